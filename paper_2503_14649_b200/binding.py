"""Thin ctypes binding of librago.so: same names as include/rago.h, argument marshalling only.

Tensors are torch CUDA tensors (device memory and streams are torch's); every computation runs in
the library's kernels.  A missing or unloadable library raises -- there is no fallback path.
"""

from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librago.so")
_lib = None

RAGO_OK = 0
STATUS_NAMES = {0: "RAGO_OK", 1: "RAGO_EINVAL", 2: "RAGO_EALIGN", 3: "RAGO_EUNSUPPORTED", 4: "RAGO_ENOMEM",
                5: "RAGO_ECUDA", 6: "RAGO_ETIMEOUT"}
RAGO_L2, RAGO_IP = 0, 1
RAGO_F32, RAGO_BF16 = 0, 1
NUM_STAGES = 5
PLAN_NAMES = ("route", "lists", "cap", "pilot_cols", "early_successor", "slots", "counts_at", "lead",
              "prefetch")
PLAN_ROUTES = ("fp32", "matrix", "lists", "tree")
STAGE_NAMES = ("coarse_scores", "probe_select", "plan", "table_scan", "merge")

EXPORTS = ("rago_index_load", "rago_index_load_pq4", "rago_index_set_coarse_tree", "rago_index_free", "rago_search_workspace_bytes", "rago_search",
           "rago_search_probes", "rago_search_probes_noalloc", "rago_search_host", "rago_host_staging_bytes", "rago_flat_search",
           "rago_flat_workspace_bytes", "rago_check", "rago_set_coarse_mode", "rago_profile_enable", "rago_profile_read",
           "rago_merge_results", "rago_q4_scores", "rago_q4_rescore", "rago_q4_rescore_backward", "rago_policy_loss", "rago_policy_workspace_bytes",
           "rago_policy_loss_backward", "rago_list_balance", "rago_list_balance_backward", "rago_selftest_wait_timeout", "rago_selftest_final_selection", "rago_debug_set_gemm_pairing", "rago_debug_search_plan", "rago_kernel_launches", "rago_last_error")


class RagoError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), message))
        self.status = status


def lib() -> ctypes.CDLL:
    """Open librago.so (built by paper_2503_14649_b200.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("librago.so is not built: run `python -m paper_2503_14649_b200.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.rago_index_load.argtypes = [ctypes.POINTER(vp), vp, ctypes.c_int, vp, vp, vp, vp, i64, i32, i32, i32,
                                      ctypes.c_int, vp]
        L.rago_index_load_pq4.argtypes = L.rago_index_load.argtypes
        L.rago_index_set_coarse_tree.argtypes = [vp, vp, vp, i32, i32, vp]
        L.rago_index_free.argtypes = [vp]
        L.rago_search_workspace_bytes.argtypes = [vp, i32, i32, i32, ctypes.POINTER(sz)]
        L.rago_host_staging_bytes.argtypes = [vp, i32, i32, ctypes.POINTER(sz)]
        L.rago_search.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        L.rago_search_probes.argtypes = [vp, vp, i32, i32, vp, vp, vp, sz, vp]
        L.rago_search_probes_noalloc.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.rago_search_host.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        L.rago_flat_search.argtypes = [vp, i64, i32, vp, i32, i32, vp, vp, vp, sz, vp]
        L.rago_flat_workspace_bytes.argtypes = [i64, i32, i32, i32, ctypes.POINTER(sz)]
        L.rago_merge_results.argtypes = [vp, vp, i32, i64, i32, i32, i32, i32, vp, vp, vp]
        f32 = ctypes.c_float
        L.rago_q4_scores.argtypes = [vp, vp, i32, i64, i32, i32, vp, i32, i32, vp, vp]
        L.rago_q4_rescore.argtypes = [vp, vp, i32, i64, i32, i32, vp, i32, i32, vp, i32, i32, vp, vp]
        L.rago_q4_rescore_backward.argtypes = [vp, vp, i32, i64, i32, i32, vp, i32, i32, vp, i32, i32, vp, vp, vp]
        L.rago_policy_loss.argtypes = [vp, vp, i32, vp, i32, i32, f32, vp, vp, vp, i32, f32, f32, vp, vp, vp, vp, vp, sz, vp]
        L.rago_policy_workspace_bytes.argtypes = [i32, i32, ctypes.POINTER(sz)]
        L.rago_policy_loss_backward.argtypes = [vp, vp, i32, vp, i32, i32, f32, vp, vp, vp, i32, f32, f32, vp, vp, vp, vp, vp,
                                                vp, vp]
        L.rago_list_balance.argtypes = [vp, i32, i32, i32, f32, vp, i32, vp, vp, vp, vp, vp]
        L.rago_list_balance_backward.argtypes = [vp, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp]
        L.rago_check.argtypes = [vp, vp]
        L.rago_selftest_wait_timeout.argtypes = [vp, ctypes.c_uint32, i32, vp]
        L.rago_selftest_final_selection.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp]
        L.rago_debug_set_gemm_pairing.argtypes = [i32]
        L.rago_debug_search_plan.argtypes = [vp, i32, i32, i32, vp]
        L.rago_set_coarse_mode.argtypes = [vp, i32]
        L.rago_profile_enable.argtypes = [vp, i32]
        L.rago_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
        L.rago_kernel_launches.restype = i64
        L.rago_last_error.restype = ctypes.c_char_p
        for name in EXPORTS:
            if name not in ("rago_kernel_launches", "rago_last_error"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != RAGO_OK:
        raise RagoError(status, lib().rago_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# The current stream as a number, without the Stream object around it (2 us a call) where torch hands it out.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream() -> ctypes.c_void_p:
    if _raw_stream is not None and torch.cuda.is_initialized():
        return ctypes.c_void_p(_raw_stream(_raw_device()))
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def rago_kernel_launches() -> int:
    return int(lib().rago_kernel_launches())


class Index:
    """Handle from rago_index_load.  Keeps references to the borrowed tensors so they outlive it."""

    def __init__(self, centroids: torch.Tensor, codebooks: torch.Tensor, codes: torch.Tensor,
                 list_offsets: torch.Tensor, ids: torch.Tensor, metric):
        metric = {"l2": RAGO_L2, "ip": RAGO_IP}.get(metric, metric)
        dtype = RAGO_BF16 if centroids.dtype == torch.bfloat16 else RAGO_F32
        nlist, d = centroids.shape
        N = codes.shape[0]
        self._keep = (centroids, codebooks, codes, list_offsets, ids)
        self._h = ctypes.c_void_p()
        if codebooks.shape[1] == 16:  # 4-bit codes, two per byte: rago_index_load_pq4
            M4 = codebooks.shape[0]
            M = M4 // 2
            _check(lib().rago_index_load_pq4(ctypes.byref(self._h), _ptr(centroids), dtype, _ptr(codebooks),
                                             _ptr(codes), _ptr(list_offsets), _ptr(ids), N, d, nlist, M4, metric,
                                             _stream()))
        else:
            M = codebooks.shape[0]
            _check(lib().rago_index_load(ctypes.byref(self._h), _ptr(centroids), dtype, _ptr(codebooks), _ptr(codes),
                                         _ptr(list_offsets), _ptr(ids), N, d, nlist, M, metric, _stream()))
        self.nlist, self.d, self.M, self.N, self.metric = nlist, d, M, N, metric
        self._ws = None

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value and _lib is not None:
            try:
                _lib.rago_index_free(self._h)
            except Exception:  # interpreter shutdown: the module globals may already be gone
                pass
            self._h = ctypes.c_void_p()

    __del__ = close

    # -- sizes ---------------------------------------------------------------------------------
    def search_workspace_bytes(self, nq: int, nprobe: int, k: int) -> int:
        out = ctypes.c_size_t()
        _check(lib().rago_search_workspace_bytes(self._h, nq, nprobe, k, ctypes.byref(out)))
        return out.value

    def host_staging_bytes(self, nq: int, k: int) -> int:
        out = ctypes.c_size_t()
        _check(lib().rago_host_staging_bytes(self._h, nq, k, ctypes.byref(out)))
        return out.value

    def workspace(self, nbytes: int, device) -> torch.Tensor:
        """A cached, 256-byte aligned scratch tensor of at least nbytes (torch allocations are)."""
        if self._ws is None or self._ws.numel() < nbytes or self._ws.device != torch.device(device):
            self._ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return self._ws

    # -- calls ---------------------------------------------------------------------------------
    def rago_search(self, queries: torch.Tensor, nprobe: int, k: int,
                    out_ids: Optional[torch.Tensor] = None, out_dists: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        nq = queries.shape[0]
        dev = queries.device
        if out_ids is None:
            out_ids = torch.empty((nq, k), dtype=torch.int64, device=dev)
        if out_dists is None:
            out_dists = torch.empty((nq, k), dtype=torch.float32, device=dev)
        if workspace is None:
            workspace = self.workspace(self.search_workspace_bytes(nq, nprobe, k), dev)
        _check(lib().rago_search(self._h, _ptr(queries), nq, nprobe, k, _ptr(out_ids), _ptr(out_dists),
                                 _ptr(workspace), workspace.numel(), _stream()))
        return out_ids, out_dists

    def rago_search_probes(self, queries: torch.Tensor, nprobe: int,
                           workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        nq = queries.shape[0]
        dev = queries.device
        lists = torch.empty((nq, nprobe), dtype=torch.int32, device=dev)
        coarse = torch.empty((nq, nprobe), dtype=torch.float32, device=dev)
        if workspace is None:
            workspace = self.workspace(self.search_workspace_bytes(nq, nprobe, 1), dev)
        _check(lib().rago_search_probes(self._h, _ptr(queries), nq, nprobe, _ptr(lists), _ptr(coarse),
                                        _ptr(workspace), workspace.numel(), _stream()))
        return lists, coarse

    def rago_search_probes_noalloc(self, queries: torch.Tensor, nprobe: int, out_lists: torch.Tensor,
                                   out_coarse: torch.Tensor):
        """rago_search_probes without a workspace: scratch is the library's built-in array, so the
        call allocates nothing (the outputs are the caller's).  Calls must not overlap on the GPU."""
        _check(lib().rago_search_probes_noalloc(self._h, _ptr(queries), queries.shape[0], nprobe, _ptr(out_lists),
                                                _ptr(out_coarse), _stream()))

    def rago_search_host(self, host_queries: torch.Tensor, nprobe: int, k: int, host_out_ids: torch.Tensor,
                         host_out_dists: torch.Tensor, workspace: torch.Tensor):
        nq = host_queries.shape[0]
        _check(lib().rago_search_host(self._h, _ptr(host_queries), nq, nprobe, k, _ptr(host_out_ids),
                                      _ptr(host_out_dists), _ptr(workspace), workspace.numel(), _stream()))

    def rago_check(self, workspace: Optional[torch.Tensor] = None):
        ws = workspace if workspace is not None else self._ws
        _check(lib().rago_check(_ptr(ws), _stream()))

    def rago_set_coarse_mode(self, mode: int):
        _check(lib().rago_set_coarse_mode(self._h, int(mode)))
        self._ws = None  # workspace sizes depend on the mode

    def rago_index_set_coarse_tree(self, level1: Optional[torch.Tensor], child_offsets: Optional[torch.Tensor], b1: int = 0):
        """Set (or, with level1 = None, remove) the level above the coarse centroids; tensors are borrowed."""
        if level1 is None:
            _check(lib().rago_index_set_coarse_tree(self._h, None, None, 0, 0, _stream()))
            self._tree = None
        else:
            _check(lib().rago_index_set_coarse_tree(self._h, _ptr(level1), _ptr(child_offsets), level1.shape[0], int(b1),
                                                    _stream()))
            self._tree = (level1, child_offsets)
        self._ws = None  # workspace sizes depend on it

    def rago_debug_search_plan(self, nq: int, nprobe: int, k: int) -> dict:
        """Which way a search of these sizes goes (see rago.h); "route" is one of PLAN_ROUTES."""
        out = (ctypes.c_int32 * len(PLAN_NAMES))()
        _check(lib().rago_debug_search_plan(self._h, nq, nprobe, k, out))
        plan = dict(zip(PLAN_NAMES, out))
        return dict(plan, route=PLAN_ROUTES[plan["route"]])

    def rago_profile_enable(self, enable: bool = True):
        _check(lib().rago_profile_enable(self._h, int(enable)))

    def rago_profile_read(self):
        out = (ctypes.c_float * NUM_STAGES)()
        _check(lib().rago_profile_read(self._h, out))
        return dict(zip(STAGE_NAMES, [float(v) for v in out]))


def rago_index_load(centroids, codebooks, codes, list_offsets, ids, metric) -> Index:
    return Index(centroids, codebooks, codes, list_offsets, ids, metric)


def rago_index_load_pq4(centroids, pq4_codebooks, packed_codes, list_offsets, ids, metric) -> Index:
    """pq4_codebooks [M4, 16, d / M4], packed_codes uint8 [N, M4 / 2] (low nibble = even sub-space)."""
    if pq4_codebooks.shape[1] != 16:
        raise ValueError("4-bit codebooks have 16 codewords per sub-space")
    return Index(centroids, pq4_codebooks, packed_codes, list_offsets, ids, metric)


def rago_debug_set_gemm_pairing(mode: int):
    """0: the library chooses the tensor-core main loop by operand size, 1: one row tile per CTA, 2: two row tiles
    per CTA, 3: two row tiles per CTA pair (cluster of two)."""
    _check(lib().rago_debug_set_gemm_pairing(int(mode)))


def rago_selftest_wait_timeout(workspace: torch.Tensor, max_polls: int, with_tmem: bool):
    """Launch the bounded-wait self-test on `workspace` (see rago.h); follow with rago_check(workspace)."""
    _check(lib().rago_selftest_wait_timeout(_ptr(workspace), int(max_polls), int(bool(with_tmem)), _stream()))


def rago_selftest_final_selection(counts: torch.Tensor, entries: torch.Tensor, k: int):
    """Flat search's final selection over counts int32 [nq, nlists] and entries int64 [nq, nlists, stride] (see rago.h)."""
    nq, nlists, stride = entries.shape
    out_ids = torch.empty((nq, k), dtype=torch.int64, device=entries.device)
    out_scores = torch.empty((nq, k), dtype=torch.float32, device=entries.device)
    _check(lib().rago_selftest_final_selection(_ptr(counts), _ptr(entries), nlists, stride, nq, k, _ptr(out_ids),
                                               _ptr(out_scores), _stream()))
    return out_ids, out_scores


def rago_check(workspace: torch.Tensor):
    """rago_check on a bare workspace tensor (Index.rago_check does the same for an index's workspace)."""
    _check(lib().rago_check(_ptr(workspace), _stream()))


def rago_flat_workspace_bytes(N: int, d: int, nq: int, k: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().rago_flat_workspace_bytes(N, d, nq, k, ctypes.byref(out)))
    return out.value


def rago_flat_search(db: torch.Tensor, queries: torch.Tensor, k: int, workspace: Optional[torch.Tensor] = None):
    N, d = db.shape
    nq = queries.shape[0]
    dev = queries.device
    out_ids = torch.empty((nq, k), dtype=torch.int64, device=dev)
    out_scores = torch.empty((nq, k), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(rago_flat_workspace_bytes(N, d, nq, k), dtype=torch.uint8, device=dev)
    _check(lib().rago_flat_search(_ptr(db), N, d, _ptr(queries), nq, k, _ptr(out_ids), _ptr(out_scores),
                                  _ptr(workspace), workspace.numel(), _stream()))
    return out_ids, out_scores


def rago_merge_results(part_ids: torch.Tensor, part_dists: torch.Tensor, k_out: int, metric,
                       out_ids: Optional[torch.Tensor] = None, out_dists: Optional[torch.Tensor] = None):
    """part_ids / part_dists: contiguous [nparts, nq, k_in] device tensors (the shards' answers side by side)."""
    metric = {"l2": RAGO_L2, "ip": RAGO_IP}.get(metric, metric)
    nparts, nq, k_in = part_ids.shape
    if part_dists.shape != part_ids.shape or not (part_ids.is_contiguous() and part_dists.is_contiguous()):
        raise ValueError("part_ids and part_dists must be contiguous tensors of one shape [nparts, nq, k_in]")
    dev = part_ids.device
    if out_ids is None:
        out_ids = torch.empty((nq, k_out), dtype=torch.int64, device=dev)
    if out_dists is None:
        out_dists = torch.empty((nq, k_out), dtype=torch.float32, device=dev)
    _check(lib().rago_merge_results(_ptr(part_ids), _ptr(part_dists), nparts, nq * k_in, nq, k_in, k_out, metric,
                                    _ptr(out_ids), _ptr(out_dists), _stream()))
    return out_ids, out_dists


# ---- what is done with the answers of a search -------------------------------------------------------------------------

POLICY_STATS = BALANCE_STATS = 4
POLICY_SPAN = 16_384  # longest row that needs no workspace
_FLOATS = {torch.float32: RAGO_F32, torch.bfloat16: RAGO_BF16}


def _current_device() -> int:
    """Number of the current CUDA device; -1 where there is none, which no tensor's device equals."""
    return _raw_device() if torch.cuda.is_initialized() else -1


def _expect(name: str, t: Optional[torch.Tensor], shape, dtypes, dev: int):
    """The library takes pointers: a tensor of another shape, type, order or device would be read as something else."""
    if t.shape == shape and t.dtype in dtypes and t.is_cuda and t.get_device() == dev and t.is_contiguous():
        return
    raise ValueError("%s must be a contiguous tensor of shape %s and type %s on the current CUDA device, not %s %s on %s"
                     % (name, list(shape), " or ".join(map(str, dtypes)), list(t.shape), t.dtype, t.device))


def _expect_q4(codes, scales, queries, group, dev):
    if codes.dim() != 2 or queries.dim() != 2 or group < 1:
        raise ValueError("codes are [N, d / 2], queries [nq, d], group is positive")
    N, d = codes.shape[0], 2 * codes.shape[1]
    _expect("codes", codes, (N, d // 2), (torch.uint8,), dev)
    _expect("scales", scales, (N, -(-d // group)), _FLOATS, dev)
    _expect("queries", queries, (queries.shape[0], d), _FLOATS, dev)
    return N, d, queries.shape[0]


def rago_q4_scores(codes: torch.Tensor, scales: torch.Tensor, queries: torch.Tensor, group: int,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """<query, row> of every row in 4 bits: codes uint8 [N, d / 2], scales [N, ceil(d / group)] -> fp32 [nq, N]."""
    dev = _current_device()
    N, d, nq = _expect_q4(codes, scales, queries, group, dev)
    if out is None:
        out = codes.new_empty((nq, N), dtype=torch.float32)
    else:
        _expect("out", out, (nq, N), (torch.float32,), dev)
    _check(lib().rago_q4_scores(codes.data_ptr(), scales.data_ptr(), _FLOATS[scales.dtype], N, d, group, queries.data_ptr(),
                                _FLOATS[queries.dtype], nq, out.data_ptr(), _stream()))
    return out


def rago_q4_rescore(codes: torch.Tensor, scales: torch.Tensor, queries: torch.Tensor, ids: torch.Tensor, group: int, metric,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Distances (or inner products) of the candidates ids int64 [nq, k] in the order of ids, fp32 [nq, k]; an id outside the
    store (a search's -1) gives +inf (L2) or -inf (IP)."""
    dev = _current_device()
    N, d, nq = _expect_q4(codes, scales, queries, group, dev)
    metric = {"l2": RAGO_L2, "ip": RAGO_IP}.get(metric, metric)
    k = ids.shape[-1]
    _expect("ids", ids, (nq, k), (torch.int64,), dev)
    if out is None:
        out = codes.new_empty((nq, k), dtype=torch.float32)
    else:
        _expect("out", out, (nq, k), (torch.float32,), dev)
    _check(lib().rago_q4_rescore(codes.data_ptr(), scales.data_ptr(), _FLOATS[scales.dtype], N, d, group, queries.data_ptr(),
                                 _FLOATS[queries.dtype], nq, ids.data_ptr(), k, metric, out.data_ptr(), _stream()))
    return out


def rago_q4_rescore_backward(codes: torch.Tensor, scales: torch.Tensor, queries: torch.Tensor, ids: torch.Tensor, group: int,
                             metric, grad_dists: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of rago_q4_rescore's distances to the queries, [nq, d] of their type."""
    dev = _current_device()
    N, d, nq = _expect_q4(codes, scales, queries, group, dev)
    metric = {"l2": RAGO_L2, "ip": RAGO_IP}.get(metric, metric)
    k = ids.shape[-1]
    _expect("ids", ids, (nq, k), (torch.int64,), dev)
    _expect("grad_dists", grad_dists, (nq, k), (torch.float32,), dev)
    if out is None:
        out = torch.empty_like(queries)
    else:
        _expect("out", out, (nq, d), (queries.dtype,), dev)
    _check(lib().rago_q4_rescore_backward(codes.data_ptr(), scales.data_ptr(), _FLOATS[scales.dtype], N, d, group,
                                          queries.data_ptr(), _FLOATS[queries.dtype], nq, ids.data_ptr(), k, metric,
                                          grad_dists.data_ptr(), out.data_ptr(), _stream()))
    return out


class PolicyLoss(NamedTuple):
    """policy, kl fp32 [nq], logp fp32 [nq, G] of the choices, and the rows' maxima and sums for the backward pass."""
    policy: torch.Tensor
    kl: torch.Tensor
    logp: torch.Tensor
    stats: torch.Tensor


def _expect_policy(scores, chosen, old_logp, advantage, ref_scores, ids, dev):
    if scores.dim() != 2 or chosen.dim() != 2:
        raise ValueError("scores are [nq, C], chosen [nq, G]")
    nq, C = scores.shape
    G = chosen.shape[1]
    _expect("scores", scores, (nq, C), _FLOATS, dev)
    _expect("chosen", chosen, (nq, G), (torch.int32,), dev)
    _expect("old_logp", old_logp, (nq, G), (torch.float32,), dev)
    _expect("advantage", advantage, (nq, G), (torch.float32,), dev)
    if ref_scores is not None:
        _expect("ref_scores", ref_scores, (nq, C), (scores.dtype,), dev)
    if ids is not None:
        _expect("ids", ids, (nq, C), (torch.int64,), dev)
    return nq, C, G


def rago_policy_workspace_bytes(nq: int, C: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().rago_policy_workspace_bytes(nq, C, ctypes.byref(out)))
    return out.value


def rago_policy_loss(scores: torch.Tensor, chosen: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, scale: float,
                     clip_low: float, clip_high: float, ref_scores: Optional[torch.Tensor] = None,
                     ids: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> PolicyLoss:
    """Clipped policy loss and KL term per query of the policy softmax(scale * scores) over its candidates (see rago.h):
    scores [nq, C], chosen int32, old_logp and advantage fp32 [nq, G]; ids int64 [nq, C] marks missing candidates (< 0)."""
    dev = _current_device()
    nq, C, G = _expect_policy(scores, chosen, old_logp, advantage, ref_scores, ids, dev)
    policy, kl = old_logp.new_empty(nq), old_logp.new_empty(nq)
    logp = torch.empty_like(old_logp)
    stats = old_logp.new_empty(nq, POLICY_STATS)
    if workspace is not None:
        _expect("workspace", workspace, workspace.shape, (workspace.dtype,), dev)
    elif C > POLICY_SPAN:
        workspace = scores.new_empty(rago_policy_workspace_bytes(nq, C), dtype=torch.uint8)
    _check(lib().rago_policy_loss(scores.data_ptr(), None if ref_scores is None else ref_scores.data_ptr(), _FLOATS[scores.dtype],
                                  None if ids is None else ids.data_ptr(), nq, C, scale, chosen.data_ptr(), old_logp.data_ptr(),
                                  advantage.data_ptr(), G, clip_low, clip_high, policy.data_ptr(), kl.data_ptr(), logp.data_ptr(),
                                  stats.data_ptr(), None if workspace is None else workspace.data_ptr(),
                                  0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))
    return PolicyLoss(policy, kl, logp, stats)


def rago_policy_loss_backward(scores: torch.Tensor, chosen: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor,
                              scale: float, clip_low: float, clip_high: float, forward: PolicyLoss, grad_policy: torch.Tensor,
                              grad_kl: Optional[torch.Tensor] = None, ref_scores: Optional[torch.Tensor] = None,
                              ids: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of sum(grad_policy * policy + grad_kl * kl) by the scores, [nq, C] of their type; `forward` is what
    rago_policy_loss returned for the same inputs."""
    dev = _current_device()
    nq, C, G = _expect_policy(scores, chosen, old_logp, advantage, ref_scores, ids, dev)
    _expect("stats", forward.stats, (nq, POLICY_STATS), (torch.float32,), dev)
    _expect("logp", forward.logp, (nq, G), (torch.float32,), dev)
    _expect("kl", forward.kl, (nq,), (torch.float32,), dev)
    _expect("grad_policy", grad_policy, (nq,), (torch.float32,), dev)
    if ref_scores is not None and grad_kl is None:
        raise ValueError("grad_kl is needed with ref_scores")
    if grad_kl is not None:
        _expect("grad_kl", grad_kl, (nq,), (torch.float32,), dev)
    if out is None:
        out = torch.empty_like(scores)
    else:
        _expect("out", out, (nq, C), (scores.dtype,), dev)
    _check(lib().rago_policy_loss_backward(scores.data_ptr(), None if ref_scores is None else ref_scores.data_ptr(),
                                           _FLOATS[scores.dtype], None if ids is None else ids.data_ptr(), nq, C, scale,
                                           chosen.data_ptr(), old_logp.data_ptr(), advantage.data_ptr(), G, clip_low, clip_high,
                                           forward.kl.data_ptr(), forward.logp.data_ptr(), forward.stats.data_ptr(),
                                           grad_policy.data_ptr(), None if grad_kl is None else grad_kl.data_ptr(),
                                           out.data_ptr(), _stream()))
    return out


class ListBalance(NamedTuple):
    """loss fp32 [1], counts int32 [nlist], and the rows' maxima and sums for the backward pass."""
    loss: torch.Tensor
    counts: torch.Tensor
    stats: torch.Tensor


def _expect_valid(valid, nq, dev):
    if valid is not None:
        _expect("valid", valid, (nq,), (torch.bool, torch.uint8), dev)


def rago_list_balance(logits: torch.Tensor, lists: torch.Tensor, scale: float, valid: Optional[torch.Tensor] = None) -> ListBalance:
    """Probes per list and the balance loss (see rago.h): logits [nq, nlist], lists int32 [nq, nprobe] as rago_search_probes
    returns them, valid bool [nq] marks the rows that are not padding."""
    if logits.dim() != 2 or lists.dim() != 2:
        raise ValueError("logits are [nq, nlist], lists [nq, nprobe]")
    dev = _current_device()
    nq, nlist = logits.shape
    nprobe = lists.shape[1]
    _expect("logits", logits, (nq, nlist), _FLOATS, dev)
    _expect("lists", lists, (nq, nprobe), (torch.int32,), dev)
    _expect_valid(valid, nq, dev)
    loss = logits.new_empty(1, dtype=torch.float32)
    counts = lists.new_empty(nlist)
    stats = logits.new_empty((nq + 1, BALANCE_STATS), dtype=torch.float32)
    _check(lib().rago_list_balance(logits.data_ptr(), _FLOATS[logits.dtype], nq, nlist, scale, lists.data_ptr(), nprobe,
                                   None if valid is None else valid.data_ptr(), loss.data_ptr(), counts.data_ptr(), stats.data_ptr(),
                                   _stream()))
    return ListBalance(loss, counts, stats)


def rago_list_balance_backward(logits: torch.Tensor, scale: float, forward: ListBalance, grad_loss: torch.Tensor,
                               valid: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of grad_loss * loss by the logits, [nq, nlist] of their type; `forward` is what rago_list_balance returned."""
    if logits.dim() != 2:
        raise ValueError("logits are [nq, nlist]")
    dev = _current_device()
    nq, nlist = logits.shape
    _expect("logits", logits, (nq, nlist), _FLOATS, dev)
    _expect("counts", forward.counts, (nlist,), (torch.int32,), dev)
    _expect("stats", forward.stats, (nq + 1, BALANCE_STATS), (torch.float32,), dev)
    _expect("grad_loss", grad_loss, (1,), (torch.float32,), dev)
    _expect_valid(valid, nq, dev)
    if out is None:
        out = torch.empty_like(logits)
    else:
        _expect("out", out, (nq, nlist), (logits.dtype,), dev)
    _check(lib().rago_list_balance_backward(logits.data_ptr(), _FLOATS[logits.dtype], nq, nlist, scale,
                                            None if valid is None else valid.data_ptr(), forward.counts.data_ptr(),
                                            forward.stats.data_ptr(), grad_loss.data_ptr(), out.data_ptr(), _stream()))
    return out


def load_index_from(data, device="cuda") -> Index:
    """rago_index_load over a synth.IvfPqData (moves its tensors to `device` first)."""
    dev = torch.device(device)
    return Index(data.centroids.to(dev).contiguous(), data.codebooks.to(dev).contiguous(),
                 data.codes.to(dev).contiguous(), data.list_offsets.to(dev).contiguous(),
                 data.ids.to(dev).contiguous(), data.metric)
