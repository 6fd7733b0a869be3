"""Rows in 4 bits with group scales on the GPU: scores of a store, candidates scored again, gradient to the queries, each against
the definition in 64 bits.

Tolerances.  u = 2^-24.  A sum of n fp32 terms in any order is off by at most (n - 1) u sum|terms| (first order); a product adds
u, the scale another u.  So |error| <= (n + 4) u * sum of the magnitudes, with 5 % for the second order.  An L2 term is
t = x - s (c - 8) in one rounding, squared: 3 u more at most.  A result stored in bf16 is off by half a step more, 2^-8.
The gradient of k distances is 2 sum g (x - w), the difference in one rounding: (k + 6) u * 2 sum |g| |x - w|, which check_candidates,
written for 2 (x sum g - sum g w), bounds by (k + 6) u * 2 sum |g| (|x| + |w|)."""

import pytest
import torch

from paper_2503_14649_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SECOND_ORDER = 1.05
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_rows(N, d, group, scale_dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (N, d // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((N, -(-d // group)), generator=g, device="cuda") * 0.02 + 1e-3).to(scale_dtype)
    return codes, scales


def make_queries(nq, d, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((nq, d), generator=g, device="cuda").to(dtype)


def values64(codes, scales, group):
    """The rows as numbers, by the definition."""
    low, high = codes.long() % 16, codes.long() // 16
    w = torch.stack((low, high), 2).flatten(1).double() - 8
    at = torch.arange(w.shape[1], device=codes.device) // group
    return w * scales.double()[:, at]


def check_scores(codes, scales, queries, group):
    got = binding.rago_q4_scores(codes, scales, queries, group)
    w, x = values64(codes, scales, group), queries.double()
    assert got.shape == (queries.shape[0], codes.shape[0]) and got.dtype == torch.float32
    tol = SECOND_ORDER * (w.shape[1] + 4) * U * (x.abs() @ w.abs().T)
    bad = ~((got.double() - x @ w.T).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:4].tolist())
    return got


@pytest.mark.parametrize("query", ["f32", "bf16"])
@pytest.mark.parametrize("scale", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,d,nq", [(1, 32, 1), (37, 96, 2), (1000, 768, 5), (33, 160, 9)])
def test_scores_match_the_definition(N, d, nq, group, scale, query):
    codes, scales = make_rows(N, d, group, DTYPES[scale])
    check_scores(codes, scales, make_queries(nq, d, DTYPES[query]), group)


@pytest.mark.parametrize("nq", [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 24, 25, 31, 33, 48, 63, 64, 65, 100, 130])
@pytest.mark.parametrize("query", ["f32", "bf16"])
def test_scores_for_any_number_of_queries(nq, query):
    codes, scales = make_rows(517, 416, 64, torch.bfloat16)
    check_scores(codes, scales, make_queries(nq, 416, DTYPES[query]), 64)


@pytest.mark.parametrize("N", [2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 2047, 4097, 20_001, 150_001])
def test_scores_for_any_number_of_rows(N):
    codes, scales = make_rows(N, 64, 32, torch.float32)
    check_scores(codes, scales, make_queries(3, 64, torch.float32), 32)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 224, 256, 288, 512, 736, 1024, 1056, 2048, 2080, 4096, 6176, 8192])
@pytest.mark.parametrize("nq,query", [(1, "f32"), (20, "f32"), (1, "bf16"), (40, "bf16")])
def test_scores_for_any_length_of_rows(d, nq, query):
    codes, scales = make_rows(301, d, 128, torch.bfloat16)
    check_scores(codes, scales, make_queries(nq, d, DTYPES[query]), 128)


def test_scores_hold_queries_of_any_size():
    """fp32 queries are not rounded to fewer bits, and their range is that of fp32."""
    codes, scales = make_rows(200, 256, 64, torch.float32)
    q = make_queries(4, 256, torch.float32)
    q[1] *= 1e30
    q[2] *= 1e-30
    q[3] = torch.where(torch.arange(256, device="cuda") % 3 == 0, q[3] * 1e4, q[3] * 1e-4)
    check_scores(codes, scales, q, 64)


@pytest.mark.parametrize("d,group,scale", [(416, 32, "bf16"), (416, 128, "f32"), (768, 32, "f32"), (768, 64, "bf16"), (768, 128, "f32"), (2048, 64, "f32")])
@pytest.mark.parametrize("query", ["f32", "bf16"])
@pytest.mark.parametrize("nq", [1, 5, 12, 20, 37, 64])
def test_scores_of_more_rows_than_one_tile_a_warp(nq, query, d, group, scale):
    """Several tiles of rows a warp (3126 and more for 1776 or 2368 warps, or half as many teams of two), with any number of tiles of columns and
    any group: rings, scales and shared sums are carried from tile to tile.  Every score is looked at."""
    for N in ((133_337,) if d > 768 else (100_003, 133_337)):
        codes, scales = make_rows(N, d, group, DTYPES[scale])
        q = make_queries(nq, d, DTYPES[query])
        got, x = binding.rago_q4_scores(codes, scales, q, group), q.double()
        for r in range(0, N, 20_000):
            w = values64(codes[r:r + 20_000], scales[r:r + 20_000], group)
            tol = SECOND_ORDER * (d + 4) * U * (x.abs() @ w.abs().T)
            assert ((got[:, r:r + 20_000].double() - x @ w.T).abs() <= tol).all(), (N, r)


@pytest.mark.parametrize("nq", [3, 12])
@pytest.mark.parametrize("query", ["f32", "bf16"])
def test_a_querys_numbers_enter_with_the_error_that_the_header_states(nq, query):
    """Rows that are 1 in one place and 0 elsewhere: the score is that number of the query, no sum rounds it."""
    d = 256
    codes = torch.full((d, d // 2), 0x88, dtype=torch.uint8, device="cuda")
    i = torch.arange(d, device="cuda")
    codes[i, i // 2] = torch.where(i % 2 == 0, 0x89, 0x98).to(torch.uint8)
    scales = torch.ones((d, d // 32), device="cuda")
    q = make_queries(nq, d, torch.float32)
    q[0] *= 2.0 ** torch.linspace(0, -40, d, device="cuda")
    q[1, :4] = torch.tensor([1 + 2 ** -11 - 2 ** -23, -1 - 2 ** -11 + 2 ** -23, 1 + 3 * 2 ** -23, 2 - 2 ** -23], device="cuda")
    q = q.to(DTYPES[query])
    got, x = binding.rago_q4_scores(codes, scales, q, 32).double(), q.double()
    top = x.abs().amax(1, keepdim=True)
    if query == "bf16":
        exact = x.abs() >= 2.0 ** -31 * top
        assert (got == x)[exact].all()
    assert ((got - x).abs() <= torch.maximum(2.0 ** -23 * x.abs(), 2.0 ** -39 * top)).all()


@pytest.mark.parametrize("nq,query", [(1, "f32"), (4, "f32"), (20, "f32"), (3, "bf16"), (40, "bf16")])
@pytest.mark.parametrize("scale,group", [("f32", 32), ("bf16", 128)])
def test_scores_hold_scales_of_any_size(nq, query, scale, group):
    """Scales up to 2e32 with queries around 1e-28 and around 1: every score, up to 1e35, is a number that fp32 holds."""
    for N in (5, 300, 20_001):
        codes, scales = make_rows(N, 256, group, DTYPES[scale])
        q = make_queries(nq, 256, torch.float32)
        scales[::3] *= 1e34
        q[::2] *= 1e-28
        check_scores(codes, scales, q.to(DTYPES[query]), group)


def test_scores_beyond_fp32_are_infinite_and_no_others():
    codes, scales = make_rows(100, 128, 64, torch.float32)
    codes[7] = 0x99                                     # ones
    scales[7] = 1e37
    q = make_queries(9, 128, torch.float32)
    q[1] = 1.0
    q[2] = -1.0
    got = binding.rago_q4_scores(codes, scales, q, 64)
    assert got[1, 7] == float("inf") and got[2, 7] == float("-inf")    # 1.28e39 either way
    scales[7] = 1e-3
    want = binding.rago_q4_scores(codes, scales, q, 64)
    rest = torch.arange(100, device="cuda") != 7
    assert torch.equal(got[:, rest], want[:, rest])


def test_a_bad_scale_or_query_stays_in_its_results():
    codes, scales = make_rows(300, 128, 32, torch.float32)
    q = make_queries(11, 128, torch.float32)
    want = binding.rago_q4_scores(codes, scales, q, 32)
    scales[17, 2] = float("nan")
    scales[40, 0] = float("inf")
    q[5, 77] = float("nan")
    q[9, 3] = float("inf")
    got = binding.rago_q4_scores(codes, scales, q, 32)
    assert got[:, 17].isnan().all() and not got[:, 40].isfinite().any()
    assert not got[5].isfinite().any()
    zero = (codes[:, 1] // 16 == 8)  # number 3 of a row: infinity times a stored 0 is NaN, times anything else infinite
    assert got[9][zero].isnan().all() and not got[9].isfinite().any()
    rows = torch.ones(300, dtype=torch.bool, device="cuda")
    rows[17] = rows[40] = False
    for i in range(11):
        if i not in (5, 9):
            assert torch.equal(got[i][rows], want[i][rows])


def test_scores_of_a_view_of_the_rows_and_with_an_output():
    codes, scales = make_rows(1000, 192, 64, torch.bfloat16)
    q = make_queries(6, 192, torch.bfloat16)
    whole = check_scores(codes, scales, q, 64)
    out = torch.full((6, 333), -7.0, device="cuda")
    assert binding.rago_q4_scores(codes[101:434], scales[101:434], q, 64, out=out) is out
    assert torch.equal(out, whole[:, 101:434])
    guard = torch.full((8, 334), -7.0, device="cuda")  # nothing is written behind the output
    inside = guard.view(-1)[:6 * 333].view(6, 333)
    binding.rago_q4_scores(codes[101:434], scales[101:434], q, 64, out=inside)
    assert torch.equal(inside, out) and (guard.view(-1)[6 * 333:] == -7.0).all()


def test_no_rows_and_no_queries():
    codes, scales = make_rows(0, 64, 32, torch.float32)
    q = make_queries(3, 64, torch.float32)
    assert binding.rago_q4_scores(codes, scales, q, 32).shape == (3, 0)
    ids = torch.zeros((3, 5), dtype=torch.int64, device="cuda")  # no row: every candidate is missing
    assert (binding.rago_q4_rescore(codes, scales, q, ids, 32, "l2") == float("inf")).all()
    assert (binding.rago_q4_rescore_backward(codes, scales, q, ids, 32, "l2", torch.ones((3, 5), device="cuda")) == 0).all()
    codes, scales = make_rows(10, 64, 32, torch.float32)
    assert binding.rago_q4_scores(codes, scales, q[:0], 32).shape == (0, 10)
    assert binding.rago_q4_rescore(codes, scales, q[:0], ids[:0], 32, "ip").shape == (0, 5)


# ---- candidates ----------------------------------------------------------------------------------------------------------

def check_candidates(codes, scales, queries, ids, group, metric, grad=None):
    d = queries.shape[1]
    N, (nq, k) = codes.shape[0], ids.shape
    got = binding.rago_q4_rescore(codes, scales, queries, ids, group, metric)
    there = (ids >= 0) & (ids < N)
    i = torch.where(there, ids, 0)
    w = values64(codes[i.flatten()], scales[i.flatten()], group).view(nq, k, d)
    x = queries.double()[:, None]
    if metric == "l2":
        t = x - w
        want = t.square().sum(2)
        tol = (d + 7) * U * want
        slope, mag = 2 * t, 2 * (x.abs() + w.abs())
    else:
        want = (x * w).sum(2)
        tol = (d + 4) * U * (x * w).abs().sum(2)
        slope, mag = w.expand(nq, k, d), w.abs()
    missing = float("inf") if metric == "l2" else float("-inf")
    assert (got[~there] == missing).all()
    bad = ~((got.double() - want).abs() <= SECOND_ORDER * tol)[there]
    assert not bad.any(), int(bad.sum())
    if grad is not None:
        gx = binding.rago_q4_rescore_backward(codes, scales, queries, ids, group, metric, grad)
        assert gx.dtype == queries.dtype and gx.shape == queries.shape
        g = torch.where(there, grad.double(), 0.0)[:, :, None]
        want = (g * slope).sum(1)
        tol = SECOND_ORDER * (k + 6) * U * (g.abs() * mag).sum(1)
        if queries.dtype == torch.bfloat16:
            tol += 2.0 ** -8 * want.abs() + 1e-38
        bad = ~((gx.double() - want).abs() <= tol)
        assert not bad.any(), int(bad.sum())
        return got, gx
    return got


def make_ids(nq, k, N, seed=2, missing=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, N, (nq, k), generator=g, device="cuda")
    if missing and k > 2:
        ids[:, k // 2] = -1
        ids[0, k - 1] = N          # just outside
        ids[nq - 1, 0] = 1 << 40   # far outside, also as 32 bits
        ids[nq - 1, 1] = ids[nq - 1, k - 2]  # twice
    return ids


@pytest.mark.parametrize("metric", ["l2", "ip"])
@pytest.mark.parametrize("query", ["f32", "bf16"])
@pytest.mark.parametrize("scale,group", [("f32", 32), ("bf16", 32), ("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("nq,k,d", [(1, 1, 32), (1, 20, 512), (5, 33, 160), (7, 100, 768), (3, 513, 96)])
def test_candidates_and_their_gradient(nq, k, d, scale, group, query, metric):
    codes, scales = make_rows(400, d, group, DTYPES[scale])
    ids = make_ids(nq, k, 400)
    grad = torch.randn((nq, k), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    check_candidates(codes, scales, make_queries(nq, d, DTYPES[query]), ids, group, metric, grad)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 192, 256, 384, 480, 1024, 1056, 2048, 2144, 4096, 8160, 8192])
@pytest.mark.parametrize("nq,k", [(1, 3), (2, 70), (150, 4)])
def test_candidates_for_any_length_of_rows(d, nq, k):
    codes, scales = make_rows(100, d, 64, torch.float32)
    grad = torch.randn((nq, k), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    for metric in ("l2", "ip"):
        check_candidates(codes, scales, make_queries(nq, d, torch.float32), make_ids(nq, k, 100), 64, metric, grad)


@pytest.mark.parametrize("nq", [1, 2, 18, 37, 74, 75, 148, 149, 300, 2000])
@pytest.mark.parametrize("k", [1, 8, 9, 65])
def test_candidates_for_any_batch(nq, k):
    codes, scales = make_rows(1000, 96, 32, torch.bfloat16)
    grad = torch.randn((nq, k), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    check_candidates(codes, scales, make_queries(nq, 96, torch.float32), make_ids(nq, k, 1000), 32, "l2", grad)


@pytest.mark.parametrize("metric", ["l2", "ip"])
@pytest.mark.parametrize("query", ["f32", "bf16"])
@pytest.mark.parametrize("nq,k,d", [(300, 513, 64), (297, 1300, 96), (40, 5000, 32), (1, 9001, 160), (2, 4097, 8192), (300, 1025, 16 * 26)])
def test_more_candidates_than_a_cta_stages_at_a_time(nq, k, d, query, metric):
    """Over 512 a CTA, alone or in a cluster, with stretches of missing ones of any length."""
    codes, scales = make_rows(1000, d, 32, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(4)
    ids = make_ids(nq, k, 1000)
    ids[nq // 2, 100:100 + k // 2] = -1
    ids[:, ::7] = -1
    grad = torch.randn((nq, k), generator=g, device="cuda")
    x = make_queries(nq, d, DTYPES[query])
    got = binding.rago_q4_rescore_backward(codes, scales, x, ids, 32, metric, grad).double()
    w = values64(codes, scales, 32)
    for r in range(nq):
        there = (ids[r] >= 0) & (ids[r] < 1000)
        rows = w[ids[r][there]]
        terms = grad[r][there].double()[:, None] * (2 * (x[r].double() - rows) if metric == "l2" else rows)
        tol = SECOND_ORDER * (k + 6) * U * terms.abs().sum(0)
        if query == "bf16":
            tol = tol + 2.0 ** -8 * terms.sum(0).abs() + 1e-38
        assert ((got[r] - terms.sum(0)).abs() <= tol).all(), r


def test_a_query_without_candidates_and_bad_gradients_of_missing_ones():
    codes, scales = make_rows(50, 64, 32, torch.float32)
    q = make_queries(3, 64, torch.float32)
    ids = make_ids(3, 6, 50, missing=False)
    ids[1] = -1
    ids[2, 4] = -5
    grad = torch.ones((3, 6), device="cuda")
    grad[1] = float("nan")
    grad[2, 4] = float("inf")
    for metric in ("l2", "ip"):
        clean = torch.where(grad.isfinite(), grad, 0.0)
        _, gx = check_candidates(codes, scales, q, ids, 32, metric, clean)
        assert (gx[1] == 0).all()
        assert torch.equal(binding.rago_q4_rescore_backward(codes, scales, q, ids, 32, metric, grad), gx)


def test_a_query_that_is_a_stored_row_has_distance_zero():
    codes, scales = make_rows(64, 128, 64, torch.float32)
    q = values64(codes, scales, 64).float()[:9].contiguous()  # the products s (c - 8) are exact in fp32 only up to a rounding
    ids = torch.arange(9, device="cuda")[:, None].contiguous()
    got = binding.rago_q4_rescore(codes, scales, q, ids, 64, "l2")
    # x is the rounded product, the row the exact one: each term is at most (u |x|)^2
    assert (got[:, 0].double() <= SECOND_ORDER * (U ** 2) * q.double().square().sum(1)).all()


@pytest.mark.parametrize("query", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 160, 768])
def test_candidates_hold_queries_and_scales_of_any_size(d, query):
    """Query numbers up to 2^119 with small scales, and scales up to 1e32 with small queries: the scaled products are ordinary ones."""
    for scale, size in ((1e-30, 2.0 ** 116), (1e34, 1e-30)):
        codes, scales = make_rows(400, d, 32, torch.float32)
        scales *= scale
        q = (make_queries(3, d, torch.float32).clamp(-8, 8) * size).to(DTYPES[query])
        check_candidates(codes, scales, q, make_ids(3, 30, 400), 32, "ip", torch.randn((3, 30), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda"))
        check_scores(codes, scales, q, 32)


@pytest.mark.parametrize("query", ["f32", "bf16"])
@pytest.mark.parametrize("near", [1.0, 0.01, 1e-3])
@pytest.mark.parametrize("nq,k,d", [(1, 700, 96), (5, 33, 160), (300, 100, 768), (2, 9, 8192)])
def test_the_gradient_of_near_candidates(nq, k, d, near, query):
    """Candidates that lie `near` times its length from their query.  A term is g (x - s (c - 8)), the difference in one rounding, so the
    error is relative to the differences, not to query and row: (k + 6) u * 2 sum |g| |x - w|."""
    g = torch.Generator(device="cuda").manual_seed(3)
    codes, scales = make_rows(400, d, 32, torch.float32)
    codes[:] = codes[0].clone()
    scales[:] = scales[0].clone() * (1 + near * torch.rand(scales.shape, generator=g, device="cuda"))
    w = values64(codes, scales, 32)
    q = (w[0] * (1 + near * torch.randn((nq, d), generator=g, device="cuda").double())).to(DTYPES[query])
    ids = make_ids(nq, k, 400)
    grad = torch.randn((nq, k), generator=g, device="cuda")
    there = (ids >= 0) & (ids < 400)
    got = binding.rago_q4_rescore_backward(codes, scales, q, ids, 32, "l2", grad).double()
    for r in range(nq):
        terms = 2 * grad[r][there[r]].double()[:, None] * (q[r].double() - w[ids[r][there[r]]])
        tol = SECOND_ORDER * (k + 6) * U * terms.abs().sum(0)
        if query == "bf16":
            tol = tol + 2.0 ** -8 * terms.sum(0).abs() + 1e-38
        assert ((got[r] - terms.sum(0)).abs() <= tol).all(), r


def test_results_do_not_change_from_call_to_call():
    codes, scales = make_rows(5000, 768, 64, torch.float32)
    q = make_queries(40, 768, torch.float32)
    ids = make_ids(40, 200, 5000)
    grad = torch.randn((40, 200), device="cuda")
    first = (binding.rago_q4_scores(codes, scales, q, 64), binding.rago_q4_rescore(codes, scales, q, ids, 64, "l2"),
             binding.rago_q4_rescore_backward(codes, scales, q, ids, 64, "l2", grad))
    for _ in range(3):
        again = (binding.rago_q4_scores(codes, scales, q, 64), binding.rago_q4_rescore(codes, scales, q, ids, 64, "l2"),
                 binding.rago_q4_rescore_backward(codes, scales, q, ids, 64, "l2", grad))
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("metric", ["l2", "ip"])
def test_the_gradient_agrees_with_differences(metric):
    """Central differences of the 64-bit distances along a direction: the distances are quadratic, so the differences are exact."""
    codes, scales = make_rows(90, 96, 32, torch.float32)
    q = make_queries(4, 96, torch.float32)
    ids = make_ids(4, 30, 90)
    there = (ids >= 0) & (ids < 90)
    g = torch.Generator(device="cuda").manual_seed(8)
    grad = torch.randn((4, 30), generator=g, device="cuda")
    along = torch.randn((4, 96), generator=g, device="cuda").double()
    w = values64(codes, scales, 32)[torch.where(there, ids, 0)]

    def loss(x):
        v = (x[:, None] - w).square().sum(2) if metric == "l2" else (x[:, None] * w).sum(2)
        return (torch.where(there, v, 0.0) * grad.double()).sum()

    slope = (loss(q.double() + 0.5 * along) - loss(q.double() - 0.5 * along))
    gx = binding.rago_q4_rescore_backward(codes, scales, q, ids, 32, metric, grad).double()
    mag = torch.where(there, grad.double().abs(), 0.0)[:, :, None] * (2 * (q.double().abs()[:, None] + w.abs()) if metric == "l2" else w.abs())
    assert abs((gx * along).sum() - slope) <= SECOND_ORDER * 36 * U * (mag.sum(1) * along.abs()).sum()


def test_rows_beyond_32_bit_byte_offsets():
    """4.4 GB of codes: the last rows lie behind offset 2^32."""
    d, N = 8192, 1_080_000
    codes = torch.zeros((N, d // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((N, d // 128), 0.5, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    tail = torch.randint(0, 256, (300, d // 2), generator=g, device="cuda", dtype=torch.uint8)
    codes[-300:] = tail
    q = make_queries(2, d, torch.bfloat16)
    w, x = values64(tail, scales[-300:], 128), q.double()
    tol = SECOND_ORDER * (d + 4) * U * (x.abs() @ w.abs().T)
    got = binding.rago_q4_scores(codes, scales, q, 128)
    assert ((got[:, -300:].double() - x @ w.T).abs() <= tol).all()
    first = (x.sum(1) * -4.0)[:, None]  # every number of a zero byte is -8 * 0.5
    assert ((got[:, :1000].double() - first).abs() <= SECOND_ORDER * (d + 4) * U * 4 * x.abs().sum(1)[:, None]).all()
    ids = torch.arange(N - 300, N, device="cuda").expand(2, 300).contiguous()
    assert ((binding.rago_q4_rescore(codes, scales, q, ids, 128, "ip").double() - x @ w.T).abs() <= tol).all()


def test_another_stream_and_a_captured_graph():
    codes, scales = make_rows(3000, 256, 64, torch.float32)
    q = make_queries(5, 256, torch.float32)
    ids = make_ids(5, 40, 3000)
    grad = torch.randn((5, 40), device="cuda")

    def calls():
        return (binding.rago_q4_scores(codes, scales, q, 64), binding.rago_q4_rescore(codes, scales, q, ids, 64, "ip"),
                binding.rago_q4_rescore_backward(codes, scales, q, ids, 64, "ip", grad))

    want = calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    q.copy_(make_queries(5, 256, torch.float32, seed=77))
    grad.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    want = calls()
    assert all(torch.equal(a, b) for a, b in zip(want, held))
