"""What the calls around a search refuse, before anything is launched (no GPU is needed: the checks are on the host)."""

import math

import pytest
import torch

from paper_2503_14649_b200 import binding

OK, EINVAL, EALIGN, EUNSUPPORTED, ENOMEM = 0, 1, 2, 3, 4
A = 4096  # an aligned address that nothing may read
F32, BF16 = binding.RAGO_F32, binding.RAGO_BF16


def call(name, defaults, **changes):
    args = dict(defaults, **changes)
    assert set(args) == set(defaults)
    L = binding.lib()
    before = binding.rago_kernel_launches()
    status = getattr(L, name)(*args.values())
    assert binding.rago_kernel_launches() == before, "something was launched"
    if status:
        assert L.rago_last_error()
    return status


ROWS = dict(codes=A, scales=A, scale_dtype=F32, N=10, d=64, group=32, queries=A, query_dtype=F32, nq=3)
SCORES = dict(ROWS, out=A, stream=None)
RESCORE = dict(ROWS, ids=A, k=5, metric=binding.RAGO_L2, out=A, stream=None)
RESCORE_BACKWARD = dict(ROWS, ids=A, k=5, metric=binding.RAGO_IP, grad=A, out=A, stream=None)

ROW_REFUSALS = [
    (EINVAL, dict(N=-1)), (EINVAL, dict(nq=-1)), (EINVAL, dict(d=0)), (EINVAL, dict(scale_dtype=2)), (EINVAL, dict(query_dtype=-1)),
    (EINVAL, dict(codes=None)), (EINVAL, dict(scales=None)), (EINVAL, dict(queries=None)), (EINVAL, dict(out=None)),
    (EALIGN, dict(codes=A + 8)), (EALIGN, dict(queries=A + 4)), (EALIGN, dict(scales=A + 2)), (EALIGN, dict(scales=A + 1, scale_dtype=BF16)),
    (EUNSUPPORTED, dict(group=16)), (EUNSUPPORTED, dict(group=96)), (EUNSUPPORTED, dict(group=0)), (EUNSUPPORTED, dict(d=48)),
    (EUNSUPPORTED, dict(d=8224)), (EUNSUPPORTED, dict(N=1 << 31)),
]


@pytest.mark.parametrize("status,changes", ROW_REFUSALS)
def test_rows_in_4_bits(status, changes):
    assert call("rago_q4_scores", SCORES, **changes) == status
    assert call("rago_q4_rescore", RESCORE, **changes) == status
    assert call("rago_q4_rescore_backward", RESCORE_BACKWARD, **changes) == status


@pytest.mark.parametrize("status,changes", [(EINVAL, dict(k=0)), (EINVAL, dict(metric=2)), (EINVAL, dict(ids=None)),
                                            (EUNSUPPORTED, dict(k=1 << 30))])
def test_candidates(status, changes):
    assert call("rago_q4_rescore", RESCORE, **changes) == status
    assert call("rago_q4_rescore_backward", RESCORE_BACKWARD, **changes) == status


def test_gradients_of_candidates():
    assert call("rago_q4_rescore_backward", RESCORE_BACKWARD, grad=None) == EINVAL
    assert call("rago_q4_rescore_backward", RESCORE_BACKWARD, out=A + 8) == EALIGN


def test_nothing_to_do_is_not_an_error():
    assert call("rago_q4_scores", SCORES, nq=0, queries=None, out=None) == OK
    assert call("rago_q4_scores", SCORES, N=0, codes=None, scales=None, out=None) == OK
    assert call("rago_q4_rescore", RESCORE, nq=0, queries=None, ids=None, out=None) == OK
    assert call("rago_q4_rescore_backward", RESCORE_BACKWARD, nq=0, queries=None, ids=None, grad=None, out=None) == OK
    assert call("rago_policy_loss", POLICY, nq=0) == OK
    assert call("rago_policy_loss_backward", POLICY_BACKWARD, nq=0) == OK
    assert call("rago_list_balance_backward", BALANCE_BACKWARD, nq=0) == OK


POLICY_IN = dict(scores=A, ref=A, dtype=F32, ids=A, nq=2, C=10, scale=1.0, chosen=A, old=A, adv=A, G=3, low=0.2, high=0.2)
POLICY = dict(POLICY_IN, policy=A, kl=A, logp=A, stats=A, workspace=None, workspace_bytes=0, stream=None)
POLICY_BACKWARD = dict(POLICY_IN, kl=A, logp=A, stats=A, grad_policy=A, grad_kl=A, grad=A, stream=None)
POLICY_REFUSALS = [
    (EINVAL, dict(nq=-1)), (EINVAL, dict(C=0)), (EINVAL, dict(G=-1)), (EINVAL, dict(dtype=5)), (EINVAL, dict(scale=0.0)),
    (EINVAL, dict(scale=math.inf)), (EINVAL, dict(scale=math.nan)), (EUNSUPPORTED, dict(scale=-3e38)), (EUNSUPPORTED, dict(scale=1.5e31)), (EINVAL, dict(low=-0.1)),
    (EINVAL, dict(low=1.5)), (EINVAL, dict(low=math.nan)), (EINVAL, dict(high=-0.1)), (EINVAL, dict(high=math.nan)),
    (EINVAL, dict(scores=None)), (EINVAL, dict(chosen=None)), (EINVAL, dict(old=None)), (EINVAL, dict(adv=None)),
    (EINVAL, dict(kl=None)), (EINVAL, dict(logp=None)), (EINVAL, dict(stats=None)),
    (EALIGN, dict(scores=A + 2)), (EALIGN, dict(ref=A + 2)), (EALIGN, dict(ids=A + 4)), (EALIGN, dict(stats=A + 8)),
    (EALIGN, dict(scores=A + 1, dtype=BF16)),
    (EUNSUPPORTED, dict(G=1025)), (EUNSUPPORTED, dict(nq=1 << 30, C=1 << 10)),
]


@pytest.mark.parametrize("status,changes", POLICY_REFUSALS)
def test_policy_loss(status, changes):
    assert call("rago_policy_loss", POLICY, **changes) == status
    assert call("rago_policy_loss_backward", POLICY_BACKWARD, **changes) == status


def test_policy_loss_outputs():
    assert call("rago_policy_loss", POLICY, policy=None) == EINVAL
    assert call("rago_policy_loss_backward", POLICY_BACKWARD, grad=None) == EINVAL
    assert call("rago_policy_loss_backward", POLICY_BACKWARD, grad_policy=None) == EINVAL
    assert call("rago_policy_loss_backward", POLICY_BACKWARD, grad_kl=None) == EINVAL
    assert call("rago_policy_loss_backward", POLICY_BACKWARD, grad=A + 2) == EALIGN


def test_policy_loss_workspace():
    long = dict(nq=3, C=100_000)
    need = binding.rago_policy_workspace_bytes(3, 100_000)
    assert need >= 3 * 7 * 20 and binding.rago_policy_workspace_bytes(5000, 16_384) == 0
    assert call("rago_policy_loss", POLICY, **long) == EINVAL
    assert call("rago_policy_loss", POLICY, workspace=A + 16, workspace_bytes=need, **long) == EALIGN
    assert call("rago_policy_loss", POLICY, workspace=A, workspace_bytes=need - 1, **long) == ENOMEM
    with pytest.raises(binding.RagoError):
        binding.rago_policy_workspace_bytes(3, 0)
    with pytest.raises(binding.RagoError):
        binding.rago_policy_workspace_bytes(-1, 5)


BALANCE = dict(logits=A, dtype=F32, nq=4, nlist=16, scale=1.0, lists=A, nprobe=2, valid=None, loss=A, counts=A, stats=A, stream=None)
BALANCE_BACKWARD = dict(logits=A, dtype=F32, nq=4, nlist=16, scale=1.0, valid=None, counts=A, stats=A, grad_loss=A, grad=A, stream=None)


@pytest.mark.parametrize("status,changes", [
    (EINVAL, dict(nq=-1)), (EINVAL, dict(nlist=0)), (EINVAL, dict(dtype=2)), (EINVAL, dict(scale=0.0)), (EINVAL, dict(scale=math.inf)),
    (EINVAL, dict(logits=None)), (EINVAL, dict(counts=None)), (EINVAL, dict(stats=None)), (EALIGN, dict(logits=A + 2)),
    (EALIGN, dict(stats=A + 4)), (EALIGN, dict(logits=A + 1, dtype=BF16))])
def test_list_balance(status, changes):
    assert call("rago_list_balance", BALANCE, **changes) == status
    assert call("rago_list_balance_backward", BALANCE_BACKWARD, **changes) == status


@pytest.mark.parametrize("scale", [9e-37, -9e-37, 1e-44])
def test_list_balance_scales_that_would_lose_differences_of_logits(scale):
    assert call("rago_list_balance", BALANCE, scale=scale) == EUNSUPPORTED
    assert call("rago_list_balance_backward", BALANCE_BACKWARD, scale=scale) == EUNSUPPORTED


def test_list_balance_inputs_and_outputs():
    assert call("rago_list_balance", BALANCE, nprobe=0) == EINVAL
    assert call("rago_list_balance", BALANCE, lists=None) == EINVAL
    assert call("rago_list_balance", BALANCE, loss=None) == EINVAL
    assert call("rago_list_balance", BALANCE, nq=1 << 20, nprobe=1 << 11) == EUNSUPPORTED
    assert call("rago_list_balance_backward", BALANCE_BACKWARD, grad_loss=None) == EINVAL
    assert call("rago_list_balance_backward", BALANCE_BACKWARD, grad=None) == EINVAL
    assert call("rago_list_balance_backward", BALANCE_BACKWARD, grad=A + 2) == EALIGN


@pytest.mark.parametrize("name,defaults,pointers", [
    ("rago_q4_scores", SCORES, {"out": 4}),
    ("rago_q4_rescore", RESCORE, {"ids": 8, "out": 4}),
    ("rago_q4_rescore_backward", RESCORE_BACKWARD, {"ids": 8, "grad": 4}),
    ("rago_policy_loss", POLICY, {"chosen": 4, "old": 4, "adv": 4, "policy": 4, "kl": 4, "logp": 4}),
    ("rago_policy_loss_backward", POLICY_BACKWARD, {"chosen": 4, "old": 4, "adv": 4, "kl": 4, "logp": 4, "grad_policy": 4, "grad_kl": 4}),
    ("rago_list_balance", BALANCE, {"lists": 4, "loss": 4, "counts": 4}),
    ("rago_list_balance_backward", BALANCE_BACKWARD, {"counts": 4, "grad_loss": 4})])
def test_pointers_that_are_not_aligned_to_their_type(name, defaults, pointers):
    for pointer, size in pointers.items():
        for off in (1, 2, size // 2, size - 1):
            assert call(name, defaults, **{pointer: A + off}) == EALIGN, pointer


# ---- the binding: tensors that the library would read as something else ----------------------------------------------------

def test_tensors_on_the_host_and_of_other_shapes_or_types():
    codes, scales = torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 2))
    q, ids = torch.zeros((2, 64)), torch.zeros((2, 5), dtype=torch.int64)
    with pytest.raises(ValueError, match="codes"):
        binding.rago_q4_scores(codes, scales, q, 32)
    with pytest.raises(ValueError, match="codes"):
        binding.rago_q4_rescore(codes.int(), scales, q, ids, 32, "l2")
    with pytest.raises(ValueError):
        binding.rago_q4_rescore_backward(codes[0], scales, q, ids, 32, "l2", torch.zeros((2, 5)))
    with pytest.raises(ValueError):
        binding.rago_q4_scores(codes, scales, q, 0)
    x, ch, f = torch.zeros((2, 6)), torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3))
    with pytest.raises(ValueError, match="scores"):
        binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2)
    with pytest.raises(ValueError):
        binding.rago_policy_loss(x[0], ch, f, f, 1.0, 0.2, 0.2)
    with pytest.raises(ValueError, match="logits"):
        binding.rago_list_balance(x, ch, 1.0)
    with pytest.raises(ValueError):
        binding.rago_list_balance(x, ch[0], 1.0)


def test_a_workspace_that_the_library_would_not_write_as_it_is(monkeypatch):
    """The other tensors stand for ones on the GPU here: the workspace is what is refused."""
    x, ch, f = torch.zeros((2, 20_000)), torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3))
    expect = binding._expect

    def only_the_workspace(name, t, *a):
        if name == "workspace":
            expect(name, t, *a)

    monkeypatch.setattr(binding, "_expect", only_the_workspace)
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    for w in (torch.zeros(4096, dtype=torch.uint8), torch.zeros(1024), torch.zeros(8192, dtype=torch.uint8)[::2], torch.zeros((2, 2048), dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace"):
            binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2, workspace=w)


def test_the_binding_knows_which_rows_need_a_workspace():
    assert binding.rago_policy_workspace_bytes(7, binding.POLICY_SPAN) == 0 < binding.rago_policy_workspace_bytes(7, binding.POLICY_SPAN + 1)


@pytest.mark.gpu
def test_workspaces_on_the_gpu():
    x, ch, f = torch.randn((2, 20_000), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda")
    need = binding.rago_policy_workspace_bytes(2, 20_000)
    want = binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2)
    room = torch.full((need + 64,), 7, dtype=torch.uint8, device="cuda")
    got = binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2, workspace=room[:need])
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and (room[need:] == 7).all()
    numbers = torch.zeros((2, need // 8), device="cuda")  # any contiguous tensor will do
    got = binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2, workspace=numbers)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for w in (torch.zeros(need, dtype=torch.uint8), torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2, workspace=w)
    with pytest.raises(binding.RagoError):
        binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2, workspace=room[:need - 1])


@pytest.mark.gpu
def test_tensors_on_the_gpu_of_other_shapes_types_or_orders():
    codes, scales = torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros((8, 2), device="cuda")
    q, ids = torch.zeros((2, 64), device="cuda"), torch.zeros((2, 5), dtype=torch.int64, device="cuda")
    g = torch.zeros((2, 5), device="cuda")
    wrong = [(codes.cpu(), scales, q), (codes, scales.cpu(), q), (codes, scales, q.cpu()), (codes, scales[:, :1], q), (codes, scales.half(), q),
             (codes, scales, q.half()), (codes, scales, q[:, :32]), (codes.t().contiguous().t(), scales, q), (codes, scales[:7], q)]
    for c, s, x in wrong:
        with pytest.raises(ValueError):
            binding.rago_q4_scores(c, s, x, 32)
        with pytest.raises(ValueError):
            binding.rago_q4_rescore(c, s, x, ids, 32, "l2")
    for i in (ids.int(), ids[:1], ids.cpu(), torch.zeros((2, 10), dtype=torch.int64, device="cuda")[:, ::2]):
        with pytest.raises(ValueError):
            binding.rago_q4_rescore(codes, scales, q, i, 32, "ip")
        with pytest.raises(ValueError):
            binding.rago_q4_rescore_backward(codes, scales, q, i, 32, "ip", g)
    with pytest.raises(ValueError):
        binding.rago_q4_rescore_backward(codes, scales, q, ids, 32, "ip", g.double())
    with pytest.raises(ValueError):
        binding.rago_q4_scores(codes, scales, q, 32, out=torch.zeros((2, 9), device="cuda"))
    with pytest.raises(binding.RagoError):
        binding.rago_q4_scores(codes, torch.zeros((8, 4), device="cuda"), q, 16)
    x, ch, f = torch.zeros((2, 6), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda")
    fwd = binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2, ref_scores=x)
    one = torch.ones(2, device="cuda")
    for bad in (dict(ref_scores=x.bfloat16()), dict(ids=torch.zeros((2, 6), dtype=torch.int32, device="cuda")), dict(ref_scores=x[:1])):
        with pytest.raises(ValueError):
            binding.rago_policy_loss(x, ch, f, f, 1.0, 0.2, 0.2, **bad)
    with pytest.raises(ValueError):
        binding.rago_policy_loss(x, ch.long(), f, f, 1.0, 0.2, 0.2)
    with pytest.raises(ValueError, match="grad_kl"):
        binding.rago_policy_loss_backward(x, ch, f, f, 1.0, 0.2, 0.2, fwd, one, ref_scores=x)
    with pytest.raises(ValueError):
        binding.rago_policy_loss_backward(x, ch, f, f, 1.0, 0.2, 0.2, fwd, one[:1], one, ref_scores=x)
    b = binding.rago_list_balance(x, ch, 1.0)
    with pytest.raises(ValueError):
        binding.rago_list_balance(x, ch, 1.0, valid=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        binding.rago_list_balance_backward(x[:, :5].contiguous(), 1.0, b, b.loss)
    with pytest.raises(ValueError):
        binding.rago_list_balance_backward(x, 1.0, b, one)
