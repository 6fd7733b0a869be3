"""The calls around a search at the largest sizes that their interface takes, where sizes and offsets stop fitting 32 bits.

Values are such that the results are known without a second computation of that size: all alike but a few."""

import math

import pytest
import torch

from paper_2503_14649_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
MOST = 2 ** 31 - 1


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("C", [MOST, 2 ** 31 - 8192, 2 ** 31 - 16_384])
def test_policy_over_the_longest_row(C):
    """Scores 0 but for three of log C: Z = C - 3 + 3 C.  Sums of at most 64 + C / 16 384 / 256 terms and the joins: log pi is off by less than
    1000 u (of 23), pi by as much of itself, and a gradient in bf16 by half a step, 2^-8."""
    s = math.log(C)
    at = [0, C // 2, C - 1]
    scores = torch.zeros((1, C), dtype=torch.bfloat16, device="cuda")
    high = torch.tensor(s, dtype=torch.bfloat16).item()
    scores[0, at] = high
    chosen = torch.tensor([[C - 1, 5, C - 2]], dtype=torch.int32, device="cuda")
    logz = math.log(C - 3 + 3 * math.exp(high))
    logp = torch.tensor([[high - logz, -logz, -logz]], dtype=torch.float64, device="cuda")
    old = (logp - 0.05).float()
    adv = torch.tensor([[1.0, -2.0, 0.5]], device="cuda")
    f = binding.rago_policy_loss(scores, chosen, old, adv, 1.0, 0.2, 0.2)
    assert ((f.logp.double() - logp).abs() <= 1000 * U).all()
    slope = -(logp - old.double()).exp() * adv.double()
    assert abs(float(f.policy[0]) - float(slope.sum())) <= 3000 * U * float(slope.abs().sum())
    grad = binding.rago_policy_loss_backward(scores, chosen, old, adv, 1.0, 0.2, 0.2, f, torch.ones(1, device="cuda"))[0]
    H = float(slope.sum())
    flat = -math.exp(-logz) * H
    own = {C - 1: float(slope[0, 0]), 5: float(slope[0, 1]), C - 2: float(slope[0, 2])}
    for i in {*at, 1, 5, 6, C // 3, C - 2, C - 3, C - 16_385, C - 8193, C - 8191}:
        want = own.get(i, 0.0) - math.exp((high if i in at else 0.0) - logz) * H
        assert abs(float(grad[i]) - want) <= (2.0 ** -8 + 4000 * U) * abs(want) + 3000 * U * abs(own.get(i, 0.0)), i
    # every other number is the same
    same = torch.tensor(flat, dtype=torch.float64, device="cuda")
    odd = 0
    for part in grad.split(1 << 28):
        odd += int(((part.double() - same).abs() > (2.0 ** -8 + 4000 * U) * abs(flat)).sum())
    assert odd == len({*at, *own})


def test_the_largest_batch_of_policies_and_of_lists():
    """2^31 - 1 rows of one and of two numbers."""
    scores = torch.zeros((MOST, 1), dtype=torch.bfloat16, device="cuda")
    none = torch.empty((MOST, 0), device="cuda")
    f = binding.rago_policy_loss(scores, none.int(), none, none, 1.0, 0.2, 0.2)
    assert not f.policy.any() and not f.kl.any()
    assert (f.stats[-3:] == torch.zeros(4, device="cuda")).all()
    out = torch.ones_like(scores)
    binding.rago_policy_loss_backward(scores, none.int(), none, none, 1.0, 0.2, 0.2, f, f.kl, out=out)
    assert not out.any()
    del f, out, scores
    torch.cuda.empty_cache()
    # all slots on list 0, p = e / (1 + e) for it: the loss is 2 p, summed over 2^26 CTAs' sums by 256 threads, 2^18 terms each
    logits = torch.zeros((MOST, 2), dtype=torch.bfloat16, device="cuda")
    logits[:, 0] = 1.0
    lists = torch.zeros((MOST, 1), dtype=torch.int32, device="cuda")
    b = binding.rago_list_balance(logits, lists, 1.0)
    p = 1 / (1 + math.exp(-1.0))
    assert b.counts.tolist() == [MOST, 0]
    assert abs(float(b.loss[0]) - 2 * p) <= 2 * p * (2 ** 18 + 100) * U
    grad = binding.rago_list_balance_backward(logits, 1.0, b, torch.full((1,), 1e9, device="cuda"))
    want = 1e9 * 2 / MOST * p * (1 - p)
    for part in grad.split(1 << 28):
        assert ((part[:, 0].double() - want).abs() <= (2.0 ** -8 + 100 * U) * want).all() and ((part[:, 1].double() + want).abs() <= (2.0 ** -8 + 100 * U) * want).all()


def test_the_longest_list_of_candidates():
    """One query, 2^31 - 1 candidates of 50 rows; all but 700 at either end have gradient 0."""
    g = torch.Generator(device="cuda").manual_seed(0)
    codes = torch.randint(0, 256, (50, 16), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.rand((50, 1), generator=g, device="cuda") + 0.1
    q = torch.randn((1, 32), generator=g, device="cuda")
    ids = torch.empty((1, MOST), dtype=torch.int64, device="cuda")
    for i in range(0, MOST, 1 << 28):
        j = min(MOST, i + (1 << 28))
        ids[0, i:j] = torch.arange(i, j, device="cuda") % 51          # row 50 is missing
    few = torch.arange(51, device="cuda")[None].contiguous()
    table = binding.rago_q4_rescore(codes, scales, q, few, 32, "l2")[0]
    assert table[50] == math.inf
    got = binding.rago_q4_rescore(codes, scales, q, ids, 32, "l2")[0]
    for i in range(0, MOST, 1 << 26):
        assert torch.equal(got[i:i + (1 << 26)], table[ids[0, i:i + (1 << 26)]])
    del got
    grad = torch.zeros((1, MOST), device="cuda")
    ends = torch.cat((torch.arange(700, device="cuda"), torch.arange(MOST - 700, MOST, device="cuda")))
    grad[0, ends] = torch.randn(1400, generator=g, device="cuda")
    gx = binding.rago_q4_rescore_backward(codes, scales, q, ids, 32, "l2", grad)[0].double()
    w = torch.stack((codes.long() % 16, codes.long() // 16), 2).flatten(1).double() - 8
    w = w * scales.double()
    there = ids[0, ends] < 50
    terms = 2 * grad[0, ends][there].double()[:, None] * (q.double() - w[ids[0, ends][there]])
    assert ((gx - terms.sum(0)).abs() <= 1.05 * 1410 * U * terms.abs().sum(0)).all()    # a term of 0 adds no rounding


@pytest.mark.parametrize("nlist", [MOST, 2 ** 31 - 5])
def test_the_largest_number_of_lists(nlist):
    """Even p, two slots: Z and the counts are whole numbers below 2^32 of few bits, sums of 8s and 1s."""
    logits = torch.zeros((2, nlist), dtype=torch.bfloat16, device="cuda")
    lists = torch.tensor([[0], [nlist - 1]], dtype=torch.int32, device="cuda")
    b = binding.rago_list_balance(logits, lists, 1.0)
    assert int(b.counts[0]) == int(b.counts[-1]) == 1 and not b.counts[1:-1].any()
    assert abs(float(b.loss[0]) - 1) <= 100 * U
    out = torch.full((2, nlist), 5.0, dtype=torch.bfloat16, device="cuda")
    binding.rago_list_balance_backward(logits, 1.0, b, torch.full((1,), 1e9, device="cuda"), out=out)
    p = 1.0 / nlist
    k = 1e9 * nlist / 2
    ends, rest = k * p * (0.5 - p), -k * p * p
    for row in out:
        assert abs(float(row[0]) - ends) <= (2.0 ** -8 + 100 * U) * ends and abs(float(row[-1]) - ends) <= (2.0 ** -8 + 100 * U) * ends
        for part in row[1:-1].split(1 << 28):
            assert ((part.double() - rest).abs() <= (2.0 ** -8 + 100 * U) * -rest).all()
