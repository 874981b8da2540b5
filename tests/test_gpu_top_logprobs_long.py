"""Top log-probabilities where the kernels for many long rows are: float16 at every length that they tell apart, up to 1024
alternatives of rows taken tile by tile, parts whose bounds let more through than a join holds.  Against sorted float64 on
the GPU, in the tolerances of test_gpu_top_logprobs.py; and a gradient against differences, every direction of which
counts."""
import math

import pytest
import torch

import paper_2510_05485_amd as tb
from paper_2510_05485_amd import losses
from test_gpu_losses import DEV, H, LP, TYPES
from test_gpu_top_logprobs import LENGTHS

pytestmark = pytest.mark.gpu


def check(x, tokens, mask, ks, at_a_time=200):
    """Rows [N, V] whose distributions exist; those of -inf and of the type's lowest value among them."""
    found = [tb.top_logprobs(x, k, tokens, mask=mask, want_entropy=True) for k in ks]
    for lo in range(0, len(x), at_a_time):
        rows = slice(lo, lo + at_a_time)
        part, live = x[rows].double(), mask[rows].unsqueeze(-1)
        order = (part + 0.0).sort(dim=-1, descending=True, stable=True)
        logp = torch.log_softmax(part, -1)
        lp = logp.gather(-1, tokens[rows].unsqueeze(-1)).squeeze(-1)
        held = logp.clamp(min=-1e6)
        h = -(held.exp() * held).sum(-1)
        for k, r in zip(ks, found):
            there = (order.values[:, :k] > -math.inf) & live
            ids = torch.where(there, order.indices[:, :k], -1)
            assert torch.equal(r.ids[rows], ids), (k, lo, (r.ids[rows] != ids).any(-1).nonzero()[:5].flatten().tolist())
            want, got = torch.where(there, logp.gather(-1, ids.clamp(min=0)), -math.inf), r.logprobs[rows].double()
            low = ~(want > -1e4)                                               # (the type's lowest value, or none)
            assert torch.equal(low, ~(got > -1e4))
            assert torch.equal(want == -math.inf, got == -math.inf)
            assert ((got - want)[~low].abs() <= LP).all(), k
            fine = mask[rows] & (lp > -1e4)
            assert ((r.token_logprobs[rows].double() - lp)[fine].abs() <= LP).all(), k
            assert ((r.entropy[rows].double() - h)[mask[rows]].abs() <= H).all(), k
            assert not r.token_logprobs[rows][~mask[rows]].any() and not r.entropy[rows][~mask[rows]].any()


def rows_of(N, V, dtype):
    """Most of them normal; below 0, large values next to one another, in order, equal, masked."""
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(N, V, generator=g, device=DEV) * 3
    x[3] -= 100
    x[4, V // 2:V // 2 + 700] += 20
    x[5] = x[5].sort().values
    x[6] = x[6].sort(descending=True).values
    x[7, :] = 1.25
    x[8, : V - 40] = -math.inf
    x[9, 40:] = torch.finfo(dtype).min
    x = x.to(dtype)
    tokens = torch.randint(0, V, (N,), generator=g, device=DEV)
    tokens[8] = V - 1
    mask = torch.ones(N, dtype=torch.bool, device=DEV)
    mask[[0, N // 6, N - 1]] = False
    return x, tokens, mask


@pytest.mark.parametrize("V", LENGTHS)
def test_many_rows_of_float16(V):
    check(*rows_of(600, V, torch.float16), (20, 300))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(300, 140_001), (300, 262_144), (600, 100_003), (200, 524_291)])
def test_many_alternatives_tile_by_tile(N, V, dtype):
    """(200 rows: two parts or three, each of them in tiles)"""
    check(*rows_of(N, V, dtype), (512, 600, 1024), at_a_time=50)


@pytest.mark.parametrize("dtype", TYPES)
def test_one_part_far_below_the_others(dtype):
    """The smallest of the parts' bounds is that of the low one, the largest K-th key lets through nearly all of the other
    parts' entries: the K-th of these is searched for."""
    V, K = 262_144, 1024
    size = torch.finfo(dtype).bits // 8
    parts = V * size // 65536
    g = torch.Generator(device=DEV).manual_seed(size)
    x = (torch.randn(3, V, generator=g, device=DEV) * 3).to(dtype)
    x[0, : V // parts] -= 50
    x[1, V - V // parts:] = -math.inf
    x[2, : V // parts] = torch.finfo(dtype).min
    # (what is let through, by the rule written out again; a part has 64 values more or fewer than another at most)
    best = x.float().view(3, parts, V // parts).topk(K, dim=-1).values
    bound = torch.maximum(best[..., -1].amax(-1), best[..., -(-K // parts) - 1].amin(-1))
    assert ((best >= bound[:, None, None]).sum((1, 2)) > 2048).all()
    tokens = torch.randint(V // parts, V - V // parts, (3,), generator=g, device=DEV)
    check(x, tokens, torch.ones(3, dtype=torch.bool, device=DEV), (K,))


def test_gradient_against_differences():
    """In float32, along random directions, of logits that lie too far apart for their order to change: 0.25, and steps
    move them by 2^-7 at most.  A difference over 2 h is off by h^2 / 6 times a third derivative and by the values' own
    errors, LP and H, over h.  Third derivatives along a direction of at most 1: of a log-probability a third central
    moment of numbers in [-1, 1], below 1; of an entropy that, and a joint fourth cumulant of these three times and of z in
    [-5, 5], below 10 * 2^3 + 3 * (10 * 2) * 2^2 = 320."""
    V, k, h = 40, 6, 2.0 ** -7
    g = torch.Generator().manual_seed(5)
    x = torch.stack([torch.randperm(V, generator=g), torch.randperm(V, generator=g)]).unsqueeze(0).float().to(DEV) * 0.25 - 5
    tokens = torch.randint(0, V, (1, 2), generator=g).to(DEV)
    d_top, d_lp, d_h = (torch.randn(*s, generator=g).to(DEV) for s in ((1, 2, k), (1, 2), (1, 2)))

    def value(y):
        r = tb.top_logprobs(y, k, tokens, want_entropy=True)
        return ((r.logprobs.double() * d_top).sum() + (r.token_logprobs.double() * d_lp).sum() + (r.entropy.double() * d_h).sum()), r.ids
    leaf = x.clone().requires_grad_()
    v, ids = value(leaf)
    grad, = torch.autograd.grad(v, leaf)
    of_lp, of_h = float(d_top.abs().sum() + d_lp.abs().sum()), float(d_h.abs().sum())
    for _ in range(8):
        step = (torch.rand(1, 2, V, generator=g) * 2 - 1).to(DEV)
        # (as far as float32 takes the logits: their differences are exact)
        high, low = x + h * step, x - h * step
        (up, ids_up), (down, ids_down) = value(high), value(low)
        assert torch.equal(ids_up, ids) and torch.equal(ids_down, ids)
        moved = float((grad.double() * (high.double() - low.double())).sum()) / (2 * h)
        allowed = h * h / 6 * (of_lp + 321 * of_h) + (LP * of_lp + H * of_h) / h
        assert abs(float(up - down) / (2 * h) - moved) <= allowed


def test_the_longest_row():
    """A row of as many values as there may be, equal ones but for some at its ends and between; and its gradient."""
    V, k = losses.VALUES_MOST, 6
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB of the GPU's memory")
    x = torch.zeros(1, V, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([V - 1, V // 2 + 1, 0, V - 70], device=DEV)
    x[0, at] = torch.tensor([9.0, 8.0, 7.0, 6.0], dtype=torch.bfloat16, device=DEV)
    token = at[1:2]
    x.requires_grad_()
    r = tb.top_logprobs(x, k, token)
    assert r.ids.tolist() == [[V - 1, V // 2 + 1, 0, V - 70, 1, 2]]
    total = V - 4 + sum(math.exp(v) for v in (9, 8, 7, 6))
    want = torch.tensor([9.0, 8.0, 7.0, 6.0, 0.0, 0.0], dtype=torch.float64, device=DEV) - math.log(total)
    assert (r.logprobs[0].double() - want).abs().max() <= LP
    assert torch.equal(r.token_logprobs, r.logprobs[:, 1])
    with torch.no_grad():
        assert (tb.token_logprobs(x, token).double() - want[1]).abs().max() <= LP
    grad, = torch.autograd.grad(r.token_logprobs.sum(), x)
    # -p of the others: 2^-31 and what the logits have; log s, and so 1 / s, is within LP, and one rounding
    for i, z in ((1, 0.0), (V - 2, 0.0), (V - 1, 9.0), (0, 7.0)):
        p = math.exp(z) / total
        assert abs(float(grad[0, i]) + p) <= p * (2.0 ** -8 + 2 * LP), i
    assert abs(float(grad[0, V // 2 + 1]) - 1) <= 2.0 ** -8
