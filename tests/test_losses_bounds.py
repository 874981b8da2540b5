"""The bounds on gradients (tests/loss_bounds.py) notice mistakes in values far from the token: planted in
the definition's own gradient, on the CPU."""
import pytest
import torch

import loss_bounds as bounds
import loss_reference as ref

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def case(V, seed=0):
    g = torch.Generator().manual_seed(seed + V)
    x = 2.5 * torch.randn(2, 3, V, generator=g)
    tokens = torch.randint(0, V, (2, 3), generator=g)
    x.scatter_add_(-1, tokens.unsqueeze(-1), 8 * torch.rand(2, 3, 1, generator=g))
    return x, tokens, torch.randn(2, 3, generator=g).double(), torch.randn(2, 3, generator=g).double()


def gradient(x, tokens, d, d_h):
    valid = torch.ones(2, 3, dtype=torch.bool)
    leaf, logp = ref.rows(x, valid, 1.0)
    value = (ref.chosen(logp, tokens, valid) * d).sum()
    if d_h is not None:
        value = value + (ref.entropies(logp, valid) * d_h).sum()
    want, = torch.autograd.grad(value, leaf)
    logp = logp.detach()
    return want, bounds.of_softmax(logp, d, bounds.at_tokens(logp, tokens, d), d_h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [64, 1031, 32000])
@pytest.mark.parametrize("entropy", [False, True])
def test_planted_mistakes_are_noticed(V, entropy, dtype):
    x, tokens, d, d_h = case(V)
    d = torch.where(d.abs() < 0.1, torch.full_like(d, 0.3), d)       # (a cotangent of 0 has a gradient of 0)
    d_h = d_h if entropy else None
    scale = 4096.0 if dtype == torch.float16 else 1.0
    want, bound = gradient(x, tokens, d, d_h)
    right = (want * scale).to(dtype)
    assert not bounds.breaches(right, want, bound, dtype, scale).any()
    # float32 all along, as a kernel would: weights, their sum, the entropy
    z = x - x.amax(-1, keepdim=True)
    p = z.exp() / z.exp().sum(-1, keepdim=True)
    f = -p * d.float().unsqueeze(-1)
    f = f.scatter_add(-1, tokens.unsqueeze(-1), d.float().unsqueeze(-1))
    if entropy:
        log_p = z - z.exp().sum(-1, keepdim=True).log()
        f = f - p * (log_p - (p * log_p).sum(-1, keepdim=True)) * d_h.float().unsqueeze(-1)
    assert not bounds.breaches((f * scale).to(dtype), want, bound, dtype, scale).any()

    def planted(change):
        wrong = right.clone()
        change(wrong)
        return bounds.breaches(wrong, want, bound, dtype, scale)
    lo = 8 if tokens[1, 2] >= 32 else 40                             # a chunk without the token
    chunk = (1, 2, slice(lo, lo + 8))

    def zero(w): w[chunk] = 0
    def twice(w): w[chunk] *= 2
    def next_chunk(w): w[chunk] = right[1, 2, lo + 8:lo + 16]
    def token_twice(w): w[0, 1, tokens[0, 1]] *= 2
    def off_by_some(w): w[chunk] *= 1.01
    # float16 holds what is below its smallest step, 6e-8 / scale, with less than that
    visible = want[chunk].abs() > 4 * bounds.STEP[dtype] / scale
    assert visible.any()
    for change in (zero, twice):
        assert planted(change)[chunk][visible].all(), change.__name__
    assert planted(next_chunk)[chunk].any()
    assert planted(token_twice)[0, 1].sum() == 1
    if not entropy:
        assert planted(off_by_some)[chunk].any() or dtype == torch.float16
    wrong = torch.zeros_like(right)                                  # all but the token's value lost
    wrong.scatter_(-1, tokens.unsqueeze(-1), right.gather(-1, tokens.unsqueeze(-1)))
    assert bounds.breaches(wrong, want, bound, dtype, scale).double().mean() > 0.9 or dtype == torch.float16
