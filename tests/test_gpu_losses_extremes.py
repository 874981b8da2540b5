"""Losses over logits of extreme size: rows whose numbers are too large for their products with log2(e) to
be exact, parts of a row that lie far apart, infinite margins, huge cotangents, wide lengths."""
import math

import pytest
import torch

import loss_bounds as bounds
import loss_reference as ref
import paper_2510_05485_amd as tb
from loss_bounds import LP

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def near(got, want, tol, what=""):
    off = (got.detach().cpu().double() - want).abs()
    assert (off <= tol).all(), (what, got, want)


def large_rows(base, V, dtype, T=4):
    """Rows around `base`: all alike, half of them impossible, some one step below, one step above the rest."""
    g = torch.Generator().manual_seed(V)
    b = torch.tensor(base, dtype=torch.float32).to(dtype)
    below, above = (torch.nextafter(b, torch.tensor(s * math.inf, dtype=dtype)) for s in (-1, 1))
    x = b.expand(2, T, V).clone()
    tokens = torch.randint(0, V, (2, T), generator=g)
    some = torch.rand(2, T, V, generator=g) < 0.5
    some = some.scatter(-1, tokens.unsqueeze(-1), False)
    x[:, 1] = torch.where(some[:, 1], torch.full_like(x[:, 1], -math.inf), x[:, 1])
    x[:, 2] = torch.where(some[:, 2], below.expand_as(x[:, 2]), x[:, 2])
    x[:, 3] = x[:, 3].scatter(-1, tokens[:, 3:], above.expand(2, 1))
    return x.to(DEV), tokens.to(DEV)


BASES = [1e6, -1e8, 3e8, 1e10, -1e10, 3e12, 1e20, -1e20, -1e30, 1e36]


@pytest.mark.parametrize("base", BASES)
@pytest.mark.parametrize("dtype,V", [(torch.float32, 64), (torch.float32, 2500), (torch.float32, 20011),
                                     (torch.bfloat16, 3), (torch.bfloat16, 1031), (torch.bfloat16, 5000),
                                     (torch.bfloat16, 50257), (torch.float32, 140000)])
def test_large_logits(dtype, V, base):
    x, tokens = large_rows(base, V, dtype)
    valid = torch.ones(2, 4, dtype=torch.bool)
    rx, logp = ref.rows(x, valid, 1.0)
    p = logp.detach()
    # what is far below has probability 0 in either: keep infinities out of the bounds
    p = p.clamp(min=-1e4)
    lp, h = ref.chosen(logp, tokens, valid), ref.entropies(logp, valid)
    d, d_h = torch.tensor([1.0, -0.5, 2.0, 0.7]).double().expand(2, 4), torch.tensor([0.3, 1.0, -1.0, 0.5]).double().expand(2, 4)
    leaf = x.clone().requires_grad_()
    got_lp, got_h = tb.token_logprobs(leaf, tokens, want_entropy=True)
    near(got_lp, lp.detach(), LP, "log-probabilities")
    near(got_h, h.detach(), bounds.H, "entropies")
    want, = torch.autograd.grad((lp * d).sum() + (h * d_h).sum(), rx, retain_graph=True)
    got, = torch.autograd.grad((got_lp, got_h), leaf, (d.float().to(DEV), d_h.float().to(DEV)))
    bounds.check(got, want, bounds.of_softmax(p, d, bounds.at_tokens(p, tokens.cpu(), d), d_h), dtype, "of both")
    want, = torch.autograd.grad((lp * d).sum(), rx)
    got, = torch.autograd.grad(tb.token_logprobs(leaf, tokens), leaf, d.float().to(DEV))
    bounds.check(got, want, bounds.of_softmax(p, d, bounds.at_tokens(p, tokens.cpu(), d)), dtype, "of log-probabilities")

    one = torch.ones(2, 4).double()
    old, a = (lp.detach() - 0.1).float().to(DEV), torch.tensor([1.0, -1.0], device=DEV)
    terms, want, _ = ref.policy(x, tokens, old, a, average="sum")
    bound = bounds.of_softmax(p, 1.2 * one, bounds.at_tokens(p, tokens.cpu(), 1.2 * one))
    bounds.check(tb.policy_loss_grad(x, tokens, old, a, average="sum").grad, want, bound, dtype, "policy")
    got, = torch.autograd.grad(tb.policy_loss(leaf, tokens, old, a, average="sum"), leaf)
    bounds.check(got, want, bound, dtype, "policy, backward")

    reference = (lp.detach() + 0.2).float().to(DEV)
    terms, want, _, margins = ref.preference(x, tokens, reference)
    bound = bounds.of_softmax(p, 0.1 * one, bounds.at_tokens(p, tokens.cpu(), 0.1 * one))
    r = tb.preference_loss_grad(x, tokens, reference)
    near(r.margins, margins, 8 * LP, "margins")
    bounds.check(r.grad, want, bound, dtype, "preference")
    got, = torch.autograd.grad(tb.preference_loss(leaf, tokens, reference), leaf)
    bounds.check(got, want, bound, dtype, "preference, backward")

    ids, teacher = tokens.unsqueeze(-1), torch.zeros(2, 4, 1, device=DEV)
    terms, want, rows = ref.distillation(x, ids, teacher, average="sum")
    bound = bounds.of_softmax(p, one, bounds.at_tokens(p, tokens.cpu(), one))
    r = tb.distillation_loss_grad(x, ids, teacher, average="sum")
    near(r.row_loss, rows, 2 * LP, "rows")
    bounds.check(r.grad, want, bound, dtype, "distillation")
    got, = torch.autograd.grad(tb.distillation_loss(leaf, ids, teacher, average="sum"), leaf)
    bounds.check(got, want, bound, dtype, "distillation, backward")


def two_peaks(V, dtype, gap):
    """All values below 0; two that share the probability, in parts of the row that different wavefronts hold:
    the one in a lane whose other values are far below, the other where a workgroup looks at every value."""
    per = 4 if dtype == torch.float32 else 8
    chunks = V // per
    threads = 256 if -(-chunks // 256) <= 8 else 512
    first, second = 3 * per + 1, per * ((min(-(-chunks // threads), 32) - 2) * threads + 100)
    x = torch.full((2, 1, V), -1.0 - gap)
    x[..., first] = x[..., second] = -1.0
    tokens = torch.tensor([[first], [second]])
    return x.to(dtype).to(DEV), tokens.to(DEV)


@pytest.mark.parametrize("gap", [20.0, 60.0, 86.5, 87.5, 88.0, 88.5, 89.0, 95.0, 120.0])
@pytest.mark.parametrize("dtype,V", [(torch.float32, 5000), (torch.bfloat16, 5000), (torch.bfloat16, 20011),
                                     (torch.float16, 50257), (torch.float32, 50257), (torch.bfloat16, 200000)])
def test_parts_of_a_row_that_lie_far_apart(dtype, V, gap):
    x, tokens = two_peaks(V, dtype, gap)
    valid = torch.ones(2, 1, dtype=torch.bool)
    rx, logp = ref.rows(x, valid, 1.0)
    p, one = logp.detach(), torch.ones(2, 1).double()
    lp, h = ref.chosen(logp, tokens, valid).detach(), ref.entropies(logp, valid).detach()
    got_lp, got_h = tb.token_logprobs(x, tokens, want_entropy=True)
    near(got_lp, lp, LP)
    near(got_h, h, bounds.H)
    near(tb.token_logprobs(x, tokens), lp, LP)
    old, a = lp.float().to(DEV) - 0.1, torch.ones(2, device=DEV)
    for kw in (dict(), dict(entropy_coef=0.1)):
        terms, want, _ = ref.policy(x, tokens, old, a, **kw)
        r = tb.policy_loss_grad(x, tokens, old, a, **kw)
        near(r.logprobs, lp, LP)
        bound = bounds.of_softmax(p, one, bounds.at_tokens(p, tokens.cpu(), one), 0.1 * one if kw else None)
        bounds.check(r.grad, want, bound, dtype, "policy")
    ids, teacher = tokens.unsqueeze(-1), torch.zeros(2, 1, 1, device=DEV)
    terms, want, rows = ref.distillation(x, ids, teacher)
    r = tb.distillation_loss_grad(x, ids, teacher)
    near(r.row_loss, rows, 2 * LP)
    bounds.check(r.grad, want, bounds.of_softmax(p, one, bounds.at_tokens(p, tokens.cpu(), one)), dtype, "distillation")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [64, 700, 5000, 20011, 140000])
def test_huge_cotangents_of_entropies(V, dtype):
    """Tokens that cannot be have no part in an entropy's gradient, however large its cotangent is."""
    g = torch.Generator().manual_seed(V)
    x, tokens = 2 * torch.randn(2, 3, V, generator=g), torch.randint(0, V, (2, 3), generator=g)
    dead = (torch.rand(2, 3, V, generator=g) < 0.3).scatter(-1, tokens.unsqueeze(-1), False)
    x = x.masked_fill(dead, -math.inf).to(dtype)
    valid, d_h = torch.ones(2, 3, dtype=torch.bool), torch.full((2, 3), 1e15)
    rx, logp = ref.rows(x, valid, 1.0)
    want, = torch.autograd.grad((ref.entropies(logp, valid) * d_h).sum(), rx)
    p = logp.detach().clamp(min=-1e4)
    bound = bounds.of_softmax(p, torch.zeros(2, 3).double(), torch.zeros_like(p), d_h.double())
    leaf = x.to(DEV).requires_grad_()
    lp, h = tb.token_logprobs(leaf, tokens.to(DEV), want_entropy=True)
    got, = torch.autograd.grad(h, leaf, d_h.to(DEV))
    assert not got[dead.to(DEV)].any()
    bounds.check(got, want, bound, dtype, "backward")
    r = tb.policy_loss_grad(x.to(DEV), tokens.to(DEV), lp.detach(), torch.zeros(2, device=DEV), entropy_coef=-1e15, average="sum")
    assert not r.grad[dead.to(DEV)].any()
    bounds.check(r.grad, want, bound, dtype, "policy")


@pytest.mark.parametrize("B,T", [(4, 3), (4, 700), (300, 2)])
@pytest.mark.parametrize("kw", [dict(), dict(beta=0.7), dict(kind="hinge"), dict(label_smoothing=0.1)])
def test_infinite_margins(B, T, kw):
    """A token of logit -inf has probability 0.  In a rejected sequence the margin is +inf: no loss (unless the
    smoothed part asks for the opposite), and no gradient; in a chosen one -inf, and the loss infinite."""
    V = 40
    g = torch.Generator().manual_seed(B + T)
    x, tokens = torch.randn(B, T, V, generator=g), torch.randint(0, V, (B, T), generator=g)
    reference = torch.full((B, T), -4.0)
    near_all = lambda r, want: near(r, want, 2 * LP * T)
    for at in (B - 1, 0):
        y = x.clone()
        y[at, 1, tokens[at, 1]] = -math.inf
        pair, pairs = at % (B // 2), B // 2
        others = [i for i in range(B) if i % pairs != pair]
        terms, grad, _, margins = ref.preference(x[others], tokens[others], reference[others], **kw)
        keep = 1.0 - 1.0 / pairs
        r = tb.preference_loss_grad(y.to(DEV), tokens.to(DEV), reference.to(DEV), **kw)
        rest = [i for i in range(pairs) if i != pair]
        near_all(r.margins[rest], margins)
        sign = 1.0 if at else -1.0
        assert float(r.margins[pair]) == sign * math.inf and float(r.terms[2]) == sign * math.inf
        if at and not kw.get("label_smoothing"):
            near_all(r.loss, float(terms[0]) * keep)
            near(r.terms[1], float(terms[1]) * keep + 1.0 / pairs, 1e-6)
            assert not r.grad[[pair, pair + pairs]].any()
            leaf = y.to(DEV).requires_grad_()
            loss = tb.preference_loss(leaf, tokens.to(DEV), reference.to(DEV), **kw)
            near_all(loss, float(terms[0]) * keep)
            assert torch.isfinite(torch.autograd.grad(loss, leaf)[0]).all()
        else:
            assert float(r.loss) == math.inf
        logp, d = torch.log_softmax(x[others].double(), -1), torch.full((len(others), T), 1.0 / pairs).double()
        bounds.check(r.grad[others], grad * keep, T * bounds.of_softmax(logp, d, bounds.at_tokens(logp, tokens[others], d)),
                     torch.float32, "the other pairs")


def test_lengths_beyond_32_bits():
    """Lengths of 64 bits are held to [0, T] as what they are, not as their lower half."""
    V, T = 64, 5
    g = torch.Generator().manual_seed(3)
    x, tokens = torch.randn(6, T, V, generator=g).to(DEV), torch.randint(0, V, (6, T), generator=g).to(DEV)
    wide = torch.tensor([(1 << 32) + 2, -(1 << 32), 3, 1 << 40, -(1 << 32) + 3, (1 << 63) - 1], device=DEV)
    held = torch.tensor([T, 0, 3, T, 0, T], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert torch.equal(tb.token_logprobs(x, tokens, lengths=wide, status=status), tb.token_logprobs(x, tokens, lengths=held))
    assert int(status) == tb.TB_DEV_LENGTH_RANGE
    status.zero_()
    tb.token_logprobs(x, tokens, lengths=held, status=status)
    assert int(status) == 0
    v, a = torch.full((6, T), -4.0, device=DEV), torch.ones(6, device=DEV)
    for f in (lambda n: tb.policy_loss_grad(x, tokens, v, a, lengths=n), lambda n: tb.preference_loss_grad(x, tokens, v, lengths=n),
              lambda n: tb.distillation_loss_grad(x, tokens.unsqueeze(-1), v.unsqueeze(-1), lengths=n)):
        for one, other in zip(f(wide), f(held)):
            assert torch.equal(one, other)
