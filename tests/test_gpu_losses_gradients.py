"""Gradients of the losses over logits, each value against what it is made of (tests/loss_bounds.py): a row of
tens of thousands of values has probabilities of 1e-7 far from its token, and these are held to 1e-4 of
themselves (and the rounding of their type), not to a share of the row's largest value.

Sizes lie on both sides of every change of kernel: rows of some lanes, of a workgroup of 256 or 512 threads with
each number of chunks, with LDS, and swept; distillation by 16 lanes, a wavefront and a workgroup."""
import pytest
import torch

import loss_bounds as bounds
import loss_reference as ref
import paper_2510_05485_amd as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# (in 16-bit values; half as many in 32 bits)
SIZES = [1, 7, 16, 33, 64, 127, 200, 301, 512, 1000, 1031, 2050, 4096, 4104, 6145, 9001, 12345, 16391, 20011, 32000, 50257,
         66000, 100003, 131072, 131090, 200003, 262144, 270003]
B, T = 2, 3


def inputs(V, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + V)
    x = 2.5 * torch.randn(B, T, V, generator=g)
    tokens = torch.randint(0, V, (B, T), generator=g)
    tokens[0, 0], tokens[1, 1] = 0, V - 1
    x.scatter_add_(-1, tokens.unsqueeze(-1), 8 * torch.rand(B, T, 1, generator=g))
    return x.to(dtype), tokens, g


def sizes():
    for dtype in TYPES:
        for V in SIZES:
            yield dtype, max(1, V // 2) if dtype == torch.float32 else V


def scale_of(dtype):
    return 4096.0 if dtype == torch.float16 else 1.0


def scored(x, temperature):
    valid = torch.ones(B, T, dtype=torch.bool)
    leaf, logp = ref.rows(x, valid, temperature)
    return leaf, logp, logp.detach(), valid


@pytest.mark.parametrize("dtype,V", sizes())
def test_of_log_probabilities_and_entropies(dtype, V):
    x, tokens, g = inputs(V, dtype)
    scale, temperature = scale_of(dtype), 0.8 if V % 2 else 1.0
    d, d_h = torch.randn(B, T, generator=g).double(), torch.randn(B, T, generator=g).double()
    leaf, logp, p, valid = scored(x, temperature)
    lp, h = ref.chosen(logp, tokens, valid), ref.entropies(logp, valid)
    y = x.to(DEV).requires_grad_()
    for both in (False, True):
        value = (lp * d).sum() + ((h * d_h).sum() if both else 0.0)
        want, = torch.autograd.grad(value, leaf, retain_graph=True)
        out = tb.token_logprobs(y, tokens.to(DEV), want_entropy=both, temperature=temperature)
        cot = [(v * scale).float().to(DEV) for v in ((d, d_h) if both else (d,))]
        got, = torch.autograd.grad(out, y, cot if both else cot[0])
        bound = bounds.of_softmax(p, d, bounds.at_tokens(p, tokens, d), d_h if both else None) / temperature
        bounds.check(got, want, bound, dtype, "with entropies" if both else "alone", scale)


@pytest.mark.parametrize("dtype,V", sizes())
def test_of_the_policy_loss(dtype, V):
    x, tokens, g = inputs(V, dtype, 1)
    scale = scale_of(dtype)
    leaf, logp, p, valid = scored(x, 1.0)
    lp = ref.chosen(logp, tokens, valid).detach()
    old, reference = (lp - 0.1).float(), (lp + 0.2).float()
    a = torch.randn(B, T, generator=g)
    for kw in (dict(), dict(kl_coef=0.3, entropy_coef=0.05)):
        terms, want, _ = ref.policy(x, tokens, old, a, reference, average="sum", **kw)
        r = tb.policy_loss_grad(x.to(DEV), tokens.to(DEV), old.to(DEV), a.to(DEV), ref_logprobs=reference.to(DEV),
                                grad_scale=scale, average="sum", **kw)
        # |ratio A| with ratio e^0.1, and of the KL term k (1 + e^0.2), whose error is a share of both parts
        d = 1.11 * a.abs().double() + kw.get("kl_coef", 0.0) * 2.3
        d_h = torch.full((B, T), kw["entropy_coef"]).double() if kw else None
        bound = bounds.of_softmax(p, d, bounds.at_tokens(p, tokens, d), d_h)
        bounds.check(r.grad, want, bound, dtype, "policy", scale)


@pytest.mark.parametrize("dtype,V", sizes())
def test_of_the_preference_loss(dtype, V):
    x, tokens, g = inputs(V, dtype, 2)
    scale = scale_of(dtype)
    leaf, logp, p, valid = scored(x, 1.0)
    lp = ref.chosen(logp, tokens, valid).detach()
    reference = (lp + 0.3 * torch.randn(B, T, generator=g)).float()
    terms, want, _, margins = ref.preference(x, tokens, reference, beta=0.5)
    r = tb.preference_loss_grad(x.to(DEV), tokens.to(DEV), reference.to(DEV), beta=0.5, grad_scale=scale)
    # the cotangent beta sigmoid(-beta h) is off by beta times the margin's error, 2 T LP, relatively to itself:
    # 3 LP, as much as a probability, for which the bound counts it twice
    d = torch.full((B, T), 0.5 * float(torch.sigmoid(-0.5 * margins[0])) * 2).double()
    bounds.check(r.grad, want, bounds.of_softmax(p, d, bounds.at_tokens(p, tokens, d)), dtype, "preference", scale)


def taught():
    """Sizes with the number of the teacher's entries: few for every size, many for some of each kernel."""
    for dtype, V in sizes():
        for K in (1, 8, 40, 65):
            if K <= V:
                yield dtype, V, K
    for dtype in TYPES:
        for V in (700, 4500, 9001, 50257):
            for K in (257, 600, 1024):
                yield dtype, V, min(K, V)


@pytest.mark.parametrize("dtype,V,K", taught())
def test_of_the_distillation_loss(dtype, V, K):
    x, _, g = inputs(V, dtype, 3)
    scale = scale_of(dtype)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(B * T)]).reshape(B, T, K)
    if K > 3:
        ids[0, 0, 1] = ids[0, 0, 3] = ids[0, 0, 0]
    teacher = (2 * torch.randn(B, T, K, generator=g)).to(dtype)
    leaf, logp, p, valid = scored(x, 1.0)
    terms, want, rows = ref.distillation(x, ids, teacher, average="sum")
    q = torch.zeros(B, T, V).double().scatter_add(-1, ids, torch.softmax(teacher.double(), -1))
    bound = bounds.of_softmax(p, torch.ones(B, T), q)
    r = tb.distillation_loss_grad(x.to(DEV), ids.to(DEV), teacher.to(DEV), average="sum", grad_scale=scale)
    bounds.check(r.grad, want, bound, dtype, "in one call", scale)
    y = x.to(DEV).requires_grad_()
    got, = torch.autograd.grad(tb.distillation_loss(y, ids.to(DEV), teacher.to(DEV), average="sum") * scale, y)
    bounds.check(got, want, bound, dtype, "backward", scale)
