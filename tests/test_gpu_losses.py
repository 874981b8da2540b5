"""Losses over logits against their definitions in float64 (tests/loss_reference.py).

Tolerances, u = 2^-24.  A log-probability is (z - m) - log s: with |z - m| <= 64 and s <= V 2^1 the
difference, the logarithm and the difference of both round by at most (64 + 13 + 77) u; the argument of
an exponential is off by 2 |a| u in the mean weight, |a| <= 12 where it matters, the instruction by 2 u,
and the sum of n terms of a thread and the tree above it by (n + 12) u, n <= 150: in all under
360 u = 2.2e-5.  LP = 3e-5 holds log-probabilities and losses per position; an entropy sums
p (z - m), |z - m| <= 64, with the same relative errors: H = 64 x as much at most, 2e-4 here because the
weights are those of a distribution (|a| <= 12 where they matter).  A gradient in float32 is its
cotangent times p, which is off by as much relatively; in another type it is rounded once more: to
2^-8 and 2^-11 of its size, or to half of float16's smallest step, 2^-25."""
import math

import pytest
import torch

import loss_reference as ref
import paper_2510_05485_amd as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LP, H = 3e-5, 2e-4
ROUND = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
STEP = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [1, 2, 3, 7, 8, 9, 15, 16, 17, 63, 64, 65, 100, 127, 129, 255, 257, 500, 512, 513, 1000, 1031, 2047, 4097,
         8200, 12289, 16385, 32000, 50257]


def inputs(seed, B, T, V, dtype=torch.float32, shift=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, T + shift, V, generator=g) * 2.5
    tokens = torch.randint(0, V, (B, T + shift), generator=g)
    x.scatter_add_(-1, tokens.unsqueeze(-1), 8 * torch.rand(B, T + shift, 1, generator=g))
    return x.to(dtype).to(DEV), tokens.to(DEV), g


def near(got, want, tol, what=""):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    tol = torch.as_tensor(tol, dtype=torch.float64).expand_as(off)
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(off[bad].max()), got[bad][:4], want[bad][:4])


def near_gradient(got, want, d, dtype, what=""):
    """d: what bounds the cotangents of a row's log-probability (and entropy), [..., 1] or a number."""
    near(got, want, LP * d + want.abs() * (ROUND[dtype] * 1.01 + LP) + STEP[dtype], what)


def spread(want):
    """The largest gradient of each row: its token's, or that of the likeliest of the others."""
    return want.abs().amax(-1, keepdim=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", SIZES)
def test_token_logprobs_and_gradient(V, dtype):
    x, tokens, g = inputs(V, 2, 3, V, dtype)
    lengths = torch.tensor([3, 2], device=DEV, dtype=torch.int32)
    d_lp, d_h = torch.randn(2, 3, generator=g), torch.randn(2, 3, generator=g)
    temperature = 0.8 if V % 2 else 1.0
    valid = ref.valid_positions((2, 3), lengths)
    rx, logp = ref.rows(x, valid, temperature)
    want_lp, want_h = ref.chosen(logp, tokens, valid), ref.entropies(logp, valid)
    kw = dict(lengths=lengths, temperature=temperature)
    near(tb.token_logprobs(x, tokens, **kw), want_lp.detach(), LP, "forward alone")
    leaf = x.clone().requires_grad_()
    lp, h = tb.token_logprobs(leaf, tokens.int(), want_entropy=True, **kw)
    near(lp, want_lp.detach(), LP, "log-probabilities")
    near(h, want_h.detach(), H, "entropies")
    want, = torch.autograd.grad((want_lp * d_lp).sum() + (want_h * d_h).sum(), rx, retain_graph=True)
    got, = torch.autograd.grad((lp, h), leaf, (d_lp.to(DEV), d_h.to(DEV)), retain_graph=True)
    size = (d_lp.abs() + 20 * d_h.abs()).unsqueeze(-1) / temperature
    near_gradient(got, want, size, dtype, "gradient of both")
    want, = torch.autograd.grad((want_lp * d_lp).sum(), rx)
    got, = torch.autograd.grad(lp, leaf, d_lp.to(DEV))
    near_gradient(got, want, d_lp.abs().unsqueeze(-1) / temperature, dtype, "gradient of the log-probabilities")
    assert not got[1, 2].any()


POLICIES = [dict(), dict(kl_coef=0.1), dict(entropy_coef=0.02, temperature=1.5),
            dict(kl_coef=0.04, entropy_coef=-0.01, average="sequence", clip_low=0.1, clip_high=0.3),
            dict(average="sum", kl_coef=0.1, temperature=0.7, clip_low=0.0, clip_high=0.0)]


def policy_inputs(seed, B, T, V, dtype, each, temperature=1.0):
    x, tokens, g = inputs(seed, B, T, V, dtype)
    valid = torch.ones(B, T, dtype=torch.bool)
    lp = ref.chosen(ref.rows(x, valid, temperature)[1], tokens, valid).detach()
    # ratios away from 1 (with clip ranges of 0) and from the other edges of the ranges
    d = torch.tensor([-0.5, -0.25, -0.15, -0.05, 0.05, 0.12, 0.24, 0.5])[torch.randint(0, 8, (B, T), generator=g)]
    old = (lp - d).float().to(DEV)
    reference = (lp + 0.3 * torch.randn(B, T, generator=g)).float().to(DEV)
    a = torch.randn(B, T, generator=g) if each else torch.randn(B, generator=g)
    return x, tokens, old, reference, a.to(DEV)


@pytest.mark.parametrize("kw", POLICIES)
@pytest.mark.parametrize("dtype,V,each", [(torch.float32, 64, True), (torch.float32, 1031, False),
                                          (torch.bfloat16, 64, False), (torch.bfloat16, 5003, True),
                                          (torch.float16, 257, True), (torch.bfloat16, 32000, False)])
def test_policy_loss(dtype, V, each, kw):
    B, T = 5, 6
    x, tokens, old, reference, a = policy_inputs(7 * V, B, T, V, dtype, each, kw.get("temperature", 1.0))
    lengths = torch.tensor([6, 0, 3, 1, 6], device=DEV)
    mask = torch.rand(B, T, generator=torch.Generator().manual_seed(V)) < 0.8
    terms, grad, lp = ref.policy(x, tokens, old, a, reference, lengths, mask, **kw)
    scale = 64.0
    args = dict(ref_logprobs=reference, lengths=lengths, mask=mask.to(DEV), **kw)
    r = tb.policy_loss_grad(x, tokens, old, a, grad_scale=scale, **args)
    near(r.logprobs, lp, LP, "log-probabilities")
    n = 30 if kw.get("average") == "sum" else 1
    size = 10 * (1 + float(a.abs().max())) * n                # of a position's loss by its log-probability
    near(r.terms, terms, LP * size, "terms")
    near_gradient(r.grad / scale if dtype == torch.float32 else r.grad.double() / scale, grad, size, dtype, "gradient")
    assert not r.grad[~ref.valid_positions((B, T), lengths, mask).to(DEV)].any()
    leaf = x.clone().requires_grad_()
    loss = tb.policy_loss(leaf, tokens, old, a, **args)
    near(loss, terms[0], LP * size, "loss")
    (3.0 * loss).backward()
    near_gradient(leaf.grad, 3 * grad, 3 * size, dtype, "backward")
    near(tb.policy_loss(x, tokens, old, a, **args), terms[0], LP * size, "loss without a gradient")


PAIRS = [dict(), dict(label_smoothing=0.2, beta=0.5), dict(kind="hinge", beta=0.3), dict(kind="ipo", beta=0.5),
         dict(temperature=1.4)]


@pytest.mark.parametrize("kw", PAIRS)
@pytest.mark.parametrize("dtype,B,T,V", [(torch.float32, 2, 1, 50), (torch.bfloat16, 6, 9, 513),
                                         (torch.float16, 4, 17, 1000), (torch.float32, 8, 5, 4097),
                                         (torch.bfloat16, 2, 3, 32000)])
def test_preference_loss(dtype, B, T, V, kw):
    x, tokens, g = inputs(3 * V + T, B, T, V, dtype)
    reference = ref.chosen(torch.log_softmax(x.cpu().double(), -1), tokens, torch.ones(B, T, dtype=torch.bool))
    reference = (reference + 0.4 * torch.randn(B, T, generator=g)).float().to(DEV)
    lengths = torch.randint(0, T + 1, (B,), generator=g).to(DEV)
    lengths[0] = T
    mask = (torch.rand(B, T, generator=g) < 0.9).to(DEV)
    terms, grad, sums, margins = ref.preference(x, tokens, reference, lengths, mask, **kw)
    assert (margins.abs() > 1e-3).all() or B > 4              # no sign hangs on the last bit
    r = tb.preference_loss_grad(x, tokens, reference, lengths=lengths, mask=mask, grad_scale=16.0, **kw)
    near(r.sequence_logprobs, sums, LP * T, "sequences")
    near(r.margins, margins, 2 * LP * T, "margins")
    size = 4.0 + 4 * float(margins.abs().max())               # of a pair's loss by its margin
    near(r.terms, terms, 2 * LP * T * size, "terms")
    near_gradient(r.grad.double() / 16, grad, T * size, dtype, "gradient")
    assert not r.grad[~ref.valid_positions((B, T), lengths, mask).to(DEV)].any()
    leaf = x.clone().requires_grad_()
    loss = tb.preference_loss(leaf, tokens, reference, lengths=lengths, mask=mask, **kw)
    near(loss, terms[0], 2 * LP * T * size, "loss")
    (2.0 * loss).backward()
    near_gradient(leaf.grad, 2 * grad, 2 * T * size, dtype, "backward")


@pytest.mark.parametrize("kw", [dict(), dict(temperature=2.0, average="sequence"), dict(average="sum", temperature=0.7)])
@pytest.mark.parametrize("dtype,V,K", [(torch.float32, 1, 1), (torch.float32, 9, 9), (torch.bfloat16, 64, 5),
                                       (torch.bfloat16, 1000, 64), (torch.float16, 1031, 65),
                                       (torch.float32, 4097, 257), (torch.bfloat16, 32000, 1024),
                                       (torch.float32, 50257, 8)])
def test_distillation_loss(dtype, V, K, kw):
    B, T = 3, 4
    x, _, g = inputs(11 * V + K, B, T, V, dtype)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] if V >= K else torch.randint(0, V, (K,), generator=g)
                       for _ in range(B * T)]).reshape(B, T, K)
    teacher = (3 * torch.randn(B, T, K, generator=g)).sort(-1, descending=True).values
    if K > 3:
        ids[0, 0, 1], ids[0, 0, 3] = ids[0, 0, 0], ids[0, 0, 0]   # entries with one id
        teacher[0, 1, K // 2:] = -math.inf                         # fewer entries: their ids are not read
        ids[0, 1, K // 2:] = -1
        teacher[0, 2], ids[0, 2] = -math.inf, 1 << 30              # none at all
    teacher = teacher.to(dtype)
    ids, teacher = ids.to(DEV), teacher.to(DEV)
    lengths = torch.tensor([4, 2, 3], device=DEV, dtype=torch.int32)
    terms, grad, rows = ref.distillation(x, ids, teacher, lengths, **kw)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tau = kw.get("temperature", 1.0)
    size = tau ** 2 * 30 * (12 if kw.get("average") == "sum" else 1)
    for wide in (ids, ids.int()):
        r = tb.distillation_loss_grad(x, wide, teacher, lengths=lengths, grad_scale=8.0, status=status, **kw)
        near(r.row_loss, rows, 2 * LP * tau ** 2, "rows")
        near(r.terms, terms, LP * size, "terms")
        near_gradient(r.grad.double() / 8, grad, size, dtype, "gradient")
    assert int(status) == 0
    leaf = x.clone().requires_grad_()
    loss = tb.distillation_loss(leaf, ids, teacher, lengths=lengths, **kw)
    near(loss, terms[0], LP * size, "loss")
    (2.0 * loss).backward()
    near_gradient(leaf.grad, 2 * grad, 2 * size, dtype, "backward")


@pytest.mark.parametrize("dtype,V", [(d, v // (2 if d == torch.float32 else 1)) for d in TYPES
                                     for v in (131064, 131072, 131082, 139264, 204802, 204820, 209001, 262144, 262152, 270003)])
def test_long_rows(dtype, V):
    """Rows that registers hold, that registers and LDS hold, and longer ones, at each boundary."""
    B, T = 2, 2
    base = torch.zeros(B, T, V + 9, dtype=dtype, device=DEV)
    x, tokens, g = inputs(V, B, T, V, dtype)
    tokens[0, 0], tokens[0, 1], tokens[1, 0] = 0, V - 1, V - 9
    old = torch.full((B, T), -10.0, device=DEV)
    a = torch.tensor([1.0, -0.5], device=DEV)
    ids = torch.stack([torch.randint(0, V, (B, T), generator=g), torch.zeros(B, T, dtype=torch.long),
                       torch.full((B, T), V - 1), torch.zeros(B, T, dtype=torch.long)], -1).to(DEV)
    teacher = torch.randn(B, T, 4, generator=g).to(DEV)
    kw = dict(kl_coef=0.1, entropy_coef=0.1)
    terms, grad, lp = ref.policy(x, tokens, old, a, old, None, None, **kw)
    d_terms, d_grad, rows = ref.distillation(x, ids, teacher)
    size = 4 * float(grad.abs().amax() + 1)
    for lo in (0, 3, 8):
        view = base[..., lo:lo + V]
        view.copy_(x)
        out = torch.full_like(base, 7.0)
        r = tb.policy_loss_grad(view, tokens, old, a, ref_logprobs=old, out=out[..., lo:lo + V], **kw)
        near(r.logprobs, lp, LP)
        near(r.terms, terms, LP * (20 + terms.abs().max()))
        near_gradient(r.grad, grad, size, dtype)
        assert (out[..., :lo] == 7).all() and (out[..., lo + V:] == 7).all()
        out.fill_(7.0)
        r = tb.distillation_loss_grad(view, ids, teacher, out=out[..., lo:lo + V])
        near(r.row_loss, rows, 2 * LP)
        near_gradient(r.grad, d_grad, 1.0, dtype)
        assert (out[..., :lo] == 7).all() and (out[..., lo + V:] == 7).all()
        near(tb.token_logprobs(view, tokens), lp, LP)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [64, 5000, 20011])
@pytest.mark.parametrize("shift", [-200.0, -30.0, 60.0, 2000.0])
def test_shifted_logits(dtype, V, shift):
    """Softmax does not change with a constant: rows below 0 throughout (log-probabilities as logits), far
    above, with tokens that cannot be among them."""
    B, T = 2, 3
    x, tokens, g = inputs(V, B, T, V)
    x = (x + shift).to(dtype)
    dead = (torch.rand(B, T, V, generator=g) < 0.3).to(DEV).scatter(-1, tokens.unsqueeze(-1), False)
    for low in (None, -math.inf, torch.finfo(dtype).min):
        y = x if low is None else torch.where(dead, torch.full_like(x, low), x)
        old, a = torch.full((B, T), -8.0, device=DEV), torch.ones(B, device=DEV)
        terms, grad, lp = ref.policy(y, tokens, old, a, None, None, None, entropy_coef=0.1)
        r = tb.policy_loss_grad(y, tokens, old, a, entropy_coef=0.1)
        # z - m is a difference of numbers of the shift's size, whose products with log2(e) are rounded
        tol = LP + 4 * abs(shift) * 2.0 ** -24
        near(r.logprobs, lp, tol)
        near(r.terms, terms, tol * (20 + terms.abs().max()))
        near(r.grad, grad, tol * 20 * (1 + float(grad.abs().max())) + grad.abs() * (ROUND[dtype] * 1.01) + STEP[dtype])
        d_terms, d_grad, rows = ref.distillation(y, tokens.unsqueeze(-1), torch.zeros(B, T, 1))
        r = tb.distillation_loss_grad(y, tokens.unsqueeze(-1), torch.zeros(B, T, 1, device=DEV))
        near(r.row_loss, rows, tol)
        near(r.grad, d_grad, tol * 20 + d_grad.abs() * (ROUND[dtype] * 1.01) + STEP[dtype])
        leaf = y.clone().requires_grad_()
        got, = torch.autograd.grad(tb.token_logprobs(leaf, tokens).sum(), leaf)
        p = torch.log_softmax(y.cpu().double(), -1).exp()
        want = torch.nn.functional.one_hot(tokens.cpu(), V) - p
        near(got, want, tol * 20 + want.abs() * (ROUND[dtype] * 1.01) + STEP[dtype])


def all_operators(x, tokens, where, seed=5, out=False):
    """Every operator on the same logits [B, T, V] (B even); a list of (name, tensor)."""
    g = torch.Generator().manual_seed(seed)
    shape = tokens.shape
    v = [torch.randn(shape, generator=g).to(DEV) for _ in range(3)]
    K = min(5, x.shape[-1])
    ids = torch.randint(0, x.shape[-1], (*shape, K), generator=g).to(DEV)
    teacher = torch.randn(*shape, K, generator=g).to(DEV)
    kw = lambda: dict(where, out=x.clone(memory_format=torch.preserve_format)) if out else where
    found = [("lp", tb.token_logprobs(x, tokens, **where))]
    r = tb.policy_loss_grad(x, tokens, v[0] - 4, v[1], ref_logprobs=v[2] - 4, kl_coef=0.1, entropy_coef=0.1, **kw())
    found += [("policy " + k, getattr(r, k)) for k in r._fields]
    r = tb.preference_loss_grad(x, tokens, v[2] - 4, **kw())
    found += [("preference " + k, getattr(r, k)) for k in r._fields]
    r = tb.distillation_loss_grad(x, ids, teacher, **kw())
    found += [("distillation " + k, getattr(r, k)) for k in r._fields]
    leaf = x.detach().clone(memory_format=torch.preserve_format).requires_grad_()
    lp, h = tb.token_logprobs(leaf, tokens, want_entropy=True, **where)
    found += [("entropy", h), ("backward", torch.autograd.grad((lp, h), leaf, (v[0], v[1]))[0])]
    return found


def same(one, other):
    for (name, a), (_, b) in zip(one, other):
        assert torch.equal(a, b), name


def alike(one, other):
    """Results of rows that begin at other addresses: sums over a row are then taken in another order."""
    for (name, a), (_, b) in zip(one, other):
        tol = 2 * LP * (20 + b.double().abs().max()) if a.dtype == torch.float32 and a.dim() < 3 else \
            2 * (LP * (1 + spread(b.double())) + ROUND[a.dtype] * b.double().abs() + STEP[a.dtype])
        near(a, b.cpu().double(), tol.cpu(), name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [5, 64, 250, 1031, 9001])
def test_what_stands_at_other_positions_is_not_read(V, dtype):
    x, tokens, _ = inputs(V, 4, 5, V, dtype)
    lengths = torch.tensor([5, 0, 2, 4], device=DEV, dtype=torch.int32)
    mask = torch.ones(4, 5, dtype=torch.bool, device=DEV)
    mask[0, 1] = mask[3, 0] = False
    where = dict(lengths=lengths, mask=mask)
    want = all_operators(x, tokens, where)
    dead = ~ref.valid_positions((4, 5), lengths, mask).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for filler in (math.nan, math.inf, -math.inf, torch.finfo(dtype).min):
        y, ids = x.clone(), tokens.clone()
        y[dead], ids[dead] = filler, 1 << 40
        same(all_operators(y, ids, dict(where, status=status)), want)
    assert int(status) == 0
    for name, t in want:
        assert torch.isfinite(t).all(), name
        if t.shape[:2] == dead.shape:
            assert not t[dead].any(), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [3, 64, 700, 5000])
def test_tokens_that_cannot_be(V, dtype):
    """Logits of -inf (or the lowest value) take no part; rows without a finite logit are NaN."""
    x, tokens, g = inputs(V + 1, 2, 4, V, dtype)
    keep = torch.rand(2, 4, V, generator=g).to(DEV) < 0.5
    keep.scatter_(-1, tokens.unsqueeze(-1), True)
    for low in (-math.inf, torch.finfo(dtype).min):
        y = torch.where(keep, x, torch.full_like(x, low))
        valid = torch.ones(2, 4, dtype=torch.bool)
        rx, logp = ref.rows(y, valid, 1.0)
        lp, h = ref.chosen(logp, tokens, valid), ref.entropies(logp, valid)
        leaf = y.clone().requires_grad_()
        got_lp, got_h = tb.token_logprobs(leaf, tokens, want_entropy=True)
        near(got_lp, lp.detach(), LP)
        near(got_h, h.detach(), H)
        grad, = torch.autograd.grad((got_lp.sum() + got_h.sum()), leaf)
        assert torch.isfinite(grad).all() and not grad[~keep].any()
    lowest = torch.full_like(x, torch.finfo(dtype).min)       # all alike: uniform
    got_lp, got_h = tb.token_logprobs(lowest, tokens, want_entropy=True)
    near(got_lp, torch.full((2, 4), -math.log(V), dtype=torch.float64), LP)
    near(got_h, torch.full((2, 4), math.log(V), dtype=torch.float64), H)
    r = tb.distillation_loss_grad(lowest, tokens.unsqueeze(-1), torch.zeros(2, 4, 1, device=DEV))
    near(r.row_loss, torch.full((2, 4), math.log(V), dtype=torch.float64), LP)
    near(r.grad.sum(-1), torch.zeros(2, 4, dtype=torch.float64), 1e-2)
    for filler in (-math.inf, math.inf, math.nan):
        y = x.clone()
        if filler == -math.inf:
            y[0, 1] = filler
        else:
            y[0, 1, V // 2] = filler
        lp, h = tb.token_logprobs(y, tokens, want_entropy=True)
        assert torch.isnan(lp[0, 1]) and torch.isnan(h[0, 1])
        assert torch.isfinite(lp).sum() == 7 and torch.isfinite(h).sum() == 7
        r = tb.policy_loss_grad(y, tokens, lp.nan_to_num(), torch.ones(2, device=DEV))
        assert torch.isnan(r.loss) and torch.isnan(r.grad[0, 1]).all()
        assert torch.isfinite(r.grad[1]).all() and torch.isfinite(r.grad[0, 0]).all()


@pytest.mark.parametrize("V", [64, 1031, 20000])
def test_strides(V):
    B, T = 4, 5
    for dtype in TYPES:
        x, tokens, g = inputs(V, B, T, V, dtype)
        where = dict(lengths=torch.tensor([5, 3, 0, 4], device=DEV))
        want = all_operators(x, tokens, where)
        wide = torch.full((B, T + 1, V + 3), math.nan, dtype=dtype, device=DEV)
        for lo in range(4):                                   # rows that begin at every address of their type
            view = wide[:, 1:, lo:lo + V]
            view.copy_(x)
            if lo == 0:
                padded = torch.full((B, T + 3), 1 << 40, dtype=torch.int64, device=DEV)
                padded[:, 2:T + 2] = tokens
                alike(all_operators(view, padded[:, 2:T + 2], where), want)
            else:
                alike(all_operators(view, tokens, where), want)
            wide.fill_(math.nan)
        turned = x.transpose(0, 1).contiguous().transpose(0, 1)
        alike(all_operators(turned, tokens.t().contiguous().t(), where), want)
        alike(all_operators(turned, tokens, where, out=True), want)      # gradients with these strides
        every_other = torch.stack([x, torch.full_like(x, math.nan)], -1).flatten(-2)[..., ::2]
        alike(all_operators(every_other, tokens, where), want)
        one = x[:1, :1].expand(B, T, V)                       # a row that all positions share
        alike(all_operators(one, tokens, where), all_operators(one.contiguous(), tokens, where))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 9, 64, 300, 1031, 9000, 50257])
def test_gradient_over_the_logits(V, dtype):
    x, tokens, g = inputs(V, 4, 3, V, dtype)
    where = dict(lengths=torch.tensor([3, 0, 2, 3], device=DEV))
    old, a = torch.zeros(4, 3, device=DEV) - 3, torch.ones(4, 3, device=DEV)
    ids = torch.randint(0, V, (4, 3, 4), generator=g).to(DEV)
    teacher = torch.randn(4, 3, 4, generator=g).to(DEV)
    for f in (lambda y, **k: tb.policy_loss_grad(y, tokens, old, a, entropy_coef=0.1, **where, **k),
              lambda y, **k: tb.preference_loss_grad(y, tokens, old, **where, **k),
              lambda y, **k: tb.distillation_loss_grad(y, ids, teacher, **where, **k)):
        want, y = f(x), x.clone()
        r = f(y, out=y)
        assert r.grad.data_ptr() == y.data_ptr()
        for p, q in zip(r, want):
            assert torch.equal(p, q)


def test_packed_positions_are_one_sequence():
    x, tokens, g = inputs(1, 1, 37, 301)
    mask = (torch.rand(1, 37, generator=g) < 0.7).to(DEV)
    old, a = torch.randn(1, 37, generator=g).to(DEV) - 4, torch.randn(1, 37, generator=g).to(DEV)
    ids, teacher = torch.randint(0, 301, (1, 37, 6), generator=g).to(DEV), torch.randn(1, 37, 6, generator=g).to(DEV)
    assert torch.equal(tb.token_logprobs(x[0], tokens[0], mask=mask[0]), tb.token_logprobs(x, tokens, mask=mask)[0])
    p, q = (tb.policy_loss_grad(*v[:4], mask=v[4]) for v in ((x, tokens, old, a, mask), (x[0], tokens[0], old[0], a[0], mask[0])))
    assert torch.equal(p.terms, q.terms) and torch.equal(p.grad[0], q.grad) and torch.equal(p.logprobs[0], q.logprobs)
    p, q = (tb.distillation_loss_grad(*v[:3], mask=v[3]) for v in ((x, ids, teacher, mask), (x[0], ids[0], teacher[0], mask[0])))
    assert torch.equal(p.terms, q.terms) and torch.equal(p.grad[0], q.grad) and torch.equal(p.row_loss[0], q.row_loss)


@pytest.mark.parametrize("shape", [(0, 4, 9), (4, 0, 9), (2, 3, 9)])
def test_nothing_that_counts(shape):
    x = torch.full(shape, math.nan, device=DEV)
    tokens = torch.zeros(shape[:2], dtype=torch.int64, device=DEV)
    v = torch.zeros(shape[:2], device=DEV)
    lengths = torch.zeros(shape[0], dtype=torch.int32, device=DEV)
    assert not tb.token_logprobs(x, tokens, lengths=lengths).any()
    for average in ("token", "sequence", "sum"):
        r = tb.policy_loss_grad(x, tokens, v, v, lengths=lengths, average=average)
        assert r.terms.tolist() == [0.0] * 4 and not r.grad.any()
        r = tb.distillation_loss_grad(x, tokens.unsqueeze(-1), v.unsqueeze(-1), lengths=lengths, average=average)
        assert r.terms.tolist() == [0.0] and not r.grad.any()
    r = tb.preference_loss_grad(x, tokens, v, lengths=lengths)
    want = math.log(2.0) if shape[0] else 0.0                # margins of 0
    assert abs(float(r.loss) - want) < 1e-6 and not r.grad.any() and not r.margins.any()
    leaf = x.clone().requires_grad_()
    tb.policy_loss(leaf, tokens, v, v, lengths=lengths).backward()
    assert leaf.grad.shape == x.shape and not leaf.grad.any()


@pytest.mark.parametrize("V", [64, 1031])
def test_wrong_ids_and_lengths_are_reported(V):
    x, tokens, g = inputs(3, 4, 3, V)
    v = torch.zeros(4, 3, device=DEV)
    for bad in (-1, V, 1 << 40):
        ids = tokens.clone()
        ids[1, 2] = bad
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        lp = tb.token_logprobs(x, ids, status=status)
        assert int(status) == tb.TB_DEV_TOKEN_RANGE and torch.isnan(lp[1, 2]) and torch.isfinite(lp).sum() == 11
        r = tb.policy_loss_grad(x, ids, v, v)
        assert torch.isnan(r.loss) and torch.isnan(r.grad[1, 2]).all() and torch.isfinite(r.grad).sum() == 11 * V
        r = tb.preference_loss_grad(x, ids, v)
        assert torch.isnan(r.loss) and torch.isnan(r.grad[1, 2]).all()
        entries = torch.stack([tokens, ids], -1)
        status.zero_()
        r = tb.distillation_loss_grad(x, entries, torch.zeros(4, 3, 2, device=DEV), status=status)
        assert int(status) == tb.TB_DEV_TOKEN_RANGE
        assert torch.isnan(r.loss) and torch.isnan(r.row_loss[1, 2]) and torch.isnan(r.grad[1, 2]).all()
        assert torch.isfinite(r.grad).sum() == 11 * V
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = tb.token_logprobs(x, tokens, lengths=torch.tensor([4, -2, 3, 1], device=DEV), status=status)
    assert int(status) == tb.TB_DEV_LENGTH_RANGE
    assert torch.equal(got, tb.token_logprobs(x, tokens, lengths=torch.tensor([3, 0, 3, 1], device=DEV)))


def test_differences():
    """The gradient along a direction against the loss's difference.  The losses are sums of about 50
    positions' values below 30, formed in float32 from log-probabilities that are off by less than
    LP/10 here (|z - m| < 20, V = 300): 2e-6 x 50 / (2 h) = 2.5e-3 with h = 0.02; the difference's own
    error is h^2/6 of a third derivative below 100 along a direction of length 1: 7e-3."""
    B, T, V, h = 4, 13, 300, 0.02
    x, tokens, old, reference, a = policy_inputs(5, B, T, V, torch.float32, True)
    g = torch.Generator().manual_seed(9)
    ids, teacher = torch.randint(0, V, (B, T, 7), generator=g).to(DEV), torch.randn(B, T, 7, generator=g).to(DEV)
    where = dict(lengths=torch.tensor([13, 0, 7, 13], device=DEV))
    losses = [lambda y: tb.policy_loss_grad(y, tokens, old, a, ref_logprobs=reference, kl_coef=0.2, entropy_coef=0.1,
                                            clip_low=0.9, clip_high=9.0, average="sum", **where),
              lambda y: tb.preference_loss_grad(y, tokens, reference, beta=0.5, **where),
              lambda y: tb.preference_loss_grad(y, tokens, reference, beta=0.5, kind="ipo", **where),
              lambda y: tb.distillation_loss_grad(y, ids, teacher, temperature=1.3, average="sum", **where)]
    for f in losses:
        r = f(x)
        for k in range(4):
            u = torch.randn(B, T, V, generator=g).to(DEV) if k else r.grad.clone()
            u = u / u.norm()
            want = (float(f(x + h * u).loss) - float(f(x - h * u).loss)) / (2 * h)
            assert abs(float((r.grad.double() * u).sum()) - want) < 1e-2


@pytest.mark.parametrize("B,T,V", [(5000, 61, 33), (2500, 121, 200), (43000, 100, 3)])
def test_more_rows_than_workgroups(B, T, V):
    """Workgroups that take row after row: what a row gives does not depend on the rows around it."""
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(B, T, V, generator=g, device=DEV).to(torch.bfloat16)
    tokens = torch.randint(0, V, (B, T), generator=g, device=DEV)
    lengths = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    old, a = -3 + torch.randn(B, T, generator=g, device=DEV), torch.randn(B, generator=g, device=DEV)
    ids, teacher = torch.randint(0, V, (B, T, 3), generator=g, device=DEV), torch.randn(B, T, 3, generator=g, device=DEV)

    def found(s):
        n = lengths[s]
        r = tb.policy_loss_grad(x[s], tokens[s], old[s], a[s], lengths=n, average="sum", entropy_coef=0.1)
        q = tb.distillation_loss_grad(x[s], ids[s], teacher[s], lengths=n, average="sum")
        leaf = x[s].clone().requires_grad_()
        lp = tb.token_logprobs(leaf, tokens[s], lengths=n)
        return [r.grad, r.logprobs, q.grad, q.row_loss, lp.detach(), torch.autograd.grad(lp, leaf, old[s])[0]], r.loss, q.loss
    whole, loss, d_loss = found(slice(0, B))
    parts = [found(slice(i, min(i + 704, B))) for i in range(0, B, 704)]   # (whole lines: rows keep their places in them)
    for k, w in enumerate(whole):
        assert torch.equal(w, torch.cat([p[0][k] for p in parts]))
    for one, other in ((loss, [p[1] for p in parts]), (d_loss, [p[2] for p in parts])):
        assert abs(float(one) - sum(map(float, other))) <= 1e-6 * (sum(abs(float(v)) for v in other) + 1)
    rows = slice(B // 3, B // 3 + 3)
    want = ref.policy(x[rows], tokens[rows], old[rows], a[rows], None, lengths[rows], None, average="sum", entropy_coef=0.1)
    near(whole[1][rows], want[2], LP)


def test_more_pairs_than_a_launch_has_threads():
    """2^24 pairs of single positions: a workgroup of 256 each would be 2^32 threads."""
    B, V = 1 << 25, 8
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(B, 1, V, generator=g, device=DEV).to(torch.bfloat16)
    tokens = torch.randint(0, V, (B, 1), generator=g, device=DEV, dtype=torch.int32)
    reference = -2 + torch.randn(B, 1, generator=g, device=DEV)
    r = tb.preference_loss_grad(x, tokens, reference, grad_scale=float(B))
    for rows in (slice(0, 50), slice(B // 4 - 7, B // 4 + 50), slice(B // 2 - 50, B // 2)):
        pair = torch.arange(B, device=DEV)[rows]
        both = torch.cat([pair, pair + B // 2])
        _, grad, sums, margins = ref.preference(x[both], tokens[both], reference[both])
        near(r.margins[pair], margins, 2 * LP)
        near(r.sequence_logprobs[both], sums, LP)
        near_gradient(r.grad[both].double() / 2, grad * len(pair), 1.0, torch.bfloat16)
    assert abs(float(r.loss) - float(torch.nn.functional.softplus(-0.1 * r.margins.double()).mean())) < 1e-6


def test_offsets_beyond_32_bits():
    V, far = 1031, (1 << 31) + 12345
    base = torch.empty(far + 3 * V, dtype=torch.bfloat16, device=DEV)
    x, tokens, g = inputs(3, 2, 2, V, torch.bfloat16)
    view = base.as_strided((2, 2, V), (far, V + 1, 1))
    view.copy_(x)
    alike(all_operators(view, tokens, {}), all_operators(x, tokens, {}))
    base_g = torch.empty_like(base)
    out = base_g.as_strided((2, 2, V), (far, V + 1, 1))
    old, a = torch.zeros(2, 2, device=DEV) - 3, torch.ones(2, device=DEV)
    r = tb.policy_loss_grad(view, tokens, old, a, out=out)
    assert r.grad is out
    alike([("gradient", out)], [("gradient", tb.policy_loss_grad(x, tokens, old, a).grad)])


@pytest.mark.parametrize("V", [64, 1031, 50257])
def test_runs_agree_and_other_streams(V):
    x, tokens, _ = inputs(V, 4, 33, V, torch.bfloat16)
    where = dict(lengths=torch.tensor([33, 20, 0, 32], device=DEV))
    want = all_operators(x, tokens, where)
    for _ in range(3):
        same(all_operators(x, tokens, where), want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        y = x.clone()
        got = all_operators(y, tokens, where)
    stream.synchronize()
    same(got, want)


@pytest.mark.parametrize("V", [64, 1031, 32000])
def test_in_a_graph(V):
    B, T = 4, 9
    x, tokens, old, reference, a = policy_inputs(2, B, T, V, torch.bfloat16, True)
    ids, teacher = tokens.unsqueeze(-1).expand(B, T, 3).contiguous(), torch.zeros(B, T, 3, device=DEV)
    lengths = torch.tensor([9, 4, 0, 9], device=DEV, dtype=torch.int32)

    def step():
        return [*tb.policy_loss_grad(x, tokens, old, a, ref_logprobs=reference, kl_coef=0.1, lengths=lengths),
                *tb.preference_loss_grad(x, tokens, reference, lengths=lengths),
                *tb.distillation_loss_grad(x, ids, teacher, lengths=lengths)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for k in range(4):
        fresh = inputs(100 + k, B, T, V, torch.bfloat16)[0]
        x.copy_(fresh)
        lengths.copy_(torch.tensor([9, k, 3, 9 - k], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, step()):
            assert torch.equal(got, want)


@pytest.mark.parametrize("V", [64, 5000])
def test_both_ways_of_marshalling(V):
    """Calls that the native code takes and calls that it leaves to the general way (lengths of 64 bits,
    values that are not contiguous) give the same."""
    B, T = 4, 6
    x, tokens, old, reference, a = policy_inputs(V, B, T, V, torch.bfloat16, True)
    ids, teacher = torch.randint(0, V, (B, T, 5)).to(DEV), torch.randn(B, T, 5).to(DEV)
    lengths = torch.tensor([6, 0, 4, 5], device=DEV, dtype=torch.int32)
    apart = lambda v: torch.stack([v, v], -1)[..., 0]

    def found(n, f):
        leaf = x.clone().requires_grad_()
        out = [*tb.token_logprobs(leaf, tokens, lengths=n, want_entropy=True)]
        out += torch.autograd.grad(out, leaf, (f(a), f(old)), retain_graph=True)
        out += torch.autograd.grad(out[1], leaf, f(old))
        for step, loss in ((tb.policy_loss_grad, tb.policy_loss), (tb.preference_loss_grad, tb.preference_loss),
                           (tb.distillation_loss_grad, tb.distillation_loss)):
            args = dict(policy_loss_grad=(tokens, f(old), f(a)), preference_loss_grad=(tokens, f(reference)),
                        distillation_loss_grad=(ids, f(teacher)))[step.__name__]
            kw = dict(ref_logprobs=f(reference), kl_coef=0.1, entropy_coef=0.1) if step is tb.policy_loss_grad else {}
            out += [*step(x, *args, lengths=n, **kw)]
            value = loss(leaf, *args, lengths=n, **kw)
            out += [value, *torch.autograd.grad(2 * value, leaf)]
            assert torch.equal(loss(x, *args, lengths=n, **kw), value) and value.dim() == 0
        return [t.detach() for t in out]
    for one, other in zip(found(lengths, lambda v: v), found(lengths.long(), apart)):
        assert torch.equal(one, other)


def test_backward_of_what_has_changed_raises():
    x, tokens, _ = inputs(1, 2, 3, 50)
    leaf = x.requires_grad_()
    y = leaf * 1.0
    loss = tb.policy_loss(y, tokens, torch.zeros(2, 3, device=DEV), torch.ones(2, device=DEV))
    y.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    loss = tb.token_logprobs(leaf, tokens).sum()
    loss.backward(retain_graph=True)
    first = leaf.grad.clone()
    loss.backward()
    assert torch.equal(leaf.grad, 2 * first)
    with pytest.raises(RuntimeError):
        loss.backward()
    with pytest.raises(RuntimeError):
        torch.autograd.grad(tb.token_logprobs(leaf, tokens).sum(), leaf, create_graph=True)


@pytest.mark.parametrize("B,T,average", [(1, 3000, "sequence"), (3, 1500, "token"), (3, 1500, "sequence"),
                                         (40, 7, "sequence"), (9000, 2, "token"), (9000, 2, "sequence"), (300, 4, "sum")])
@pytest.mark.parametrize("masked", [False, True])
def test_averages_over_many_positions(B, T, average, masked):
    V = 17
    x, tokens, g = inputs(B + T, B, T, V)
    lengths = torch.randint(0, T + 1, (B,), generator=g).to(DEV)
    mask = (torch.rand(B, T, generator=g) < 0.6).to(DEV) if masked else None
    old, a = torch.full((B, T), -3.0, device=DEV), torch.ones(B, device=DEV)
    terms, grad, _ = ref.policy(x, tokens, old, a, None, lengths, mask, average=average)
    r = tb.policy_loss_grad(x, tokens, old, a, lengths=lengths, mask=mask, average=average)
    n = B * T if average == "sum" else 1
    near(r.terms, terms, LP * (20 * n + terms.abs().max()))
    near_gradient(r.grad, grad, spread(grad) + grad.abs().max(), torch.float32)
    reference = torch.full((B, T), -4.0, device=DEV)
    half = B // 2 * 2
    if half:
        cut = dict(lengths=lengths[:half], mask=None if mask is None else mask[:half])
        terms, grad, sums, margins = ref.preference(x[:half], tokens[:half], reference[:half], beta=0.01, **cut)
        r = tb.preference_loss_grad(x[:half], tokens[:half], reference[:half], beta=0.01, **cut)
        near(r.sequence_logprobs, sums, LP * T)
        near(r.margins, margins, 2 * LP * T)
        near(r.terms[:1], terms[:1], 2 * LP * T)
        near(r.terms[2:], terms[2:], 2 * LP * T)
        near_gradient(r.grad, grad, spread(grad) + grad.abs().max(), torch.float32)


def test_refusals():
    x, tokens, _ = inputs(1, 4, 3, 50)
    v, one = torch.zeros(4, 3, device=DEV), torch.zeros(4, device=DEV)
    ids, q = tokens.unsqueeze(-1), torch.zeros(4, 3, 1, device=DEV)

    def refused(f, *args, **kw):
        with pytest.raises(tb.TensorBLEUError):
            f(*args, **kw)
    lp = tb.token_logprobs
    refused(lp, x.cpu(), tokens)
    refused(lp, x.double(), tokens)
    refused(lp, x[0, 0], tokens[0, 0])
    refused(lp, x, tokens[:, :2])
    refused(lp, x, tokens.float())
    refused(lp, x, tokens.cpu())
    refused(lp, x, tokens, lengths=torch.zeros(3, dtype=torch.int32, device=DEV))
    refused(lp, x, tokens, lengths=one)
    refused(lp, x[0], tokens[0], lengths=torch.zeros(1, dtype=torch.int32, device=DEV))
    refused(lp, x, tokens, mask=v)
    refused(lp, x, tokens, mask=torch.ones(4, 2, dtype=torch.bool, device=DEV))
    refused(lp, x, tokens, status=one)
    for t in (0.0, -1.0, math.inf, math.nan):
        refused(lp, x, tokens, temperature=t)
    for f in (tb.policy_loss, tb.policy_loss_grad):
        refused(f, x, tokens, v.double(), v)
        refused(f, x, tokens, v, v[:, :2])
        refused(f, x, tokens, v, one[:3])
        refused(f, x, tokens, v, one, kl_coef=0.1)
        refused(f, x, tokens, v, one, kl_coef=-0.1, ref_logprobs=v)
        refused(f, x, tokens, v, one, clip_low=-0.1)
        refused(f, x, tokens, v, one, average="mean")
    for f in (tb.preference_loss, tb.preference_loss_grad):
        refused(f, x[:3], tokens[:3], v[:3])
        refused(f, x[0], tokens[0], v[0])
        refused(f, x, tokens, one)
        refused(f, x, tokens, v, beta=0.0)
        refused(f, x, tokens, v, kind="other")
        refused(f, x, tokens, v, label_smoothing=0.6)
        refused(f, x, tokens, v, kind="ipo", label_smoothing=0.1)
    for f in (tb.distillation_loss, tb.distillation_loss_grad):
        refused(f, x, ids.float(), q)
        refused(f, x, ids, q.double())
        refused(f, x, ids, q[:, :2])
        refused(f, x, ids.expand(4, 3, 1025), q.expand(4, 3, 1025))
        refused(f, x, ids[..., :0], q[..., :0])
    r = tb.policy_loss_grad
    refused(r, x, tokens, v, one, out=torch.empty(4, 3, 51, device=DEV))
    refused(r, x, tokens, v, one, out=torch.empty(4, 3, 50, device=DEV, dtype=torch.bfloat16))
    refused(r, x, tokens, v, one, out=torch.empty(4, 50, 3, device=DEV).transpose(1, 2))
    refused(r, x, tokens, v, one, out=torch.empty(1, 3, 50, device=DEV).expand(4, 3, 50))   # rows overlap
    room = torch.zeros(4 * 3 * 50 + 8, device=DEV)
    shifted = room[8:].view(4, 3, 50)
    refused(r, room[:600].view(4, 3, 50), tokens, v, one, out=shifted)                       # half over the logits
