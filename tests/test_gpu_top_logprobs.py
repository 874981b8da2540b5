"""Top log-probabilities against their definition in float64 (tests/top_reference.py).

Ids have to be equal.  Log-probabilities and entropies are held to LP and H, which tests/test_gpu_losses.py
derives for the same sums; gradients value by value to what tests/loss_bounds.py derives, a row's cotangents of
K + 1 log-probabilities being as many terms of its softmax part: their sum, rounded K + 1 times at 2^-24 of its
size, is within LP of the sum of their magnitudes for K up to 500, and of 2 LP for 1024."""
import gc
import math

import pytest
import torch

import loss_bounds as bounds
import loss_reference as ref
import paper_2510_05485_amd as tb
import top_reference as plain
from test_gpu_losses import DEV, H, LP, TYPES, inputs, near

pytestmark = pytest.mark.gpu
# of every kernel and about its limits, in 16-bit and (half as long) in 32-bit types
SIZES = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 1031,
         2047, 2049, 4096, 4097, 4111, 8200, 12289, 16385, 16393, 32000, 40961, 50257, 65537, 98304, 100003, 131072, 131073]


def check_values(r, x, k, tokens, valid, temperature=1.0, entropy=True, what="", tol=LP):
    _, logp, ids, lps = plain.top(x, k, valid, temperature)
    assert torch.equal(r.ids.cpu().long(), ids), (what, (r.ids.cpu() != ids).nonzero()[:4].tolist())
    there = ids >= 0
    got = r.logprobs.cpu().double()
    assert (got[~there] == -math.inf).all(), what
    near(torch.where(there, got, 0.0), torch.where(there, lps.detach(), torch.zeros_like(lps)), tol, what)
    if tokens is None:
        assert r.token_logprobs is None
    else:
        near(r.token_logprobs, ref.chosen(logp, tokens, valid).detach(), tol, what)
    if entropy:
        near(r.entropy, ref.entropies(logp, valid).detach(), H, what)
    else:
        assert r.entropy is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", SIZES)
def test_values(V, dtype):
    x, tokens, g = inputs(V, 2, 3, V, dtype)
    lengths = torch.tensor([3, 2], device=DEV, dtype=torch.int32)
    valid = ref.valid_positions((2, 3), lengths)
    temperature = 0.8 if V % 2 else 1.0
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kw = dict(lengths=lengths, temperature=temperature, status=status)
    for k in sorted({1, min(V, 5), min(V, 20), min(V, 64), min(V, 257)}):
        r = tb.top_logprobs(x, k, tokens, want_entropy=True, **kw)
        check_values(r, x, k, tokens, valid, temperature, what=k)
        assert r.ids.dtype == torch.int64
        other = tb.top_logprobs(x, k, id_dtype=torch.int32, want_entropy=True, **kw)
        assert other.ids.dtype == torch.int32 and torch.equal(other.ids.long(), r.ids)
        assert torch.equal(other.logprobs, r.logprobs) and other.token_logprobs is None
        check_values(tb.top_logprobs(x, k, **kw), x, k, None, valid, temperature, entropy=False, what=k)
    assert int(status) == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(300, 300), (512, 512), (1024, 1024), (1500, 1000), (4000, 1024), (5000, 600), (33333, 1024),
                                 (50257, 512), (262144, 1024), (300000, 256)])
def test_many_alternatives(V, K, dtype):
    x, tokens, _ = inputs(V + K, 1, 2, V, dtype)
    valid = torch.ones(1, 2, dtype=torch.bool)
    check_values(tb.top_logprobs(x, K, tokens, want_entropy=True), x, K, tokens, valid)


# rows of every length that kernels for many rows tell apart: chunks of 16 bytes a thread of 256, their first and last
LENGTHS = [c * 2048 + d for c in range(2, 27) for d in (-70, 3)] + [26 * 2048 - 1, 26 * 2048, 26 * 2048 + 1, 26 * 2048 + 9, 28 * 2048, 2 * 24 * 2048,
                                                                   2 * 24 * 2048 - 150, 2 * 24 * 2048 + 150, 131072, 150001]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", LENGTHS)
def test_many_rows(V, half):
    """Against sorted float64 on the GPU, some of the rows with large values next to one another or below 0."""
    V, dtype, rows = (V, torch.bfloat16, 600) if half else (V // 2 + 1, torch.float32, 600)
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(rows, V, generator=g, device=DEV) * 3
    x[3] -= 100
    x[4, V // 2:V // 2 + 700] += 20
    x[5] = x[5].sort().values
    x[6] = x[6].sort(descending=True).values
    x[7, :] = 1.25
    x[8, : V - 40] = -math.inf
    x[9, 40:] = torch.finfo(dtype).min
    x = x.to(dtype)
    tokens = torch.randint(0, V, (rows,), generator=g, device=DEV)
    tokens[8] = V - 1
    mask = torch.ones(rows, dtype=torch.bool, device=DEV)
    mask[[0, 100, 599]] = False
    order = (x.double() + 0.0).sort(dim=-1, descending=True, stable=True)
    logp = torch.log_softmax(x.double(), -1)
    for k in (20, 300):
        r = tb.top_logprobs(x, k, tokens, mask=mask, want_entropy=True)
        there = (order.values[:, :k] > -math.inf) & mask.unsqueeze(-1)
        ids = torch.where(there, order.indices[:, :k], -1)
        assert torch.equal(r.ids, ids), (k, (r.ids != ids).any(-1).nonzero()[:5].flatten().tolist())
        want = torch.where(there, logp.gather(-1, ids.clamp(min=0)), -math.inf)
        low = ~(want > -1e4)
        assert torch.equal(low, ~(r.logprobs > -1e4))
        assert ((r.logprobs.double() - want)[~low].abs() <= LP).all()
        lp = logp.gather(-1, tokens.unsqueeze(-1)).squeeze(-1)
        fine = mask & (lp > -1e4)
        assert ((r.token_logprobs.double() - lp)[fine].abs() <= LP).all()
        held = logp.clamp(min=-1e6)
        h = -(held.exp() * held).sum(-1)
        assert ((r.entropy.double() - h)[mask].abs() <= H).all()
    del order, logp


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [33, 130, 255, 285, 300, 511, 600, 635, 1000, 1023, 1100, 2000, 2047, 2512, 4000])
def test_many_alternatives_of_short_rows(V, dtype):
    """Every number of alternatives that the kernels for wavefronts tell apart, with ties and masked tokens."""
    x, tokens, g = inputs(V, 3, 40, V, dtype)
    x[0, 0] = x[0, 0].abs() * -1
    x[0, 1] = (x[0, 1] * 0.5).round()
    x[0, 2] = 3.0
    x[0, 3, torch.randperm(V, generator=g)[: V - 20].to(DEV)] = -math.inf
    x[0, 4] = torch.where(x[0, 4] > 1, x[0, 4], torch.full_like(x[0, 4], torch.finfo(dtype).min))
    valid = torch.ones(3, 40, dtype=torch.bool)
    for k in sorted({min(V, k) for k in (9, 16, 17, 32, 33, 64, 65, 100, 127, 128, 129, 192, 200, 255, 256, 257)}):
        r = tb.top_logprobs(x, k)
        _, _, ids, lps = plain.top(x, k, valid)
        assert torch.equal(r.ids.cpu(), ids), (k, (r.ids.cpu() != ids).any(-1).nonzero()[:4].tolist())
        got, want = r.logprobs.cpu().double(), lps.detach()
        low = ~(want > -1e4)
        assert torch.equal(low, ~(got > -1e4))
        near(got.masked_fill(low, 0.0), want.masked_fill(low, 0.0), LP, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [60, 500, 3000, 20011, 140000])
def test_ties(V, dtype):
    """Equal logits are taken by their ids, 0 and -0 alike: few values, one value, values of both signs."""
    g = torch.Generator().manual_seed(V)
    rows = torch.stack([torch.randint(0, 3, (V,), generator=g).float(),           # many equal ones
                        torch.zeros(V).where(torch.rand(V, generator=g) < 0.5, torch.tensor(-0.0)),
                        torch.full((V,), 2.5), torch.full((V,), -2.5),
                        -torch.randint(0, 4, (V,), generator=g).float(),
                        torch.full((V,), torch.finfo(dtype).min).scatter(0, torch.tensor([V - 1, V // 2]), 1.0),
                        torch.full((V,), -1e-30).scatter(0, torch.tensor([V - 2]), 1e-30)])
    x = rows.to(dtype).unsqueeze(0).to(DEV)
    n = rows.shape[0]
    valid = torch.ones(1, n, dtype=torch.bool)
    for k in (1, 8, min(V, 20), min(V, 300)):
        r = tb.top_logprobs(x, k)
        _, _, ids, lps = plain.top(x, k, valid)
        assert torch.equal(r.ids.cpu(), ids), [(i, (r.ids[0, i].cpu() != ids[0, i]).sum()) for i in range(n)]
        # (the lowest value has a log-probability of about itself, or -inf where float32 ends)
        want = lps.detach().float().double()
        low = want < -1e4
        got = r.logprobs.cpu().double()
        near(got.masked_fill(low, 0.0), want.masked_fill(low, 0.0), LP)
        assert (got[low] <= want[low] * (1 - 2.0 ** -22)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 400, 3000, 20011, 140000])
def test_places_of_the_largest(V, dtype):
    """All large values next to one another, at the beginning, the end and in between, or in ascending or
    descending order: bounds that go by lanes then let many through."""
    ramp = torch.arange(V, dtype=torch.float64) / V * 20 - 10
    rows = [ramp, ramp.flip(0), -ramp.abs()]
    for at in (0, V // 2, V - min(V, 300)):
        few = torch.randn(V, generator=torch.Generator().manual_seed(at + 1)).double() - 30
        few[at:at + 300] += 40
        rows.append(few)
    x = torch.stack(rows).to(dtype).unsqueeze(0).to(DEV)
    valid = torch.ones(1, len(rows), dtype=torch.bool)
    for k in (1, min(V, 33), min(V, 256), min(V, 1000)):
        check_values(tb.top_logprobs(x, k), x, k, None, valid, entropy=False, what=k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [9, 64, 700, 9001, 150000])
def test_masked_vocabulary(V, dtype):
    """Tokens of -inf are none of the alternatives; rows with fewer finite logits than entries; rows without a
    finite logit, with +inf or with NaN have no distribution."""
    x, tokens, g = inputs(V + 3, 1, 8, V, dtype)
    k = min(V, 40)
    keep = torch.rand(1, 8, V, generator=g) < 0.5
    keep[0, 1], keep[0, 2] = False, False
    keep[0, 1, [V - 1, V // 3]] = True                     # two are left
    keep[0, 2, V // 2] = True                              # one
    keep[0, 3] = False                                     # none
    x = torch.where(keep.to(DEV), x, torch.full_like(x, -math.inf))
    x[0, 4, V - 1], x[0, 5, 0], x[0, 6] = math.inf, math.nan, math.nan
    r = tb.top_logprobs(x, k, tokens, want_entropy=True)
    fine = [0, 1, 2, 7]
    _, _, ids, lps = plain.top(x[:, fine], k, torch.ones(1, 4, dtype=torch.bool))
    assert torch.equal(r.ids[:, fine].cpu(), ids)
    got, want = r.logprobs[:, fine].cpu().double(), lps.detach()
    assert torch.equal(got == -math.inf, want == -math.inf)
    near(got.masked_fill(ids < 0, 0.0), want.masked_fill(ids < 0, 0.0), LP)
    near(r.entropy[:, fine], ref.entropies(torch.log_softmax(x[:, fine].cpu().double(), -1),
                                           torch.ones(1, 4, dtype=torch.bool)), H)
    lost = [3, 4, 5, 6]
    assert (r.ids[:, lost] == -1).all() and r.logprobs[:, lost].isnan().all()
    assert r.token_logprobs[:, lost].isnan().all() and r.entropy[:, lost].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [64, 900, 5000, 20011, 150000])
@pytest.mark.parametrize("shift", [-2000.0, -30.0, 2000.0])
def test_shifted_logits(V, dtype, shift):
    """Softmax does not change with a constant: log-probabilities as logits, or values far from 0."""
    x, tokens, _ = inputs(V, 2, 2, V)
    x = (x + shift).to(dtype)
    valid = torch.ones(2, 2, dtype=torch.bool)
    tol = LP + 4 * abs(shift) * 2.0 ** -24       # (products of the shift's size with log2(e) are rounded)
    check_values(tb.top_logprobs(x, 17, tokens), x, 17, tokens, valid, entropy=False, tol=tol)


@pytest.mark.parametrize("V", [64, 700, 9001, 150000])
def test_extreme_logits(V):
    """Logits of 1e30 and parts of a row 88 and more apart."""
    x, tokens, _ = inputs(V, 1, 4, V)
    x[0, 0] *= 1e30
    x[0, 1, : V // 2] += 90
    x[0, 2, V // 2:] += 1000
    x[0, 3] = x[0, 3].abs() * -1e30
    valid = torch.ones(1, 4, dtype=torch.bool)
    r = tb.top_logprobs(x, 9, tokens, want_entropy=True)
    _, logp, ids, lps = plain.top(x, 9, valid)
    assert torch.equal(r.ids.cpu(), ids)
    want = lps.detach()
    near(r.logprobs, want, LP + want.abs() * 2.0 ** -22 + 4000 * 2.0 ** -24)
    assert torch.isfinite(r.entropy).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [3, 64, 250, 1031, 9001, 150000])
def test_positions_that_do_not_count(V, dtype):
    x, tokens, _ = inputs(V, 4, 5, V, dtype)
    lengths = torch.tensor([5, 0, 2, 4], device=DEV)
    mask = torch.ones(4, 5, dtype=torch.bool, device=DEV)
    mask[0, 1] = mask[3, 0] = False
    k = min(V, 7)
    kw = dict(lengths=lengths, mask=mask, want_entropy=True)
    want = tb.top_logprobs(x, k, tokens, **kw)
    valid = ref.valid_positions((4, 5), lengths, mask)
    check_values(want, x, k, tokens, valid)
    dead = ~valid.to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for filler in (math.nan, math.inf, -math.inf, torch.finfo(dtype).min):
        y, ids = x.clone(), tokens.clone()
        y[dead], ids[dead] = filler, 1 << 40
        for a, b in zip(tb.top_logprobs(y, k, ids, status=status, **kw), want):
            assert torch.equal(a, b)
    assert int(status) == 0
    assert (want.ids[dead] == -1).all() and (want.logprobs[dead] == -math.inf).all()
    assert not want.token_logprobs[dead].any() and not want.entropy[dead].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [61, 600, 5003, 140003])
def test_strides_and_alignments(V, dtype):
    """Views into wider rows at every alignment, shifted positions, sequences behind positions, packed rows."""
    B, T, k = 2, 3, 11
    x, tokens, _ = inputs(V, B, T, V, dtype)
    valid = torch.ones(B, T, dtype=torch.bool)
    wide = torch.full((B, T, V + 9), math.nan, dtype=dtype, device=DEV)
    for lo in (0, 1, 3, 8):
        view = wide[..., lo:lo + V]
        view.copy_(x)
        check_values(tb.top_logprobs(view, k, tokens), x, k, tokens, valid, entropy=False, what=lo)
        wide.fill_(math.nan)
    want = tb.top_logprobs(x, k, tokens, want_entropy=True)
    turned = x.transpose(0, 1).contiguous().transpose(0, 1)
    longer = torch.cat([x, x[:, :1]], 1)[:, :T]
    ids = torch.cat([tokens[:, :1], tokens], 1)[:, 1:].int()
    across = x.transpose(1, 2).contiguous().transpose(1, 2)            # values of a row apart
    for y in (turned, longer, across):
        r = tb.top_logprobs(y, k, ids, want_entropy=True)
        assert torch.equal(r.ids, want.ids)
        near(r.logprobs, want.logprobs.cpu().double(), 2 * LP)
    r = tb.top_logprobs(x.flatten(0, 1), k, tokens.flatten(), mask=torch.tensor([1, 1, 0, 1, 1, 1], device=DEV).bool())
    assert torch.equal(r.ids[[0, 1, 3, 4, 5]], want.ids.flatten(0, 1)[[0, 1, 3, 4, 5]]) and (r.ids[2] == -1).all()
    r = tb.top_logprobs(x[:1].expand(3, T, V), k)                      # one row of memory for all sequences
    assert torch.equal(r.ids, want.ids[:1].expand(3, T, k))


def gradients(x, k, tokens, valid, d_top, d_lp, d_h, temperature):
    """(gradient, what its bounds are made of) in float64."""
    rx, logp, ids, lps = plain.top(x, k, valid, temperature)
    there = ids >= 0
    d_top = torch.where(there, d_top.double(), torch.zeros((), dtype=torch.float64))
    total = (torch.where(there, lps, torch.zeros_like(lps)) * d_top).sum()
    extra = torch.zeros_like(logp).detach().scatter_add_(-1, ids.clamp(min=0), d_top.abs())
    size = d_top.abs().sum(-1)
    if d_lp is not None:
        d_lp = torch.where(valid, d_lp.double(), torch.zeros((), dtype=torch.float64))
        total = total + (ref.chosen(logp, tokens, valid) * d_lp).sum()
        extra += bounds.at_tokens(extra, torch.where(valid, tokens.cpu().long(), 0), d_lp)
        size = size + d_lp.abs()
    if d_h is not None:
        d_h = torch.where(valid, d_h.double(), torch.zeros((), dtype=torch.float64))
        total = total + (ref.entropies(logp, valid) * d_h).sum()
    grad, = torch.autograd.grad(total, rx)
    held = torch.where(valid.unsqueeze(-1), logp.detach(), torch.full_like(logp.detach(), -math.inf))
    bound = bounds.of_softmax(held, size, extra, d_h)
    return grad, 2 * bound / temperature


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 33, 64, 100, 257, 512, 1031, 4097, 8200, 20011, 50257, 140000])
def test_gradient(V, dtype):
    B, T = 2, 3
    x, tokens, g = inputs(V + 1, B, T, V, dtype)
    lengths = torch.tensor([3, 2], device=DEV, dtype=torch.int32)
    valid = ref.valid_positions((B, T), lengths)
    temperature = 1.3 if V % 2 else 1.0
    k = min(V, 20)
    with torch.no_grad():
        tokens[0, 0] = x[0, 0].argmax()                                # (the token is an alternative, too)
    d_top, d_lp, d_h = torch.randn(B, T, k, generator=g), torch.randn(B, T, generator=g), torch.randn(B, T, generator=g)
    for use_tokens, use_h in ((True, True), (False, False), (True, False), (False, True)):
        leaf = x.clone().requires_grad_()
        r = tb.top_logprobs(leaf, k, tokens if use_tokens else None, lengths=lengths, temperature=temperature,
                            want_entropy=use_h)
        values, given = [r.logprobs], [d_top.to(DEV)]
        if use_tokens:
            values, given = values + [r.token_logprobs], given + [d_lp.to(DEV)]
        if use_h:
            values, given = values + [r.entropy], given + [d_h.to(DEV)]
        got, = torch.autograd.grad(values, leaf, given)
        want, bound = gradients(x, k, tokens, valid, d_top, d_lp if use_tokens else None, d_h if use_h else None, temperature)
        bounds.check(got, want, bound, dtype, (use_tokens, use_h))
        assert not got[1, 2].any()
    # of a part of the values
    leaf = x.clone().requires_grad_()
    r = tb.top_logprobs(leaf, k, tokens, lengths=lengths, temperature=temperature, want_entropy=True)
    got, = torch.autograd.grad(r.token_logprobs, leaf, d_lp.to(DEV))
    want, bound = gradients(x, k, tokens, valid, torch.zeros_like(d_top), d_lp, None, temperature)
    bounds.check(got, want, bound, dtype, "token log-probabilities alone")


def test_gradient_against_differences():
    """In float32, by differences of the values themselves along random directions."""
    V, k = 40, 6
    x, tokens, g = inputs(5, 1, 2, V)
    d_top, d_lp, d_h = torch.randn(1, 2, k, generator=g).to(DEV), torch.randn(1, 2, generator=g).to(DEV), torch.randn(1, 2, generator=g).to(DEV)

    def value(y):
        r = tb.top_logprobs(y, k, tokens, want_entropy=True)
        return ((r.logprobs.double() * d_top).sum() + (r.token_logprobs.double() * d_lp).sum() + (r.entropy.double() * d_h).sum()), r.ids
    leaf = x.clone().requires_grad_()
    v, ids = value(leaf)
    grad, = torch.autograd.grad(v, leaf)
    for i in range(8):
        step = torch.randn(1, 2, V, generator=g).to(DEV)
        h = 2.0 ** -7
        (up, ids_up), (down, ids_down) = value(x + h * step), value(x - h * step)
        if not (torch.equal(ids_up, ids) and torch.equal(ids_down, ids)):
            continue
        # third derivatives of log-probabilities and entropies times |step|^3 h^2 / 6, and values off by LP each
        slope = float((grad.double() * step).sum())
        size = float(d_top.abs().sum() + d_lp.abs().sum() + 20 * d_h.abs().sum())
        assert abs(float(up - down) / (2 * h) - slope) <= size * (30 * h * h + 1e-6 / h)


def test_alternatives_teach():
    """Ids and log-probabilities are a teacher's of distillation_loss: the divergence from oneself is 0 up to the tail
    that is left out, and that from another model is that of its definition."""
    x, tokens, _ = inputs(3, 3, 4, 1000, torch.bfloat16)
    student, _, _ = inputs(4, 3, 4, 1000, torch.bfloat16)
    lengths = torch.tensor([4, 0, 2], device=DEV, dtype=torch.int32)
    for k in (1, 50, 1000):
        best = tb.top_logprobs(x, k, lengths=lengths)
        r = tb.distillation_loss_grad(student, best.ids, best.logprobs, lengths=lengths)
        terms, grad, rows = ref.distillation(student, best.ids, best.logprobs, lengths)
        near(r.row_loss, rows, 2 * LP)
        if k == 1000:
            p, q = (torch.log_softmax(t.cpu().double(), -1) for t in (x, student))
            want = (p.exp() * (p - q)).sum(-1) * ref.valid_positions((3, 4), lengths)
            near(r.row_loss, want, 4 * LP)
            near(tb.distillation_loss_grad(x, best.ids, best.logprobs, lengths=lengths).row_loss, torch.zeros(3, 4).double(), 2 * LP)


def test_two_streams_at_once():
    """Calls that share nothing but the logits, on two streams at the same time, and results that are read on a third."""
    x, tokens, _ = inputs(9, 4, 300, 50257, torch.bfloat16)
    few = x[:1, :3].clone()
    big = torch.randn(2, 1, 400000, device=DEV)
    want = tb.top_logprobs(x, 20, tokens, want_entropy=True), tb.top_logprobs(few, 300), tb.top_logprobs(big, 9)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    found = []
    for i in range(9):
        with torch.cuda.stream(streams[i % 3]):
            found.append((tb.top_logprobs(x, 20, tokens, want_entropy=True), tb.top_logprobs(few, 300), tb.top_logprobs(big, 9)))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for calls in found:
        for got, ref_ in zip(calls, want):
            assert all(a is b or torch.equal(a, b) for a, b in zip(got, ref_))


def test_wrong_tokens_and_lengths():
    x, tokens, _ = inputs(3, 2, 3, 5000)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    wrong = tokens.clone()
    wrong[0, 1], wrong[1, 0] = -1, 5000
    r = tb.top_logprobs(x, 5, wrong, status=status, want_entropy=True)
    want = tb.top_logprobs(x, 5, tokens, want_entropy=True)
    assert int(status) == tb.TB_DEV_TOKEN_RANGE
    assert torch.equal(r.ids, want.ids) and torch.equal(r.logprobs, want.logprobs) and torch.equal(r.entropy, want.entropy)
    assert r.token_logprobs[0, 1].isnan() and r.token_logprobs[1, 0].isnan() and int(r.token_logprobs.isnan().sum()) == 2
    leaf = x.clone().requires_grad_()
    tb.top_logprobs(leaf, 5, wrong).token_logprobs.nan_to_num(0.0).sum().backward()
    assert leaf.grad[0, 1].isnan().all() and leaf.grad[1, 0].isnan().all() and torch.isfinite(leaf.grad[0, 0]).all()
    for V in (60, 600, 5000, 300000):
        x, tokens, _ = inputs(3, 2, 3, V)
        status.zero_()
        long = tb.top_logprobs(x, 5, tokens, lengths=torch.tensor([4, -1], device=DEV, dtype=torch.int32), status=status)
        want = tb.top_logprobs(x, 5, tokens, lengths=torch.tensor([3, 0], device=DEV, dtype=torch.int32))
        assert int(status) == tb.TB_DEV_LENGTH_RANGE
        assert all(torch.equal(a, b) for a, b in zip(long[:3], want[:3]))


def test_nothing_to_do():
    for shape in ((0, 4, 50), (3, 0, 50), (0, 50)):
        x = torch.empty(shape, device=DEV, requires_grad=True)
        r = tb.top_logprobs(x, 5, torch.empty(shape[:-1], dtype=torch.int64, device=DEV), want_entropy=True)
        assert r.ids.shape == r.logprobs.shape == (*shape[:-1], 5) and r.entropy.shape == shape[:-1]
        (r.logprobs.sum() + r.token_logprobs.sum()).backward()
        assert x.grad.shape == shape


def test_refusals():
    x, tokens, _ = inputs(1, 2, 3, 50)
    for k in (0, -1, 51, 1025, 2.0, True, None):
        with pytest.raises(tb.TensorBLEUError, match="k must be"):
            tb.top_logprobs(x, k, tokens)
    with pytest.raises(tb.TensorBLEUError, match="id_dtype"):
        tb.top_logprobs(x, 3, id_dtype=torch.int16)
    for bad in (tokens[:1], tokens.float(), tokens.cpu()):
        with pytest.raises(tb.TensorBLEUError):
            tb.top_logprobs(x, 3, bad)
    with pytest.raises(tb.TensorBLEUError):
        tb.top_logprobs(x.double(), 3)
    with pytest.raises(tb.TensorBLEUError):
        tb.top_logprobs(x, 3, temperature=0.0)
    with pytest.raises(tb.TensorBLEUError, match="mask"):
        tb.top_logprobs(x.flatten(0, 1), 3, lengths=torch.ones(2, device=DEV))
    leaf = x.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="differentiated twice"):
        torch.autograd.grad(tb.top_logprobs(leaf, 3).logprobs.sum(), leaf, create_graph=True)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(tb.TensorBLEUError, match="tangent"):
            tb.top_logprobs(dual, 3)


def test_general_way_and_hooks():
    """int64 lengths go through the general way, whose results and gradients are the native ones' bit by bit; hooks on saved
    tensors may give back other memory and strides; changed logits are noticed."""
    x, tokens, g = inputs(6, 3, 4, 700, torch.bfloat16)
    lengths = torch.tensor([4, 1, 3], device=DEV, dtype=torch.int32)
    d = torch.randn(3, 4, 5, generator=g).to(DEV), torch.randn(3, 4, generator=g).to(DEV)

    def step(n, hooks=None):
        leaf = x.clone().requires_grad_()
        with hooks or torch.enable_grad():
            r = tb.top_logprobs(leaf, 5, tokens, lengths=n, want_entropy=True)
        return [t.detach() for t in r] + list(torch.autograd.grad([r.logprobs, r.token_logprobs, r.entropy], leaf, [*d, d[1]]))
    want = step(lengths)
    moved = torch.autograd.graph.saved_tensors_hooks(
        lambda t: t.cpu(), lambda t: t.to(DEV).transpose(0, -1).contiguous().transpose(0, -1))
    for got in (step(lengths.long()), step(lengths, moved), step(lengths.long(), torch.autograd.graph.save_on_cpu())):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    leaf = x.clone().requires_grad_()
    y = leaf * 1
    r = tb.top_logprobs(y, 5)
    y.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        r.logprobs.sum().backward()
    r = tb.top_logprobs(leaf, 5, tokens)
    assert not r.ids.requires_grad and r.logprobs.requires_grad and r.token_logprobs.requires_grad and r.entropy is None


@pytest.mark.parametrize("V,k", [(64, 9), (700, 9), (700, 200), (9001, 9), (50257, 300), (300000, 9)])
def test_streams_graphs_and_order(V, k):
    """On a stream of its own; captured and replayed with eager work between; the same bits every time."""
    T = 7
    x, tokens, g = inputs(V, 2, T, V, torch.bfloat16)
    others = [inputs(V + i, 2, T, V, torch.bfloat16)[0] for i in (1, 2, 3)]
    eager = [tb.top_logprobs(y, k, tokens, want_entropy=True) for y in others]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        r = [tb.top_logprobs(y, k, tokens, want_entropy=True) for y in others]
    torch.cuda.current_stream().wait_stream(stream)
    for a, b in zip(r, eager):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    still = x.clone()
    d = torch.randn(2, T, k, generator=g).to(DEV)

    def step():
        leaf = still.detach().requires_grad_()
        out = tb.top_logprobs(leaf, k, tokens, want_entropy=True)
        return [t.detach() for t in out] + list(torch.autograd.grad([out.logprobs, out.entropy], leaf, [d, d[..., 0]]))
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for y in others + others:
        still.copy_(y)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want))


@pytest.mark.parametrize("lengths", [None, torch.int64])
def test_a_capture_beside_an_eager_graph(lengths):
    """A leaf that a graph from outside holds: the captured backward pass is refused; without that graph it runs."""
    x, tokens, _ = inputs(9, 2, 6, 700, torch.float32)
    leaf = x.clone().requires_grad_()
    where = {} if lengths is None else dict(lengths=torch.tensor([6, 2], device=DEV, dtype=lengths))
    f = lambda: tb.top_logprobs(leaf, 5, tokens, **where).token_logprobs.sum()
    held = f()
    want, = torch.autograd.grad(held, leaf, retain_graph=True)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="outside the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            torch.autograd.grad(f(), leaf)
    del held
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, = torch.autograd.grad(f(), leaf)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [8, 17, 64, 100, 256, 511, 1000])
def test_few_alternatives_of_short_rows(V, dtype):
    """One to eight of rows with ties, 0 and -0 and masks, some of which leave less than K; ragged, so that wavefronts
    hold rows that do not count, and a number of rows that fills no wavefront."""
    x, tokens, g = inputs(V, 5, 41, V, dtype)
    x = (x * 2).round() / 2
    x[0, :9] = x[0, :9].masked_fill((torch.rand(9, V, generator=g) < 0.9).to(DEV), -math.inf)
    x[1, 3], x[1, 4, V // 2], x[1, 5] = -math.inf, math.nan, -0.0
    lengths = torch.tensor([41, 7, 0, 20, 33], device=DEV, dtype=torch.int32)
    valid = ref.valid_positions((5, 41), lengths)
    lost = valid & ((x == -math.inf).all(-1) | x.isnan().any(-1)).cpu()           # (rows without a distribution)
    assert lost[1, 3] and lost[1, 4]
    for k in range(1, 9):
        r = tb.top_logprobs(x, k, tokens, lengths=lengths, want_entropy=True)
        assert (r.ids.cpu()[lost] == -1).all() and r.logprobs.cpu()[lost].isnan().all()
        _, _, ids, lps = plain.top(x.masked_fill(lost.to(DEV).unsqueeze(-1), 0.0), k, valid & ~lost)
        assert torch.equal(r.ids.cpu().long(), ids)
        got = r.logprobs.cpu().double()
        there, none = ids >= 0, (ids < 0) & ~lost.unsqueeze(-1)
        assert (got[none] == -math.inf).all()
        near(torch.where(there, got, 0.0), torch.where(there, lps.detach(), torch.zeros_like(lps)), LP, k)
