"""The losses over logits as parts of torch's graph: saved tensors that hooks replace, gradients written over
what is saved, tangents.

A hook gives back other memory than the forward pass's, which is gone by then, with other strides; the
gradient is the one without hooks, bit by bit where rows begin at the same addresses modulo 128 (the
clones here do: every allocation begins at a multiple of 512, and strides are kept or all rows are read
in the same order)."""
import math

import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2510_05485_amd as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def apart(v):
    """The same values, not contiguous: the general way of marshalling."""
    return torch.stack([v, v], -1)[..., 0]


def operators(V, seed=0, B=4, T=6, native=True):
    """Logits, and functions of logits: a scalar each, through every operator."""
    g = torch.Generator().manual_seed(seed + V)
    x = (torch.randn(B, T, V, generator=g) * 2).to(DEV)
    tokens = torch.randint(0, V, (B, T), generator=g).to(DEV)
    old, reference = (-3 + torch.randn(B, T, generator=g).to(DEV) for _ in range(2))
    a = torch.randn(B, generator=g).to(DEV)
    K = min(V, 5)
    ids, teacher = torch.randint(0, V, (B, T, K), generator=g).to(DEV), torch.randn(B, T, K, generator=g).to(DEV)
    d = torch.randn(2, B, T, generator=g).to(DEV)
    lengths = torch.tensor([6, 0, 4, 5], device=DEV, dtype=torch.int32)
    mask = (torch.rand(B, T, generator=g) < 0.8).to(DEV)
    if not native:
        lengths, old, reference, teacher = lengths.long(), apart(old), apart(reference), apart(teacher)
    where = dict(lengths=lengths, mask=mask, temperature=0.9)

    def scores(y):
        lp, h = tb.token_logprobs(y, tokens, want_entropy=True, **where)
        return (lp * d[0]).sum() + (h * d[1]).sum()
    return x, dict(
        scores=scores,
        logprobs=lambda y: (tb.token_logprobs(y, tokens, **where) * d[0]).sum(),
        policy=lambda y: tb.policy_loss(y, tokens, old, a, ref_logprobs=reference, kl_coef=0.1, entropy_coef=0.1, **where),
        preference=lambda y: tb.preference_loss(y, tokens, reference, beta=0.5, **where),
        distillation=lambda y: tb.distillation_loss(y, ids, teacher, **where))


def gradient_of(f, x):
    leaf = x.clone().requires_grad_()
    # (logits are the product of a layer, so that nothing but the loss's saved tensors holds them)
    return torch.autograd.grad(3 * f(leaf * 1.5), leaf)[0]


class Replaced(torch.autograd.graph.saved_tensors_hooks):
    """Saved tensors live on the host and come back through `restore`."""

    def __init__(self, restore=lambda t: t):
        self.saved = 0

        def pack(t):
            self.saved += 1
            return t.detach().cpu().clone()
        super().__init__(pack, lambda t: restore(t.to(DEV)))


def litter(x):
    """What the forward pass's memory holds next: NaN, in every size that it may have come from."""
    rows = x.numel() // x.shape[-1]
    return [torch.full((n,), math.nan, device=DEV) for n in (1, rows, 2 * rows, 4 * rows, 5 * rows, x.numel()) for _ in range(4)]


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("V", [3, 64, 1031, 9001])
def test_saved_tensors_from_the_host(V, native):
    x, all_of = operators(V, native=native)
    for name, f in all_of.items():
        want = gradient_of(f, x)
        leaf = x.clone().requires_grad_()
        hooks = Replaced()
        with hooks:
            loss = 3 * f(leaf * 1.5)
        assert hooks.saved
        over = litter(x)
        got, = torch.autograd.grad(loss, leaf)
        assert torch.equal(got, want), name
        del over


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("V", [64, 1031])
def test_saved_tensors_with_other_strides(V, native):
    """What a hook gives back need not be laid out as it was."""
    def turned(t):
        if t.dim() < 2:
            return apart(t) if t.dim() else t
        return t.transpose(-1, -2).contiguous().transpose(-1, -2)
    x, all_of = operators(V, native=native)
    for name, f in all_of.items():
        want = gradient_of(f, x)
        leaf = x.clone().requires_grad_()
        with Replaced(turned):
            loss = 3 * f(leaf * 1.5)
        got, = torch.autograd.grad(loss, leaf)
        assert torch.equal(got, want), name


def test_views_that_come_back_whole():
    """Logits that are a view of a longer model output: a copy of them has other strides."""
    x, all_of = operators(64)
    for name, f in all_of.items():
        wide = torch.zeros(4, 7, 64, device=DEV)
        wide[:, :6] = x
        leaf = wide.requires_grad_()
        want, = torch.autograd.grad(f((leaf * 1.0)[:, :-1]), leaf)
        with Replaced():
            loss = f((leaf * 1.0)[:, :-1])
        over = litter(wide)
        got, = torch.autograd.grad(loss, leaf)
        assert torch.equal(got, want) and not got[:, 6:].any(), name
        del over


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("V", [64, 1031, 9001])
def test_checkpoint(V, native):
    """The head and its loss computed anew in the backward pass, twice in a row."""
    x, all_of = operators(V, native=native)
    for name, f in all_of.items():
        want = gradient_of(f, x)
        leaf = x.clone().requires_grad_()
        losses = [checkpoint(lambda y: f(y * 1.5), leaf, use_reentrant=False) for _ in range(2)]
        over = litter(x)
        got, = torch.autograd.grad(3 * losses[0], leaf)
        assert torch.equal(got, want), name
        (3 * losses[1]).backward()
        assert torch.equal(leaf.grad, want), name
        del over


def test_save_on_cpu():
    x, all_of = operators(300)
    for name, f in all_of.items():
        want = gradient_of(f, x)
        leaf = x.clone().requires_grad_()
        with torch.autograd.graph.save_on_cpu():
            loss = 3 * f(leaf * 1.5)
        over = litter(x)
        assert torch.equal(torch.autograd.grad(loss, leaf)[0], want), name
        del over


def test_hooks_that_give_back_something_else():
    """Another shape or type than was saved is refused, not read."""
    x, all_of = operators(64)
    for cut in (lambda t: t[..., :-1] if t.dim() == 3 and t.shape[-1] == 64 else t,
                lambda t: t.double() if t.dim() == 3 and t.shape[-1] == 64 else t,
                lambda t: t[:-1] if t.dtype == torch.int32 else t,
                lambda t: t[:, :-1] if t.dtype == torch.bool else t,
                lambda t: t[:, :3] if t.dim() == 3 and t.shape[-1] == 4 else t,
                lambda t: t.cpu() if t.dtype == torch.int32 else t):
        for name, f in all_of.items():
            leaf = x.clone().requires_grad_()
            y = leaf * 1.5
            with Replaced(cut):
                loss = f(y)
            with pytest.raises(RuntimeError):
                torch.autograd.grad(loss, leaf)


def with_gradient(native):
    """Every operator that returns its gradient, as a function of logits and `out`."""
    x, _ = operators(64)
    g = torch.Generator().manual_seed(1)
    tokens, ids = torch.randint(0, 64, (4, 6), generator=g).to(DEV), torch.randint(0, 64, (4, 6, 5), generator=g).to(DEV)
    v, a, teacher = torch.full((4, 6), -4.0, device=DEV), torch.ones(4, device=DEV), torch.zeros(4, 6, 5, device=DEV)
    if not native:
        v, teacher = apart(v), apart(teacher)
    return x, tokens, [lambda y, out: tb.policy_loss_grad(y, tokens, v, a, out=out),
                       lambda y, out: tb.preference_loss_grad(y, tokens, v, out=out),
                       lambda y, out: tb.distillation_loss_grad(y, ids, teacher, out=out)]


@pytest.mark.parametrize("native", [True, False])
def test_a_gradient_written_over_saved_logits_is_noticed(native):
    x, tokens, all_of = with_gradient(native)
    for f in all_of:
        for of in (lambda y: y.detach(), lambda y: y):
            leaf = x.clone().requires_grad_()
            y = leaf * 1.5
            loss = tb.token_logprobs(y, tokens).sum() + torch.logsumexp(y, -1).sum()
            want, = torch.autograd.grad(loss, leaf, retain_graph=True)
            before = y._version
            r = f(of(y), of(y))
            assert y._version > before and r.grad.data_ptr() == y.data_ptr()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                torch.autograd.grad(loss, leaf)
        # the gradient itself goes on into the model from there
        leaf = x.clone().requires_grad_()
        y = leaf * 1.5
        expected = f(y.detach(), None).grad
        f(y.detach(), y.detach())
        y.backward(y.detach().clone())
        assert torch.equal(leaf.grad, 1.5 * expected)
        # elsewhere than the logits: these have not changed
        out = torch.empty_like(x)
        before, at = x._version, out._version
        f(x, out)
        assert out._version > at and x._version == before


@pytest.mark.parametrize("native", [True, False])
def test_out_in_inference_mode(native):
    """Tensors of inference mode have no version to count."""
    x, tokens, all_of = with_gradient(native)
    for f in all_of:
        want = f(x, None).grad
        with torch.inference_mode():
            out = torch.empty_like(x)
            assert torch.equal(f(x, out).grad, want)
        assert torch.equal(f(x, out).grad, want)


@pytest.mark.parametrize("native", [True, False])
def test_tangents_are_refused(native):
    """Forward-mode differentiation: a result without a tangent would stand for one of 0."""
    x, _, given = with_gradient(native)
    _, all_of = operators(64, native=native)
    with torch.autograd.forward_ad.dual_level():
        for leaf in (x, x.clone().requires_grad_()):
            dual = torch.autograd.forward_ad.make_dual(leaf, torch.ones_like(x))
            for f in list(all_of.values()) + [lambda y, f=f: f(y, None) for f in given]:
                with pytest.raises(tb.TensorBLEUError, match="forward-mode"):
                    f(dual)
        for f in all_of.values():                # without a tangent, as outside
            assert torch.isfinite(f(x))


def test_entropies_that_any_true_value_asks_for():
    x, _ = operators(64)
    tokens = torch.zeros(4, 6, dtype=torch.int64, device=DEV)
    lp, h = tb.token_logprobs(x, tokens, want_entropy=True)
    for yes in (1, "yes"):
        found = tb.token_logprobs(x, tokens, want_entropy=yes)
        assert isinstance(found, tuple) and torch.equal(found[0], lp) and torch.equal(found[1], h)
    for no in (0, None):
        assert torch.equal(tb.token_logprobs(x, tokens, want_entropy=no), lp)
