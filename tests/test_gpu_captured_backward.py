"""Backward passes that are captured while a graph from outside the capture holds a leaf that they end at: refused by
every operator, however far the leaf is, before torch's engine takes the default stream into the capture.  What
does not go on to that leaf is captured and replayed."""
import gc

import pytest
import torch

import paper_2510_05485_amd as tb
from test_gpu_losses_autograd import operators

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ["scores", "logprobs", "policy", "preference", "distillation", "top"]


class Doubled(torch.autograd.Function):
    """A Function of Python between the leaf and the operator."""
    @staticmethod
    def forward(ctx, x):
        return 2 * x

    @staticmethod
    def backward(ctx, d):
        return 2 * d


BETWEEN = dict(nothing=lambda x: x, product=lambda x: x * 1.5, cast=lambda x: x.to(torch.bfloat16), function=Doubled.apply,
               chain=lambda x: (x.transpose(0, 1).to(torch.float16) * 0.5).transpose(0, 1))


def functions(native, V=700):
    x, all_of = operators(V, native=native)
    tokens = torch.zeros(x.shape[:2], dtype=torch.long, device=DEV)
    mask = torch.ones_like(tokens, dtype=torch.bool) if native else torch.ones(*x.shape[:2], 2, dtype=torch.bool, device=DEV)[..., 0]
    all_of["top"] = lambda y: tb.top_logprobs(y, 5, tokens, mask=mask).token_logprobs.sum()
    table = torch.randn(50, 24, device=DEV)
    ids = torch.randint(0, 50, (2, 30), device=DEV)
    lengths = torch.tensor([30, 11], device=DEV, dtype=torch.int32 if native else torch.int64)
    return x, all_of, table, lambda y: tb.embedding(y, ids, scale=2.0, lengths=lengths).float().square().sum()


def refused_then_captured(x, f, between):
    leaf = x.clone().requires_grad_()
    step = lambda: torch.autograd.grad(f(between(leaf)), leaf)[0]
    want = step()
    held = leaf * 1.0                                          # (a graph of the default stream that holds the leaf)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="outside the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step()
    del held
    gc.collect()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("between", BETWEEN)
def test_losses(between, name, native):
    x, all_of, _, _ = functions(native)
    refused_then_captured(x, all_of[name], BETWEEN[between])


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("between", BETWEEN)
def test_embedding(between, native):
    _, _, table, f = functions(native)
    refused_then_captured(table, f, BETWEEN[between])


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES + ["embedding"])
def test_gradients_that_stop_before_the_leaf(name, native):
    """Those of logits (or of a scaled table) alone: the leaf behind them may be held by what it likes."""
    x, all_of, table, lookup = functions(native)
    x, f = (table, lookup) if name == "embedding" else (x, all_of[name])
    leaf = x.clone().requires_grad_()
    held = leaf * 1.0

    def step():
        y = leaf * 1.5
        return torch.autograd.grad(f(y), y)[0]
    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    assert torch.equal(held, x)
