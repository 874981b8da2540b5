"""The gradient of lookups in tables of more than two million rows by more than 65536 positions: the sort parts the
positions by eleven bits of their tokens, and workgroups that share a digit take a range of its rows each.  Tolerances are
those of test_gpu_embeddings.py."""
import math

import pytest
import torch

import paper_2510_05485_amd as tb
import top_reference as plain
from test_gpu_embeddings import check_sums

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tokens_of(kind, N, V, D, g):
    low = max(0, math.ceil(math.log2(128 / D))) if D < 128 else 0             # (neighbours that share a digit)
    if kind == "uniform":
        return torch.randint(0, V, (N,), generator=g)
    # tokens of the digit 7, on both sides of every end of a range (1024 rows of the digit), and the table's last rows
    rows = torch.tensor([r for e in range(0, V >> 11, 1024) for r in range(e - 3, e + 4)] + [(V >> 11) - 1])
    rows = rows[(rows >= 0) & (rows < V >> 11)]
    few = ((rows >> low << 11 | 7) << low | (rows & ((1 << low) - 1))).tolist()
    few = torch.tensor([t for t in few if t < V] + [V - 1, V - 2, 0])
    at = torch.randint(0, len(few), (N,), generator=g)
    if kind == "one":
        at[torch.rand(N, generator=g) < 0.9] = len(few) // 2
    mixed = torch.randint(0, V, (N,), generator=g)
    return torch.where(torch.rand(N, generator=g) < (0.5 if kind == "ends" else 0.95), few[at], mixed)


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)])
@pytest.mark.parametrize("kind", ["uniform", "ends", "one"])
@pytest.mark.parametrize("N,V,D", [(65537, 2_097_152, 5), (65537, 2_097_153, 5), (70001, 2_100_000, 130), (90000, 5_000_000, 16),
                                   (300_000, 5_000_000, 1), (66000, 30_000_000, 2), (1_000_000, 3_000_000, 8)])
def test_gradient(N, V, D, kind, dtype, out):
    g = torch.Generator().manual_seed(N + V + D)
    ids = tokens_of(kind, N, V, D, g)
    rows = torch.randn(N, D, generator=g).to(dtype)
    mask = torch.rand(N, generator=g) < 0.9
    touched, inverse = ids[mask].unique(return_inverse=True)
    places = torch.zeros(N, dtype=torch.long)
    places[mask] = inverse
    grad, size, counts = plain.embedding_grad(rows, places, len(touched), mask, 3.0)
    at, ids, rows, valid = touched.to(DEV), ids.to(DEV), rows.to(DEV), mask.to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = tb.embedding_grad(rows, ids, V, scale=3.0, mask=valid, dtype=out, status=status)
    check_sums(got[at], grad, size, counts)
    assert torch.equal(got, tb.embedding_grad(rows, ids.int(), V, scale=3.0, mask=valid, dtype=out))
    got[at] = 0
    assert not got.any() and int(status) == 0
    # added to what is there: no other row is touched
    old = torch.randn(len(touched), D, generator=g).to(out)
    held = torch.full((V, D), math.nan, dtype=out, device=DEV)
    held[at] = old.to(DEV)
    tb.embedding_grad(rows, ids, V, scale=3.0, mask=valid, out=held, accumulate=True)
    check_sums(held[at], grad, size, counts, old)
    held[at] = math.nan
    assert held.isnan().all()


def test_wrong_tokens_and_none():
    N, V, D = 70000, 2_500_000, 3
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(0, V, (N,), generator=g).to(DEV)
    rows = torch.randn(N, D, generator=g).to(DEV)
    wrong = ids.clone()
    wrong[5], wrong[N - 1], wrong[N // 2] = -1, V, 1 << 40
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = tb.embedding_grad(rows, wrong, V, status=status)
    assert int(status) == tb.TB_DEV_TOKEN_RANGE
    assert torch.equal(got, tb.embedding_grad(rows, ids, V, mask=wrong == ids))
    assert not tb.embedding_grad(rows, ids, V, mask=torch.zeros(N, dtype=torch.bool, device=DEV)).any()


def test_replays_of_a_captured_call():
    N, V, D = 70000, 2_500_000, 6
    g = torch.Generator().manual_seed(2)
    draws = [(torch.randint(0, V, (N,), generator=g).to(DEV), torch.randn(N, D, generator=g).to(DEV)) for _ in range(3)]
    ids, rows = draws[0][0].clone(), draws[0][1].clone()
    tb.embedding_grad(rows, ids, V)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = tb.embedding_grad(rows, ids, V)
    for i, r in draws + draws:
        ids.copy_(i)
        rows.copy_(r)
        want = tb.embedding_grad(rows, ids, V)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
