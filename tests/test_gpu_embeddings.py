"""Embeddings and their gradient against their definitions in float64 (tests/top_reference.py).

An embedding is a product in float32, rounded once: 2^-24 and half a step of the type.  A sum of n rows in float32
adds at most n numbers one after the other, and no more than 256 of a slice, then at most n / 16 + 130 sums of
slices: each addition rounds by 2^-24 of a number that the sum of magnitudes bounds, and so do the product with the
scale and an addition to what is there."""
import gc
import math

import pytest
import torch

import loss_reference as ref
import paper_2510_05485_amd as tb
import top_reference as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
STEP = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 63, 64, 65, 100, 127, 128, 129, 200, 256, 257, 500, 512, 513, 768, 1000, 1024,
          2048, 2049, 4099]


def inputs(seed, B, T, V, D, dtype, low=0):
    g = torch.Generator().manual_seed(seed)
    table = torch.randn(V, D, generator=g).to(dtype).to(DEV)
    tokens = torch.randint(low, V, (B, T), generator=g).to(DEV)
    rows = torch.randn(B, T, D, generator=g).to(dtype).to(DEV)
    return table, tokens, rows, g


def check_rows(got, want, dtype):
    got = got.detach().cpu().double()
    assert got.shape == want.shape
    off = (got - want).abs()
    assert (off <= want.abs() * (ROUND[dtype] + U) * (1 + 2 * U) + STEP[dtype]).all(), float(off.max())


def check_sums(got, grad, size, counts, old=None):
    dtype = got.dtype
    got = got.detach().cpu().double()
    n = counts.double().unsqueeze(-1)
    depth = torch.minimum(n, 256 + n / 16 + 130) + 3
    want, bound = grad, depth * U * size
    if old is not None:
        old = old.cpu().double()
        want, bound = grad + old, bound + U * (old.abs() + size)
    off = (got - want).abs()
    allowed = bound + (want.abs() + bound) * ROUND[dtype] + STEP[dtype]
    bad = ~(off <= allowed)
    assert got.shape == want.shape and not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), off[bad][:4], want[bad][:4])


def check_gradient(rows, tokens, V, valid, scale=1.0, **kw):
    grad, size, counts = plain.embedding_grad(rows, tokens, V, valid, scale)
    got = tb.embedding_grad(rows, tokens, V, scale=scale, **kw)
    assert got.dtype == kw.get("dtype", rows.dtype)
    check_sums(got, grad, size, counts)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_values_and_gradient(D, dtype):
    B, T, V = 3, 7, 40
    table, tokens, rows, _ = inputs(D, B, T, V, D, dtype)
    lengths = torch.tensor([7, 0, 4], device=DEV, dtype=torch.int32)
    valid = ref.valid_positions((B, T), lengths)
    scale = D ** 0.5
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kw = dict(lengths=lengths, status=status)
    out = tb.embedding(table, tokens, scale=scale, **kw)
    assert out.dtype == dtype
    check_rows(out, plain.embedding(table, tokens, valid, scale), dtype)
    assert not out[~valid.to(DEV)].any()
    got = check_gradient(rows, tokens, V, valid, scale, **kw)
    check_gradient(rows, tokens.int(), V, valid, scale, dtype=torch.float32, **kw)
    leaf = table.clone().requires_grad_()
    out = tb.embedding(leaf, tokens, scale=scale, **kw)
    assert torch.equal(torch.autograd.grad(out, leaf, rows)[0], got)
    assert int(status) == 0


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                       (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
                                       (torch.float16, torch.float32)])
@pytest.mark.parametrize("B,T,V,D", [(1, 1, 1, 1), (1, 1, 50257, 64), (2, 8, 1, 24), (1, 17, 3, 100), (4, 100, 30, 40),
                                     (5, 333, 1000, 129), (16, 256, 32000, 33), (3, 1000, 2, 600), (7, 2000, 5000, 16),
                                     (2, 40000, 64, 8), (5, 20000, 300, 5), (3, 30000, 50257, 12), (100, 700, 7, 70),
                                     (1, 131073, 1, 16), (4, 9, 262144, 8), (2, 33000, 262144, 4), (40000, 2, 700, 16),
                                     (3, 5, 5_000_000, 4), (1, 70000, 5_000_000, 4),
                                     (300, 512, 64, 64), (90, 1000, 100, 37), (150, 500, 31, 131),
                                     (2, 40000, 255, 16), (3, 30000, 16, 256), (1, 2_000_000, 3, 9), (66000, 2, 256, 8), (70, 1000, 1, 129)])
def test_gradient(B, T, V, D, dtype, out):
    """One position to many, one token to many, tokens with one position to all: tokens inside a slice, over the end
    of one, over many slices."""
    _, tokens, rows, g = inputs(B + T + V, B, T, V, D, dtype)
    words = torch.rand(B, T, generator=g) < 0.5                                 # half of them distributed like words
    likely = torch.floor(torch.exp(torch.rand(B, T, generator=g).double() * math.log(V + 1))).long() - 1
    tokens = torch.where(words.to(DEV), likely.clamp(0, V - 1).to(DEV), tokens)
    lengths = torch.randint(0, T + 1, (B,), generator=g).to(DEV)
    lengths[0] = T
    mask = torch.rand(B, T, generator=g) < 0.9
    valid = ref.valid_positions((B, T), lengths, mask)
    got = check_gradient(rows, tokens, V, valid, 3.0, lengths=lengths, mask=mask.to(DEV), dtype=out)
    again = tb.embedding_grad(rows, tokens, V, scale=3.0, lengths=lengths, mask=mask.to(DEV), dtype=out)
    assert torch.equal(got, again)
    everything = torch.ones(B, T, dtype=torch.bool)
    check_gradient(rows, tokens, V, everything, dtype=out)
    # added to what is there: rows of other tokens stay as they are, whatever they are
    at = tokens.cpu()[valid]
    there = torch.zeros(V, dtype=torch.bool)
    there[at] = True
    old = torch.randn(V, D, generator=g).to(out)
    old[~there] = math.nan
    held = old.to(DEV)
    same = tb.embedding_grad(rows, tokens, V, scale=3.0, lengths=lengths, mask=mask.to(DEV), out=held, accumulate=True)
    assert same is held
    grad, size, counts = plain.embedding_grad(rows, tokens, V, valid, 3.0)
    assert held.cpu()[~there].isnan().all()
    check_sums(held[there.to(DEV)], grad[there], size[there], counts[there], old[there])


@pytest.mark.parametrize("N", [1, 15, 16, 17, 4096, 65536, 65537, 70001])
def test_one_token_has_all_positions(N):
    D = 20
    _, _, rows, _ = inputs(N, 1, N, 1, D, torch.float32)
    for V, token in ((1, 0), (9, 8), (1000, 511), (50257, 50256)):
        tokens = torch.full((N,), token, device=DEV)
        got = check_gradient(rows[0], tokens, V, torch.ones(N, dtype=torch.bool))
        assert not got[:token].any() and not got[token + 1:].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [40, 70000])
def test_what_stands_at_other_positions_is_not_read(N, dtype):
    B, V, D = 4, 50, 24
    T = N // B
    table, tokens, rows, g = inputs(N, B, T, V, D, dtype)
    lengths = torch.tensor([T, 0, T // 2, 1], device=DEV, dtype=torch.int32)
    mask = (torch.rand(B, T, generator=g) < 0.7).to(DEV)
    dead = ~ref.valid_positions((B, T), lengths, mask).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kw = dict(lengths=lengths, mask=mask, status=status)
    want = tb.embedding(table, tokens, **kw), tb.embedding_grad(rows, tokens, V, **kw)
    ids, filled = tokens.clone(), rows.clone()
    ids[dead], filled[dead] = 1 << 40, math.nan
    assert torch.equal(tb.embedding(table, ids, **kw), want[0])
    assert torch.equal(tb.embedding_grad(filled, ids, V, **kw), want[1])
    assert int(status) == 0 and not want[0][dead].any() and torch.isfinite(want[1]).all()
    none = dict(kw, lengths=torch.zeros_like(lengths))
    assert not tb.embedding(table, tokens, **none).any() and not tb.embedding_grad(rows, tokens, V, **none).any()


@pytest.mark.parametrize("N", [12, 70000])
def test_wrong_tokens_and_lengths(N):
    B, V, D = 2, 30, 16
    T = N // B
    table, tokens, rows, _ = inputs(N, B, T, V, D, torch.float32)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    wrong = tokens.clone()
    wrong[0, 1], wrong[1, 0], wrong[1, T - 1] = -1, V, 1 << 40
    bad = wrong != tokens
    out = tb.embedding(table, wrong, status=status)
    assert int(status) == tb.TB_DEV_TOKEN_RANGE
    assert out[bad].isnan().all() and torch.equal(out[~bad], table[tokens][~bad])
    status.zero_()
    got = tb.embedding_grad(rows, wrong, V, status=status)
    assert int(status) == tb.TB_DEV_TOKEN_RANGE
    assert torch.equal(got, tb.embedding_grad(rows, tokens, V, mask=~bad))
    for f in (lambda **kw: tb.embedding(table, tokens, **kw), lambda **kw: tb.embedding_grad(rows, tokens, V, **kw)):
        status.zero_()
        long = f(lengths=torch.tensor([T + 1, -1], device=DEV, dtype=torch.int32), status=status)
        assert int(status) == tb.TB_DEV_LENGTH_RANGE
        assert torch.equal(long, f(lengths=torch.tensor([T, 0], device=DEV, dtype=torch.int32)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [5, 24, 129, 700])
def test_strides_and_alignments(D, dtype):
    """Tables, rows and gradients inside wider ones at every alignment, sequences behind positions, rows that are
    broadcast, packed positions."""
    B, T, V = 3, 5, 12
    table, tokens, rows, _ = inputs(D, B, T, V, D, dtype)
    want = tb.embedding(table, tokens), tb.embedding_grad(rows, tokens, V)
    for lo in (0, 1, 3, 8):
        wide = torch.full((V, D + 9), math.nan, dtype=dtype, device=DEV)
        wide[:, lo:lo + D] = table
        assert torch.equal(tb.embedding(wide[:, lo:lo + D], tokens), want[0])
        many = torch.full((B, T, D + 9), math.nan, dtype=dtype, device=DEV)
        many[..., lo:lo + D] = rows
        assert torch.equal(tb.embedding_grad(many[..., lo:lo + D], tokens, V), want[1])
        wide.fill_(7.0)
        tb.embedding_grad(rows, tokens, V, out=wide[:, lo:lo + D])
        assert torch.equal(wide[:, lo:lo + D], want[1]) and (wide[:, :lo] == 7).all() and (wide[:, lo + D:] == 7).all()
    turned = rows.transpose(0, 1).contiguous().transpose(0, 1)
    across = rows.transpose(1, 2).contiguous().transpose(1, 2)
    ids = tokens.t().contiguous().t()
    for y in (turned, across):
        assert torch.equal(tb.embedding_grad(y, ids, V), want[1])
    assert torch.equal(tb.embedding(table.t().contiguous().t(), ids), want[0])
    assert torch.equal(tb.embedding(table, tokens.flatten()), want[0].flatten(0, 1))
    packed = tb.embedding_grad(rows.flatten(0, 1), tokens.flatten(), V)
    assert torch.equal(packed, want[1])
    one = rows[:1, :1].expand(B, T, D)
    assert torch.equal(tb.embedding_grad(one, tokens, V), tb.embedding_grad(one.contiguous(), tokens, V))
    leaf = table.clone().requires_grad_()
    tb.embedding(leaf, tokens).sum().backward()                           # (a gradient of stride 0)
    counts = torch.bincount(tokens.flatten(), minlength=V).to(dtype)
    assert torch.equal(leaf.grad, counts.unsqueeze(-1).expand(V, D))
    assert torch.equal(tb.embedding(table[:, :1].expand(V, D), tokens), table[:, :1].expand(V, D)[tokens])


def test_gradient_against_differences():
    V, D = 6, 5
    table, tokens, rows, g = inputs(1, 2, 9, V, D, torch.float32)
    grad = tb.embedding_grad(rows, tokens, V, scale=1.5)
    step = torch.randn(V, D, generator=g).to(DEV)
    up, down = (((tb.embedding(table + h * step, tokens, scale=1.5).double()) * rows).sum() for h in (0.5, -0.5))
    size = float((tb.embedding(table, tokens, scale=1.5).double() * rows).abs().sum() + (grad.double() * step).abs().sum())
    assert abs(float(up - down) - float((grad.double() * step).sum())) <= 40 * U * size      # (linear: rounding is all)


def test_two_uses_of_a_table():
    """A table that is looked up twice and is the head, too: autograd adds the parts up, and so does accumulate."""
    V, D = 20, 16
    table, tokens, rows, g = inputs(2, 2, 6, V, D, torch.float32)
    leaf = table.clone().requires_grad_()
    x = tb.embedding(leaf, tokens, scale=4.0)
    y = tb.embedding(leaf, tokens.flip(1).int())
    logits = torch.tanh(x + y) @ leaf.t()
    loss = (tb.top_logprobs(logits, 3, tokens, want_entropy=True).token_logprobs * rows[..., 0]).sum()
    got, = torch.autograd.grad(loss, leaf)
    wide = table.cpu().double().requires_grad_()
    t = tokens.cpu()
    out = torch.log_softmax(torch.tanh(wide[t] * 4 + wide[t.flip(1)]) @ wide.t(), -1)
    want, = torch.autograd.grad((out.gather(-1, t.unsqueeze(-1)).squeeze(-1) * rows[..., 0].cpu().double()).sum(), wide)
    # float32 throughout: log-probabilities to 3e-5, products of 16 terms and sums of 12 positions
    assert (got.cpu().double() - want).abs().max() <= 12 * 3e-5 * (1 + want.abs().max())


def test_nothing_to_do():
    table = torch.randn(9, 4, device=DEV, requires_grad=True)
    for shape in ((0, 3), (3, 0), (0,)):
        tokens = torch.empty(shape, dtype=torch.int64, device=DEV)
        out = tb.embedding(table, tokens)
        assert out.shape == (*shape, 4)
        g = tb.embedding_grad(torch.empty(*shape, 4, device=DEV), tokens, 9)
        assert g.shape == (9, 4) and not g.any()
        held = torch.ones(9, 4, device=DEV)
        tb.embedding_grad(torch.empty(*shape, 4, device=DEV), tokens, 9, out=held, accumulate=True)
        assert (held == 1).all()
        grad, = torch.autograd.grad(out.sum(), table)
        assert not grad.any()


def test_refusals():
    table, tokens, rows, _ = inputs(3, 2, 3, 10, 8, torch.float32)
    E = tb.TensorBLEUError
    for f in (lambda: tb.embedding(table.double(), tokens), lambda: tb.embedding(table.cpu(), tokens),
              lambda: tb.embedding(table[0], tokens), lambda: tb.embedding(table, tokens.float()),
              lambda: tb.embedding(table, tokens.cpu()), lambda: tb.embedding(table, tokens.unsqueeze(0)),
              lambda: tb.embedding(table[:0], tokens), lambda: tb.embedding(table[:, :0], tokens),
              lambda: tb.embedding(table, tokens, lengths=torch.ones(3, device=DEV, dtype=torch.int32)),
              lambda: tb.embedding(table, tokens.flatten(), lengths=torch.ones(1, device=DEV, dtype=torch.int32)),
              lambda: tb.embedding(table, tokens, mask=torch.ones(2, 2, device=DEV, dtype=torch.bool)),
              lambda: tb.embedding(table, tokens, status=torch.zeros(1, device=DEV)),
              lambda: tb.embedding_grad(rows[:1], tokens, 10), lambda: tb.embedding_grad(rows, tokens, 0),
              lambda: tb.embedding_grad(rows, tokens, 10.0), lambda: tb.embedding_grad(rows, tokens, 10, dtype=torch.bfloat16),
              lambda: tb.embedding_grad(rows, tokens, 10, accumulate=True),
              lambda: tb.embedding_grad(rows, tokens, 10, out=table[:9].clone()),
              lambda: tb.embedding_grad(rows, tokens, 10, out=table.clone().requires_grad_()),
              lambda: tb.embedding_grad(rows, tokens, 10, out=table.clone().requires_grad_() * 2),
              lambda: tb.embedding_grad(rows.bfloat16(), tokens, 10, out=table.half()),
              lambda: tb.embedding_grad(rows, tokens, 6, out=rows.view(6, 8))):
        with pytest.raises(E):
            f()
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(table, torch.ones_like(table))
        with pytest.raises(E, match="tangent"):
            tb.embedding(dual, tokens)
    leaf = table.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="differentiated twice"):
        torch.autograd.grad(tb.embedding(leaf, tokens).sum(), leaf, create_graph=True)


def test_a_gradient_written_to_out_counts_as_a_change():
    table, tokens, rows, _ = inputs(3, 2, 3, 10, 8, torch.float32)
    leaf = torch.ones(10, 8, device=DEV, requires_grad=True)
    held = torch.ones(10, 8, device=DEV)
    loss = (leaf * held).sum()
    tb.embedding_grad(rows, tokens, 10, out=held)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_saved_tensor_hooks_and_changed_ids():
    table, tokens, rows, _ = inputs(5, 3, 4, 12, 24, torch.bfloat16)
    lengths = torch.tensor([4, 1, 3], device=DEV)
    want = tb.embedding_grad(rows, tokens, 12, lengths=lengths)
    leaf = table.clone().requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: t.to(DEV).t().contiguous().t() if t.dim() > 1 else t.to(DEV)):
        out = tb.embedding(leaf, tokens, lengths=lengths)
    assert torch.equal(torch.autograd.grad(out, leaf, rows)[0], want)
    out = torch.utils.checkpoint.checkpoint(lambda: tb.embedding(leaf, tokens, lengths=lengths.int()), use_reentrant=False)
    assert torch.equal(torch.autograd.grad(out, leaf, rows)[0], want)
    ids = tokens.clone()
    out = tb.embedding(leaf, ids)
    ids.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_two_streams_at_once():
    """Gradients of the same rows on several streams at the same time."""
    _, tokens, rows, _ = inputs(8, 3, 30000, 4000, 40, torch.bfloat16)
    want = tb.embedding_grad(rows, tokens, 4000), tb.embedding_grad(rows[:, :500], tokens[:, :500], 4000)
    torch.cuda.synchronize()
    streams, found = [torch.cuda.Stream() for _ in range(3)], []
    for i in range(9):
        with torch.cuda.stream(streams[i % 3]):
            found.append((tb.embedding_grad(rows, tokens, 4000), tb.embedding_grad(rows[:, :500], tokens[:, :500], 4000)))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for calls in found for a, b in zip(calls, want))


def test_wide_offsets():
    """A table and a gradient whose last values lie beyond 2^31 (and their bytes beyond 2^32)."""
    V, D = 280_000, 8192
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of the GPU's memory")
    table = torch.empty(V, D, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator().manual_seed(1)
    tokens = torch.tensor([V - 1, 0, V - 2, V - 1, 262145, V - 1], device=DEV)
    table[tokens] = torch.randn(6, D, generator=g).bfloat16().to(DEV)
    out = tb.embedding(table, tokens)
    assert torch.equal(out, table[tokens])
    grad = tb.embedding_grad(out, tokens, V, out=table)           # (over the table: its rows are not needed any more)
    rows, size, counts = plain.embedding_grad(out, torch.tensor([3, 0, 2, 3, 1, 3]), 4, torch.ones(6, dtype=torch.bool))
    check_sums(grad[[0, 262145, V - 2, V - 1]], rows, size, counts)
    assert not grad[1:262145].any() and not grad[262146:V - 2].any()


@pytest.mark.parametrize("N,V,D", [(14, 50, 24), (900, 40000, 33), (70000, 300, 20)])
def test_streams_and_graphs(N, V, D):
    """On a stream of its own; captured, forward and backward, and replayed with eager work between."""
    table, tokens, rows, g = inputs(N, 1, N, V, D, torch.bfloat16)
    others = [(torch.randint(0, V, (1, N), generator=g).to(DEV), torch.randn(1, N, D, generator=g).bfloat16().to(DEV)) for _ in range(3)]
    still = tokens.clone(), rows.clone()

    def step():
        leaf = table.detach().requires_grad_()
        out = tb.embedding(leaf, still[0], scale=2.0)
        return out.detach(), *torch.autograd.grad(out, leaf, still[1]), tb.embedding_grad(still[1], still[0], V, dtype=torch.float32)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        aside = step()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(a, b) for a, b in zip(aside, step()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for ids, r in others + others:
        still[0].copy_(ids)
        still[1].copy_(r)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


@pytest.mark.parametrize("lengths", [None, torch.int64])
def test_a_capture_beside_an_eager_graph(lengths):
    """A leaf that a graph from outside holds: the captured backward pass is refused; without that graph it runs."""
    table, tokens, rows, _ = inputs(6, 2, 30, 50, 24, torch.float32)
    leaf = table.clone().requires_grad_()
    where = {} if lengths is None else dict(lengths=torch.tensor([30, 11], device=DEV, dtype=lengths))
    held = tb.embedding(leaf, tokens, **where)
    want, = torch.autograd.grad(held, leaf, rows, retain_graph=True)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="outside the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            torch.autograd.grad(tb.embedding(leaf, tokens, **where), leaf, rows)
    del held
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, = torch.autograd.grad(tb.embedding(leaf, tokens, **where), leaf, rows)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
