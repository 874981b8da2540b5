"""Top log-probabilities over a vocabulary and embeddings of token ids, with their gradients, as cases
to be timed.

Both ends of a policy that is trained on rewards of its token ids.  A case is one call of one of these
operators on tensors that live on the GPU:

  top      log-probabilities of given tokens with the K likeliest alternatives of every position (what a
           server returns, or a teacher leaves for a distillation), with the entropy and the gradient where
           asked for
  lookup   rows of an embedding table by token ids, scaled
  grad     the gradient of such a lookup in the table, all of its rows
  train    both through autograd, as a training step runs them

Fields of a case
  B, T, V      sequences, positions of each, vocabulary
  packed       positions are [T] (B is 1) with a mask instead of lengths
  dtype, ids   types of logits, tables and gradients, and of token ids
  low          lengths are uniform in [low * T, T]; 1.0: every position counts
  K            top: alternatives
  temperature  top: divides the logits
  tokens       top: log-probabilities of given tokens come along
  entropy      top: entropies come along
  backward     top: the gradient of given cotangents comes along
  D            width of the table
  scale        of the embeddings
  zipf         token ids are distributed like words (the i-th likeliest has a share of 1 / i), else uniformly

With `own` set, run() calls the framework's operators, otherwise it computes them from elementary
operations in 32 bits.
"""
import math

import torch

DEVICE = "cuda:0"
own = False

DEFAULTS = dict(B=16, T=256, V=32000, packed=False, dtype="bfloat16", ids="int64", low=0.5, K=0, temperature=1.0,
                tokens=False, entropy=False, backward=False, D=0, scale=1.0, zipf=True)


def _case(op, name=None, **kw):
    case = dict(DEFAULTS, op=op, **kw)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # serving: a sampled token's log-probability and the 20 likeliest of its position
        _case("top", "top_1x1_v50257_k20", B=1, T=1, V=50257, K=20, low=1.0, tokens=True),
        # four sequences served together over a large vocabulary (benchmark configuration 4's), in float32
        _case("top", "top_4x1_v262144_k8_f32", B=4, T=1, V=262144, K=8, low=1.0, dtype="float32", temperature=0.7,
              tokens=True, entropy=True),
        # a teacher's 64 best for a distillation of one prompt's rollouts (benchmark configuration 1)
        _case("top", "top_16x256_v32000_k64", K=64),
        # many ragged sequences over a tiny vocabulary (benchmark configuration 5)
        _case("top", "top_4096x512_v64_k5", B=4096, T=512, V=64, K=5, ids="int32", low=0.06, tokens=True),
        # packed positions over a large vocabulary, many alternatives
        _case("top", "top_2047_v262144_k256_f16", B=1, T=2047, V=262144, packed=True, K=256, low=0.8,
              dtype="float16"),
        # an auxiliary loss on alternatives, log-probabilities and entropies, in float32
        _case("top", "top_train_8x511_v50257_k20_f32", B=8, T=511, V=50257, K=20, dtype="float32", low=0.9,
              tokens=True, entropy=True, backward=True),
        # the largest: statistics of a whole batch of rollouts
        _case("top", "top_16x1024_v50257_k20", B=16, T=1024, V=50257, K=20, low=0.25, tokens=True, entropy=True),
        # serving: the embedding of one token
        _case("lookup", "lookup_1x1_v50257_d768", B=1, T=1, V=50257, D=768, low=1.0, scale=768 ** 0.5),
        # the policy's own forward pass over a batch of rollouts
        _case("lookup", "lookup_32x1024_v50257_d2048", B=32, T=1024, V=50257, D=2048, low=0.25, scale=2048 ** 0.5),
        # one micro-batch in float32: lookup and gradient
        _case("train", "train_16x256_v32000_d1024_f32", D=1024, dtype="float32", scale=32.0),
        # the gradient of a batch of rollouts
        _case("grad", "grad_32x1024_v50257_d2048", B=32, T=1024, V=50257, D=2048, low=0.25, scale=2048 ** 0.5),
        # two million positions of a tiny vocabulary (benchmark configuration 5)
        _case("grad", "grad_4096x512_v64_d64", B=4096, T=512, V=64, D=64, ids="int32", low=0.06, zipf=False),
    ]


MOST = 3 << 29          # bytes that a drawn case may read and write


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["top", "top", "top", "lookup", "grad", "grad", "train"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    size = 4 if dtype == "float32" else 2
    case = _case(op, dtype=dtype, ids=rng.choice(["int32", "int64"]), low=rng.choice([1.0, 0.9, 0.5, 0.1]),
                 V=_log_int(rng, 64, 262144))
    if op == "top":
        case["tokens"], case["entropy"] = rng.random() < 0.6, rng.random() < 0.4
        case["backward"], case["temperature"] = rng.random() < 0.3, rng.choice([1.0, 1.0, 0.7, 2.0])
        case["K"] = _log_int(rng, 1, min(case["V"], 256))
        row = case["V"] * size * (3 if case["backward"] else 1) + 12 * case["K"]
    else:
        case["D"], case["zipf"] = _log_int(rng, 16, 8192), rng.random() < 0.7
        if case["V"] * case["D"] * size > MOST // 4:
            case["V"] = max(64, MOST // 4 // (case["D"] * size))
        case["scale"] = rng.choice([1.0, case["D"] ** 0.5])
        row = case["D"] * size * (3 if op == "train" else 2)
    rows = _log_int(rng, 1, max(1, min(1 << 20, MOST // 2 // row)))
    T = _log_int(rng, 1, max(1, min(2048, rows)))
    case["B"], case["T"] = max(1, rows // T), T
    if rng.random() < 0.3:
        case["B"], case["T"], case["packed"] = 1, case["B"] * T, True
    return case


def _zipf(shape, V, gen):
    """Token ids whose i-th likeliest has a share of 1 / i."""
    share = 1.0 / torch.arange(1, V + 1, dtype=torch.float64, device=DEVICE)
    edges = share.cumsum(0)
    u = torch.rand(*shape, generator=gen, device=DEVICE, dtype=torch.float64) * edges[-1]
    return torch.searchsorted(edges, u).clamp(max=V - 1)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) * 1_000_003 + 31)
    B, T, V, D, dtype = case["B"], case["T"], case["V"], case["D"], getattr(torch, case["dtype"])

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE)

    s = {"case": case, "lengths": None, "mask": None}
    if case["packed"]:
        s["mask"] = torch.rand(T, generator=gen, device=DEVICE) < (1 + case["low"]) / 2
    elif case["low"] < 1:
        s["lengths"] = torch.randint(max(1, int(case["low"] * T)), T + 1, (B,), generator=gen, device=DEVICE,
                                     dtype=torch.int32)
    if case["op"] == "top":
        # a model's logits: a broad floor, and the sampled tokens from there up to where half of the
        # probability is
        logits = torch.empty(B, T, V, dtype=dtype, device=DEVICE)
        logits.normal_(0.0, 2.5, generator=gen)
        tokens = torch.randint(0, V, (B, T), generator=gen, device=DEVICE)
        most = case["temperature"] * (math.log(V) + 3.1 / case["temperature"] ** 2)
        high = most * torch.rand(B, T, 1, generator=gen, device=DEVICE)
        logits.scatter_(-1, tokens.unsqueeze(-1), high.to(dtype))
        if case["backward"]:
            s["d_top"], s["d_logprobs"], s["d_entropy"] = normal(B, T, case["K"]), normal(B, T), normal(B, T)
        s["logits"] = logits
    else:
        tokens = _zipf((B, T), V, gen) if case["zipf"] else torch.randint(0, V, (B, T), generator=gen, device=DEVICE)
        if case["op"] != "grad":
            s["table"] = (0.02 * normal(V, D)).to(dtype)
        if case["op"] != "lookup":
            s["d_rows"] = torch.empty(B, T, D, dtype=dtype, device=DEVICE).normal_(0.0, 0.01, generator=gen)
    s["tokens"] = tokens.to(getattr(torch, case["ids"]))
    if case["packed"]:
        s.update({k: s[k][0] for k in ("logits", "tokens", "d_top", "d_logprobs", "d_entropy", "d_rows") if k in s})
    return s


def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _run_own(s, case):
    import paper_2510_05485_amd as tb
    where = dict(lengths=s["lengths"], mask=s["mask"])
    if case["op"] == "lookup":
        return tb.embedding(s["table"], s["tokens"], scale=case["scale"], **where)
    if case["op"] == "grad":
        return tb.embedding_grad(s["d_rows"], s["tokens"], case["V"], scale=case["scale"], **where)
    if case["op"] == "train":
        table = s["table"].detach().requires_grad_()
        out = tb.embedding(table, s["tokens"], scale=case["scale"], **where)
        return [out.detach(), *torch.autograd.grad(out, table, s["d_rows"])]
    x = s["logits"].detach().requires_grad_() if case["backward"] else s["logits"]
    r = tb.top_logprobs(x, case["K"], s["tokens"] if case["tokens"] else None, temperature=case["temperature"],
                        want_entropy=case["entropy"], **where)
    values, given = [r.logprobs], [s["d_top"]] if case["backward"] else []
    if case["tokens"]:
        values.append(r.token_logprobs)
        given += [s["d_logprobs"]] if case["backward"] else []
    if case["entropy"]:
        values.append(r.entropy)
        given += [s["d_entropy"]] if case["backward"] else []
    if not case["backward"]:
        return [r.ids, *values]
    return [r.ids, *(v.detach() for v in values), *torch.autograd.grad(values, x, given)]


def _valid(s, case):
    """Which positions count, of the tokens' shape."""
    if s["mask"] is not None:
        return s["mask"]
    if s["lengths"] is not None:
        return torch.arange(case["T"], device=DEVICE) < s["lengths"].unsqueeze(-1)
    return torch.ones(s["tokens"].shape, dtype=torch.bool, device=DEVICE)


def _table_gradient(s, case, valid):
    """Sums over equal tokens; of few tokens with many positions as products, part by part, with the matrix
    that says which position holds which token."""
    V, D = case["V"], case["D"]
    at, rows = s["tokens"][valid].long(), s["d_rows"][valid].float()
    if V * at.numel() <= 1 << 29 and at.numel() >= 16 * V:
        part = 4096
        more = -at.numel() % part
        at = torch.nn.functional.pad(at, (0, more), value=-1).reshape(-1, 1, part)
        rows = torch.nn.functional.pad(rows, (0, 0, 0, more)).reshape(-1, part, D)
        grad = torch.bmm((at == torch.arange(V, device=DEVICE).unsqueeze(-1)).float(), rows).sum(0)
    else:
        grad = torch.zeros(V, D, device=DEVICE).index_add_(0, at, rows)
    return (grad * case["scale"]).to(s["d_rows"].dtype)


def _run_plain(s, case):
    valid = _valid(s, case)
    if case["op"] == "grad":
        return _table_gradient(s, case, valid)
    zero = torch.zeros((), device=DEVICE)
    if case["op"] in ("lookup", "train"):
        rows = s["table"][s["tokens"].long()].float() * case["scale"]
        out = torch.where(valid.unsqueeze(-1), rows, zero).to(s["table"].dtype)
        return out if case["op"] == "lookup" else [out, _table_gradient(s, case, valid)]

    # the order of the logits as one of whole numbers: by value, equal ones by their places
    V, K = case["V"], case["K"]
    bits = (s["logits"].float() + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * V + torch.arange(V - 1, -1, -1, device=DEVICE)
    ids = V - 1 - order.topk(K).values % V
    del bits, order
    z = s["logits"].float() / case["temperature"]
    z = z - z.amax(-1, keepdim=True)
    e = z.exp()
    total = e.sum(-1, keepdim=True)
    log_total = total.log()
    at = valid.unsqueeze(-1)
    out = [torch.where(at, ids, -1), torch.where(at, z.gather(-1, ids) - log_total, -math.inf)]
    tokens = s["tokens"].long().unsqueeze(-1)
    if case["tokens"]:
        out.append(torch.where(valid, (z.gather(-1, tokens) - log_total).squeeze(-1), zero))
    p = e / total
    if case["entropy"]:
        entropy = log_total.squeeze(-1) - (p * z).sum(-1)
        out.append(torch.where(valid, entropy, zero))
    if case["backward"]:
        weight = s["d_top"].sum(-1, keepdim=True)
        if case["tokens"]:
            weight = weight + s["d_logprobs"].unsqueeze(-1)
        if case["entropy"]:
            weight = weight + s["d_entropy"].unsqueeze(-1) * (z - (log_total - entropy.unsqueeze(-1)))
        grad = -p * weight
        grad.scatter_add_(-1, ids, s["d_top"])
        if case["tokens"]:
            grad.scatter_add_(-1, tokens, s["d_logprobs"].unsqueeze(-1))
        out.append(torch.where(at, grad / case["temperature"], zero).to(s["logits"].dtype))
    return out


def exact(case, seed):
    """The definitions in 64 bits, some rows at a time; a table's gradient by
    sorted tokens, as differences of running sums."""
    s = prepare(case, seed)
    N, V, D, K = case["B"] * case["T"], case["V"], case["D"], case["K"]
    count = torch.ones(N, dtype=torch.bool, device=DEVICE)
    if case["packed"]:
        count = s["mask"].clone()
    elif s["lengths"] is not None:
        place = torch.arange(N, device=DEVICE)
        count = place % case["T"] < s["lengths"].long().repeat_interleave(case["T"])
    tokens = s["tokens"].reshape(N).long()

    if case["op"] != "top":
        out = []
        if case["op"] != "grad":
            rows = torch.zeros(N, D, dtype=torch.float64, device=DEVICE)
            rows[count] = s["table"].double().index_select(0, tokens[count]) * case["scale"]
            out.append(rows.reshape(*s["tokens"].shape, D))
        if case["op"] != "lookup":
            which, order = tokens[count].sort()
            rows = s["d_rows"].reshape(N, D)[count][order].double()
            ends = torch.searchsorted(which, torch.arange(V, device=DEVICE), right=True)
            sums = torch.zeros(V, D, dtype=torch.float64, device=DEVICE)
            step = max(1, (1 << 27) // max(1, rows.shape[0]))
            for d in range(0, D, step):
                running = torch.nn.functional.pad(rows[:, d:d + step].t().contiguous().cumsum(1), (1, 0))
                sums[:, d:d + step] = running[:, ends].diff(dim=1, prepend=running[:, :1]).t()
            out.append(sums * case["scale"])
        return out if case["op"] == "train" else out[0]

    x = s["logits"].reshape(N, V)
    step = max(1, (1 << 27) // V)
    parts = []
    for i in range(0, N, step):
        values, held = x[i:i + step].double(), count[i:i + step]
        least = values.topk(K).values[:, -1:]
        above, equal = values > least, values == least
        taken = above | (equal & (equal.cumsum(1) <= K - above.sum(1, keepdim=True)))
        ids = taken.nonzero()[:, 1].reshape(-1, K)                 # by place, then by value
        ids = ids.gather(1, values.gather(1, ids).sort(dim=1, descending=True, stable=True).indices)
        values.requires_grad_(case["backward"])
        lp = torch.log_softmax(values / case["temperature"], 1)
        found = [lp.gather(1, ids)]
        if case["tokens"]:
            found.append(lp.gather(1, tokens[i:i + step, None]).squeeze(1))
        if case["entropy"]:
            found.append(-(lp.exp() * lp).sum(1))
        row = [ids.masked_fill(~held[:, None], -1), found[0].detach().masked_fill(~held[:, None], -math.inf)]
        row += [f.detach().masked_fill(~held, 0.0) for f in found[1:]]
        if case["backward"]:
            given = [s["d_top"].reshape(N, K)]
            given += [s["d_logprobs"].reshape(N)] if case["tokens"] else []
            given += [s["d_entropy"].reshape(N)] if case["entropy"] else []
            loss = 0.0
            for f, d in zip(found, given):
                each = f * d[i:i + step].double()
                loss = loss + (each.sum(1) if each.dim() == 2 else each)
            grad, = torch.autograd.grad((loss * held).sum(), values)
            row.append(grad)
        parts.append(row)
    shape = tuple(s["tokens"].shape)
    return [torch.cat(p).reshape(shape + p[0].shape[1:]) for p in zip(*parts)]


def _rows_touched(case, n):
    """Expected rows of the table that n positions read."""
    if not case["zipf"]:
        return case["V"] * -math.expm1(n * math.log1p(-1.0 / case["V"]))
    share = 1.0 / torch.arange(1, case["V"] + 1, dtype=torch.float64)
    return float(-torch.expm1(n * torch.log1p(-share / (share.sum() + 1e-9))).sum())


def work(case):
    """Logits of the positions that count (expected lengths) and rows of the table that are looked up read
    once; embeddings, gradients of all positions and of the whole table written once; ids and values of
    each position; some operations a value."""
    N, V, D, K = case["B"] * case["T"], case["V"], case["D"], case["K"]
    low = (1 + case["low"]) / 2 if case["packed"] else (max(1, int(case["low"] * case["T"])) + case["T"]) / 2 / case["T"]
    if case["low"] >= 1:
        low = 1.0
    size, id_size = 4 if case["dtype"] == "float32" else 2, 8 if case["ids"] == "int64" else 4
    if case["op"] == "top":
        moved = low * N * V * size + N * K * 12 + N * 4 * (case["tokens"] + case["entropy"])
        moved += low * N * id_size * case["tokens"]
        if case["backward"]:
            moved += N * V * size + low * N * 4 * (K + case["tokens"] + case["entropy"])
        return {"bytes": moved, "flops": low * N * V * (10 if case["backward"] else 5)}
    moved, ops = low * N * id_size, 0
    if case["op"] != "grad":
        moved += (_rows_touched(case, low * N) + N) * D * size
        ops += low * N * D
    if case["op"] != "lookup":
        moved += (low * N + V) * D * size
        ops += low * N * D
    return {"bytes": moved, "flops": ops}
