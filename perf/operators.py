"""Losses over a policy's logits with their gradients, as cases to be timed.

A training loop that rewards sampled sequences goes on from the rewards to a loss over the logits of
the model that it trains.  A case is one call of one of these operators on logits that live on the GPU:

  score     log-probabilities of given tokens (of the sampling or reference model), with the entropy
            and the gradient where asked for
  policy    the clipped policy loss with a KL term against a reference and an entropy bonus
  prefer    the loss of paired log ratios: the first half of the sequences is chosen, the second rejected
  distill   Kullback-Leibler divergence from a teacher's K top logits

Fields of a case
  B, T, V      sequences, positions of each, vocabulary; logits are [B, T, V]
  packed       logits are [T, V] (B is 1) with a mask over the positions instead of lengths
  shifted      logits and tokens are views [:, :-1] and [:, 1:] of a model's output and its input ids
  dtype, ids   types of logits (and gradient) and of token ids
  low          lengths are uniform in [low * T, T]; 1.0: every position counts
  temperature  divides the logits
  entropy      entropies come along (score) or enter with a coefficient (policy)
  backward     score: the gradient of given cotangents comes along
  kl           coefficient of the KL term; 0 for none (no reference log-probabilities)
  each         advantages are given for every position, not for every sequence
  average      "token", "sequence" or "sum"
  kind         prefer: "sigmoid", "hinge" or "ipo"; smooth: label smoothing
  K, counts    distill: entries of the teacher a position; counts: 1 to K of them, the others -inf

With `own` set, run() calls the framework's operators, otherwise it computes them from elementary
operations in 32 bits.
"""
import math

import torch

DEVICE = "cuda:0"
own = False

BETA = {"sigmoid": 0.1, "hinge": 0.1, "ipo": 0.5}
CLIP_LOW, CLIP_HIGH = 0.2, 0.25
ENTROPY = 0.01          # coefficient of the entropy bonus
SCALE = {"float16": 4096.0, "bfloat16": 1.0, "float32": 1.0}   # of gradients that leave in this type

DEFAULTS = dict(B=16, T=256, V=32000, packed=False, shifted=False, dtype="bfloat16", ids="int64",
                low=0.5, temperature=1.0, entropy=False, backward=False, kl=0.0, each=False,
                average="token", kind="sigmoid", smooth=0.0, K=0, counts=False)


def _case(op, name=None, **kw):
    case = dict(DEFAULTS, op=op, **kw)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # serving: the log-probability of one sampled token
        _case("score", "score_1x1_v50257", B=1, T=1, V=50257, low=1.0),
        # the reference model's log-probabilities of one prompt's rollouts (benchmark configuration 1)
        _case("score", "score_16x256_v32000"),
        # an auxiliary loss written by the user on log-probabilities and entropies, in float32, on
        # logits shifted against the ids
        _case("score", "logprobs_train_8x511_v50257_f32", B=8, T=511, V=50257, dtype="float32",
              shifted=True, entropy=True, backward=True, low=0.9),
        # one micro-batch of short answers: latency counts
        _case("policy", "policy_16x32_v32000", T=32, kl=0.04),
        # many ragged sequences over a tiny vocabulary (benchmark configuration 5)
        _case("policy", "policy_4096x512_v64", B=4096, T=512, V=64, ids="int32", low=0.06,
              average="sequence", each=True),
        # the largest: a whole policy step with KL and entropy terms
        _case("policy", "policy_32x1024_v50257", B=32, T=1024, V=50257, low=0.25, kl=0.04, entropy=True),
        # two pairs of short answers
        _case("prefer", "prefer_4x64_v32000_f16", B=4, T=64, dtype="float16"),
        # a batch of sixteen pairs, smoothed labels
        _case("prefer", "prefer_32x512_v50257", B=32, T=512, V=50257, low=0.3, smooth=0.1),
        # two long pairs over a large vocabulary (benchmark configuration 4's)
        _case("prefer", "prefer_4x1024_v262144_ipo", B=4, T=1024, V=262144, low=0.8, kind="ipo"),
        # online distillation of a few positions, in float32
        _case("distill", "distill_17_v50257_k8_f32", B=1, T=17, V=50257, packed=True, dtype="float32",
              low=1.0, K=8),
        # a batch of answers against the teacher's 64 best, softened
        _case("distill", "distill_16x256_v32000_k64", temperature=2.0, K=64),
        # packed positions over a large vocabulary, ragged entries
        _case("distill", "distill_2047_v262144_k256", B=1, T=2047, V=262144, packed=True, low=0.8, K=256,
              counts=True, ids="int32"),
    ]


MOST = 1 << 30          # logits of a drawn case


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["score", "score", "policy", "policy", "prefer", "distill"])
    V = _log_int(rng, 64, 262144)
    rows = _log_int(rng, 1, max(1, min(1 << 20, MOST // V)))
    T = _log_int(rng, 1, max(1, min(2048, rows)))
    case = _case(op, B=max(1, rows // T), T=T, V=V,
                 dtype=rng.choice(["bfloat16", "bfloat16", "float16", "float32"]),
                 ids=rng.choice(["int32", "int64"]), low=rng.choice([1.0, 0.9, 0.5, 0.1]),
                 temperature=rng.choice([1.0, 1.0, 0.7, 2.0]), shifted=rng.random() < 0.3)
    if op == "score":
        case["entropy"], case["backward"] = rng.random() < 0.4, rng.random() < 0.4
    if op == "policy":
        case["entropy"], case["kl"] = rng.random() < 0.4, rng.choice([0.0, 0.04, 0.1])
        case["each"], case["average"] = rng.random() < 0.5, rng.choice(["token", "token", "sequence", "sum"])
    if op == "prefer":
        case["B"] = max(2, case["B"] // 2 * 2)
        case["T"] = max(8, min(case["T"], MOST // (case["B"] * V)))
        case["kind"], case["smooth"] = rng.choice([("sigmoid", 0.0), ("sigmoid", 0.1), ("hinge", 0.0), ("ipo", 0.0)])
    if op == "distill":
        case["K"], case["counts"] = _log_int(rng, 1, min(V, 256)), rng.random() < 0.4
        case["average"] = rng.choice(["token", "sequence", "sum"])
        if rng.random() < 0.4:
            case["B"], case["T"], case["packed"], case["shifted"] = 1, case["B"] * case["T"], True, False
    return case


def _chosen(logits, tokens, temperature):
    """Log-probabilities of the tokens, some rows at a time."""
    B, T, V = logits.shape
    out = torch.empty(B, T, device=logits.device)
    step = max(1, (1 << 27) // V)
    for b in range(B):
        for t in range(0, T, step):
            z = logits[b, t:t + step].float() / temperature
            out[b, t:t + step] = z.gather(-1, tokens[b, t:t + step].long().unsqueeze(-1)).squeeze(-1) - z.logsumexp(-1)
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) * 1_000_003 + 29)
    B, T, V, dtype = case["B"], case["T"], case["V"], getattr(torch, case["dtype"])

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=DEVICE)

    more = 1 if case["shifted"] else 0
    s = {"case": case}
    # a model's logits: a broad floor, and the sampled tokens from there up to where half of the
    # probability is
    logits = torch.empty(B, T + more, V, dtype=dtype, device=DEVICE)
    logits.normal_(0.0, 2.5, generator=gen)
    ids = torch.randint(0, V, (B, T + more), generator=gen, device=DEVICE)
    tokens = ids[:, more:]
    view = logits[:, :T]
    at = tokens.unsqueeze(-1)
    top = case["temperature"] * (math.log(V) + 3.1 / case["temperature"] ** 2)
    view.scatter_(-1, at, (top * uniform(B, T, 1)).to(dtype))
    s["lengths"], s["mask"] = None, None
    if case["packed"]:
        s["mask"] = uniform(T) < (1 + case["low"]) / 2 if case["low"] < 1 else torch.ones(T, dtype=torch.bool, device=DEVICE)
    elif case["low"] < 1:
        s["lengths"] = torch.randint(max(1, int(case["low"] * T)), T + 1, (B,), generator=gen, device=DEVICE,
                                     dtype=torch.int32)
    if case["op"] == "score" and case["backward"]:
        s["d_logprobs"], s["d_entropy"] = normal(B, T), normal(B, T) if case["entropy"] else None
    if case["op"] == "policy":
        lp = _chosen(view, tokens, case["temperature"])
        # the sampling policy is a little older than the one that is trained.  No ratio lies on the
        # edge of the clip range, where the last bit would decide whether a position has a gradient
        d = 0.1 * normal(B, T)
        edge = ((-d).exp() / (1 + CLIP_HIGH) - 1).abs().minimum(((-d).exp() / (1 - CLIP_LOW) - 1).abs()) < 1e-3
        s["old"] = lp + torch.where(edge, torch.zeros_like(d), d)
        s["ref"] = lp + 0.2 * normal(B, T) if case["kl"] else None
        s["advantages"] = normal(B, T) if case["each"] else normal(B)
    if case["op"] == "prefer":
        # the trained model has moved away from the reference, towards the chosen sequences
        moved = 0.4 / T ** 0.5 * torch.where(torch.arange(B, device=DEVICE) < B // 2, 1.0, -1.0).unsqueeze(-1)
        s["ref"] = _chosen(view, tokens, case["temperature"]) + 0.2 * normal(B, T) - moved
    if case["op"] == "distill":
        K = case["K"]
        stride = next(p for p in (7919, 7907, 7901) if V % p)   # no two entries of a row are alike
        first = torch.randint(0, V, (B, T, 1), generator=gen, device=DEVICE)
        at = (first + stride * torch.arange(K, device=DEVICE)) % V
        best = (3 * normal(B, T, K)).sort(-1, descending=True).values
        view.scatter_(-1, at, (view.gather(-1, at).float() + 5 + 0.7 * best).to(dtype))
        if case["counts"]:
            none = torch.arange(K, device=DEVICE) >= torch.randint(1, K + 1, (B, T, 1), generator=gen, device=DEVICE)
            best, at = best.masked_fill(none, float("-inf")), at.masked_fill(none, -1)
        at, best = at.to(getattr(torch, case["ids"])), best.to(dtype)
        s["teacher_ids"], s["teacher_logits"] = (at[0], best[0]) if case["packed"] else (at, best)
    ids = ids.to(getattr(torch, case["ids"]))
    s["logits"], s["tokens"] = (view[0], ids[0]) if case["packed"] else (view, ids[:, more:])
    return s


def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _run_own(s, case):
    import paper_2510_05485_amd as tb
    where = dict(lengths=s["lengths"], mask=s["mask"], temperature=case["temperature"])
    if case["op"] != "score":
        where["grad_scale"] = SCALE[case["dtype"]]
    if case["op"] == "score":
        x = s["logits"].detach().requires_grad_() if case["backward"] else s["logits"]
        out = tb.token_logprobs(x, s["tokens"], want_entropy=case["entropy"], **where)
        if not case["backward"]:
            return out
        if case["entropy"]:
            return [*out, *torch.autograd.grad(out, x, (s["d_logprobs"], s["d_entropy"]))]
        return [out, *torch.autograd.grad(out, x, s["d_logprobs"])]
    if case["op"] == "policy":
        r = tb.policy_loss_grad(s["logits"], s["tokens"], s["old"], s["advantages"], ref_logprobs=s["ref"],
                                clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=case["kl"],
                                entropy_coef=ENTROPY if case["entropy"] else 0.0, average=case["average"], **where)
        return [r.terms, r.grad, r.logprobs]
    if case["op"] == "prefer":
        r = tb.preference_loss_grad(s["logits"], s["tokens"], s["ref"], beta=BETA[case["kind"]], kind=case["kind"],
                                    label_smoothing=case["smooth"], **where)
        return [r.terms, r.grad, r.sequence_logprobs, r.margins]
    r = tb.distillation_loss_grad(s["logits"], s["teacher_ids"], s["teacher_logits"], average=case["average"], **where)
    return [r.terms, r.grad, r.row_loss]


def _valid(s, case):
    """Which positions count, [B, T], and how many of each sequence."""
    if s["mask"] is not None:
        valid = s["mask"].reshape(1, -1)
    elif s["lengths"] is not None:
        valid = torch.arange(case["T"], device=DEVICE) < s["lengths"].unsqueeze(-1)
    else:
        valid = torch.ones(case["B"], case["T"], dtype=torch.bool, device=DEVICE)
    return valid, valid.sum(-1, keepdim=True)


def _weights(valid, counts, average):
    w = valid.float()
    if average == "token":
        return w / counts.sum().clamp(min=1)
    if average == "sequence":
        return w / (counts.clamp(min=1) * (counts > 0).sum().clamp(min=1))
    return w


def _softmax(logits, temperature):
    """(z, log s, p): logits over the temperature less their maximum, the logarithm of the sum of the
    exponentials of these, and probabilities; all in 32 bits."""
    z = logits.float() / temperature
    z = z - z.amax(-1, keepdim=True)
    e = z.exp()
    total = e.sum(-1, keepdim=True)
    return z, total.log(), e / total


def _run_plain(s, case):
    B, T, V, c = case["B"], case["T"], case["V"], 1.0 / case["temperature"]
    logits = s["logits"].reshape(1, T, V) if case["packed"] else s["logits"]
    valid, counts = _valid(s, case)
    w = _weights(valid, counts, case["average"])
    zero = torch.zeros((), device=DEVICE)
    z, log_total, p = _softmax(logits, case["temperature"])
    log_total = log_total.squeeze(-1)

    scale = 1.0 if case["op"] == "score" else SCALE[case["dtype"]]

    def back(grad):
        grad = torch.where(valid.unsqueeze(-1), grad, zero).to(logits.dtype)
        return grad.reshape(s["logits"].shape)

    if case["op"] == "distill":
        K = case["K"]
        ids = s["teacher_ids"].reshape(B, T, K).long().clamp(min=0)
        zt, log_qt, q = _softmax(s["teacher_logits"].reshape(B, T, K), case["temperature"])
        kl = torch.where(q > 0, q * ((zt - log_qt) - (z.gather(-1, ids) - log_total.unsqueeze(-1))), zero).sum(-1)
        rows = torch.where(valid, kl * case["temperature"] ** 2, zero)
        grad = p.scatter_add(-1, ids, -q) * (w * (case["temperature"] * scale)).unsqueeze(-1)
        return [(rows * w).sum().reshape(1), back(grad), rows.reshape(s["logits"].shape[:-1])]

    tokens = s["tokens"].reshape(B, T).long().unsqueeze(-1)
    lp = z.gather(-1, tokens).squeeze(-1) - log_total
    entropy = log_total - (p * z).sum(-1) if case["entropy"] else None

    def gradient(d_lp, d_entropy):
        grad = -p * d_lp.unsqueeze(-1)
        grad.scatter_add_(-1, tokens, d_lp.unsqueeze(-1))
        if d_entropy is not None:
            grad -= p * (z - (log_total - entropy).unsqueeze(-1)) * d_entropy.unsqueeze(-1)
        return back(grad * (c * scale))

    if case["op"] == "score":
        out = [torch.where(valid, lp, zero).reshape(s["tokens"].shape)]
        if case["entropy"]:
            out.append(torch.where(valid, entropy, zero).reshape(s["tokens"].shape))
        if case["backward"]:
            out.append(gradient(s["d_logprobs"], s["d_entropy"]))
        return out if len(out) > 1 else out[0]

    if case["op"] == "policy":
        advantages = s["advantages"] if case["each"] else s["advantages"].unsqueeze(-1)
        ratio = (lp - s["old"]).exp()
        gain = torch.minimum(ratio * advantages, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * advantages)
        clipped = ((advantages > 0) & (ratio > 1 + CLIP_HIGH)) | ((advantages < 0) & (ratio < 1 - CLIP_LOW))
        loss, d_lp = -gain, torch.where(clipped, zero, -ratio * advantages)
        kl = zero
        if case["kl"]:
            r = s["ref"] - lp
            kl = r.exp() - r - 1
            loss, d_lp = loss + case["kl"] * kl, d_lp + case["kl"] * (1 - r.exp())
        d_entropy = None
        if case["entropy"]:
            loss, d_entropy = loss - ENTROPY * entropy, -ENTROPY * w
        terms = [(x * w).sum() for x in (loss, kl, clipped.float(), entropy if case["entropy"] else zero)]
        return [torch.stack(terms), gradient(d_lp * w, d_entropy), torch.where(valid, lp, zero)]

    lp = torch.where(valid, lp, zero)
    ratios = torch.where(valid, lp - s["ref"], zero).sum(-1)
    share = torch.ones(B, device=DEVICE)
    if case["kind"] == "ipo":
        share = 1.0 / counts.squeeze(-1).clamp(min=1)
    pairs, beta = B // 2, BETA[case["kind"]]
    d = ratios * share
    margins = d[:pairs] - d[pairs:]
    h = beta * margins
    if case["kind"] == "ipo":
        off = margins - 0.5 / beta
        losses, d_margin = off * off, 2 * off
    elif case["kind"] == "hinge":
        losses, d_margin = (1 - h).clamp(min=0), torch.where(h < 1, -beta, 0.0)
    else:
        e = case["smooth"]
        low = torch.log1p((-h.abs()).exp())               # softplus(-h) and softplus(h) without overflow
        losses = (1 - e) * (low + (-h).clamp(min=0)) + e * (low + h.clamp(min=0))
        d_margin = beta * (e / (1 + (-h).exp()) - (1 - e) / (1 + h.exp()))
    d_sequence = torch.cat([d_margin, -d_margin]) * share / pairs
    terms = torch.stack([losses.mean(), (margins > 0).float().mean(), margins.mean()])
    return [terms, gradient(torch.where(valid, d_sequence.unsqueeze(-1), zero), None), lp.sum(-1), margins]


def exact(case, seed):
    """The definitions in 64 bits, the gradients by differentiation of the definition: of the loss
    with respect to the log-probabilities, then of these with respect to the logits, rows by rows."""
    s = prepare(case, seed)
    V, tau = case["V"], case["temperature"]
    rows = s["logits"].reshape(-1, V) if s["logits"].is_contiguous() else s["logits"].flatten(0, 1)
    N = rows.shape[0]
    step = max(1, (1 << 27) // V)
    if s["mask"] is not None:
        valid = s["mask"].reshape(1, N)
    else:
        n = s["lengths"].long() if s["lengths"] is not None else torch.full((case["B"],), case["T"], device=DEVICE)
        valid = torch.arange(case["T"], device=DEVICE).unsqueeze(0) < n.unsqueeze(1)
    count = valid.double().sum(1)
    if case["average"] == "token":
        w = valid.double() / count.sum().clamp(min=1)
    elif case["average"] == "sequence":
        w = valid.double() / count.clamp(min=1).unsqueeze(1) / (count > 0).sum().clamp(min=1)
    else:
        w = valid.double()

    def log_p(x):
        return torch.log_softmax(x / tau, -1)

    def pull_back(of_rows):
        """of_rows(log-probabilities, first, last): a scalar; its gradient in all logits."""
        grad = torch.empty(N, V, dtype=torch.float64, device=DEVICE)
        for i in range(0, N, step):
            x = rows[i:i + step].double().requires_grad_()
            grad[i:i + step] = torch.autograd.grad(of_rows(log_p(x), i, i + step), x)[0]
        if case["op"] != "score":
            grad *= SCALE[case["dtype"]]
        return grad.reshape(s["logits"].shape)

    if case["op"] == "distill":
        K = case["K"]
        ids = s["teacher_ids"].reshape(N, K).long()
        log_q = torch.log_softmax(s["teacher_logits"].reshape(N, K).double() / tau, -1)
        held = log_q > float("-inf")
        q, log_q, ids = log_q.exp(), log_q.masked_fill(~held, 0.0), ids.masked_fill(~held, 0)

        def divergence(lp, i, j):
            return tau ** 2 * (q[i:j] * (log_q[i:j] - lp.gather(1, ids[i:j]))).sum(1) * valid.reshape(-1)[i:j]

        with torch.no_grad():
            each = torch.cat([divergence(log_p(rows[i:i + step].double()), i, i + step) for i in range(0, N, step)])
        grad = pull_back(lambda lp, i, j: (divergence(lp, i, j) * w.reshape(-1)[i:j]).sum())
        return [(each * w.reshape(-1)).sum().reshape(1), grad, each.reshape(s["logits"].shape[:-1])]

    tokens = s["tokens"].reshape(N, 1).long()
    lp, entropy = [], []
    with torch.no_grad():
        for i in range(0, N, step):
            a = log_p(rows[i:i + step].double())
            lp.append(a.gather(1, tokens[i:i + step]).squeeze(1))
            entropy.append(-(a.exp() * a).sum(1))
    shape = (case["B"], case["T"])
    lp = (torch.cat(lp).reshape(shape) * valid).requires_grad_()
    entropy = (torch.cat(entropy).reshape(shape) * valid).requires_grad_()

    def from_values(d_lp, d_entropy):
        d_lp, d_entropy = (d_lp * valid).reshape(-1), (d_entropy * valid).reshape(-1)

        def of_rows(a, i, j):
            total = (a.gather(1, tokens[i:j]).squeeze(1) * d_lp[i:j]).sum()
            return total - ((a.exp() * a).sum(1) * d_entropy[i:j]).sum() if case["entropy"] else total
        return pull_back(of_rows)

    none = torch.zeros(shape, dtype=torch.float64, device=DEVICE)
    if case["op"] == "score":
        out = [lp.detach().reshape(s["tokens"].shape)]
        if case["entropy"]:
            out.append(entropy.detach().reshape(s["tokens"].shape))
        if case["backward"]:
            out.append(from_values(s["d_logprobs"].double(), s["d_entropy"].double() if case["entropy"] else none))
        return out if len(out) > 1 else out[0]

    if case["op"] == "policy":
        a = s["advantages"].double().reshape(shape[0], -1).expand(shape)
        ratio = torch.exp(lp - s["old"].double())
        held = torch.where(a > 0, ratio.clamp(max=1 + CLIP_HIGH), ratio.clamp(min=1 - CLIP_LOW))
        r = s["ref"].double() - lp if case["kl"] else none
        kl = torch.exp(r) - r - 1
        loss = ((case["kl"] * kl - held * a - (ENTROPY if case["entropy"] else 0.0) * entropy) * w).sum()
        d_lp, d_entropy = torch.autograd.grad(loss, (lp, entropy), materialize_grads=True, allow_unused=True)
        parts = [loss, (kl * w).sum(), ((held != ratio) & (a != 0)).double().mul(w).sum(),
                 (entropy * w).sum() if case["entropy"] else none.sum()]
        return [torch.stack(parts).detach(), from_values(d_lp, d_entropy), lp.detach()]

    beta, half = BETA[case["kind"]], shape[0] // 2
    d = torch.where(valid, lp - s["ref"].double(), none).sum(1)
    if case["kind"] == "ipo":
        d = d / count.clamp(min=1)
    margin = d[:half] - d[half:]
    if case["kind"] == "ipo":
        loss = (margin - 1 / (2 * beta)).square().mean()
    elif case["kind"] == "hinge":
        loss = torch.relu(1 - beta * margin).mean()
    else:
        e = case["smooth"]
        loss = -((1 - e) * torch.nn.functional.logsigmoid(beta * margin)
                 + e * torch.nn.functional.logsigmoid(-beta * margin)).mean()
    d_lp, = torch.autograd.grad(loss, lp)
    margin = margin.detach()
    return [torch.stack([loss.detach(), (margin > 0).double().mean(), margin.mean()]), from_values(d_lp, none),
            lp.detach().sum(1), margin]


def work(case):
    """Logits of the positions that count read once (expected lengths), a gradient of all of them
    written once, the values given and returned for each position; about six operations a value."""
    B, T, V = case["B"], case["T"], case["V"]
    low = (1 + case["low"]) / 2 if case["packed"] else (max(1, int(case["low"] * T)) + T) / 2 / T
    if case["low"] >= 1:
        low = 1.0
    size = 4 if case["dtype"] == "float32" else 2
    id_size = 8 if case["ids"] == "int64" else 4
    rows, graded = B * T, case["op"] != "score" or case["backward"]
    moved = low * rows * V * size + (rows * V * size if graded else 0)
    if case["op"] == "distill":
        moved += low * rows * case["K"] * (id_size + size) + 4 * rows
    else:
        given = {"score": 4 * graded * (1 + case["entropy"]), "policy": 4 + 4 * (case["kl"] > 0) + 4 * case["each"], "prefer": 4}
        moved += low * rows * (id_size + given[case["op"]])
        moved += rows * 4 * {"score": 1 + case["entropy"], "policy": 1, "prefer": 0}[case["op"]]
    return {"bytes": moved, "flops": low * rows * V * (6 if graded else 4)}
