"""How far a gradient in the logits may be off, value by value.

Row of logits z = x / temperature with probabilities p.  Its gradient is a sum of a few terms of known
size: -p d (the softmax's part of a log-probability with cotangent d), d more at the chosen token, and
-d_H p (log p + H) of an entropy.  LP and H are the bounds on log-probabilities and entropies that
tests/test_gpu_losses.py derives; a weight 2^a is off by at most LP relatively there (2 |a| u of its
argument, |a| <= 126, and 2 u of the instruction), and so are their sum, and the ratio exp(lp - old) that a
cotangent may hold.  So the softmax's part is off by 3 LP of itself, what stands at the token by 2 LP of the
cotangent, and the entropy's part by that of its factors: no value is allowed more than it is made of.
A result in 16 bits is rounded once more."""
import torch

LP, H = 3e-5, 2e-4
ROUND = {torch.float32: 2.0 ** -22, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
STEP = {torch.float32: 1e-36, torch.bfloat16: 1e-36, torch.float16: 2.0 ** -25}


def of_softmax(logp, d, extra, d_entropy=None):
    """Bound of a gradient before its last rounding.  logp: log-probabilities of the rows [.., V]; d [..]: size
    of the cotangents of lp; extra [.., V]: what is added beside the softmax's part (cotangents at tokens, a
    teacher's probabilities); d_entropy [..]: cotangents of the entropy."""
    p = logp.exp()
    bound = 3 * LP * p * d.abs().unsqueeze(-1) + 2 * LP * extra.abs()
    if d_entropy is not None:
        held = logp.clamp(min=-1e4)
        h = -(p * held).sum(-1, keepdim=True)
        bound = bound + p * d_entropy.abs().unsqueeze(-1) * (3 * LP * (held.abs() + h) + LP + H)
    return bound


def at_tokens(logp, tokens, d):
    """Zeros but for |d| at the tokens, of the shape of logp."""
    return torch.zeros_like(logp).scatter(-1, tokens.unsqueeze(-1), d.abs().unsqueeze(-1))


def breaches(got, want, bound, dtype, scale=1.0):
    """Where a result of `dtype` is further off than the bound and its rounding; scale: it was multiplied by."""
    got = got.detach().cpu().double() / scale
    allowed = bound + want.abs() * (1.01 * ROUND[dtype]) + STEP[dtype] / scale
    return ~((got - want).abs() <= allowed)


def check(got, want, bound, dtype, what="", scale=1.0):
    assert got.shape == want.shape and torch.isfinite(want).all(), what
    bad = breaches(got, want, bound, dtype, scale)
    off = (got.detach().cpu().double() / scale - want)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), off[bad][:3].tolist(), want[bad][:3].tolist())
