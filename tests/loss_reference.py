"""Plain definitions of the losses over logits in float64 on the CPU, with autograd for the gradients.

Positions that do not count are replaced before anything is computed, so whatever stands there has no
part in it."""
import torch


def valid_positions(shape, lengths=None, mask=None):
    valid = torch.ones(shape, dtype=torch.bool)
    if lengths is not None:
        valid &= torch.arange(shape[-1]) < lengths.cpu().long().unsqueeze(-1)
    if mask is not None:
        valid &= mask.cpu() != 0
    return valid


def weights(valid, average):
    """[B, T] weights (a packed row of positions is one sequence)."""
    v = valid.double().reshape(-1, valid.shape[-1])
    n = v.sum(1, keepdim=True)
    if average == "token":
        v = v / max(float(n.sum()), 1.0)
    elif average == "sequence":
        v = v / n.clamp(min=1) / max(int((n > 0).sum()), 1)
    return v.reshape(valid.shape)


def rows(logits, valid, temperature):
    """(x, log softmax of x / temperature) with x a float64 leaf; zeros where a position does not count."""
    x = torch.where(valid.unsqueeze(-1), logits.detach().cpu().double(), torch.zeros((), dtype=torch.float64))
    x.requires_grad_()
    return x, torch.log_softmax(x / temperature, -1)


def chosen(logp, tokens, valid):
    ids = torch.where(valid, tokens.cpu().long(), torch.zeros((), dtype=torch.long))
    lp = logp.gather(-1, ids.unsqueeze(-1)).squeeze(-1)
    return torch.where(valid, lp, torch.zeros_like(lp))


def entropies(logp, valid):
    h = -(logp.exp() * logp.masked_fill(logp == -float("inf"), 0.0)).sum(-1)   # (0 log 0 is 0, its slope, too)
    return torch.where(valid, h, torch.zeros_like(h))


def given(t, valid):
    """A value for each position in float64; 0 where the position does not count."""
    return torch.where(valid, t.detach().cpu().double(), torch.zeros((), dtype=torch.float64))


def policy(logits, tokens, old, advantages, ref=None, lengths=None, mask=None, clip_low=0.2, clip_high=0.2,
           kl_coef=0.0, entropy_coef=0.0, average="token", temperature=1.0):
    """(terms, gradient, log-probabilities)"""
    valid = valid_positions(logits.shape[:-1], lengths, mask)
    w = weights(valid, average)
    x, logp = rows(logits, valid, temperature)
    lp, h = chosen(logp, tokens, valid), entropies(logp, valid)
    a = advantages.detach().cpu().double()
    a = given(a if a.dim() == lp.dim() else a.unsqueeze(-1).expand(lp.shape), valid)
    ratio = torch.exp(lp - given(old, valid))
    held = torch.where(a > 0, ratio.clamp(max=1 + clip_high), ratio.clamp(min=1 - clip_low))
    kl = torch.zeros_like(lp)
    if kl_coef:
        d = given(ref, valid) - lp
        kl = torch.expm1(d) - d
    loss = (w * (-held * a + kl_coef * kl - entropy_coef * h)).sum()
    grad, = torch.autograd.grad(loss, x)
    clipped = ((held != ratio) & (a != 0)).double()
    terms = [loss, (w * kl).sum(), (w * clipped).sum(), (w * h).sum() if entropy_coef else torch.zeros(())]
    return torch.stack([t.detach().double() for t in terms]), grad, lp.detach()


def preference(logits, tokens, ref, lengths=None, mask=None, beta=0.1, kind="sigmoid", label_smoothing=0.0,
               temperature=1.0):
    """(terms, gradient, sequence log-probabilities, margins)"""
    valid = valid_positions(logits.shape[:-1], lengths, mask)
    x, logp = rows(logits, valid, temperature)
    lp = chosen(logp, tokens, valid)
    d = (lp - given(ref, valid)).sum(1)
    if kind == "ipo":
        d = d / valid.sum(1).clamp(min=1)
    half = d.shape[0] // 2
    h = d[:half] - d[half:]
    if kind == "ipo":
        loss = (h - 1 / (2 * beta)).square().mean()
    elif kind == "hinge":
        loss = torch.relu(1 - beta * h).mean()
    else:
        sp = torch.nn.functional.softplus
        loss = ((1 - label_smoothing) * sp(-beta * h) + label_smoothing * sp(beta * h)).mean()
    grad, = torch.autograd.grad(loss, x)
    h = h.detach()
    return (torch.stack([loss.detach(), (h > 0).double().mean(), h.mean()]), grad, lp.detach().sum(1), h)


def distillation(logits, ids, teacher, lengths=None, mask=None, temperature=1.0, average="token"):
    """(terms, gradient, row losses)"""
    valid = valid_positions(logits.shape[:-1], lengths, mask)
    w = weights(valid, average)
    x, logp = rows(logits, valid, temperature)
    t = teacher.detach().cpu().double() / temperature
    entry = (t > -float("inf")) & valid.unsqueeze(-1)
    t = t.masked_fill(~entry, -1e300)
    q = torch.where(entry, torch.softmax(t, -1), torch.zeros_like(t))
    log_q = torch.where(q > 0, torch.log_softmax(t, -1), torch.zeros_like(t))
    lp = logp.gather(-1, torch.where(entry, ids.cpu().long(), torch.zeros((), dtype=torch.long)))
    each = temperature ** 2 * torch.where(q > 0, q * (log_q - lp), torch.zeros_like(q)).sum(-1)
    loss = (w * each).sum()
    grad, = torch.autograd.grad(loss, x)
    return loss.detach().reshape(1), grad, each.detach()
