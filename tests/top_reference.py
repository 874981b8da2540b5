"""Plain definitions of top log-probabilities and of embeddings with their gradients, in float64 on the CPU."""
import math

import torch

import loss_reference as ref


def top(logits, k, valid, temperature=1.0):
    """(x, log softmax, ids, log-probabilities): x the float64 leaf; entries that are not there: -1 and -inf."""
    x, logp = ref.rows(logits, valid, temperature)
    order = (x.detach() + 0.0).sort(dim=-1, descending=True, stable=True)      # (equal ones by their ids)
    ids, values = order.indices[..., :k], order.values[..., :k]
    there = (values > -math.inf) & valid.unsqueeze(-1)
    lp = logp.gather(-1, ids)
    return x, logp, torch.where(there, ids, -1), torch.where(there, lp, torch.full_like(lp, -math.inf))


def embedding(table, tokens, valid, scale=1.0):
    ids = torch.where(valid, tokens.cpu().long(), torch.zeros((), dtype=torch.long))
    out = table.detach().cpu().double()[ids] * scale
    return torch.where(valid.unsqueeze(-1), out, torch.zeros((), dtype=torch.float64))


def embedding_grad(d_rows, tokens, V, valid, scale=1.0):
    """(gradient, sum of the magnitudes of what each of its values is made of, positions of each token)"""
    at, rows = tokens.cpu().long()[valid], d_rows.detach().cpu().double()[valid] * scale
    D = d_rows.shape[-1]
    grad = torch.zeros(V, D, dtype=torch.float64).index_add_(0, at, rows)
    size = torch.zeros(V, D, dtype=torch.float64).index_add_(0, at, rows.abs())
    return grad, size, torch.bincount(at, minlength=V)
