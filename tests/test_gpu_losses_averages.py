"""Means over positions and sequences on both sides of the rule that decides where they are added up: in every
workgroup, or by launches before (many sequences times many workgroups, masks of more than 2048 positions)."""
import pytest
import torch

import loss_bounds as bounds
import loss_reference as ref
import paper_2510_05485_amd as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("average", ["token", "sequence"])
@pytest.mark.parametrize("B,T,V", [(1450, 2, 2100), (1450, 4, 2100), (2100, 2, 2100), (3000, 2, 70), (4, 512, 2100),
                                   (4, 513, 2100), (1, 2048, 40), (1, 2049, 40)])
@pytest.mark.parametrize("masked", [False, True])
def test_means(B, T, V, average, masked):
    g = torch.Generator().manual_seed(B + T + V)
    x, tokens = torch.randn(B, T, V, generator=g), torch.randint(0, V, (B, T), generator=g)
    lengths = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
    mask = torch.rand(B, T, generator=g) < 0.7 if masked else None
    old, a = torch.full((B, T), -8.0), torch.randn(B, generator=g)
    where = dict(lengths=lengths.to(DEV), mask=None if mask is None else mask.to(DEV), average=average)
    terms, want, lp = ref.policy(x, tokens, old, a, None, lengths, mask, average=average)
    r = tb.policy_loss_grad(x.to(DEV), tokens.to(DEV), old.to(DEV), a.to(DEV), **where)
    logp = torch.log_softmax(x.double(), -1)
    valid = ref.valid_positions((B, T), lengths, mask)
    # a weight is off by 2^-22 of itself: within the 3 LP of what it weighs
    d = ref.weights(valid, average) * a.abs().double().unsqueeze(-1) * torch.exp(lp + 8.0)     # |ratio A|
    bounds.check(r.grad, want, bounds.of_softmax(logp, d, bounds.at_tokens(logp, tokens, d)), torch.float32, "policy")
    assert abs(float(r.loss) - float(terms[0])) <= 3 * bounds.LP * float(d.sum()) + 1e-9

    ids, teacher = tokens.unsqueeze(-1), torch.zeros(B, T, 1)
    terms, want, rows = ref.distillation(x, ids, teacher, lengths, mask, average=average)
    r = tb.distillation_loss_grad(x.to(DEV), ids.to(DEV), teacher.to(DEV), **where)
    d = ref.weights(valid, average)
    bounds.check(r.grad, want, bounds.of_softmax(logp, d, bounds.at_tokens(logp, tokens, d)), torch.float32, "distillation")
    assert abs(float(r.loss) - float(terms[0])) <= 4 * bounds.LP
