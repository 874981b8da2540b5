"""Tokens at the type's lowest value, as masks leave them, are there: their log-probabilities are of about that size, and
-inf only where it lies beyond float32.  In every kernel.

z = (x - m) / temperature is rounded at most four times (the difference, the temperature's inverse, their product, the
subtraction of log s), or six times as a product with log2(e) and back: within 6 * 2^-24 of itself."""
import math

import pytest
import torch

import paper_2510_05485_amd as tb
from test_gpu_losses import DEV, LP, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("temperature", [1.0, 2.0, 0.5])
@pytest.mark.parametrize("rows,V,k", [(3, 5, 5), (3, 40, 8), (40, 1000, 7), (9, 300, 33), (9, 600, 100), (9, 3000, 64), (9, 9001, 200),
                                      (3, 50257, 600), (600, 30001, 20), (600, 110_001, 20), (2, 262_144, 50)])
def test_lowest_values(rows, V, k, temperature, dtype):
    g = torch.Generator(device=DEV).manual_seed(V)
    lowest = torch.finfo(dtype).min
    x = torch.full((rows, V), lowest, dtype=dtype, device=DEV)
    ids = torch.randint(0, V, (rows, k - 2), generator=g, device=DEV)           # fewer than k tokens are left
    x.scatter_(1, ids, torch.randn(rows, k - 2, generator=g, device=DEV).to(dtype))
    tokens = (x == lowest).long().argmax(-1)
    r = tb.top_logprobs(x, k, tokens, temperature=temperature, want_entropy=True)
    logp = torch.log_softmax(x.double() / temperature, -1)
    order = x.double().sort(dim=-1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(r.ids, order)
    want = logp.gather(-1, order)
    low = x.gather(-1, order) == lowest
    assert low[:, -1].all() and not low[:, 0].any()
    assert ((r.logprobs.double() - want)[~low].abs() <= LP).all()
    for got, want in ((r.logprobs[low], want[low]), (r.token_logprobs, logp.gather(-1, tokens.unsqueeze(-1)).squeeze(-1))):
        beyond = want.float() == -math.inf
        assert (got[beyond] == -math.inf).all()
        assert (got.double() - want)[~beyond].abs().le(want[~beyond].abs() * (6 * 2.0 ** -24)).all()
    assert beyond.all() if temperature < 1 and dtype != torch.float16 else not beyond.any()
