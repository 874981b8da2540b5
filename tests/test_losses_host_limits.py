"""Host side of the losses: scales that float32 cannot hold are refused before any launch."""
import ctypes

import pytest

from paper_2510_05485_amd import losses
from test_losses_host import HERE, lib, logits, positions  # noqa: F401  (lib is a fixture)


@pytest.mark.parametrize("temperature", [1e-45, 1e-39, 2.9e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_reciprocal_is_not_finite(lib, temperature):  # noqa: F811
    """The kernels multiply by log2(e) / temperature: 1.4427 / 4.2e-39 is beyond 3.4e38, the reciprocal of
    the last three alone is not."""
    l, p = logits(temperature=temperature), positions()
    assert lib.tensorloss_token_logprobs(ctypes.byref(l), ctypes.byref(p), HERE, None, None, None, None) == 1
    w = losses.workspace_bytes(4, 3)
    q = losses.tb_policy_t(old_logprobs=HERE, ref_logprobs=HERE, advantages=HERE, clip_low=0.2, clip_high=0.2)
    assert lib.tensorloss_policy(ctypes.byref(l), ctypes.byref(p), ctypes.byref(q), None, HERE, HERE, None, None, None,
                                 None, HERE, w, None) == 1
