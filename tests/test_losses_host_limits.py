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


@pytest.mark.parametrize("type_", [0, 1, 2])
@pytest.mark.parametrize("V,rc", [(losses.VALUES_MOST, 0), (losses.VALUES_MOST + 1, 1), (2 ** 31 - 8, 1), (2 ** 31 - 1, 1)])
def test_rows_whose_end_is_no_number_of_32_bits(lib, V, rc, type_):  # noqa: F811
    """The kernels count a row's chunks and look at places up to a workgroup behind its end in 32 bits."""
    l, p = logits(V=V, B=0, type=type_, pos_stride=V, seq_stride=3 * V), positions()
    top = losses.tb_top_t(ids=HERE, logprobs=HERE, id_bytes=8, K=4)
    g = losses.tb_gradient_t(data=HERE << 24, seq_stride=3 * V, pos_stride=V, scale=1.0)
    ref = ctypes.byref
    assert lib.tensorloss_token_logprobs(ref(l), ref(p), HERE, None, None, None, None) == rc
    assert lib.tensorloss_top_logprobs(ref(l), ref(p), ref(top), HERE, None, None, None, None, 0, None) == rc
    assert lib.tensorloss_top_logprobs_grad(ref(l), ref(p), ref(top), HERE, HERE, HERE, None, ref(g), None) == rc
