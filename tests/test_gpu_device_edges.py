"""Arguments at their ends, on a B200: scales and caps of every size, lengths up to the limit, page tables and logits that hold what they should not."""
import pytest
import torch

from tests.test_gpu_device_ops import attention_case, check_attention, status, ws  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [-0.125, 0.0, 1e-39, -1e-3])
@pytest.mark.parametrize("q,kv", [([1, 1, 1], [75, 40, 200]), ([70, 3, 16], [75, 40, 200]), ([4], [2000])])
@pytest.mark.parametrize("cap,window,prefix,bias", [(0.0, 0, 0, False), (0.0, 17, 21, False), (30.0, 0, 0, False), (0.0, 0, 0, True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_of_scales_that_are_not_positive(scale, q, kv, cap, window, prefix, bias, dtype, ws, status):
    """The smallest key's score is the largest, or all are alike; masked keys stay at -infinity.  (No scale is above head_dim^-1/2, which check_attention's
    tolerance is made for.)"""
    c = attention_case(11, kv, q, 8, 2, 64, dtype, cap, window, prefix, bias)
    c["scale"] = scale
    check_attention(c, ws, status)
