"""Limits of the stand-alone operators on the device: empty batches."""
import pytest
import torch

from paper_2508_17624_b200 import binding, build

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


@pytest.mark.parametrize("n_slots", [1, 5])
@pytest.mark.parametrize("top_k", [1, 6])
def test_no_tokens(top_k, n_slots):
    """A step without tokens: results without rows, nothing reported."""
    q, scales = binding.quant_pack(torch.ones((n_slots, 16, 64), dtype=BF16, device="cuda"), 32)
    x, slots = torch.empty((0, 64), dtype=BF16, device="cuda"), torch.empty((0, top_k), dtype=torch.int32, device="cuda")
    y = binding.quant_mv(x, q, scales, slots)
    assert y.shape == (0, 16) and y.dtype == BF16
    assert binding.quant_mv(x, q, scales, slots, out_dtype=FP32).dtype == FP32
    assert binding.quant_mv(x, q[:1], scales[:1]).shape == (0, 16)
    p = torch.empty((0,), device="cuda")
    assert binding.swiglu(y).shape == (0, 8) and binding.swiglu(y, p).shape == (0, 8)
    dh, dp = binding.swiglu_grad(torch.empty((0, 8), dtype=BF16, device="cuda"), y, p)
    assert dh.shape == (0, 16) and dp.shape == (0,)
    assert binding.last_operator_error() == 0
