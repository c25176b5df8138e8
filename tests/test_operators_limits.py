"""Limits of the stand-alone operators' arguments, on the host: nothing is launched, no GPU is needed."""
import pytest
import torch

from paper_2508_17624_b200 import binding, build

INVALID, NO_DEVICE = 1, 9
BF16, FP16, FP32 = 0, 1, 2
X, W, OFF, OUT, SCALES = 0x1000, 0x2000, 0x3000, 0x4000, 0x5000        # addresses that are never read


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def mv(lib, device=-1, x=X, ldx=64, slots=OFF, pairs=12, per=6, n_slots=4, n=16, k=64, group=32, y=OUT, ldy=16):
    return lib.ew_quant_mv(device, BF16, BF16, x, ldx, W, SCALES, slots, pairs, per, n_slots, n, k, group, y, ldy, None)


def test_an_empty_batch_needs_no_slot_ids(lib):
    """A tensor without entries has no address: [0, top_k] slot ids are not the call without slot ids."""
    assert mv(lib, pairs=0, slots=None, x=None, y=None, n_slots=64) == NO_DEVICE
    assert mv(lib, pairs=6, slots=None, n_slots=64) == INVALID


def test_operands_that_autograd_records_are_refused():
    """A result without a gradient would go unnoticed."""
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((2, 64, 64), dtype=torch.bfloat16)
    offsets, p, q, scales = torch.zeros(3, dtype=torch.int32), torch.ones(4), torch.zeros((2, 64, 32), dtype=torch.uint8), torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    recorded = [t.clone().requires_grad_() for t in (x, w, p, scales)]
    xr, wr, pr, sr = recorded
    calls = [lambda: binding.grouped_mm(xr, w, offsets), lambda: binding.grouped_mm(x, wr, offsets), lambda: binding.grouped_mm_dx(xr, w, offsets),
             lambda: binding.grouped_mm_dx(x, wr, offsets), lambda: binding.grouped_mm_dw(xr, x, offsets), lambda: binding.grouped_mm_dw(x, xr, offsets),
             lambda: binding.quant_mv(xr, q, scales), lambda: binding.quant_mv(x, q, sr), lambda: binding.swiglu(xr), lambda: binding.swiglu(x, pr),
             lambda: binding.swiglu_grad(xr, x), lambda: binding.swiglu_grad(x[:, :32], xr), lambda: binding.swiglu_grad(x[:, :32], x, pr)]
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):      # the next check
            call()
