"""Limits of the stand-alone operators' arguments, on the host: nothing is launched, no GPU is needed."""
import pytest

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
