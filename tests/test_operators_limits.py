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


class Huge:
    """What the binding asks of a device tensor, for one of any size; its address is what the library would be called with."""
    requires_grad = False

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def stride(self, d=None):
        strides = [self.shape[i + 1:].numel() for i in range(len(self.shape))]
        return tuple(strides) if d is None else strides[d]

    def new_empty(self, shape, dtype=None):
        return Huge(*shape, dtype=dtype or self.dtype)

    def data_ptr(self):
        raise AssertionError("the call went on")


def test_sizes_beyond_32_bits_are_refused():
    """The library's sizes have 32 bits and ctypes cuts larger ones down to them: 2^32 + 5 rows would have been five."""
    far, i32, f32, u8 = 2 ** 32 + 5, torch.int32, torch.float32, torch.uint8
    offsets = Huge(3, dtype=i32)
    calls = [lambda: binding.grouped_mm(Huge(far, 8), Huge(2, 8, 8), offsets), lambda: binding.grouped_mm(Huge(4, 8), Huge(2, far, 8), offsets),
             lambda: binding.grouped_mm_dx(Huge(4, far), Huge(2, far, 8), offsets), lambda: binding.grouped_mm(Huge(4, far), Huge(2, 8, far), offsets),
             lambda: binding.grouped_mm(Huge(4, 8), Huge(far, 8, 8), Huge(far + 1, dtype=i32)), lambda: binding.grouped_mm_dw(Huge(far, 8), Huge(far, 8), offsets),
             lambda: binding.grouped_mm_dw(Huge(4, far), Huge(4, 8), offsets), lambda: binding.grouped_mm_dw(Huge(4, 8), Huge(4, 8), Huge(far + 1, dtype=i32)),
             lambda: binding.quant_mv(Huge(1, 32), Huge(2, 8, 16, dtype=u8), Huge(2, 1, 8), Huge(far, dtype=i32)),
             lambda: binding.quant_mv(Huge(1, 32), Huge(far, 8, 16, dtype=u8), Huge(far, 1, 8), Huge(1, dtype=i32)),
             lambda: binding.quant_mv(Huge(1, 32), Huge(2, far, 16, dtype=u8), Huge(2, 1, far), Huge(1, dtype=i32)),
             lambda: binding.quant_mv(Huge(far, 32), Huge(1, 8, 16, dtype=u8), Huge(1, 1, 8)),
             lambda: binding.quant_pack(Huge(far, 8, 32), 32), lambda: binding.quant_pack(Huge(1, far, 32), 32),
             lambda: binding.swiglu(Huge(far, 2)), lambda: binding.swiglu(Huge(4, 2 * far)), lambda: binding.swiglu(Huge(far, 2), Huge(far, dtype=f32)),
             lambda: binding.swiglu_grad(Huge(far, 1), Huge(far, 2))]
    for call in calls:
        with pytest.raises(ValueError, match="the library takes up to"):
            call()
    with pytest.raises(AssertionError, match="went on"):
        binding.swiglu(Huge(2 ** 31 - 1, 2))


def test_quant_mv_widths_near_two_to_the_31(lib):
    """The widths that the header names, and nothing beyond them, wherever a sum of sizes may pass 31 bits."""
    assert mv(lib, n_slots=1, n=33554400, ldy=33554400) == NO_DEVICE
    for n_slots, n in ((1, 33554408), (1, 0x7ffffff8), (1, 0x7fffffe8), (64, 33554432), (2048, 1048576)):
        assert mv(lib, n_slots=n_slots, n=n, ldy=n) == INVALID, (n_slots, n)


def test_strides_of_groups(lib):
    """Groups one behind the other or row by row; a stride whose product with the rows passes 64 bits is not taken for a small one."""
    def mm(fn, ld, stride, groups=3, n=64, k=64):
        return getattr(lib, fn)(-1, BF16, BF16, X, 64, W, ld, stride, OFF, 8, groups, n, k, OUT, max(n, k), None)

    def dw(ld, stride, groups=3, n=64, k=64):
        return lib.ew_grouped_mm_dw(-1, BF16, FP32, X, max(n, 64), W, 64, OFF, 8, groups, n, k, 0, OUT, ld, stride, None)

    def pack(ld, stride, groups=3, n=64, k=64):
        return lib.ew_quant_pack(-1, BF16, X, ld, stride, groups, n, k, 32, W, OUT, None)

    for call in (lambda *a, **b: mm("ew_grouped_mm", *a, **b), lambda *a, **b: mm("ew_grouped_mm_dx", *a, **b), dw, pack):
        assert call(64, 64 * 64) == call(72, 63 * 72 + 64) == call(3 * 64, 64) == call(2 * 72 + 64, 72) == NO_DEVICE
        assert call(64, 0, groups=1) == NO_DEVICE and (call is pack or call(64, 64, n=1) == NO_DEVICE)
        for ld, stride in ((64, 63 * 64), (72, 63 * 72 + 56), (2 * 64 + 56, 64), (3 * 64, 56), (3 * 64, 0), (64, -64 * 64), (3 * 64, -64)):
            assert call(ld, stride) == INVALID, (ld, stride)
    # (2^31 - 65536) rows of 2^37 elements pass 2^64
    assert dw(2 ** 37, 64, n=0x7fff0000) == NO_DEVICE and dw(2 ** 37, 56, n=0x7fff0000) == INVALID
    assert dw(2 ** 33 + 2 ** 18, 2 ** 40, n=0x7fff0000) == INVALID and mm("ew_grouped_mm", 2 ** 37, 2 ** 37 + 8, n=0x7fff0000) == INVALID


def test_results_that_autograd_records_are_refused():
    """Written by the library, they would change under autograd's hands."""
    def out(*shape, dtype=torch.bfloat16):
        t = Huge(*shape, dtype=dtype)
        t.requires_grad = True
        return t

    x, w, offsets = Huge(4, 64), Huge(2, 64, 64), Huge(3, dtype=torch.int32)
    calls = [lambda: binding.grouped_mm(x, w, offsets, out=out(4, 64)), lambda: binding.grouped_mm_dx(x, w, offsets, out=out(4, 64)),
             lambda: binding.grouped_mm_dw(x, x, offsets, out=out(2, 64, 64), accumulate=True), lambda: binding.swiglu(x, out=out(4, 32)),
             lambda: binding.swiglu_grad(Huge(4, 32), x, out=out(4, 64)),
             lambda: binding.quant_mv(x, Huge(1, 64, 32, dtype=torch.uint8), Huge(1, 2, 64), out=out(4, 64))]
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
