"""Refusals of the stand-alone operators, on the host: nothing is launched, no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2508_17624_b200 import binding, build

INVALID, NO_DEVICE = 1, 9
BF16, FP16, FP32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


# Addresses that are never read: every call below is refused before the device is touched.
X, W, OFF, OUT = 0x1000, 0x2000, 0x3000, 0x4000


def mm(lib, fn="ew_grouped_mm", device=-1, dtype=BF16, out_dtype=BF16, x=X, ldx=64, w=W, ldw=64, gs=64 * 64, off=OFF, rows=8, groups=2, n=64, k=64, out=OUT, ldo=64):
    return getattr(lib, fn)(device, dtype, out_dtype, x, ldx, w, ldw, gs, off, rows, groups, n, k, out, ldo, None)


@pytest.mark.parametrize("fn", ["ew_grouped_mm", "ew_grouped_mm_dx"])
def test_grouped_mm_refuses(lib, fn):
    assert mm(lib, fn) == NO_DEVICE                                          # everything else is in order
    assert mm(lib, fn, rows=0) == NO_DEVICE
    bad = [dict(dtype=FP32), dict(out_dtype=FP16), dict(dtype=FP16, out_dtype=BF16), dict(dtype=7), dict(rows=-1), dict(groups=0), dict(groups=2049),
           dict(n=0), dict(k=0), dict(off=None), dict(off=OFF + 2), dict(out=None), dict(out=OUT + 1), dict(out_dtype=FP32, out=OUT + 2),
           dict(x=None), dict(x=X + 8), dict(ldx=60), dict(ldx=68), dict(w=None), dict(w=W + 2), dict(ldw=56), dict(ldw=65), dict(gs=64 * 63), dict(gs=64 * 64 + 4), dict(ldo=63)]
    for change in bad:
        assert mm(lib, fn, **change) == INVALID, change
        assert binding.lib().ew_last_error_string()
    assert mm(lib, fn, groups=1, gs=0) == NO_DEVICE                          # a single group has no stride


def dw(lib, device=-1, dtype=BF16, out_dtype=FP32, dy=X, lddy=64, x=W, ldx=64, off=OFF, rows=8, groups=2, n=64, k=64, acc=0, out=OUT, ld=64, gs=64 * 64):
    return lib.ew_grouped_mm_dw(device, dtype, out_dtype, dy, lddy, x, ldx, off, rows, groups, n, k, acc, out, ld, gs, None)


def test_grouped_mm_dw_refuses(lib):
    assert dw(lib) == NO_DEVICE
    assert dw(lib, rows=0, dy=None, x=None) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(out_dtype=FP16), dict(rows=-1), dict(groups=0), dict(groups=4096), dict(n=0), dict(k=-3), dict(off=None), dict(out=None),
                   dict(out=OUT + 2), dict(dy=None), dict(dy=X + 4), dict(lddy=63), dict(lddy=65), dict(x=W + 4), dict(ldx=68), dict(ld=63), dict(gs=4095)]:
        assert dw(lib, **change) == INVALID, change


def mv(lib, device=-1, dtype=BF16, out_dtype=BF16, x=X, ldx=64, q=W, sc=0x5000, slots=OFF, pairs=12, per=6, n_slots=4, n=16, k=64, group=32, y=OUT, ldy=16):
    return lib.ew_quant_mv(device, dtype, out_dtype, x, ldx, q, sc, slots, pairs, per, n_slots, n, k, group, y, ldy, None)


def test_quant_mv_refuses(lib):
    assert mv(lib) == mv(lib, pairs=0, x=None, y=None) == mv(lib, slots=None, n_slots=1, per=1) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(out_dtype=FP16), dict(x=None), dict(x=X + 8), dict(ldx=63), dict(ldx=68), dict(q=None), dict(q=W + 8), dict(sc=None), dict(sc=X + 2),
                   dict(slots=None), dict(slots=OFF + 1), dict(pairs=-6), dict(pairs=13), dict(per=0), dict(n_slots=0), dict(n_slots=2049), dict(n=12), dict(n=0), dict(k=48),
                   dict(k=0), dict(group=16), dict(group=96, k=96, ldx=96), dict(group=128), dict(y=None), dict(y=OUT + 1), dict(ldy=15)]:
        assert mv(lib, **change) == INVALID, change


def test_quant_pack_refuses(lib):
    def pack(device=-1, dtype=BF16, w=X, ldw=64, stride=1024, n_slots=2, n=16, k=64, group=32, q=W, sc=OUT):
        return lib.ew_quant_pack(device, dtype, w, ldw, stride, n_slots, n, k, group, q, sc, None)

    assert pack() == pack(n_slots=1, stride=0) == pack(ldw=65, stride=1040) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(w=None), dict(w=X + 1), dict(ldw=63), dict(stride=1023), dict(n_slots=0), dict(n=4), dict(n=12), dict(k=65), dict(group=48, k=96, ldw=96),
                   dict(q=None), dict(q=W + 8), dict(sc=None), dict(sc=OUT + 2)]:
        assert pack(**change) == INVALID, change


def test_swiglu_refuses(lib):
    def act(device=-1, dtype=BF16, h=X, ldh=32, p=W, rows=4, inter=16, out=OUT, ldo=16):
        return lib.ew_swiglu(device, dtype, h, ldh, p, rows, inter, out, ldo, None)

    def grad(device=-1, dtype=BF16, da=X, ldda=16, h=X, ldh=32, p=W, rows=4, inter=16, out=OUT, ldo=32, dp=OFF):
        return lib.ew_swiglu_grad(device, dtype, da, ldda, h, ldh, p, rows, inter, out, ldo, dp, None)

    assert act() == act(p=None) == act(rows=0, h=None, out=None, p=None) == grad() == grad(dp=None) == grad(p=None, dp=None) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(h=None), dict(h=X + 1), dict(ldh=31), dict(p=W + 2), dict(rows=-1), dict(inter=0), dict(out=None), dict(out=OUT + 1), dict(ldo=15)]:
        assert act(**change) == INVALID, change
    for change in [dict(dtype=FP32), dict(da=None), dict(da=X + 1), dict(ldda=15), dict(h=None), dict(ldh=31), dict(p=None), dict(rows=-1), dict(inter=-1), dict(out=None),
                   dict(ldo=31), dict(dp=OFF + 2)]:
        assert grad(**change) == INVALID, change


def test_operator_error_word_refuses(lib):
    assert lib.ew_last_operator_error(0, None) == INVALID
    assert lib.ew_last_operator_error(-1, C.byref(C.c_int32())) == NO_DEVICE


def test_python_checks_before_the_library():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(2, 8, 8, dtype=torch.bfloat16)
    offsets = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.grouped_mm(x, w, offsets)
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.grouped_mm_dw(x, x, offsets)
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.swiglu(x)
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.quant_pack(w, 32)
