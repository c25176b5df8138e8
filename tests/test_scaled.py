"""Refusals of the operators in 8-bit floating point and of the norm, on the host: nothing is launched, no GPU is needed."""
import pytest
import torch

from paper_2508_17624_b200 import binding, build

INVALID, NO_DEVICE = 1, 9
BF16, FP16, FP32, E4M3, E5M2 = range(5)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


# Addresses that are never read: every call below is refused before the device is touched.
X, W, OFF, OUT, SX, SW = 0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000


@pytest.mark.parametrize("fn", ["ew_scaled_mm", "ew_scaled_mm_dx"])
def test_scaled_mm_refuses(lib, fn):
    def mm(device=-1, dtype=E4M3, out_dtype=BF16, x=X, ldx=128, sx=SX, lds=4, w=W, ldw=128, gs=128 * 128, sw=SW, off=OFF, rows=8, groups=2, n=128, k=128, out=OUT, ldo=128):
        return getattr(lib, fn)(device, dtype, out_dtype, x, ldx, sx, lds, w, ldw, gs, sw, off, rows, groups, n, k, out, ldo, None)

    good = [dict(), dict(dtype=E5M2, out_dtype=FP32), dict(out_dtype=FP16), dict(rows=0, x=None, sx=None, out=None), dict(groups=1, gs=0, off=None), dict(sw=SW + 1), dict(sx=SX + 1, lds=5),
            dict(n=100, k=100, ldo=100), dict(gs=128, ldw=256)]
    for change in good:
        assert mm(**change) == NO_DEVICE, change
    bad = [dict(dtype=BF16), dict(dtype=FP32), dict(dtype=7), dict(out_dtype=E4M3), dict(out_dtype=-1), dict(rows=-1), dict(groups=0), dict(groups=2049), dict(n=0), dict(k=0),
           dict(off=None), dict(off=OFF + 2), dict(out=None), dict(out=OUT + 1), dict(out_dtype=FP32, out=OUT + 2), dict(x=None), dict(x=X + 8), dict(ldx=120), dict(ldx=136),
           dict(sx=None), dict(lds=0), dict(w=None), dict(w=W + 8), dict(ldw=112), dict(ldw=130), dict(gs=128 * 127), dict(gs=128 * 128 + 8), dict(sw=None),
           dict(ldo=127)]
    for change in bad:
        assert mm(**change) == INVALID, change
        assert lib.ew_last_error_string()


def test_scaled_rows_refuses(lib):
    def rows(device=-1, dtype=BF16, to=E4M3, x=X, ldx=200, rows=3, width=200, q=W, ldq=200, s=SX, lds=2):
        return lib.ew_scaled_rows(device, dtype, to, x, ldx, rows, width, q, ldq, s, lds, None)

    assert rows() == rows(to=E5M2, dtype=FP16) == rows(q=W + 1, s=SX + 1, x=X + 2) == rows(rows=0, x=None, q=None, s=None) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(dtype=E4M3), dict(to=BF16), dict(to=9), dict(x=None), dict(x=X + 1), dict(ldx=199), dict(rows=-1), dict(width=0), dict(q=None), dict(ldq=199),
                   dict(s=None), dict(lds=1)]:
        assert rows(**change) == INVALID, change


def test_swiglu_scaled_refuses(lib):
    def act(device=-1, dtype=BF16, h=X, ldh=400, p=OFF, rows=3, inter=200, q=W, ldq=200, s=SX, lds=2):
        return lib.ew_swiglu_scaled(device, dtype, h, ldh, p, rows, inter, q, ldq, s, lds, None)

    assert act() == act(p=None) == act(rows=0, h=None, q=None, s=None) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(h=None), dict(h=X + 1), dict(ldh=399), dict(p=OFF + 2), dict(rows=-1), dict(inter=0), dict(q=None), dict(ldq=199), dict(s=None), dict(lds=1)]:
        assert act(**change) == INVALID, change


def test_scaled_pack_refuses(lib):
    def pack(device=-1, dtype=BF16, w=X, ldw=64, stride=1024, n_slots=2, n=16, k=64, q=W, ldq=64, qs=1024, s=SX):
        return lib.ew_scaled_pack(device, dtype, w, ldw, stride, n_slots, n, k, q, ldq, qs, s, None)

    assert pack() == pack(n_slots=1, stride=0, qs=0) == pack(ldw=65, stride=1040) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(w=None), dict(w=X + 1), dict(ldw=63), dict(stride=1023), dict(n_slots=0), dict(n_slots=2049), dict(n=0), dict(k=0), dict(q=None), dict(ldq=63),
                   dict(qs=1023), dict(s=None)]:
        assert pack(**change) == INVALID, change


def test_rms_norm_refuses(lib):
    def norm(device=-1, dtype=BF16, x=X, ldx=64, res=W, ldr=64, w=OFF, eps=1e-6, rows=4, width=64, t=OUT, ldt=64, y=SX, ldy=64, q=SW, ldq=64, s=0x7000, lds=1):
        return lib.ew_rms_norm(device, dtype, x, ldx, res, ldr, w, eps, rows, width, t, ldt, y, ldy, q, ldq, s, lds, None)

    assert norm() == norm(res=None, t=None) == norm(q=None, s=None) == norm(y=None) == norm(t=W) == norm(rows=0, x=None, w=None, y=None, q=None) == norm(eps=0.0) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(dtype=E4M3), dict(x=None), dict(x=X + 1), dict(ldx=63), dict(res=W + 1), dict(ldr=63), dict(w=None), dict(w=OFF + 1), dict(eps=-1.0),
                   dict(eps=float("nan")), dict(eps=float("inf")), dict(rows=-1), dict(width=0), dict(width=16385, ldx=16385), dict(t=None), dict(t=OUT + 1), dict(ldt=63),
                   dict(y=None, q=None), dict(y=SX + 1), dict(ldy=63), dict(ldq=63), dict(s=None), dict(lds=0)]:
        assert norm(**change) == INVALID, change


def test_rms_norm_grad_refuses(lib):
    def grad(device=-1, dtype=BF16, dy=X, lddy=64, t=W, ldt=64, w=OFF, more=SX, ldm=64, eps=1e-6, rows=4, width=64, dt=OUT, lddt=64, dw=SW, room=0x7000):
        return lib.ew_rms_norm_grad(device, dtype, dy, lddy, t, ldt, w, more, ldm, eps, rows, width, dt, lddt, dw, room, None)

    assert grad() == grad(more=None) == grad(rows=0, dy=None, t=None, dt=None, room=None) == grad(room=None) == grad(rows=10 ** 6) == NO_DEVICE
    for change in [dict(dtype=FP32), dict(dy=None), dict(dy=X + 1), dict(lddy=63), dict(t=None), dict(ldt=63), dict(w=None), dict(more=SX + 1), dict(ldm=63), dict(eps=-1e-6), dict(rows=-1),
                   dict(width=0), dict(width=16385), dict(dt=None), dict(dt=OUT + 1), dict(lddt=63), dict(dw=None), dict(dw=SW + 2), dict(rows=10 ** 6, room=None), dict(room=0x7002)]:
        assert grad(**change) == INVALID, change
    assert lib.ew_rms_norm_grad_parts(0, 64) == lib.ew_rms_norm_grad_parts(1, 64) == 0 and 1 < lib.ew_rms_norm_grad_parts(1 << 30, 64) <= 4096
    assert lib.ew_rms_norm_grad_parts(1, 16384) == 1


def test_python_checks_before_the_library():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(2, 8, 8, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 8, dtype=torch.float8_e4m3fn), torch.zeros(4, 1, dtype=torch.float8_e8m0fnu)
    for call in (lambda: binding.scaled_rows(x), lambda: binding.scaled_pack(w), lambda: binding.swiglu_scaled(x), lambda: binding.rms_norm(x, x[0]),
                 lambda: binding.rms_norm_scaled(x, x[0]), lambda: binding.rms_norm_grad(x, x, x[0]), lambda: binding.scaled_mm(q, s, q[None], s[None])):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="float8"):
        binding.scaled_rows(x, torch.float16)
    with pytest.raises(ValueError, match="float8"):
        binding.scaled_mm(x, s, q[None], s[None])
