"""The norm's gradient where its kernels change (384 rows, 2048 columns and below), in place, and beyond 2^31 elements.

Tolerances as in the tests of the formula: sums of squares off by at most 2^-18, results by half a step of their type.
"""
import os
import subprocess
import sys

import pytest
import torch

from paper_2508_17624_b200 import binding

from test_gpu_scaled import NORM, grad_ref, randn, uneven

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# one launch up to 384 rows of 2048, of which a team of warps takes every 64th
SIZES = [(64, 2048), (65, 2048), (128, 2048), (129, 1024), (200, 999), (333, 2048), (384, 2048), (385, 2048), (384, 2049), (384, 2056), (65, 1333), (333, 1333), (384, 1025), (130, 1), (384, 7)]


def inputs(rows, width, dtype, with_dt, pad, seed=1):
    t, dy = uneven((rows, width), dtype, seed, 0.5, pad), randn((rows, width), dtype, seed + 1, 0.1, pad)
    return dy, t, (1 + 0.2 * randn((width,), FP32, seed + 2)).to(dtype), randn((rows, width), dtype, seed + 3, 0.1, pad) if with_dt else None


def check(got, dw, dy, t, w, dt, eps):
    rows, dtype = t.shape[0], t.dtype
    ref, mag, ref_dw, mag_dw = grad_ref(dy, t, w, dt, eps)
    tiny = 2.0 ** -25 if dtype == FP16 else 2.0 ** -134
    assert ((got.double() - ref).abs() <= torch.finfo(dtype).eps / 2 * ref.abs() + 4 * NORM * mag + tiny).all()
    # a thread's own additions (six rows a team, four teams, sixteen CTAs; otherwise as many rows as a CTA meets, and a tree)
    assert ((dw.double() - ref_dw).abs() <= (NORM + (rows / 592 + 40) * 2.0 ** -24) * mag_dw + 1e-40).all()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("with_dt", [True, False])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("rows,width", SIZES)
def test_norm_grad_of_few_rows(rows, width, pad, with_dt, dtype):
    """Two sets of inputs in turn, so that a value of an earlier row or call would show."""
    sets = [inputs(rows, width, dtype, with_dt, pad, seed) for seed in (1, 31)]
    first = [binding.rms_norm_grad(*s, 1e-5) for s in sets]
    for s, got in zip(sets, first):
        check(*got, *s, 1e-5)
    for _ in range(5):
        for s, got in zip(sets, first):
            again = binding.rms_norm_grad(*s, 1e-5)
            assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("rows,width,pad", [(333, 2048, 0), (333, 1333, 1), (385, 2048, 0), (2500, 256, 8), (2500, 512, 0), (9000, 1024, 0), (3000, 2048, 0), (3000, 1999, 1), (2500, 300, 1),
                                            (1500, 4096, 0), (700, 8192, 0), (600, 16384, 0), (600, 12345, 0)])
def test_norm_grad_in_place(rows, width, pad):
    """dt may be the result: each row is read before it is written, rows that are asked for ahead among them."""
    dy, t, w, dt = inputs(rows, width, BF16, True, pad)
    want, dw = binding.rms_norm_grad(dy, t, w, dt)
    for _ in range(3):
        there = torch.full((rows, width + pad), 7.0, dtype=BF16, device="cuda")
        at = there[:, pad:] if pad % 8 else there[:, : width]
        at.copy_(dt)
        got, dw2 = binding.rms_norm_grad(dy, t, w, at, out=at)
        assert got is at and torch.equal(got, want) and torch.equal(dw, dw2)
        assert (there[:, :pad] == 7).all() if pad % 8 else (there[:, width:] == 7).all()


def test_norm_grad_beyond_two_to_the_31_elements():
    """9 M rows of 256 whose last 64 alone are not zero, into a result that was NaN: as of those rows alone."""
    rows, width = 9_000_000, 256
    dy, t = (torch.zeros((rows, width), dtype=BF16, device="cuda") for _ in range(2))
    w = (1 + 0.2 * randn((width,), FP32, 3)).to(BF16)
    dy[-64:], t[-64:] = randn((64, width), BF16, 1), randn((64, width), BF16, 2)
    out = torch.full((rows, width), float("nan"), dtype=BF16, device="cuda")
    dt, dw = binding.rms_norm_grad(dy, t, w, out=out)
    assert dt is out and not out[:-64].any()
    check(dt[-64:], dw, dy[-64:], t[-64:], w, None, 1e-6)
    del dy, out
    dt, dw = binding.rms_norm_grad(t, t, w, t)
    assert not dt[:-64].any()
    check(dt[-64:], dw, t[-64:], t[-64:], w, t[-64:], 1e-6)


def test_norm_grad_of_few_rows_in_the_portable_cluster():
    """Where no cluster of sixteen CTAs fits: the same tests in a process that takes the one of eight, and its sums are of another order."""
    code = ("import sys, torch; sys.path.insert(0, 'tests'); import test_gpu_norm_limits as t\n"
            "for rows, width in t.SIZES:\n"
            "    for pad in (0, 3):\n"
            "        for with_dt in (True, False):\n"
            "            t.test_norm_grad_of_few_rows(rows, width, pad, with_dt, torch.bfloat16)\n"
            "dw = t.binding.rms_norm_grad(*t.inputs(384, 2048, torch.bfloat16, True, 0))[1]\n"
            "print('sum', dw.view(torch.int32).long().sum().item())\n")

    def run(**env):
        r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT, **env})
        assert r.returncode == 0, r.stderr[-2000:]
        return r.stdout.split()[-1]

    assert run(EW_DISABLE_CLUSTER16="1") != run()
