"""The stand-alone expert operators against their formulas in 64 bits.

Tolerances.  A result rounded to type t is off by at most eps(t)/2 relative (`torch.finfo(t).eps / 2`).  Sums are kept in
fp32: the tensor core adds 16 products and the running sum at a time, each addend cut off below the 24 bits of the largest
one, so a step adds at most 17 units of 2^-23 of S = sum |a b| and a sum of t terms is off by at most
(t/16 + 1) * 17 * 2^-23 * S.
"""
import numpy as np
import pytest
import torch

from paper_2508_17624_b200 import binding

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def near(got, ref, mag, terms, what=""):
    """Elementwise: half a step of the result's type plus the sum's own error (`mag` = sum of |products|)."""
    tol = torch.finfo(got.dtype).eps / 2 * ref.abs() + (terms / 16 + 1) * 17 * 2.0 ** -23 * mag
    if got.dtype == FP16:
        tol = tol + 2.0 ** -25                          # half a step of the subnormals
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((off / tol.clamp(min=1e-300)).max()), bad.nonzero()[:4].tolist())


def make_counts(rows, groups, seed, empty=()):
    r = np.random.RandomState(seed)
    p = np.exp(r.randn(groups))
    for g in empty:
        p[g] = 0
    return r.multinomial(rows, p / p.sum())


def randn(shape, dtype, seed, scale=1.0, pad=0):
    """A device tensor; `pad` more elements between its rows than they are long."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn((*shape[:-1], shape[-1] + pad), device="cuda", generator=g) * scale
    return wide.to(dtype)[..., : shape[-1]]


def up8(v):
    return (8 - v % 8) % 8


def check_three(counts, n, k, dtype, out_dtype, seed=0, first=0, behind=0, pad=0):
    """All three products of one grouping.  `first` rows before the first group, `behind` after the last, all NaN."""
    rows, groups = first + int(sum(counts)) + behind, len(counts)
    ends = [first] + (first + np.cumsum(counts)).tolist()
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x = randn((rows, k), dtype, seed + 1, 1.0, pad + up8(k))
    dy = randn((rows, n), dtype, seed + 2, 0.25, pad + up8(n))
    w = randn((groups, n, k), dtype, seed + 3, 0.05, pad + up8(k))
    for t in (x, dy):
        t[:first] = float("nan")
        t[ends[-1]:] = float("nan")
    y = torch.full((rows, n), 7.0, dtype=out_dtype, device="cuda")
    dx = torch.full((rows, k), 7.0, dtype=out_dtype, device="cuda")
    assert binding.grouped_mm(x, w, offsets, out=y) is y
    binding.grouped_mm_dx(dy, w, offsets, out=dx)
    dw = binding.grouped_mm_dw(dy, x, offsets, out_dtype=out_dtype)
    more = binding.grouped_mm_dw(dy, x, offsets, out=torch.ones_like(dw), accumulate=True)
    torch.cuda.synchronize()
    for g in range(groups):
        i, j = ends[g], ends[g + 1]
        xd, yd, wd = x[i:j].double(), dy[i:j].double(), w[g].double()
        near(y[i:j], xd @ wd.t(), xd.abs() @ wd.abs().t(), k, ("y", g))
        near(dx[i:j], yd @ wd, yd.abs() @ wd.abs(), n, ("dx", g))
        ref, mag = yd.t() @ xd, yd.abs().t() @ xd.abs()
        near(dw[g], ref, mag, j - i, ("dw", g))
        near(more[g], ref + 1, mag + 1, j - i + 16, ("dw accumulated", g))
        if i == j:
            assert not dw[g].any() and (more[g] == 1).all()
    for t in (y, dx):
        assert (t[:first] == 7).all() and (t[ends[-1]:] == 7).all()
    assert binding.last_operator_error() == 0


@pytest.mark.parametrize("counts", [[1], [0, 1, 0], [3, 0, 17, 1], [16, 15, 33, 64], [65, 0, 129, 1, 0], [257, 300, 0, 2], [511, 768, 1]],
                         ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("n,k", [(8, 8), (40, 72), (128, 64), (264, 200), (513, 331)], ids=lambda v: str(v))
def test_products_ragged(counts, n, k):
    check_three(counts, n, k, BF16, BF16)


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, FP32), (FP16, FP16), (FP16, FP32)], ids=str)
@pytest.mark.parametrize("counts", [[0, 5, 70, 2], [300, 0, 40]], ids=lambda c: "-".join(map(str, c)))
def test_products_types(counts, dtype, out_dtype):
    check_three(counts, 136, 264, dtype, out_dtype, seed=3)


@pytest.mark.parametrize("counts", [[5, 0, 40], [400, 130]], ids=lambda c: "-".join(map(str, c)))
def test_products_strides_and_rows_outside(counts):
    check_three(counts, 72, 136, BF16, BF16, seed=5, first=3, behind=21, pad=24)


@pytest.mark.parametrize("rows,groups,n,k", [(1536, 96, 704, 512), (700, 5, 2816, 256), (4097, 16, 512, 1408), (6, 64, 2816, 2048)])
def test_products_layer_sizes(rows, groups, n, k):
    check_three(make_counts(rows, groups, 1, empty=(1,)), n, k, BF16, FP32, seed=9)


def test_no_rows():
    w = randn((3, 16, 24), BF16, 0)
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    x, dy = randn((0, 24), BF16, 1), randn((0, 16), BF16, 2)
    assert binding.grouped_mm(x, w, offsets).shape == (0, 16)
    assert binding.grouped_mm_dx(dy, w, offsets).shape == (0, 24)
    assert not binding.grouped_mm_dw(dy, x, offsets).any()
    kept = torch.ones((3, 16, 24), dtype=FP32, device="cuda")
    assert (binding.grouped_mm_dw(dy, x, offsets, out=kept, accumulate=True) == 1).all()
