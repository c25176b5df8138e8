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


def near(got, ref, mag, terms, what="", more=0.0):
    """Elementwise: half a step of the result's type plus the sum's own error (`mag` = sum of |products|) plus `more`."""
    tol = torch.finfo(got.dtype).eps / 2 * ref.abs() + (terms / 16 + 1) * 17 * 2.0 ** -23 * mag + more
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


@pytest.mark.parametrize("counts,n,k", [([2100, 0, 1025], 264, 200), ([3, 40, 0, 7], 1100, 2056), ([300, 700], 2049, 1032)], ids=str)
def test_products_long_sums_in_parts(counts, n, k):
    """Contractions beyond 1024 terms with fp32 results: summed in parts, rows and gradients alike."""
    check_three(counts, n, k, BF16, FP32, seed=11)


def test_no_rows():
    w = randn((3, 16, 24), BF16, 0)
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    x, dy = randn((0, 24), BF16, 1), randn((0, 16), BF16, 2)
    assert binding.grouped_mm(x, w, offsets).shape == (0, 16)
    assert binding.grouped_mm_dx(dy, w, offsets).shape == (0, 24)
    assert not binding.grouped_mm_dw(dy, x, offsets).any()
    kept = torch.ones((3, 16, 24), dtype=FP32, device="cuda")
    assert (binding.grouped_mm_dw(dy, x, offsets, out=kept, accumulate=True) == 1).all()


# ------------------------------------------------------------------------------------------ 4-bit weights
PLACE = [0, 4, 1, 5, 2, 6, 3, 7]                        # nibble of weight 0..7 in its 32-bit word


def unpacked(q, scales):
    """The weights that (q, scales) stand for, in 64 bits."""
    s, n, half = q.shape
    words = q.cpu().numpy().view("<u4").astype(np.int64)
    levels = np.stack([(words >> (4 * p)) & 15 for p in PLACE], axis=-1).reshape(s, n, 2 * half)
    group = 2 * half // scales.shape[1]
    return (torch.from_numpy(levels).cuda() - 8).double() * scales.double().transpose(1, 2).repeat_interleave(group, dim=2)


def check_quant(slots, n_slots, n, k, group, dtype=BF16, out_dtype=None, per_row=None, seed=0, pad=0):
    pairs = slots.numel() if slots is not None else per_row
    rows = pairs // per_row if slots is not None else pairs
    x = randn((rows, k), dtype, seed + 1, 1.0, pad)
    q, scales = binding.quant_pack(randn((n_slots, n, k), dtype, seed, 0.05), group)
    y = binding.quant_mv(x, q, scales, slots, out_dtype=out_dtype)
    torch.cuda.synchronize()
    assert y.shape == (pairs, n) and y.dtype == (out_dtype or dtype)
    w, flat = unpacked(q, scales), [0] * pairs if slots is None else slots.reshape(-1).tolist()
    step = 1 if slots is None else per_row
    for s in sorted(set(flat)):
        at = [i for i, v in enumerate(flat) if v == s]
        if not 0 <= s < n_slots:
            assert not y[at].any()
            continue
        xd = x[[i // step for i in at]].double()
        # x may enter as fixed-point numbers whose largest in a group is above 4177855: rounding them costs at most 1/2, i.e.
        # 1/8355711 of the group's largest x, a weight
        most = xd.view(len(at), k // group, group).abs().amax(2, keepdim=True).expand(-1, -1, group).reshape(len(at), k)
        near(y[at], xd @ w[s].t(), xd.abs() @ w[s].abs().t(), 2 * k, ("slot", s), (most / 8355711 @ w[s].abs().t()))


def some_slots(tokens, per, n_slots, seed=0):
    r = np.random.RandomState(seed)
    return torch.from_numpy(np.stack([r.choice(n_slots, per, replace=False) for _ in range(tokens)]).astype(np.int32)).cuda()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("group,k", [(32, 32), (32, 96), (64, 192), (128, 128), (128, 1408), (64, 2048)])
@pytest.mark.parametrize("n", [8, 24, 264])
def test_quant_sizes(dtype, group, k, n):
    check_quant(some_slots(5, 2, 7), 7, n, k, group, dtype, per_row=2)
    check_quant(None, 1, n, k, group, dtype, FP32, per_row=3, seed=4, pad=8)


@pytest.mark.parametrize("tokens,per,n_slots", [(1, 1, 1), (1, 6, 64), (7, 3, 3), (40, 1, 1), (33, 2, 2), (150, 6, 8), (256, 6, 96), (600, 4, 300)])
@pytest.mark.parametrize("per_row", ["token", "pair"])
def test_quant_batches(tokens, per, n_slots, per_row):
    check_quant(some_slots(tokens, per, n_slots, 3), n_slots, 72, 512, 64, BF16, FP32, per_row=per if per_row == "token" else 1, seed=2)


@pytest.mark.parametrize("group", [32, 128])
def test_quant_longest_rows(group):
    """k = 16384: few rows of x fit a CTA at a time."""
    check_quant(some_slots(3, 2, 4), 4, 24, 16384, group, BF16, per_row=2)
    check_quant(None, 1, 40, 16384, group, FP16, FP32, per_row=50, seed=3)
    slots = torch.arange(2048, dtype=torch.int32, device="cuda").flip(0).contiguous()
    check_quant(slots, 2048, 8, 128, group, BF16, per_row=1)


def test_quant_pairs_without_a_slot():
    slots = some_slots(12, 6, 20, 5)
    slots[3] = -1
    slots[7, 2:] = -5
    check_quant(slots, 20, 48, 256, 32, per_row=6)
    check_quant(torch.full((4, 2), -1, dtype=torch.int32, device="cuda"), 3, 16, 128, 128, per_row=1)
    assert binding.last_operator_error() == 0
    slots[0, 0] = 20                                    # beyond the last slot: a row of zeros, reported
    check_quant(slots, 20, 48, 256, 32, per_row=6)
    assert binding.last_operator_error() == 1 and binding.last_operator_error() == 0


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
def test_quant_outliers_leave_the_other_values_their_bits(dtype):
    """One value of a group 2000 times the others, where the weights are zero: what is left is as exact as without it."""
    x, w = randn((2, 256), dtype, 1), randn((1, 64, 256), dtype, 2, 0.05)
    x[0, 77], w[:, :, 77] = 6000.0, 0
    q, scales = binding.quant_pack(w, 128)
    assert (unpacked(q, scales)[0, :, 77] == 0).all()
    y = binding.quant_mv(x, q, scales, out_dtype=FP32)
    ref = x.double() @ unpacked(q, scales)[0].t()
    rest = x.double().clone()
    rest[0, 77] = 0
    # fixed point: half a step, 6000 / 8355711, a value, against sums of 255 values of about 1
    assert (y - ref).norm() / ref.norm() <= 1e-3
    assert ((y - ref).abs() <= 6000 / 8355711 * unpacked(q, scales)[0].abs().sum(1) + 1e-5 * (rest.abs() @ unpacked(q, scales)[0].abs().t())).all()


def test_quant_rows_do_not_touch_one_another():
    slots = torch.tensor([[0, 1], [-1, -1], [1, 0]], dtype=torch.int32, device="cuda")
    x = randn((3, 256), BF16, 1)
    q, scales = binding.quant_pack(randn((2, 40, 256), BF16, 2, 0.05), 64)
    clean = binding.quant_mv(x, q, scales, slots)
    x[1] = float("nan")
    out = torch.full((6, 48), 7.0, dtype=BF16, device="cuda")
    binding.quant_mv(x, q, scales, slots, out=out[:, :40])
    assert torch.equal(out[:, :40], clean) and (out[:, 40:] == 7).all()
    x[0] = float("inf")
    got = binding.quant_mv(x, q, scales, slots)
    assert not got[:2].isfinite().any() and torch.equal(got[2:], clean[2:])


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("shape,group", [((1, 8, 32), 32), ((3, 40, 192), 64), ((5, 72, 640), 128), ((2, 8, 2048), 32)])
def test_quant_pack(dtype, shape, group):
    w = randn(shape, dtype, 8, 0.1, pad=3)
    w[0, 0, :group] = 0                                 # a group of zeros
    w[0, 1, 0] = 40.0                                   # a group with an outlier
    q, scales = binding.quant_pack(w, group)
    s, n, k = shape
    most = w.float().view(s, n, k // group, group).abs().amax(-1)
    assert torch.equal(scales, (most / torch.full_like(most, 7.0)).to(dtype).transpose(1, 2))
    wide = scales.float().transpose(1, 2).repeat_interleave(group, dim=2)
    level = torch.where(wide > 0, (w.float() / wide).round().clamp(-8, 7), torch.zeros_like(wide))
    assert torch.equal(unpacked(q, scales), level.double() * wide.double())
    assert ((unpacked(q, scales) - w.double()).abs() <= wide.double() * 0.5 + most.double().repeat_interleave(group, 2) * torch.finfo(dtype).eps / 2).all()


# ------------------------------------------------------------------------------------------------ SwiGLU
def swiglu_ref(h, p, da=None):
    """The formulas in 64 bits: act, or (dh, dp), each with the size of what is summed up in it."""
    g, u = h.double().chunk(2, dim=1)
    s, pp = torch.sigmoid(g), 1.0 if p is None else p.double()[:, None]
    if da is None:
        return pp * g * s * u, (pp * g * s * u).abs()
    d = da.double()
    dg, du, dp = pp * d * u * s * (1 + g * (1 - s)), pp * d * g * s, d * g * s * u
    return torch.cat((dg, du), 1), torch.cat(((pp * d * u * s).abs() * (1 + g.abs() * (1 - s)), du.abs()), 1), dp.sum(1), dp.abs().sum(1)


def close(got, ref, mag, sums=0):
    """Half a step of the type, and the fast exponential's error: at most 2 + 1.2 |g| steps of 2^-23, two more for the
    division and a handful of products, 20 for |g| < 8; `sums`: length of a sum in fp32."""
    tol = torch.finfo(got.dtype).eps / 2 * ref.abs() + (20 + sums) * 2.0 ** -23 * mag + (2.0 ** -25 if got.dtype == FP16 else 2.0 ** -134 if got.dtype == BF16 else 0)
    assert ((got.double() - ref).abs() <= tol).all(), float(((got.double() - ref).abs() / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("rows,inter,pad", [(1, 1, 0), (1, 1408, 0), (3, 7, 5), (70, 264, 8), (6000, 24, 0), (5000, 131, 1), (2, 9000, 0)])
def test_swiglu(rows, inter, pad, weights, dtype):
    h, da = randn((rows, 2 * inter), dtype, 1, 1.5, pad).clamp(-7.9, 7.9), randn((rows, inter), dtype, 2, 0.5, pad)
    h = randn((rows, 2 * inter), dtype, 1, 1.5, pad)
    h.clamp_(-7.9, 7.9)
    p = torch.rand(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) if weights else None
    out = torch.full((rows, inter + 3), 7.0, dtype=dtype, device="cuda")
    act = binding.swiglu(h, p, out=out[:, :inter])
    close(act, *swiglu_ref(h, p))
    assert (out[:, inter:] == 7).all()
    got = binding.swiglu_grad(da, h, p)
    dh, dh_mag, dp, dp_mag = swiglu_ref(h, p, da)
    close(got[0] if weights else got, dh, dh_mag)
    if weights:
        close(got[1], dp, dp_mag, inter)


def test_swiglu_extremes():
    """Saturated gates, infinities and NaN come out as the formula's."""
    g = torch.tensor([-200.0, -100.0, -88.5, 88.5, 100.0, 200.0, 0.0, float("inf"), float("-inf"), float("nan")], device="cuda")
    h = torch.cat((g, torch.full_like(g, 2.0))).to(BF16)[None]
    act = binding.swiglu(h)[0].float()
    assert torch.equal(act[:3], torch.zeros(3, device="cuda") * act[:3]) and (act[:3].abs() < 1e-30).all()
    assert torch.equal(act[3:6], (2 * h[0, 3:6].float()).to(BF16).float()) and act[6] == 0
    assert act[7] == float("inf") and act[8:].isnan().all()
    da = torch.ones_like(h[:, :10])
    dh = binding.swiglu_grad(da, h)[0].float()
    assert (dh[:3].abs() < 1e-30).all() and (dh[3:6] == 2).all() and dh[6] == 1


def test_swiglu_gradient_by_differences():
    """d act / d h along a random direction against (act(h + e v) - act(h - e v)) / 2 e of the formula in 64 bits."""
    h, da = randn((5, 48), FP16, 4, 1.0), randn((5, 24), FP16, 5, 1.0)
    p = torch.rand(5, device="cuda")
    dh, dp = binding.swiglu_grad(da, h, p)
    v, e = randn((5, 48), FP32, 6).double(), 1e-4

    def act(at, w):
        g, u = at.chunk(2, 1)
        return (w[:, None] * g * torch.sigmoid(g) * u * da.double()).sum()

    by_h = (act(h.double() + e * v, p.double()) - act(h.double() - e * v, p.double())) / (2 * e)
    # dh is rounded to fp16: each term is off by half a step; the differences by e^2 times a third derivative, below 1e-6
    assert abs(float((dh.double() * v).sum() - by_h)) <= float((dh.double() * v).abs().sum()) * 2.0 ** -11 + 1e-5
    q = torch.rand(5, device="cuda").double()
    by_p = (act(h.double(), p.double() + e * q) - act(h.double(), p.double() - e * q)) / (2 * e)
    assert abs(float((dp.double() * q).sum() - by_p)) <= 1e-4
