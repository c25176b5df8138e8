"""The operators in 8-bit floating point (blocks of 128 with a power-of-two scale) against their formulas in 64 bits.

Tolerances.  Blocks of given numbers are equal to the formula's.  A result rounded to type t is off by at most eps(t)/2 relative
(`torch.finfo(t).eps / 2`), and half a step of the type's smallest numbers.  The tensor core multiplies 8-bit values exactly and
adds 32 products and the running sum at a time, each addend cut off below the 24 bits of the largest one: a step
adds at most 33 units of 2^-23 of S = sum |a b|, and a sum of t terms is off by at most (t/32 + 1) * 33 * 2^-23 * S.
"""
import numpy as np
import pytest
import torch

from paper_2508_17624_b200 import binding

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
POWERS = torch.tensor([2.0 ** e for e in range(-127, 128)], dtype=torch.float64)


def randn(shape, dtype, seed, scale=1.0, pad=0):
    """A device tensor; `pad` more elements between its rows than they are long."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn((*shape[:-1], shape[-1] + pad), device="cuda", generator=g) * scale
    return wide.to(dtype)[..., : shape[-1]]


def room(width, step):
    return (width + step - 1) // step * step


def power(most, to):
    """The smallest power of two from 2^-127 on that is at least most / largest, in 64 bits."""
    powers = POWERS.to(most.device)
    return powers[torch.searchsorted(powers * LARGEST[to], most.double().contiguous())]


def as_bits(t):
    return t.contiguous().view(torch.uint8)


def ref_rows(x, to):
    """(q, scales) of finite rows whose values 32 bits hold."""
    rows, width = x.shape
    wide = torch.zeros((rows, room(width, 128)), dtype=torch.float64, device=x.device)
    wide[:, :width] = x.double()
    wide = wide.view(rows, -1, 128)
    s = power(wide.abs().amax(2), to)
    return (wide / s[..., None]).view(rows, -1)[:, :width].float().to(to), s.float().to(E8M0)


def ref_squares(w):
    g, n, k = w.shape
    wide = torch.zeros((g, room(n, 128), room(k, 128)), dtype=torch.float64, device=w.device)
    wide[:, :n, :k] = w.double()
    wide = wide.view(g, -1, 128, wide.shape[2] // 128, 128)
    s = power(wide.abs().amax((2, 4)), E4M3)
    return (wide / s[:, :, None, :, None]).reshape(g, wide.shape[1] * 128, -1)[:, :n, :k].float().to(E4M3), s.float().to(E8M0)


def values(q, scales):
    s = scales.float().double()
    if q.dim() == 2:
        return q.float().double() * s.repeat_interleave(128, 1)[:, : q.shape[1]]
    return q.float().double() * s.repeat_interleave(128, 1)[:, : q.shape[1]].repeat_interleave(128, 2)[:, :, : q.shape[2]]


def uneven(shape, dtype, seed, scale=1.0, pad=0):
    """Rows and columns of different sizes, so that a block's scale is its own."""
    x = randn(shape, dtype, seed, scale, pad)
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    x *= torch.exp2(torch.randint(-6, 7, (*shape[:-1], 1), device="cuda", generator=g)).to(dtype)
    blocks = torch.exp2(torch.randint(-4, 5, ((shape[-1] + 127) // 128,), device="cuda", generator=g)).repeat_interleave(128)[: shape[-1]]
    return x.mul_(blocks.to(dtype))


# ------------------------------------------------------------------------------------------ rows and weights
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("to", [E4M3, E5M2], ids=str)
@pytest.mark.parametrize("rows,width,pad", [(1, 1, 0), (1, 2048, 0), (3, 127, 0), (5, 128, 8), (2, 129, 7), (70, 264, 0), (4000, 520, 8), (3000, 333, 0), (3, 9000, 0)])
def test_rows(rows, width, pad, to, dtype):
    x = uneven((rows, width), dtype, 1, 0.5, pad)
    x[0, 0] = 0
    q, s = binding.scaled_rows(x, to)
    rq, rs = ref_rows(x, to)
    assert q.dtype == to and s.dtype == E8M0 and torch.equal(as_bits(s), as_bits(rs)) and torch.equal(as_bits(q), as_bits(rq))


def test_rows_every_exponent():
    """Largest values at and next to the powers of two where the scale changes, and down to the smallest numbers; zeros."""
    for to in (E4M3, E5M2):
        most = torch.cat([LARGEST[to] * 2.0 ** torch.arange(-100.0, 80.0, dtype=torch.float64), torch.tensor([0.0, 1e-40, 9.2e-41, 3e38])])
        for factor in (1.0, 1 + 2.0 ** -7, 1 - 2.0 ** -8):
            x = torch.zeros((most.numel(), 128), dtype=BF16, device="cuda")
            x[:, 5] = (most * factor).to(BF16)
            x[:, 6] = (most * factor / 3).to(BF16)
            x[:, 7] = (most * factor / 1000).to(BF16)
            q, s = binding.scaled_rows(x, to)
            rq, rs = ref_rows(x, to)
            assert torch.equal(as_bits(s), as_bits(rs)) and torch.equal(as_bits(q), as_bits(rq))


@pytest.mark.parametrize("width,pad", [(256, 0), (255, 0)])
def test_rows_not_finite(width, pad):
    x = randn((4, width), BF16, 3)
    clean_q, clean_s = binding.scaled_rows(x)
    x[0, 3], x[0, 130], x[1, 7], x[2, :128] = float("inf"), float("nan"), float("-inf"), float("nan")
    q, s = binding.scaled_rows(x)
    bad = ~x.isfinite()
    assert torch.equal(q.float().isnan(), bad)
    x[bad] = 0                                          # the others are as if these were not there
    rq, rs = ref_rows(x, E4M3)
    assert torch.equal(as_bits(s), as_bits(rs)) and torch.equal(q[~bad].float(), rq[~bad].float()) and torch.equal(as_bits(q[3]), as_bits(clean_q[3]))


def test_rows_into_place():
    """Results in the middle of larger tensors: what is around them stays."""
    x = randn((9, 200), BF16, 1)
    for left in (0, 1):
        q = torch.full((9, 240), 7, dtype=torch.uint8, device="cuda")
        s = torch.full((9, 9), 7, dtype=torch.uint8, device="cuda")
        out = q.view(E4M3)[:, left:left + 200], s.view(E8M0)[:, left:left + 2]
        got = binding.scaled_rows(x, out=out)
        rq, rs = ref_rows(x, E4M3)
        assert torch.equal(as_bits(got[0]), as_bits(rq)) and torch.equal(as_bits(got[1]), as_bits(rs))
        assert (q[:, :left] == 7).all() and (q[:, left + 200:] == 7).all() and (s[:, :left] == 7).all() and (s[:, left + 2:] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("shape,pad", [((1, 1, 1), 0), ((1, 128, 128), 0), ((3, 129, 130), 0), ((2, 300, 264), 8), ((5, 40, 640), 3), ((2048, 1, 16), 0)])
def test_pack(shape, pad, dtype):
    w = uneven(shape, dtype, 8, 0.1, pad)
    q, s = binding.scaled_pack(w)
    rq, rs = ref_squares(w)
    assert torch.equal(as_bits(s), as_bits(rs)) and torch.equal(as_bits(q), as_bits(rq))
    w[0, 0, 0] = float("inf")
    q, s = binding.scaled_pack(w)
    w[0, 0, 0] = 0
    rq, rs = ref_squares(w)
    assert torch.equal(as_bits(s), as_bits(rs)) and q[0, 0, 0].float().isnan() and torch.equal(as_bits(q).flatten()[1:], as_bits(rq).flatten()[1:])


# ------------------------------------------------------------------------------------------------- products
def near(got, ref, mag, terms, what="", more=0.0):
    tol = torch.finfo(got.dtype).eps / 2 * ref.abs() + (terms / 32 + 1) * 33 * 2.0 ** -23 * mag + more
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


def check_both(counts, n, k, row_type=E4M3, out_dtype=BF16, seed=0, first=0, behind=0):
    """Product and input gradient of one grouping.  `first` rows before the first group, `behind` after the last, all NaN."""
    rows, groups = first + int(sum(counts)) + behind, len(counts)
    ends = [first] + (first + np.cumsum(counts)).tolist()
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    w, ws = binding.scaled_pack(uneven((groups, n, k), BF16, seed + 3, 0.05))
    for call, width, wide in ((binding.scaled_mm, k, n), (binding.scaled_mm_dx, n, k)):
        x = uneven((rows, width), BF16, seed + 1, 2.0 ** -6)
        x[:first], x[ends[-1]:] = float("nan"), float("nan")
        q, s = binding.scaled_rows(x, row_type)
        out = torch.full((rows, wide), 7.0, dtype=out_dtype, device="cuda")
        assert call(q, s, w, ws, offsets, out=out) is out
        torch.cuda.synchronize()
        xd, wd = values(q, s), values(w, ws)
        if call is binding.scaled_mm:
            wd = wd.transpose(1, 2)
        for g in range(groups):
            i, j = ends[g], ends[g + 1]
            near(out[i:j], xd[i:j] @ wd[g], xd[i:j].abs() @ wd[g].abs(), width, (call.__name__, g))
        assert (out[:first] == 7).all() and (out[ends[-1]:] == 7).all()
    assert binding.last_operator_error() == 0


@pytest.mark.parametrize("n,k", [(128, 128), (16, 32), (128, 512), (256, 640), (40, 72), (264, 200), (513, 331)], ids=lambda v: str(v))
@pytest.mark.parametrize("counts", [[1], [0, 1, 0], [3, 0, 17, 1], [16, 15, 33, 64], [65, 0, 129, 1, 0], [257, 300, 0, 2], [511, 768, 1]],
                         ids=lambda c: "-".join(map(str, c)))
def test_products_ragged(counts, n, k):
    check_both(counts, n, k)


@pytest.mark.parametrize("row_type,out_dtype", [(E4M3, FP32), (E5M2, BF16), (E5M2, FP32), (E4M3, FP16)], ids=str)
@pytest.mark.parametrize("counts", [[0, 5, 70, 2], [300, 0, 440]], ids=lambda c: "-".join(map(str, c)))
def test_products_types(counts, row_type, out_dtype):
    check_both(counts, 136, 264, row_type, out_dtype, seed=3)


@pytest.mark.parametrize("counts", [[5, 0, 40], [400, 130]], ids=lambda c: "-".join(map(str, c)))
def test_products_rows_outside(counts):
    check_both(counts, 72, 136, seed=5, first=3, behind=21)


@pytest.mark.parametrize("rows,groups,n,k", [(1536, 96, 704, 512), (700, 5, 2816, 256), (4097, 16, 512, 1408), (6, 64, 2816, 2048)])
def test_products_layer_sizes(rows, groups, n, k):
    check_both(make_counts(rows, groups, 1, empty=(1,)), n, k, E4M3, FP32, seed=9)


@pytest.mark.parametrize("counts,n,k,out_dtype", [([210, 0, 1025], 264, 2200, FP32), ([3, 40, 0, 7], 1100, 2056, FP32), ([300, 700], 2049, 1032, FP32), ([40, 3], 24, 16700, FP16),
                                                  ([900, 3], 24, 16700, FP16), ([12], 40, 70000, BF16)], ids=str)
def test_products_long_sums_in_parts(counts, n, k, out_dtype):
    check_both(counts, n, k, E4M3, out_dtype, seed=11)


@pytest.mark.parametrize("rows", [40, 700])
@pytest.mark.parametrize("n,k", [(264, 2048), (2048, 520), (136, 5000)])
def test_products_of_one_sign_in_the_2_norm(n, k, rows):
    """fp32 results of positive operands: off by at most 1.5e-5 (two steps of 2^-23 of the sum an instruction of 32 terms, 2048 terms a part), which
    neither a 16-bit rounding on the way (1.4e-4 for fp16) nor a summed element left out (1/k) would pass."""
    w, ws = binding.scaled_pack(uneven((1, n, k), BF16, 1).abs_())
    for call, width in ((binding.scaled_mm, k), (binding.scaled_mm_dx, n)):
        q, s = binding.scaled_rows(uneven((rows, width), BF16, 2).abs_())
        got, wd = call(q, s, w, ws, out_dtype=FP32).double(), values(w, ws)[0]
        ref = values(q, s) @ (wd.t() if call is binding.scaled_mm else wd)
        assert (got - ref).norm() / ref.norm() <= 1.5e-5 and ((got - ref).abs() <= 1.5e-5 * ref).all()


@pytest.mark.parametrize("rows", [3000, 300000])
def test_products_most_groups(rows):
    check_both(make_counts(rows, 2048, 4, empty=range(0, 2048, 3)), 24, 32, out_dtype=FP32, seed=6)


def test_products_groups_that_take_turns():
    """Weights whose matrices interleave their rows, results in the middle of a larger tensor."""
    w = uneven((3, 72, 256), BF16, 1, 0.1)
    packed = binding.scaled_pack(w)
    turns = torch.zeros((72, 3, 272), dtype=torch.uint8, device="cuda").view(E4M3).transpose(0, 1)[:, :, :256]
    turned = binding.scaled_pack(w, out=(turns, torch.empty_like(packed[1])))
    assert torch.equal(as_bits(turned[0]), as_bits(packed[0])) and turned[0] is turns
    offsets = torch.tensor([0, 30, 31, 50], dtype=torch.int32, device="cuda")
    for call, width, wide in ((binding.scaled_mm, 256, 72), (binding.scaled_mm_dx, 72, 256)):
        q, s = binding.scaled_rows(uneven((50, width), BF16, 2))
        want = call(q, s, *packed, offsets)
        for left, room_ in ((8, 96 if wide == 72 else 280), (3, wide + 8), (0, wide + 1)):
            out = torch.full((50, room_), 7.0, dtype=BF16, device="cuda")
            call(q, s, *turned, offsets, out=out[:, left:left + wide])
            assert torch.equal(out[:, left:left + wide], want) and (out[:, :left] == 7).all() and (out[:, left + wide:] == 7).all()


def test_input_gradient_by_differences():
    """Whole numbers that e4m3 holds, so that every sum is exact: <dy, y(x + v) - y(x - v)> = 2 <dx, v>, to the last bit."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def whole(shape, most):
        return torch.randint(-most, most + 1, shape, device="cuda", generator=g).to(BF16)

    offsets = torch.tensor([0, 3, 3, 40, 300], dtype=torch.int32, device="cuda")
    x, v, dy, w = whole((300, 200), 6), whole((300, 200), 1), whole((300, 136), 4), whole((4, 136, 200), 4)
    packed = binding.scaled_pack(w)
    plus, minus = (binding.scaled_mm(*binding.scaled_rows(t), *packed, offsets, out_dtype=FP32).double() for t in (x + v, x - v))
    dx = binding.scaled_mm_dx(*binding.scaled_rows(dy, E5M2), *packed, offsets, out_dtype=FP32).double()
    assert torch.equal(values(*binding.scaled_rows(x + v)), (x + v).double()) and torch.equal(values(*binding.scaled_rows(dy, E5M2)), dy.double())
    assert float((dy.double() * (plus - minus)).sum()) == 2 * float((dx * v.double()).sum())


def test_products_without_offsets():
    w, ws = binding.scaled_pack(uneven((1, 200, 300), BF16, 1, 0.1))
    q, s = binding.scaled_rows(uneven((37, 300), FP16, 2))
    offsets = torch.tensor([0, 37], dtype=torch.int32, device="cuda")
    assert torch.equal(binding.scaled_mm(q, s, w, ws), binding.scaled_mm(q, s, w, ws, offsets))
    none = binding.scaled_mm(q[:0], s[:0], w, ws)
    assert none.shape == (0, 200) and none.dtype == BF16


# ------------------------------------------------------------------------------------------------- norm
def blocks_near(q, s, ref, rel, what=""):
    """Blocks of values known to `rel` relative: the scale is that of a value within rel of the largest, each value within half a step
    (of the type's smallest numbers at least) and rel of the formula's."""
    rows, width = ref.shape
    wide = torch.zeros((rows, room(width, 128)), dtype=torch.float64, device=ref.device)
    wide[:, :width] = ref
    most = wide.view(rows, -1, 128).abs().amax(2)
    scale = s.float().double()
    assert ((scale >= power(most * (1 - rel), q.dtype)) & (scale <= power(most * (1 + rel), q.dtype))).all(), what
    each = scale.repeat_interleave(128, 1)[:, :width]
    tol = (torch.finfo(q.dtype).eps / 2 * (1 + rel) + rel) * ref.abs() + each * 2.0 ** -10
    off = (values(q, s) - ref).abs()
    assert (off <= tol).all(), (what, float((off / tol.clamp(min=1e-300)).max()))


def norm_ref(t, w, eps):
    td = t.double()
    return td / ((td ** 2).mean(1, keepdim=True) + eps).sqrt() * w.double()


# A row's sum of squares is off by at most 72 steps of 2^-24 (eight adds a span and up to eight spans a lane, then trees), the root by half of
# that, and a few more for the root itself and two products: 2^-18 in all.
NORM = 2.0 ** -18


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("rows,width,pad", [(1, 1, 0), (1, 2048, 0), (3, 129, 0), (5, 300, 4), (70, 264, 8), (2500, 512, 0), (2500, 1000, 0), (1500, 2048, 8), (1500, 1333, 0), (3, 4000, 0),
                                            (2, 8192, 0), (2, 16384, 0), (2, 12345, 1)])
def test_norm(rows, width, pad, dtype):
    x, res = uneven((rows, width), dtype, 1, 0.5, pad), uneven((rows, width), dtype, 2, 1.0, pad)
    w = (1 + 0.2 * randn((width,), FP32, 3)).to(dtype)
    total = (x.float() + res.float()).to(dtype)
    tiny = 2.0 ** -25 if dtype == FP16 else 2.0 ** -134

    def check(y, ref):
        assert ((y.double() - ref).abs() <= (torch.finfo(dtype).eps / 2 + NORM) * ref.abs() + tiny).all()

    check(binding.rms_norm(x, w, eps=1e-5), norm_ref(x, w, 1e-5))
    y, t = binding.rms_norm(x, w, res, 1e-5)
    assert torch.equal(t, total)
    check(y, norm_ref(total, w, 1e-5))
    q, s = binding.rms_norm_scaled(x, w)
    blocks_near(q, s, norm_ref(x, w, 1e-6), NORM)
    q, s, y2, t2 = binding.rms_norm_scaled(x, w, res, 1e-5, with_y=True)
    assert torch.equal(y2, y) and torch.equal(t2, total)
    blocks_near(q, s, norm_ref(total, w, 1e-5), NORM)
    # in place: the residual stream is overwritten by its next value
    stream = res.clone()
    got = binding.rms_norm_scaled(x, w, stream, 1e-5, sum_out=stream)
    assert got[2] is stream and torch.equal(stream, total) and torch.equal(as_bits(got[0]), as_bits(q))


def test_norm_zeros_and_not_finite():
    x = randn((5, 256), BF16, 1)
    w = torch.ones(256, dtype=BF16, device="cuda")
    clean = binding.rms_norm(x, w)
    x[0], x[1, 3], x[2, 200] = 0, float("nan"), float("inf")
    y = binding.rms_norm(x, w)
    q, s = binding.rms_norm_scaled(x, w)
    assert not y[0].any() and y[1].isnan().all() and torch.equal(y[3:], clean[3:])
    assert not q[0].float().any() and q[1].float().isnan().all() and q[2, 200].float().isnan() and not q[2, :200].float().any()
    assert not binding.rms_norm(x[:1], w, eps=0.0).isfinite().any()          # 0 / 0


def grad_ref(dy, t, w, dt, eps):
    td, g = t.double(), dy.double() * w.double()
    r = 1 / ((td ** 2).mean(1, keepdim=True) + eps).sqrt()
    u = td * r
    out = r * (g - u * (g * u).mean(1, keepdim=True))
    mag = r * (g.abs() + u.abs() * (g * u).abs().mean(1, keepdim=True))
    if dt is not None:
        out, mag = out + dt.double(), mag + dt.double().abs()
    return out, mag, (dy.double() * u).sum(0), (dy.double() * u).abs().sum(0)


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("with_dt", [True, False])
@pytest.mark.parametrize("rows,width,pad", [(1, 1, 0), (1, 2048, 0), (3, 129, 0), (70, 264, 8), (593, 300, 4), (2500, 512, 0), (1300, 1333, 0), (3, 4000, 0), (700, 8192, 0), (900, 16384, 0),
                                            (2, 12345, 1)])
def test_norm_grad(rows, width, pad, with_dt, dtype):
    t, dy = uneven((rows, width), dtype, 1, 0.5, pad), randn((rows, width), dtype, 2, 0.1, pad)
    w = (1 + 0.2 * randn((width,), FP32, 3)).to(dtype)
    dt = randn((rows, width), dtype, 4, 0.1, pad) if with_dt else None
    got, dw = binding.rms_norm_grad(dy, t, w, dt, 1e-5)
    ref, mag, ref_dw, mag_dw = grad_ref(dy, t, w, dt, 1e-5)
    tiny = 2.0 ** -25 if dtype == FP16 else 2.0 ** -134
    assert ((got.double() - ref).abs() <= torch.finfo(dtype).eps / 2 * ref.abs() + 4 * NORM * mag + tiny).all()
    assert dw.dtype == FP32 and ((dw.double() - ref_dw).abs() <= (NORM + (rows / 592 + 40) * 2.0 ** -24) * mag_dw + 1e-40).all()
    again = binding.rms_norm_grad(dy, t, w, dt, 1e-5)
    assert torch.equal(again[0], got) and torch.equal(again[1], dw)


@pytest.mark.parametrize("with_dt", [True, False])
@pytest.mark.parametrize("rows,width", [(4000, 256), (2500, 512), (3000, 1000), (9000, 1024), (2500, 2048), (1500, 4096), (700, 8192), (900, 16384), (3000, 300)])
def test_norm_grad_reads_no_earlier_row(rows, width, with_dt):
    """Two sets of inputs in turn: what a call finds in shared memory is of the other set, and must not show."""
    sets = [(randn((rows, width), BF16, s, 0.1), randn((rows, width), BF16, s + 1, 0.5), 1 + randn((width,), BF16, s + 2, 0.2),
             randn((rows, width), BF16, s + 3, 0.1) if with_dt else None) for s in (10, 20)]
    first = [binding.rms_norm_grad(dy, t, w, dt) for dy, t, w, dt in sets]
    for (dy, t, w, dt), (got, dw) in zip(sets, first):
        ref, mag, ref_dw, mag_dw = grad_ref(dy, t, w, dt, 1e-6)
        assert ((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 4 * NORM * mag + 2.0 ** -134).all()
        assert ((dw.double() - ref_dw).abs() <= (NORM + (rows / 592 + 40) * 2.0 ** -24) * mag_dw + 1e-40).all()
    for _ in range(20):
        for (dy, t, w, dt), (got, dw) in zip(sets, first):
            again = binding.rms_norm_grad(dy, t, w, dt)
            assert torch.equal(again[0], got) and torch.equal(again[1], dw)


def test_norm_grad_by_differences():
    """Along a random direction against (f(t + e v) - f(t - e v)) / 2 e of the formula in 64 bits."""
    t, dy, w = randn((5, 48), FP16, 4), randn((5, 48), FP16, 5), (1 + 0.2 * randn((48,), FP32, 6)).to(FP16)
    dt, dw = binding.rms_norm_grad(dy, t, w)
    v, e = randn((5, 48), FP32, 7).double(), 1e-4

    def f(at, weight):
        return (at / ((at ** 2).mean(1, keepdim=True) + 1e-6).sqrt() * weight * dy.double()).sum()

    by_t = (f(t.double() + e * v, w.double()) - f(t.double() - e * v, w.double())) / (2 * e)
    # dt is rounded to fp16: each term is off by half a step; the differences by e^2 times a third derivative, below 1e-6
    assert abs(float((dt.double() * v).sum() - by_t)) <= float((dt.double() * v).abs().sum()) * 2.0 ** -11 + 1e-5
    z = randn((48,), FP32, 8).double()
    by_w = (f(t.double(), w.double() + e * z) - f(t.double(), w.double() - e * z)) / (2 * e)
    assert abs(float((dw.double() * z).sum() - by_w)) <= 1e-4


def test_norm_no_rows():
    x, w = randn((0, 64), BF16, 1), randn((64,), BF16, 2)
    assert binding.rms_norm(x, w).shape == (0, 64) and binding.rms_norm_scaled(x, w)[1].shape == (0, 1)
    dt, dw = binding.rms_norm_grad(x, x, w)
    assert dt.shape == (0, 64) and not dw.any()


# ------------------------------------------------------------------------------------------------- SwiGLU
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("rows,inter,pad", [(1, 1, 0), (1, 1408, 0), (3, 7, 5), (70, 264, 8), (6000, 24, 0), (5000, 131, 1), (3000, 1408, 0), (2, 9000, 0)])
def test_swiglu(rows, inter, pad, weights, dtype):
    h = randn((rows, 2 * inter), dtype, 1, 1.5, pad)
    h.clamp_(-7.9, 7.9)
    p = torch.rand(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) if weights else None
    g, u = h.double().chunk(2, dim=1)
    ref = g * torch.sigmoid(g) * u * (1.0 if p is None else p.double()[:, None])
    q, s = binding.swiglu_scaled(h, p)
    # the fast exponential and division: 2 + 1.2 |g| steps of 2^-23, two more for the division and a handful of products: 20 for |g| < 8
    blocks_near(q, s, ref, 20 * 2.0 ** -23)


@pytest.mark.parametrize("inter", [256, 200, 131])
def test_swiglu_large_weights_and_zeros(inter):
    """Row weights above one beside blocks of zeros and of the smallest numbers, weights of zero beside infinities."""
    h = randn((7, 2 * inter), BF16, 1).clamp_(-7.9, 7.9)
    p = torch.tensor([3.0, 100.0, 1e30, 2.5, 0.0, -4.0, 1e-30], device="cuda")
    h[0], h[1, :128], h[2, inter:] = 0, 0, 1e-37
    q, s = binding.swiglu_scaled(h, p)
    g, u = h.double().chunk(2, dim=1)
    ref = g * torch.sigmoid(g) * u * p.double()[:, None]
    blocks_near(q, s, ref, 20 * 2.0 ** -23)
    h[4, 5] = float("inf")                              # times a weight of zero
    q, s = binding.swiglu_scaled(h, p)
    assert q[4, 5].float().isnan() and q[4, 6:].float().isfinite().all() and not q[4, 6:].float().any()
