"""Limits of the stand-alone operators on the device: empty batches, long sums, the error word, failed calls, autograd."""
import ctypes as C

import pytest
import torch

from paper_2508_17624_b200 import binding, build
from paper_2508_17624_b200 import workloads as wl

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


# ---------------------------------------------------------------------------------------------- long sums
# The tensor core adds 16 products to the running sum at a time and cuts off at most two units of 2^-23 of it.  A running sum of
# terms of one sign averages half its end, so a part of `part` terms loses at most part / 16 units of its end, all parts
# together as much of the whole; the parts are added up in fp32, half a unit each.
PART = {FP16: 8192, BF16: 65536, FP32: 1024}
UNIT = 2.0 ** -23


def one_sign(shape, dtype, seed, top):
    """Values in (top / 2, top)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return ((torch.rand(shape, device="cuda", generator=g) * 0.5 + 0.5) * top).to(dtype)


def near_long(got, ref, mag, terms):
    part = min(terms, PART[got.dtype])
    tol = torch.finfo(got.dtype).eps / 2 * ref.abs() + (part / 16 + terms / part) * UNIT * mag + (2.0 ** -25 if got.dtype == FP16 else 0)
    off = (got.double() - ref).abs()
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("dtype,out_dtype,terms", [(FP16, FP16, 70001), (BF16, BF16, 300001), (FP16, FP32, 20003)], ids=str)
def test_long_sums_of_one_sign_keep_their_mean(dtype, out_dtype, terms):
    """A sum that is cut off term by term drifts towards zero; one made in parts does not, whatever its length."""
    dy, x = one_sign((terms, 64), dtype, 1, 16384 / terms), one_sign((terms, 72), dtype, 2, 1.0)
    ref = dy.double().t() @ x.double()
    ends = torch.tensor([0, terms], dtype=torch.int32, device="cuda")
    wide = terms + (-terms) % 8
    flat = [torch.nn.functional.pad(t.t(), (0, wide - terms)).contiguous()[:, :terms] for t in (dy, x)]
    results = [binding.grouped_mm_dw(dy, x, ends, out_dtype=out_dtype)[0]]
    # the same sums as a product and as an input gradient; 1 row block a group on one CTA, five on CTA pairs
    for copies in (1, 5):
        rows = flat[0].repeat(copies, 1) if copies > 1 else flat[0]
        rows = torch.nn.functional.pad(rows, (0, wide - terms)).contiguous()[:, :terms]
        o = torch.tensor([0, rows.shape[0]], dtype=torch.int32, device="cuda")
        y = binding.grouped_mm(rows, flat[1][None], o, out_dtype=out_dtype)
        dx = binding.grouped_mm_dx(rows, x[None], o, out_dtype=out_dtype)
        results += list(y.split(64)) + list(dx.split(64))
    half = torch.finfo(out_dtype).eps / 2
    for got in results:
        near_long(got, ref, ref, terms)
        # roundings of either sign: uniform within half a step, their mean over the elements within four deviations of zero
        drift = float(((got.double() - ref) / ref).mean())
        assert abs(drift) <= PART[out_dtype] / 16 * UNIT + 4 * half / (3 * ref.numel()) ** 0.5 + terms / PART[out_dtype] * UNIT, drift


@pytest.mark.parametrize("out_dtype", [FP16, FP32], ids=str)
@pytest.mark.parametrize("empty", [0, 400])
def test_long_and_short_groups_in_turn(empty, out_dtype):
    """Groups of many parts, of one and of none take turns in a CTA pair's accumulators; results repeat to the bit."""
    counts = [9000, 10, 17000, 0, 300, 8193, 8192, 64, 24577, 0, 16384, 1] + [0] * empty
    ends = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    g = torch.Generator(device="cuda").manual_seed(7)
    dy, x = ((torch.randn((sum(counts), w), device="cuda", generator=g) * 0.1).to(FP16) for w in (1000, 1096))
    dw = binding.grouped_mm_dw(dy, x, ends, out_dtype=out_dtype)
    more = binding.grouped_mm_dw(dy, x, ends, out=torch.ones_like(dw), accumulate=True)
    at = 0
    for i, c in enumerate(counts):
        a, b = dy[at:at + c].double(), x[at:at + c].double()
        at += c
        ref, mag = a.t() @ b, a.abs().t() @ b.abs()
        near_long(dw[i], ref, mag, max(c, 16))
        near_long(more[i], ref + 1, mag + 1, max(c, 16))
    for _ in range(5):
        assert torch.equal(dw, binding.grouped_mm_dw(dy, x, ends, out_dtype=out_dtype))
    assert binding.last_operator_error() == 0


@pytest.mark.parametrize("rows", [40, 700])
def test_long_contractions_over_many_tiles(rows):
    """y and dx of 16-bit results with a summed axis of several parts, more tiles than CTAs; short sums before and after."""
    k, n, groups = 8192 * 2 + 72, 1096, 6
    g = torch.Generator(device="cuda").manual_seed(rows)
    offsets = torch.tensor([0, 5, 5, rows // 2, rows - 9, rows - 8, rows], dtype=torch.int32, device="cuda")
    x, w = torch.randn((rows, k), device="cuda", generator=g).to(FP16), (torch.randn((groups, n, k), device="cuda", generator=g) * 0.05).to(FP16)
    y = binding.grouped_mm(x, w, offsets)
    wt = w.transpose(1, 2).contiguous()
    dx = binding.grouped_mm_dx(x, wt, offsets)
    for s, (i, j) in enumerate(zip(offsets.tolist()[:-1], offsets.tolist()[1:])):
        ref, mag = x[i:j].double() @ w[s].double().t(), x[i:j].double().abs() @ w[s].double().abs().t()
        near_long(y[i:j], ref, mag, k)
        near_long(dx[i:j], ref, mag, k)
    assert torch.equal(y, binding.grouped_mm(x, w, offsets)) and torch.equal(dx, binding.grouped_mm_dx(x, wt, offsets))
    assert binding.last_operator_error() == 0


# ---------------------------------------------------------------------------------------------- the error word
class _Device(C.Structure):                             # what the library keeps of a device
    _fields_ = [("sm_count", C.c_int), ("err", C.c_void_p), ("encode", C.c_void_p)]


def test_what_was_not_reported_stays_in_the_error_word():
    """A timeout and a bad index: the first call reports the one, the second the other.  (No operator's wait runs out, so the
    word is written by the test.)"""
    assert binding.last_operator_error() == 0
    device = C.POINTER(_Device)()
    assert binding.lib()._ZN2ew3ops12device_stateEiPPKNS0_6DeviceE(0, C.byref(device)) == 0
    for bits, codes in ((2 | 4, [7, 1, 0]), (2, [7, 0]), (4, [1, 0])):
        word = C.c_int(bits)
        assert C.CDLL("libcuda.so.1").cuMemcpyHtoD_v2(C.c_uint64(device.contents.err), C.byref(word), C.c_size_t(4)) == 0
        assert [binding.last_operator_error() for _ in codes] == codes


def test_a_failed_call_does_not_fail_the_next_one():
    """An operator on a device that is not there fails; the pool's next call of the same thread does not see that error."""
    cfg = wl.CONFIGS["c0"]
    pool = binding.Pool.from_config(cfg)
    binding.load_model(pool, cfg, adapters=[])
    ids = torch.zeros((8, cfg.top_k), dtype=torch.int32, device="cuda")
    aid = torch.full((8,), -1, dtype=torch.int32, device="cuda")
    h, out = torch.zeros((4, 32), dtype=BF16, device="cuda"), torch.zeros((4, 16), dtype=BF16, device="cuda")
    lib = binding.lib()
    assert lib.ew_swiglu(63, 0, h.data_ptr(), 32, None, 4, 16, out.data_ptr(), 16, None) == 6          # EW_ERR_CUDA
    assert lib.ew_last_error_string()
    pool.reroute(0, ids, aid)
    assert lib.ew_last_operator_error(63, C.byref(C.c_int32())) == 6
    pool.reroute(0, ids, aid)
    pool.destroy()


# ---------------------------------------------------------------------------------------------- autograd
class Experts(torch.autograd.Function):
    """An expert FFN over sorted rows, the operators in both of its halves."""

    @staticmethod
    def forward(ctx, x, w13, w2, p, offsets):
        h = binding.grouped_mm(x, w13, offsets)
        act = binding.swiglu(h, p)
        ctx.save_for_backward(x, w13, w2, p, offsets, h, act)
        return binding.grouped_mm(act, w2, offsets)

    @staticmethod
    def backward(ctx, dy):
        x, w13, w2, p, offsets, h, act = ctx.saved_tensors
        dh, dp = binding.swiglu_grad(binding.grouped_mm_dx(dy, w2, offsets), h, p)
        return binding.grouped_mm_dx(dh, w13, offsets), binding.grouped_mm_dw(dh, x, offsets), binding.grouped_mm_dw(dy, act, offsets), dp, None


def test_operators_inside_an_autograd_function():
    """Parameters that need gradients reach the operators through a Function; by themselves they are refused, except for packing."""
    g = torch.Generator(device="cuda").manual_seed(3)
    offsets = torch.tensor([0, 7, 7, 30], dtype=torch.int32, device="cuda")
    x, w13, w2 = (torch.randn(s, device="cuda", generator=g).mul_(f).to(FP16).requires_grad_() for s, f in (((30, 64), 1.0), ((3, 96, 64), 0.1), ((3, 64, 48), 0.1)))
    p = torch.rand(30, device="cuda", generator=g).requires_grad_()
    with pytest.raises(ValueError, match="autograd"):
        binding.grouped_mm(x, w13, offsets)
    y = Experts.apply(x, w13, w2, p, offsets)
    dy = torch.randn(y.shape, device="cuda", generator=g).to(FP16)
    y.backward(dy)
    x64, a64, b64, p64 = (t.detach().double().requires_grad_() for t in (x, w13, w2, p))
    parts = []
    for s, (i, j) in enumerate(((0, 7), (7, 7), (7, 30))):
        gate, up = (x64[i:j] @ a64[s].t()).chunk(2, 1)
        parts.append((p64[i:j, None] * gate * torch.sigmoid(gate) * up) @ b64[s].t())
    ref = torch.cat(parts)
    ref.backward(dy.double())
    # the fp16 roundings on the way (h, act, d_act, dh, the result) are half a step each, h's through silu's slope on both halves
    for got, want in ((y, ref), (x.grad, x64.grad), (w13.grad, a64.grad), (w2.grad, b64.grad), (p.grad, p64.grad)):
        assert float((got.detach().double() - want.detach()).norm() / want.detach().norm()) <= 6 * 2.0 ** -11
    q, scales = binding.quant_pack(w13, 32)
    assert not scales.requires_grad
    with torch.no_grad():
        assert not binding.quant_mv(x, q[:1], scales[:1]).requires_grad


def test_as_many_pairs_as_a_call_takes():
    """2^31 - 1 pairs of one row of x, a million launches: the last ones, and some of the others."""
    pairs = 2 ** 31 - 1
    g = torch.Generator(device="cuda").manual_seed(2)
    x, (q, scales) = torch.randn((1, 32), device="cuda", generator=g).to(BF16), binding.quant_pack(torch.randn((3, 8, 32), device="cuda", generator=g).to(BF16), 32)
    slots = torch.zeros((pairs,), dtype=torch.int32, device="cuda")
    slots[-9:] = torch.tensor([1, 2, 0, -1, 2, 1, 0, 0, 2], dtype=torch.int32)
    slots[1000003::1000003] = 1
    every = torch.cat([binding.quant_mv(x, q, scales, torch.full((1,), s, dtype=torch.int32, device="cuda")) for s in (0, 1, 2, -1)])
    y = binding.quant_mv(x, q, scales, slots)
    for at in (slice(0, 5000), slice(pairs - 5000, pairs), slice(1000003, None, 1000003), slice(7, None, 999983)):
        assert torch.equal(y[at], every[slots[at].long()])
    assert binding.last_operator_error() == 0


@pytest.mark.parametrize("n,k", [(72, 136), (300, 264)])
def test_groups_that_take_turns_row_by_row(n, k):
    """w, dw and what is packed as the middle dimension of an [n, groups, k] tensor: the same bits as with groups apart."""
    groups, counts = 4, [5, 0, 150, 70]
    offsets = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    g = torch.Generator(device="cuda").manual_seed(n)
    x, dy = (torch.randn((sum(counts), v), device="cuda", generator=g).to(BF16) for v in (k, (n + 7) // 8 * 8))
    dy = dy[:, :n]
    w = (torch.randn((groups, n, k), device="cuda", generator=g) * 0.05).to(BF16)
    turns = w.transpose(0, 1).contiguous().transpose(0, 1)
    assert turns.stride() == (k, groups * k, 1)
    for fn, rows in ((binding.grouped_mm, x), (binding.grouped_mm_dx, dy)):
        assert torch.equal(fn(rows, turns, offsets), fn(rows, w, offsets))
    for rows in (slice(None), slice(0, 0)):
        ends = offsets if rows == slice(None) else torch.zeros_like(offsets)
        whole = torch.full((n, groups + 1, k), 7.0, device="cuda")
        out = whole[:, :groups].transpose(0, 1)
        want = binding.grouped_mm_dw(dy[rows], x[rows], ends, out_dtype=FP32)
        assert torch.equal(binding.grouped_mm_dw(dy[rows], x[rows], ends, out=out), want) and (whole[:, groups] == 7).all()
        assert torch.equal(binding.grouped_mm_dw(dy[rows], x[rows], ends, out=out, accumulate=True), 2 * want)
    if n % 8 == 0:
        for a, b in zip(binding.quant_pack(turns[:, :, :128], 64), binding.quant_pack(w[:, :, :128], 64)):
            assert torch.equal(a, b)
