"""The operators in 8-bit floating point as a user runs them: a decode layer from the norm to the combined result, a training
step through autograd, captured and replayed calls, streams and threads, and what documentation allows and sizes make rare."""
import threading

import numpy as np
import pytest
import torch

from paper_2508_17624_b200 import binding

from test_gpu_operators_run import HALF_STEP, Layer, rel
from test_gpu_scaled import as_bits, near, randn, ref_rows, uneven, values

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
E4M3_STEP = 2.0 ** -4                                   # half a step, relative


def rows_of(blocks, index):
    """Rows of blocks by index, as a dispatch gathers them."""
    return tuple(t.view(torch.uint8)[index].view(t.dtype) for t in blocks)


@pytest.mark.parametrize("n", [1, 5, None])
def test_decode_layer_with_eight_bit_experts(n):
    """Norm with the residual, routing with the pool, the experts' products from 8-bit weights and rows, the sum over a token's experts:
    against the formula in 64 bits with the values that the blocks stand for, and near the layer with 16-bit weights."""
    L = Layer()
    cfg = L.cfg
    n = cfg.n_tokens if n is None else n
    hidden, k = L.x[:n], cfg.top_k
    residual, w_norm = randn((n, cfg.hidden), BF16, 1), (1 + 0.1 * randn((cfg.hidden,), FP32, 2)).to(BF16)
    w13, w2 = binding.scaled_pack(L.w13), binding.scaled_pack(L.w2)

    q, s, y, stream = binding.rms_norm_scaled(hidden, w_norm, residual, with_y=True, sum_out=residual)
    ids, slots = (torch.empty((n, k), dtype=torch.int32, device="cuda") for _ in range(2))
    p, counts = torch.empty((n, k), device="cuda"), torch.empty((cfg.num_slots,), dtype=torch.int32, device="cuda")
    L.pool.route_noalloc(0, y, L.aid[:n].contiguous(), ids, p, slots, counts)
    offsets = torch.cat((counts.new_zeros(1), counts.cumsum(0))).to(torch.int32)
    order = slots.reshape(-1).argsort(stable=True)
    token, row_p = order // k, p.reshape(-1)[order].contiguous()
    h = binding.scaled_mm(*rows_of((q, s), token), *w13, offsets)
    act = binding.swiglu_scaled(h, row_p)
    out = torch.zeros((n, cfg.hidden), device="cuda").index_add(0, token, binding.scaled_mm(*act, *w2, offsets, out_dtype=FP32))

    assert residual is stream
    td = stream.double()
    y64 = td / ((td ** 2).mean(1, keepdim=True) + 1e-6).sqrt() * w_norm.double()
    assert rel(values(q, s), y64) <= E4M3_STEP and rel(y, y64) <= HALF_STEP
    flat = slots.reshape(-1)[order].long()
    g, u = torch.einsum("ri,roi->ro", values(q, s)[token], values(*w13)[flat]).chunk(2, 1)
    act64 = row_p.double()[:, None] * g * torch.sigmoid(g) * u
    # h is rounded to bf16, act to e4m3 (uniform within a step: a third of the largest error in the 2-norm is an upper estimate of
    # the mean; the whole is allowed)
    assert rel(values(*act), act64) <= E4M3_STEP + 2 * HALF_STEP
    ref = torch.zeros_like(td).index_add(0, token, torch.einsum("ri,rhi->rh", values(*act), values(*w2)[flat]))
    assert rel(out, ref) <= 1e-5
    # and the layer with 16-bit weights: five roundings to e4m3 on the way of each term (y, gate, up, act, down), independent of one another
    g, u = torch.einsum("ri,roi->ro", y.double()[token], L.w13.double()[flat]).chunk(2, 1)
    full = torch.zeros_like(td).index_add(0, token, torch.einsum("ri,rhi->rh", row_p.double()[:, None] * g * torch.sigmoid(g) * u, L.w2.double()[flat]))
    assert rel(out, full) <= 5 ** 0.5 * E4M3_STEP
    assert L.pool.last_device_error() == 0 and binding.last_operator_error() == 0


class Experts(torch.autograd.Function):
    """Norm and experts with 8-bit products: forward and input gradients from blocks, weight gradients from the 16-bit rows."""

    @staticmethod
    def forward(ctx, x, residual, w_norm, w13, w2, offsets):
        q, s, y, t = binding.rms_norm_scaled(x, w_norm, residual, with_y=True)
        p13, p2 = binding.scaled_pack(w13), binding.scaled_pack(w2)
        h = binding.scaled_mm(q, s, *p13, offsets)
        act = binding.swiglu(h)
        ctx.save_for_backward(t, w_norm, y, h, act, offsets, *p13, *p2)
        return binding.scaled_mm(*binding.scaled_rows(act), *p2, offsets), t

    @staticmethod
    def backward(ctx, d_out, dt):
        t, w_norm, y, h, act, offsets, *packed = ctx.saved_tensors
        d_out = d_out.contiguous()
        d_act = binding.scaled_mm_dx(*binding.scaled_rows(d_out, E5M2), *packed[2:], offsets)
        dw2 = binding.grouped_mm_dw(d_out, act, offsets)
        dh = binding.swiglu_grad(d_act, h)
        dw13 = binding.grouped_mm_dw(dh, y, offsets)
        dy = binding.scaled_mm_dx(*binding.scaled_rows(dh, E5M2), *packed[:2], offsets)
        dx, dw = binding.rms_norm_grad(dy, t, w_norm, dt.contiguous())
        return dx, dx, dw.to(w_norm.dtype), dw13, dw2, None


def training_leaves(rows=200, groups=4, hidden=384, inter=256):
    counts = np.array([0, 70, 1, rows - 71])
    offsets = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda")
    leaves = [randn((rows, hidden), BF16, 1), randn((rows, hidden), BF16, 2), (1 + 0.1 * randn((hidden,), FP32, 3)).to(BF16),
              randn((groups, 2 * inter, hidden), BF16, 4, 0.05), randn((groups, hidden, inter), BF16, 5, 0.05)]
    return [t.requires_grad_() for t in leaves], offsets, randn((rows, hidden), BF16, 6, 0.1), randn((rows, hidden), BF16, 7, 0.1)


def test_training_step_through_autograd():
    """Gradients of the whole chain against the formula's in 64 bits without any rounding to 8 bits."""
    leaves, offsets, g_out, g_t = training_leaves()
    out, t = Experts.apply(*leaves, offsets)
    torch.autograd.backward((out, t), (g_out, g_t))
    exact = [v.detach().double().requires_grad_() for v in leaves]
    x, r, w, w13, w2 = exact
    s = x + r
    y = s / ((s ** 2).mean(1, keepdim=True) + 1e-6).sqrt() * w
    ref = []
    for g, (i, j) in enumerate(zip(offsets.tolist()[:-1], offsets.tolist()[1:])):
        a, b = (y[i:j] @ w13[g].t()).chunk(2, 1)
        ref.append((a * torch.sigmoid(a) * b) @ w2[g].t())
    ref = torch.cat(ref)
    torch.autograd.backward((ref, s), (g_out.double(), g_t.double()))
    assert rel(out.detach(), ref.detach()) <= 5 ** 0.5 * E4M3_STEP
    # what lies between a gradient and its exact value: roundings to e4m3 (half a step 2^-4 at most) and e5m2 (2^-3), a dozen at most on
    # the longest way, independent of one another
    for got, want in zip(leaves, exact):
        assert rel(got.grad, want.grad) <= (6 * 2.0 ** -8 + 6 * 2.0 ** -6) ** 0.5
    assert not leaves[3].grad[0].any()                  # a group without rows


def test_backward_captured_while_an_eager_graph_lives():
    leaves, offsets, g_out, g_t = training_leaves()
    Experts.apply(*leaves, offsets)                     # warm
    alive = Experts.apply(*leaves, offsets)             # an eager graph of the same leaves
    torch.cuda.synchronize()

    def step():
        with torch.no_grad():
            q, s, y, t = binding.rms_norm_scaled(leaves[0], leaves[2], leaves[1], with_y=True)
            return binding.rms_norm_grad(g_out, t, leaves[2], g_t)

    eager = [v.clone() for v in step()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, eager))
    torch.autograd.backward(alive, (g_out, g_t))
    assert leaves[0].grad.isfinite().all()


def test_training_step_captured():
    """Forward and backward through autograd in a graph: replays give the eager step's gradients."""
    leaves, offsets, g_out, g_t = training_leaves()

    def step():
        for v in leaves:
            v.grad = None
        torch.autograd.backward(Experts.apply(*leaves, offsets), (g_out, g_t))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    eager = [v.grad.clone() for v in leaves]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for v in leaves:
        v.grad.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(v.grad, e) for v, e in zip(leaves, eager))


def every_operator(seed=0):
    """One call of each, and their results as bits."""
    x, r, w = uneven((300, 512), BF16, seed + 1), uneven((300, 512), BF16, seed + 2), randn((512,), BF16, seed + 3)
    weights = randn((8, 384, 512), BF16, seed + 4, 0.05)
    many = uneven((700, 512), BF16, seed + 5)           # beyond the rows that the norm's gradient takes in one launch
    offsets = torch.tensor([0, 10, 10, 90, 130, 200, 201, 280, 300], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()

    def call():
        q, s, y, t = binding.rms_norm_scaled(x, w, r, with_y=True)
        packed = binding.scaled_pack(weights)
        h = binding.scaled_mm(q, s, *packed, offsets)
        act = binding.swiglu_scaled(h, torch.ones(300, device="cuda"))
        back = binding.scaled_mm_dx(*binding.scaled_rows(h, E5M2), *packed, offsets, out_dtype=FP32)
        dense = binding.scaled_mm(q[:7], s[:7], packed[0][:1], packed[1][:1])
        return [q, s, y, t, *packed, h, *act, back, dense, binding.rms_norm(x, w), *binding.rms_norm_grad(y, t, w, r), *binding.rms_norm_grad(many, many, w)]
    return call


def equal(a, b):
    return all(torch.equal(as_bits(u.contiguous()) if u.element_size() == 1 else u, as_bits(v.contiguous()) if v.element_size() == 1 else v) for u, v in zip(a, b))


def test_streams_and_repeated_calls_give_the_same_bits():
    call = every_operator()
    first = call()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for _ in range(5):
        for st in streams:
            with torch.cuda.stream(st):
                results.append(call())
    torch.cuda.synchronize()
    assert all(equal(first, r) for r in results) and binding.last_operator_error() == 0


def test_two_captured_graphs():
    """Two graphs of every operator, replayed in turn and at once on two streams: each keeps its own workspace."""
    calls = [every_operator(s) for s in (0, 50)]
    eager = [c() for c in calls]
    torch.cuda.synchronize()
    graphs, got = [], []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(c())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert equal(got[0], eager[0]) and equal(got[1], eager[1])


def test_threads():
    """Calls from several threads at once, each the thread's first on the GPU."""
    call = every_operator(9)
    first, results, errors = call(), [None] * 4, []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                results[i] = call()
                torch.cuda.current_stream().synchronize()
        except Exception as e:                          # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and all(equal(first, r) for r in results)


@pytest.mark.parametrize("ends", [[0, 9, 5, 20, 30], [0, 5, 9, 40, 30], [-3, 5, 9, 20, 30]], ids=str)
def test_bad_offsets_are_clamped_and_reported(ends):
    x, w = uneven((30, 256), BF16, 1), binding.scaled_pack(randn((4, 128, 256), BF16, 2, 0.05))
    blocks = binding.scaled_rows(x)
    out = torch.full((30, 128), 7.0, dtype=BF16, device="cuda")
    binding.scaled_mm(*blocks, *w, torch.tensor(ends, dtype=torch.int32, device="cuda"), out=out)
    assert binding.last_operator_error() == 1 and binding.last_operator_error() == 0
    fixed = np.maximum.accumulate(np.clip(ends, 0, 30)).tolist()
    assert torch.equal(out, binding.scaled_mm(*blocks, *w, torch.tensor(fixed, dtype=torch.int32, device="cuda"), out=torch.full_like(out, 7.0)))


@pytest.mark.parametrize("out_dtype", [BF16, FP32], ids=str)
def test_not_finite_values_stay_in_their_rows(out_dtype):
    x, w = uneven((300, 256), BF16, 1), binding.scaled_pack(randn((2, 136, 256), BF16, 2, 0.05))
    offsets = torch.tensor([0, 290, 300], dtype=torch.int32, device="cuda")
    clean = binding.scaled_mm(*binding.scaled_rows(x), *w, offsets, out_dtype=out_dtype)
    x[3, 77], x[250, 0], x[295, 255] = float("nan"), float("inf"), float("-inf")
    got = binding.scaled_mm(*binding.scaled_rows(x), *w, offsets, out_dtype=out_dtype)
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[[3, 250, 295]] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], clean[~bad])
    # a NaN among the scales
    q, s = binding.scaled_rows(torch.ones_like(x))
    s.view(torch.uint8)[5, 1] = 255
    got = binding.scaled_mm(q, s, *w, offsets, out_dtype=out_dtype)
    assert got[5].isnan().all() and got[:5].isfinite().all() and got[6:].isfinite().all()


@pytest.mark.parametrize("x_exp,w_exp", [(-100, 60), (60, -100), (-60, -60), (100, 20), (-127, 120), (127, -120), (-127, 0)])
def test_scales_over_their_whole_range(x_exp, w_exp):
    """Exponents far from one another: the products as the values say, results down to fp32's smallest normal number."""
    x, w = randn((20, 256), BF16, 1).clamp(-3, 3), randn((1, 136, 256), BF16, 2).clamp(-3, 3)
    (q, s), (wq, ws) = binding.scaled_rows(x), binding.scaled_pack(w)
    s.view(torch.uint8).copy_(torch.full(s.shape, 127 + x_exp, device="cuda"))
    ws.view(torch.uint8).fill_(127 + w_exp)
    s.view(torch.uint8)[:, 1] -= 1 if x_exp > -127 else 0
    got = binding.scaled_mm(q, s, wq, ws, out_dtype=FP32)
    xd, wd = values(q, s), values(wq, ws)[0]
    ref, mag = xd @ wd.t(), xd.abs() @ wd.abs().t()
    fits = mag < 2.0 ** 127                             # no sum on the way leaves fp32's range, 2^128
    near(got[fits], ref[fits], mag[fits], 256, more=256 * 2.0 ** -126)
    assert not got[ref.abs() >= 2.0 ** 128].isfinite().any() and fits.all() == (x_exp + w_exp < 100)


def test_rows_scales_at_any_address():
    q, s = binding.scaled_rows(uneven((40, 700), BF16, 1))
    w = binding.scaled_pack(uneven((1, 72, 700), BF16, 2, 0.1))
    want = binding.scaled_mm(q, s, *w)
    for left, ld in ((0, 6), (0, 8), (4, 12), (1, 7), (3, 13)):
        wide = torch.full((40, ld + left), 255, dtype=torch.uint8, device="cuda")
        wide[:, left:left + 6] = s.view(torch.uint8)
        assert torch.equal(binding.scaled_mm(q, wide.view(E8M0)[:, left:left + 6], *w), want)


def test_gradient_in_place():
    t, dy, w, dt = randn((50, 264), BF16, 1), randn((50, 264), BF16, 2), randn((264,), BF16, 3), randn((50, 264), BF16, 4)
    want, dw = binding.rms_norm_grad(dy, t, w, dt)
    got, dw2 = binding.rms_norm_grad(dy, t, w, dt, out=dt)
    assert got is dt and torch.equal(got, want) and torch.equal(dw, dw2)


def test_results_beyond_two_to_the_31_elements():
    """9 M rows of 256: the last ones lie behind 2^31 elements."""
    rows, k, n = 9_000_000, 32, 256
    x = torch.zeros((rows, k), dtype=torch.uint8, device="cuda").view(E4M3)
    s = torch.full((rows, 1), 127, dtype=torch.uint8, device="cuda").view(E8M0)
    last = randn((64, k), BF16, 1)
    lq, ls = binding.scaled_rows(last)
    x.view(torch.uint8)[-64:], s.view(torch.uint8)[-64:] = lq.view(torch.uint8), ls.view(torch.uint8)
    w = binding.scaled_pack(randn((1, n, k), BF16, 2))
    out = binding.scaled_mm(x, s, *w)
    assert not out[:1000].any() and torch.equal(out[-64:], binding.scaled_mm(lq, ls, *w))
    del x, s
    q, s = binding.scaled_rows(out)
    rq, rs = ref_rows(out[-64:], E4M3)
    assert torch.equal(as_bits(q[-64:]), as_bits(rq)) and torch.equal(as_bits(s[-64:]), as_bits(rs))
    y = binding.rms_norm(out, torch.ones(n, dtype=BF16, device="cuda"))
    assert torch.equal(y[-64:], binding.rms_norm(out[-64:], torch.ones(n, dtype=BF16, device="cuda")))
    dt, dw = binding.rms_norm_grad(y, out, torch.ones(n, dtype=BF16, device="cuda"), out=y)
    assert dt[-64:].isfinite().all() and dw.isfinite().all()


def test_recorded_operands_are_refused():
    x, w = randn((8, 256), BF16, 1), randn((256,), BF16, 2)
    xr, wr = x.clone().requires_grad_(), w.clone().requires_grad_()
    for call in (lambda: binding.scaled_rows(xr), lambda: binding.swiglu_scaled(xr), lambda: binding.rms_norm(xr, w), lambda: binding.rms_norm(x, wr), lambda: binding.rms_norm(x, w, xr),
                 lambda: binding.rms_norm_scaled(xr, w), lambda: binding.rms_norm_grad(xr, x, w), lambda: binding.rms_norm_grad(x, xr, w), lambda: binding.rms_norm_grad(x, x, wr),
                 lambda: binding.rms_norm_grad(x, x, w, xr), lambda: binding.rms_norm(x, w, out=torch.empty_like(x).requires_grad_())):
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad():
            call()
    assert binding.scaled_pack(xr[None])[0].shape == (1, 8, 256)             # data from a parameter


def test_python_refusals():
    x, w = randn((8, 256), BF16, 1), randn((256,), BF16, 2)
    q, s = binding.scaled_rows(x)
    wq, ws = binding.scaled_pack(randn((2, 64, 256), BF16, 3))
    offsets = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    for call in (lambda: binding.scaled_mm(q[:, :128], s, wq, ws, offsets), lambda: binding.scaled_mm(q, s[:, :1], wq, ws, offsets), lambda: binding.scaled_mm(q, s[:4], wq, ws, offsets),
                 lambda: binding.scaled_mm(q, s, wq, ws[:1], offsets), lambda: binding.scaled_mm(q, s, wq, ws, offsets[:2]), lambda: binding.scaled_mm(q, s, wq, ws),
                 lambda: binding.scaled_mm(q, s.view(torch.uint8), wq, ws, offsets), lambda: binding.scaled_mm(q, s, wq.view(torch.uint8), ws, offsets),
                 lambda: binding.scaled_mm(q, s, wq, ws, offsets, out_dtype=torch.float64), lambda: binding.scaled_mm(q, s, wq, ws, offsets, out=torch.empty((8, 65), device="cuda")),
                 lambda: binding.scaled_rows(x, BF16), lambda: binding.rms_norm(x, w[:255]), lambda: binding.rms_norm(x, w.float()),
                 lambda: binding.rms_norm(x, w, x[:4]), lambda: binding.rms_norm(x, w, sum_out=x), lambda: binding.rms_norm_scaled(x, w, out=(q, s, x)),
                 lambda: binding.rms_norm_grad(x[:4], x, w), lambda: binding.swiglu_scaled(x[:, :255])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.scaled_rows(x.float()), lambda: binding.rms_norm(x.float(), w.float()), lambda: binding.rms_norm(x, w, eps=-1.0),
                 lambda: binding.scaled_mm(q[:, :200].contiguous(), s, wq[:, :, :200], ws, offsets),            # rows off 16-byte boundaries
                 lambda: binding.scaled_rows(x[:1].expand(8, 256)), lambda: binding.rms_norm(torch.zeros((2, 16392), dtype=BF16, device="cuda"), torch.zeros(16392, dtype=BF16, device="cuda"))):
        with pytest.raises(binding.EwError):
            call()
    assert binding.last_operator_error() == 0
