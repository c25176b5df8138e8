"""The stand-alone expert operators as a user runs them: a training step of an adapter's experts next to the pool's
forward, a decode layer with 4-bit experts, streams, graphs, and indexes that are out of range."""
import numpy as np
import pytest
import torch

from paper_2508_17624_b200 import binding, build
from paper_2508_17624_b200 import workloads as wl

from helpers import to_dev

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = 2.0 ** -8                                   # of bf16, relative


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def rel(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


class Layer:
    """The c0 layer in a pool and, slot by slot, as stacked tensors w13 [P, 2I, H] and w2 [P, H, I]."""

    def __init__(self, n_tokens=None):
        self.cfg = cfg = wl.CONFIGS["c0"]
        bank = wl.NoiseBank(cfg.seed)
        self.pool = binding.Pool.from_config(cfg)
        self.tuned, bases = binding.load_model(self.pool, cfg, bank)
        base = bases[0]
        self.w13 = torch.zeros((cfg.num_slots, 2 * cfg.inter, cfg.hidden), dtype=BF16, device="cuda")
        self.w2 = torch.zeros((cfg.num_slots, cfg.hidden, cfg.inter), dtype=BF16, device="cuda")
        self.put(0, base.routed)
        for i in range(cfg.max_adapters):
            self.put(cfg.num_experts + i * cfg.e_max, wl.gen_adapter_layer(cfg, i, 0, self.tuned[i][0], bank))
        self.shared = [to_dev(a) for a in (base.shared.w_gate, base.shared.w_up, base.shared.w_down)]
        self.x, self.aid = to_dev(wl.gen_tokens(cfg)), to_dev(wl.gen_adapter_ids(cfg))
        r = self.pool.moe_forward_debug(0, self.x, self.aid)
        self.out, self.p, self.slots, self.offsets = r["out"], r["topk_w"], r["slot_ids"], r["offsets"]
        # the row of each pair in slot order, and back: token and weight of each row
        inv = r["inv"].reshape(-1).long()
        self.token = torch.empty_like(inv)
        self.token[inv] = torch.arange(inv.numel(), device="cuda") // cfg.top_k
        self.row_p = torch.empty_like(self.p.reshape(-1))
        self.row_p[inv] = self.p.reshape(-1)

    def put(self, at, e):
        n = e.n
        self.w13[at:at + n, :self.cfg.inter], self.w13[at:at + n, self.cfg.inter:], self.w2[at:at + n] = to_dev(e.w_gate), to_dev(e.w_up), to_dev(e.w_down)

    def shared_out(self, x):
        g, u, d = (w.to(x.dtype) for w in self.shared)
        return sum((torch.nn.functional.silu(x @ g[s].t()) * (x @ u[s].t())) @ d[s].t() for s in range(g.shape[0]))


def test_training_step_of_an_adapters_experts():
    """Forward and backward through the experts with the operators: the forward equals the pool's, the gradients those of the
    formula in 64 bits, and the pool serves the experts that a step with them has changed."""
    L = Layer()
    cfg, I = L.cfg, L.cfg.inter
    rows_x = L.x[L.token]

    def forward():
        h = binding.grouped_mm(rows_x, L.w13, L.offsets)
        act = binding.swiglu(h, L.row_p)
        y = binding.grouped_mm(act, L.w2, L.offsets, out_dtype=FP32)
        out = L.shared_out(L.x.float())
        return h, act, out.index_add(0, L.token, y)

    h, act, out = forward()
    # both round h's successor act to bf16 and sum in fp32; here h is rounded too, there only the output
    assert rel(out, L.out.double()) <= 4 * HALF_STEP

    g_out = (torch.randn(out.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 0.1).to(BF16)
    dy = g_out[L.token]
    d_act = binding.grouped_mm_dx(dy, L.w2, L.offsets)
    dw2 = binding.grouped_mm_dw(dy, act, L.offsets, out_dtype=FP32)
    dh, dp = binding.swiglu_grad(d_act, h, L.row_p)
    dw13 = binding.grouped_mm_dw(dh, rows_x, L.offsets, out_dtype=FP32)
    dx = torch.zeros_like(out).index_add(0, L.token, binding.grouped_mm_dx(dh, L.w13, L.offsets, out_dtype=FP32))

    leaves = [t.double().requires_grad_() for t in (L.x, L.w13, L.w2, L.row_p)]
    x64, a64, b64, p64 = leaves
    ends = L.offsets.tolist()
    ref = 0
    for s, (i, j) in enumerate(zip(ends[:-1], ends[1:])):
        if j > i:
            g, u = (x64[L.token[i:j]] @ a64[s].t()).chunk(2, dim=1)
            y = (p64[i:j, None] * g * torch.sigmoid(g) * u) @ b64[s].t()
            ref = ref + torch.zeros_like(x64).index_add(0, L.token[i:j], y)
    (ref * g_out.double()).sum().backward()
    # the bf16 roundings on the way: h, act, d_act, dh, each at most half a step in the 2-norm, h's through silu's slope (at
    # most 1.1) on both of its halves
    for got, leaf in ((dx, x64), (dw13, a64), (dw2, b64), (dp, p64)):
        assert rel(got, leaf.grad) <= 6 * HALF_STEP
    assert not dw13[torch.diff(L.offsets) == 0].any()

    # a step along the gradient on adapter 1's experts, straight from device memory into the pool
    a, at = 1, cfg.num_experts + cfg.e_max
    n = len(L.tuned[a][0])
    L.w13[at:at + n] = (L.w13[at:at + n].float() - 0.5 * dw13[at:at + n]).to(BF16)
    L.w2[at:at + n] = (L.w2[at:at + n].float() - 0.5 * dw2[at:at + n]).to(BF16)
    L.pool.unload_adapter(a)
    L.pool.load_adapter(a, np.array([n]), L.tuned[a][0], L.w13[at:at + n, :I].contiguous(), L.w13[at:at + n, I:].contiguous(), L.w2[at:at + n].contiguous())
    served = L.pool.moe_forward(0, L.x, L.aid)
    assert not torch.equal(served, L.out)
    assert rel(forward()[2], served.double()) <= 4 * HALF_STEP
    assert L.pool.last_device_error() == 0 and binding.last_operator_error() == 0


def test_decode_layer_with_four_bit_experts():
    """Route with the pool, then the experts from 4-bit weights: against the formula in 64 bits with the weights that the
    4-bit values stand for, and near the 16-bit layer."""
    L = Layer()
    cfg = L.cfg
    q13, s13 = binding.quant_pack(L.w13, 64)
    q2, s2 = binding.quant_pack(L.w2, 32)
    for n in (1, 5, cfg.n_tokens):
        x, slots, p = L.x[:n], L.slots[:n].contiguous(), L.p[:n].reshape(-1).contiguous()
        h = binding.quant_mv(x, q13, s13, slots)
        act = binding.swiglu(h, p)
        y = binding.quant_mv(act, q2, s2, slots, out_dtype=FP32)
        out = y.view(n, cfg.top_k, cfg.hidden).sum(1)
        from test_gpu_operators import unpacked
        w13, w2, flat = unpacked(q13, s13), unpacked(q2, s2), slots.reshape(-1).long()
        g, u = torch.einsum("pk,pnk->pn", x.double().repeat_interleave(cfg.top_k, 0), w13[flat]).chunk(2, 1)
        ref = torch.einsum("pi,phi->ph", p.double()[:, None] * g * torch.sigmoid(g) * u, w2[flat]).view(n, cfg.top_k, -1).sum(1)
        assert rel(out, ref) <= 4 * HALF_STEP              # h and act are rounded to bf16, x to 15 bits a group
        full = L.out[:n].double() - L.shared_out(x.double())
        # 4-bit weights of N(0, s): a step of max/7, about 2.6 s / 7 in a group of 64; its rounding is step / sqrt(12) rms,
        # a tenth of s, for each of gate, up and down: sqrt(3) tenths, and half as much again for groups with larger maxima
        assert rel(out, full) <= 0.3


def test_two_streams_and_repeated_calls_give_the_same_bits():
    x = torch.randn((300, 512), device="cuda").to(BF16)
    w = (torch.randn((8, 384, 512), device="cuda") * 0.05).to(BF16)
    offsets = torch.tensor([0, 10, 10, 90, 130, 200, 201, 280, 300], dtype=torch.int32, device="cuda")
    q, s = binding.quant_pack(w, 128)
    slots = torch.randint(0, 8, (300,), dtype=torch.int32, device="cuda")
    dy = torch.randn((300, 384), device="cuda").to(BF16)

    def all_of_them():
        return [binding.grouped_mm(x, w, offsets), binding.grouped_mm_dx(dy, w, offsets, out_dtype=FP32), binding.grouped_mm_dw(dy, x, offsets, out_dtype=FP32),
                binding.quant_mv(x, q, s, slots), binding.quant_mv(x[:20], q, s, slots[:20]), binding.swiglu(x), *binding.swiglu_grad(x[:, :256].contiguous(), x, torch.ones(300, device="cuda"))]

    first = all_of_them()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for st in streams:
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got.append(all_of_them())
    torch.cuda.synchronize()
    for some in got:
        for a, b in zip(first, some):
            assert torch.equal(a, b)


def test_busy_slots_in_several_batches_give_the_same_bits_every_time():
    """1536 pairs over 20 slots: a CTA works through several batches of rows, partial tiles in each."""
    x = torch.randn((256, 2048), device="cuda").to(BF16)
    q, s = binding.quant_pack((torch.randn((20, 328, 2048), device="cuda") * 0.05).to(BF16), 64)
    slots = torch.randint(0, 20, (256, 6), dtype=torch.int32, device="cuda")
    first = binding.quant_mv(x, q, s, slots, out_dtype=FP32)
    for _ in range(40):
        assert torch.equal(first, binding.quant_mv(x, q, s, slots, out_dtype=FP32))


def test_captured_and_replayed_with_new_inputs():
    """Two graphs over the same weights, replayed in turn with changing inputs, offsets and slots."""
    w = (torch.randn((6, 264, 256), device="cuda") * 0.05).to(BF16)
    q, s = binding.quant_pack(w, 64)
    x = torch.randn((40, 256), device="cuda").to(BF16)
    offsets = torch.tensor([0, 5, 9, 9, 30, 31, 40], dtype=torch.int32, device="cuda")
    slots = torch.arange(40, dtype=torch.int32, device="cuda") % 6

    def step():
        h = binding.grouped_mm(x, w, offsets)
        return h, binding.swiglu(h), binding.grouped_mm_dw(h, x, offsets, out_dtype=FP32), binding.quant_mv(x, q, s, slots)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        step()
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(step())
            graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(4):
        x.copy_(torch.randn_like(x))
        offsets.copy_(torch.tensor([[0, 5, 9, 9, 30, 31, 40], [0, 40, 40, 40, 40, 40, 40], [0, 1, 2, 3, 4, 5, 40], [0, 0, 0, 17, 33, 39, 40]][turn], dtype=torch.int32))
        slots.copy_(torch.randint(-1, 6, (40,), dtype=torch.int32))
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        for a, b in zip(outs[turn % 2], step()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("offsets", [[0, 10, 5, 20], [-3, 4, 8, 20], [0, 4, 99, 20], [7, 3, 3, 3], [0, 20, 0, 20]], ids=str)
def test_offsets_out_of_order_or_range_are_clamped_and_reported(offsets):
    """No access outside the matrices: every group ends where the largest offset so far, inside the matrix, says."""
    x, w = torch.randn((20, 64), device="cuda").to(BF16), torch.randn((3, 72, 64), device="cuda").to(BF16)
    ends = np.maximum.accumulate(np.clip(offsets, 0, 20))
    good, bad = (torch.tensor(list(o), dtype=torch.int32, device="cuda") for o in (ends, offsets))
    out = [torch.full((20, 72), 7.0, dtype=BF16, device="cuda") for _ in range(2)]
    for o, y in zip((good, bad), out):
        assert binding.last_operator_error() == 0
        binding.grouped_mm(x, w, o, out=y)
    assert binding.last_operator_error() == 1              # EW_ERR_INVALID_ARG, once
    assert torch.equal(out[0], out[1])
    dw = [binding.grouped_mm_dw(y.nan_to_num(), x, o, out_dtype=FP32) for o, y in zip((good, bad), out)]
    assert binding.last_operator_error() == 1 and torch.equal(dw[0], dw[1])


def test_results_beyond_two_to_the_31_elements():
    """2.2 G elements of y, of dh and of dw: the last rows against the formula."""
    rows, n, k = 1_100_003, 2048, 64
    x, w = torch.randn((rows, k), device="cuda").to(BF16), torch.randn((3, n, k), device="cuda").to(BF16)
    offsets = torch.tensor([0, 500_001, 500_001, rows], dtype=torch.int32, device="cuda")
    y = binding.grouped_mm(x, w, offsets)
    for at, g in ((slice(0, 70), 0), (slice(rows - 70, rows), 2)):
        assert rel(y[at], x[at].double() @ w[g].double().t()) <= HALF_STEP
    dh = binding.swiglu_grad(y[:, :1024], y)
    g, u, d = y[-9:, :1024].double(), y[-9:, 1024:].double(), y[-9:, :1024].double()
    sig = torch.sigmoid(g)
    assert rel(dh[-9:], torch.cat((d * u * sig * (1 + g * (1 - sig)), d * g * sig), 1)) <= HALF_STEP
    del y, dh
    groups, n, k = 540, 2040, 2048
    dy, x = torch.randn((groups, n), device="cuda").to(FP16), torch.randn((groups, k), device="cuda").to(FP16)
    dw = binding.grouped_mm_dw(dy, x, torch.arange(groups + 1, dtype=torch.int32, device="cuda"))
    for g in (0, groups - 1):
        assert rel(dw[g], torch.outer(dy[g].double(), x[g].double())) <= 2.0 ** -11
    assert binding.last_operator_error() == 0


def test_more_pairs_than_one_launch_takes():
    """5000 pairs of 250 tokens, 20 a token, over 40 slots, some without one: the launches divide inside a token's pairs."""
    slots = torch.randint(-1, 40, (250, 20), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    w = (torch.randn((40, 48, 160), device="cuda") * 0.05).to(FP16)
    q, s = binding.quant_pack(w, 32)
    x = torch.randn((250, 160), device="cuda").to(FP16)
    y = binding.quant_mv(x, q, s, slots, out_dtype=FP32)
    from test_gpu_operators import unpacked
    flat = slots.reshape(-1).long()
    ref = torch.einsum("pk,pnk->pn", x.double().repeat_interleave(20, 0), unpacked(q, s)[flat.clamp(min=0)]) * (flat >= 0)[:, None]
    assert rel(y, ref) <= 1e-6 and not y[flat < 0].any()


def test_python_refuses_what_does_not_fit():
    x, w = torch.zeros((4, 64), dtype=BF16, device="cuda"), torch.zeros((2, 72, 64), dtype=BF16, device="cuda")
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    q, s = binding.quant_pack(w, 64)
    slots = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    p = torch.ones(4, device="cuda")
    bad = [lambda: binding.grouped_mm(x, w[:, :, :32], offsets), lambda: binding.grouped_mm(x, w, offsets[:2]), lambda: binding.grouped_mm(x, w, offsets.long()),
           lambda: binding.grouped_mm(x.half(), w, offsets), lambda: binding.grouped_mm(x.float(), w.float(), offsets), lambda: binding.grouped_mm(x, w, offsets.cpu()),
           lambda: binding.grouped_mm(x.t(), w, offsets), lambda: binding.grouped_mm(x, w, offsets, out=torch.zeros((4, 64), dtype=BF16, device="cuda")),
           lambda: binding.grouped_mm(x, w, offsets, out_dtype=torch.int32), lambda: binding.grouped_mm_dw(x, x[:3], offsets),
           lambda: binding.grouped_mm_dw(x, x, offsets, accumulate=True), lambda: binding.quant_mv(x.half(), q, s, slots), lambda: binding.quant_mv(x, q, s, slots.long()),
           lambda: binding.quant_mv(x, q, s[:1], slots), lambda: binding.quant_mv(x[:3], q, s, slots), lambda: binding.quant_mv(x, q.float(), s, slots),
           lambda: binding.quant_pack(w, 48), lambda: binding.quant_pack(w.float(), 32), lambda: binding.swiglu(x[:, :63]), lambda: binding.swiglu(x, p.double()),
           lambda: binding.swiglu(x, p[:3]), lambda: binding.swiglu_grad(x, x), lambda: binding.swiglu_grad(x[:, :32].half(), x)]
    bad += [lambda: binding.grouped_mm(x, w, offsets, out_dtype=FP16), lambda: binding.quant_mv(x, q, s, None), lambda: binding.grouped_mm(x[:, 1:57], w[:, :, :56], offsets),
            lambda: binding.quant_pack(torch.zeros((1, 12, 64), dtype=BF16, device="cuda"), 64)]
    for call in bad:
        with pytest.raises((ValueError, binding.EwError)):          # the binding's or the library's refusal
            call()
    assert binding.last_operator_error() == 0
