"""Measured cases of the stand-alone expert operators: grouped products with their gradients, matrix-vector products
with 4-bit expert weights, and the SwiGLU between the two linears of an expert with its gradient.

`run` computes a case in its plain form (elementary torch operations in 32 bits, rounded once at the end), or, with
`own` set, through the framework's entry points in `paper_2508_17624_b200.binding`.

Sizes are those of the framework's layer: hidden 2048, expert intermediate 1408 (gate and up stacked: 2816), 64 base
experts, 32 tuned ones, six experts a token; the drawn cases spread below them.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# where k = 0..7 of a 32-bit word's eight weights sit among its nibbles: even ones in the low half, odd ones in the high
NIBBLE = [0, 4, 1, 5, 2, 6, 3, 7]


# ----------------------------------------------------------------------------------------------------------- cases
def products(name, way, rows, groups, n, k, dtype="bf16", out="same"):
    return {"name": name, "op": "products", "way": way, "rows": rows, "groups": groups, "n": n, "k": k, "dtype": dtype, "out": out}


def quant(name, tokens, per_token, slots, n, k, group, rows="token", dtype="bf16", out="same"):
    return {"name": name, "op": "quant", "tokens": tokens, "per_token": per_token, "slots": slots, "n": n, "k": k, "group": group, "rows": rows, "dtype": dtype,
            "out": out}


def swiglu(name, way, rows, inter, weights=True, dtype="bf16"):
    return {"name": name, "op": "swiglu", "way": way, "rows": rows, "inter": inter, "weights": weights, "dtype": dtype}


def listed():
    return [
        # one decoded token through the gate and up weights of its six experts: a weight stream of 69 MB
        products("products 1 token", "y", 6, 64, 2816, 2048),
        # a decode batch of 256 tokens over the base experts and four adapters' copies: a weight stream of 1.1 GB
        products("products decode", "y", 1536, 96, 2816, 2048),
        # the gate and up products of an 8192-token prompt batch: bound by arithmetic
        products("products prompt", "y", 49152, 64, 2816, 2048),
        # training: the down projection's input gradient for 4097 tokens
        products("products dx", "dx", 24582, 64, 2048, 1408),
        # training: the gate and up weights' gradient of 32 tuned experts, kept in 32 bits for accumulation over steps
        products("products dw fp32", "dw", 12289, 32, 2816, 2048, out="fp32"),
        # training: the down weights' gradient, rounded to the weights' own type
        products("products dw fp16", "dw", 6151, 32, 2048, 1408, "fp16"),
        # one decoded token with 4-bit experts: latency and 18 MB of weights
        quant("quant 1 token", 1, 6, 64, 2816, 2048, 128),
        # sixteen tokens through the 4-bit down projections; a pair's own activation row
        quant("quant down 16", 16, 6, 96, 2048, 1408, 128, "pair"),
        # the 256-token decode batch with 4-bit experts: 300 MB of weights, some sixteen rows an expert
        quant("quant decode 256", 256, 6, 96, 2816, 2048, 64),
        # a dense projection of four tokens, small groups, results in 32 bits for a sum over ranks
        quant("quant dense 4", 4, 1, 1, 2048, 2048, 32, "token", "fp16", "fp32"),
        # the activation of the prompt batch, routing weights folded in
        swiglu("swiglu prompt", "y", 49152, 1408),
        # its gradient, with the routing weights' own
        swiglu("swiglu grad", "grad", 24582, 1408),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["products", "quant", "swiglu"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "products":
        way = rng.choice(["y", "dx", "dw"])
        case = products("", way, _log(rng, 1, 49152), _log(rng, 1, 96), 8 * _log(rng, 8, 352), 8 * _log(rng, 8, 256), dtype, rng.choice(["same", "fp32"]))
    elif op == "quant":
        group = rng.choice([32, 64, 128])
        per = rng.choice([1, 2, 6, 8])
        case = quant("", _log(rng, 1, 256), per, rng.randint(per, 96), 8 * _log(rng, 8, 352), group * rng.randint(1, 2048 // group), group, rng.choice(["token", "pair"]), dtype,
                     rng.choice(["same", "fp32"]))
    else:
        case = swiglu("", rng.choice(["y", "grad"]), _log(rng, 1, 49152), _log(rng, 8, 1408), rng.random() < 0.7, dtype)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------- inputs
def _counts(case, seed):
    """Rows a group, as routing gives them: popular experts and rare ones, some without a row."""
    r = np.random.RandomState(seed % (1 << 31))
    rows, groups = case["rows"], case["groups"]
    if rows <= groups:                                # one token's experts are distinct
        c = np.zeros(groups, np.int64)
        c[r.choice(groups, rows, replace=False)] = 1
        return c
    p = np.exp(0.4 * r.randn(groups))
    return r.multinomial(rows, p / p.sum())


def _randn(gen, shape, dtype, scale=1.0):
    return torch.empty(shape, dtype=torch.float32 if math.prod(shape) < 1 << 20 else dtype, device="cuda").normal_(0.0, scale, generator=gen).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    state = {"case": case, "out": TYPES.get(case.get("out"), dtype)}
    if case["op"] == "products":
        counts = _counts(case, seed)
        rows, groups, n, k = (case[f] for f in ("rows", "groups", "n", "k"))
        state["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
        state["most"] = int(counts.max())             # the longest group: the plain form pads to it
        if case["way"] == "y":
            state["a"], state["b"] = _randn(gen, (rows, k), dtype), _randn(gen, (groups, n, k), dtype, 0.02)
        elif case["way"] == "dx":
            state["a"], state["b"] = _randn(gen, (rows, n), dtype), _randn(gen, (groups, n, k), dtype, 0.02)
        else:
            state["a"], state["b"] = _randn(gen, (rows, n), dtype, 0.1), _randn(gen, (rows, k), dtype)
    elif case["op"] == "quant":
        tokens, per, slots, n, k = (case[f] for f in ("tokens", "per_token", "slots", "n", "k"))
        state["x"] = _randn(gen, (tokens * per if case["rows"] == "pair" else tokens, k), dtype)
        levels = torch.empty((slots, n, k), dtype=torch.float16, device="cuda").normal_(7.5, 2.5, generator=gen).clamp_(0, 15).to(torch.uint8)
        state["q"] = (levels[..., 0::2] | (levels[..., 1::2] << 4)).contiguous()
        state["scales"] = torch.empty((slots, k // case["group"], n), device="cuda").uniform_(0.004, 0.012, generator=gen).to(dtype)
        state["slots"] = None
        if slots > 1:
            state["slots"] = torch.rand((tokens, slots), device="cuda", generator=gen).argsort(dim=1)[:, :per].to(torch.int32).contiguous()
    else:
        rows, inter = case["rows"], case["inter"]
        state["h"] = _randn(gen, (rows, 2 * inter), dtype)
        state["p"] = torch.rand((rows,), device="cuda", generator=gen) if case["weights"] else None
        state["da"] = _randn(gen, (rows, inter), dtype, 0.1) if case["way"] == "grad" else None
    return state


# ------------------------------------------------------------------------------------------------------ plain forms
def _padded(t, offsets, most):
    """[groups, most, width] in 32 bits: each group's rows, zeros behind them."""
    at = offsets[:-1, None].long() + torch.arange(most, device=t.device)
    inside = at < offsets[1:, None]
    return t[at.clamp_(max=t.shape[0] - 1)].float() * inside[..., None]


def _rows(padded, offsets, rows):
    """The rows of a padded tensor in their order."""
    r = torch.arange(rows, device=padded.device)
    group = torch.searchsorted(offsets[1:].contiguous(), r.int(), right=True)
    return padded[group, r - offsets[group]]


def _plain_products(s):
    offsets, most, way = s["offsets"], s["most"], s["case"]["way"]
    a = _padded(s["a"], offsets, most)
    if way == "dw":
        return torch.bmm(a.transpose(1, 2), _padded(s["b"], offsets, most)).to(s["out"])
    w = s["b"].float()
    y = torch.bmm(a, w.transpose(1, 2) if way == "y" else w)
    return _rows(y, offsets, s["case"]["rows"]).to(s["out"])


def _unpacked(q, scales, group):
    """The weights that the 4-bit values stand for, in 32 bits."""
    g, n, half = q.shape
    place = torch.stack((q & 15, q >> 4), dim=-1).view(g, n, half // 4, 8)
    level = place[..., NIBBLE].view(g, n, 2 * half)
    return (level.float() - 8.0) * scales.float().transpose(1, 2).repeat_interleave(group, dim=2)


def _plain_quant(s):
    w = _unpacked(s["q"], s["scales"], s["case"]["group"])
    every = torch.matmul(s["x"].float(), w.transpose(1, 2))               # [slots, rows of x, n]
    if s["slots"] is None:
        return every[0].to(s["out"])
    slot = s["slots"].reshape(-1).long()
    pair = torch.arange(slot.numel(), device=slot.device)
    y = every[slot.clamp(min=0), pair // (slot.numel() // s["x"].shape[0])]
    return (y * (slot >= 0)[:, None]).to(s["out"])


def _plain_swiglu(s):
    inter, dtype = s["case"]["inter"], s["h"].dtype
    gate, up = s["h"][:, :inter].float(), s["h"][:, inter:].float()
    sig = 1.0 / (1.0 + torch.exp(-gate))
    p = 1.0 if s["p"] is None else s["p"][:, None]
    if s["da"] is None:
        return (gate * sig * up * p).to(dtype)
    da = s["da"].float()
    d_gate = da * p * up * sig * (1.0 + gate * (1.0 - sig))
    d_up = da * p * gate * sig
    dh = torch.cat((d_gate, d_up), dim=1).to(dtype)
    return dh if s["p"] is None else (dh, (da * gate * sig * up).sum(dim=1))


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2508_17624_b200 import binding
        if op == "products":
            call = {"y": binding.grouped_mm, "dx": binding.grouped_mm_dx, "dw": binding.grouped_mm_dw}[state["case"]["way"]]
            return call(state["a"], state["b"], state["offsets"], out_dtype=state["out"])
        if op == "quant":
            return binding.quant_mv(state["x"], state["q"], state["scales"], state["slots"], out_dtype=state["out"])
        if state["da"] is None:
            return binding.swiglu(state["h"], state["p"])
        return binding.swiglu_grad(state["da"], state["h"], state["p"])
    return {"products": _plain_products, "quant": _plain_quant, "swiglu": _plain_swiglu}[op](state)


# ------------------------------------------------------------------------------------------------------------- work
def work(case):
    two, out = 2, {"fp32": 4}.get(case.get("out"), 2)
    if case["op"] == "products":
        rows, groups, n, k = (case[f] for f in ("rows", "groups", "n", "k"))
        live = rows if rows <= groups else groups * (1.0 - math.exp(-rows / groups))
        flops = 2.0 * rows * n * k
        if case["way"] == "dw":
            return {"bytes": rows * (n + k) * two + groups * n * k * out, "flops": flops}
        wide, other = (n, k) if case["way"] == "y" else (k, n)
        return {"bytes": live * n * k * two + rows * other * two + rows * wide * out, "flops": flops}
    if case["op"] == "quant":
        tokens, per, slots, n, k = (case[f] for f in ("tokens", "per_token", "slots", "n", "k"))
        live = slots * (1.0 - (1.0 - per / slots) ** tokens)
        weights = n * k / 2 + n * (k // case["group"]) * two
        rows = tokens * per if case["rows"] == "pair" else tokens
        return {"bytes": live * weights + rows * k * two + tokens * per * n * out, "flops": 2.0 * tokens * per * n * k}
    rows, inter = case["rows"], case["inter"]
    if case["way"] == "y":
        return {"bytes": rows * inter * 3 * two + rows * 4 * case["weights"], "flops": 6.0 * rows * inter}
    return {"bytes": rows * inter * 5 * two + rows * 8 * case["weights"], "flops": 14.0 * rows * inter}


# ------------------------------------------------------------------------------------------------ exact, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "products":
        ends = s["offsets"].tolist()
        spans = list(zip(ends[:-1], ends[1:]))
        a, b = s["a"], s["b"]
        if case["way"] == "dw":
            return torch.stack([a[i:j].double().t() @ b[i:j].double() for i, j in spans])
        rule = "rk,nk->rn" if case["way"] == "y" else "rn,nk->rk"
        return torch.cat([torch.einsum(rule, a[i:j].double(), b[g].double()) for g, (i, j) in enumerate(spans) if j > i])
    if case["op"] == "quant":
        x, q, scales, group = s["x"], s["q"], s["scales"], case["group"]
        n, k = case["n"], case["k"]
        slots = [0] * x.shape[0] if s["slots"] is None else s["slots"].reshape(-1).tolist()
        share = len(slots) // x.shape[0]
        y = torch.zeros((len(slots), n), dtype=torch.float64, device=x.device)
        for slot in sorted(set(slots)):
            if slot < 0:
                continue
            word = q[slot].contiguous().view(torch.int32).long() & 0xFFFFFFFF    # eight weights a word
            w = torch.empty((n, k), dtype=torch.float64, device=x.device)
            for j in range(8):
                w[:, j::8] = ((word >> (4 * (j // 2) + 16 * (j % 2))) & 15).double() - 8
            for c in range(k // group):
                w[:, c * group:(c + 1) * group] *= scales[slot, c].double()[:, None]
            pairs = [i for i, v in enumerate(slots) if v == slot]
            y[pairs] = x[[i // share for i in pairs]].double() @ w.t()
        return y
    inter = case["inter"]
    gate, up = s["h"].double().split(inter, dim=1)
    p = torch.ones((case["rows"], 1), dtype=torch.float64, device=gate.device) if s["p"] is None else s["p"].double()[:, None]
    silu = gate * torch.sigmoid(gate)
    if case["way"] == "y":
        return p * silu * up
    g = p * s["da"].double()
    slope = torch.sigmoid(gate) * (1 + gate - silu)
    dh = torch.empty((case["rows"], 2 * inter), dtype=torch.float64, device=gate.device)
    dh[:, :inter], dh[:, inter:] = g * up * slope, g * silu
    return dh if s["p"] is None else (dh, (s["da"].double() * silu * up).sum(1))
