"""Measured cases of the experts' operators in 8-bit floating point: grouped products of operands with a scale for each block
of 128 values and their input gradient, the operators that make such operands (RMS norm with the residual's addition, SwiGLU,
rows and weights as they are), and the norm's gradient.

`run` computes a case in its plain form (elementary torch operations in 32 bits, rounded once at the end), or, with
`own` set, through the framework's entry points in `paper_2508_17624_b200.binding`.

A block of 128 values is held as 8-bit floats q (e4m3 or e5m2) and one 8-bit exponent, a power of two s, and stands for q s.
s is the smallest power of two for which the block's largest value fits the type (448 or 57344).  Rows have a scale for each
128 neighbouring values, weights one for each 128 x 128.

Sizes are those of the framework's layer: hidden 2048, expert intermediate 1408 (gate and up stacked: 2816), 64 base
experts, 32 tuned ones, six experts a token; the drawn cases spread below them.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
EPS = 1e-6


# ----------------------------------------------------------------------------------------------------------- cases
def products(name, way, rows, groups, n, k, dtype="e4m3", out="bf16"):
    return {"name": name, "op": "products", "way": way, "rows": rows, "groups": groups, "n": n, "k": k, "dtype": dtype, "out": out}


def norm(name, rows, width, outs, residual=True, dtype="bf16"):
    return {"name": name, "op": "norm", "rows": rows, "width": width, "outs": outs, "residual": residual, "dtype": dtype}


def norm_grad(name, rows, width, residual=True, dtype="bf16"):
    return {"name": name, "op": "norm grad", "rows": rows, "width": width, "residual": residual, "dtype": dtype}


def swiglu(name, rows, inter, weights=True, dtype="bf16"):
    return {"name": name, "op": "swiglu", "rows": rows, "inter": inter, "weights": weights, "dtype": dtype}


def blocks(name, what, groups, rows, width, to="e4m3", dtype="bf16"):
    return {"name": name, "op": "blocks", "what": what, "groups": groups, "rows": rows, "width": width, "to": to, "dtype": dtype}


def listed():
    return [
        # one decoded token through the gate and up weights of its six experts: a weight stream of 35 MB
        products("products 1 token", "y", 6, 64, 2816, 2048),
        # a decode batch of 256 tokens over the base experts and four adapters' copies: a weight stream of 550 MB
        products("products decode", "y", 1536, 96, 2816, 2048),
        # the gate and up products of an 8192-token prompt batch: bound by arithmetic
        products("products prompt", "y", 49152, 64, 2816, 2048),
        # training: the down projection's input gradient for 4097 tokens, the arriving gradient in the wider-ranged type
        products("products dx", "dx", 24582, 64, 2048, 1408, "e5m2"),
        # the norm before the layer for one decoded token: 8 bits for the experts, 16 for the router; latency
        norm("norm 1 token", 1, 2048, "both"),
        # the same for the prompt batch
        norm("norm prompt", 8192, 2048, "both"),
        # training: its gradient for the prompt batch, the residual stream's own gradient joined in
        norm_grad("norm grad prompt", 8192, 2048),
        # the gradient of a short batch of an odd number of tokens
        norm_grad("norm grad 333", 333, 2048, True, "fp16"),
        # the activation of the prompt batch, routing weights folded in, ready for the down projections
        swiglu("swiglu prompt", 49152, 1408),
        # the activation of the decode batch
        swiglu("swiglu decode", 1536, 1408),
        # training: the gradient that arrives at the down projections, made ready for their input gradient
        blocks("rows e5m2", "rows", 1, 24582, 2048, "e5m2"),
        # an adapter's or the base model's gate and up weights as they are loaded
        blocks("weights", "weights", 64, 2816, 2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["products", "products", "norm", "norm grad", "swiglu", "blocks"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    # widths in steps of 16 are the rule; an odd one now and then
    width = rng.choice([16, 16, 16, 1])
    if op == "products":
        case = products("", rng.choice(["y", "y", "dx"]), _log(rng, 1, 49152), _log(rng, 1, 96), 16 * _log(rng, 4, 176), 16 * _log(rng, 4, 128),
                        rng.choice(["e4m3", "e4m3", "e5m2"]), rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    elif op == "norm":
        case = norm("", _log(rng, 1, 16384), width * _log(rng, 128 // width, 2048 // width), rng.choice(["both", "scaled", "plain"]), rng.random() < 0.7, dtype)
    elif op == "norm grad":
        case = norm_grad("", _log(rng, 1, 16384), width * _log(rng, 128 // width, 2048 // width), rng.random() < 0.7, dtype)
    elif op == "swiglu":
        case = swiglu("", _log(rng, 1, 49152), width * _log(rng, 64 // width, 1408 // width), rng.random() < 0.7, dtype)
    elif rng.random() < 0.5:
        case = blocks("", "rows", 1, _log(rng, 1, 49152), width * _log(rng, 128 // width, 2048 // width), rng.choice(["e4m3", "e5m2"]), dtype)
    else:
        case = blocks("", "weights", _log(rng, 1, 64), 16 * _log(rng, 4, 176), 16 * _log(rng, 4, 128), "e4m3", dtype)
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


def _activations(gen, rows, width, dtype):
    """Normal values of rows of different sizes, some channels larger than the others."""
    channel = 1.0 + 15.0 * (torch.rand((width,), device="cuda", generator=gen) < 0.01)
    row = torch.empty((rows, 1), device="cuda").normal_(0.0, 0.5, generator=gen).exp_()
    return _randn(gen, (rows, width), dtype).mul_(channel.to(dtype)).mul_(row.to(dtype))


def _room(width, step):
    return (width + step - 1) // step * step


def _in_rows(values, to):
    """Rows in blocks of 128: (q [rows, width], scales [rows, blocks]), q's rows on 16-byte boundaries and the scales' on
    four-byte ones, as the framework's own operators lay them out."""
    rows, width = values.shape
    wide = torch.zeros((rows, _room(width, 128)), dtype=torch.float32, device="cuda")
    wide[:, :width] = values
    wide = wide.view(rows, -1, 128)
    s = _scale(wide.abs().amax(2), to)
    scales = torch.zeros((rows, _room(s.shape[1], 4)), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)[:, : s.shape[1]]
    scales.copy_(s)
    q = torch.zeros((rows, _room(width, 16)), dtype=torch.uint8, device="cuda").view(to)[:, :width]
    q.copy_((wide / s[..., None]).view(rows, -1)[:, :width])
    return q, scales


def _in_squares(w, to):
    """Weights [groups, n, k] in blocks of 128 x 128: (q, scales [groups, n blocks, k blocks]), a part of the groups at a time."""
    (groups, n, k), parts = w.shape, max(1, w.numel() >> 27)
    if parts > 1:
        done = [_in_squares(p, to) for p in w.chunk(parts)]
        return tuple(torch.cat([d[i].view(torch.uint8) for d in done]).view(done[0][i].dtype) for i in range(2))
    wide = torch.zeros((groups, _room(n, 128), _room(k, 128)), dtype=torch.float32, device="cuda")
    wide[:, :n, :k] = w
    wide = wide.view(groups, -1, 128, wide.shape[2] // 128, 128)
    s = _scale(wide.abs().amax((2, 4)), to)
    q = (wide / s[:, :, None, :, None]).reshape(groups, wide.shape[1] * 128, -1)[:, :n, :k].contiguous().to(to)
    return q, s.to(torch.float8_e8m0fnu)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype = case["op"], TYPES[case["dtype"]]
    state = {"case": case}
    if op == "products":
        counts = _counts(case, seed)
        rows, groups, n, k = (case[f] for f in ("rows", "groups", "n", "k"))
        state["out"] = TYPES[case["out"]]
        state["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
        state["most"] = int(counts.max())             # the longest group: the plain form pads to it
        state["a"], state["a_scales"] = _in_rows(_activations(gen, rows, k if case["way"] == "y" else n, torch.bfloat16), dtype)
        w = _randn(gen, (groups, n, k), torch.bfloat16, 0.02)
        state["b"], state["b_scales"] = _in_squares(w, torch.float8_e4m3fn)
    elif op == "norm":
        rows, width = case["rows"], case["width"]
        state["x"], state["w"] = _randn(gen, (rows, width), dtype, 0.5), (1.0 + 0.2 * torch.randn((width,), device="cuda", generator=gen)).to(dtype)
        state["residual"] = _activations(gen, rows, width, dtype) if case["residual"] else None
    elif op == "norm grad":
        rows, width = case["rows"], case["width"]
        state["s"], state["w"] = _activations(gen, rows, width, dtype), (1.0 + 0.2 * torch.randn((width,), device="cuda", generator=gen)).to(dtype)
        state["dy"] = _randn(gen, (rows, width), dtype, 0.1)
        state["ds"] = _randn(gen, (rows, width), dtype, 0.1) if case["residual"] else None
    elif op == "swiglu":
        state["h"] = _randn(gen, (case["rows"], 2 * case["inter"]), dtype)
        state["p"] = torch.rand((case["rows"],), device="cuda", generator=gen) if case["weights"] else None
    elif case["what"] == "rows":
        state["x"] = _activations(gen, case["rows"], case["width"], dtype)
    else:
        state["x"] = _randn(gen, (case["groups"], case["rows"], case["width"]), dtype, 0.02)
    return state


# ------------------------------------------------------------------------------------------------------ plain forms
def _scale(most, to):
    """The smallest power of two s with most / s <= the type's largest, down to 2^-127."""
    top, top_exponent = math.frexp(LARGEST[to])
    fraction, exponent = torch.frexp(most)            # without a division, whose rounding could pass a power of two
    exponent = (exponent - top_exponent + (fraction > top)).clamp(-127, 127)
    exponent = torch.where(most == 0, torch.full_like(exponent, -127), exponent)
    bits = torch.where(exponent < -126, torch.full_like(exponent, 1 << 22), (exponent + 127) << 23)      # 2^-127 has no leading one
    return bits.to(torch.int32).view(torch.float32)


def _padded(t, offsets, most):
    """[groups, most, width]: each group's rows, zeros behind them."""
    at = offsets[:-1, None].long() + torch.arange(most, device=t.device)
    inside = at < offsets[1:, None]
    return t[at.clamp_(max=t.shape[0] - 1)] * inside[..., None]


def _rows(padded, offsets, rows):
    """The rows of a padded tensor in their order."""
    r = torch.arange(rows, device=padded.device)
    group = torch.searchsorted(offsets[1:].contiguous(), r.int(), right=True)
    return padded[group, r - offsets[group]]


def _values(q, scales):
    """What 8-bit rows stand for, in 32 bits."""
    return q.float() * scales.float().repeat_interleave(128, dim=1)[:, : q.shape[1]]


def _square_values(q, scales):
    (_, n, k), s = q.shape, scales.float()
    return q.float() * s.repeat_interleave(128, dim=1)[:, :n].repeat_interleave(128, dim=2)[:, :, :k]


def _plain_products(s):
    a = _padded(_values(s["a"], s["a_scales"]), s["offsets"], s["most"])
    w = _square_values(s["b"], s["b_scales"])
    y = torch.bmm(a, w.transpose(1, 2) if s["case"]["way"] == "y" else w)
    return _rows(y, s["offsets"], s["case"]["rows"]).to(s["out"])


def _plain_norm(s):
    x, dtype, outs = s["x"].float(), s["x"].dtype, s["case"]["outs"]
    if s["residual"] is not None:
        total = (x + s["residual"].float()).to(dtype)
        x = total.float()                             # the norm is of the stream as it is kept
    y = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * s["w"].float()
    got = list(_in_rows(y, torch.float8_e4m3fn)) if outs != "plain" else []
    got += [y.to(dtype)] if outs != "scaled" else []
    return got + ([total] if s["residual"] is not None else [])


def _plain_norm_grad(s):
    x, dy, w = s["s"].float(), s["dy"].float(), s["w"].float()
    r = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    unit, g = x * r, dy * w
    dx = r * (g - unit * (g * unit).mean(dim=1, keepdim=True))
    if s["ds"] is not None:
        dx = dx + s["ds"].float()
    return dx.to(s["s"].dtype), (dy * unit).sum(dim=0)


def _plain_swiglu(s):
    gate, up = s["h"].float().chunk(2, dim=1)
    act = gate / (1.0 + torch.exp(-gate)) * up
    return _in_rows(act if s["p"] is None else act * s["p"][:, None], torch.float8_e4m3fn)


def _plain_blocks(s):
    to = TYPES[s["case"]["to"]]
    return _in_rows(s["x"].float(), to) if s["case"]["what"] == "rows" else _in_squares(s["x"], to)


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2508_17624_b200 import binding
        if op == "products":
            call = binding.scaled_mm if case["way"] == "y" else binding.scaled_mm_dx
            return call(state["a"], state["a_scales"], state["b"], state["b_scales"], state["offsets"], out_dtype=state["out"])
        if op == "norm":
            if case["outs"] == "plain":
                return binding.rms_norm(state["x"], state["w"], state["residual"], EPS)
            return binding.rms_norm_scaled(state["x"], state["w"], state["residual"], EPS, with_y=case["outs"] == "both")
        if op == "norm grad":
            return binding.rms_norm_grad(state["dy"], state["s"], state["w"], state["ds"], EPS)
        if op == "swiglu":
            return binding.swiglu_scaled(state["h"], state["p"])
        if case["what"] == "rows":
            return binding.scaled_rows(state["x"], TYPES[case["to"]])
        return binding.scaled_pack(state["x"])
    got = {"products": _plain_products, "norm": _plain_norm, "norm grad": _plain_norm_grad, "swiglu": _plain_swiglu, "blocks": _plain_blocks}[op](state)
    return got[0] if op == "norm" and len(got) == 1 else got


# ------------------------------------------------------------------------------------------------------------- work
def work(case):
    two, op = 2, case["op"]
    if op == "products":
        rows, groups, n, k = (case[f] for f in ("rows", "groups", "n", "k"))
        live = rows if rows <= groups else groups * (1.0 - math.exp(-rows / groups))
        wide, other = (n, k) if case["way"] == "y" else (k, n)
        scales = live * _blocks(n) * _blocks(k) + rows * _blocks(other)
        return {"bytes": live * n * k + rows * other + scales + rows * wide * (4 if case["out"] == "fp32" else two), "flops": 2.0 * rows * n * k}
    if op == "norm":
        rows, width = case["rows"], case["width"]
        held = {"both": 3, "scaled": 1, "plain": 2}[case["outs"]] * width + (0 if case["outs"] == "plain" else _blocks(width))
        return {"bytes": rows * (width * two * (3 if case["residual"] else 1) + held) + width * two, "flops": 6.0 * rows * width}
    if op == "norm grad":
        rows, width = case["rows"], case["width"]
        return {"bytes": rows * width * two * (4 if case["residual"] else 3) + width * 6, "flops": 12.0 * rows * width}
    if op == "swiglu":
        rows, inter = case["rows"], case["inter"]
        return {"bytes": rows * (inter * 5 + _blocks(inter) + 4 * case["weights"]), "flops": 8.0 * rows * inter}
    groups, rows, width = case["groups"], case["rows"], case["width"]
    each = rows * width * 3 + _blocks(width) * (rows if case["what"] == "rows" else _blocks(rows))
    return {"bytes": groups * each, "flops": 3.0 * groups * rows * width}


def _blocks(width):
    return (width + 127) // 128


# ------------------------------------------------------------------------------------------------ exact, in 64 bits
def _power(most, largest):
    """2^ceil(log2(most / largest)) by counting powers of two, which 64 bits hold exactly; 2^-127 at least."""
    powers = torch.tensor([2.0 ** e for e in range(-127, 128)], dtype=torch.float64, device=most.device)
    return powers[torch.searchsorted(powers * largest, most).clamp(max=254)]


def _to_rows(values, to):
    """(q, scales) of rows in 64 bits, block by block.  The one rounding to 8 bits is done on a number of 32 bits, which holds
    every 8-bit step's half exactly; numbers next to such a half are first pushed off it."""
    rows, width = values.shape
    q, scales = torch.empty((rows, width), dtype=to, device="cuda"), []
    for at in range(0, width, 128):
        block = values[:, at:at + 128]
        p = _power(block.abs().amax(1), LARGEST[to])
        q[:, at:at + 128] = _to_eight(block / p[:, None], to)
        scales.append(p.to(torch.float32).to(torch.float8_e8m0fnu).view(torch.uint8))
    return q, torch.stack(scales, 1).view(torch.float8_e8m0fnu)


def _to_eight(v, to):
    narrow = v.float()
    back = narrow.double()
    toward = torch.where(back < v, torch.full_like(narrow, float("inf")), torch.full_like(narrow, -float("inf")))
    half = narrow.view(torch.int32).bitwise_and((1 << 17) - 1) == 0      # may be half of a step: a few significant bits
    return torch.where((back != v) & half, torch.nextafter(narrow, toward), narrow).to(to)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "products":
        ends, rows = s["offsets"].tolist(), s["a"].shape[0]
        wide = case["n"] if case["way"] == "y" else case["k"]
        y = torch.empty((rows, wide), dtype=torch.float64, device="cuda")
        a_power, b_power = s["a_scales"].view(torch.uint8).double() - 127, s["b_scales"].view(torch.uint8).double() - 127
        row, col = torch.arange(case["n"], device="cuda") // 128, torch.arange(case["k"], device="cuda") // 128
        across = col if case["way"] == "y" else row
        for g, (i, j) in enumerate(zip(ends[:-1], ends[1:])):
            if j > i:
                w = s["b"][g].double() * 2.0 ** b_power[g][row][:, col]
                a = s["a"][i:j].double() * 2.0 ** a_power[i:j][:, across]
                y[i:j] = a @ w.t() if case["way"] == "y" else a @ w
        return y
    if op == "norm":
        x, got = s["x"], []
        if s["residual"] is not None:
            x = (x.double() + s["residual"].double()).float().to(x.dtype)
        x64 = x.double()
        y = x64 / ((x64 ** 2).sum(1, keepdim=True) / case["width"] + EPS).sqrt() * s["w"].double()
        if case["outs"] != "plain":
            got += list(_to_rows(y, torch.float8_e4m3fn))
        if case["outs"] != "scaled":
            got.append(y)
        if s["residual"] is not None:
            got.append(x64)
        return got[0] if len(got) == 1 else got
    if op == "norm grad":
        x, dy, w = s["s"].double(), s["dy"].double(), s["w"].double()
        m = (x ** 2).sum(1, keepdim=True) / case["width"] + EPS
        dx = dy * w / m.sqrt() - x * (dy * w * x).sum(1, keepdim=True) / (case["width"] * m ** 1.5)
        return dx if s["ds"] is None else dx + s["ds"].double(), (dy * x / m.sqrt()).sum(0)
    if op == "swiglu":
        inter = case["inter"]
        gate, up = s["h"][:, :inter].double(), s["h"][:, inter:].double()
        act = gate * torch.sigmoid(gate) * up
        return _to_rows(act if s["p"] is None else act * s["p"].double()[:, None], torch.float8_e4m3fn)
    to = TYPES[case["to"]]
    if case["what"] == "rows":
        return _to_rows(s["x"].double(), to)
    q = torch.empty(s["x"].shape, dtype=to, device="cuda")
    scales = torch.empty((case["groups"], _blocks(case["rows"]), _blocks(case["width"])), dtype=torch.uint8, device="cuda")
    for g in range(case["groups"]):
        for i in range(scales.shape[1]):
            band = s["x"][g, 128 * i:128 * i + 128].double()
            most = torch.stack([band[:, c:c + 128].abs().max() for c in range(0, case["width"], 128)])
            p = _power(most, LARGEST[to])
            scales[g, i] = (torch.log2(p) + 127).to(torch.uint8)
            q[g, 128 * i:128 * i + 128] = _to_eight(band / p.repeat_interleave(128)[: case["width"]], to)
    return q, scales.view(torch.float8_e8m0fnu)
