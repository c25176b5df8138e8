"""Limits of the operators in 8-bit floating point: sums next to the last bit of what the tensor core keeps, and each form of the
product's kernel over what it may be given.

Tolerances.  An instruction adds 32 products (16 of 16-bit operands) to the running sum.  It cuts each addend off below 2^-25 of the
largest one's power of two, and the sum behind its 24th bit: (32 + 1) 2^-25 + 2^-23 = 9.25 * 2^-23 of S = sum |a b| at most
(5.25 * 2^-23 for 16).  The parts of a long sum each lose that of their own S, and are added up with half a step of fp32 each.
"""
import numpy as np
import pytest
import torch

from paper_2508_17624_b200 import binding

from test_gpu_scaled import near, uneven, values

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
TERMS = {FP32: 2048, FP16: 8192, BF16: 65536}           # of a part


def loss(terms, out_dtype, parts_of, instruction):
    """What a sum of so many terms may be off by, of sum |a b|: its own rounding and the parts' losses and additions."""
    parts = -(-terms // parts_of[out_dtype])
    of_part = min(terms + 128 if parts == 1 else parts_of[out_dtype], parts_of[out_dtype])       # (whole blocks of 128)
    rounding = torch.finfo(out_dtype).eps / 2
    return rounding + (of_part / instruction * ((instruction + 1) * 2.0 ** -25 + 2.0 ** -23) + parts * 2.0 ** -24) * (1 + rounding)


@pytest.mark.parametrize("out_dtype,k", [(FP32, 1024), (FP32, 2048), (FP32, 2208), (FP32, 8192), (FP16, 8192), (BF16, 70016)], ids=str)
def test_sums_next_to_the_last_bit(out_dtype, k):
    """One large term, and all others of one size 2^-e below it: most is lost where they lie just below what an addition keeps."""
    blocks = k // 128 + (k % 128 > 0)
    for first in (1, 128):                              # large terms
        for m in (1.0, 1.875):
            x = torch.full((31, k), m, device="cuda")
            x[:, :128] = 0
            x[:, :first] = 1
            q, s = x.to(E4M3), torch.full((31, (blocks + 3) // 4 * 4), 127, dtype=torch.uint8, device="cuda")
            s[:, 1:] -= torch.arange(31, dtype=torch.uint8, device="cuda")[:, None]          # row e
            s = s.view(E8M0)[:, :blocks]
            w, ws = binding.scaled_pack(torch.ones((1, 16, k), dtype=BF16, device="cuda"))
            ref = values(q, s).sum(1)[:, None]
            off = (binding.scaled_mm(q, s, w, ws, out_dtype=out_dtype).double() - ref).abs() / ref
            assert (off <= loss(k, out_dtype, TERMS, 32)).all(), (first, m, float(off.max()))


@pytest.mark.parametrize("dtype,out_dtype,k", [(BF16, FP32, 1024), (BF16, FP32, 5000), (FP16, FP16, 8192), (BF16, BF16, 70000)], ids=str)
def test_sums_of_16_bit_products_next_to_the_last_bit(dtype, out_dtype, k):
    """The same for the grouped products and their gradients."""
    parts_of, most = {FP32: 1024, FP16: 8192, BF16: 65536}, 31 if dtype == BF16 else 14       # (fp16 ends at 2^-14)
    offsets = torch.tensor([0, most], dtype=torch.int32, device="cuda")
    for first in (1, 64):
        for m in (1.0, 1.9921875):
            x = torch.exp2(-torch.arange(most, device="cuda").double())[:, None] * torch.full((1, k), m, dtype=torch.float64, device="cuda")
            x[:, :64] = 0
            x[:, :first] = 1
            x = x.to(dtype)
            ref = x.double().sum(1)
            for call, w in ((binding.grouped_mm, torch.ones((1, 16, k), dtype=dtype, device="cuda")), (binding.grouped_mm_dx, torch.ones((1, k, 16), dtype=dtype, device="cuda"))):
                off = (call(x, w, offsets, out_dtype=out_dtype).double() - ref[:, None]).abs() / ref[:, None]
                assert (off <= loss(k, out_dtype, parts_of, 16)).all(), (call.__name__, first, m, float(off.max()))
            rows = torch.ones((k, 16), dtype=dtype, device="cuda")
            wide = torch.zeros((k, 32), dtype=dtype, device="cuda")[:, :most].copy_(x.t())
            got = binding.grouped_mm_dw(wide, rows, torch.tensor([0, k], dtype=torch.int32, device="cuda"), out_dtype=out_dtype)[0].double()
            off = (got - ref[:, None]).abs() / ref[:, None]
            assert (off <= loss(k, out_dtype, parts_of, 16)).all(), ("dw", first, m, float(off.max()))


# ---------------------------------------------------------------------------------------------- forms of the product's kernel
RAGGED = (700, 0, 1, 257, 563)
# the form on 148 SMs (0 one CTA, 1 a pair with eight epilogue warps, 2 a pair with four), input gradient, rows a group, n, k, types of rows and results, elements
# more between the result's rows
FORMS = [
    (2, False, RAGGED, 2816, 1408, E4M3, BF16, 0),
    (2, False, RAGGED, 2816, 1408, E5M2, FP16, 0),
    (2, False, RAGGED, 2816, 1408, E4M3, FP32, 0),
    (2, False, RAGGED, 2817, 1424, E4M3, BF16, 0),          # results value by value
    (2, False, RAGGED, 2816, 1424, E5M2, FP16, 5),          # the same for their stride
    (2, False, RAGGED, 2824, 2208, E4M3, FP32, 3),          # two parts, added up in the result
    (2, False, RAGGED, 2816, 16704, E4M3, FP16, 0),         # three parts, in tensor memory
    (2, False, RAGGED, 2816, 16704, E5M2, FP16, 1),
    (2, False, RAGGED, 2816, 8200 * 2, E5M2, FP32, 0),      # nine parts
    (2, False, (900, 700), 2816, 66000, E4M3, BF16, 0),     # two parts
    (2, True, RAGGED, 1408, 2816, E5M2, BF16, 0),
    (2, True, RAGGED, 1408, 2816, E4M3, FP16, 0),
    (2, True, RAGGED, 1403, 2824, E5M2, FP32, 0),           # the summed axis ends inside a block
    (2, True, RAGGED, 2200, 2817, E4M3, BF16, 0),
    (2, True, RAGGED, 2208, 2816, E5M2, FP32, 7),
    (2, True, RAGGED, 16700, 2816, E4M3, FP16, 0),
    (2, True, (4001, 224, 225, 223), 1040, 1000, E5M2, BF16, 0),
    (1, False, RAGGED, 2816, 1024, E4M3, BF16, 0),
    (1, False, RAGGED, 2816, 528, E5M2, FP16, 0),
    (1, False, RAGGED, 2817, 144, E4M3, FP32, 0),
    (1, True, RAGGED, 1024, 2816, E5M2, BF16, 0),
    (1, True, RAGGED, 519, 2824, E4M3, FP16, 3),
    (0, False, (128, 0, 1, 60, 100), 2816, 1408, E4M3, BF16, 0),
    (0, False, (128, 0, 1, 60, 100), 2816, 16704, E5M2, FP16, 0),
    (0, True, (128, 0, 1, 60, 100), 2200, 2817, E5M2, FP32, 0),
]


def form(grad, counts, n, k, rows_more=0, sm_count=None):
    sm_count = sm_count or torch.cuda.get_device_properties(0).multi_processor_count
    return binding.lib().ew_scaled_mm_form(int(grad), sum(counts) + rows_more, len(counts), n, k, sm_count)


def operands(grad, counts, n, k, row_type, first=0, behind=0, seed=0):
    """(rows in blocks, weights in blocks, ends): `first` rows before the first group, `behind` after the last, all NaN."""
    ends = [first] + (first + np.cumsum(counts)).tolist()
    x = uneven((ends[-1] + behind, n if grad else k), BF16, seed + 1, 2.0 ** -10)
    x[:first], x[ends[-1]:] = float("nan"), float("nan")
    return binding.scaled_rows(x, row_type), binding.scaled_pack(uneven((len(counts), n, k), BF16, seed + 3, 0.05)), ends


@pytest.mark.parametrize("case", FORMS, ids=lambda c: "-".join(str(v) for v in c if not isinstance(v, tuple)))
def test_forms(case):
    want, grad, counts, n, k, row_type, out_dtype, more = case
    first, behind = 3, 18
    assert form(grad, counts, n, k, first + behind) == want
    rows, weights, ends = operands(grad, counts, n, k, row_type, first, behind)
    offsets, wide = torch.tensor(ends, dtype=torch.int32, device="cuda"), k if grad else n
    call, terms = (binding.scaled_mm_dx, n) if grad else (binding.scaled_mm, k)
    out = torch.full((ends[-1] + behind, wide + more), 7.0, dtype=out_dtype, device="cuda")
    call(*rows, *weights, offsets, out=out[:, more:])
    for g, (i, j) in enumerate(zip(ends[:-1], ends[1:])):
        xd, wd = values(rows[0][i:j], rows[1][i:j]), values(weights[0][g:g + 1], weights[1][g:g + 1])[0]
        wd = wd if grad else wd.t()
        near(out[i:j, more:], xd @ wd, xd.abs() @ wd.abs(), terms, g)
    assert (out[:first] == 7).all() and (out[ends[-1]:] == 7).all() and (out[:, :more] == 7).all()
    again = torch.full_like(out, 7.0)
    for _ in range(3):
        call(*rows, *weights, offsets, out=again[:, more:])
        assert torch.equal(again, out)
    assert binding.last_operator_error() == 0


@pytest.mark.parametrize("out_dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("grad,n,k", [(False, 2816, 1408), (True, 1408, 2816)])
def test_a_pair_keeps_not_finite_values_in_their_rows(grad, n, k, out_dtype):
    counts = (700, 0, 1, 257, 563)
    assert form(grad, counts, n, k) == 2
    rows, weights, ends = operands(grad, counts, n, k, E4M3)
    offsets, call = torch.tensor(ends, dtype=torch.int32, device="cuda"), binding.scaled_mm_dx if grad else binding.scaled_mm
    clean = call(*rows, *weights, offsets, out_dtype=out_dtype)
    bad = torch.zeros(ends[-1], dtype=torch.bool, device="cuda")
    bad[[0, 130, 255, 699, 700, 901, 1520]] = True
    rows[0].view(torch.uint8)[bad, 77] = 0x7f             # NaN
    rows[1].view(torch.uint8)[701, 3] = 255               # and a NaN among the scales
    bad[701] = True
    got = call(*rows, *weights, offsets, out_dtype=out_dtype)
    assert got[bad].isnan().all() and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("ends", [[0, 900, 500, 1200, 1500], [0, 300, 900, 1700, 1500], [-3, 300, 900, 1200, 1500], [7, 7, 7, 1493, 1400]], ids=str)
def test_a_pair_clamps_and_reports_bad_offsets(ends):
    assert form(False, (375,) * 4, 2816, 1408) == 2
    rows, weights, _ = operands(False, (375,) * 4, 2816, 1408, E4M3)
    got, want = (torch.full((1500, 2816), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    binding.scaled_mm(*rows, *weights, torch.tensor(ends, dtype=torch.int32, device="cuda"), out=got)
    assert binding.last_operator_error() == 1 and binding.last_operator_error() == 0
    fixed = np.maximum.accumulate(np.clip(ends, 0, 1500)).tolist()
    binding.scaled_mm(*rows, *weights, torch.tensor(fixed, dtype=torch.int32, device="cuda"), out=want)
    assert torch.equal(got, want) and binding.last_operator_error() == 0


def test_rows_gathered_by_index():
    """As the README does: a token's rows, once for each of its experts, by indexing both parts of the blocks."""
    tokens, hidden, inter, experts = 50, 512, 128, 4
    q, s, x, t = binding.rms_norm_scaled(uneven((tokens, hidden), BF16, 1), torch.ones(hidden, dtype=BF16, device="cuda"), uneven((tokens, hidden), BF16, 2), with_y=True)
    w = binding.scaled_pack(uneven((experts, 2 * inter, hidden), BF16, 3, 0.05))
    token = torch.arange(2 * tokens, device="cuda") % tokens
    offsets = torch.tensor([0, 30, 30, 31, 100], dtype=torch.int32, device="cuda")
    y = binding.scaled_mm(q[token], s[token], *w, offsets)
    for g, (i, j) in enumerate(zip(offsets.tolist()[:-1], offsets.tolist()[1:])):
        xd, wd = values(q, s)[token[i:j]], values(w[0][g:g + 1], w[1][g:g + 1])[0].t()
        near(y[i:j], xd @ wd, xd.abs() @ wd.abs(), hidden, g)
