"""Limits of the operators in 8-bit floating point: sums next to the last bit of what the tensor core keeps.

Tolerances.  An instruction adds 32 products (16 of 16-bit operands) to the running sum.  It cuts each addend off below 2^-25 of the
largest one's power of two, and the sum behind its 24th bit: (32 + 1) 2^-25 + 2^-23 = 9.25 * 2^-23 of S = sum |a b| at most
(5.25 * 2^-23 for 16).  The parts of a long sum each lose that of their own S, and are added up with half a step of fp32 each.
"""
import pytest
import torch

from paper_2508_17624_b200 import binding

from test_gpu_scaled import values

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
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
