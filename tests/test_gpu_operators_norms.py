"""fp32 results of the stand-alone operators in the 2-norm.

The bounds per element that hold for every input grow with the number of terms and let a result of 16 bits through; over random
terms the errors of a sum cancel, and the 2-norm shows whether fp32 results are fp32 ones.

Grouped products: parts of at most 1024 terms, 64 steps of the tensor core that cut off at most two units of 2^-23 of a running sum
which grows like the square root of its length: at most 64 * 2 * 2/3 * 2^-23 = 1e-5 of the result if all steps cut in its
direction, of which the random signs leave a fraction; bounded by 3e-6 here.  One sign: 1e-5 (half of the running sum's end, two
units, 64 steps: 7.6e-6) and the additions of the parts.
4-bit products: sums of a group are exact (bytes) or 8 steps of fp32 (16 bits); the groups are added up with rounding, half a
unit each: 1e-6.  Two bytes of x instead of three would be 1e-5, a missing line of 256 of 16384 terms 0.12.
"""
import pytest
import torch

from paper_2508_17624_b200 import binding, build
from test_gpu_operators import randn, some_slots, unpacked

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def rel(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("sign", ["random", "one"])
@pytest.mark.parametrize("rows,terms", [(70, 1024), (70, 2056), (600, 1032), (600, 2816), (50, 16384)])
def test_grouped_products_in_fp32(rows, terms, sign, dtype):
    ends = [0, rows // 3, rows // 3, rows]
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, w = randn((rows, terms), dtype, 1), randn((3, 264, terms), dtype, 2, 0.05)
    tall = [randn((3 * terms, v), dtype, v) for v in (264, 136)]
    if sign == "one":
        x, w, tall = x.abs(), w.abs(), [t.abs() for t in tall]
    most = 3e-6 if sign == "random" else 1e-5 + terms / 1024 * 2.0 ** -24
    y = binding.grouped_mm(x, w, offsets, out_dtype=FP32)
    dx = binding.grouped_mm_dx(x, w.transpose(1, 2).contiguous(), offsets, out_dtype=FP32)
    for g in (0, 2):
        i, j = ends[g], ends[g + 1]
        ref = x[i:j].double() @ w[g].double().t()
        assert rel(y[i:j], ref) <= most and rel(dx[i:j], ref) <= most
    offsets = torch.tensor([0, terms, 3 * terms], dtype=torch.int32, device="cuda")
    dw = binding.grouped_mm_dw(*tall, offsets, out_dtype=FP32)
    more = binding.grouped_mm_dw(*tall, offsets, out=torch.zeros_like(dw), accumulate=True)
    for g, (i, j) in enumerate(((0, terms), (terms, 3 * terms))):
        ref = tall[0][i:j].double().t() @ tall[1][i:j].double()
        assert rel(dw[g], ref) <= most + (2 * 2.0 ** -24 if sign == "one" else 0)
        assert torch.equal(more[g], dw[g])


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,per,n_slots", [(1, 6, 8), (3, 2, 6), (40, 2, 5), (70, 1, 3)])
@pytest.mark.parametrize("k", [512, 2048, 16384])
def test_four_bit_products_in_fp32(k, tokens, per, n_slots, group, dtype):
    """Both forms (bytes for up to eight pairs or few a slot, 16 bits for many), one batch of rows and several."""
    slots = some_slots(tokens, per, n_slots, k)
    x = randn((tokens, k), dtype, 1)
    q, scales = binding.quant_pack(randn((n_slots, 72, k), dtype, 2, 0.05), group)
    w = unpacked(q, scales)
    y = binding.quant_mv(x, q, scales, slots, out_dtype=FP32).view(tokens, per, 72)
    ref = torch.einsum("tk,tpnk->tpn", x.double(), w[slots.long()]) if tokens * per * k <= 2 ** 18 else torch.stack(
        [torch.stack([w[s] @ x[t].double() for s in slots[t].tolist()]) for t in range(tokens)])
    assert rel(y, ref) <= 1e-6
    for t in range(tokens):                             # and no pair by itself hides in the others
        assert rel(y[t], ref[t]) <= 2e-6
