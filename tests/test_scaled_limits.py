"""Limits of the stand-alone operators that the host decides; no GPU is needed."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2508_17624_b200 import binding, build

from test_gpu_scaled_limits import FORMS, form

BF16, E4M3, E8M0 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu


def test_operands_with_a_tangent_are_refused():
    """A tangent would be lost without a word, under torch.no_grad() too."""
    x, w, weight = torch.ones((4, 64), dtype=BF16), torch.ones((2, 64, 64), dtype=BF16), torch.ones(64, dtype=BF16)
    offsets, p, q4, scales = torch.zeros(3, dtype=torch.int32), torch.ones(4), torch.zeros((2, 64, 32), dtype=torch.uint8), torch.ones((2, 1, 64), dtype=BF16)
    q, s, wq, ws = x.to(E4M3), torch.ones((4, 1)).to(E8M0), w.to(E4M3), torch.ones((2, 1, 1)).to(E8M0)
    with forward_ad.dual_level():
        xd, wd, pd, sd, vd, qd, wqd = (forward_ad.make_dual(t, t.clone()) for t in (x, w, p, scales, weight, q, wq))
        calls = [lambda: binding.grouped_mm(xd, w, offsets), lambda: binding.grouped_mm(x, wd, offsets), lambda: binding.grouped_mm_dx(xd, w, offsets), lambda: binding.grouped_mm_dw(x, xd, offsets),
                 lambda: binding.grouped_mm_dw(xd, x, offsets), lambda: binding.quant_mv(xd, q4, scales), lambda: binding.quant_mv(x, q4, sd), lambda: binding.swiglu(xd),
                 lambda: binding.swiglu(x, pd), lambda: binding.swiglu_grad(xd, x), lambda: binding.swiglu_grad(x[:, :32], xd), lambda: binding.swiglu_grad(x[:, :32], x, pd),
                 lambda: binding.scaled_rows(xd), lambda: binding.scaled_mm(qd, s, wq, ws, offsets), lambda: binding.scaled_mm(q, s, wqd, ws, offsets),
                 lambda: binding.scaled_mm_dx(qd, s, wq, ws, offsets), lambda: binding.swiglu_scaled(xd), lambda: binding.swiglu_scaled(x, pd), lambda: binding.rms_norm(xd, weight),
                 lambda: binding.rms_norm(x, vd), lambda: binding.rms_norm(x, weight, xd), lambda: binding.rms_norm_scaled(xd, weight), lambda: binding.rms_norm_grad(xd, x, weight),
                 lambda: binding.rms_norm_grad(x, xd, weight), lambda: binding.rms_norm_grad(x, x, vd), lambda: binding.rms_norm_grad(x, x, weight, xd)]
        for call in calls:
            with pytest.raises(ValueError, match="tangent"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                call()
        with pytest.raises(ValueError, match="tangent"):
            binding._result(xd, (4, 64), BF16, x)
        with pytest.raises(ValueError, match="CUDA tensor"):                 # the next check, of operands without one
            binding.rms_norm(forward_ad.unpack_dual(xd).primal, weight, x)


def test_operators_inside_a_function_with_a_jvp():
    """What autograd hands to the halves of a torch.autograd.Function has no tangent: the calls go on to the next check."""
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            with pytest.raises(ValueError, match="CUDA tensor"):
                binding.rms_norm(x, weight)
            return x.clone()

        @staticmethod
        def jvp(ctx, dx, dweight):
            return dx

    x, weight = torch.ones((4, 64), dtype=BF16), torch.ones(64, dtype=BF16)
    with forward_ad.dual_level():
        out = Norm.apply(forward_ad.make_dual(x, 2 * x), weight)
        assert torch.equal(forward_ad.unpack_dual(out).tangent, 2 * x)


def test_the_listed_sizes_reach_every_form():
    """A rule that changes must not leave a form of the product's kernel without its tests."""
    build.build()
    assert [form(grad, counts, n, k, 21, 148) for _, grad, counts, n, k, *_ in FORMS] == [case[0] for case in FORMS]
    for want in range(3):
        assert {case[1] for case in FORMS if case[0] == want} == {False, True}
        assert {case[6] for case in FORMS if case[0] == want} == {BF16, torch.float16, torch.float32}
    assert form(False, (768,) * 64, 2816, 2048, 0, 148) == form(True, (384,) * 64, 2048, 1408, 0, 148) == 2 and form(False, (16,) * 96, 2816, 2048, 0, 148) == 0
