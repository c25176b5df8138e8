"""The stand-alone operators and the pool's forward called from other threads than the main one."""
import ctypes as C
import threading

import pytest
import torch

from paper_2508_17624_b200 import binding, build
from paper_2508_17624_b200 import workloads as wl

from helpers import to_dev

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def in_threads(calls):
    """Each call in a thread of its own, all at the same time; their results, or the first exception."""
    results, errors, gate = [None] * len(calls), [], threading.Barrier(len(calls))

    def go(i):
        try:
            gate.wait()
            results[i] = calls[i]()
        except Exception as e:                          # noqa: BLE001 (handed to the test)
            errors.append(e)

    threads = [threading.Thread(target=go, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]
    return results


class Case:
    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(1)
        self.x, self.dy = (torch.randn((300, n), device="cuda", generator=g).to(BF16) for n in (512, 384))
        self.w = (torch.randn((8, 384, 512), device="cuda", generator=g) * 0.05).to(BF16)
        self.offsets = torch.tensor([0, 10, 10, 90, 130, 200, 201, 280, 300], dtype=torch.int32, device="cuda")
        self.q, self.s = binding.quant_pack(self.w, 128)
        self.slots = torch.randint(0, 8, (300,), dtype=torch.int32, device="cuda", generator=g)
        self.ones = torch.ones(300, device="cuda")

    def calls(self):
        return [lambda: binding.grouped_mm(self.x, self.w, self.offsets), lambda: binding.grouped_mm_dx(self.dy, self.w, self.offsets),
                lambda: binding.grouped_mm_dw(self.dy, self.x, self.offsets, out_dtype=FP32), lambda: binding.quant_mv(self.x, self.q, self.s, self.slots),
                lambda: binding.quant_pack(self.w, 64)[0], lambda: binding.swiglu(self.x), lambda: binding.swiglu_grad(self.x[:, :256], self.x, self.ones)[0]]


@pytest.mark.parametrize("which", range(7))
def test_the_first_call_of_a_thread(which):
    """A thread that has made no CUDA call yet has no context either."""
    call = Case().calls()[which]
    want = call()
    torch.cuda.synchronize()
    (got,) = in_threads([call])
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_pools_forward_as_the_first_call_of_a_thread():
    cfg = wl.CONFIGS["c0"]
    pool = binding.Pool.from_config(cfg)
    binding.load_model(pool, cfg)
    x, aid = to_dev(wl.gen_tokens(cfg)), to_dev(wl.gen_adapter_ids(cfg))
    want = pool.moe_forward(0, x, aid)
    torch.cuda.synchronize()
    (got,) = in_threads([lambda: pool.moe_forward(0, x, aid)])
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    pool.destroy()


def test_several_threads_at_once_on_streams_of_their_own():
    case = Case()
    want = [c() for c in case.calls()]
    torch.cuda.synchronize()

    def loop():
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            got = [[c() for c in case.calls()] for _ in range(20)]
        st.synchronize()
        return got

    for got in in_threads([loop] * 4):
        for some in got:
            for a, b in zip(some, want):
                assert torch.equal(a, b)
    assert binding.last_operator_error() == 0


def test_a_threads_own_context_stays_current():
    """A thread that works in a context it made itself is still in it after a call.  (The call sees the device and has nothing to
    do, so nothing of the main context is used in the other one.)"""
    cu, lib = C.CDLL("libcuda.so.1"), binding.lib()
    x = torch.ones((4, 32), dtype=BF16, device="cuda")
    want = binding.swiglu(x)                            # the device's constants are there

    def call():
        mine, now = C.c_void_p(), C.c_void_p()
        assert cu.cuCtxCreate_v2(C.byref(mine), 0, 0) == 0
        # no rows, added to what is there
        assert lib.ew_grouped_mm_dw(0, 0, 2, None, 64, None, 64, 0x1000, 0, 1, 64, 64, 1, 0x1000, 64, 0, None) == 0
        assert cu.cuCtxGetCurrent(C.byref(now)) == 0
        same = now.value == mine.value
        assert cu.cuCtxDestroy_v2(mine) == 0
        return same

    assert in_threads([call]) == [True]
    assert torch.equal(binding.swiglu(x), want)
