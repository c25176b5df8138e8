"""ctypes binding over libexpertweave.so: argument marshalling only.

Function names mirror the C ABI (`include/expertweave.h`).  Host weights are numpy uint16 arrays of
bf16 bit patterns; device operands are torch CUDA tensors, passed by data pointer together with the
current CUDA stream.  There is no CPU fallback: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libexpertweave.so")

EW_OK = 0
STATUS_NAMES = ["EW_OK", "EW_ERR_INVALID_ARG", "EW_ERR_OOM", "EW_ERR_SLOT_IN_USE", "EW_ERR_NOT_LOADED",
                "EW_ERR_TOO_MANY_EXPERTS", "EW_ERR_CUDA", "EW_ERR_TIMEOUT", "EW_ERR_BAD_ADAPTER_ID_IN_BATCH",
                "EW_ERR_NO_DEVICE"]
EXPORTS = ["ew_pool_create", "ew_pool_destroy", "ew_load_base", "ew_load_adapter", "ew_unload_adapter",
           "ew_pool_trim", "ew_moe_forward", "ew_moe_forward_debug", "ew_moe_forward_host", "ew_profile_enable",
           "ew_profile_read", "ew_reroute", "ew_reroute_unfused", "ew_route_logits", "ew_route_noalloc", "ew_selftest_bounded_wait", "ew_get_expert_map",
           "ew_moe_forward_partial", "ew_ep_finish", "ew_moe_forward_scatter", "ew_ep_finish_gathered", "ew_pool_stats", "ew_last_device_error", "ew_slot_address", "ew_grouped_mm", "ew_grouped_mm_dx", "ew_grouped_mm_dw",
           "ew_quant_mv", "ew_quant_pack", "ew_swiglu", "ew_swiglu_grad", "ew_scaled_rows", "ew_scaled_pack", "ew_scaled_mm", "ew_scaled_mm_dx", "ew_scaled_mm_form",
           "ew_swiglu_scaled", "ew_rms_norm", "ew_rms_norm_grad", "ew_rms_norm_grad_parts", "ew_last_operator_error", "ew_status_str", "ew_last_error_string"]


class EwConfig(C.Structure):
    _fields_ = [("device", C.c_int32), ("num_layers", C.c_int32), ("hidden", C.c_int32), ("inter", C.c_int32),
                ("num_experts", C.c_int32), ("num_shared", C.c_int32), ("top_k", C.c_int32),
                ("max_adapters", C.c_int32), ("e_max", C.c_int32), ("max_tokens", C.c_int32),
                ("renormalize", C.c_int32), ("routed_scale", C.c_float), ("pool_mode", C.c_int32),
                ("ep_size", C.c_int32), ("page_bytes", C.c_uint64), ("prealloc_pages", C.c_uint64),
                ("max_pages", C.c_uint64), ("ep_rank", C.c_int32), ("reserved0", C.c_int32)]


class EwStats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in
                ("page_bytes", "va_reserved_bytes", "pages_mapped", "pages_free", "pages_created_total",
                 "physical_bytes", "live_expert_bytes", "padding_bytes", "live_experts", "adapters_loaded",
                 "workspace_bytes", "last_forward_kernels")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class EwError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{where}: {name}" + (f" ({detail})" if detail else ""))


_lib = None


def lib():
    """Load the shared library (raises if it has not been built: there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2508_17624_b200.build` "
                               "(the CUDA extension is required; there is no CPU fallback)")
        loaded = C.CDLL(LIB_PATH)
        loaded.ew_status_str.restype = C.c_char_p
        loaded.ew_last_error_string.restype = C.c_char_p
        for name in EXPORTS:
            getattr(loaded, name)
        # the stand-alone operators are called with plain integers (addresses among them)
        i32, i64, ptr = C.c_int32, C.c_int64, C.c_void_p
        for name in ("ew_grouped_mm", "ew_grouped_mm_dx"):
            getattr(loaded, name).argtypes = [i32, i32, i32, ptr, i64, ptr, i64, i64, ptr, i32, i32, i32, i32, ptr, i64, ptr]
        loaded.ew_grouped_mm_dw.argtypes = [i32, i32, i32, ptr, i64, ptr, i64, ptr, i32, i32, i32, i32, i32, ptr, i64, i64, ptr]
        loaded.ew_quant_mv.argtypes = [i32, i32, i32, ptr, i64, ptr, ptr, ptr, i32, i32, i32, i32, i32, i32, ptr, i64, ptr]
        loaded.ew_quant_pack.argtypes = [i32, i32, ptr, i64, i64, i32, i32, i32, i32, ptr, ptr, ptr]
        loaded.ew_swiglu.argtypes = [i32, i32, ptr, i64, ptr, i32, i32, ptr, i64, ptr]
        loaded.ew_swiglu_grad.argtypes = [i32, i32, ptr, i64, ptr, i64, ptr, i32, i32, ptr, i64, ptr, ptr]
        loaded.ew_scaled_rows.argtypes = [i32, i32, i32, ptr, i64, i32, i32, ptr, i64, ptr, i64, ptr]
        loaded.ew_scaled_pack.argtypes = [i32, i32, ptr, i64, i64, i32, i32, i32, ptr, i64, i64, ptr, ptr]
        for name in ("ew_scaled_mm", "ew_scaled_mm_dx"):
            getattr(loaded, name).argtypes = [i32, i32, i32, ptr, i64, ptr, i64, ptr, i64, i64, ptr, ptr, i32, i32, i32, i32, ptr, i64, ptr]
        loaded.ew_swiglu_scaled.argtypes = [i32, i32, ptr, i64, ptr, i32, i32, ptr, i64, ptr, i64, ptr]
        loaded.ew_rms_norm.argtypes = [i32, i32, ptr, i64, ptr, i64, ptr, C.c_float, i32, i32, ptr, i64, ptr, i64, ptr, i64, ptr, i64, ptr]
        loaded.ew_rms_norm_grad.argtypes = [i32, i32, ptr, i64, ptr, i64, ptr, ptr, i64, C.c_float, i32, i32, ptr, i64, ptr, ptr, ptr]
        _lib = loaded                                      # (complete: another thread may be waiting for it to be there)
    return _lib


def _check(rc: int, where: str):
    if rc != EW_OK:
        detail = lib().ew_last_error_string().decode() if rc == 6 or rc == 2 or rc == 1 else ""
        raise EwError(rc, where, detail)


def _host(a, dtype=np.uint16) -> Optional[np.ndarray]:
    if a is None:
        return None
    return np.ascontiguousarray(a, dtype=dtype)


def _hp(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _dp(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class Pool:
    """Owner of one `ew_pool_t`.  Methods carry the names of the C entry points without the prefix."""

    def __init__(self, *, device: int = 0, num_layers: int = 1, hidden: int, inter: int, num_experts: int,
                 num_shared: int, top_k: int, max_adapters: int, e_max: int, max_tokens: int,
                 renormalize: int = 0, routed_scale: float = 1.0, pool_mode: int = 0, page_bytes: int = 0,
                 prealloc_pages: int = 0, max_pages: int = 0, ep_size: int = 0, ep_rank: int = 0):
        self.cfg = EwConfig(device, num_layers, hidden, inter, num_experts, num_shared, top_k, max_adapters,
                            e_max, max_tokens, renormalize, routed_scale, pool_mode, ep_size, page_bytes,
                            prealloc_pages, max_pages, ep_rank, 0)
        self._h = C.c_void_p()
        _check(lib().ew_pool_create(C.byref(self.cfg), C.byref(self._h)), "ew_pool_create")

    @classmethod
    def from_config(cls, cfg, *, device: int = 0, max_tokens: Optional[int] = None, **kw) -> "Pool":
        """`cfg` is a `workloads.MoEConfig`."""
        return cls(device=device, num_layers=cfg.num_layers, hidden=cfg.hidden, inter=cfg.inter,
                   num_experts=cfg.num_experts, num_shared=cfg.num_shared, top_k=cfg.top_k,
                   max_adapters=cfg.max_adapters, e_max=cfg.e_max, max_tokens=max_tokens or cfg.n_tokens, **kw)

    @property
    def num_slots(self) -> int:
        return self.cfg.num_experts + self.cfg.max_adapters * self.cfg.e_max

    def destroy(self):
        if self._h:
            _check(lib().ew_pool_destroy(self._h), "ew_pool_destroy")
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def load_base(self, layer, router_w, w_gate, w_up, w_down, sh_gate=None, sh_up=None, sh_down=None):
        arrs = [_host(a) for a in (router_w, w_gate, w_up, w_down, sh_gate, sh_up, sh_down)]
        _check(lib().ew_load_base(self._h, layer, *[_hp(a) for a in arrs]), "ew_load_base")

    def load_adapter(self, adapter_id, counts, expert_ids, w_gate, w_up, w_down):
        """Weights: numpy arrays of bf16 bit patterns (host), or torch tensors (host or device) taken as they are."""
        counts = _host(counts, np.int32)
        expert_ids = _host(expert_ids, np.int32)
        keep = [a if hasattr(a, "data_ptr") else _host(a) for a in (w_gate, w_up, w_down)]   # alive during the call
        g, u, d = [_dp(a) if hasattr(a, "data_ptr") else _hp(a) for a in keep]
        _check(lib().ew_load_adapter(self._h, adapter_id, _hp(counts), _hp(expert_ids), g, u, d), "ew_load_adapter")

    def unload_adapter(self, adapter_id):
        _check(lib().ew_unload_adapter(self._h, adapter_id), "ew_unload_adapter")

    def trim(self):
        _check(lib().ew_pool_trim(self._h), "ew_pool_trim")

    def moe_forward(self, layer, x, adapter_ids, out=None):
        import torch
        if out is None:
            out = torch.empty_like(x)
        _check(lib().ew_moe_forward(self._h, layer, _dp(x), _dp(adapter_ids), x.shape[0], _dp(out), _stream()),
               "ew_moe_forward")
        return out

    def moe_forward_partial(self, layer, x, adapter_ids, partial=None):
        """This rank's unrounded partial sums, fp32 [n_tokens, H] (expert parallelism; see the header)."""
        import torch
        if partial is None:
            partial = torch.empty(x.shape, dtype=torch.float32, device=x.device)
        _check(lib().ew_moe_forward_partial(self._h, layer, _dp(x), _dp(adapter_ids), x.shape[0], _dp(partial), _stream()),
               "ew_moe_forward_partial")
        return partial

    def ep_finish(self, summed, out=None):
        """bf16 result from the sum of all ranks' partials."""
        import torch
        if out is None:
            out = torch.empty(summed.shape, dtype=torch.bfloat16, device=summed.device)
        _check(lib().ew_ep_finish(self._h, _dp(summed), summed.shape[0], _dp(out), _stream()), "ew_ep_finish")
        return out

    def moe_forward_scatter(self, layer, x, adapter_ids, gather_ptrs):
        """Partial forward whose last kernel stores the partial sums into every rank's gather buffer; `gather_ptrs`:
        device int64 tensor with the ep_size buffer addresses (see the header)."""
        _check(lib().ew_moe_forward_scatter(self._h, layer, _dp(x), _dp(adapter_ids), x.shape[0], _dp(gather_ptrs), _stream()),
               "ew_moe_forward_scatter")

    def ep_finish_gathered(self, gathered, out=None):
        """bf16 result from this rank's gather buffer [ep_size, n_tokens, H] (blocks added in rank order)."""
        import torch
        if out is None:
            out = torch.empty(gathered.shape[1:], dtype=torch.bfloat16, device=gathered.device)
        _check(lib().ew_ep_finish_gathered(self._h, _dp(gathered), gathered.shape[1], _dp(out), _stream()), "ew_ep_finish_gathered")
        return out

    def moe_forward_debug(self, layer, x, adapter_ids):
        import torch
        B, k, P = x.shape[0], self.cfg.top_k, self.num_slots
        dev = x.device
        out = torch.empty_like(x)
        r = dict(topk_ids=torch.empty((B, k), dtype=torch.int32, device=dev),
                 topk_w=torch.empty((B, k), dtype=torch.float32, device=dev),
                 slot_ids=torch.empty((B, k), dtype=torch.int32, device=dev),
                 counts=torch.empty((P,), dtype=torch.int32, device=dev),
                 inv=torch.empty((B, k), dtype=torch.int32, device=dev),
                 offsets=torch.empty((P + 1,), dtype=torch.int32, device=dev))
        _check(lib().ew_moe_forward_debug(self._h, layer, _dp(x), _dp(adapter_ids), B, _dp(out), _stream(),
                                          _dp(r["topk_ids"]), _dp(r["topk_w"]), _dp(r["slot_ids"]), _dp(r["counts"]),
                                          _dp(r["inv"]), _dp(r["offsets"])), "ew_moe_forward_debug")
        r["out"] = out
        return r

    def moe_forward_host(self, layer, x_host, adapter_ids_host, out_host, n_tokens=None):
        """x_host / out_host: pinned torch CPU tensors (or numpy arrays); asynchronous on the current stream."""
        def hp(t):
            return C.c_void_p(t.data_ptr()) if hasattr(t, "data_ptr") else t.ctypes.data_as(C.c_void_p)
        n = x_host.shape[0] if n_tokens is None else n_tokens
        _check(lib().ew_moe_forward_host(self._h, layer, hp(x_host), hp(adapter_ids_host), n, hp(out_host),
                                         _stream()), "ew_moe_forward_host")
        return out_host

    def profile_enable(self, on: bool):
        _check(lib().ew_profile_enable(self._h, int(on)), "ew_profile_enable")

    def profile_read(self):
        """-> (dict kernel -> total ms, forwards measured)"""
        ms = (C.c_double * 5)()
        n = C.c_int32(0)
        _check(lib().ew_profile_read(self._h, ms, C.byref(n)), "ew_profile_read")
        names = ("route", "permute", "gemm1", "gemm2", "combine")
        return {k: float(v) for k, v in zip(names, ms)}, int(n.value)

    def reroute(self, layer, topk_ids, adapter_ids, slot_ids=None, counts=None, want_counts=True):
        import torch
        if slot_ids is None:
            slot_ids = torch.empty_like(topk_ids)
        if counts is None and want_counts:
            counts = torch.empty((self.num_slots,), dtype=torch.int32, device=topk_ids.device)
        _check(lib().ew_reroute(self._h, layer, _dp(topk_ids), _dp(adapter_ids), topk_ids.shape[0], _dp(slot_ids),
                                _dp(counts), _stream()), "ew_reroute")
        return slot_ids, counts

    def reroute_unfused(self, layer, topk_ids, adapter_ids, slot_ids=None, counts=None, want_counts=True, scratch=None):
        """The same rewrite as `reroute`, as one kernel per elementary tensor operation (ablation)."""
        import torch
        if slot_ids is None:
            slot_ids = torch.empty_like(topk_ids)
        if counts is None and want_counts:
            counts = torch.empty((self.num_slots,), dtype=torch.int32, device=topk_ids.device)
        if scratch is None:
            scratch = torch.empty((2 * topk_ids.numel(),), dtype=torch.int32, device=topk_ids.device)
        _check(lib().ew_reroute_unfused(self._h, layer, _dp(topk_ids), _dp(adapter_ids), topk_ids.shape[0], _dp(slot_ids),
                                        _dp(counts), _dp(scratch), _stream()), "ew_reroute_unfused")
        return slot_ids, counts

    def route_logits(self, layer, logits, adapter_ids):
        """Softmax + top-k + rerouting + per-slot counts from fp32 logits [n, M] (device tensors)."""
        import torch
        n, k, dev = logits.shape[0], self.cfg.top_k, logits.device
        ids = torch.empty((n, k), dtype=torch.int32, device=dev)
        w = torch.empty((n, k), dtype=torch.float32, device=dev)
        slots = torch.empty((n, k), dtype=torch.int32, device=dev)
        counts = torch.empty((self.num_slots,), dtype=torch.int32, device=dev)
        _check(lib().ew_route_logits(self._h, layer, _dp(logits), _dp(adapter_ids), n, _dp(ids), _dp(w), _dp(slots),
                                     _dp(counts), _stream()), "ew_route_logits")
        return ids, w, slots, counts

    def route_noalloc(self, layer, x, adapter_ids, topk_ids, topk_w, slot_ids, counts, device_status=None):
        """Routing into caller-provided device tensors; the library allocates nothing (see the header)."""
        _check(lib().ew_route_noalloc(self._h, layer, _dp(x), _dp(adapter_ids), x.shape[0], _dp(topk_ids),
                                      _dp(topk_w), _dp(slot_ids), _dp(counts), _dp(device_status), _stream()),
               "ew_route_noalloc")

    def selftest_bounded_wait(self):
        _check(lib().ew_selftest_bounded_wait(self._h, _stream()), "ew_selftest_bounded_wait")

    def get_expert_map(self, layer) -> np.ndarray:
        out = np.empty((self.cfg.max_adapters, self.cfg.num_experts), np.int32)
        _check(lib().ew_get_expert_map(self._h, layer, _hp(out)), "ew_get_expert_map")
        return out

    def stats(self) -> dict:
        s = EwStats()
        _check(lib().ew_pool_stats(self._h, C.byref(s)), "ew_pool_stats")
        return s.as_dict()

    def last_device_error(self) -> int:
        code = C.c_int32(0)
        _check(lib().ew_last_device_error(self._h, C.byref(code)), "ew_last_device_error")
        return code.value

    def slot_address(self, layer, which, slot) -> int:
        p = C.c_void_p()
        _check(lib().ew_slot_address(self._h, layer, which, slot, C.byref(p)), "ew_slot_address")
        return p.value or 0


# ---------------------------------------------------------------------------------------------------------------------
# Stand-alone operators (no pool): argument checks, output allocation, one library call on the current stream.  A small
# call takes the GPU less time than the host, so the checks of a good call are a handful of comparisons; only when one of
# them fails does `_on` find out which and say so.  autograd does not see the calls: an operand that it is recording, or that carries
# a tangent of forward-mode differentiation, is refused, since a result without one would go unnoticed (torch.autograd.Function runs
# its halves unrecorded and without tangents).
class _Torch:
    """What the operators need of torch, resolved on first use (the package imports without it)."""
    ready = False

    @classmethod
    def load(cls):
        import torch
        from torch.autograd import forward_ad
        cls.forward = forward_ad
        cls.codes = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
        cls.int32, cls.float32, cls.uint8, cls.bfloat16 = torch.int32, torch.float32, torch.uint8, torch.bfloat16
        cls.e4m3, cls.e5m2, cls.exponent = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
        cls.eights = {torch.float8_e4m3fn: 3, torch.float8_e5m2: 4}
        cls.recording, cls.empty_like, cls.empty = torch.is_grad_enabled, torch.empty_like, torch.empty_strided      # (half a microsecond less than new_empty)
        cls.stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
        cls.ready = True
        return cls


def _torch():
    return _Torch if _Torch.ready else _Torch.load()


def _on(t, like=None, ndim=2, name="operand", dtype=None):
    """Checks a device tensor: dimensions, type, contiguous innermost dimension, the same device as `like`."""
    if not t.is_cuda or t.dim() != ndim:
        raise ValueError(f"{name}: a {ndim}-dimensional CUDA tensor is wanted, got {tuple(t.shape)} on {t.device}")
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, the other operands on {like.device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, {dtype} is wanted")
    if t.numel() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the innermost dimension is not contiguous")
    return t


def _recorded(where):
    raise ValueError(f"{where}: autograd is recording an operand and would lose its gradient here; call it under torch.no_grad() or inside "
                     "a torch.autograd.Function, and the gradient's operators in its backward")


def _without_tangents(where, *operands):
    """For calls while forward-mode differentiation is on (torch.no_grad() leaves it on)."""
    for t in operands:
        if t is not None and _Torch.forward.unpack_dual(t).tangent is not None:
            raise ValueError(f"{where}: forward-mode autograd's tangent of a tensor would be lost here; pass what torch.autograd.forward_ad.unpack_dual "
                             "gives, or call it inside a torch.autograd.Function that has a jvp")


def _code(T, dtype) -> int:
    code = T.codes.get(dtype)
    if code is None:
        raise ValueError(f"dtype {dtype} is not supported: bfloat16, float16 (results also float32)")
    return code


_MOST = 2 ** 31 - 1                                     # of a size: the library takes 32-bit ones, and ctypes would cut a larger one down


def _too_large(what, *sizes):
    raise ValueError(f"{what}: sizes of {', '.join(map(str, sizes))}; the library takes up to {_MOST}")


def _good(t, dev, dtype, ndim) -> bool:
    """Whether `t` is what `_on` wants (contiguity of the last dimension apart)."""
    return t.get_device() == dev and t.dtype is dtype and t.dim() == ndim


def _matrix(t, dev, dtype, name, like):
    """(rows, width, elements between rows) of a matrix; one row alone has no stride of its own."""
    if t.get_device() != dev or t.dtype is not dtype or t.dim() != 2 or dev < 0:
        _on(t, like, 2, name, dtype)
    (rows, width), (ld, one) = t.shape, t.stride()
    if one != 1 and width > 1 and rows:
        _on(t, like, 2, name, dtype)
    if rows > _MOST or width > _MOST:
        _too_large(name, rows, width)
    return rows, width, ld if rows > 1 else (width + 7) // 8 * 8


def _matrices(t, dev, dtype, name, like):
    """(matrices, rows, width, elements between rows, between matrices)."""
    if t.get_device() != dev or t.dtype is not dtype or t.dim() != 3 or dev < 0:
        _on(t, like, 3, name, dtype)
    (g, n, k), (stride, ld, one) = t.shape, t.stride()
    if one != 1 and k > 1:
        _on(t, like, 3, name, dtype)
    if g > _MOST or n > _MOST or k > _MOST:
        _too_large(name, g, n, k)
    ld = ld if n > 1 else (k + 7) // 8 * 8
    return g, n, k, ld, stride if g > 1 else n * ld


def _offsets(offsets, dev, T, like):
    n = offsets.numel()
    if offsets.get_device() != dev or offsets.dtype is not T.int32 or offsets.dim() != 1 or n < 2 or not offsets.is_contiguous():
        _on(offsets, like, 1, "offsets")
        raise ValueError("offsets: a contiguous int32 tensor with one more entry than groups is wanted")
    if n - 1 > _MOST:
        _too_large("offsets", n)
    return n - 1


def _result(out, shape, dtype, like, name="out"):
    if out is None:
        return like.new_empty(shape, dtype=dtype)
    if out.requires_grad and _torch().recording():
        raise ValueError(f"{name}: autograd is recording it and would not see it overwritten; pass it under torch.no_grad(), or a tensor of its own")
    if _torch().forward._current_level >= 0:
        _without_tangents(name, out)
    _on(out, like, len(shape), name)
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype:
        raise ValueError(f"{name}: {tuple(shape)} of {dtype} is wanted, got {tuple(out.shape)} of {out.dtype}")
    return out


def _rows_product(fn, where, a, w, offsets, out, out_dtype, grad):
    T, dev, dtype = _torch(), a.get_device(), a.dtype
    if (a.requires_grad or w.requires_grad) and T.recording():
        _recorded(where)
    if T.forward._current_level >= 0:
        _without_tangents(where, a, w)
    code = _code(T, dtype)
    rows, width, lda = _matrix(a, dev, dtype, "the rows' operand", None)
    groups, n, k, ldw, stride = _matrices(w, dev, dtype, "w", a)
    if _offsets(offsets, dev, T, a) != groups:
        raise ValueError(f"offsets has {offsets.shape[0]} entries for {groups} groups")
    if width != (n if grad else k):
        raise ValueError(f"rows of {width} do not match w of {tuple(w.shape)}")
    if out_dtype is None:
        out_dtype = dtype if out is None else out.dtype
    wide = k if grad else n
    if out is None:
        out, ldo = a.new_empty((rows, wide)) if out_dtype is dtype else a.new_empty((rows, wide), dtype=out_dtype), wide
    else:
        out = _result(out, (rows, wide), out_dtype, a)
        ldo = out.stride(0) if rows > 1 else wide
    rc = fn(dev, code, _code(T, out_dtype), a.data_ptr(), lda, w.data_ptr(), ldw, stride, offsets.data_ptr(), rows, groups, n, k,
            out.data_ptr(), ldo, T.stream(dev))
    if rc:
        _check(rc, where)
    return out


def grouped_mm(x, w, offsets, out=None, out_dtype=None):
    """y[r] = x[r] w[g]^T for the rows offsets[g] <= r < offsets[g+1] of each group: x [rows, k], w [groups, n, k], offsets
    int32 [groups + 1] (all on one device).  Rows outside the offsets are left as they were in `out`, and undefined in a
    new result.  out_dtype: x's type
    or float32.  See the header for alignment."""
    return _rows_product(lib().ew_grouped_mm, "ew_grouped_mm", x, w, offsets, out, out_dtype, False)


def grouped_mm_dx(dy, w, offsets, out=None, out_dtype=None):
    """The gradient of `grouped_mm` with respect to x: dx[r] = dy[r] w[g]; dy [rows, n] -> [rows, k]."""
    return _rows_product(lib().ew_grouped_mm_dx, "ew_grouped_mm_dx", dy, w, offsets, out, out_dtype, True)


def grouped_mm_dw(dy, x, offsets, out=None, out_dtype=None, accumulate=False):
    """The gradient of `grouped_mm` with respect to w: dw[g] = dy_g^T x_g -> [groups, n, k]; a group without rows gets zeros.
    accumulate: adds to `out` instead (required then), as over the steps of a large batch."""
    T, dev, dtype = _torch(), dy.get_device(), dy.dtype
    if (dy.requires_grad or x.requires_grad) and T.recording():
        _recorded("ew_grouped_mm_dw")
    if T.forward._current_level >= 0:
        _without_tangents("ew_grouped_mm_dw", dy, x)
    code = _code(T, dtype)
    rows, n, lddy = _matrix(dy, dev, dtype, "dy", None)
    x_rows, k, ldx = _matrix(x, dev, dtype, "x", dy)
    groups = _offsets(offsets, dev, T, dy)
    if x_rows != rows:
        raise ValueError(f"dy has {rows} rows, x {x_rows}")
    if accumulate and out is None:
        raise ValueError("accumulate adds to `out`: pass it")
    if out_dtype is None:
        out_dtype = dtype if out is None else out.dtype
    if out is None:
        out, ldo, stride = dy.new_empty((groups, n, k), dtype=out_dtype), k, n * k
    else:
        out = _result(out, (groups, n, k), out_dtype, dy)
        ldo = out.stride(1) if n > 1 else k
        stride = out.stride(0) if groups > 1 else n * ldo
    rc = lib().ew_grouped_mm_dw(dev, code, _code(T, out_dtype), dy.data_ptr(), lddy, x.data_ptr(), ldx, offsets.data_ptr(), rows, groups, n, k,
                                1 if accumulate else 0, out.data_ptr(), ldo, stride, T.stream(dev))
    if rc:
        _check(rc, "ew_grouped_mm_dw")
    return out


def quant_pack(w, group, out=None):
    """4-bit weights and group scales of w [slots, n, k] (bf16 or fp16) for `quant_mv`: (q uint8 [slots, n, k/2], scales
    [slots, k/group, n] of w's type).  The header has the format.  Not differentiable: w may be a parameter, the result is data."""
    T, dev, dtype = _torch(), w.get_device(), w.dtype
    code = _code(T, dtype)
    slots, n, k, ld, stride = _matrices(w, dev, dtype, "w", None)
    if group not in (32, 64, 128) or k % group:
        raise ValueError(f"groups of 32, 64 or 128 weights that divide k = {k} are wanted, got {group}")
    q, scales = out or (None, None)
    q = _result(q, (slots, n, k // 2), T.uint8, w, "q")
    scales = _result(scales, (slots, k // group, n), dtype, w, "scales")
    if not (q.is_contiguous() and scales.is_contiguous()):
        raise ValueError("q and scales are contiguous")
    _check(lib().ew_quant_pack(dev, code, w.data_ptr(), ld, stride, slots, n, k, group, q.data_ptr(), scales.data_ptr(), T.stream(dev)), "ew_quant_pack")
    return q, scales


def quant_mv(x, q, scales, slots=None, out=None, out_dtype=None):
    """y[p] = x[p // per_row] W[slots[p]]^T with the 4-bit weights of `quant_pack`.  x [rows, k]; slots int32, one entry a
    pair in any shape ([tokens, top_k] as the router writes it), per_row = pairs / rows of x; negative: a row of zeros.
    slots None: one matrix, a pair a row.  -> [pairs, n]; out_dtype: x's type or float32."""
    T, dev, dtype = _torch(), x.get_device(), x.dtype
    if (x.requires_grad or scales.requires_grad) and T.recording():
        _recorded("ew_quant_mv")
    if T.forward._current_level >= 0:
        _without_tangents("ew_quant_mv", x, scales)
    code = _code(T, dtype)
    rows, k, ldx = _matrix(x, dev, dtype, "x", None)
    if not _good(q, dev, T.uint8, 3):
        _on(q, x, 3, "q", T.uint8)
    if not _good(scales, dev, dtype, 3):
        _on(scales, x, 3, "scales", dtype)
    (n_slots, n, half), (s_slots, groups, s_n) = q.shape, scales.shape
    if half * 2 != k or groups < 1 or k % groups or s_slots != n_slots or s_n != n or not q.is_contiguous() or not scales.is_contiguous():
        raise ValueError(f"x {tuple(x.shape)}, q {tuple(q.shape)} and scales {tuple(scales.shape)} do not belong together")
    pairs, per_row = rows, 1
    if slots is not None:
        if slots.get_device() != dev or slots.dtype is not T.int32 or not slots.is_contiguous():
            raise ValueError("slots: a contiguous int32 tensor on x's device is wanted")
        pairs = slots.numel()
        if pairs and (rows == 0 or pairs % rows):
            raise ValueError(f"{pairs} pairs for {rows} rows of x")
        per_row = pairs // rows if pairs else 1
    if pairs > _MOST or n_slots > _MOST or n > _MOST:
        _too_large("slots and q", pairs, n_slots, n)
    if out_dtype is None:
        out_dtype = dtype if out is None else out.dtype
    if out is None:
        out, ldo = x.new_empty((pairs, n)) if out_dtype is dtype else x.new_empty((pairs, n), dtype=out_dtype), n
    else:
        out = _result(out, (pairs, n), out_dtype, x)
        ldo = out.stride(0) if pairs > 1 else n
    rc = lib().ew_quant_mv(dev, code, _code(T, out_dtype), x.data_ptr(), ldx, q.data_ptr(), scales.data_ptr(), None if slots is None else slots.data_ptr(), pairs, per_row, n_slots, n, k,
                           k // groups, out.data_ptr(), ldo, T.stream(dev))
    if rc:
        _check(rc, "ew_quant_mv")
    return out


def _row_weights(p, dev, T, rows, like):
    if p is None:
        return None
    if not _good(p, dev, T.float32, 1) or not p.is_contiguous():
        _on(p, like, 1, "row_weights", T.float32)
    if p.shape[0] != rows:
        raise ValueError(f"{p.shape[0]} row weights for {rows} rows")
    return p.data_ptr()


def swiglu(h, row_weights=None, out=None):
    """row_weights[r] * silu(h[r, :inter]) * h[r, inter:] -> [rows, inter]: the activation between an expert's linears, the
    routing weights (float32, or None) folded in."""
    T, dev, dtype = _torch(), h.get_device(), h.dtype
    if (h.requires_grad or (row_weights is not None and row_weights.requires_grad)) and T.recording():
        _recorded("ew_swiglu")
    if T.forward._current_level >= 0:
        _without_tangents("ew_swiglu", h, row_weights)
    code = _code(T, dtype)
    rows, two, ldh = _matrix(h, dev, dtype, "h", None)
    if two < 2 or two % 2:
        raise ValueError(f"h holds a gate and an up block side by side: an even width is wanted, got {two}")
    inter = two // 2
    p = _row_weights(row_weights, dev, T, rows, h)
    if out is None:
        out, ldo = h.new_empty((rows, inter)), inter
    else:
        out = _result(out, (rows, inter), dtype, h)
        ldo = out.stride(0) if rows > 1 else inter
    rc = lib().ew_swiglu(dev, code, h.data_ptr(), ldh if rows > 1 else two, p, rows, inter, out.data_ptr(), ldo, T.stream(dev))
    if rc:
        _check(rc, "ew_swiglu")
    return out


def swiglu_grad(dact, h, row_weights=None, out=None):
    """The gradient of `swiglu`: dh [rows, 2 inter], and with row_weights also theirs, float32 [rows] -> dh or (dh, dp)."""
    T, dev, dtype = _torch(), h.get_device(), h.dtype
    if (h.requires_grad or dact.requires_grad or (row_weights is not None and row_weights.requires_grad)) and T.recording():
        _recorded("ew_swiglu_grad")
    if T.forward._current_level >= 0:
        _without_tangents("ew_swiglu_grad", dact, h, row_weights)
    code = _code(T, dtype)
    rows, two, ldh = _matrix(h, dev, dtype, "h", None)
    d_rows, inter, ldd = _matrix(dact, dev, dtype, "dact", h)
    if two < 2 or d_rows != rows or inter * 2 != two:
        raise ValueError(f"dact {tuple(dact.shape)} does not belong to h {tuple(h.shape)}")
    p = _row_weights(row_weights, dev, T, rows, h)
    if out is None:
        out, ldo = h.new_empty((rows, two)), two
    else:
        out = _result(out, (rows, two), dtype, h)
        ldo = out.stride(0) if rows > 1 else two
    dp = None if p is None else h.new_empty((rows,), dtype=T.float32)
    rc = lib().ew_swiglu_grad(dev, code, dact.data_ptr(), ldd if rows > 1 else inter, h.data_ptr(), ldh if rows > 1 else two, p, rows, inter, out.data_ptr(),
                              ldo, None if dp is None else dp.data_ptr(), T.stream(dev))
    if rc:
        _check(rc, "ew_swiglu_grad")
    return out if dp is None else (out, dp)


# 8-bit floating point in blocks of 128: q (float8_e4m3fn or float8_e5m2) and scales (float8_e8m0fnu, powers of two).  Rows of
# q lie on 16-byte boundaries, as the products want them, and rows of scales on 4-byte ones, as they like them: results are views of
# padded tensors where the width is no multiple of 16 or 512.
def _eight(T, dtype, name) -> int:
    code = T.eights.get(dtype)
    if code is None:
        raise ValueError(f"{name}: dtype {dtype} is not supported: float8_e4m3fn, float8_e5m2")
    return code


def _room(width, step):
    return (width + step - 1) // step * step


def _row_blocks(out, rows, width, dtype, T, like):
    """(q, scales, elements between q's rows, between the scales') of a result in blocks."""
    if out is None:
        wide, blocks = (width + 15) // 16 * 16, (width + 127) // 128
        room = (blocks + 3) // 4 * 4
        at = like.device
        q, scales = T.empty((rows, wide), (wide, 1), dtype=dtype, device=at), T.empty((rows, room), (room, 1), dtype=T.exponent, device=at)
        return q if wide == width else q[:, :width], scales if room == blocks else scales[:, :blocks], wide, room
    q, scales = out
    q, scales = _result(q, (rows, width), dtype, like, "q"), _result(scales, (rows, (width + 127) // 128), T.exponent, like, "scales")
    return q, scales, q.stride(0) if rows > 1 else width, scales.stride(0) if rows > 1 else scales.shape[1]


def scaled_rows(x, dtype=None, out=None):
    """Rows x [rows, width] (bf16 or fp16) as 8-bit blocks for `scaled_mm`: (q [rows, width] of dtype, float8_e4m3fn by default, scales
    [rows, ceil(width / 128)]).  The header has the form."""
    T, dev = _torch(), x.get_device()
    if x.requires_grad and T.recording():
        _recorded("ew_scaled_rows")
    if T.forward._current_level >= 0:
        _without_tangents("ew_scaled_rows", x)
    code = _code(T, x.dtype)
    if dtype is None:
        dtype = T.e4m3
    to = _eight(T, dtype, "scaled_rows")
    rows, width, ldx = _matrix(x, dev, x.dtype, "x", None)
    q, scales, ldq, lds = _row_blocks(out, rows, width, dtype, T, x)
    rc = lib().ew_scaled_rows(dev, code, to, x.data_ptr(), ldx, rows, width, q.data_ptr(), ldq, scales.data_ptr(), lds, T.stream(dev))
    if rc:
        _check(rc, "ew_scaled_rows")
    return q, scales


def scaled_pack(w, out=None):
    """8-bit weights for `scaled_mm` from w [slots, n, k] (bf16 or fp16): (q float8_e4m3fn [slots, n, k], scales [slots, ceil(n / 128),
    ceil(k / 128)]).  Not differentiable: w may be a parameter, the result is data."""
    T, dev, dtype = _torch(), w.get_device(), w.dtype
    code = _code(T, dtype)
    slots, n, k, ld, stride = _matrices(w, dev, dtype, "w", None)
    shape = (slots, (n + 127) // 128, (k + 127) // 128)
    if out is None:
        wide = _room(k, 16)
        q, scales = w.new_empty((slots, n, wide), dtype=T.e4m3), w.new_empty(shape, dtype=T.exponent)
        q = q if wide == k else q[:, :, :k]
    else:
        q, scales = _result(out[0], (slots, n, k), T.e4m3, w, "q"), _result(out[1], shape, T.exponent, w, "scales")
        if not scales.is_contiguous():
            raise ValueError("scales of weights are contiguous")
    ldq = q.stride(1) if n > 1 else k
    rc = lib().ew_scaled_pack(dev, code, w.data_ptr(), ld, stride, slots, n, k, q.data_ptr(), ldq, q.stride(0) if slots > 1 else n * ldq, scales.data_ptr(),
                              T.stream(dev))
    if rc:
        _check(rc, "ew_scaled_pack")
    return q, scales


def _scaled_product(where, a, a_scales, w, w_scales, offsets, out, out_dtype, grad):
    T, dev = _torch(), a.get_device()
    if (a.requires_grad or w.requires_grad) and T.recording():
        _recorded(where)
    if T.forward._current_level >= 0:
        _without_tangents(where, a, w)
    row_type = _eight(T, a.dtype, "the rows' operand")
    rows, width, lda = _matrix(a, dev, a.dtype, "the rows' operand", None)
    groups, n, k, ldw, stride = _matrices(w, dev, T.e4m3, "w", a)
    if width != (n if grad else k):
        raise ValueError(f"rows of {width} do not match w of {tuple(w.shape)}")
    blocks, nb, kb = (width + 127) // 128, (n + 127) // 128, (k + 127) // 128
    if a_scales.get_device() != dev or a_scales.dtype is not T.exponent:
        _on(a_scales, a, 2, "the rows' scales", T.exponent)
    if w_scales.get_device() != dev or w_scales.dtype is not T.exponent:
        _on(w_scales, a, 3, "w's scales", T.exponent)
    if a_scales.shape != (rows, blocks) or (blocks > 1 and rows and a_scales.stride(1) != 1):
        raise ValueError(f"the rows' scales: ({rows}, {blocks}), a row's side by side, are wanted, got {tuple(a_scales.shape)}")
    if w_scales.shape != (groups, nb, kb) or not w_scales.is_contiguous():
        raise ValueError(f"w's scales: contiguous ({groups}, {nb}, {kb}) are wanted, got {tuple(w_scales.shape)}")
    offsets_at = None
    if offsets is not None:
        if _offsets(offsets, dev, T, a) != groups:
            raise ValueError(f"offsets has {offsets.shape[0]} entries for {groups} groups")
        offsets_at = offsets.data_ptr()
    elif groups != 1:
        raise ValueError(f"without offsets there is one matrix, got {groups}")
    # a row, a matrix alone has no stride of its own
    if rows > 1:
        lds = a_scales.stride(0)
    else:
        lda, lds = (width + 15) // 16 * 16, (blocks + 3) // 4 * 4
    if n == 1:
        ldw = (k + 15) // 16 * 16
    if groups == 1:
        stride = n * ldw
    wide = k if grad else n
    if out_dtype is None:
        out_dtype = T.bfloat16 if out is None else out.dtype
    code = _code(T, out_dtype)
    if out is None:
        out, ldo = T.empty((rows, wide), (wide, 1), dtype=out_dtype, device=a.device), wide
    else:
        _result(out, (rows, wide), out_dtype, a)
        ldo = out.stride(0) if rows > 1 else wide
    fn = lib().ew_scaled_mm_dx if grad else lib().ew_scaled_mm
    rc = fn(dev, row_type, code, a.data_ptr(), lda, a_scales.data_ptr(), lds, w.data_ptr(), ldw, stride, w_scales.data_ptr(), offsets_at, rows, groups, n, k,
            out.data_ptr(), ldo, T.stream(dev))
    if rc:
        _check(rc, where)
    return out


def scaled_mm(x, x_scales, w, w_scales, offsets=None, out=None, out_dtype=None):
    """y[r] = x[r] w[g]^T of the values that 8-bit blocks stand for, for the rows offsets[g] <= r < offsets[g+1] of each group: x, x_scales
    from `scaled_rows`, `rms_norm_scaled` or `swiglu_scaled`, w, w_scales from `scaled_pack`.  offsets None: one matrix, all
    rows.  out_dtype: bfloat16 (default), float16 or float32.  Rows outside the offsets as in `grouped_mm`."""
    return _scaled_product("ew_scaled_mm", x, x_scales, w, w_scales, offsets, out, out_dtype, False)


def scaled_mm_dx(dy, dy_scales, w, w_scales, offsets=None, out=None, out_dtype=None):
    """The gradient of `scaled_mm` with respect to x's values: dx[r] = dy[r] w[g]; dy, dy_scales [rows, n] from `scaled_rows`, often in
    float8_e5m2.  (The weights' gradient: `grouped_mm_dw` of the 16-bit rows.)"""
    return _scaled_product("ew_scaled_mm_dx", dy, dy_scales, w, w_scales, offsets, out, out_dtype, True)


def swiglu_scaled(h, row_weights=None, out=None):
    """`swiglu` with its result as 8-bit blocks of rows: (q float8_e4m3fn [rows, inter], scales [rows, ceil(inter / 128)])."""
    T, dev, dtype = _torch(), h.get_device(), h.dtype
    if (h.requires_grad or (row_weights is not None and row_weights.requires_grad)) and T.recording():
        _recorded("ew_swiglu_scaled")
    if T.forward._current_level >= 0:
        _without_tangents("ew_swiglu_scaled", h, row_weights)
    code = _code(T, dtype)
    rows, two, ldh = _matrix(h, dev, dtype, "h", None)
    if two < 2 or two % 2:
        raise ValueError(f"h holds a gate and an up block side by side: an even width is wanted, got {two}")
    p = _row_weights(row_weights, dev, T, rows, h)
    q, scales, ldq, lds = _row_blocks(out, rows, two // 2, T.e4m3, T, h)
    rc = lib().ew_swiglu_scaled(dev, code, h.data_ptr(), ldh if rows > 1 else two, p, rows, two // 2, q.data_ptr(), ldq, scales.data_ptr(), lds, T.stream(dev))
    if rc:
        _check(rc, "ew_swiglu_scaled")
    return q, scales


def _norm_operands(x, weight, T, dev):
    dtype = x.dtype
    code = T.codes.get(dtype)
    if code is None:
        _code(T, dtype)
    rows, width, ldx = _matrix(x, dev, dtype, "x", None)
    if weight.get_device() != dev or weight.dtype is not dtype or weight.shape != (width,) or not weight.is_contiguous():
        _on(weight, x, 1, "weight", dtype)
        raise ValueError(f"weight: a contiguous tensor of {width} is wanted, got {tuple(weight.shape)}")
    return code, rows, width, ldx


def _beside(t, rows, width, name, like, dev):
    """(address, elements between rows) of an operand that has x's shape and type."""
    t_rows, t_width, ld = _matrix(t, dev, like.dtype, name, like)
    if t_rows != rows or t_width != width:
        raise ValueError(f"{name}: {(rows, width)} is wanted, got {tuple(t.shape)}")
    return t.data_ptr(), ld


def _like(out, rows, width, name, like):
    """(tensor, elements between rows) of a result that has x's shape and type."""
    if out is None:
        return _Torch.empty_like(like), width
    _result(out, (rows, width), like.dtype, like, name)
    return out, out.stride(0) if rows > 1 else width


def _norm(x, weight, residual, eps, y, with_y, blocks, with_blocks, total):
    T, dev = _torch(), x.get_device()
    if (x.requires_grad or weight.requires_grad or (residual is not None and residual.requires_grad)) and T.recording():
        _recorded("ew_rms_norm")
    if T.forward._current_level >= 0:
        _without_tangents("ew_rms_norm", x, weight, residual)
    code, rows, width, ldx = _norm_operands(x, weight, T, dev)
    res = total_at = y_at = q_at = scales_at = None
    ldr = ldt = ldy = ldq = lds = 0
    got = ()
    if with_blocks:
        q, scales, ldq, lds = _row_blocks(blocks, rows, width, T.e4m3, T, x)
        q_at, scales_at, got = q.data_ptr(), scales.data_ptr(), (q, scales)
    if with_y:
        y, ldy = _like(y, rows, width, "out", x)
        y_at, got = y.data_ptr(), got + (y,)
    if residual is not None:
        res, ldr = _beside(residual, rows, width, "residual", x, dev)
        total, ldt = _like(total, rows, width, "sum_out", x)
        total_at, got = total.data_ptr(), got + (total,)
    elif total is not None:
        raise ValueError("sum_out is for the sum with a residual")
    rc = lib().ew_rms_norm(dev, code, x.data_ptr(), ldx, res, ldr, weight.data_ptr(), eps, rows, width, total_at, ldt, y_at, ldy, q_at, ldq, scales_at, lds, T.stream(dev))
    if rc:
        _check(rc, "ew_rms_norm")
    return got[0] if len(got) == 1 else got


def rms_norm(x, weight, residual=None, eps=1e-6, out=None, sum_out=None):
    """t / sqrt(mean(t^2) + eps) * weight of each row, t = x + residual rounded to their type (or x): y, or (y, t) with a residual.
    x, residual [rows, width] and weight [width] bf16 or fp16.  sum_out: where t goes; it may be the residual itself."""
    return _norm(x, weight, residual, eps, out, True, None, False, sum_out)


def rms_norm_scaled(x, weight, residual=None, eps=1e-6, with_y=False, out=None, sum_out=None):
    """`rms_norm` with its result as 8-bit blocks of rows: (q float8_e4m3fn, scales), then y in 16 bits if asked for with_y (for a router,
    say), then t with a residual.  out: (q, scales), or (q, scales, y)."""
    if out is not None and len(out) != (3 if with_y else 2):
        raise ValueError("out: (q, scales), and y if it is wanted")
    return _norm(x, weight, residual, eps, out[2] if out is not None and with_y else None, with_y, None if out is None else out[:2], True, sum_out)


def rms_norm_grad(dy, t, weight, dt=None, eps=1e-6, out=None):
    """The gradient of `rms_norm` (and, for the blocks' values, of `rms_norm_scaled`) from dy and t, the normed stream (x, or its sum with
    the residual): (dt [rows, width], the gradient of x and of the residual each, dweight float32 [width]).  dt: the
    gradient that reaches t past the norm, added in; it may be `out`."""
    T, dev = _torch(), t.get_device()
    if (dy.requires_grad or t.requires_grad or weight.requires_grad or (dt is not None and dt.requires_grad)) and T.recording():
        _recorded("ew_rms_norm_grad")
    if T.forward._current_level >= 0:
        _without_tangents("ew_rms_norm_grad", dy, t, weight, dt)
    code, rows, width, ldt = _norm_operands(t, weight, T, dev)
    dy_at, lddy = _beside(dy, rows, width, "dy", t, dev)
    dt_at, lddt = (None, 0) if dt is None else _beside(dt, rows, width, "dt", t, dev)
    out, ldo = _like(out, rows, width, "out", t)
    fn = lib()
    parts, room, room_at = fn.ew_rms_norm_grad_parts(rows, width), None, None
    dw = T.empty((width,), (1,), dtype=T.float32, device=t.device)
    if parts:
        room = T.empty((parts, width), (width, 1), dtype=T.float32, device=t.device)
        room_at = room.data_ptr()
    rc = fn.ew_rms_norm_grad(dev, code, dy_at, lddy, t.data_ptr(), ldt, weight.data_ptr(), dt_at, lddt, eps, rows, width, out.data_ptr(), ldo, dw.data_ptr(), room_at,
                             T.stream(dev))
    if rc:
        _check(rc, "ew_rms_norm_grad")
    return out, dw


def last_operator_error(device: int = 0) -> int:
    """Read and clear the stand-alone operators' error word of a device (a status code; waits for the device)."""
    code = C.c_int32(0)
    _check(lib().ew_last_operator_error(int(device), C.byref(code)), "ew_last_operator_error")
    return code.value


def load_model(pool: Pool, cfg, bank=None, layers=None, adapters=None, tuned=None):
    """Fill a pool with the seeded synthetic model of `cfg` (a workloads.MoEConfig): base weights of the
    given layers, then the given adapters.  Returns (tuned sets, dict layer -> BaseLayer) for the tests."""
    from . import workloads as wl
    bank = bank or wl.NoiseBank(cfg.seed)
    layers = list(range(cfg.num_layers)) if layers is None else layers
    tuned = wl.tuned_sets(cfg) if tuned is None else tuned
    bases = {}
    for l in layers:
        b = wl.gen_base_layer(cfg, l, bank)
        pool.load_base(l, b.router_w, b.routed.w_gate, b.routed.w_up, b.routed.w_down,
                       b.shared.w_gate, b.shared.w_up, b.shared.w_down)
        bases[l] = b
    adapters = list(range(cfg.max_adapters)) if adapters is None else adapters
    for i in adapters:
        per_layer = [wl.gen_adapter_layer(cfg, i, l, tuned[i][l], bank) for l in range(cfg.num_layers)]
        counts = np.array([len(tuned[i][l]) for l in range(cfg.num_layers)], np.int32)
        ids = np.concatenate([tuned[i][l] for l in range(cfg.num_layers)]).astype(np.int32)
        pool.load_adapter(i, counts, ids, np.concatenate([e.w_gate for e in per_layer]),
                          np.concatenate([e.w_up for e in per_layer]), np.concatenate([e.w_down for e in per_layer]))
    return tuned, bases
