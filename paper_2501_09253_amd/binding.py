"""ctypes binding of the C ABI in include/pserve.h: argument marshalling only.

Every step of the path runs in the HIP kernels of libpserve.so; torch is used for device
memory and streams.  There is no CPU fallback: if the library is missing, loading fails.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from functools import lru_cache
from itertools import chain
from typing import Dict, List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))

F32, BF16 = 0, 1
MSE_STATIC_MAX_PATCHES = 16384      # PSERVE_MSE_STATIC_MAX_PATCHES
STAGE_KIND = {"RES1": 1, "RES2": 2, "SATTN": 3, "XATTN": 4, "FFN": 5, "LSATTN": 6, "LXATTN": 7, "LFFN": 8, "RES2T": 9, "ASATTN": 10, "AMLP": 11, "MMDIT": 12}
TABLES = {"perm": 0, "request_offset": 1, "res_offset": 2, "res_hw": 3, "patch_owner": 4,
          "patch_rc": 5, "neighbour": 6, "halo_src": 7, "cu_seqlens": 8, "seq_len": 9}
SLOT_H1, SLOT_R, SLOT_K, SLOT_V, SLOT_Y = 0, 1, 2, 3, 4
MAX_STAGES, MAX_PARAMS = 8, 24

# parameter order per stage kind (same as the header)
PARAM_ORDER = {
    "RES1": ["gn_g", "gn_b", "conv_w", "conv_b"],
    "RES2": ["gn_a_g", "gn_a_b", "conv_a_w", "conv_a_b", "gn_b_g", "gn_b_b", "conv_b_w", "conv_b_b"],
    "SATTN": ["gn_g", "gn_b", "wq", "wk", "wv", "wo", "bo"],
    "XATTN": ["wq", "wk", "wv", "wo", "bo"],
    "FFN": ["w1", "b1", "w2", "b2"],
    "LSATTN": ["ln_g", "ln_b", "wq", "wk", "wv", "wo", "bo"],
    "LXATTN": ["ln_g", "ln_b", "wq", "wk", "wv", "wo", "bo"],
    "LFFN": ["ln_g", "ln_b", "w1", "b1", "w2", "b2"],
    "MMDIT": [X + "." + n for X in ("img", "txt") for n in ("wm", "bm", "wq", "wk", "wv", "wo", "bo", "w1", "b1", "w2", "b2")],
    "ASATTN": ["wm", "bm", "wq", "wk", "wv", "wo", "bo"],
    "AMLP": ["wm", "bm", "w1", "b1", "w2", "b2"],
    "RES2T": ["gn_a_g", "gn_a_b", "conv_a_w", "conv_a_b", "gn_b_g", "gn_b_b", "conv_b_w", "conv_b_b", "wt", "bt"],
}


class PserveError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"pserve status {status}: {msg}")
        self.status = status


class _PlanInfo(C.Structure):
    _fields_ = [("n", C.c_int32), ("R", C.c_int32), ("P", C.c_int32), ("ph", C.c_int32), ("pw", C.c_int32),
                ("ring", C.c_int32), ("T", C.c_int64), ("text_len", C.c_int32), ("text_patches", C.c_int32)]


class _BlockDesc(C.Structure):
    _fields_ = [("n_stages", C.c_int32), ("stages", C.c_int32 * MAX_STAGES), ("C", C.c_int32), ("G", C.c_int32),
                ("heads", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_float), ("ctx_len", C.c_int32),
                ("ctx_dim", C.c_int32), ("ffn_mult", C.c_int32), ("temb_dim", C.c_int32)]


class _ProfEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("calls", C.c_int32), ("total_ms", C.c_float)]


class _Task(C.Structure):
    _fields_ = [("id", C.c_int64), ("H", C.c_int32), ("W", C.c_int32), ("steps_left", C.c_int32),
                ("arrival", C.c_double), ("ddl", C.c_double), ("standalone", C.c_double)]


class _LatencyModel(C.Structure):
    _fields_ = [("w", C.c_double * 4)]


class _BlockParams(C.Structure):
    _fields_ = [("p", (C.c_void_p * MAX_PARAMS) * MAX_STAGES)]


class _PromptDesc(C.Structure):
    _fields_ = [("n", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("causal", C.c_int32), ("scale", C.c_float), ("max_q", C.c_int32), ("max_k", C.c_int32), ("q_tokens", C.c_int64),
                ("k_tokens", C.c_int64), ("q_stride", C.c_int64 * 2), ("k_stride", C.c_int64 * 2), ("v_stride", C.c_int64 * 2),
                ("o_stride", C.c_int64 * 2)]


def library_path() -> str:
    return os.path.join(_HERE, "libpserve.so")


_lib = None


def lib() -> C.CDLL:
    """Load libpserve.so (built by paper_2501_09253_amd.build); fails loudly if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} not found: build it with `python -m paper_2501_09253_amd.build` "
                          "(there is no CPU fallback)")
    L = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    L.pserve_last_error.restype = C.c_char_p
    L.pserve_last_error.argtypes = []
    L.pserve_plan.argtypes = [C.POINTER(i32), i32, i32, i32, vp, C.POINTER(vp)]
    L.pserve_plan_free.argtypes = [vp]
    L.pserve_plan_free.restype = None
    L.pserve_plan_info.argtypes = [vp, C.POINTER(_PlanInfo)]
    L.pserve_plan_table.argtypes = [vp, C.c_int, C.c_int, C.POINTER(C.POINTER(i32)), C.POINTER(i64)]
    L.pserve_plan_text.argtypes = [C.POINTER(i32), i32, i32, i32, i32, vp, C.POINTER(vp)]
    L.pserve_text_scatter.argtypes = [vp, vp, i32, C.c_int, vp, vp]
    L.pserve_text_gather.argtypes = [vp, vp, i32, C.c_int, vp, vp]
    L.pserve_split.argtypes = [vp, C.POINTER(vp), i32, C.c_int, vp, vp]
    L.pserve_split_stats.argtypes = [vp, C.POINTER(vp), i32, C.c_int, vp, vp, vp]
    L.pserve_reassemble.argtypes = [vp, vp, i32, C.c_int, C.POINTER(vp), vp]
    L.pserve_block_create.argtypes = [C.POINTER(_BlockDesc), C.POINTER(_BlockParams), vp, C.POINTER(vp)]
    L.pserve_block_free.argtypes = [vp]
    L.pserve_block_free.restype = None
    L.pserve_cache_create.argtypes = [vp, vp, C.c_int, C.POINTER(vp)]
    L.pserve_cache_free.argtypes = [vp]
    L.pserve_cache_free.restype = None
    L.pserve_cache_load.argtypes = [vp, C.c_int, C.c_int, vp, vp]
    L.pserve_cache_read.argtypes = [vp, C.c_int, C.c_int, vp, vp]
    L.pserve_block_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    L.pserve_block_forward_temb.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.pserve_set_kernel_mode.argtypes = [C.c_int]
    L.pserve_profile_enable.argtypes = [C.c_int]
    L.pserve_profile_select.argtypes = [C.c_char_p]
    L.pserve_profile_sample.argtypes = [C.c_int]
    L.pserve_patch_mse.argtypes = [vp, vp, vp, i32, C.c_int, vp, vp]
    L.pserve_patch_mse_static.argtypes = [vp, vp, vp, i32, C.c_int, vp, vp]
    L.pserve_probe_mfma_bf16.argtypes = [C.c_int, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_double), vp]
    L.pserve_probe_mfma_mix.argtypes = [C.c_int, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_double), vp]
    L.pserve_probe_copy.argtypes = [vp, vp, C.c_size_t, C.c_int, C.POINTER(C.c_double), vp]
    L.pserve_cache_sets.argtypes = [vp, C.POINTER(C.c_int64), vp, C.POINTER(C.c_int64), C.POINTER(i32),
                                    C.POINTER(C.c_uint8), vp, vp]
    L.pserve_cache_migrate.argtypes = [vp, vp, vp, vp, vp]
    L.pserve_profile_read.argtypes = [C.POINTER(_ProfEntry), i32, C.POINTER(i32)]
    L.pserve_latency_predict.argtypes = [C.POINTER(_LatencyModel), C.POINTER(_Task), i32, i32, i32, C.POINTER(C.c_double)]
    L.pserve_latency_fit.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_double), i32, C.POINTER(_LatencyModel)]
    L.pserve_slack.argtypes = [C.POINTER(_Task), C.c_double, C.c_double, C.POINTER(C.c_double)]
    L.pserve_schedule.argtypes = [C.POINTER(_Task), i32, C.POINTER(_Task), i32, C.c_double, C.POINTER(_LatencyModel), i32, i32,
                                  C.c_double, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
    L.pserve_resample_create.argtypes = [C.c_int, i32, i32, C.c_int, vp, vp, vp, C.POINTER(vp)]
    L.pserve_resample_free.argtypes = [vp]
    L.pserve_resample_free.restype = None
    L.pserve_resample_workspace.argtypes = [vp, vp, C.POINTER(C.c_size_t)]
    L.pserve_resample_forward.argtypes = [vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
    st2 = C.POINTER(i64)
    L.pserve_prompt_attention_workspace.argtypes = [C.POINTER(_PromptDesc), C.POINTER(C.c_size_t)]
    L.pserve_prompt_attention.argtypes = [C.POINTER(_PromptDesc), vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
    L.pserve_kv8_create.argtypes = [i64, i32, i32, vp, C.POINTER(vp)]
    L.pserve_kv8_free.argtypes = [vp]
    L.pserve_kv8_free.restype = None
    L.pserve_kv8_write.argtypes = [vp, vp, vp, C.c_int, st2, st2, vp, i64, vp]
    L.pserve_kv8_read.argtypes = [vp, vp, i64, C.c_int, vp, vp, vp]
    L.pserve_kv8_attention.argtypes = [vp, C.POINTER(_PromptDesc), vp, vp, vp, vp, i32, i32, vp, C.c_size_t, vp, vp]
    L.pserve_linear8_create.argtypes = [i32, i32, C.c_int, vp, vp, vp, C.POINTER(vp)]
    L.pserve_linear8_free.argtypes = [vp]
    L.pserve_linear8_free.restype = None
    L.pserve_linear8_workspace.argtypes = [vp, i64, C.POINTER(C.c_size_t)]
    L.pserve_linear8_forward.argtypes = [vp, vp, i64, i64, vp, vp, C.c_size_t, vp, vp]
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise PserveError(status, lib().pserve_last_error().decode())


def _stream() -> int:
    import torch
    if torch.cuda.is_initialized():         # the handle alone: no Stream object per call (0.4 us against 1.3)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _torch_dtype(dtype: int):
    import torch
    return torch.bfloat16 if dtype == BF16 else torch.float32


def set_kernel_mode(mode: int):
    """0 = fastest kernels for the shapes, 1 = plain reference kernels only."""
    _check(lib().pserve_set_kernel_mode(mode))


def profile_enable(on: bool):
    """Bracket every kernel of pserve_block_forward with HIP events (pserve_profile_enable)."""
    _check(lib().pserve_profile_enable(int(on)))


def profile_select(label: Optional[str]):
    """Time only the kernels with this label; None = all kernels (pserve_profile_select)."""
    _check(lib().pserve_profile_select(None if not label else label.encode()))


def profile_sample(every: int):
    """Bracket the kernels of every n-th forward call only (pserve_profile_sample)."""
    _check(lib().pserve_profile_sample(int(every)))


def probe_mfma_bf16(iters: int = 20000, random_operands: bool = False):
    """pserve_probe_mfma_bf16: (dense bf16 TFLOP/s of a register-resident MFMA stream, shader clock in MHz inside it)."""
    out, mhz = C.c_double(0.0), C.c_double(0.0)
    _check(lib().pserve_probe_mfma_bf16(iters, 1 if random_operands else 0, C.byref(out), C.byref(mhz), _stream()))
    return out.value, mhz.value


def probe_mfma_mix(mix: int, iters: int = 20000):
    """pserve_probe_mfma_mix: (bf16 TFLOP/s of the 32 x 32 x 16 MFMAs, shader clock in MHz) of an MFMA stream on
    standard-normal operands with the instruction mix `mix` between the MFMAs (19: attention inner loop, 8: convolution)."""
    out, mhz = C.c_double(0.0), C.c_double(0.0)
    _check(lib().pserve_probe_mfma_mix(iters, int(mix), C.byref(out), C.byref(mhz), _stream()))
    return out.value, mhz.value


def probe_copy(dst, src, reps: int = 5) -> float:
    """pserve_probe_copy: GB/s (read + written) of a plain copy between two equally sized device tensors."""
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes and src.is_contiguous() and dst.is_contiguous()
    out = C.c_double(0.0)
    _check(lib().pserve_probe_copy(dst.data_ptr(), src.data_ptr(), nbytes, reps, C.byref(out), _stream()))
    return out.value


def profile_read() -> Dict[str, Dict[str, float]]:
    """Collect {kernel label: {"calls": n, "total_ms": t}} since the last read (pserve_profile_read)."""
    buf = (_ProfEntry * 64)()
    n = C.c_int32()
    _check(lib().pserve_profile_read(buf, 64, C.byref(n)))
    return {buf[i].name.decode(): {"calls": int(buf[i].calls), "total_ms": float(buf[i].total_ms)}
            for i in range(n.value)}


class Plan:
    """pserve_plan: Compressed Sparse Patch tables of one batch composition."""

    def __init__(self, resolutions: Sequence[Sequence[int]], ph: int = 0, pw: int = 0, text_len: int = 0):
        res = self._flat(resolutions)
        self._h = C.c_void_p()
        _check(lib().pserve_plan_text((C.c_int32 * len(res)).from_buffer(res), len(res) // 2, ph, pw, text_len, _stream(),
                                      C.byref(self._h)))
        info = _PlanInfo()
        _check(lib().pserve_plan_info(self._h, C.byref(info)))
        self.n, self.R, self.P, self.ph, self.pw, self.ring, self.T = (info.n, info.R, info.P, info.ph, info.pw,
                                                                      info.ring, info.T)
        self.text_len, self.text_patches = info.text_len, info.text_patches
        self.resolutions = list(zip(res[::2], res[1::2]))

    @staticmethod
    def _flat(resolutions) -> array:
        """h0, w0, h1, w1, ... as int32.  Lists of pairs of whole numbers, a batch's usual form, without an ndarray on the way
        (24 requests: 3 us against 5); anything else as numpy converts it, with numpy's errors."""
        if type(resolutions) in (list, tuple) and set(map(type, resolutions)) <= {list, tuple} and set(map(len, resolutions)) == {2}:
            try:
                return array("i", chain.from_iterable(resolutions))
            except (TypeError, OverflowError):
                pass
        return array("i", np.ascontiguousarray(np.asarray(resolutions, dtype=np.int32).reshape(-1, 2)).tobytes())

    def text_scatter(self, text, x):
        """pserve_text_scatter: text [n, text_len, C] (caller order) into the text patches of x[T, C] (in place)."""
        assert text.is_contiguous() and x.is_contiguous() and text.dtype == x.dtype
        assert text.shape == (self.n, self.text_len, x.shape[1]) and x.shape[0] == self.T
        import torch
        dt = BF16 if x.dtype == torch.bfloat16 else F32
        _check(lib().pserve_text_scatter(self._h, text.data_ptr(), x.shape[1], dt, x.data_ptr(), _stream()))
        return x

    def text_gather(self, x):
        """pserve_text_gather: the text tokens of every request out of x[T, C]: [n, text_len, C] in caller order."""
        import torch
        assert x.is_contiguous() and x.shape[0] == self.T
        out = torch.empty((self.n, self.text_len, x.shape[1]), dtype=x.dtype, device=x.device)
        dt = BF16 if x.dtype == torch.bfloat16 else F32
        _check(lib().pserve_text_gather(self._h, x.data_ptr(), x.shape[1], dt, out.data_ptr(), _stream()))
        return out

    def table(self, name: str) -> np.ndarray:
        """Host mirror of a table as a numpy int32 array (copy)."""
        ptr = C.POINTER(C.c_int32)()
        cnt = C.c_int64()
        _check(lib().pserve_plan_table(self._h, TABLES[name], 0, C.byref(ptr), C.byref(cnt)))
        a = np.empty(cnt.value, dtype=np.int32)
        if cnt.value:
            C.memmove(C.byref(C.c_int32.from_buffer(a)), ptr, a.nbytes)
        shape = {"res_hw": (-1, 2), "patch_rc": (-1, 2), "neighbour": (-1, 8), "halo_src": (self.P, -1)}.get(name)
        return a.reshape(shape) if shape else a

    def table_device_ptr(self, name: str) -> int:
        ptr = C.POINTER(C.c_int32)()
        cnt = C.c_int64()
        _check(lib().pserve_plan_table(self._h, TABLES[name], 1, C.byref(ptr), C.byref(cnt)))
        return C.cast(ptr, C.c_void_p).value

    def split(self, images, out=None, cache=None):
        """Per-request NCHW device tensors (caller order) -> patch-major token matrix x[T, C].  With `cache` (a Cache of
        this plan) the pass also leaves the input's GroupNorm moments behind for the cache's next forward call on x
        (pserve_split_stats)."""
        import torch
        Cc = images[0].shape[0]
        dt = BF16 if images[0].dtype == torch.bfloat16 else F32
        if out is None:
            out = torch.empty((self.T, Cc), dtype=images[0].dtype, device=images[0].device)
        ptrs = (C.c_void_p * self.n)(*[im.data_ptr() for im in images])
        for im, (h, w) in zip(images, self.resolutions):
            assert im.is_contiguous() and im.shape == (Cc, h, w) and im.dtype == images[0].dtype
        if cache is not None:
            _check(lib().pserve_split_stats(self._h, ptrs, Cc, dt, out.data_ptr(), cache._h, _stream()))
        else:
            _check(lib().pserve_split(self._h, ptrs, Cc, dt, out.data_ptr(), _stream()))
        return out

    def reassemble(self, y, images=None):
        """Patch-major y[T, C] -> per-request NCHW tensors in caller order."""
        import torch
        Cc = y.shape[1]
        dt = BF16 if y.dtype == torch.bfloat16 else F32
        assert y.is_contiguous() and y.shape[0] == self.T
        if images is None:
            images = [torch.empty((Cc, h, w), dtype=y.dtype, device=y.device) for h, w in self.resolutions]
        ptrs = (C.c_void_p * self.n)(*[im.data_ptr() for im in images])
        _check(lib().pserve_reassemble(self._h, y.data_ptr(), Cc, dt, ptrs, _stream()))
        return images

    def patch_mse(self, a, b):
        """pserve_patch_mse: per-patch mean squared error of two patch batches [T, C] -> float32 [P] (plan order)."""
        import torch
        assert a.shape == b.shape and a.dtype == b.dtype and a.is_contiguous() and b.is_contiguous() and a.shape[0] == self.T
        out = torch.empty(self.P, dtype=torch.float32, device=a.device)
        dt = BF16 if a.dtype == torch.bfloat16 else F32
        _check(lib().pserve_patch_mse(self._h, a.data_ptr(), b.data_ptr(), a.shape[1], dt, out.data_ptr(), _stream()))
        return out

    def patch_mse_static(self, a, b, out=None):
        """pserve_patch_mse_static: the same result through the library's fixed device scratch; allocates nothing when
        `out` (float32 [P]) is given."""
        import torch
        assert a.shape == b.shape and a.dtype == b.dtype and a.is_contiguous() and b.is_contiguous() and a.shape[0] == self.T
        if out is None:
            out = torch.empty(self.P, dtype=torch.float32, device=a.device)
        dt = BF16 if a.dtype == torch.bfloat16 else F32
        _check(lib().pserve_patch_mse_static(self._h, a.data_ptr(), b.data_ptr(), a.shape[1], dt, out.data_ptr(), _stream()))
        return out

    def cache_sets(self, ids, old_plan: "Plan", old_ids):
        """pserve_cache_sets with this plan as the new batch: returns (req_src, expired, patch_src device tensor)."""
        import torch
        new_ids = np.ascontiguousarray(np.asarray(ids, dtype=np.int64))
        prev_ids = np.ascontiguousarray(np.asarray(old_ids, dtype=np.int64))
        assert new_ids.shape == (self.n,) and prev_ids.shape == (old_plan.n,)
        req_src = np.empty(self.n, dtype=np.int32)
        expired = np.empty(old_plan.n, dtype=np.uint8)
        patch_src = torch.empty(self.P, dtype=torch.int32, device="cuda")
        _check(lib().pserve_cache_sets(old_plan._h, prev_ids.ctypes.data_as(C.POINTER(C.c_int64)), self._h,
                                       new_ids.ctypes.data_as(C.POINTER(C.c_int64)),
                                       req_src.ctypes.data_as(C.POINTER(C.c_int32)),
                                       expired.ctypes.data_as(C.POINTER(C.c_uint8)), patch_src.data_ptr(), _stream()))
        return req_src, expired, patch_src

    def close(self):
        if self._h:
            lib().pserve_plan_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Block:
    """pserve_block: block description + packed weights (params: per stage dict name -> device tensor)."""

    def __init__(self, stages: Sequence[str], params: List[Dict[str, "object"]], *, C_: int, G: int, heads: int,
                 dtype: int, eps: float = 1e-5, ctx_len: int = 0, ctx_dim: int = 0, ffn_mult: int = 4, temb_dim: int = 0):
        desc = _BlockDesc()
        desc.n_stages = len(stages)
        for i, s in enumerate(stages):
            desc.stages[i] = STAGE_KIND[s]
        desc.C, desc.G, desc.heads, desc.dtype, desc.eps = C_, G, heads, dtype, eps
        desc.ctx_len, desc.ctx_dim, desc.ffn_mult, desc.temb_dim = ctx_len, ctx_dim, ffn_mult, temb_dim
        bp = _BlockParams()
        keep = []
        for i, (s, p) in enumerate(zip(stages, params)):
            for k, name in enumerate(PARAM_ORDER[s]):
                t = p[name]
                assert t.is_contiguous() and t.dtype == _torch_dtype(dtype), (s, name, t.dtype)
                keep.append(t)
                bp.p[i][k] = t.data_ptr()
        self._h = C.c_void_p()
        _check(lib().pserve_block_create(C.byref(desc), C.byref(bp), _stream(), C.byref(self._h)))
        self.stages, self.C, self.dtype = tuple(stages), C_, dtype

    def close(self):
        if self._h:
            lib().pserve_block_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Cache:
    """pserve_cache: cached operand tensors + scratch of one (plan, block) pair."""

    def __init__(self, plan: Plan, block: Block, with_slots: bool = False):
        self._h = C.c_void_p()
        _check(lib().pserve_cache_create(plan._h, block._h, int(with_slots), C.byref(self._h)))
        self.plan, self.block = plan, block

    def load(self, stage: int, slot: int, src):
        assert src.is_contiguous() and src.shape == (self.plan.T, self.block.C)
        _check(lib().pserve_cache_load(self._h, stage, slot, src.data_ptr(), _stream()))

    def read(self, stage: int, slot: int):
        import torch
        dst = torch.empty((self.plan.T, self.block.C), dtype=_torch_dtype(self.block.dtype), device="cuda")
        _check(lib().pserve_cache_read(self._h, stage, slot, dst.data_ptr(), _stream()))
        return dst

    def migrate_from(self, old_cache: "Cache", patch_src):
        """pserve_cache_migrate: take the Common Set's slots from the cache of the previous batch; returns valid[P]."""
        import torch
        assert patch_src.dtype == torch.int32 and patch_src.numel() == self.plan.P and patch_src.is_contiguous()
        valid = torch.empty(self.plan.P, dtype=torch.uint8, device="cuda")
        _check(lib().pserve_cache_migrate(old_cache._h, self._h, patch_src.data_ptr(), valid.data_ptr(), _stream()))
        return valid

    def forward(self, x, ctx=None, reuse_mask=None, y=None, temb=None):
        """pserve_block_forward (pserve_block_forward_temb when temb is given) on the current torch stream; returns y[T, C]."""
        import torch
        assert x.is_contiguous() and x.shape == (self.plan.T, self.block.C)
        assert x.dtype == _torch_dtype(self.block.dtype)
        if y is None:
            y = torch.empty_like(x)
        if ctx is not None:
            assert ctx.is_contiguous() and ctx.dtype == x.dtype
        if reuse_mask is not None:
            assert reuse_mask.dtype == torch.uint8 and reuse_mask.numel() == self.plan.P and reuse_mask.is_contiguous()
        mask_p = reuse_mask.data_ptr() if reuse_mask is not None else None
        ctx_p = ctx.data_ptr() if ctx is not None else None
        if temb is not None:
            assert temb.is_contiguous() and temb.dtype == x.dtype
            _check(lib().pserve_block_forward_temb(self.plan._h, x.data_ptr(), ctx_p, temb.data_ptr(), self.block._h,
                                                   self._h, mask_p, y.data_ptr(), _stream()))
        else:
            _check(lib().pserve_block_forward(self.plan._h, x.data_ptr(), ctx_p, self.block._h, self._h, mask_p,
                                              y.data_ptr(), _stream()))
        return y

    def close(self):
        if self._h:
            lib().pserve_cache_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


DOWN2, UP2 = 1, 2


class Resample:
    """pserve_resample: stride-2 (DOWN2) or nearest-up (UP2) 3x3 convolution between two plans with the same patch grid."""

    def __init__(self, kind: int, w, b, dtype: int):
        assert w.is_contiguous() and b.is_contiguous() and w.dtype == _torch_dtype(dtype) and b.dtype == w.dtype
        self.kind, self.dtype, self.C_out, self.C_in = kind, dtype, int(w.shape[0]), int(w.shape[1])
        self._h = C.c_void_p()
        _check(lib().pserve_resample_create(kind, self.C_in, self.C_out, dtype, w.data_ptr(), b.data_ptr(), _stream(),
                                            C.byref(self._h)))
        self._ws = None

    def workspace_bytes(self, plan_in: "Plan") -> int:
        n = C.c_size_t()
        _check(lib().pserve_resample_workspace(self._h, plan_in._h, C.byref(n)))
        return int(n.value)

    def forward(self, plan_in: "Plan", plan_out: "Plan", x, y=None, workspace=None):
        import torch
        assert x.is_contiguous() and x.shape == (plan_in.T, self.C_in) and x.dtype == _torch_dtype(self.dtype)
        if workspace is None:
            need = self.workspace_bytes(plan_in)
            if self._ws is None or self._ws.numel() < need:
                self._ws = torch.empty(need, dtype=torch.uint8, device=x.device)
            workspace = self._ws
        if y is None:
            y = torch.empty((plan_out.T, self.C_out), dtype=x.dtype, device=x.device)
        _check(lib().pserve_resample_forward(self._h, plan_in._h, plan_out._h, x.data_ptr(), workspace.data_ptr(),
                                             workspace.numel() * workspace.element_size(), y.data_ptr(), _stream()))
        return y

    def close(self):
        if self._h:
            lib().pserve_resample_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- the prompt side: causal attention over packed prompts, the 8-bit key/value store, 8-bit linear layers
EINVAL = -1


def _need(cond, msg: str):
    """Argument checks of the calls below: PserveError as for those the library refuses itself."""
    if not cond:
        raise PserveError(EINVAL, msg)


def _whole(who: str, name: str, x, least: int = 0, most: int = 2 ** 31 - 1) -> int:
    """A number that the library takes in 32 bits (or `most`): ctypes would pass on the low half of a larger one."""
    x = int(x)
    if not least <= x <= most:
        raise PserveError(EINVAL, f"{who}: {name} {x}")
    return x


def _here(who: str, *tensors):
    """Tensors (None: absent) on the current device: the library's kernels run there."""
    import torch
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:         # -1: not on a GPU
            raise PserveError(EINVAL, f"{who}: a tensor on {t.device}, the current device is cuda:{dev}")


def _ints(who: str, t, dtype, shape, name: str):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise PserveError(EINVAL, f"{who}: {name} must be contiguous {dtype} {tuple(shape)}")


def _workspace(need: int, workspace, device, who: str):
    """The caller's workspace, or one from torch's allocator for this call: (pointer, bytes, what keeps it alive)."""
    import torch
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        return workspace.data_ptr(), need, workspace
    _need(workspace.is_contiguous(), f"{who}: the workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _apart(who: str, out, *inputs):
    """`out` shares no byte with an input (dense or strided: the extents are compared)."""
    def extent(t):
        last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
        return t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()
    if out.numel() == 0:
        return
    o0, o1 = extent(out)
    for t in inputs:
        if t is not None and t.numel():
            a0, a1 = extent(t)
            _need(a1 <= o0 or o1 <= a0, f"{who}: the output overlaps an input")


def _number(scale):
    """The value of a scale that may be an array of one: the descriptors below are kept by value."""
    return None if scale is None else float(scale)


@lru_cache(maxsize=1024)
def _prompt_desc(n: int, heads: int, kv_heads: int, dim: int, dtype: int, causal: bool, scale: Optional[float], max_q: int, max_k: int,
                 q_tokens: int, k_tokens: int, q_stride, k_stride, v_stride, o_stride):
    """(pserve_prompt_desc, bytes of workspace) of these sizes: decoding steps ask for the same one again and again (7 us each)."""
    d = _PromptDesc()
    d.n, d.heads, d.kv_heads, d.head_dim, d.dtype = n, heads, kv_heads, dim, dtype
    d.causal, d.scale = int(causal), (dim ** -0.5 if scale is None else scale)
    d.max_q, d.max_k, d.q_tokens, d.k_tokens = max_q, max_k, q_tokens, k_tokens
    d.q_stride[:], d.k_stride[:], d.v_stride[:], d.o_stride[:] = q_stride[:2], k_stride[:2], v_stride[:2], o_stride[:2]
    need = C.c_size_t()
    _check(lib().pserve_prompt_attention_workspace(C.byref(d), C.byref(need)))
    return C.byref(d), need.value


def _prompt_out(who: str, q, out, *inputs):
    """The output tensor: the caller's, checked, or a new one."""
    import torch
    if q.dtype != torch.bfloat16 and q.dtype != torch.float32:
        raise PserveError(EINVAL, f"{who}: dtype {q.dtype} is neither bfloat16 nor float32")
    if q.stride(2) != 1:
        raise PserveError(EINVAL, f"{who}: the values of a head must be consecutive")
    if out is None:
        return torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _need(out.shape == q.shape and out.dtype == q.dtype, f"{who}: out must have q's shape and dtype")
    _need(out.stride(2) == 1, f"{who}: the values of a head must be consecutive")
    (T, H, D), (st, sh, _) = out.shape, out.stride()        # heads inside tokens or tokens inside heads
    _need(out.numel() == 0 or (H == 1 or sh >= D) and (T == 1 or st >= (H - 1) * (sh if H > 1 else 0) + D)
          or (T == 1 or st >= D) and (H == 1 or sh >= (T - 1) * (st if T > 1 else 0) + D), f"{who}: rows of out overlap")
    _apart(who, out, q, *inputs)
    return out


def prompt_attention(q, k, v, cu_q, cu_k=None, causal: bool = True, scale: Optional[float] = None, max_q: int = 0, max_k: int = 0,
                     out=None, workspace=None):
    """pserve_prompt_attention: q [Tq, heads, D], k and v [Tk, kv_heads, D] (any strides between tokens and heads that are
    multiples of 16 bytes), cu_q and cu_k int32 [n + 1] on the device (cu_k = None: those of the queries); scale defaults to
    1 / sqrt(D).  Rows of no sequence are not written.  `out` must lie apart from q, k and v, from its first to its last
    byte.  Returns out [Tq, heads, D]."""
    import torch
    who = "prompt_attention"
    cu_k = cu_q if cu_k is None else cu_k
    _here(who, q, k, v, cu_q, cu_k, out, workspace)
    _need(cu_q.dim() == 1 and cu_q.shape[0] >= 2, f"{who}: cu_q must be int32 [n + 1], n > 0")
    _ints(who, cu_q, torch.int32, cu_q.shape, "cu_q")
    _ints(who, cu_k, torch.int32, cu_q.shape, "cu_k")
    if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape or k.shape[2] != q.shape[2] or 0 in q.shape[1:] or 0 in k.shape[1:]:
        raise PserveError(EINVAL, f"{who}: q [Tq, heads, D], k and v [Tk, kv_heads, D]")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise PserveError(EINVAL, f"{who}: q, k and v must have one dtype")
    sk, sv = k.stride(), v.stride()
    if sk[2] != 1 or sv[2] != 1:
        raise PserveError(EINVAL, f"{who}: the values of a head must be consecutive")
    out = _prompt_out(who, q, out, k, v)
    d, need = _prompt_desc(cu_q.shape[0] - 1, q.shape[1], k.shape[1], q.shape[2], BF16 if q.dtype == torch.bfloat16 else F32, bool(causal), _number(scale),
                           _whole(who, "max_q", max_q), _whole(who, "max_k", max_k), q.shape[0], k.shape[0], q.stride(), sk, sv, out.stride())
    ws, nws, keep = _workspace(need, workspace, q.device, who)
    _check(lib().pserve_prompt_attention(d, q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(),
                                         ws, nws, out.data_ptr(), _stream()))
    return out


@lru_cache(maxsize=1024)
def _strides(token: int, head: int):
    return (C.c_int64 * 2)(token, head)


class KV8:
    """pserve_kv8: keys and values of `places` tokens in 8 bits, a scale for each token and head."""

    def __init__(self, places: int, kv_heads: int, head_dim: int):
        self._h, who = C.c_void_p(), "KV8"
        self.places, self.kv_heads, self.head_dim = (_whole(who, name, x, 1) for name, x in (("places", places), ("kv_heads", kv_heads), ("head_dim", head_dim)))
        _check(lib().pserve_kv8_create(self.places, self.kv_heads, self.head_dim, _stream(), C.byref(self._h)))

    def write(self, k, v, places):
        """k and v [T, kv_heads, D] into places int64 [T] (on the device; negative or out of range: not written; the last row
        of a place counts)."""
        import torch
        who = "KV8.write"
        _here(who, k, v, places)
        if k.dim() != 3 or k.shape[1] != self.kv_heads or k.shape[2] != self.head_dim or v.shape != k.shape or v.dtype != k.dtype or \
                (k.dtype != torch.bfloat16 and k.dtype != torch.float32):
            raise PserveError(EINVAL, f"{who}: k and v must be [T, {self.kv_heads}, {self.head_dim}], both bfloat16 or both float32")
        sk, sv = k.stride(), v.stride()
        if sk[2] != 1 or sv[2] != 1:
            raise PserveError(EINVAL, f"{who}: the values of a head must be consecutive")
        _ints(who, places, torch.int64, k.shape[:1], "places")
        _check(lib().pserve_kv8_write(self._h, k.data_ptr(), v.data_ptr(), BF16 if k.dtype == torch.bfloat16 else F32, _strides(sk[0], sk[1]),
                                      _strides(sv[0], sv[1]), places.data_ptr(), k.shape[0], _stream()))

    def read(self, places, dtype: int, k=None, v=None):
        """The values held at places int64 [T], as (k, v) [T, kv_heads, D] of dtype F32 or BF16; zeros where out of range."""
        import torch
        who = "KV8.read"
        _here(who, places, k, v)
        _need(dtype in (F32, BF16), f"{who}: unknown dtype {dtype}")
        _need(places.dim() == 1, f"{who}: places must be int64 [T]")
        _ints(who, places, torch.int64, places.shape, "places")
        shape = (places.shape[0], self.kv_heads, self.head_dim)
        given = [t for t in (k, v) if t is not None]
        for t in given:
            _need(t.shape == shape and t.is_contiguous() and t.dtype == _torch_dtype(dtype), f"{who}: k and v must be contiguous {shape} of dtype")
        k = torch.empty(shape, dtype=_torch_dtype(dtype), device=places.device) if k is None else k
        v = torch.empty(shape, dtype=_torch_dtype(dtype), device=places.device) if v is None else v
        if given:
            _apart(who, k, v, places)
            _apart(who, v, places)
        _check(lib().pserve_kv8_read(self._h, places.data_ptr(), places.shape[0], dtype, k.data_ptr(), v.data_ptr(), _stream()))
        return k, v

    def attention(self, q, cu_q, key_len, table, page: int, causal: bool = True, scale: Optional[float] = None, max_q: int = 0,
                  max_k: int = 0, out=None, workspace=None):
        """pserve_kv8_attention: q [Tq, heads, D], cu_q int32 [n + 1], key_len int32 [n], table int32 [n, max_pages]: key j of
        sequence s lies at place table[s, j // page] * page + j % page.  As prompt_attention otherwise."""
        import torch
        who = "KV8.attention"
        _here(who, q, cu_q, key_len, table, out, workspace)
        _need(cu_q.dim() == 1 and cu_q.shape[0] >= 2, f"{who}: cu_q must be int32 [n + 1], n > 0")
        n = cu_q.shape[0] - 1
        _ints(who, cu_q, torch.int32, cu_q.shape, "cu_q")
        _ints(who, key_len, torch.int32, (n,), "key_len")
        _need(table.dim() == 2, f"{who}: table must be int32 [n, max_pages]")
        _ints(who, table, torch.int32, (n, table.shape[1]), "table")
        page = _whole(who, "page", page, 1)
        _need(q.dim() == 3 and q.shape[1] > 0 and q.shape[2] == self.head_dim, f"{who}: q must be [Tq, heads, {self.head_dim}]")
        out = _prompt_out(who, q, out)
        d, need = _prompt_desc(n, q.shape[1], self.kv_heads, self.head_dim, BF16 if q.dtype == torch.bfloat16 else F32, bool(causal), _number(scale),
                               _whole(who, "max_q", max_q), _whole(who, "max_k", max_k), q.shape[0], 0, q.stride(), (0, 0), (0, 0), out.stride())
        ws, nws, keep = _workspace(need, workspace, q.device, who)
        _check(lib().pserve_kv8_attention(self._h, d, q.data_ptr(), cu_q.data_ptr(), key_len.data_ptr(), table.data_ptr(),
                                          table.shape[1], page, ws, nws, out.data_ptr(), _stream()))
        return out

    def close(self):
        if self._h:
            lib().pserve_kv8_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Linear8:
    """pserve_linear8: y = x W + b (+ residual), x and W in 8-bit integers with a scale for each token and output channel.
    w [K, N], b [N] or None; the weights are quantised here, once."""

    def __init__(self, w, b, dtype: int):
        who = "Linear8"
        _here(who, w, b)
        _need(dtype in (F32, BF16) and w.dim() == 2 and w.is_contiguous() and w.dtype == _torch_dtype(dtype), f"{who}: w must be contiguous [K, N] of the given dtype")
        _need(b is None or (tuple(b.shape) == (w.shape[1],) and b.is_contiguous() and b.dtype == w.dtype), f"{who}: b must be [N] of the given dtype")
        self.dtype, self.K, self.N = dtype, int(w.shape[0]), int(w.shape[1])
        self._h = C.c_void_p()
        _check(lib().pserve_linear8_create(self.K, self.N, dtype, w.data_ptr(), None if b is None else b.data_ptr(), _stream(), C.byref(self._h)))
        self._dtype, self._row_bytes = w.dtype, self.workspace_bytes(1)         # (workspace_bytes is linear in the rows)

    def workspace_bytes(self, rows: int) -> int:
        n = C.c_size_t()
        _check(lib().pserve_linear8_workspace(self._h, rows, C.byref(n)))
        return int(n.value)

    def forward(self, x, res=None, y=None, workspace=None):
        """x [rows, K] (rows may lie further apart), res [rows, N] or None (it may be y)."""
        import torch
        who = "Linear8.forward"
        _here(who, x, res, y, workspace)
        if x.dim() != 2 or x.shape[1] != self.K or x.dtype != self._dtype:
            raise PserveError(EINVAL, f"{who}: x must be [rows, {self.K}] of the layer's dtype")
        rows = x.shape[0]
        ldx, one = x.stride()
        if rows <= 1:
            ldx = self.K
        if (one != 1 and self.K > 1) or ldx < self.K:
            raise PserveError(EINVAL, f"{who}: the values of a row must be consecutive, rows must not overlap")
        for t in (y, res):
            if t is not None and (t.shape != (rows, self.N) or not t.is_contiguous() or t.dtype != x.dtype):
                raise PserveError(EINVAL, f"{who}: res and y must be contiguous [rows, {self.N}] of the layer's dtype")
        if y is None:
            y = torch.empty((rows, self.N), dtype=x.dtype, device=x.device)
        else:
            _apart(who, y, x, *([res] if res is not None and res.data_ptr() != y.data_ptr() else []))
        ws, nws, keep = _workspace(rows * self._row_bytes, workspace, x.device, who)
        _check(lib().pserve_linear8_forward(self._h, x.data_ptr(), ldx, rows, None if res is None else res.data_ptr(), ws, nws, y.data_ptr(), _stream()))
        return y

    def close(self):
        if self._h:
            lib().pserve_linear8_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- host-side scheduler pieces (tasks are tuples (id, H, W, steps_left, arrival, ddl, standalone), times in ms)
def _tasks(ts):
    arr = (_Task * max(1, len(ts)))()
    for i, t in enumerate(ts):
        arr[i] = _Task(*t)
    return arr


def _model(w):
    m = _LatencyModel()
    for i in range(4):
        m.w[i] = float(w[i])
    return m


def latency_predict(w, batch, ph, pw) -> float:
    out = C.c_double()
    _check(lib().pserve_latency_predict(C.byref(_model(w)), _tasks(batch), len(batch), ph, pw, C.byref(out)))
    return out.value


def latency_fit(X, y):
    import numpy as np
    X = np.ascontiguousarray(X, dtype=np.float64)
    y = np.ascontiguousarray(y, dtype=np.float64)
    m = _LatencyModel()
    _check(lib().pserve_latency_fit(X.ctypes.data_as(C.POINTER(C.c_double)), y.ctypes.data_as(C.POINTER(C.c_double)),
                                    X.shape[0], C.byref(m)))
    return [m.w[i] for i in range(4)]


def slack(task, now, latency) -> float:
    out = C.c_double()
    _check(lib().pserve_slack(_tasks([task]), now, latency, C.byref(out)))
    return out.value


def schedule(wait, active, now, w, ph, pw, relaxed_slack):
    """pserve_schedule: returns (admitted, discarded), indices into `wait` in the order decided."""
    n = len(wait)
    adm, dis = (C.c_int32 * max(1, n))(), (C.c_int32 * max(1, n))()
    na, nd = C.c_int32(), C.c_int32()
    _check(lib().pserve_schedule(_tasks(wait), n, _tasks(active), len(active), now, C.byref(_model(w)), ph, pw,
                                 relaxed_slack, adm, C.byref(na), dis, C.byref(nd)))
    return list(adm[:na.value]), list(dis[:nd.value])
