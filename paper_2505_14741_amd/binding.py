"""ctypes binding of the HIP C-ABI library: argument marshalling only.

Every function has the name of the C entry point it calls.  PyTorch supplies device
memory (tensors) and the stream; all arithmetic runs in the library's kernels.  The
library must have been built (`python -m paper_2505_14741_amd.build` or
`__graft_entry__.build()`); if it is missing this module raises at import of the
library handle -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import List, Optional, Sequence

import numpy as np
import torch

from .inputs import DiTConfig

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libparastep_hip.so")
_lib = None

PS_F32, PS_BF16 = 0, 1
KERNEL_CLASSES = ("attention", "gemm_qkv", "gemm_oproj", "gemm_fc1", "gemm_fc2", "ln_modulate", "other")


PS_ERR_SHAPE, PS_ERR_DTYPE = -2, -3


class PsError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().ps_strerror(status).decode()} (status {status})")


class _DitConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("layers", "hidden", "heads", "head_dim", "mlp_ratio", "in_channels",
                                       "patch", "frames", "height", "width", "text_tokens",
                                       "time_embed_dim", "dtype")] + [("ln_eps", C.c_float), ("rope_theta", C.c_float)]


class _Schedule(C.Structure):
    _fields_ = [("steps", C.c_int), ("timesteps", C.POINTER(C.c_int32)), ("coef_a", C.POINTER(C.c_double)),
                ("coef_b", C.POINTER(C.c_double)), ("warmup", C.c_int), ("n_cycles", C.c_int),
                ("cycle_len", C.POINTER(C.c_int32)), ("batched", C.c_int), ("mode", C.c_int)]


class _CrossShape(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("batch", "q_len", "kv_len", "heads", "kv_heads", "head_dim", "dtype")] + [("scale", C.c_float)] + [
        (f"{t}_{n}", C.c_int64) for t in "qkvo" for n in ("batch", "token", "head")] + [("mask_batch", C.c_int64)]


class _GroupNormShape(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("batch", "positions", "channels", "groups", "act", "dtype")] + [("eps", C.c_float)] + [
        (n, C.c_int64) for n in ("x_batch", "x_position", "out_batch", "out_position")]


class _QkNormShape(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("batch", "tokens", "heads", "kv_heads", "head_dim", "rotated", "norm", "halves", "dtype")] + [("eps", C.c_float)] + [
        (f"{t}_{n}", C.c_int64) for t in ("q", "k", "q_out", "k_out") for n in ("batch", "token", "head")] + [("table_batch", C.c_int64)]


class _PackedShape(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("samples", "q_tokens", "kv_tokens", "heads", "kv_heads", "head_dim", "dtype", "own_offsets", "causal", "frame")] + [
        ("scale", C.c_float), ("cap", C.c_float)] + [(f"{t}_{n}", C.c_int64) for t in "qkvo" for n in ("token", "head")]


class SamplerState(C.Structure):
    """Host part of a run's state between two steps (`sampler_state`); plain data, may be stored."""
    _fields_ = [("step", C.c_int32), ("cycle", C.c_int32), ("round", C.c_int32), ("toggle", C.c_int32),
                ("eps_prev", C.c_int32), ("calls", C.c_int32), ("src", C.c_int32 * 16)]


def lib():
    """Load the shared library once; fail loudly if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it first (python -m paper_2505_14741_amd.build)")
    L = C.CDLL(_LIB_PATH)
    vp, sz, i32, f32 = C.c_void_p, C.c_size_t, C.c_int, C.c_float
    sig = {
        "ps_strerror": (C.c_char_p, [i32]),
        "dit_set_kernel_path": (i32, [vp, i32]),
        "dit_get_kernel_path": (i32, [vp]),
        "dit_num_weights": (i32, [i32]),
        "dit_create": (i32, [C.POINTER(_DitConfig), C.POINTER(vp), i32, C.POINTER(vp)]),
        "dit_destroy": (i32, [vp]),
        "dit_workspace_bytes": (sz, [vp, i32]),
        "dit_forward": (i32, [vp, vp, vp, C.POINTER(C.c_int32), vp, i32, vp, sz, vp]),
        "dit_profile_enable": (i32, [vp, i32]),
        "dit_profile_read": (i32, [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
        "ps_mfma_probe": (i32, [i32, vp, C.POINTER(C.c_double), vp]),
        "attn3d_workspace_bytes": (sz, [i32, i32, i32, i32, i32]),
        "attn3d": (i32, [vp, vp, vp, vp, i32, i32, i32, i32, f32, i32, i32, vp, sz, vp]),
        "dit_linear_workspace_bytes": (C.c_size_t, [i32, i32, i32, i32, i32]),
        "dit_linear": (i32, [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, C.c_size_t, vp]),
        "cross_attn_workspace_bytes": (sz, [C.POINTER(_CrossShape)]),
        "cross_attn": (i32, [vp, vp, vp, vp, vp, vp, C.POINTER(_CrossShape), vp, sz, vp]),
        "fp8_quantize": (i32, [vp, vp, vp, i32, i32, C.c_int64, i32, vp]),
        "dit_linear_fp8_workspace_bytes": (sz, [i32, i32, i32]),
        "dit_linear_fp8": (i32, [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp]),
        "group_norm_workspace_bytes": (sz, [i32, i32, i32, i32, i32]),
        "group_norm": (i32, [vp, vp, vp, vp, C.POINTER(_GroupNormShape), vp, sz, vp]),
        "fp4_quantize": (i32, [vp, vp, vp, i32, i32, C.c_int64, i32, vp]),
        "fp4_dequantize": (i32, [vp, vp, vp, i32, i32, C.c_int64, i32, vp]),
        "dit_linear_fp4_workspace_bytes": (sz, [i32, i32, i32]),
        "dit_linear_fp4": (i32, [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp]),
        "rope_table": (i32, [vp, C.c_int64, i32, C.POINTER(i32), C.POINTER(C.c_double), vp, i32, vp]),
        "qk_norm_rope": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, C.POINTER(_QkNormShape), vp]),
        "packed_attn_workspace_bytes": (sz, [C.POINTER(_PackedShape)]),
        "packed_attn": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, C.POINTER(_PackedShape), vp, sz, vp]),
        "sampler_step_workspace_bytes": (sz, [sz]),
        "sampler_step": (i32, [vp, vp, vp, vp, C.c_double, C.c_double, sz, vp, vp, sz, vp]),
        "sampler_step_noalloc": (i32, [vp, vp, vp, vp, C.c_double, C.c_double, sz, vp, vp]),
        "rel_mae_workspace_bytes": (sz, [sz]),
        "rel_mae": (i32, [vp, vp, sz, vp, vp, sz, vp]),
        "ddim_coefficients": (i32, [i32, C.c_double, C.c_double, i32, C.POINTER(C.c_int32),
                                    C.POINTER(C.c_double), C.POINTER(C.c_double)]),
        "euler_discrete_coefficients": (i32, [i32, C.c_double, C.c_double, i32, C.POINTER(C.c_int32),
                                              C.POINTER(C.c_double), C.POINTER(C.c_double)]),
        "flow_euler_coefficients": (i32, [i32, i32, C.POINTER(C.c_int32), C.POINTER(C.c_double),
                                          C.POINTER(C.c_double)]),
        "sampler_workspace_bytes": (sz, [vp, C.POINTER(_Schedule)]),
        "sampler_state_bytes": (sz, [vp, C.POINTER(_Schedule)]),
        "sampler_run_steps": (i32, [vp, C.POINTER(_Schedule), C.POINTER(SamplerState), i32, vp, vp, vp, vp, vp, vp, sz,
                                    vp]),
        "sampler_run": (i32, [vp, C.POINTER(_Schedule), vp, vp, vp, vp, vp, C.POINTER(i32), vp, sz, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    _lib = L
    return L


EXPORTED = ("ps_strerror", "ps_mfma_probe", "dit_set_kernel_path", "dit_get_kernel_path", "sampler_step_noalloc", "dit_num_weights", "dit_create", "dit_destroy",
            "dit_workspace_bytes", "dit_forward", "dit_profile_enable", "dit_profile_read",
            "attn3d_workspace_bytes", "attn3d", "dit_linear_workspace_bytes", "dit_linear", "sampler_step_workspace_bytes", "sampler_step",
            "rel_mae_workspace_bytes", "rel_mae", "ddim_coefficients", "euler_discrete_coefficients",
            "flow_euler_coefficients", "sampler_workspace_bytes", "sampler_run", "sampler_state_bytes",
            "sampler_run_steps", "cross_attn_workspace_bytes", "cross_attn", "fp8_quantize", "dit_linear_fp8_workspace_bytes",
            "dit_linear_fp8", "group_norm_workspace_bytes", "group_norm", "fp4_quantize", "fp4_dequantize", "dit_linear_fp4_workspace_bytes",
            "dit_linear_fp4", "rope_table", "qk_norm_rope", "packed_attn_workspace_bytes", "packed_attn")


def _check(status: int, where: str):
    if status != 0:
        raise PsError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()      # (void* arguments take an int as it is)


def _stream():
    """Handle of torch's current stream on the current device."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


@functools.lru_cache(maxsize=1024)
def _bytes_on(device: int, entry: str, *args) -> int:
    return getattr(lib(), entry)(*args)


def _bytes(entry: str, *args) -> int:
    """What a workspace-size function of the library returns for these sizes on the current device (asking it through
    ctypes is a microsecond)."""
    return _bytes_on(torch._C._cuda_getDevice(), entry, *args)


def _dt(name: str) -> int:
    return {"f32": PS_F32, "bf16": PS_BF16}[name]


def torch_dtype(name: str):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _workspace(nbytes: int, device) -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


# ---------------------------------------------------------------------------- predictor
class Dit:
    """Owner of a `dit*` handle and of the weight tensors it borrows."""

    def __init__(self, cfg: DiTConfig, weights: Sequence[torch.Tensor]):
        L = lib()
        self.cfg = cfg
        self.weights = list(weights)            # keep alive
        c = _DitConfig(cfg.layers, cfg.hidden, cfg.heads, cfg.head_dim, cfg.mlp_ratio, cfg.in_channels,
                       cfg.patch, cfg.frames, cfg.height, cfg.width, cfg.text_tokens, cfg.time_embed_dim,
                       _dt(cfg.dtype), cfg.ln_eps, cfg.rope_theta)
        arr = (C.c_void_p * len(self.weights))(*[w.data_ptr() for w in self.weights])
        h = C.c_void_p()
        _check(L.dit_create(C.byref(c), arr, len(self.weights), C.byref(h)), "dit_create")
        self.handle = h
        self._ws = {}

    def close(self):
        if getattr(self, "handle", None):
            lib().dit_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, batch: int) -> torch.Tensor:
        if batch not in self._ws:
            n = lib().dit_workspace_bytes(self.handle, batch)
            if n == 0:
                raise PsError(-2, "dit_workspace_bytes")
            self._ws[batch] = _workspace(n, self.weights[0].device)
        return self._ws[batch]


def dit_create(cfg: DiTConfig, weights: Sequence[torch.Tensor]) -> Dit:
    return Dit(cfg, weights)


def dit_set_kernel_path(d: Dit, path: int):
    _check(lib().dit_set_kernel_path(d.handle, int(path)), "dit_set_kernel_path")


def dit_forward(d: Dit, x: torch.Tensor, ctx: Optional[torch.Tensor], t: Sequence[int],
                eps_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    B = x.shape[0]
    if eps_out is None:
        eps_out = torch.empty_like(x)
    ws = d.workspace(B)
    tt = (C.c_int32 * B)(*[int(v) for v in t])
    _check(lib().dit_forward(d.handle, _ptr(x), _ptr(ctx), tt, _ptr(eps_out), B, _ptr(ws), ws.numel(), _stream()),
           "dit_forward")
    return eps_out


def dit_profile_enable(d: Dit, on):
    """on: False/0 off, True/1 every kernel class, 2 the attention class only."""
    _check(lib().dit_profile_enable(d.handle, int(on)), "dit_profile_enable")


def dit_profile_read(d: Dit):
    ms = (C.c_double * 7)()
    cnt = (C.c_int64 * 7)()
    _check(lib().dit_profile_read(d.handle, ms, cnt), "dit_profile_read")
    return {k: (ms[i], cnt[i]) for i, k in enumerate(KERNEL_CLASSES)}


def ps_mfma_probe(iters: int, sink: torch.Tensor) -> float:
    """Enqueue the MFMA-only launch; returns the operations it performs (time it with events)."""
    flops = C.c_double(0.0)
    _check(lib().ps_mfma_probe(int(iters), _ptr(sink), C.byref(flops), _stream()), "ps_mfma_probe")
    return flops.value


# ---------------------------------------------------------------------------- attention
def attn3d(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float,
           out: Optional[torch.Tensor] = None, kernel_path: int = 0) -> torch.Tensor:
    B, N, H, d = q.shape
    dt = PS_BF16 if q.dtype == torch.bfloat16 else PS_F32
    if out is None:
        out = torch.empty_like(q)
    n = _bytes("attn3d_workspace_bytes", B, N, H, d, dt)
    ws = _workspace(n, q.device)
    _check(lib().attn3d(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, N, H, d, float(scale), dt, int(kernel_path),
                        _ptr(ws), n, _stream()), "attn3d")
    return out


def dit_linear(a: torch.Tensor, w: torch.Tensor, bias: torch.Tensor, act: int = 0,
               out: Optional[torch.Tensor] = None, use_workspace: bool = True, kernel_path: int = 0) -> torch.Tensor:
    M, K = a.shape
    Nn = w.shape[0]
    dt = PS_BF16 if a.dtype == torch.bfloat16 else PS_F32
    if out is None:
        out = torch.empty(M, Nn, dtype=a.dtype, device=a.device)
    nb = _bytes("dit_linear_workspace_bytes", M, Nn, K, dt, int(kernel_path)) if use_workspace else 0
    ws = _workspace(nb, a.device)
    _check(lib().dit_linear(_ptr(a), _ptr(w), _ptr(bias), _ptr(out), M, Nn, K, int(act), dt, int(kernel_path),
                            _ptr(ws), nb, _stream()), "dit_linear")
    return out


# ------------------------------------- operators of a conditioned predictor block
_CODE = {torch.float32: PS_F32, torch.bfloat16: PS_BF16}


def _need(ok: bool, where: str, what: str, status: int = PS_ERR_SHAPE):
    if not ok:
        raise PsError(status, f"{where}: {what}")


def _need_extents(where: str, *extents: int):
    """The library's sizes are 32-bit integers, into which ctypes would cut larger ones."""
    _need(max(extents) < 1 << 31, where, "extents must be below 2^31")


def _need_here(where: str, first: torch.Tensor, *others: Optional[torch.Tensor]):
    """Kernels run on the current device and its current stream, on memory of that device."""
    dev = first.get_device()
    ok = dev >= 0 and dev == torch._C._cuda_getDevice()
    for t in others:
        ok = ok and (t is None or t.get_device() == dev)
    if not ok:
        raise PsError(PS_ERR_SHAPE, f"{where}: tensors must lie on the current GPU")


# What a call checks and computes from types, shapes and strides alone is done once for each (these are microseconds); addresses and devices
# are looked at in every call.
@functools.lru_cache(maxsize=1024)
def _cross_plan(dtypes, q, qs, k, ks, v, vs, o, os_, lens, mask, scale, device):
    w = "cross_attn"
    _need(len(q) == 4 and len(k) == 4 and v == k, w, "q [B, Nq, H, d], k and v [B, Nk, Hkv, d]")
    B, N, H, d = q
    _need(k[0] == B and k[3] == d, w, "k and v must have q's batch and head_dim")
    dt = _CODE.get(dtypes[0])
    _need(dt is not None and dtypes[1] == dtypes[0] and dtypes[2] == dtypes[0], w, "float32 or bfloat16, the same for q, k and v", PS_ERR_DTYPE)
    _need_extents(w, *q, *k)
    _need(o == q, w, "out must have q's shape")
    _need(dtypes[3] == dtypes[0], w, "out must have q's type", PS_ERR_DTYPE)
    _need(qs[3] == ks[3] == vs[3] == os_[3] == 1, w, "the elements of a head must be contiguous")
    mask_batch = 0
    if lens is not None:
        _need(lens[0] == torch.int32, w, "kv_lens must be int32", PS_ERR_DTYPE)
        _need(lens[1] == (B,) and (B <= 1 or lens[2] == (1,)), w, "kv_lens must be [B], contiguous")
    if mask is not None:
        _need(mask[0] in (torch.bool, torch.uint8), w, "key_mask must be bool or uint8", PS_ERR_DTYPE)
        _need(mask[1] == (B, k[1]) and (k[1] <= 1 or mask[2][1] == 1), w, "key_mask must be [B, Nk], rows contiguous")
        mask_batch = mask[2][0] if B > 1 else 0
    s = _CrossShape(B, N, k[1], H, k[2], d, dt, scale, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                    os_[0], os_[1], os_[2], mask_batch)
    return C.byref(s), lib().cross_attn_workspace_bytes(C.byref(s))


def cross_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float, kv_lens: Optional[torch.Tensor] = None,
               key_mask: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q [B, Nq, H, d]; k, v [B, Nk, Hkv, d], any strides whose elements of a head are contiguous; kv_lens int32 [B]; key_mask bool
    or uint8 [B, Nk], also expanded from one sample's.  A query without a key that counts gets zeros."""
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    shape, n = _cross_plan((q.dtype, k.dtype, v.dtype, out.dtype), q.shape, q.stride(), k.shape, k.stride(), v.shape, v.stride(), out.shape, out.stride(),
                           None if kv_lens is None else (kv_lens.dtype, kv_lens.shape, kv_lens.stride()),
                           None if key_mask is None else (key_mask.dtype, key_mask.shape, key_mask.stride()), float(scale), q.get_device())
    _need_here("cross_attn", q, k, v, out, kv_lens, key_mask)
    ws = _workspace(n, q.device)
    _check(lib().cross_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(kv_lens), _ptr(key_mask), out.data_ptr(), shape, _ptr(ws), n, _stream()),
           "cross_attn")
    return out


def fp8_quantize(x: torch.Tensor):
    """x [rows, cols], float32 or bfloat16, rows any distance apart -> (q float8_e4m3fn [rows, kp], scale float8_e8m0fnu [kp / 128,
    pitch]): kp is cols rounded up to 128, pitch is rows rounded up to 16, both filled up as include/parastep.h says."""
    w = "fp8_quantize"
    _need(x.dim() == 2 and x.shape[1] >= 1, w, "x must be [rows, cols]")
    dt = _CODE.get(x.dtype)
    _need(dt is not None, w, "float32 or bfloat16", PS_ERR_DTYPE)
    rows, cols = x.shape
    _need_extents(w, rows, cols)
    _need(x.stride(1) == 1 or cols == 1, w, "the elements of a row must be contiguous")
    _need_here(w, x)
    blocks = (cols + 127) // 128
    q = torch.empty((rows, blocks * 128), dtype=torch.float8_e4m3fn, device=x.device)
    scale = torch.empty((blocks, (rows + 15) // 16 * 16), dtype=torch.float8_e8m0fnu, device=x.device)
    _check(lib().fp8_quantize(x.data_ptr(), q.data_ptr(), scale.data_ptr(), rows, cols, x.stride(0), dt, _stream()), w)
    return q, scale


@functools.lru_cache(maxsize=1024)
def _fp8_plan(dtypes, a, a_scale, w, w_scale, bias, out, use_workspace, device):
    f = "dit_linear_fp8"
    _need(len(a) == 2 and len(w) == 2 and a[1] == w[1] and a[1] % 128 == 0 and a[1] > 0, f, "a [M, kp] and w [n_out, kp], kp a multiple of 128")
    M, K = a
    Nn = w[0]
    _need_extents(f, M, K, Nn)
    _need(dtypes[:4] == (torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float8_e4m3fn, torch.float8_e8m0fnu), f,
          "values in float8_e4m3fn, scales in float8_e8m0fnu", PS_ERR_DTYPE)
    _need(dtypes[4] == torch.float32, f, "bias must be float32", PS_ERR_DTYPE)
    _need(a_scale == (K // 128, (M + 15) // 16 * 16) and w_scale == (K // 128, (Nn + 15) // 16 * 16), f, "scales [kp / 128, rows rounded up to 16]")
    _need(bias == (Nn,), f, "bias must be [n_out]")
    _need(out == (M, Nn), f, "out must be [M, n_out]")
    _need(dtypes[5] == torch.bfloat16, f, "out must be bfloat16", PS_ERR_DTYPE)
    return M, Nn, K, lib().dit_linear_fp8_workspace_bytes(M, Nn, K) if use_workspace else 0


def dit_linear_fp8(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: torch.Tensor, act: int = 0,
                   out: Optional[torch.Tensor] = None, use_workspace: bool = True) -> torch.Tensor:
    """act(a w^T + bias) of operands from fp8_quantize: a of [M, K] and w of [n_out, K]; bias float32 [n_out], out bfloat16."""
    f = "dit_linear_fp8"
    _need(0 <= act <= 1, f, "act 0 or 1")
    if out is None:
        _need(a.dim() == 2 and w.dim() == 2, f, "a [M, kp] and w [n_out, kp]")
        out = torch.empty((a.shape[0], w.shape[0]), dtype=torch.bfloat16, device=a.device)
    M, Nn, K, nb = _fp8_plan((a.dtype, a_scale.dtype, w.dtype, w_scale.dtype, bias.dtype, out.dtype), a.shape, a_scale.shape, w.shape, w_scale.shape,
                             bias.shape, out.shape, use_workspace, a.get_device())
    _need(a.is_contiguous() and a_scale.is_contiguous() and w.is_contiguous() and w_scale.is_contiguous() and bias.is_contiguous() and
          out.is_contiguous(), f, "operands must be contiguous")
    _need_here(f, a, a_scale, w, w_scale, bias, out)
    ws = _workspace(nb, a.device)
    _check(lib().dit_linear_fp8(a.data_ptr(), a_scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(), bias.data_ptr(), out.data_ptr(), M, Nn, K, int(act),
                                _ptr(ws), nb, _stream()), f)
    return out


@functools.lru_cache(maxsize=1024)
def _gnorm_plan(dtypes, x, xs, o, os_, affine, groups, eps, act, device):
    w = "group_norm"
    _need(len(x) == 3 and x[2] >= 1, w, "x must be [B, positions, C]")
    dt = _CODE.get(dtypes[0])
    _need(dt is not None, w, "float32 or bfloat16", PS_ERR_DTYPE)
    _need_extents(w, *x)
    _need(1 <= groups <= x[2] and 0 <= act <= 2, w, "1 to C groups, act 0, 1 or 2")
    _need(o == x, w, "out must have x's shape")
    _need(dtypes[1] == dtypes[0], w, "out must have x's type", PS_ERR_DTYPE)
    _need(x[2] == 1 or (xs[2] == 1 and os_[2] == 1), w, "channels must be contiguous")
    for t in affine:
        _need(t is None or t[0] == torch.float32, w, "gamma and beta must be float32", PS_ERR_DTYPE)
        _need(t is None or (t[1] == (x[2],) and (x[2] == 1 or t[2] == (1,))), w, "gamma and beta must be [C], contiguous")
    s = _GroupNormShape(x[0], x[1], x[2], groups, act, dt, eps, xs[0], xs[1], os_[0], os_[1])
    return C.byref(s), lib().group_norm_workspace_bytes(x[0], x[1], x[2], groups, dt)


def group_norm(x: torch.Tensor, groups: int, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, eps: float = 1e-5,
               act: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [B, positions, C] (channels contiguous, other strides free), float32 or bfloat16; gamma, beta float32 [C]; act 0 none, 1
    tanh-GELU, 2 SiLU.  out may be x."""
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    shape, n = _gnorm_plan((x.dtype, out.dtype), x.shape, x.stride(), out.shape, out.stride(),
                           (None if gamma is None else (gamma.dtype, gamma.shape, gamma.stride()),
                            None if beta is None else (beta.dtype, beta.shape, beta.stride())), int(groups), float(eps), int(act), x.get_device())
    _need_here("group_norm", x, out, gamma, beta)
    ws = _workspace(n, x.device)
    _check(lib().group_norm(x.data_ptr(), _ptr(gamma), _ptr(beta), out.data_ptr(), shape, _ptr(ws), n, _stream()), "group_norm")
    return out


# ------------------------------------- operators of self-attention on packed samples
@functools.lru_cache(maxsize=1024)
def _fp4_quantize_plan(dtype, shape, stride):
    w = "fp4_quantize"
    _need(len(shape) == 2 and shape[1] >= 1, w, "x must be [rows, cols]")
    dt = _CODE.get(dtype)
    _need(dt is not None, w, "float32 or bfloat16", PS_ERR_DTYPE)
    rows, cols = shape
    _need_extents(w, rows, cols)
    _need(stride[1] == 1 or cols == 1, w, "the elements of a row must be contiguous")
    kp = (cols + 127) // 128 * 128
    return dt, (rows, kp // 2), (kp // 32, (rows + 15) // 16 * 16)


def fp4_quantize(x: torch.Tensor):
    """x [rows, cols], float32 or bfloat16, rows any distance apart -> (q uint8 [rows, kp / 2], two e2m1 codes to a byte, scale float8_e8m0fnu
    [kp / 32, pitch]): kp is cols rounded up to 128, pitch is rows rounded up to 16, both filled up as include/parastep.h says."""
    shape, stride = x.shape, x.stride()
    dt, of_q, of_scale = _fp4_quantize_plan(x.dtype, shape, stride)
    _need_here("fp4_quantize", x)
    dev = x.device
    q = torch.empty(of_q, dtype=torch.uint8, device=dev)
    scale = torch.empty(of_scale, dtype=torch.float8_e8m0fnu, device=dev)
    _check(lib().fp4_quantize(x.data_ptr(), q.data_ptr(), scale.data_ptr(), shape[0], shape[1], stride[0], dt, _stream()), "fp4_quantize")
    return q, scale


def fp4_dequantize(q: torch.Tensor, scale: torch.Tensor, cols: Optional[int] = None, dtype: torch.dtype = torch.bfloat16,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values [rows, cols] of fp4_quantize's result (cols: all kp), float32 or bfloat16; NaN where a block was not finite."""
    w = "fp4_dequantize"
    _need(q.dim() == 2 and q.shape[1] % 64 == 0 and q.shape[1] > 0, w, "q must be [rows, kp / 2], kp a multiple of 128")
    _need(q.dtype == torch.uint8 and scale.dtype == torch.float8_e8m0fnu, w, "codes in uint8, scales in float8_e8m0fnu", PS_ERR_DTYPE)
    rows, kp = q.shape[0], 2 * q.shape[1]
    cols = kp if cols is None else int(cols)
    _need_extents(w, rows, kp)
    _need(kp - 128 < cols <= kp, w, "cols must be what kp is rounded up from")
    _need(scale.shape == (kp // 32, (rows + 15) // 16 * 16), w, "scale must be [kp / 32, rows rounded up to 16]")
    _need(q.is_contiguous() and scale.is_contiguous(), w, "q and scale must be contiguous")
    if out is None:
        _need(dtype in _CODE, w, "float32 or bfloat16", PS_ERR_DTYPE)
        out = torch.empty((rows, cols), dtype=dtype, device=q.device)
    dt = _CODE.get(out.dtype)
    _need(dt is not None, w, "float32 or bfloat16", PS_ERR_DTYPE)
    _need(out.shape == (rows, cols) and (out.stride(1) == 1 or cols == 1), w, "out must be [rows, cols], rows contiguous")
    _need_here(w, q, scale, out)
    _check(lib().fp4_dequantize(q.data_ptr(), scale.data_ptr(), out.data_ptr(), rows, cols, out.stride(0), dt, _stream()), w)
    return out


@functools.lru_cache(maxsize=1024)
def _fp4_plan(dtypes, a, a_scale, w, w_scale, bias, out, use_workspace, device):
    f = "dit_linear_fp4"
    _need(len(a) == 2 and len(w) == 2 and a[1] == w[1] and a[1] % 64 == 0 and a[1] > 0, f, "a [M, kp / 2] and w [n_out, kp / 2], kp a multiple of 128")
    M, K = a[0], 2 * a[1]
    Nn = w[0]
    _need_extents(f, M, K, Nn)
    _need(dtypes[:4] == (torch.uint8, torch.float8_e8m0fnu, torch.uint8, torch.float8_e8m0fnu), f, "codes in uint8, scales in float8_e8m0fnu", PS_ERR_DTYPE)
    _need(dtypes[4] == torch.float32, f, "bias must be float32", PS_ERR_DTYPE)
    _need(a_scale == (K // 32, (M + 15) // 16 * 16) and w_scale == (K // 32, (Nn + 15) // 16 * 16), f, "scales [kp / 32, rows rounded up to 16]")
    _need(bias == (Nn,), f, "bias must be [n_out]")
    _need(out == (M, Nn), f, "out must be [M, n_out]")
    _need(dtypes[5] == torch.bfloat16, f, "out must be bfloat16", PS_ERR_DTYPE)
    return M, Nn, K, lib().dit_linear_fp4_workspace_bytes(M, Nn, K) if use_workspace else 0


def dit_linear_fp4(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: torch.Tensor, act: int = 0,
                   out: Optional[torch.Tensor] = None, use_workspace: bool = True) -> torch.Tensor:
    """act(a w^T + bias) of operands from fp4_quantize: a of [M, K] and w of [n_out, K]; bias float32 [n_out], out bfloat16."""
    f = "dit_linear_fp4"
    _need(0 <= act <= 1, f, "act 0 or 1")
    if out is None:
        _need(a.dim() == 2 and w.dim() == 2, f, "a [M, kp / 2] and w [n_out, kp / 2]")
        out = torch.empty((a.shape[0], w.shape[0]), dtype=torch.bfloat16, device=a.device)
    M, Nn, K, nb = _fp4_plan((a.dtype, a_scale.dtype, w.dtype, w_scale.dtype, bias.dtype, out.dtype), a.shape, a_scale.shape, w.shape, w_scale.shape,
                             bias.shape, out.shape, use_workspace, a.get_device())
    _need(a.is_contiguous() and a_scale.is_contiguous() and w.is_contiguous() and w_scale.is_contiguous() and bias.is_contiguous() and
          out.is_contiguous(), f, "operands must be contiguous")
    _need_here(f, a, a_scale, w, w_scale, bias, out)
    ws = _workspace(nb, a.device)
    _check(lib().dit_linear_fp4(a.data_ptr(), a_scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(), bias.data_ptr(), out.data_ptr(), M, Nn, K, int(act),
                                _ptr(ws), nb, _stream()), f)
    return out


@functools.lru_cache(maxsize=1024)
def _rope_plan(dtype, shape, stride, dims, thetas):
    w, n = "rope_table", len(dims)
    _need(len(shape) == 2 and 1 <= n <= 4 and shape[1] == n, w, "positions must be [tokens, axes], 1 to 4 axes of axis_dims")
    _need(dtype == torch.float32, w, "positions must be float32", PS_ERR_DTYPE)
    thetas = thetas if isinstance(thetas, tuple) else (thetas,) * n
    _need(len(thetas) == n, w, "theta must be one number, or one for each axis")
    _need(all(0 < d <= 256 and d % 2 == 0 for d in dims), w, "axis_dims must be even, 256 in all at most")
    _need_extents(w, shape[0])
    _need(n == 1 or stride[1] == 1 or shape[0] == 0, w, "a token's positions must be contiguous")
    return n, (C.c_int * n)(*dims), (C.c_double * n)(*thetas), (shape[0], sum(dims) // 2, 2)


def rope_table(positions: torch.Tensor, axis_dims: Sequence[int], theta=10000.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """positions float32 [tokens, axes] -> float32 [tokens, sum(axis_dims) / 2, 2] of (cos, sin); theta one number, or one for each axis."""
    w, stride = "rope_table", positions.stride()
    n, dims, thetas, shape = _rope_plan(positions.dtype, positions.shape, stride, tuple(int(d) for d in axis_dims),
                                        tuple(float(t) for t in theta) if isinstance(theta, (list, tuple)) else float(theta))
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=positions.device)
    else:
        _need(out.dtype == torch.float32, w, "out must be float32", PS_ERR_DTYPE)
        _need(out.shape == shape and out.is_contiguous(), w, "out must be [tokens, sum(axis_dims) / 2, 2], contiguous")
    _need_here(w, positions, out)
    _check(lib().rope_table(positions.data_ptr(), stride[0], n, dims, thetas, out.data_ptr(), shape[0], _stream()), w)
    return out


def _like(t: Optional[torch.Tensor]):
    return None if t is None else (t.dtype, t.shape, t.stride())


@functools.lru_cache(maxsize=1024)
def _qk_plan(q, k, qo, ko, table, norm, eps, halves):
    w = "qk_norm_rope"
    _need(len(q[1]) == 4, w, "q must be [B, N, H, d]")
    B, N, H, d = q[1]
    dt = _CODE.get(q[0])
    _need(dt is not None, w, "float32 or bfloat16", PS_ERR_DTYPE)
    _need((k is None) == (ko is None), w, "k_out goes with k")
    _need(k is None or (len(k[1]) == 4 and k[1][:2] == (B, N) and k[1][3] == d and k[1][2] >= 1), w, "k must be [B, N, Hkv, d]")
    _need(qo[1] == q[1] and (k is None or ko[1] == k[1]), w, "outputs must have their inputs' shapes")
    for t in (k, qo, ko):
        _need(t is None or t[0] == q[0], w, "one type for all", PS_ERR_DTYPE)
    for t in (q, k, qo, ko):
        _need(t is None or t[2][3] == 1, w, "the elements of a head must be contiguous")
    _need(0 <= norm <= 2, w, "norm 0, 1 or 2")
    _need_extents(w, B, N, H, d, k[1][2] if k else 0)
    rotated = table_batch = 0
    if table is not None:
        _need(table[0] == torch.float32, w, "table must be float32", PS_ERR_DTYPE)
        shape, stride = (table[1], table[2]) if len(table[1]) == 4 else ((B,) + tuple(table[1]), (0,) + tuple(table[2]))
        _need(len(shape) == 4 and shape[0] == B and shape[1] == N and shape[3] == 2 and 1 <= shape[2] <= 128, w, "table must be [N, pairs, 2] or [B, N, pairs, 2]")
        rotated, table_batch = 2 * shape[2], stride[0] if B > 1 else 0
        _need(stride[3] == 1 and (shape[2] == 1 or stride[2] == 2) and (N <= 1 or stride[1] == rotated), w, "a sample's table must be contiguous")
    none = (None, (0, 0, 0), (0, 0, 0))
    kk, oo = k or none, ko or none
    s = _QkNormShape(B, N, H, k[1][2] if k else 0, d, rotated, norm, int(halves), dt, eps, *q[2][:3], *kk[2][:3], *qo[2][:3], *oo[2][:3], table_batch)
    return C.byref(s)


def qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], table: Optional[torch.Tensor], gamma_q: Optional[torch.Tensor] = None,
                 gamma_k: Optional[torch.Tensor] = None, beta_q: Optional[torch.Tensor] = None, beta_k: Optional[torch.Tensor] = None, norm: int = 1,
                 eps: float = 1e-6, halves: bool = False, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """q [B, N, H, d] and k [B, N, Hkv, d] (or None), elements of a head contiguous, normalised over each head (norm 0 none, 1 by the root of the mean
    square, 2 by mean and deviation; gamma, beta float32 [d]) and turned by table, [N, pairs, 2] or [B, N, pairs, 2] from rope_table (None: not
    turned): neighbouring values, or with halves the first pairs values with the next.  Returns (q_out, k_out), which may be q and k."""
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k_out is None and k is not None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    shape = _qk_plan(_like(q), _like(k), _like(q_out), _like(k_out), _like(table), int(norm), float(eps), bool(halves))
    for t in (gamma_q, gamma_k, beta_q, beta_k):
        if t is not None:
            _need(t.dtype is torch.float32, "qk_norm_rope", "gamma and beta must be float32", PS_ERR_DTYPE)
            _need(t.shape == q.shape[3:] and t.is_contiguous(), "qk_norm_rope", "gamma and beta must be [d], contiguous")
    _need_here("qk_norm_rope", q, k, q_out, k_out, table, gamma_q, gamma_k, beta_q, beta_k)
    _check(lib().qk_norm_rope(q.data_ptr(), _ptr(k), _ptr(table), _ptr(gamma_q), _ptr(beta_q), _ptr(gamma_k), _ptr(beta_k), q_out.data_ptr(), _ptr(k_out),
                              shape, _stream()), "qk_norm_rope")
    return q_out, k_out


@functools.lru_cache(maxsize=1024)
def _packed_plan(q, k, v, o, q_offsets, kv_offsets, prefix_lens, slopes, scale, frame, causal, cap, device):
    w = "packed_attn"
    _need(len(q[1]) == 3 and len(k[1]) == 3 and v[1] == k[1], w, "q [Tq, H, d], k and v [Tk, Hkv, d]")
    T, H, d = q[1]
    _need(k[1][2] == d, w, "k and v must have q's head_dim")
    dt = _CODE.get(q[0])
    _need(dt is not None and k[0] == q[0] and v[0] == q[0], w, "float32 or bfloat16, the same for q, k and v", PS_ERR_DTYPE)
    _need(o[1] == q[1], w, "out must have q's shape")
    _need(o[0] == q[0], w, "out must have q's type", PS_ERR_DTYPE)
    _need(q[2][2] == k[2][2] == v[2][2] == o[2][2] == 1, w, "the elements of a head must be contiguous")
    _need(len(q_offsets[1]) == 1 and q_offsets[1][0] >= 1, w, "q_offsets must be [samples + 1]")
    n = q_offsets[1][0] - 1
    _need_extents(w, T, H, d, *k[1], n, frame)
    for t, m in ((q_offsets, n + 1), (kv_offsets, n + 1), (prefix_lens, n)):
        _need(t is None or t[0] == torch.int32, w, "offsets and prefix_lens must be int32", PS_ERR_DTYPE)
        _need(t is None or (t[1] == (m,) and (m <= 1 or t[2] == (1,))), w, "kv_offsets must be [samples + 1] and prefix_lens [samples], contiguous")
    _need(slopes is None or slopes[0] == torch.float32, w, "slopes must be float32", PS_ERR_DTYPE)
    _need(slopes is None or (slopes[1] == (H,) and (H == 1 or slopes[2] == (1,))), w, "slopes must be [H], contiguous")
    _need(kv_offsets is not None or k[1][0] == T, w, "without kv_offsets, keys must be as many as queries")
    s = _PackedShape(n, T, k[1][0], H, k[1][1], d, dt, int(kv_offsets is not None), int(causal), frame, scale, cap, *q[2][:2], *k[2][:2], *v[2][:2], *o[2][:2])
    return C.byref(s), lib().packed_attn_workspace_bytes(C.byref(s))


def packed_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float, q_offsets: torch.Tensor, kv_offsets: Optional[torch.Tensor] = None,
                prefix_lens: Optional[torch.Tensor] = None, frame: int = 1, causal: bool = False, cap: float = 0.0,
                slopes: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q [Tq, H, d]; k, v [Tk, Hkv, d], any strides whose elements of a head are contiguous; sample s has the queries q_offsets[s] .. q_offsets[s + 1] - 1
    (int32 [samples + 1]) and the keys of kv_offsets (None: the queries'), its queries being its last tokens.  Behind the sample's first prefix_lens[s]
    tokens (int32 [samples]) tokens lie in frames of `frame`; causal: a query sees the prefix and the frames up to its own; slopes (float32 [H]):
    scores less slope * distance in frames; cap: scores capped by cap * tanh(score / cap).  A query that sees no key gets zeros; rows of out
    outside all samples are not written."""
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    shape, n = _packed_plan(_like(q), _like(k), _like(v), _like(out), _like(q_offsets), _like(kv_offsets), _like(prefix_lens), _like(slopes), float(scale),
                            int(frame), bool(causal), float(cap), q.get_device())
    _need_here("packed_attn", q, k, v, out, q_offsets, kv_offsets, prefix_lens, slopes)
    ws = _workspace(n, q.device)
    _check(lib().packed_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), q_offsets.data_ptr(), _ptr(kv_offsets), _ptr(prefix_lens), _ptr(slopes),
                             out.data_ptr(), shape, _ptr(ws), n, _stream()), "packed_attn")
    return out


# ---------------------------------------------------------------- scheduler and metric
def sampler_step(x: torch.Tensor, eps: torch.Tensor, eps_prev: Optional[torch.Tensor], a: float, b: float,
                 x_out: Optional[torch.Tensor] = None, want_sums: bool = True):
    n = x.numel()
    if x_out is None:
        x_out = torch.empty_like(x)
    sums = torch.empty(4, dtype=torch.float32, device=x.device) if want_sums else None
    nb = _bytes("sampler_step_workspace_bytes", n) if want_sums else 0
    ws = _workspace(nb, x.device)
    _check(lib().sampler_step(_ptr(x), _ptr(eps), _ptr(eps_prev), _ptr(x_out), float(a), float(b), n, _ptr(sums),
                              _ptr(ws), nb, _stream()), "sampler_step")
    return x_out, sums


def sampler_step_noalloc(x: torch.Tensor, eps: torch.Tensor, eps_prev: Optional[torch.Tensor], a: float, b: float,
                         x_out: torch.Tensor, sums: Optional[torch.Tensor]):
    """The caller supplies every buffer; neither this wrapper nor the library allocates."""
    _check(lib().sampler_step_noalloc(_ptr(x), _ptr(eps), _ptr(eps_prev), _ptr(x_out), float(a), float(b), x.numel(),
                                      _ptr(sums), _stream()), "sampler_step_noalloc")
    return x_out, sums


def rel_mae(a: torch.Tensor, b: torch.Tensor) -> torch.Tensor:
    n = a.numel()
    out = torch.empty(3, dtype=torch.float32, device=a.device)
    nb = _bytes("rel_mae_workspace_bytes", n)
    ws = _workspace(nb, a.device)
    _check(lib().rel_mae(_ptr(a), _ptr(b), n, _ptr(out), _ptr(ws), nb, _stream()), "rel_mae")
    return out


def ddim_coefficients(steps: int, train_steps: int = 1000, beta_start: float = 1e-4, beta_end: float = 2e-2):
    ts = (C.c_int32 * steps)()
    a = (C.c_double * steps)()
    b = (C.c_double * steps)()
    _check(lib().ddim_coefficients(train_steps, beta_start, beta_end, steps, ts, a, b), "ddim_coefficients")
    return (np.array(ts[:], dtype=np.int32), np.array(a[:], dtype=np.float64), np.array(b[:], dtype=np.float64))


def euler_discrete_coefficients(steps: int, train_steps: int = 1000, beta_start: float = 1e-4, beta_end: float = 2e-2):
    ts = (C.c_int32 * steps)()
    a = (C.c_double * steps)()
    b = (C.c_double * steps)()
    _check(lib().euler_discrete_coefficients(train_steps, beta_start, beta_end, steps, ts, a, b),
           "euler_discrete_coefficients")
    return (np.array(ts[:], dtype=np.int32), np.array(a[:], dtype=np.float64), np.array(b[:], dtype=np.float64))


def flow_euler_coefficients(steps: int, train_steps: int = 1000):
    ts = (C.c_int32 * steps)()
    a = (C.c_double * steps)()
    b = (C.c_double * steps)()
    _check(lib().flow_euler_coefficients(train_steps, steps, ts, a, b), "flow_euler_coefficients")
    return (np.array(ts[:], dtype=np.int32), np.array(a[:], dtype=np.float64), np.array(b[:], dtype=np.float64))


# ------------------------------------------------------------------ reuse-then-predict
class Schedule:
    """Host arrays behind a `sampler_schedule` (kept alive while the struct is in use)."""

    def __init__(self, timesteps, coef_a, coef_b, warmup: int, cycle_len: Sequence[int], batched: bool = False,
                 mode: int = 0):
        self.ts = np.ascontiguousarray(timesteps, dtype=np.int32)
        self.a = np.ascontiguousarray(coef_a, dtype=np.float64)
        self.b = np.ascontiguousarray(coef_b, dtype=np.float64)
        self.cyc = np.ascontiguousarray(cycle_len, dtype=np.int32)
        self.c = _Schedule(len(self.ts), self.ts.ctypes.data_as(C.POINTER(C.c_int32)),
                           self.a.ctypes.data_as(C.POINTER(C.c_double)), self.b.ctypes.data_as(C.POINTER(C.c_double)),
                           int(warmup), len(self.cyc), self.cyc.ctypes.data_as(C.POINTER(C.c_int32)),
                           int(batched), int(mode))


def sampler_run(d: Dit, sched: Schedule, x_T: torch.Tensor, ctx: Optional[torch.Tensor],
                want_trajectory: bool = False):
    """Returns (x0, step_sums [steps,4], predictor launches), plus the per-step samples [steps, ...] if asked."""
    L = lib()
    nb = L.sampler_workspace_bytes(d.handle, C.byref(sched.c))
    if nb == 0:
        raise PsError(-5, "sampler_workspace_bytes")
    ws = _workspace(nb, x_T.device)
    x0 = torch.empty_like(x_T)
    sums = torch.zeros(len(sched.ts), 4, dtype=torch.float32, device=x_T.device)
    traj = (torch.empty((len(sched.ts),) + tuple(x_T.shape), dtype=torch.float32, device=x_T.device)
            if want_trajectory else None)
    calls = C.c_int(0)
    _check(L.sampler_run(d.handle, C.byref(sched.c), _ptr(x_T), _ptr(ctx), _ptr(x0), _ptr(sums), _ptr(traj),
                         C.byref(calls), _ptr(ws), nb, _stream()), "sampler_run")
    if want_trajectory:
        return x0, sums, calls.value, traj
    return x0, sums, calls.value


def sampler_workspace(d: Dit, sched: Schedule, device) -> torch.Tensor:
    nb = lib().sampler_workspace_bytes(d.handle, C.byref(sched.c))
    if nb == 0:
        raise PsError(-5, "sampler_workspace_bytes")
    return _workspace(nb, device)


def sampler_state_bytes(d: Dit, sched: Schedule) -> int:
    return lib().sampler_state_bytes(d.handle, C.byref(sched.c))


def sampler_run_steps(d: Dit, sched: Schedule, state: SamplerState, stop_step: int, x_T: Optional[torch.Tensor],
                      ctx: Optional[torch.Tensor], ws: torch.Tensor, x_out: Optional[torch.Tensor] = None,
                      step_sums: Optional[torch.Tensor] = None, trajectory: Optional[torch.Tensor] = None):
    """Advance a run from state.step to stop_step; `ws` (from sampler_workspace) carries the tensors of the state."""
    _check(lib().sampler_run_steps(d.handle, C.byref(sched.c), C.byref(state), int(stop_step), _ptr(x_T), _ptr(ctx),
                                   _ptr(x_out), _ptr(step_sums), _ptr(trajectory), _ptr(ws), ws.numel(), _stream()),
           "sampler_run_steps")
    return x_out


def weights_to_device(cfg: DiTConfig, weights, device="cuda") -> List[torch.Tensor]:
    """Upload a weight list (name, fp32 ndarray): matrices in cfg.dtype, biases fp32."""
    out = []
    for _, w in weights:
        t = torch.from_numpy(np.ascontiguousarray(w))
        if w.ndim == 2:
            t = t.to(torch_dtype(cfg.dtype))
        out.append(t.to(device).contiguous())
    return out
