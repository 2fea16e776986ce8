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
            "dit_linear_fp8", "group_norm_workspace_bytes", "group_norm")


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
