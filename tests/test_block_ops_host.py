"""Operators of a conditioned predictor block: what they refuse, on the host and before any launch."""
import ctypes as C

import pytest
import torch

from paper_2505_14741_amd import binding as B

FAKE = 0x10000                                                   # never dereferenced: every call below is refused or has nothing to do


def cross_shape(**over):
    s = dict(batch=2, q_len=5, kv_len=7, heads=4, kv_heads=2, head_dim=64, dtype=1, scale=0.125, q_batch=5 * 256, q_token=256, q_head=64,
             k_batch=7 * 128, k_token=128, k_head=64, v_batch=7 * 128, v_token=128, v_head=64, o_batch=5 * 256, o_token=256, o_head=64, mask_batch=0)
    s.update(over)
    return B._CrossShape(**s)


def call_cross(shape, q=FAKE, k=2 * FAKE, v=3 * FAKE, o=4 * FAKE, lens=None, mask=None, ws=None, ws_bytes=0):
    return B.lib().cross_attn(q, k, v, lens, mask, o, C.byref(shape) if shape else None, ws, ws_bytes, None)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=2), -3), (dict(head_dim=48), -2), (dict(head_dim=0), -2), (dict(batch=-1), -2), (dict(q_len=-1), -2), (dict(kv_len=-1), -2), (dict(heads=0), -2),
    (dict(kv_heads=3), -2), (dict(kv_heads=0), -2), (dict(scale=0.0), -2), (dict(scale=-1.0), -2), (dict(scale=float("nan")), -2),
    (dict(scale=float("inf")), -2), (dict(q_token=252), -2), (dict(q_head=-64), -2), (dict(k_token=100), -2), (dict(v_batch=-8), -2), (dict(o_token=0), -2),
    (dict(o_head=0), -2), (dict(o_batch=0), -2), (dict(mask_batch=-1), -2), (dict(batch=65536), -2), (dict(q_len=(1 << 24) + 1), -2),
    (dict(kv_len=(1 << 24) + 1), -2), (dict(k_token=1 << 41), -2), (dict(batch=60000, q_len=1 << 20), -2)])
def test_cross_attention_refuses(over, status):
    assert call_cross(cross_shape(**over)) == status
    assert B.lib().cross_attn_workspace_bytes(C.byref(cross_shape(**over))) == 0


def test_cross_attention_refuses_pointers():
    ok = cross_shape()
    assert call_cross(None) == -1 and B.lib().cross_attn_workspace_bytes(None) == 0
    for name in ("q", "k", "v", "o"):
        assert call_cross(ok, **{name: None}) == -1
        assert call_cross(ok, **{name: 5 * FAKE + 8}) == -2
    assert call_cross(ok, lens=FAKE + 2) == -2
    for same in (FAKE, 2 * FAKE, 3 * FAKE):
        assert call_cross(ok, o=same) == -2
    # nothing to do: no pointer is looked at, extents of one have no stride
    assert call_cross(cross_shape(batch=0), q=None, k=None, v=None, o=None) == 0
    assert call_cross(cross_shape(q_len=0), q=None, k=None, v=None, o=None) == 0
    assert call_cross(cross_shape(kv_len=0), o=None) == -1


def test_cross_attention_workspace():
    """Few rows over many keys need scratch; a missing, small or misaligned one is refused."""
    s = cross_shape(batch=1, q_len=1, kv_len=100000)
    n = B.lib().cross_attn_workspace_bytes(C.byref(s))
    assert n > 0 and n % 256 == 0
    assert call_cross(s) == -4 and call_cross(s, ws=FAKE, ws_bytes=n - 1) == -4 and call_cross(s, ws=FAKE + 128, ws_bytes=n) == -4
    two = cross_shape(batch=2, q_len=1, kv_len=100000)
    assert B.lib().cross_attn_workspace_bytes(C.byref(two)) == 2 * n          # a sample's plan does not depend on the batch
    assert B.lib().cross_attn_workspace_bytes(C.byref(cross_shape(q_len=17550, kv_len=226))) == 0


def test_quantize_refuses():
    L = B.lib()
    call = lambda x=FAKE, q=2 * FAKE, s=3 * FAKE, rows=4, cols=100, x_row=100, dtype=1: L.fp8_quantize(x, q, s, rows, cols, x_row, dtype, None)  # noqa: E731
    assert call(dtype=2) == -3
    for bad in (dict(rows=-1), dict(cols=0), dict(rows=(1 << 24) + 1), dict(cols=(1 << 22) + 1), dict(x_row=99), dict(x_row=1 << 41),
                dict(rows=1 << 24, cols=1 << 15, x_row=1 << 15), dict(rows=1 << 24, cols=2048, x_row=2048), dict(x=FAKE + 1), dict(q=2 * FAKE + 8), dict(s=3 * FAKE + 4), dict(q=FAKE), dict(s=FAKE)):
        assert call(**bad) == -2, bad
    for name in ("x", "q", "s"):
        assert call(**{name: None}) == -1
    assert call(rows=0, x=None, q=None, s=None) == 0


def test_product_refuses():
    L = B.lib()

    def call(a=FAKE, a_s=2 * FAKE, w=3 * FAKE, w_s=4 * FAKE, bias=5 * FAKE, out=6 * FAKE, m=4, n=8, k=128, act=0, ws=None, nb=0):
        return L.dit_linear_fp8(a, a_s, w, w_s, bias, out, m, n, k, act, ws, nb, None)
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(m=(1 << 24) + 1), dict(n=(1 << 24) + 1), dict(k=(1 << 22) + 1), dict(act=2), dict(act=-1), dict(m=1 << 24, n=1 << 24), dict(m=1 << 18, n=1 << 18),
                dict(a=FAKE + 8), dict(a_s=FAKE + 8), dict(w=FAKE + 8), dict(w_s=FAKE + 4), dict(bias=FAKE + 4), dict(out=FAKE + 2), dict(out=FAKE), dict(out=3 * FAKE)):
        assert call(**bad) == -2, bad
    for name in ("a", "a_s", "w", "w_s", "bias", "out"):
        assert call(**{name: None}) == -1
    assert call(ws=FAKE + 128, nb=1 << 20) == -4
    assert call(m=0, a=None, a_s=None, out=None) == 0
    assert L.dit_linear_fp8_workspace_bytes(0, 8, 128) == 0 and L.dit_linear_fp8_workspace_bytes(4, 8, (1 << 22) + 1) == 0


def test_group_norm_refuses():
    L = B.lib()

    def call(x=FAKE, gamma=None, beta=None, out=2 * FAKE, ws=None, nb=0, shape=True, **over):
        s = dict(batch=2, positions=5, channels=64, groups=8, act=0, dtype=1, eps=1e-5, x_batch=320, x_position=64, out_batch=320, out_position=64)
        s.update(over)
        return L.group_norm(x, gamma, beta, out, C.byref(B._GroupNormShape(**s)) if shape else None, ws, nb, None)
    assert call(shape=False) == -1 and call(dtype=3) == -3
    for bad in (dict(batch=-1), dict(positions=-1), dict(channels=0), dict(groups=0), dict(groups=7), dict(act=3), dict(act=-1), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(batch=65536), dict(positions=(1 << 24) + 1), dict(channels=65544), dict(x_batch=-1),
                dict(x_position=-64), dict(out_batch=0), dict(out_position=32), dict(x_batch=1 << 41), dict(x=FAKE + 1), dict(out=FAKE + 1), dict(gamma=FAKE + 2),
                dict(out=FAKE, out_position=72, out_batch=360)):
        assert call(**bad) == -2, bad
    assert call(x=None) == -1 and call(out=None) == -1
    assert call(batch=0, x=None, out=None) == 0 and call(positions=0, x=None, out=None) == 0
    n = L.group_norm_workspace_bytes(1, 70200, 512, 32, 1)
    assert n > 0 and n % 256 == 0 and L.group_norm_workspace_bytes(3, 70200, 512, 32, 1) == 3 * n
    big = dict(batch=1, positions=70200, channels=512, groups=32, x_position=512, out_position=512)
    assert call(**big) == -4 and call(ws=FAKE, nb=n - 1, **big) == -4 and call(ws=FAKE + 16, nb=n, **big) == -4
    assert L.group_norm_workspace_bytes(1, 5, 64, 7, 1) == 0


def test_binding_refuses_tensors():
    """Wrong types, shapes, strides and places raise before the library is called."""
    q, k = torch.zeros(2, 5, 4, 64), torch.zeros(2, 7, 2, 64)
    x = torch.zeros(4, 128)
    q8, s8 = torch.zeros(4, 128, dtype=torch.float8_e4m3fn), torch.zeros(1, 16, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    bias = torch.zeros(4)
    shape, dtype = -2, -3
    calls = [
        (lambda: B.cross_attn(q[0], k, k, 1.0), shape), (lambda: B.cross_attn(q, k, k[:, :6], 1.0), shape), (lambda: B.cross_attn(q, k[:1], k[:1], 1.0), shape),
        (lambda: B.cross_attn(q, k[..., :32], k[..., :32], 1.0), shape), (lambda: B.cross_attn(q.half(), k.half(), k.half(), 1.0), dtype),
        (lambda: B.cross_attn(q, k, k.bfloat16(), 1.0), dtype), (lambda: B.cross_attn(q, k, k, 1.0, out=q[:, :4]), shape),
        (lambda: B.cross_attn(q, k, k, 1.0, out=torch.empty_like(q, dtype=torch.bfloat16)), dtype),
        (lambda: B.cross_attn(q.transpose(2, 3).contiguous().transpose(2, 3), k, k, 1.0), shape),
        (lambda: B.cross_attn(q, k, k, 1.0, kv_lens=torch.zeros(2, dtype=torch.int64)), dtype),
        (lambda: B.cross_attn(q, k, k, 1.0, kv_lens=torch.zeros(3, dtype=torch.int32)), shape),
        (lambda: B.cross_attn(q, k, k, 1.0, key_mask=torch.zeros(2, 7)), dtype), (lambda: B.cross_attn(q, k, k, 1.0, key_mask=torch.zeros(2, 6, dtype=torch.bool)), shape),
        (lambda: B.cross_attn(q, k, k, 1.0, key_mask=torch.zeros(7, 2, dtype=torch.bool).t()), shape),
        (lambda: B.cross_attn(q, k, k, 1.0), shape),             # not on the GPU
        (lambda: B.fp8_quantize(x[0]), shape), (lambda: B.fp8_quantize(x.half()), dtype), (lambda: B.fp8_quantize(x.t()), shape), (lambda: B.fp8_quantize(x), shape),
        (lambda: B.dit_linear_fp8(x, s8, q8, s8, bias), dtype), (lambda: B.dit_linear_fp8(q8, s8.view(torch.uint8), q8, s8, bias), dtype),
        (lambda: B.dit_linear_fp8(q8[:, :64], s8, q8[:, :64], s8, bias), shape), (lambda: B.dit_linear_fp8(q8, s8[:, :4], q8, s8, bias), shape),
        (lambda: B.dit_linear_fp8(q8, s8, q8, s8, bias[:3]), shape), (lambda: B.dit_linear_fp8(q8, s8, q8, s8, bias.double()), dtype),
        (lambda: B.dit_linear_fp8(q8, s8, q8, s8, bias, out=torch.zeros(4, 5, dtype=torch.bfloat16)), shape),
        (lambda: B.dit_linear_fp8(q8, s8, q8, s8, bias, out=torch.zeros(4, 4)), dtype), (lambda: B.dit_linear_fp8(q8, s8, q8, s8, bias), shape),
        (lambda: B.group_norm(x, 8), shape), (lambda: B.group_norm(x[None].half(), 8), dtype), (lambda: B.group_norm(x[None].transpose(1, 2), 4), shape),
        (lambda: B.group_norm(x[None], 8, gamma=torch.zeros(64)), shape), (lambda: B.group_norm(x[None], 8, beta=torch.zeros(128).bfloat16()), dtype),
        (lambda: B.group_norm(x[None], 8, out=torch.zeros(1, 4, 127)), shape), (lambda: B.group_norm(x[None], 8, out=x[None].bfloat16()), dtype),
        (lambda: B.group_norm(x[None], 8), shape)]
    for i, (call, status) in enumerate(calls):
        with pytest.raises(B.PsError) as e:
            call()
        assert e.value.status == status, i
