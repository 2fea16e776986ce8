"""Operators of a conditioned predictor block at the ends of their ranges: what is not finite, values and scores as large as their types
hold, addresses on no border, the largest grids."""
import math

import pytest
import torch

from paper_2505_14741_amd import binding as B
from test_block_edges_host import PRODUCTS
from test_gpu_block_ops import (DEV, NAN, U, block_data, check_cross, check_gnorm, check_quantize, conditioned_block, cross_ref, fp8_ref, gen,
                                randn)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- cross attention
# (few rows; rows whose keys are divided; all keys in LDS in bf16 up to heads of 64)
SIZES = [(3, 100), (40, 2600), (300, 226)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("nq,nk", SIZES)
def test_rows_without_a_key_are_zero_whatever_their_query_holds(dtype, d, nq, nk):
    """An empty place of a padded batch, its queries never written: a mask of zeros, a length of zero.  Beside it a sample with the same
    queries and all keys."""
    print(f"cross_attn empty rows {dtype} d={d} q={nq} k={nk}", flush=True)
    g = gen(nq + nk + d)
    q, k, v = randn(g, 3, nq, 2, d).to(dtype), randn(g, 3, nk, 2, d).to(dtype), randn(g, 3, nk, 2, d).to(dtype)
    junk = torch.tensor([NAN, float("inf"), -float("inf"), 1.0], device=DEV).to(dtype)
    q[:2] = junk[torch.randint(0, 4, (2, nq, 2, d), generator=g, device=DEV)]
    mask = torch.ones(3, nk, dtype=torch.bool, device=DEV)
    mask[0] = False
    lens = torch.tensor([nk, 0, nk], dtype=torch.int32, device=DEV)
    out = B.cross_attn(q, k, v, 1.0 / math.sqrt(d), kv_lens=lens, key_mask=mask)
    assert bool((out[:2] == 0).all())
    assert torch.equal(out[2:], B.cross_attn(q[2:], k[2:], v[2:], 1.0 / math.sqrt(d), kv_lens=lens[2:], key_mask=mask[2:]))
    check_cross(q[2:], k[2:], v[2:], 1.0 / math.sqrt(d))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq,nk", SIZES)
def test_a_query_that_is_not_finite_spoils_its_own_row_only(dtype, nq, nk):
    g = gen(nq + nk)
    q, k, v = randn(g, 1, nq, 2, 64).to(dtype), randn(g, 1, nk, 2, 64).to(dtype), randn(g, 1, nk, 2, 64).to(dtype)
    whole = torch.ones(1, nk, dtype=torch.bool, device=DEV)
    ref, tol = cross_ref(q, k, v, 0.125, whole)
    for mask in (None, torch.arange(nk, device=DEV)[None] >= 70):            # (nothing of the first 64 keys)
        if mask is not None:
            ref, tol = cross_ref(q, k, v, 0.125, mask)
        for bad in (NAN, float("inf")):
            p = q.clone()
            p[0, 1, 0, 5] = bad
            out = B.cross_attn(p, k, v, 0.125, key_mask=mask)
            good = torch.ones(1, nq, 2, 64, dtype=torch.bool, device=DEV)
            good[0, 1, 0] = False
            assert bool(((out.double() - ref).abs() <= tol * 1.001)[good].all())
            assert bool(torch.isnan(out[0, 1, 0]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [16, 64])
@pytest.mark.parametrize("growth", [0.0, 11.0, 15.0, 30.0])
@pytest.mark.parametrize("nq,nk", [(5, 200), (40, 2600), (300, 200), (300, 640)])
def test_values_as_large_as_their_sums_allow(dtype, d, growth, nq, nk):
    """|v| * keys * 2^8 below 2^128, under scores that grow by `growth` behind the first 64 keys (by 15: e^15 = 2^21.6 times 2^110)."""
    print(f"cross_attn large values {dtype} d={d} q={nq} k={nk} growth={growth}", flush=True)
    g = gen(26)
    q, k = randn(g, 1, nq, 1, d) * 0.25, randn(g, 1, nk, 1, d) * 0.25
    q[..., 0], k[0, :64, 0, 0], k[0, 64:, 0, 0] = 1.0, 0.0, growth
    v = randn(g, 1, nk, 1, d)
    v *= 2.0 ** (118 - math.ceil(math.log2(nk))) / v.abs().max()
    assert float(v.abs().max()) * nk * 256 < 2.0 ** 128
    assert bool(torch.isfinite(check_cross(q.to(dtype), k.to(dtype), v.to(dtype), 1.0)).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("first", [1, 64, 70])
@pytest.mark.parametrize("nq,nk", [(5, 200), (40, 2600), (300, 200), (300, 640)])
def test_scores_whose_difference_is_beyond_their_type(dtype, first, nq, nk):
    """Scores of -1.75 * 2^127 and then 1.75 * 2^127 under a scale of 1e-38: 6 apart in the exponent, so that the first keys, whose values
    alone are not zero, count for exp(-6) each."""
    g = gen(27)
    q, k = torch.zeros(1, nq, 1, 64, device=DEV), torch.zeros(1, nk, 1, 64, device=DEV)
    q[..., 0], k[0, :first, 0, 0], k[0, first:, 0, 0] = 2.0 ** 63, -1.75 * 2.0 ** 64, 1.75 * 2.0 ** 64
    v = randn(g, 1, nk, 1, 64) * 100.0
    v[:, first:] = 0.0
    for flip in (False, True):
        kk, vv = (k.flip(1), v.flip(1)) if flip else (k, v)
        mask = torch.ones(1, nk, dtype=torch.bool, device=DEV)
        check_cross(q.to(dtype), kk.to(dtype).contiguous(), vv.to(dtype).contiguous(), 1e-38)
        mask[0, 1 if first == 1 else 0] = False                  # (other paths where a key is out)
        check_cross(q.to(dtype), kk.to(dtype).contiguous(), vv.to(dtype).contiguous(), 1e-38, key_mask=mask)


@pytest.mark.parametrize("batch,heads,nq", [(512, 65535, 1), (1, 65535, 8192)])
def test_cross_attention_on_the_largest_grids(batch, heads, nq):
    """The most samples x heads x tokens, one key each: the result is its value.  2^25 workgroups over samples, and 2^22 of 128 rows in one."""
    print(f"cross_attn batch={batch} heads={heads} q={nq}", flush=True)
    g = gen(29)
    v = torch.randn(batch, 1, heads, 16, generator=g, device=DEV, dtype=torch.bfloat16)
    q = torch.ones(1, 1, 1, 16, device=DEV, dtype=torch.bfloat16).expand(batch, nq, heads, 16)
    out = B.cross_attn(q, v, v, 0.25)
    for at in range(0, nq, 1024):
        part = out[:, at:at + 1024]
        assert torch.equal(part, v.expand_as(part))


# ------------------------------------------------------------------------------------------------- 8-bit products
@pytest.mark.parametrize("rows,n_out,k", [s for shapes in PRODUCTS.values() for s in shapes])
@pytest.mark.parametrize("act", [0, 1])
def test_products_of_every_tile(rows, n_out, k, act):
    """The bounds of test_product_of_blocks; what lies behind the last row stays; a row has the same bits on the tiles of few rows."""
    print(f"dit_linear_fp8 {rows}x{n_out}x{k} act={act}", flush=True)
    g = gen(rows + n_out + k)
    a, a_scale = B.fp8_quantize(randn(g, rows, k) * torch.exp(2 * randn(g, rows, 1)) * torch.exp(randn(g, k)))
    w, w_scale = B.fp8_quantize(randn(g, n_out, k) / math.sqrt(k))
    bias = randn(g, n_out)
    buf = torch.full((rows + 3, n_out), 5.0, dtype=torch.bfloat16, device=DEV)
    out = B.dit_linear_fp8(a, a_scale, w, w_scale, bias, act=act, out=buf[:rows], use_workspace=False)
    ref, off = fp8_ref(a, a_scale, w, w_scale, bias, act)
    tol = 1.13 * off + U[torch.bfloat16] * ref.abs() + (2.0 ** -20 * (ref.abs() + 1.0) if act else 0.0) + 1e-30
    assert bool(((out.double() - ref).abs() <= tol).all()), float(((out.double() - ref).abs() / tol).max())
    assert bool((buf[rows:] == 5.0).all())
    few = min(rows, 48)
    assert torch.equal(B.dit_linear_fp8(a[-few:], scales_of_last(a_scale, rows, few), w, w_scale, bias, act=act, use_workspace=False), out[-few:])


def scales_of_last(scale, rows, few):
    """The scales of the last `few` rows as an operand of their own: [blocks, few rounded up to 16], filled up with zeros."""
    s = torch.zeros(scale.shape[0], (few + 15) // 16 * 16, dtype=torch.uint8, device=DEV)
    s[:, :few] = scale.view(torch.uint8)[:, rows - few:rows]
    return s.view(scale.dtype)


# ------------------------------------------------------------------------------------------------- group norm
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off,channels", [(3, 256), (1, 324)])
def test_group_norm_of_slices_on_no_border_beyond_the_caches(dtype, off, channels):
    """Results over 32 MB, which are stored past L2, from and into channel slices at odd elements: loads and stores of 8 and 4 channels."""
    positions = 70200
    g = gen(28)
    wide = torch.full((1, positions + 1, channels + 5), 9.0, dtype=dtype, device=DEV)
    x = randn(g, 1, positions, channels + 7).to(dtype)[:, :, off:off + channels]
    gamma, beta = randn(g, channels + 1)[1:], randn(g, channels + 1)[1:]
    got = check_gnorm(x, 4, gamma, beta, act=2, out=wide[:, :-1, off:off + channels])
    rest = torch.ones_like(wide, dtype=torch.bool)
    rest[:, :-1, off:off + channels] = False
    assert bool((wide[rest] == 9.0).all())
    assert torch.equal(got, B.group_norm(x.contiguous(), 4, gamma.clone(), beta.clone(), act=2))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_outputs_that_interleave(dtype):
    """Samples between the heads of a token, tokens between samples, positions between samples: no overlap, and every other value stays."""
    g = gen(30)
    q, k = randn(g, 2, 70, 4, 64).to(dtype), randn(g, 2, 90, 4, 64).to(dtype)
    for strides in ((64, 640, 160), (64, 128, 2 * 70 * 64), (4 * 64, 2 * 4 * 64, 64)):
        buf = torch.full((2 * 70 * 640,), 7.0, dtype=dtype, device=DEV)
        out = buf.as_strided((2, 70, 4, 64), (*strides, 1))
        check_cross(q, k, k, 0.125, out=out)
        kept = out.clone()
        out.fill_(7.0)
        assert bool((buf == 7.0).all())
        assert torch.equal(kept, B.cross_attn(q, k, k, 0.125))
    x = randn(g, 2, 300, 64).to(dtype)
    for strides in ((96, 160), (64, 128)):
        buf = torch.full((300 * 160 + 200,), 7.0, dtype=dtype, device=DEV)
        out = buf.as_strided((2, 300, 64), (*strides, 1))
        check_gnorm(x, 8, out=out)
        kept = out.clone()
        out.fill_(7.0)
        assert bool((buf == 7.0).all())
        assert torch.equal(kept, B.group_norm(x, 8))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq,nk", SIZES)
def test_cross_attention_of_the_largest_scale(dtype, nq, nk):
    """Scores of 0 to 3 under a scale of 2^127, from queries of 2^-60 and keys of 2^-67 times small whole numbers (exact products)."""
    g = gen(31)
    q, k = torch.zeros(1, nq, 2, 64, device=DEV), torch.zeros(1, nk, 2, 64, device=DEV)
    q[..., 3] = 2.0 ** -60 * torch.randint(0, 2, (1, nq, 2), generator=g, device=DEV)
    k[..., 3] = 2.0 ** -67 * torch.randint(0, 4, (1, nk, 2), generator=g, device=DEV)
    check_cross(q.to(dtype), k.to(dtype), randn(g, 1, nk, 2, 64).to(dtype), 2.0 ** 127)


# ------------------------------------------------------------------------------------------------- the largest sizes
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq", [1, 40])
def test_cross_attention_over_the_most_keys(dtype, nq):
    """2^24 keys of equal scores, values 0 and 1: every sum is a whole number up to 2^24, exact in fp32, so the result is their quotient, rounded;
    with a length that ends inside a tile and garbage behind it."""
    nk = 1 << 24
    g = gen(32)
    q, k = torch.zeros(1, nq, 1, 16, dtype=dtype, device=DEV), torch.ones(1, 1, 1, 16, dtype=dtype, device=DEV).expand(1, nk, 1, 16)
    v = torch.randint(0, 2, (1, nk, 1, 16), generator=g, device=DEV, dtype=torch.int8).to(dtype)
    for n in (nk, nk - 37):
        v[:, n:] = NAN
        out = B.cross_attn(q, k, v, 1.0, kv_lens=torch.tensor([n], dtype=torch.int32, device=DEV))
        want = v[0, :n, 0].sum(0, dtype=torch.float64) / n
        assert bool(((out[0, :, 0].double() - want).abs() <= (U[dtype] + 4 * 2.0 ** -24) * want).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cross_attention_of_the_most_tokens(dtype):
    g = gen(33)
    q, k, v = torch.randn(1, 1 << 24, 1, 16, generator=g, device=DEV, dtype=dtype), randn(g, 1, 3, 1, 16).to(dtype), randn(g, 1, 3, 1, 16).to(dtype)
    out = B.cross_attn(q, k, v, 0.25)
    for at in (0, 1 << 23, (1 << 24) - 1000):
        ref, tol = cross_ref(q[:, at:at + 1000], k, v, 0.25, torch.ones(1, 3, dtype=torch.bool, device=DEV))
        assert bool(((out[:, at:at + 1000].double() - ref).abs() <= tol * 1.001).all())


@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("rows,n_out", [(3, 5), (70, 300)])
def test_products_of_the_most_columns(rows, n_out, use_workspace):
    """k = 2^22, values -1, 0 and 1: whole sums, exact in fp32."""
    k = 1 << 22
    g = gen(34)
    x, w = (torch.randint(-1, 2, (n, k), generator=g, device=DEV, dtype=torch.int8).float() for n in (rows, n_out))
    out = B.dit_linear_fp8(*B.fp8_quantize(x), *B.fp8_quantize(w.bfloat16()), torch.zeros(n_out, device=DEV), use_workspace=use_workspace)
    want = x.double() @ w.double().t().contiguous()
    assert bool(((out.double() - want).abs() <= U[torch.bfloat16] * want.abs()).all())


def test_products_of_the_most_rows():
    """2^24 rows of one column against one, as the operand of many rows and as that of many columns."""
    n = 1 << 24
    g = gen(35)
    x = torch.randint(-16, 17, (n, 1), generator=g, device=DEV).bfloat16()
    q, s = B.fp8_quantize(x)
    w = B.fp8_quantize(torch.full((1, 1), 3.0, device=DEV))
    assert torch.equal(B.dit_linear_fp8(q, s, *w, torch.zeros(1, device=DEV)), 3.0 * x)
    assert torch.equal(B.dit_linear_fp8(*w, q, s, torch.zeros(n, device=DEV)), (3.0 * x).t())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,positions,groups", [(1, 1, 1), (2, 3, 32), (1, 50, 1), (1, 600, 65536), (1, 40, 16384)])
def test_group_norm_of_the_most_channels(dtype, batch, positions, groups):
    print(f"group_norm {dtype} {batch}x{positions}x65536/{groups}", flush=True)
    g = gen(36)
    x = (randn(g, batch, positions, 65536) * torch.exp(randn(g, 65536)) + randn(g, 65536)).to(dtype)
    check_gnorm(x, groups, randn(g, 65536), randn(g, 65536), act=2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("positions", [20, 5000])
def test_group_norm_keeps_what_is_not_finite_in_its_group(dtype, positions):
    g = gen(37)
    x = randn(g, 2, positions, 96).to(dtype)
    want = B.group_norm(x, 12)
    for bad in (NAN, float("inf")):
        y = x.clone()
        y[1, positions - 1, 17] = bad                            # group 2 of the second sample
        out = B.group_norm(y, 12)
        spoilt = torch.zeros_like(out, dtype=torch.bool)
        spoilt[1, :, 16:24] = True
        assert bool(torch.isnan(out[spoilt]).all()) and torch.equal(out[~spoilt], want[~spoilt])


# ------------------------------------------------------------------------------------------------- together
def check_linear(x, w, bias):
    """Quantization exact, the product within its bound (see test_product_of_blocks); the result."""
    a, a_scale = check_quantize(x)
    ref, off = fp8_ref(a, a_scale, *w, bias, 0)
    out = B.dit_linear_fp8(a, a_scale, *w, bias)
    assert bool(((out.double() - ref).abs() <= off + U[torch.bfloat16] * ref.abs() + 1e-30).all())
    return out


def test_a_conditioned_block_step_by_step():
    """Each operator on what the one before it gave, within its own bound; the block in one go has the same bits."""
    x, states, lens, p, _ = block_data(38)
    Bn, N, D = x.shape
    L, heads = states.shape[1], 5
    h = check_gnorm(x, 32, p["gamma"], p["beta"], act=2)
    q = check_linear(h.view(Bn * N, D), p["wq"], p["bq"]).view(Bn, N, heads, D // heads)
    kv = check_linear(states.view(Bn * L, -1), p["wkv"], p["bkv"]).view(Bn, L, 2, heads, D // heads)
    o = check_cross(q, kv[:, :, 0], kv[:, :, 1], 1.0 / math.sqrt(D // heads), kv_lens=lens)
    y = x + check_linear(o.view(Bn * N, D), p["wo"], p["bo"]).view(Bn, N, D)
    assert torch.equal(y, conditioned_block(x, states, lens, p, heads))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq,nk", SIZES)
def test_cross_attention_of_the_smallest_scale(dtype, nq, nk):
    """Below the normal range: the weights are equal; and with scores of 2^126, which such a scale leaves as small."""
    g = gen(39)
    q, k, v = randn(g, 1, nq, 2, 64), randn(g, 1, nk, 2, 64), randn(g, 1, nk, 2, 64).to(dtype)
    for size in (1.0, 2.0 ** 59):
        check_cross((q * size).to(dtype), (k * size).to(dtype), v, 2.0 ** -149)
