"""Operators of self-attention on packed samples at the ends of their ranges: values as large as their type holds under scores that grow behind the first
keys."""
import ctypes as C
import math

import pytest
import torch

from paper_2505_14741_amd import binding as B
from test_gpu_packed_ops import DEV, U, check_packed, gen, ints, offsets, packed_ref, randn, widen
from test_packed_edges_host import PRODUCTS, WIDE_HEADS, WIDE_KEYS, WIDE_LENS

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def grown(dtype, d, nq, nk, heads, level, high, dims):
    """Keys 0 .. 31 of every 64 have the score 0, the others level / 16 in powers of two (for the scale ln 2 / 16); values of `high` in [high / 2, high] in
    the dimensions whose d % 8 lies in dims, and of order one in the others."""
    g = gen(nq + nk + level + d)
    q, k = torch.zeros(nq, heads, d, device=DEV), torch.zeros(nk, heads, d, device=DEV)
    q[..., 0] = 1.0
    k[torch.arange(nk, device=DEV) % 64 >= 32, :, 0] = float(level)
    v = randn(g, nk, heads, d)
    far = torch.isin(torch.arange(d, device=DEV) % 8, torch.tensor(dims, device=DEV))
    v[..., far] = high * (0.5 + 0.5 * torch.rand(nk, heads, int(far.sum()), generator=g, device=DEV))
    return q.to(dtype), k.to(dtype), v.to(dtype)


SCALE = math.log(2.0) / 16.0


# The largest value times the keys times 2^8 is below 2^128 in each case.  (100, 3000): 11 pieces of 256 keys and more, whose values overflow under weights of 2^16
# relative to their first keys (23 + 108 - 1 bits), so that those rows are computed again.  (200, 1500) of 60 heads: 4 pieces.  (5, 3000): two pieces of few rows.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dims", [(0, 1, 2, 3), (4, 5, 6, 7), (1,), (6,), tuple(range(8))])
@pytest.mark.parametrize("nq,nk,heads", [(100, 3000, 1), (200, 1500, 60), (5, 3000, 2)])
def test_values_that_overflow_in_some_dimensions_under_divided_keys(dtype, d, dims, nq, nk, heads):
    print(f"packed_attn {dtype} d={d} dims={dims} {nq}x{nk}x{heads}", flush=True)
    q, k, v = grown(dtype, d, nq, nk, heads, 16 * 16, 2.0 ** 108, list(dims))
    check_packed(q, k, v, SCALE, [0, nq], [0, nk])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 64, 128])
def test_values_that_overflow_under_moderate_sums(dtype, d):
    """40 keys, the last 8 with the weight 1960: sums of 2^13.9, within 2^14, times 2^114.7 are no fp32 number."""
    high = 2.0 ** 114 * 1.59375
    assert high * 40 * 256 < torch.finfo(torch.float32).max
    q, k, v = grown(dtype, d, 40, 40, 3, 175, high, [2, 5])
    v[..., 2], v[..., 5] = high, -high
    got = check_packed(q, k, v, SCALE, [0, 40])
    assert bool(torch.isfinite(got).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("nq,nk,heads,level,power", [(100, 3000, 1, 12, 108), (200, 1500, 60, 11, 109), (70, 20000, 2, 12, 105), (5, 3000, 2, 12, 108)])
def test_pieces_whose_sums_overflow_only_together(dtype, d, nq, nk, heads, level, power):
    """Each piece's sum of weights times values is below 2^128, the sum over the pieces is not."""
    print(f"packed_attn {dtype} d={d} {nq}x{nk}x{heads}", flush=True)
    assert 2.0 ** power * nk * 256 < torch.finfo(torch.float32).max
    q, k, v = grown(dtype, d, nq, nk, heads, 16 * level, 2.0 ** power, [0, 3, 4])
    check_packed(q, k, v, SCALE, [0, nq], [0, nk])


# ------------------------------------------------------------------------------------------------- capped scores
# cap * tanh(x / cap) is off by 2^-19 of |x| at most: where |x| >= cap / 4 the quotient's four roundings and the exponential's (two of 2^-23 and the angle's) count
# 8 * 2^-23 of it together at |x| = cap / 4 and less above; below it is a series.  bf16, caps of at most 256: 2^-21 of the cap, far below the weights' 2^-8.
def check_capped(q, k, v, scale, q_off, kv_off, cap, slack, **kw):
    """slack: a score's relative error beside the cap's."""
    o, _ = packed_ref(q, k, v, scale, q_off, kv_off or q_off, None, 1, False, cap, None)
    near, _ = packed_ref(q, k, v.abs(), scale, q_off, kv_off or q_off, None, 1, False, cap, None)
    got = B.packed_attn(q, k, v, scale, ints(*q_off), kv_offsets=None if kv_off is None else ints(*kv_off), cap=cap).double()
    share = q.shape[1] // k.shape[1]
    size = float(torch.stack([(q[:, h].double().abs() @ k[:, h // share].double().abs().t()).amax() for h in range(q.shape[1])]).amax()) * scale
    es = (slack + 2.0 ** -19) * size + (2.0 ** -21 * cap if q.dtype == torch.bfloat16 and cap <= 256.0 else 0.0)
    off = 2 * es + (k.shape[0] + 32) * 2.0 ** -24 + (U[q.dtype] if q.dtype == torch.bfloat16 else 0.0)
    tol = off * near + U[q.dtype] * o.abs() + 1e-37
    bad = ~((got - o).abs() <= tol * 1.001)
    assert not bad.any(), (cap, float(((got - o).abs() / tol).max()), es)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("nq,nk", [(70, None), (300, None), (3, 200), (2, 3000), (100, 3000)])
@pytest.mark.parametrize("cap", [3.0, 50.0, 256.0, 300.0, 1e4, 1e5, 1e6, 1e9, 1e30])
def test_caps_far_above_the_scores(dtype, d, nq, nk, cap):
    """Scores of order one, which such a cap leaves nearly as they are."""
    print(f"packed_attn {dtype} d={d} {nq}x{nk} cap={cap}", flush=True)
    g = gen(nq + d)
    q, k, v = randn(g, nq, 4, d).to(dtype), randn(g, nk or nq, 2, d).to(dtype), randn(g, nk or nq, 2, d).to(dtype)
    check_capped(q, k, v, 1.0 / math.sqrt(d), [0, nq], None if nk is None else [0, nk], cap, (d + 4) * 2.0 ** -24)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nq,nk", [(70, None), (3, 200), (100, 3000)])
@pytest.mark.parametrize("cap", [40.0, 256.0, 300.0, 1000.0])
def test_scores_on_both_sides_of_the_cap(dtype, nq, nk, cap):
    """Scores up to four times the cap, exact in fp32, across every branch of the function."""
    g = gen(nq)
    n = nk or nq
    q, k, v = torch.zeros(nq, 1, 64, device=DEV), torch.zeros(n, 1, 64, device=DEV), randn(g, n, 1, 64)
    q[:, 0, 0] = torch.exp2(-torch.arange(nq, device=DEV) % 9 - 1.0)              # (down to scores that the cap leaves as they are)
    k[:, 0, 0] = torch.linspace(-8.0, 8.0, n, device=DEV)[torch.randperm(n, generator=g, device=DEV)] * cap
    check_capped(q.to(dtype), k.to(dtype), v.to(dtype), 1.0, [0, nq], None if nk is None else [0, nk], cap, 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("frame,prefix", [(1, 0), (7, 5), (100, 226)])
def test_large_caps_with_frames_prefixes_and_biases(dtype, d, frame, prefix):
    """A cap above 256 has kernels of its own: lengths that end inside tiles, masks, biases, kept keys, values and keys that are not finite."""
    lens = [130, 401, 1, 0, 700]
    g = gen(frame + d)
    n = sum(lens)
    q, k, v = (randn(g, n, 2, d).to(dtype) for _ in range(3))
    slopes = torch.tensor([0.5, -0.02], device=DEV)
    prefixes = [prefix, prefix // 2, 0, 3, prefix]
    for kw in ({}, {"slopes": slopes}):
        for causal in (True, False):
            print(f"packed_attn {dtype} d={d} frame={frame} prefix={prefix} {sorted(kw)} {causal}", flush=True)
            check_packed(q, k, v, 2.0 / math.sqrt(d), offsets(lens), prefix=prefixes, frame=frame, causal=causal, cap=300.0, **kw)
            check_packed(q[:43], k, v, 2.0 / math.sqrt(d), [0, 1, 41, 41, 41, 43], offsets([1, 401, 130, 0, 700]), prefix=prefixes, frame=frame, causal=causal, cap=300.0, **kw)
        want = B.packed_attn(q, k, v, 0.2, ints(*offsets(lens)), causal=True, cap=300.0, **kw)
        kk, vv = k.clone(), v.clone()
        kk[300], vv[300] = float("nan"), float("inf")
        got = B.packed_attn(q, kk, vv, 0.2, ints(*offsets(lens)), causal=True, cap=300.0, **kw)
        assert torch.equal(got[:300], want[:300]) and torch.equal(got[531:], want[531:]) and bool(torch.isnan(got[300:531]).all())


# ------------------------------------------------------------------------------------------------- many samples with kept keys
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples", [60, 64, 65, 150])
def test_a_token_for_each_of_many_samples(dtype, samples):
    """Keys of 0 to 4096, 16 heads over 4: divided and whole ones next to each other, the same bits as alone; nothing behind the workspace is written."""
    g = gen(samples)
    nks = [(0, 1, 1279, 1280, 2048, 4096, 700)[i % 7] for i in range(samples)]
    nqs = [(1, 1, 2, 1, 0, 1, 9, 1)[i % 8] for i in range(samples)]
    q, k, v = randn(g, sum(nqs), 16, 64).to(dtype), randn(g, sum(nks), 4, 64).to(dtype), randn(g, sum(nks), 4, 64).to(dtype)
    qo, ko = offsets(nqs), offsets(nks)
    whole = check_packed(q, k, v, 0.125, qo, ko, causal=True, prefix=[5] * samples)
    for s in range(0, samples, 5):
        a, b, ka, kb = qo[s], qo[s + 1], ko[s], ko[s + 1]
        alone = B.packed_attn(q[a:b].contiguous(), k[ka:kb].contiguous(), v[ka:kb].contiguous(), 0.125, ints(0, b - a), kv_offsets=ints(0, kb - ka),
                              prefix_lens=ints(5), causal=True)
        assert torch.equal(whole[a:b], alone), s
    shape = B._PackedShape(samples, sum(nqs), sum(nks), 16, 4, 64, B._CODE[dtype], 1, 1, 1, 0.125, 0.0, 1024, 64, 256, 64, 256, 64, 1024, 64)
    n = B.lib().packed_attn_workspace_bytes(C.byref(shape))
    ws = torch.full((n + 65536,), 77, dtype=torch.uint8, device=DEV)
    prefix = ints(*[5] * samples)
    fall = ints(*[0, sum(nqs)] * (samples // 2 + 1))[:samples + 1].contiguous(), ints(*[0, sum(nks)] * (samples // 2 + 1))[:samples + 1].contiguous()
    for dq, dk in ((ints(*qo), ints(*ko)), fall):
        out = torch.empty_like(q)
        rc = B.lib().packed_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), dq.data_ptr(), dk.data_ptr(), prefix.data_ptr(), None, out.data_ptr(), C.byref(shape),
                                 ws.data_ptr(), n, B._stream())
        torch.cuda.synchronize()
        assert rc == 0 and bool((ws[n:] == 77).all())
        assert dq is fall[0] or torch.equal(out, whole)


# ------------------------------------------------------------------------------------------------- blocks of 256 rows
def check_wide(q, k, v, scale, kv_lens, each=None, **kw):
    """The call, in blocks of 256 rows, against 64 bits, and each sample's bits against those of a call of its own, in blocks of 128."""
    qo, ko = offsets(WIDE_LENS), offsets(kv_lens or WIDE_LENS)
    if each is None:
        whole = check_packed(q, k, v, scale, qo, ko if kv_lens else None, **kw)
    else:
        whole = each
    call = dict(kw)
    prefix = call.pop("prefix", None)
    for s in range(len(WIDE_LENS)):
        a, b, ka, kb = qo[s], qo[s + 1], ko[s], ko[s + 1]
        alone = B.packed_attn(q[a:b].contiguous(), k[ka:kb].contiguous(), v[ka:kb].contiguous(), scale, ints(0, b - a), kv_offsets=ints(0, kb - ka) if kv_lens else None,
                              prefix_lens=None if prefix is None else ints(prefix[s]), **call)
        assert torch.equal(whole[a:b].view(torch.int16), alone.view(torch.int16)), (s, kw)


def wide_data(d, kv_lens, seed):
    g = gen(seed + d)
    n, m = sum(WIDE_LENS), sum(kv_lens or WIDE_LENS)
    return g, randn(g, n, WIDE_HEADS, d).bfloat16(), randn(g, m, WIDE_HEADS, d).bfloat16(), randn(g, m, WIDE_HEADS, d).bfloat16()


@pytest.mark.parametrize("d", [16, 32, 64])
@pytest.mark.parametrize("kv_lens", [None, WIDE_KEYS])
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_wide_blocks(d, kv_lens, cap):
    """Masks, prefixes, frames shorter and longer than a tile, biases, capped scores, kept keys in pieces."""
    _, q, k, v = wide_data(d, kv_lens, 1)
    slopes = torch.linspace(-0.01, 0.4, WIDE_HEADS, device=DEV)
    prefix = [i * 23 % 90 for i in range(len(WIDE_LENS))]
    for kw in ({}, {"causal": True}, {"causal": True, "frame": 7, "prefix": prefix}, {"causal": True, "frame": 100, "prefix": prefix}, {"slopes": slopes},
               {"slopes": slopes, "causal": True, "frame": 9, "prefix": prefix}, {"slopes": slopes, "causal": True, "frame": 130, "prefix": prefix}, {"slopes": slopes, "frame": 64}):
        print(f"packed_attn wide d={d} own={kv_lens is not None} cap={cap} {sorted(kw)} frame={kw.get('frame')}", flush=True)
        check_wide(q, k, v, 1.0 / math.sqrt(d), kv_lens, cap=cap, **kw)


@pytest.mark.parametrize("d", [16, 32, 64])
@pytest.mark.parametrize("kv_lens", [None, WIDE_KEYS])
def test_wide_blocks_of_rows_that_are_computed_again(d, kv_lens):
    """Scores of hundreds in some rows only, values that overflow under scores that grow, values and keys that are not finite."""
    g, q, k, v = wide_data(d, kv_lens, 2)
    loud = q.clone()
    loud[::3] *= 60.0
    check_wide(loud, k, v, 1.0 / math.sqrt(d), kv_lens)
    check_wide(loud, k, v, 1.0 / math.sqrt(d), kv_lens, causal=True, frame=40)
    qq, kk, vv = torch.zeros_like(q), torch.zeros_like(k), v.clone()
    qq[..., 0] = 1.0
    kk[torch.arange(k.shape[0], device=DEV) % 64 >= 32, :, 0] = 256.0
    vv[..., [3, 6]] = (2.0 ** 107 * (0.5 + 0.5 * torch.rand(k.shape[0], WIDE_HEADS, 2, generator=g, device=DEV))).bfloat16()
    check_wide(qq, kk, vv, SCALE, kv_lens)
    qo, ko = offsets(WIDE_LENS), offsets(kv_lens or WIDE_LENS)
    kk, vv = k.clone(), v.clone()
    at = [ko[7] + 300, ko[2] + 40, ko[10] + 129]
    kk[at[0]], vv[at[1], :, 2], vv[at[2], :, 1] = float("nan"), float("inf"), float("nan")
    args = {"causal": True, "frame": 11}
    dk = ints(*ko) if kv_lens else None
    want = B.packed_attn(q, k, v, 0.2, ints(*qo), kv_offsets=dk, **args)
    got = B.packed_attn(q, kk, vv, 0.2, ints(*qo), kv_offsets=dk, **args)
    check_wide(q, kk, vv, 0.2, kv_lens, each=got, **args)
    for s in range(len(WIDE_LENS)):
        if s not in (7, 2, 10):
            assert torch.equal(got[qo[s]:qo[s + 1]], want[qo[s]:qo[s + 1]])
    exact, tol = packed_ref(q, k, v, 0.2, qo, ko, None, 11, True, 0.0, None)
    for s, key, dim in ((7, 300, None), (2, 40, 2), (10, 129, 1)):
        nq, nk = WIDE_LENS[s], (kv_lens or WIDE_LENS)[s]
        pos = torch.arange(nk - nq, nk, device=DEV)
        sees = torch.div(pos, 11, rounding_mode="floor") >= key // 11
        part, ref = got[qo[s]:qo[s + 1]], want[qo[s]:qo[s + 1]]
        assert torch.equal(part[~sees], ref[~sees])
        assert not torch.isfinite(part[sees] if dim is None else part[sees][..., dim]).any()
        if dim is not None:
            # (a row whose sum is above 2^8 is computed again, so with another reference, as for values that overflow: other roundings of the same weights)
            rest = [i for i in range(d) if i != dim]
            far = (part.double() - exact[qo[s]:qo[s + 1]]).abs() <= tol[qo[s]:qo[s + 1]] * 1.001
            assert bool(far[sees][..., rest].all())


# ------------------------------------------------------------------------------------------------- 4-bit product
# K products and a bias summed in fp32; GELU's slope is below 1.13, its own arithmetic good for 2^-20 of its argument
@pytest.mark.parametrize("shape,tile", PRODUCTS)
def test_product_of_4_bit_blocks_on_every_tile(shape, tile):
    rows, n_out, k = shape
    print(f"dit_linear_fp4 {rows}x{n_out}x{k} tile {tile}", flush=True)
    g = gen(rows + n_out + k)
    a = B.fp4_quantize(randn(g, rows, k) * torch.exp(2 * randn(g, rows, 1)) * torch.exp(randn(g, k)))
    w = B.fp4_quantize(randn(g, n_out, k) / math.sqrt(k))
    bias = randn(g, n_out)
    A, W = widen(*a), widen(*w).t().contiguous()
    y = A @ W + bias.double()
    off = (k + 16) * 2.0 ** -24 * (A.abs() @ W.abs() + bias.double().abs())
    for act in (0, 1):
        ref = torch.nn.functional.gelu(y, approximate="tanh") if act else y
        tol = 1.13 * off + U[torch.bfloat16] * ref.abs() + (2.0 ** -20 * (ref.abs() + 1.0) if act else 0.0) + 1e-30
        err = (B.dit_linear_fp4(*a, *w, bias, act=act).double() - ref).abs()
        assert bool((err <= tol).all()), (act, float((err / tol).max()))
