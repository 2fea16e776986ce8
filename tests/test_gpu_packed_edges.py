"""Operators of self-attention on packed samples at the ends of their ranges: values as large as their type holds under scores that grow behind the first
keys."""
import ctypes as C
import math

import pytest
import torch

from paper_2505_14741_amd import binding as B
from test_gpu_packed_ops import DEV, U, check_packed, gen, ints, offsets, packed_ref, randn

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
