"""Operators of self-attention on packed samples at the ends of their ranges: values as large as their type holds under scores that grow behind the first
keys."""
import math

import pytest
import torch

from test_gpu_packed_ops import DEV, check_packed, gen, randn

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
