"""Operators of a conditioned predictor block against plain forms in 64 bits: cross attention, 8-bit quantization and product, group
norm, and a run of them together.  Bounds count roundings: half a step is 2^-8 of a value in bf16 and 2^-24 in fp32; an fp32 sum of n
terms is off by n * 2^-24 of the sum of their magnitudes at most."""
import math

import pytest
import torch

from paper_2505_14741_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
NAN = float("nan")


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


# ------------------------------------------------------------------------------------------------- cross attention
def cross_ref(q, k, v, scale, counts):
    """(output, bound of its error): 64 bits; counts [B, Nk] says which keys count."""
    Bn, N, H, d = q.shape
    share = H // k.shape[2]
    o = torch.zeros(Bn, N, H, d, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(o)
    u = U[q.dtype]
    for b in range(Bn):
        at = counts[b].nonzero()[:, 0]
        if not len(at):
            continue
        for h in range(H):
            qq, kk, vv = q[b, :, h].double(), k[b, at, h // share].double(), v[b, at, h // share].double()
            s = qq @ kk.t().contiguous() * scale
            p = torch.softmax(s, 1)
            o[b, :, h] = p @ vv
            spread = p @ vv.abs()
            # a score's products are summed in fp32, and it is multiplied and subtracted from the reference once more
            es = (d + 4) * 2.0 ** -24 * (qq.abs() @ kk.abs().t().contiguous()).amax(1, keepdim=True) * scale
            rounding = 2 * es + (len(at) + 32) * 2.0 ** -24 + (u if q.dtype == torch.bfloat16 else 0.0)      # probabilities in bf16
            tol[b, :, h] = rounding * spread + u * o[b, :, h].abs() + 1e-37
    return o, tol


def check_cross(q, k, v, scale, kv_lens=None, key_mask=None, out=None):
    counts = torch.ones(q.shape[0], k.shape[1], dtype=torch.bool, device=q.device)
    if kv_lens is not None:
        counts &= torch.arange(k.shape[1], device=q.device) < kv_lens[:, None]
    if key_mask is not None:
        counts &= key_mask != 0
    got = B.cross_attn(q, k, v, scale, kv_lens=kv_lens, key_mask=key_mask, out=out)
    ref, tol = cross_ref(q, k, v, scale, counts)
    bad = ~((got.double() - ref).abs() <= tol * 1.001)
    assert not bad.any(), (float((got.double() - ref).abs().max()), int(bad.sum()), bad.nonzero()[:4].tolist())
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 300), (5, 15), (63, 64), (64, 65), (65, 16), (257, 129), (130, 700), (3, 5000)])
def test_cross_attention_lengths_and_head_dims(dtype, d, nq, nk):
    print(f"cross_attn {dtype} d={d} q={nq} k={nk}", flush=True)
    g = gen(nq * 1000 + nk + d)
    q, k, v = (randn(g, 2, n, 3, d).to(dtype) for n in (nq, nk, nk))
    check_cross(q, k, v, 1.0 / math.sqrt(d))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,kv_heads", [(6, 1), (6, 2), (10, 2), (4, 4)])
def test_cross_attention_shared_key_heads(dtype, heads, kv_heads):
    g = gen(heads * 10 + kv_heads)
    for nq, nk in ((1, 77), (33, 200), (29, 2100)):
        print(f"cross_attn {dtype} heads={heads}/{kv_heads} q={nq} k={nk}", flush=True)
        q, k, v = randn(g, 2, nq, heads, 64).to(dtype), randn(g, 2, nk, kv_heads, 64).to(dtype), randn(g, 2, nk, kv_heads, 64).to(dtype)
        check_cross(q, k, v, 0.125)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("nq,nk", [(1, 130), (20, 226), (300, 226), (7, 3000)])
def test_cross_attention_masks_with_garbage_behind_them(dtype, d, nq, nk):
    """Lengths 0, 1, in the middle of a tile and whole, masks that leave nothing, one key, and whole tiles out; NaN, infinities and
    the type's extremes lie in keys that do not count."""
    print(f"cross_attn masked {dtype} d={d} q={nq} k={nk}", flush=True)
    g = gen(nq + nk + d)
    Bn = 7
    q, k, v = (randn(g, Bn, n, 2, d).to(dtype) for n in (nq, nk, nk))
    lens = torch.tensor([0, 1, nk // 2, nk, nk, nk, nk + 5], dtype=torch.int32, device=DEV)     # (past the end: clamped)
    mask = torch.rand(Bn, nk, generator=g, device=DEV) < 0.7
    mask[1] = True
    mask[3] = False                                              # nothing counts
    mask[4] = False
    mask[4, nk - 1] = True                                       # the last key alone
    mask[5] = True
    mask[5, 64:128] = False                                      # a whole tile out
    counts = mask & (torch.arange(nk, device=DEV) < lens[:, None])
    junk = torch.tensor([NAN, float("inf"), -float("inf"), torch.finfo(dtype).max, torch.finfo(dtype).min], device=DEV).to(dtype)
    fill = junk[torch.randint(0, 5, (Bn, nk, 2, d), generator=g, device=DEV)]
    k, v = (torch.where(counts[:, :, None, None], t, fill) for t in (k, v))
    got = check_cross(q, k, v, 1.0 / math.sqrt(d), kv_lens=lens, key_mask=mask)
    assert bool((got[0] == 0).all()) and bool((got[3] == 0).all())
    check_cross(q[:3], k[:3], v[:3], 1.0 / math.sqrt(d), kv_lens=lens[:3], key_mask=mask[:3].to(torch.uint8) * 255)
    # one mask for all samples, and negative lengths (clamped to 0)
    one = torch.arange(nk, device=DEV) % 3 != 1
    kk, vv = (torch.where(one[None, :, None, None], randn(g, Bn, nk, 2, d).to(dtype), torch.full((), NAN, dtype=dtype, device=DEV)) for _ in "kv")
    check_cross(q, kk, vv, 1.0 / math.sqrt(d), key_mask=one[None].expand(Bn, nk))
    assert bool((B.cross_attn(q, kk, vv, 0.5, kv_lens=torch.full((Bn,), -3, dtype=torch.int32, device=DEV)) == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cross_attention_of_many_tokens(dtype):
    """Half a million query rows; the last ones as in a call of their own (from a multiple of the rows of a workgroup on)."""
    n, cut = (1 << 19) + 7, 384 * 1365
    g = gen(22)
    q, k, v = randn(g, 1, n, 1, 64).to(dtype), randn(g, 1, 77, 1, 64).to(dtype), randn(g, 1, 77, 1, 64).to(dtype)
    out = B.cross_attn(q, k, v, 0.125)
    check_cross(q[:, cut:], k, v, 0.125)
    assert torch.equal(out[:, cut:], B.cross_attn(q[:, cut:], k, v, 0.125))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cross_attention_empty_extents(dtype):
    many = torch.ones(2, 300, 2, 32, dtype=dtype, device=DEV)
    assert bool((B.cross_attn(many, many[:, :0], many[:, :0], 0.2) == 0).all())
    some = B.cross_attn(many, many[:, :40], many[:, :40], 0.2, kv_lens=torch.tensor([0, 40], dtype=torch.int32, device=DEV))
    assert bool((some[0] == 0).all()) and bool((some[1] == 1).all())
    q = torch.ones(2, 5, 2, 32, dtype=dtype, device=DEV)
    none = torch.empty(2, 0, 2, 32, dtype=dtype, device=DEV)
    assert bool((B.cross_attn(q, none, none, 0.2) == 0).all())
    assert B.cross_attn(q[:, :0], q, q, 0.2).shape == (2, 0, 2, 32)
    assert B.cross_attn(q[:0], q[:0], q[:0], 0.2).shape == (0, 5, 2, 32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq", [3, 70])
def test_cross_attention_large_scores(dtype, nq):
    """Scores of thousands, growing, falling and in any order along the keys: the reference of the exponents moves or not."""
    g = gen(5)
    nk = 400
    for order in ("up", "down", "any"):
        q = randn(g, 1, nq, 2, 64).to(dtype)
        size = torch.linspace(0.1, 60.0, nk, device=DEV)
        size = size.flip(0) if order == "down" else size[torch.randperm(nk, generator=g, device=DEV)] if order == "any" else size
        k = (randn(g, 1, nk, 2, 64) * size[None, :, None, None]).to(dtype)
        check_cross(q, k, randn(g, 1, nk, 2, 64).to(dtype), 1.0)
    same = torch.full((1, nk, 2, 64), 3.0, device=DEV).to(dtype)
    v = randn(g, 1, nk, 2, 64).to(dtype)
    check_cross(torch.full((1, nq, 2, 64), -9.0, device=DEV).to(dtype), same, v, 0.3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq,nk", [(5, 200), (40, 2600), (300, 200)])
def test_cross_attention_of_huge_scores(dtype, nq, nk):
    """Scores of 2^10 to 2^100 that are exact, so that the weights are: one key far ahead, wherever it stands, or two that share the first place;
    and values of 2^60 under scores that grow by 40."""
    g = gen(24)
    v = randn(g, 1, nk, 1, 64).to(dtype)
    for power in (10, 14, 24, 40, 100):
        for best in ([0], [nk - 1], [70, nk - 3], [1, 2]):
            q, k = torch.zeros(1, nq, 1, 64, device=DEV), torch.zeros(1, nk, 1, 64, device=DEV)
            q[..., 0] = 2.0 ** (power // 2)
            k[0, :, 0, 0] = 2.0 ** (power - power // 2) * (1.0 - 2.0 ** -2 * torch.rand(nk, generator=g, device=DEV).round().add(1.0))
            k[0, best, 0, 0] = 2.0 ** (power - power // 2)
            for sign in (1.0, -1.0):                             # (below zero: the best are the smallest in size)
                kk = k.clone()
                if sign < 0:
                    kk[0, :, 0, 0] = -2.0 ** (power - power // 2) * 2
                    kk[0, best, 0, 0] = -2.0 ** (power - power // 2)
                out = B.cross_attn(q.to(dtype), kk.to(dtype), v, 1.0).double()
                want = v.double()[:, best].mean(1, keepdim=True).expand_as(out)
                # (at 2^10 the others are 2^8 behind: exp(-256) of the sum)
                assert bool(((out - want).abs() <= 2 * U[dtype] * v.double()[:, best].abs().mean(1, keepdim=True) + 1e-6).all()), (power, best, sign)
    q, k = torch.zeros(1, nq, 1, 64, device=DEV), torch.zeros(1, nk, 1, 64, device=DEV)
    q[..., 0], k[0, 64:, 0, 0] = 1.0, 40.0
    big = (v.float() * 2.0 ** 60).to(dtype)
    check_cross(q.to(dtype), k.to(dtype), big, 1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq,nk", [(5, 200), (40, 2600), (300, 200)])
def test_cross_attention_of_a_tiny_scale(dtype, nq, nk):
    g = gen(25)
    check_cross(*(randn(g, 1, n, 1, 64).to(dtype) for n in (nq, nk, nk)), 1e-38)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cross_attention_strides(dtype):
    """Halves of one projection, head-major tensors, operands that samples and heads share, an output inside a wider one whose other
    values stay."""
    g = gen(6)
    for nq, nk in ((70, 90), (2, 1500)):
        print(f"cross_attn strides {dtype} q={nq} k={nk}", flush=True)
        kv = randn(g, 3, nk, 2, 4, 64).to(dtype)
        q = randn(g, 3, 4, nq, 64).to(dtype).permute(0, 2, 1, 3)
        wide = torch.full((3, nq + 2, 6, 64), 7.0, dtype=dtype, device=DEV)
        check_cross(q, kv[:, :, 0], kv[:, :, 1], 0.125, out=wide[:, 1:-1, 1:5])
        rest = torch.ones_like(wide, dtype=torch.bool)
        rest[:, 1:-1, 1:5] = False
        assert bool((wide[rest] == 7.0).all())
        check_cross(q, kv[:1, :, 0].expand(3, nk, 4, 64), kv[:, :, 1, :1].expand(3, nk, 4, 64), 0.125)
        # what lies beyond the keys is not read into the result
        pool = torch.full((3, nk + 64, 4, 64), NAN, dtype=dtype, device=DEV)
        pool[:, :nk] = kv[:, :, 0]
        check_cross(q, pool[:, :nk], kv[:, :, 1], 0.125)


def test_cross_attention_offsets_beyond_32_bits():
    """Keys 2^20 elements apart: the last ones lie 5.9 GB behind the first."""
    nk, step = 2800, 1 << 20
    big = torch.zeros(nk * step, dtype=torch.bfloat16, device=DEV)
    g = gen(7)
    k, v = (big.as_strided((1, nk, 2, 64), (0, step, 64, 1), off) for off in (0, 128))
    k.copy_(randn(g, 1, nk, 2, 64))
    v.copy_(randn(g, 1, nk, 2, 64))
    q = randn(g, 1, 40, 2, 64).bfloat16()
    check_cross(q, k, v, 0.125)
    out = big.as_strided((1, 40, 2, 64), (0, 70 * step, 64, 1), 256)
    check_cross(q, k.contiguous(), v.contiguous(), 0.125, out=out)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nq,nk", [(1, 226), (40, 3000), (500, 226)])
def test_cross_attention_of_a_batch_equals_its_samples(dtype, nq, nk):
    g = gen(8)
    q, k, v = (randn(g, 5, n, 4, 64).to(dtype) for n in (nq, nk, nk))
    lens = torch.tensor([nk, nk // 3, 7, nk - 1, 0], dtype=torch.int32, device=DEV)
    whole = B.cross_attn(q, k, v, 0.125, kv_lens=lens)
    for b in range(5):
        assert torch.equal(whole[b:b + 1], B.cross_attn(q[b:b + 1], k[b:b + 1], v[b:b + 1], 0.125, kv_lens=lens[b:b + 1]))
    assert torch.equal(whole, B.cross_attn(q, k, v, 0.125, kv_lens=lens))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,heads,kv_heads", [(16, 3, 3), (32, 4, 2), (64, 2, 2), (64, 3, 1), (128, 2, 2)])
def test_cross_attention_many_rows(dtype, d, heads, kv_heads):
    """Rows enough to go over the keys again and again, key counts around whole tiles and around what a workgroup can hold, masks that
    leave nothing in the first tile or at all, scores that grow far beyond the first tile's."""
    g = gen(d + heads)
    for nq, nk in ((300, 1), (256, 64), (257, 65), (700, 226), (1111, 256), (300, 257), (431, 448), (333, 832)):
        print(f"cross_attn {dtype} d={d} heads={heads}/{kv_heads} q={nq} k={nk}", flush=True)
        q, k, v = randn(g, 4, nq, heads, d).to(dtype), randn(g, 4, nk, kv_heads, d).to(dtype), randn(g, 4, nk, kv_heads, d).to(dtype)
        mask = torch.rand(4, nk, generator=g, device=DEV) < 0.8
        mask[0] = True
        mask[1, :64] = False
        mask[2] = False
        lens = torch.tensor([nk, nk, nk, (nk + 1) // 2], dtype=torch.int32, device=DEV)
        check_cross(q, k, v, 1.0 / math.sqrt(d))
        check_cross(q, k, v, 1.0 / math.sqrt(d), kv_lens=lens, key_mask=mask)
        steep = (k.float() * torch.linspace(0.01, 150.0, nk, device=DEV)[None, :, None, None]).to(dtype)
        check_cross(q, steep, v, 1.0, kv_lens=lens)
        check_cross(q, steep.flip(1), v, 1.0, kv_lens=lens)
        whole = B.cross_attn(q, k, v, 0.2, kv_lens=lens, key_mask=mask)
        for b in range(4):
            assert torch.equal(whole[b:b + 1], B.cross_attn(q[b:b + 1], k[b:b + 1], v[b:b + 1], 0.2, kv_lens=lens[b:b + 1], key_mask=mask[b:b + 1]))


# ------------------------------------------------------------------------------------------------- 8-bit blocks
def quantize_ref(x):
    """(values q, scales) in 64 bits from the definition."""
    rows, cols = x.shape
    blocks = (cols + 127) // 128
    v = torch.zeros(rows, blocks * 128, dtype=torch.float64, device=x.device)
    v[:, :cols] = x.double()
    v = v.view(rows, blocks, 128)
    top = torch.where(torch.isfinite(v), v.abs(), 0.0).amax(2)
    s = torch.full_like(top, 2.0 ** -127)
    for e in range(-127, 121):                                   # the least power of two that reaches
        s = torch.where(top > 448.0 * 2.0 ** e, 2.0 ** (e + 1), s)
    y = v / s[:, :, None]
    finite = torch.isfinite(y)
    a = torch.where(finite, y.abs(), 0.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3.0)
    q = torch.round(a / step) * step * torch.sign(y)
    return torch.where(finite, q, NAN).view(rows, -1), s


def check_quantize(x):
    q, scale = B.fp8_quantize(x)
    rq, rs = quantize_ref(x)
    rows = x.shape[0]
    assert q.shape == rq.shape and scale.shape == (rs.shape[1], (rows + 15) // 16 * 16)
    assert torch.equal(scale[:, :rows].double().t(), rs)
    assert bool((scale.view(torch.uint8)[:, rows:] == 0).all())
    assert torch.equal(torch.nan_to_num(q.double(), nan=999.0), torch.nan_to_num(rq, nan=999.0))
    return q, scale


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 127), (17, 129), (16, 1920), (33, 1000), (257, 77), (5, 4100)])
def test_quantize_is_exact(dtype, rows, cols):
    print(f"fp8_quantize {dtype} {rows}x{cols}", flush=True)
    g = gen(rows * cols)
    x = (randn(g, rows, cols) * torch.exp(3 * randn(g, rows, 1))).to(dtype)
    check_quantize(x)
    check_quantize(x * 2.0 ** 100)
    check_quantize(x * 2.0 ** -120)                              # below the normal range in fp32
    wide = torch.full((rows, cols + 3), NAN, dtype=dtype, device=DEV)      # rows that no vector load can take
    wide[:, 1:1 + cols] = x
    check_quantize(wide[:, 1:1 + cols])


def test_quantize_at_the_edges_of_the_format():
    """Values next to 448 times a power of two, ties, zeros, subnormal results, infinities and NaN."""
    vals = [0.0, -0.0, 448.0, 448.0001, 447.99, 256.0, 464.0, 480.0, 512.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, -448.0, 0.4375]
    x = torch.zeros(len(vals) + 6, 256, device=DEV)
    for i, t in enumerate(vals):
        x[i, 0], x[i, 1], x[i, 130] = t, 448.0, t
    x[-1, 3], x[-1, 200] = float("inf"), NAN
    x[-2, :128] = float("inf")
    x[-3, 5], x[-3, 6] = -float("inf"), 3.0e38
    x[-4] = 2.0 ** -149
    x[-5] = torch.linspace(-500, 500, 256, device=DEV)
    x[-6] = torch.finfo(torch.float32).max
    check_quantize(x)
    check_quantize(x.bfloat16())
    assert B.fp8_quantize(x[:0])[0].shape == (0, 256)


def fp8_ref(a, a_scale, w, w_scale, bias, act):
    def wide(q, s):
        return (q.double().view(q.shape[0], -1, 128) * s[:, :q.shape[0]].double().t()[:, :, None]).view(q.shape)
    A, W = wide(a, a_scale), wide(w, w_scale)
    Wt = W.t().contiguous()
    y = A @ Wt + bias.double()
    # of 8 adjacent products, the instruction cuts the 7 smaller ones at 2^-13 of the largest (or of more: the largest of each operand)
    cut = 7 * 2.0 ** -13 * A.abs().view(A.shape[0], -1, 8).amax(2) @ W.abs().view(W.shape[0], -1, 8).amax(2).t().contiguous()
    size = A.abs() @ Wt.abs() + bias.double().abs()
    return (torch.nn.functional.gelu(y, approximate="tanh") if act else y), cut + (A.shape[1] + 8) * 2.0 ** -24 * size


# K products and a bias summed in fp32 behind the cut; GELU's slope is below 1.13, its own arithmetic good for 2^-20 of its argument
@pytest.mark.parametrize("rows,n_out,k", [(1, 1, 1), (1, 1920, 1920), (2, 63, 100), (15, 64, 128), (16, 65, 129), (17, 5760, 256), (33, 130, 7680),
                                          (112, 1920, 7680), (64, 6, 700), (129, 257, 640), (300, 1908, 1920), (1100, 1920, 512), (2500, 2052, 300)])
@pytest.mark.parametrize("act", [0, 1])
def test_product_of_blocks(rows, n_out, k, act):
    print(f"dit_linear_fp8 {rows}x{n_out}x{k} act={act}", flush=True)
    g = gen(rows + n_out + k)
    a, a_scale = B.fp8_quantize(randn(g, rows, k) * torch.exp(2 * randn(g, rows, 1)) * torch.exp(randn(g, k)))
    w, w_scale = B.fp8_quantize(randn(g, n_out, k) / math.sqrt(k))
    bias = randn(g, n_out)
    ref, off = fp8_ref(a, a_scale, w, w_scale, bias, act)
    for kw in ({}, {"use_workspace": False}):
        out = B.dit_linear_fp8(a, a_scale, w, w_scale, bias, act=act, **kw)
        tol = 1.13 * off + U[torch.bfloat16] * ref.abs() + (2.0 ** -20 * (ref.abs() + 1.0) if act else 0.0) + 1e-30
        err = (out.double() - ref).abs()
        assert bool((err <= tol).all()), (kw, float((err / tol).max()))


def test_product_rows_do_not_depend_on_their_neighbours():
    """Summed whole, a row has the same bits in a call of its own (64 x 64 tiles) and among hundreds and thousands (the other tiles)."""
    g = gen(20)
    for n_out, k in ((1920, 1920), (516, 300)):
        a, s = B.fp8_quantize(randn(g, 4600, k))
        w, bias = B.fp8_quantize(randn(g, n_out, k)), randn(g, n_out)
        full = B.dit_linear_fp8(a, s, *w, bias, act=1, use_workspace=False)
        for rows in (16, 48, 448, 1104):
            part = B.dit_linear_fp8(a[:rows], s[:, :rows].contiguous(), *w, bias, act=1, use_workspace=False)
            assert torch.equal(part, full[:rows]), (n_out, k, rows)


def test_quantize_and_product_beyond_32_bits():
    """600000 rows of 7680: 4.6 10^9 values; the last rows as in a call of their own."""
    rows, k = 600000, 7680
    g = gen(21)
    x = randn(g, 1000, k).bfloat16().repeat(rows // 1000, 1)
    x[-100:] = randn(g, 100, k).bfloat16()
    w, bias = B.fp8_quantize(randn(g, 64, k)), randn(g, 64)
    a, s = B.fp8_quantize(x)
    b, t = B.fp8_quantize(x[-100:])
    assert torch.equal(a[-100:].view(torch.uint8), b.view(torch.uint8)) and torch.equal(s[:, -100:].contiguous().view(torch.uint8), t[:, :100].contiguous().view(torch.uint8))
    out = B.dit_linear_fp8(a, s, *w, bias, use_workspace=False)
    assert torch.equal(out[-100:], B.dit_linear_fp8(b, t, *w, bias, use_workspace=False))


def test_product_spreads_nan_along_its_row_only():
    g = gen(9)
    x, w = randn(g, 40, 300), randn(g, 70, 300)
    x[7, 299], w[11, 0] = NAN, float("inf")
    a, w8 = B.fp8_quantize(x), B.fp8_quantize(w)
    out = B.dit_linear_fp8(*a, *w8, torch.zeros(70, device=DEV))
    bad = torch.zeros(40, 70, dtype=torch.bool, device=DEV)
    bad[7], bad[:, 11] = True, True
    assert torch.equal(torch.isnan(out), bad)


def test_product_writes_its_rows_only():
    """Rows behind the last one stay as they were, at sizes that end inside a tile."""
    g = gen(10)
    for rows, n_out, k in ((5, 68, 128), (70, 30, 1000), (1, 512, 7680)):
        a, w = B.fp8_quantize(randn(g, rows, k)), B.fp8_quantize(randn(g, n_out, k))
        buf = torch.full((rows + 3, n_out), 5.0, dtype=torch.bfloat16, device=DEV)
        B.dit_linear_fp8(*a, *w, torch.zeros(n_out, device=DEV), out=buf[:rows])
        assert bool((buf[rows:] == 5.0).all())
    assert B.dit_linear_fp8(*B.fp8_quantize(randn(g, 0, 128)), *B.fp8_quantize(randn(g, 4, 128)), torch.zeros(4, device=DEV)).shape == (0, 4)


# ------------------------------------------------------------------------------------------------- group norm
def gnorm_ref(x, groups, gamma, beta, eps, act):
    b, n, ch = x.shape
    v = x.double().reshape(b, n, groups, ch // groups)
    var, mean = torch.var_mean(v, (1, 3), correction=0, keepdim=True)
    z = (v - mean) / torch.sqrt(var + eps)
    # deviations of fp32 means (roundings of the mean's own size) and of the variance, relative to the standard deviation
    rough = 2.0 ** -24 * (600.0 * mean.abs() / torch.sqrt(var + eps) + 600.0 * z.abs() + 8.0)
    z, rough = z.reshape(b, n, ch), rough.expand_as(z).reshape(b, n, ch)
    ga = torch.ones(ch, device=x.device) if gamma is None else gamma
    be = torch.zeros(ch, device=x.device) if beta is None else beta
    y = z * ga.double() + be.double()
    tol = rough * ga.double().abs() + 2.0 ** -23 * (y.abs() + be.double().abs())
    r = torch.nn.functional.gelu(y, approximate="tanh") if act == 1 else y * torch.sigmoid(y) if act == 2 else y
    return r, 1.13 * tol + 2.0 ** -20 * y.abs() * (act > 0)


def check_gnorm(x, groups, gamma=None, beta=None, eps=1e-5, act=0, out=None):
    ref, tol = gnorm_ref(x, groups, gamma, beta, eps, act)
    got = B.group_norm(x, groups, gamma, beta, eps=eps, act=act, out=out)
    err = (got.double() - ref).abs()
    assert bool((err <= tol + U[x.dtype] * ref.abs() + 1e-30).all()), float((err / (tol + U[x.dtype] * ref.abs() + 1e-30)).max())
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,positions,channels,groups", [(1, 1, 1, 1), (2, 1, 64, 32), (3, 7, 30, 3), (1, 345, 320, 32), (2, 1000, 512, 32), (1, 9000, 77, 7),
                                                             (1, 400, 2048, 1), (2, 33, 4100, 2), (1, 20000, 256, 256), (1, 5001, 96, 32), (1, 3, 1500, 500)])
@pytest.mark.parametrize("act", [0, 1, 2])
def test_group_norm(dtype, batch, positions, channels, groups, act):
    print(f"group_norm {dtype} {batch}x{positions}x{channels}/{groups} act={act}", flush=True)
    g = gen(positions + channels)
    x = (randn(g, batch, positions, channels) * torch.exp(randn(g, channels)) + randn(g, channels)).to(dtype)
    gamma, beta = randn(g, channels), randn(g, channels)
    got = check_gnorm(x, groups, gamma, beta, act=act)
    check_gnorm(x, groups, None, None, eps=1e-3, act=act)
    for b in range(batch):                                       # a sample's result does not depend on its batch
        assert torch.equal(got[b:b + 1], B.group_norm(x[b:b + 1], groups, gamma, beta, act=act))
    assert torch.equal(B.group_norm(x.clone(), groups, gamma, beta, act=act), got)
    same = x.clone()
    assert B.group_norm(same, groups, gamma, beta, act=act, out=same) is same and torch.equal(same, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_group_norm_far_means_outliers_and_constants(dtype):
    """A mean a thousand deviations away, a first value far from all others, groups without any spread."""
    g = gen(11)
    for positions in (50, 6000):
        x = (randn(g, 1, positions, 128) + 1000.0 * torch.sign(randn(g, 128))).to(dtype)
        check_gnorm(x, 128)
        check_gnorm(x, 8, act=2)
        x = randn(g, 1, positions, 128)
        x[0, 0] = 3000.0
        check_gnorm(x.to(dtype), 8)
        assert bool((check_gnorm(torch.full((1, positions, 128), 3.0, dtype=dtype, device=DEV), 8) == 0).all())


def test_group_norm_beyond_32_bits():
    """2^22 positions of 768 channels are 3.2 10^9 values: a block of 4096 positions over and over has the block's moments."""
    g = gen(23)
    block = randn(g, 1, 4096, 768).bfloat16()
    x = block.expand(1024, 4096, 768).reshape(1, 1 << 22, 768)
    out = B.group_norm(x, 32, act=2, out=x)                     # (in place)
    ref, tol = gnorm_ref(block, 32, None, None, 1e-5, 2)
    for at in (0, 1 << 21, (1 << 22) - 4096):
        err = (out[:, at:at + 4096].double() - ref).abs()
        assert bool((err <= tol + U[torch.bfloat16] * ref.abs() + 1e-30).all()), at


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_group_norm_strides(dtype):
    """A channel slice of a wider tensor into another one, a channels-first tensor's view refused, an input repeated over the batch."""
    g = gen(12)
    for off, positions in ((8, 200), (3, 9000)):                 # on 16-byte borders and not
        x = randn(g, 2, positions, 200).to(dtype)[:, :, off:off + 96]
        wide = torch.full((2, positions + 1, 130), 9.0, dtype=dtype, device=DEV)
        check_gnorm(x, 12, act=2, out=wide[:, :-1, off:off + 96])
        rest = torch.ones_like(wide, dtype=torch.bool)
        rest[:, :-1, off:off + 96] = False
        assert bool((wide[rest] == 9.0).all())
        check_gnorm(x[:1].expand(3, positions, 96), 12)
    assert B.group_norm(x[:0], 12).shape == (0, 9000, 96) and B.group_norm(x[:, :0], 12).shape == (2, 0, 96)


# ------------------------------------------------------------------------------------------------- together
def conditioned_block(x, states, lens, p, heads):
    """x [B, N, D] channels-last, states [B, L, E]: x + out(cross_attn(query(norm(x)), keys and values(states))), projections in 8 bits."""
    Bn, N, D = x.shape
    L = states.shape[1]
    h = B.group_norm(x, 32, p["gamma"], p["beta"], act=2)
    q = B.dit_linear_fp8(*B.fp8_quantize(h.view(Bn * N, D)), *p["wq"], p["bq"])
    kv = B.dit_linear_fp8(*B.fp8_quantize(states.view(Bn * L, -1)), *p["wkv"], p["bkv"]).view(Bn, L, 2, heads, D // heads)
    o = B.cross_attn(q.view(Bn, N, heads, -1), kv[:, :, 0], kv[:, :, 1], 1.0 / math.sqrt(D // heads), kv_lens=lens)
    return x + B.dit_linear_fp8(*B.fp8_quantize(o.view(Bn * N, D)), *p["wo"], p["bo"]).view(Bn, N, D)


def block_data(seed, Bn=2, N=345, D=320, L=77, E=200):
    g = gen(seed)
    mats = {"wq": randn(g, D, D) / math.sqrt(D), "wkv": randn(g, 2 * D, E) / math.sqrt(E), "wo": randn(g, D, D) / math.sqrt(D)}
    p = {n: B.fp8_quantize(m) for n, m in mats.items()}
    p.update(gamma=1 + 0.2 * randn(g, D), beta=0.2 * randn(g, D), bq=randn(g, D), bkv=randn(g, 2 * D), bo=randn(g, D))
    x, states = randn(g, Bn, N, D).bfloat16(), randn(g, Bn, L, E).bfloat16()
    lens = torch.tensor([L, L // 3], dtype=torch.int32, device=DEV)
    return x, states, lens, p, mats


def test_a_conditioned_block():
    """Against the block in 64 bits without any 8-bit rounding.  A value in e4m3 is off by 2^-4 of itself at most, 2^-4 / sqrt(3) in the
    mean square; a product of two such operands with independent errors by 0.051 of its norm.  The update is linear in wo (0.051, of which
    values already carry 0.051 from wkv) and smooth in the scores (errors of 0.051 of scores of order one): below 0.13 together."""
    x, states, lens, p, mats = block_data(13)
    heads, D = 5, 320
    got = conditioned_block(x, states, lens, p, heads).double() - x.double()
    h, _ = gnorm_ref(x, 32, p["gamma"], p["beta"], 1e-5, 2)
    q = h @ mats["wq"].double().t() + p["bq"].double()
    kv = states.double() @ mats["wkv"].double().t() + p["bkv"].double()
    q, kv = q.view(2, 345, heads, 64), kv.view(2, 77, 2, heads, 64)
    o = torch.zeros_like(q)
    for b in range(2):
        for hd in range(heads):
            n = int(lens[b])
            s = q[b, :, hd] @ kv[b, :n, 0, hd].t().contiguous() / 8.0
            o[b, :, hd] = torch.softmax(s, 1) @ kv[b, :n, 1, hd].contiguous()
    ref = o.reshape(2, 345, D) @ mats["wo"].double().t() + p["bo"].double()
    assert float((got - ref).norm() / ref.norm()) < 0.13


def test_a_captured_block_replays():
    """The block in a graph, replayed with new inputs and with eager calls between, equals the eager result each time; two graphs live."""
    data = [block_data(s) for s in (14, 15)]
    x, states, lens, p, _ = data[0]
    conditioned_block(x, states, lens, p, 5)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = conditioned_block(x, states, lens, p, 5)
        graphs.append((gr, out))
    originals = [(d[0].clone(), d[1].clone()) for d in data]
    for turn in range(4):
        nx, ns = originals[turn % 2]
        x.copy_(nx)
        states.copy_(ns)
        want = conditioned_block(x, states, lens, p, 5)
        torch.cuda.synchronize()
        for gr, out in graphs:
            out.zero_()
            gr.replay()
        conditioned_block(*data[1][:4], 5)
        torch.cuda.synchronize()
        for gr, out in graphs:
            assert torch.equal(out, want), turn


def test_block_on_two_streams_at_once():
    data = [block_data(s) for s in (16, 17)]
    want = [conditioned_block(*d[:4], 5) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    got = [[], []]
    for _ in range(3):
        for i, (d, st) in enumerate(zip(data, streams)):
            with torch.cuda.stream(st):
                got[i].append(conditioned_block(*d[:4], 5))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(t, want[i]) for t in got[i])
