"""Operators of self-attention on packed samples against plain forms in 64 bits: 4-bit quantization, reading back and product, rotary tables, norms
with rotation, packed attention, and a run of them together.  Bounds count roundings: half a step is 2^-8 of a value in bf16 and 2^-24 in
fp32; an fp32 sum of n terms is off by n * 2^-24 of the sum of their magnitudes at most."""
import math

import pytest
import torch

from paper_2505_14741_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
NAN = float("nan")
TYPES = [torch.bfloat16, torch.float32]


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------------- 4-bit blocks
def quantize_ref(x):
    """(values, scales) in 64 bits from the definition, NaN scales for blocks that are not finite."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % 128)).view(rows, -1, 32)
    top = v.abs().amax(2)
    s = torch.full_like(top, 2.0 ** -127)
    for e in range(-127, 126):                                   # the least power of two that reaches
        s = torch.where(top > 6.0 * 2.0 ** e, 2.0 ** (e + 1), s)
    y = v / s[:, :, None]
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    q = torch.zeros_like(y)
    for i in range(1, 8):                                        # ties go to the even code
        mid = (grid[i - 1] + grid[i]) / 2
        q = torch.where((y.abs() > mid) | ((y.abs() == mid) & (i % 2 == 0)), grid[i], q)
    bad = ~torch.isfinite(top)
    s = torch.where(bad, NAN, s)
    q = torch.where(bad[:, :, None], 0.0, q * torch.sign(y))
    return q.view(rows, -1), s


def check_quantize(x):
    q, scale = B.fp4_quantize(x)
    rq, rs = quantize_ref(x)
    rows, cols = x.shape
    assert q.shape == (rows, rq.shape[1] // 2) and scale.shape == (rs.shape[1], (rows + 15) // 16 * 16)
    byte = scale.view(torch.uint8)
    assert bool((byte[:, rows:] == 0).all())
    want = torch.where(torch.isnan(rs), 255.0, torch.log2(torch.nan_to_num(rs, nan=1.0)) + 127.0)
    assert torch.equal(byte[:, :rows].double().t(), want)
    code = torch.stack([q & 15, q >> 4], 2).view(rows, -1)
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)[(code & 7).long()]
    assert torch.equal(torch.where(code >= 8, -mag, mag) + 0.0, rq + 0.0)
    value = (rq.view(rows, -1, 32) * rs[:, :, None]).view(rows, -1)
    for dt in TYPES:
        for n in {cols, rq.shape[1]}:
            back = B.fp4_dequantize(q, scale, cols=n, dtype=dt)
            most = torch.finfo(dt).max                           # (fp32's largest numbers are rounded to 2^128)
            assert back.dtype == dt and torch.equal(torch.nan_to_num(back.double(), nan=1e300), torch.nan_to_num(value[:, :n].clamp(-most, most), nan=1e300))
    wide = torch.full((rows, cols + 3), 7.0, device=DEV)
    B.fp4_dequantize(q, scale, cols=cols, out=wide[:, 1:1 + cols])
    assert torch.equal(torch.nan_to_num(wide[:, 1:1 + cols].double(), nan=1e300), torch.nan_to_num(value[:, :cols].clamp(-most, most), nan=1e300))
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 1 + cols:] == 7.0).all())
    return q, scale


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 127), (17, 129), (16, 1920), (33, 1000), (257, 77), (5, 4100), (15, 512), (48, 513)])
def test_quantize_4_bit_is_exact(dtype, rows, cols):
    print(f"fp4_quantize {dtype} {rows}x{cols}", flush=True)
    g = gen(rows * cols)
    x = (randn(g, rows, cols) * torch.exp(3 * randn(g, rows, 1))).to(dtype)
    check_quantize(x)
    check_quantize(x * 2.0 ** 100)
    check_quantize(x * 2.0 ** -120)                              # below the normal range in fp32
    wide = torch.full((rows, cols + 3), NAN, dtype=dtype, device=DEV)      # rows that no vector load can take
    wide[:, 1:1 + cols] = x
    check_quantize(wide[:, 1:1 + cols])


def test_quantize_4_bit_at_the_edges_of_the_format():
    """Ties, values next to 6 times a power of two, zeros, the smallest and largest numbers, infinities and NaN."""
    x = torch.zeros(64, 256, device=DEV)
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    for i, t in enumerate(ties):
        near = torch.tensor([t], device=DEV)
        x[i, 0], x[i, 1], x[i, 2], x[i, 3], x[i, 5] = 6.0, t, torch.nextafter(near, near + 1)[0], torch.nextafter(near, near - 1)[0], -t
    for i, t in enumerate([6.0, 6.0000005, 5.9999995, 4.0, 8.0, 7.0, 12.0, 2.0 ** -126, 2.0 ** -149, 3.0e38, torch.finfo(torch.float32).max, 1.5 * 2.0 ** -126, -6.0]):
        x[8 + i, 40] = t
    x[30, 3], x[31, 200], x[32, 64:96] = float("inf"), NAN, -float("inf")
    x[33, 127], x[33, 128] = NAN, 3.0
    x[34] = torch.linspace(-9, 9, 256, device=DEV)
    check_quantize(x)
    check_quantize(x.bfloat16())
    q, s = B.fp4_quantize(x[:0])
    assert q.shape == (0, 128) and s.shape == (8, 0) and B.fp4_dequantize(q, s).shape == (0, 256)


def widen(q, scale):
    return B.fp4_dequantize(q, scale, dtype=torch.float32).double()


# K products and a bias summed in fp32 (an instruction's 128 products as exactly as that); GELU's slope is below 1.13, its own arithmetic good for 2^-20 of its argument
@pytest.mark.parametrize("rows,n_out,k", [(1, 1, 1), (1, 1920, 1920), (2, 63, 100), (15, 64, 128), (16, 65, 129), (17, 5760, 256), (33, 130, 7680), (5, 70, 300), (130, 4, 513),
                                          (112, 1920, 7680), (64, 6, 700), (129, 257, 640), (300, 1908, 1920), (1100, 1920, 512), (2500, 2052, 300), (4516, 1920, 900)])
@pytest.mark.parametrize("act", [0, 1])
def test_product_of_4_bit_blocks(rows, n_out, k, act):
    print(f"dit_linear_fp4 {rows}x{n_out}x{k} act={act}", flush=True)
    g = gen(rows + n_out + k)
    a = B.fp4_quantize(randn(g, rows, k) * torch.exp(2 * randn(g, rows, 1)) * torch.exp(randn(g, k)))
    w = B.fp4_quantize(randn(g, n_out, k) / math.sqrt(k))
    bias = randn(g, n_out)
    A, W = widen(*a), widen(*w).t().contiguous()
    y = A @ W + bias.double()
    off = (k + 16) * 2.0 ** -24 * (A.abs() @ W.abs() + bias.double().abs())
    ref = torch.nn.functional.gelu(y, approximate="tanh") if act else y
    tol = 1.13 * off + U[torch.bfloat16] * ref.abs() + (2.0 ** -20 * (ref.abs() + 1.0) if act else 0.0) + 1e-30
    for kw in ({}, {"use_workspace": False}):
        err = (B.dit_linear_fp4(*a, *w, bias, act=act, **kw).double() - ref).abs()
        assert bool((err <= tol).all()), (kw, float((err / tol).max()))


def test_4_bit_product_rows_do_not_depend_on_their_neighbours():
    """Summed whole, a row has the same bits in a call of its own and among hundreds and thousands."""
    g = gen(20)
    for n_out, k in ((1920, 1920), (516, 300), (5760, 640)):
        a, s = B.fp4_quantize(randn(g, 4600, k))
        w, bias = B.fp4_quantize(randn(g, n_out, k)), randn(g, n_out)
        full = B.dit_linear_fp4(a, s, *w, bias, act=1, use_workspace=False)
        for rows in (16, 48, 448, 1104, 2048):
            part = B.dit_linear_fp4(a[:rows], s[:, :rows].contiguous(), *w, bias, act=1, use_workspace=False)
            assert torch.equal(part, full[:rows]), (n_out, k, rows)


def test_4_bit_blocks_and_product_beyond_32_bits():
    """600000 rows of 7680: 4.6 10^9 values; the last rows as in a call of their own."""
    rows, k = 600000, 7680
    g = gen(21)
    x = randn(g, 1000, k).bfloat16().repeat(rows // 1000, 1)
    x[-100:] = randn(g, 100, k).bfloat16()
    w, bias = B.fp4_quantize(randn(g, 64, k)), randn(g, 64)
    a, s = B.fp4_quantize(x)
    b, t = B.fp4_quantize(x[-100:])
    assert torch.equal(a[-100:], b) and torch.equal(s[:, -100:].contiguous().view(torch.uint8), t[:, :100].contiguous().view(torch.uint8))
    out = B.dit_linear_fp4(a, s, *w, bias, use_workspace=False)
    assert torch.equal(out[-100:], B.dit_linear_fp4(b, t, *w, bias, use_workspace=False))
    back = B.fp4_dequantize(a, s, out=x)
    assert torch.equal(back[-100:], B.fp4_dequantize(b, t))


def test_4_bit_product_spreads_nan_along_its_row_only():
    g = gen(9)
    for k in (300, 256):
        x, w = randn(g, 40, k), randn(g, 70, k)
        x[7, k - 1], w[11, 0] = NAN, float("inf")
        out = B.dit_linear_fp4(*B.fp4_quantize(x), *B.fp4_quantize(w), torch.zeros(70, device=DEV))
        bad = torch.zeros(40, 70, dtype=torch.bool, device=DEV)
        bad[7], bad[:, 11] = True, True
        assert torch.equal(torch.isnan(out), bad)


def test_4_bit_product_writes_its_rows_only():
    g = gen(10)
    for rows, n_out, k in ((5, 68, 128), (70, 30, 1000), (1, 512, 7680), (200, 1923, 640)):
        a, w = B.fp4_quantize(randn(g, rows, k)), B.fp4_quantize(randn(g, n_out, k))
        buf = torch.full((rows + 3, n_out), 5.0, dtype=torch.bfloat16, device=DEV)
        if buf[:rows].data_ptr() % 16 == 0:
            B.dit_linear_fp4(*a, *w, torch.zeros(n_out, device=DEV), out=buf[:rows])
            assert bool((buf[rows:] == 5.0).all())
    assert B.dit_linear_fp4(*B.fp4_quantize(randn(g, 0, 128)), *B.fp4_quantize(randn(g, 4, 128)), torch.zeros(4, device=DEV)).shape == (0, 4)


# ------------------------------------------------------------------------------------------------- tables, norms and rotations
def angles(positions, dims, thetas):
    parts = []
    for a, d in enumerate(dims):
        i = torch.arange(d // 2, dtype=torch.float64, device=DEV)
        parts.append(positions[:, a].double()[:, None] / thetas[a] ** (2.0 * i / d))
    return torch.cat(parts, 1)


@pytest.mark.parametrize("dims,thetas", [((64,), (10000.0,)), ((16, 24, 24), (10000.0, 10000.0, 10000.0)), ((2, 2, 2, 2), (100.0, 1e6, 1.0, 0.5)), ((256,), (500000.0,)),
                                         ((100, 156), (10.0, 10000.0))])
def test_rope_table(dims, thetas):
    g = gen(len(dims))
    pos = torch.randint(-20000, 20000, (777, len(dims)), generator=g, device=DEV).float()
    pos[100:200] += 0.25
    pos[0], pos[1], pos[2] = 0.0, 2.0 ** 24, -(2.0 ** 24) + 1
    t = B.rope_table(pos, dims, list(thetas))
    turn = angles(pos, dims, thetas)
    ref = torch.stack([turn.cos(), turn.sin()], 2)
    # rounded once to 32 bits; the angle in 64 bits is off by a few of its last places, its frequency among them
    assert bool(((t.double() - ref).abs() <= 2.0 ** -25 + 2.0 ** -49 * turn.abs()[:, :, None] + 1e-15).all())
    assert bool((t[0, :, 0] == 1.0).all()) and bool((t[0, :, 1] == 0.0).all())
    wide = torch.full((777, len(dims) + 2), NAN, device=DEV)
    wide[:, 1:-1] = pos
    assert torch.equal(B.rope_table(wide[:, 1:-1], dims, list(thetas)), t)
    assert torch.equal(B.rope_table(pos[5:6].expand(7, len(dims)), dims, list(thetas)), t[5:6].expand(7, *t.shape[1:]))
    assert B.rope_table(pos[:0], dims).shape == (0, sum(dims) // 2, 2)
    if len(set(thetas)) == 1:
        assert torch.equal(B.rope_table(pos, dims, thetas[0]), t)


def norm_ref(x, norm, gamma, beta, eps):
    """(normalised values, bound of their error)"""
    x = x.double()
    d = x.shape[-1]
    if norm == 0:
        return x, torch.zeros_like(x)
    ga = torch.ones(d, device=DEV).double() if gamma is None else gamma.double()
    be = torch.zeros(d, device=DEV).double() if beta is None else beta.double()
    size = x.abs().mean(-1, keepdim=True)
    if norm == 2:
        x = x - x.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    z = x * r
    # sums of d terms; a mean's error counts in every deviation, and again in their squares (z is at most sqrt(d))
    off = (d + 8) * 2.0 ** -24 * z.abs() + ((d + 2) * 2.0 ** -24 * size * r * (1.0 + z.abs()) if norm == 2 else 0.0)
    return z * ga + be, off * ga.abs() + 2.0 ** -23 * ((z * ga).abs() + be.abs())


def turn_ref(y, off, table, halves):
    if table is None:
        return y, off
    t = table.double()
    t = t[None] if t.dim() == 3 else t
    n = t.shape[2]
    c, s = t[:, :, None, :, 0], t[:, :, None, :, 1]

    def turned(v, sign, c, s):
        r = v[..., :2 * n]
        a, b = (r[..., :n], r[..., n:]) if halves else (r[..., 0::2], r[..., 1::2])
        u, w = a * c - sign * b * s, a * s + sign * sign * b * c
        r = torch.cat([u, w], -1) if halves else torch.stack([u, w], -1).flatten(-2)
        return torch.cat([r, v[..., 2 * n:]], -1)
    out = turned(y, 1.0, c, s)
    mag = turned(y.abs(), -1.0, c.abs(), s.abs())                # |a cos| + |b sin|
    return out, turned(off, -1.0, c.abs(), s.abs()) + 3 * 2.0 ** -24 * mag


def check_qk(q, k, table, gq=None, gk=None, bq=None, bk=None, norm=1, eps=1e-6, halves=False, q_out=None, k_out=None):
    refs = []
    for x, ga, be in ((q, gq, bq), (k, gk, bk)):
        refs.append(None if x is None else turn_ref(*norm_ref(x, norm, ga, be, eps), table, halves))
    got = B.qk_norm_rope(q, k, table, gq, gk, bq, bk, norm=norm, eps=eps, halves=halves, q_out=q_out, k_out=k_out)
    for o, r in zip(got, refs):
        if r is None:
            assert o is None
            continue
        ref, tol = r
        tol = tol + U[o.dtype] * (ref.abs() + tol) + 1e-37
        err = (o.double() - ref).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("d,rotated,halves", [(8, 8, False), (16, 16, True), (24, 8, False), (32, 32, True), (64, 64, False), (64, 32, True), (72, 64, True), (96, 96, True),
                                              (104, 0, False), (128, 120, False), (256, 256, True), (256, 248, False), (128, 128, True)])
def test_norm_and_rotation(dtype, norm, d, rotated, halves):
    print(f"qk_norm_rope {dtype} d={d} rotated={rotated} halves={halves} norm={norm}", flush=True)
    g = gen(d + rotated)
    for batch, tokens, heads, kv_heads in ((1, 1, 1, 1), (2, 7, 5, 1), (3, 66, 9, 3), (1, 259, 30, 30)):
        q, k = (randn(g, batch, tokens, h, d).to(dtype) * torch.exp(randn(g, tokens, h, 1)).to(dtype) for h in (heads, kv_heads))
        table = None
        if rotated:
            turn = 30.0 * randn(g, batch, tokens, rotated // 2)
            table = torch.stack([turn.cos(), turn.sin()], 3)
            table = table if batch == 3 else table[0]
        gq, gk, bq, bk = (randn(g, d) for _ in range(4))
        check_qk(q, k, table, gq, gk, bq, bk, norm=norm, halves=halves)
        got = check_qk(q, k, table, gq, None, None, bk, norm=norm, eps=1e-3, halves=halves)
        assert torch.equal(B.qk_norm_rope(q, None, table, gq, norm=norm, eps=1e-3, halves=halves)[0], got[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_and_rotation_in_place_and_strides(dtype):
    """Inside a projection of odd pitch, head-major, repeated inputs; what lies between stays."""
    g = gen(6)
    turn = randn(g, 200, 32)
    table = torch.stack([turn.cos(), turn.sin()], 2)
    for pad in (0, 8, 3):                                        # on 16-byte borders and not
        wide = randn(g, 2, 200, 7 * 64 + pad).to(dtype)
        heads = wide[:, :, pad:].view(2, 200, 7, 64) if pad == 0 else wide.as_strided((2, 200, 7, 64), (200 * (448 + pad), 448 + pad, 64, 1), pad)
        want = B.qk_norm_rope(heads[:, :, :4].contiguous(), heads[:, :, 4:5].contiguous(), table)
        before = wide.clone()
        check_qk(heads[:, :, :4], heads[:, :, 4:5], table)
        q, k = B.qk_norm_rope(heads[:, :, :4], heads[:, :, 4:5], table, q_out=heads[:, :, :4], k_out=heads[:, :, 4:5])
        assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(heads[:, :, :4], want[0])
        assert torch.equal(wide[:, :, :pad], before[:, :, :pad]) and torch.equal(wide[:, :, pad + 320:], before[:, :, pad + 320:])
    q = randn(g, 2, 6, 200, 64).to(dtype).transpose(1, 2)
    check_qk(q, q[:, :, :1].expand(2, 200, 3, 64), table, q_out=torch.empty(2, 6, 200, 64, dtype=dtype, device=DEV).transpose(1, 2))
    check_qk(q[:1].expand(2, 200, 6, 64), q, table, norm=2)
    assert B.qk_norm_rope(q[:0], q[:0], table)[0].shape == (0, 200, 6, 64) and B.qk_norm_rope(q[:, :0], q[:, :0], table[:0])[1].shape == (2, 0, 6, 64)


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_unusual_heads(dtype):
    """Zeros, constants, far means, the largest squares that sum to a finite value, tiny values; NaN and infinity stay in their head."""
    g = gen(7)
    q = randn(g, 1, 8, 5, 64)
    q[0, 0, 0], q[0, 1, 0], q[0, 2, 0] = 0.0, 3.0, 1000.0 + q[0, 2, 0]
    q[0, 3, 0] = 2.0e18 * torch.sign(q[0, 3, 0])
    q[0, 4, 0] *= 1e-20
    q = q.to(dtype)
    for norm in (1, 2):
        check_qk(q, None, None, norm=norm)
    assert bool((B.qk_norm_rope(q, None, None, norm=2)[0][0, 1, 0] == 0).all())
    turn = randn(g, 8, 32)
    table = torch.stack([turn.cos(), turn.sin()], 2)
    for norm in (0, 1, 2):
        for halves in (False, True):
            want = B.qk_norm_rope(q, None, table, norm=norm, halves=halves)[0]
            bad = q.clone()
            bad[0, 5, 2, 40], bad[0, 6, 1, 0] = NAN, float("inf")
            got = B.qk_norm_rope(bad, None, table, norm=norm, halves=halves)[0]
            here = torch.zeros(1, 8, 5, dtype=torch.bool, device=DEV)
            here[0, 5, 2] = here[0, 6, 1] = True
            assert torch.equal(got[~here], want[~here]) and not torch.isfinite(got[here]).all(1).any()


def test_norm_and_rotation_beyond_32_bits():
    """2^18 tokens of 128 heads of 128 are 4.3 10^9 values, in place: a block of tokens over and over has the block's result."""
    g = gen(8)
    block = randn(g, 1, 64, 128, 128).bfloat16()
    turn = randn(g, 64, 64)
    table = torch.stack([turn.cos(), turn.sin()], 2)
    want = B.qk_norm_rope(block, None, table)[0]
    x = block.expand(4096, 64, 128, 128).reshape(1, 4096 * 64, 128, 128)
    out = B.qk_norm_rope(x, None, table.repeat(4096, 1, 1), q_out=x)[0]
    for at in (0, 2048 * 64, 4095 * 64):
        assert torch.equal(out[:, at:at + 64], want)


# ------------------------------------------------------------------------------------------------- packed attention
def packed_ref(q, k, v, scale, q_off, kv_off, prefix, frame, causal, cap, slopes):
    """(output, bound of its error) in 64 bits; offsets and prefix as lists."""
    H, d = q.shape[1:]
    share = H // k.shape[1]
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.full_like(o, 1e-37)
    u = U[q.dtype]
    for s in range(len(q_off) - 1):
        (a, b), (ka, kb) = q_off[s:s + 2], kv_off[s:s + 2]
        nq, nk = b - a, kb - ka
        if nq == 0 or nk == 0:
            continue
        P = min(max(prefix[s], 0), nk) if prefix else 0
        i, j = torch.arange(nk - nq, nk, device=DEV), torch.arange(nk, device=DEV)
        fi, fj = (torch.floor((t - P).double() / frame) for t in (i, j))
        seen = torch.ones(nq, nk, dtype=torch.bool, device=DEV)
        if causal:
            seen = (j < P)[None] | ((i >= P)[:, None] & (fj[None] <= fi[:, None]))
        some = seen.any(1, keepdim=True)
        for h in range(H):
            qq, kk, vv = q[a:b, h].double(), k[ka:kb, h // share].double(), v[ka:kb, h // share].double()
            x = qq @ torch.nan_to_num(kk, posinf=0.0, neginf=0.0).t().contiguous() * scale
            size = (qq.abs() @ torch.nan_to_num(kk, posinf=0.0, neginf=0.0).abs().t().contiguous() * scale)
            size = torch.where(seen, size, 0.0).amax(1, keepdim=True)
            es = (d + 4) * 2.0 ** -24 * size                     # a score's products are summed in fp32
            if cap:
                x = cap * torch.tanh(x / cap)
                es = es + 2.0 ** -20 * cap
            if slopes is not None:
                far = (fi[:, None] - fj[None]).abs() * ((i >= P)[:, None] & (j >= P)[None])
                bias = slopes[h].double() * far
                x = x - bias
                es = es + 2.0 ** -22 * (torch.where(seen, bias.abs() + x.abs(), 0.0)).amax(1, keepdim=True)
            x = torch.where(seen, x, -float("inf"))
            p = torch.where(some, torch.softmax(torch.where(some, x, 0.0), 1), 0.0)
            clean = torch.where(seen.any(0)[:, None], vv, 0.0)
            assert bool(torch.isfinite(clean).all())
            o[a:b, h] = p @ clean
            rounding = 2 * es + (nk + 32) * 2.0 ** -24 + (u if q.dtype == torch.bfloat16 else 0.0)      # probabilities in bf16
            tol[a:b, h] = rounding * (p @ clean.abs()) + u * o[a:b, h].abs() + 1e-37
    return o, tol


def offsets(lens, at=0):
    out = [at]
    for n in lens:
        out.append(out[-1] + n)
    return out


def check_packed(q, k, v, scale, q_off, kv_off=None, prefix=None, frame=1, causal=False, cap=0.0, slopes=None, out=None):
    got = B.packed_attn(q, k, v, scale, ints(*q_off), kv_offsets=None if kv_off is None else ints(*kv_off), prefix_lens=None if prefix is None else ints(*prefix),
                        frame=frame, causal=causal, cap=cap, slopes=slopes, out=out)
    ref, tol = packed_ref(q, k, v, scale, q_off, kv_off or q_off, prefix, frame, causal, cap, slopes)
    here = slice(q_off[0], q_off[-1])
    bad = ~((got[here].double() - ref[here]).abs() <= tol[here] * 1.001)
    assert not bad.any(), (float((got[here].double() - ref[here]).abs().max()), int(bad.sum()), bad.nonzero()[:4].tolist())
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("lens", [[1], [5, 0, 1, 63], [64, 65, 127], [0, 129, 0, 300], [700], [2, 1, 1, 31, 33, 256, 255, 257]])
def test_packed_attention_lengths_and_head_dims(dtype, d, lens):
    print(f"packed_attn {dtype} d={d} lens={lens}", flush=True)
    n = sum(lens)
    g = gen(n + d)
    q, k, v = (randn(g, n, 3, d).to(dtype) for _ in range(3))
    for causal in (False, True):
        check_packed(q, k, v, 1.0 / math.sqrt(d), offsets(lens), causal=causal)
        check_packed(q, k, v, 1.0 / math.sqrt(d), offsets(lens), causal=causal, prefix=[3] * len(lens), frame=7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("frame,prefix", [(1, 0), (1, 5), (3, 77), (16, 64), (50, 226), (64, 0), (100, 1), (300, 30), (1 << 30, 10), (7, 10000)])
def test_packed_attention_frames(dtype, frame, prefix):
    """Frames behind a prefix; a prefix longer than its sample, frames longer than all of them."""
    lens = [130, 401, 1, 700]
    g = gen(frame % 1000 + prefix)
    q, k, v = (randn(g, sum(lens), 2, 64).to(dtype) for _ in range(3))
    slopes = torch.tensor([0.5, -0.02], device=DEV)
    for kw in ({}, {"cap": 2.0}, {"slopes": slopes}, {"cap": 5.0, "slopes": slopes}):
        print(f"packed_attn {dtype} frame={frame} prefix={prefix} {sorted(kw)}", flush=True)
        for causal in (True, False):
            check_packed(q, k, v, 0.125, offsets(lens), prefix=[prefix, prefix // 2, 0, prefix], frame=frame, causal=causal, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(6, 1), (6, 2), (10, 2), (3, 3)])
def test_packed_attention_of_the_last_tokens(dtype, d, heads, kv_heads):
    """Single tokens, a few, a frame, more queries than keys, samples without either; keys divided among workgroups and not."""
    g = gen(heads * 10 + kv_heads + d)
    for nqs, nks in (([1], [1]), ([1, 1, 1], [77, 1300, 5000]), ([3, 0, 40, 2], [1279, 5, 4000, 0]), ([100, 7], [90, 2]), ([200, 65], [1400, 3001]), ([1], [1280])):
        print(f"packed_attn {dtype} d={d} heads={heads}/{kv_heads} q={nqs} k={nks}", flush=True)
        q, k, v = randn(g, sum(nqs), heads, d).to(dtype), randn(g, sum(nks), kv_heads, d).to(dtype), randn(g, sum(nks), kv_heads, d).to(dtype)
        slopes = torch.exp2(-torch.arange(heads, device=DEV) - 1.0)
        for kw in ({}, {"causal": True}, {"causal": True, "frame": 60, "prefix": [20] * len(nqs)}, {"causal": True, "slopes": slopes, "prefix": [3] * len(nqs)},
                   {"cap": 3.0}, {"cap": 20.0, "slopes": slopes, "frame": 9}):
            check_packed(q, k, v, 1.0 / math.sqrt(d), offsets(nqs), offsets(nks), **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 64, 128])
def test_packed_attention_with_garbage_where_nothing_counts(dtype, d):
    """NaN, infinities and the type's extremes: outside all samples, and in keys and values that some of a tile's queries see and others do not.
    Those that see a value which is not finite get one; the others get what they would without it."""
    g = gen(d)
    lens = [70, 200, 0, 333]
    n = sum(lens) + 11
    off = offsets(lens, 4)
    junk = torch.tensor([NAN, float("inf"), -float("inf"), torch.finfo(dtype).max, torch.finfo(dtype).min], device=DEV).to(dtype)
    q, k, v = (randn(g, n, 2, d).to(dtype) for _ in range(3))
    outside = torch.ones(n, dtype=torch.bool, device=DEV)
    outside[off[0]:off[-1]] = False
    for t in (q, k, v):
        t[outside] = junk[torch.randint(0, 5, (int(outside.sum()), 2, d), generator=g, device=DEV)]
    slopes = torch.tensor([0.3, 0.1], device=DEV)
    for kw in ({}, {"cap": 4.0}, {"slopes": slopes}):
        for causal in (False, True):
            out = torch.full_like(q, 7.0)
            check_packed(q, k, v, 0.2, off, causal=causal, out=out, **kw)
            assert bool((out[outside] == 7.0).all())
        for at, bad in ((100, NAN), (150, float("inf")), (273, -float("inf")), (off[-1] - 1, NAN)):
            print(f"packed_attn {dtype} d={d} bad token {at} {sorted(kw)}", flush=True)
            want = B.packed_attn(q, k, v, 0.2, ints(*off), causal=True, **kw)
            kk, vv = k.clone(), v.clone()
            kk[at], vv[at, :, 1] = NAN, bad
            s = [i for i in range(4) if off[i] <= at < off[i + 1]][0]
            got = B.packed_attn(q, kk, vv, 0.2, ints(*off), causal=True, **kw)
            for a, b in ((off[0], at), (off[s + 1], off[-1])):           # those that do not see it
                assert torch.equal(got[a:b], want[a:b])
            assert bool(torch.isnan(got[at:off[s + 1]]).all())
            got = B.packed_attn(q, k, vv, 0.2, ints(*off), causal=True, **kw)
            assert torch.equal(got[off[0]:at], want[off[0]:at]) and torch.equal(got[off[s + 1]:off[-1]], want[off[s + 1]:off[-1]])
            see = got[at:off[s + 1]]
            assert not torch.isfinite(see[:, :, 1]).any()
            rest = [i for i in range(d) if i != 1]
            assert torch.equal(see[:, :, rest], want[at:off[s + 1]][:, :, rest])


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_attention_of_a_sample_does_not_depend_on_the_others(dtype):
    g = gen(8)
    for nqs, nks, kw in (([345, 1, 130, 0, 260], None, {"causal": True, "frame": 13}), ([345, 1, 130, 0, 260], None, {}),
                         ([1, 3, 90, 700, 1], [1300, 5000, 2000, 1500, 9], {"causal": True}), ([1, 3, 90, 700, 1], [1300, 5000, 2000, 1500, 9], {"cap": 9.0})):
        nk = nks or nqs
        q, k, v = randn(g, sum(nqs), 6, 64).to(dtype), randn(g, sum(nk), 2, 64).to(dtype), randn(g, sum(nk), 2, 64).to(dtype)
        qo, ko = offsets(nqs), offsets(nk)
        whole = B.packed_attn(q, k, v, 0.125, ints(*qo), kv_offsets=ints(*ko) if nks else None, **kw)
        for s in range(5):
            a, b, ka, kb = qo[s], qo[s + 1], ko[s], ko[s + 1]
            alone = B.packed_attn(q[a:b].contiguous(), k[ka:kb].contiguous(), v[ka:kb].contiguous(), 0.125, ints(0, b - a),
                                  kv_offsets=ints(0, kb - ka) if nks else None, **kw)
            assert torch.equal(whole[a:b], alone), s
        assert torch.equal(whole, B.packed_attn(q, k, v, 0.125, ints(*qo), kv_offsets=ints(*ko) if nks else None, **kw))


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_attention_many_samples(dtype):
    """5000 samples of up to 9 tokens, more than a wave looks at in one step, and one long one at the end."""
    g = gen(9)
    lens = torch.randint(0, 10, (5000,), generator=torch.Generator().manual_seed(1)).tolist() + [500]
    n = sum(lens)
    q, k, v = (randn(g, n, 1, 16).to(dtype) for _ in range(3))
    got = B.packed_attn(q, k, v, 0.25, ints(*offsets(lens)))
    off = offsets(lens)
    sample = torch.repeat_interleave(torch.arange(len(lens), device=DEV), torch.tensor(lens, device=DEV))
    x = (q[:, 0].double() @ k[:, 0].double().t().contiguous()) * 0.25
    p = torch.softmax(torch.where(sample[:, None] == sample[None], x, -float("inf")), 1)
    ref = (p @ v[:, 0].double())[:, None]
    es = 20 * 2.0 ** -24 * 0.25 * float((q.float().norm(dim=2).max() * k.float().norm(dim=2).max()))
    tol = (2 * es + 600 * 2.0 ** -24 + U[dtype] * (dtype == torch.bfloat16)) * (p @ v[:, 0].double().abs())[:, None] + U[dtype] * ref.abs()
    assert bool(((got.double() - ref).abs() <= tol * 1.001).all())
    assert torch.equal(got[off[-2]:], B.packed_attn(q[off[-2]:], k[off[-2]:], v[off[-2]:], 0.25, ints(0, 500)))


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_attention_many_samples_with_divided_keys(dtype):
    """80 samples, some with keys for several workgroups, some without any: the table and the partial sums share the workspace; alone, and replayed from
    a graph with other offsets, each sample gives the same bits."""
    g = gen(12)
    nqs = [(1, 3, 0, 2, 70)[i % 5] for i in range(80)]
    nks = [(40, 1500, 7, 0, 90, 2600, 1279)[i % 7] for i in range(80)]
    q, k, v = randn(g, sum(nqs), 4, 64).to(dtype), randn(g, sum(nks), 2, 64).to(dtype), randn(g, sum(nks), 2, 64).to(dtype)
    qo, ko = offsets(nqs), offsets(nks)
    kw = {"causal": True, "frame": 30, "prefix": [i % 50 for i in range(80)], "slopes": torch.tensor([0.5, 0.1, 0.02, 0.0], device=DEV)}
    whole = check_packed(q, k, v, 0.125, qo, ko, **kw)
    call = {**kw, "prefix_lens": ints(*kw["prefix"])}
    del call["prefix"]
    for s in range(80):
        a, b, ka, kb = qo[s], qo[s + 1], ko[s], ko[s + 1]
        alone = B.packed_attn(q[a:b].contiguous(), k[ka:kb].contiguous(), v[ka:kb].contiguous(), 0.125, ints(0, b - a), kv_offsets=ints(0, kb - ka),
                              **{**call, "prefix_lens": call["prefix_lens"][s:s + 1]})
        assert torch.equal(whole[a:b], alone), s
    dq, dk = ints(*qo), ints(*ko)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = B.packed_attn(q, k, v, 0.125, dq, kv_offsets=dk, **call)
    other = offsets(list(reversed(nks)))
    for keys in (ko, other, ko, other):
        dk.copy_(ints(*keys))
        want = B.packed_attn(q, k, v, 0.125, ints(*qo), kv_offsets=ints(*keys), **call)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples", [50, 400])
def test_packed_attention_of_offsets_that_fall_stays_inside(dtype, samples):
    """Every second sample has all the tokens: far more blocks, and pieces of their keys, than rising offsets could have."""
    g = gen(13)
    q, k, v = (randn(g, 1500, 2, 64).to(dtype) for _ in range(3))
    wide = torch.full((1500, 4, 64), 7.0, dtype=dtype, device=DEV)
    fall = ints(*[0, 1500] * (samples // 2), 0)
    B.packed_attn(q, k, v, 0.125, fall, kv_offsets=fall, out=wide[:, 1:3])
    B.packed_attn(q[:20], k, v, 0.125, fall, kv_offsets=fall, out=wide[:20, 1:3])
    B.packed_attn(q, k, v, 0.125, fall, out=wide[:, 1:3])
    torch.cuda.synchronize()
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 3] == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_attention_strides_and_offsets_outside(dtype):
    """Parts of one projection, head-major tensors, repeated operands, an output inside a wider one; offsets before 0 and behind the end are
    clamped."""
    g = gen(6)
    qkv = randn(g, 300, 8, 64).to(dtype)
    wide = torch.full((300, 6, 64), 7.0, dtype=dtype, device=DEV)
    check_packed(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], 0.125, [0, 100, 300], causal=True, out=wide[:, 1:5])
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 5] == 7.0).all())
    q = randn(g, 4, 300, 64).to(dtype).transpose(0, 1)
    check_packed(q, qkv[:, :1].expand(300, 4, 64), qkv[:1, :4].expand(300, 4, 64), 0.125, [0, 130, 300])
    same = B.packed_attn(q, qkv[:, :4], qkv[:, 4:], 0.125, ints(0, 200, 300))
    assert torch.equal(same, B.packed_attn(q, qkv[:, :4], qkv[:, 4:], 0.125, ints(-7, 200, 1000)))
    assert torch.equal(same, B.packed_attn(q, qkv[:, :4], qkv[:, 4:], 0.125, ints(-7, 200, 1000), kv_offsets=ints(-2 ** 31, 200, 2 ** 31 - 1)))
    # offsets that fall give nothing particular, but stay inside
    B.packed_attn(q, qkv[:, :4], qkv[:, 4:], 0.125, ints(250, 10, 299, 3), kv_offsets=ints(300, 300, 0, 300), causal=True, out=wide[:, 1:5])
    torch.cuda.synchronize()
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 5] == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_attention_empty_extents(dtype):
    t = torch.ones(10, 2, 32, dtype=dtype, device=DEV)
    assert B.packed_attn(t[:0], t[:0], t[:0], 0.2, ints(0)).shape == (0, 2, 32)
    out = torch.full_like(t, 3.0)
    assert B.packed_attn(t, t, t, 0.2, ints(0), out=out) is out and bool((out == 3.0).all())
    assert bool((B.packed_attn(t, t[:0], t[:0], 0.2, ints(0, 10), kv_offsets=ints(0, 0)) == 0).all())
    assert bool((B.packed_attn(t, t[:3], t[:3], 0.2, ints(0, 10), kv_offsets=ints(0, 3), causal=True)[:7] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nq,nk", [(300, 300), (5, 3000)])
def test_packed_attention_of_large_scores(dtype, nq, nk):
    """Scores of thousands, growing, falling and in any order along the keys; exact ones up to 2^100, one key far ahead; a tiny scale."""
    g = gen(5)
    for order in ("up", "down", "any"):
        q = randn(g, nq, 2, 64).to(dtype)
        size = torch.linspace(0.1, 60.0, nk, device=DEV)
        size = size.flip(0) if order == "down" else size[torch.randperm(nk, generator=g, device=DEV)] if order == "any" else size
        k = (randn(g, nk, 2, 64) * size[:, None, None]).to(dtype)
        check_packed(q, k, randn(g, nk, 2, 64).to(dtype), 1.0, [0, nq], [0, nk])
    v = randn(g, nk, 1, 64).to(dtype)
    for power in (10, 14, 24, 40, 100):
        for best in ([0], [nk - 1], [70, nk - 3], [1, 2]):
            q, k = torch.zeros(nq, 1, 64, device=DEV), torch.zeros(nk, 1, 64, device=DEV)
            q[..., 0] = 2.0 ** (power // 2)
            k[:, 0, 0] = 2.0 ** (power - power // 2) * 0.5
            k[best, 0, 0] = 2.0 ** (power - power // 2)
            for shift in (0.0, 1.5):                             # (below zero: the best are the smallest in size)
                kk = k - shift * 2.0 ** (power - power // 2) * (torch.arange(64, device=DEV) == 0)
                out = B.packed_attn(q.to(dtype), kk.to(dtype), v, 1.0, ints(0, nq), kv_offsets=ints(0, nk)).double()
                want = v.double()[best].mean(0).expand_as(out)
                assert bool(((out - want).abs() <= 2 * U[dtype] * v.double()[best].abs().mean(0) + 1e-6).all()), (power, best, shift)
    check_packed(*(randn(g, n, 1, 64).to(dtype) for n in (nq, nk, nk)), 1e-38, [0, nq], [0, nk])


def test_packed_attention_offsets_beyond_32_bits():
    """Keys 2^20 elements apart: the last ones lie 5.9 GB behind the first; samples of one token to a thousand."""
    nk, step = 2800, 1 << 20
    big = torch.zeros(nk * step, dtype=torch.bfloat16, device=DEV)
    g = gen(7)
    k, v, q = (big.as_strided((nk, 2, 64), (step, 64, 1), off) for off in (0, 128, 256))
    for t in (k, v, q):
        t.copy_(randn(g, nk, 2, 64))
    out = big.as_strided((nk, 2, 64), (step, 64, 1), 384)
    check_packed(q, k, v, 0.125, [0, 1, 1000, 1801, nk], causal=True, out=out)
    check_packed(q[:2], k, v, 0.125, [0, 1, 2], [0, 100, nk], causal=True)


def test_packed_attention_of_one_sample_equals_full_attention():
    """The same definition as attn3d: one sample, no mask."""
    g = gen(12)
    q, k, v = (randn(g, 1000, 4, 64).bfloat16() for _ in range(3))
    a, b = B.packed_attn(q, k, v, 0.125, ints(0, 1000)).double(), B.attn3d(q[None], k[None], v[None], 0.125)[0].double()
    assert float((a - b).norm() / b.norm()) < 2.0 ** -7                  # (both round probabilities and results to bf16)


# ------------------------------------------------------------------------------------------------- together
def sublayer(x, off, prefix, frame, table, p, heads, kv_heads):
    """x [T, D]: x + out(attention(rotated norms of q and k, v)), projections in 4 bits, samples packed along T."""
    T, D = x.shape
    qkv = B.dit_linear_fp4(*B.fp4_quantize(x), *p["wqkv"], p["bqkv"]).view(1, T, heads + 2 * kv_heads, -1)
    q, k = qkv[:, :, :heads], qkv[:, :, heads:heads + kv_heads]
    B.qk_norm_rope(q, k, table, p["gq"], p["gk"], q_out=q, k_out=k)
    o = B.packed_attn(q[0], k[0], qkv[0, :, heads + kv_heads:], 1.0 / math.sqrt(q.shape[3]), off, prefix_lens=prefix, frame=frame, causal=True)
    return x + B.dit_linear_fp4(*B.fp4_quantize(o.view(T, -1)), *p["wo"], p["bo"])


def sublayer_data(seed, lens=(345, 77, 200), D=320, heads=5, kv_heads=5, prefix=17, frame=40):
    g = gen(seed)
    d = D // heads
    mats = {"wqkv": randn(g, (heads + 2 * kv_heads) * d, D) / math.sqrt(D), "wo": randn(g, D, D) / math.sqrt(D)}
    p = {n: B.fp4_quantize(m) for n, m in mats.items()}
    p.update(gq=1 + 0.2 * randn(g, d), gk=1 + 0.2 * randn(g, d), bqkv=0.1 * randn(g, (heads + 2 * kv_heads) * d), bo=0.1 * randn(g, D))
    x = randn(g, sum(lens), D).bfloat16()
    pos = torch.cat([torch.arange(n, device=DEV) for n in lens]).float()
    table = B.rope_table(torch.stack([pos // frame, pos % frame], 1), [d // 2, d // 2])
    return (x, ints(*offsets(lens)), ints(*([prefix] * len(lens))), frame, table, p, heads, kv_heads), mats


def test_a_sublayer_on_packed_samples():
    """Against the sublayer in 64 bits without any 4-bit rounding.  Blocks of 32 normal values hold steps of 0.5, 1 and 2 under a largest value of 3 to 6: errors of
    0.13 of the norm at most in the mean square.  A product of two such operands with independent errors: 0.18.  Values carry 0.18 and the output projection
    0.13 twice more: 0.26; queries and keys of 0.18 each move scores of order one by 0.25 and the weighted sums with them: 0.36 together."""
    args, mats = sublayer_data(13)
    x, off, prefix, frame, table, p, heads, kv_heads = args
    got = sublayer(*args).double() - x.double()
    T, D = x.shape
    y = (x.double() @ mats["wqkv"].double().t() + p["bqkv"].double()).view(1, T, heads + 2 * kv_heads, -1)
    q, k = (turn_ref(*norm_ref(t, 1, ga, None, 1e-6), table, False)[0][0] for t, ga in ((y[:, :, :heads], p["gq"]), (y[:, :, heads:heads + kv_heads], p["gk"])))
    o, _ = packed_ref(q.float(), k.float(), y[0, :, heads + kv_heads:].float(), 1.0 / 8.0, off.tolist(), off.tolist(), prefix.tolist(), frame, True, 0.0, None)
    ref = o.reshape(T, D) @ mats["wo"].double().t() + p["bo"].double()
    assert float((got - ref).norm() / ref.norm()) < 0.4


def test_new_tokens_against_kept_keys_equal_the_whole():
    """The last frame's queries against all keys give what the whole sample's pass gave them, up to the order of sums."""
    g = gen(15)
    n, frame, prefix = 226 + 4 * 300, 300, 226
    q, k, v = randn(g, n, 6, 64).bfloat16(), randn(g, n, 2, 64).bfloat16(), randn(g, n, 2, 64).bfloat16()
    whole = B.packed_attn(q, k, v, 0.125, ints(0, n), prefix_lens=ints(prefix), frame=frame, causal=True).double()
    for new in (300, 1, 17):
        last = B.packed_attn(q[n - new:], k, v, 0.125, ints(0, new), kv_offsets=ints(0, n), prefix_lens=ints(prefix), frame=frame, causal=True).double()
        assert float((last - whole[n - new:]).norm() / last.norm()) < 2.0 ** -7


def test_a_captured_sublayer_replays():
    """In a graph, replayed with new inputs and new lengths and with eager calls between, equal to the eager result each time; two graphs live."""
    data = [sublayer_data(s, lens)[0] for s, lens in ((14, (345, 77, 200)), (15, (10, 600, 12)))]
    x, off, prefix, frame, table, p, heads, kv_heads = data[0]
    nq = [torch.arange(0, 4 * m, m, dtype=torch.int32, device=DEV) for m in (1,)][0]
    kept = torch.empty(4000, 2 * kv_heads, 64, dtype=torch.bfloat16, device=DEV).normal_(generator=gen(3))
    ko = ints(0, 1500, 1500, 4000)

    def step():
        out = sublayer(x, off, prefix, frame, table, p, heads, kv_heads)
        return out, B.packed_attn(out[:3].view(3, heads, 64), kept[:, :kv_heads], kept[:, kv_heads:], 0.125, nq, kv_offsets=ko, causal=True)
    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = step()
        graphs.append((gr, out))
    originals = [(d[0].clone(), d[1].clone(), d[4].clone()) for d in data]
    for turn in range(4):
        for t, n in zip((x, off, table), originals[turn % 2]):
            t.copy_(n)
        want = step()
        torch.cuda.synchronize()
        for gr, out in graphs:
            out[0].zero_()
            out[1].zero_()
            gr.replay()
        sublayer(*data[1])
        torch.cuda.synchronize()
        for gr, out in graphs:
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), turn


def test_sublayer_on_two_streams_at_once():
    data = [sublayer_data(s)[0] for s in (16, 17)]
    want = [sublayer(*d) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    got = [[], []]
    for _ in range(3):
        for i, (d, st) in enumerate(zip(data, streams)):
            with torch.cuda.stream(st):
                got[i].append(sublayer(*d))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(t, want[i]) for t in got[i])
