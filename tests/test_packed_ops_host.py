"""Operators of self-attention on packed samples: what they refuse, on the host and before any launch, and the rules that divide their work."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

from paper_2505_14741_amd import binding as B
from paper_2505_14741_amd import build

FAKE = 0x10000                                                   # never dereferenced: every call below is refused or has nothing to do


@pytest.mark.parametrize("entry", ["fp4_quantize", "fp4_dequantize"])
def test_4_bit_blocks_refuse(entry):
    f = getattr(B.lib(), entry)

    def call(a=FAKE, b=2 * FAKE, c=3 * FAKE, rows=4, cols=100, row=100, dtype=1):
        return f(a, b, c, rows, cols, row, dtype, None)
    assert call(dtype=2) == -3
    for bad in (dict(rows=-1), dict(cols=0), dict(rows=(1 << 24) + 1), dict(cols=(1 << 22) + 1), dict(row=99), dict(row=1 << 41), dict(rows=1 << 24, cols=1 << 15, row=1 << 15),
                dict(rows=1 << 24, cols=8192, row=8192), dict(b=2 * FAKE + 8)):
        assert call(**bad) == -2, bad
    x, q, s = ("a", "b", "c") if entry == "fp4_quantize" else ("c", "a", "b")
    for bad in ({x: 9 * FAKE + 1}, {q: 9 * FAKE + 8}, {s: 9 * FAKE + 4}):
        assert call(**bad) == -2, bad
    for name in "abc":
        assert call(**{name: None}) == -1
    assert call(b=FAKE) == -2 if entry == "fp4_quantize" else call(c=FAKE) == -2
    assert call(rows=0, a=None, b=None, c=None) == 0


def test_4_bit_product_refuses():
    L = B.lib()

    def call(a=FAKE, a_s=2 * FAKE, w=3 * FAKE, w_s=4 * FAKE, bias=5 * FAKE, out=6 * FAKE, m=4, n=8, k=128, act=0, ws=None, nb=0):
        return L.dit_linear_fp4(a, a_s, w, w_s, bias, out, m, n, k, act, ws, nb, None)
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(m=(1 << 24) + 1), dict(n=(1 << 24) + 1), dict(k=(1 << 22) + 1), dict(act=2), dict(act=-1), dict(m=1 << 24, n=1 << 24), dict(m=1 << 18, n=1 << 18),
                dict(a=FAKE + 8), dict(a_s=FAKE + 8), dict(w=FAKE + 8), dict(w_s=FAKE + 4), dict(bias=FAKE + 4), dict(out=FAKE + 2), dict(out=FAKE), dict(out=3 * FAKE)):
        assert call(**bad) == -2, bad
    for name in ("a", "a_s", "w", "w_s", "bias", "out"):
        assert call(**{name: None}) == -1
    assert call(ws=FAKE + 128, nb=1 << 20) == -4
    assert call(m=0, a=None, a_s=None, out=None) == 0
    assert L.dit_linear_fp4_workspace_bytes(0, 8, 128) == 0 and L.dit_linear_fp4_workspace_bytes(4, 8, (1 << 22) + 1) == 0


def test_rope_table_refuses():
    L = B.lib()

    def call(pos=FAKE, row=2, dims=(16, 24), thetas=(1e4, 1e4), table=2 * FAKE, tokens=5, axes=None):
        n = len(dims)
        return L.rope_table(pos, row, n if axes is None else axes, (C.c_int * n)(*dims), (C.c_double * n)(*thetas), table, tokens, None)
    for bad in (dict(axes=0), dict(dims=(2,) * 5, thetas=(1.0,) * 5), dict(dims=(16, 23)), dict(dims=(0, 16)), dict(dims=(-2, 16)), dict(dims=(200, 58)), dict(dims=(2, (1 << 31) - 2)),
                dict(thetas=(1e4, 0.0)), dict(thetas=(-1.0, 1.0)), dict(thetas=(float("nan"), 1.0)), dict(thetas=(float("inf"), 1.0)), dict(tokens=-1), dict(tokens=(1 << 24) + 1),
                dict(row=-1), dict(row=1 << 41), dict(pos=FAKE + 2), dict(table=2 * FAKE + 4), dict(table=FAKE)):
        assert call(**bad) == -2, bad
    assert call(pos=None) == -1 and call(table=None) == -1 and L.rope_table(FAKE, 1, 1, None, None, 2 * FAKE, 1, None) == -1
    assert call(tokens=0, pos=None, table=None) == 0


def test_norm_and_rotation_refuse():
    L = B.lib()

    def call(q=FAKE, k=2 * FAKE, table=3 * FAKE, qo=4 * FAKE, ko=5 * FAKE, gq=None, bk=None, shape=True, **over):
        s = dict(batch=2, tokens=5, heads=4, kv_heads=2, head_dim=64, rotated=64, norm=1, halves=0, dtype=1, eps=1e-6, q_batch=1280, q_token=256, q_head=64, k_batch=640,
                 k_token=128, k_head=64, q_out_batch=1280, q_out_token=256, q_out_head=64, k_out_batch=640, k_out_token=128, k_out_head=64, table_batch=0)
        s.update(over)
        return L.qk_norm_rope(q, k, table, gq, None, None, bk, qo, ko, C.byref(B._QkNormShape(**s)) if shape else None, None)
    assert call(shape=False) == -1 and call(dtype=2) == -3
    for bad in (dict(batch=-1), dict(tokens=-1), dict(heads=0), dict(kv_heads=-1), dict(batch=65536), dict(heads=65536), dict(kv_heads=65536), dict(tokens=(1 << 24) + 1),
                dict(batch=4, tokens=1 << 24), dict(head_dim=60), dict(head_dim=0), dict(head_dim=264), dict(rotated=60), dict(rotated=72), dict(rotated=-8), dict(halves=1, rotated=40),
                dict(halves=2), dict(norm=3), dict(norm=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(table_batch=-1), dict(table_batch=1 << 41),
                dict(q_token=-1), dict(k_head=-64), dict(q_out_token=-256), dict(q_out_head=32), dict(k_out_token=64), dict(q_out_batch=0), dict(q_batch=1 << 41),
                dict(q=FAKE + 1), dict(qo=FAKE + 1), dict(k=FAKE + 1), dict(ko=FAKE + 1), dict(table=FAKE + 2), dict(gq=FAKE + 2), dict(bk=FAKE + 1),
                dict(qo=2 * FAKE), dict(ko=FAKE), dict(qo=5 * FAKE), dict(qo=FAKE, q_token=264, q_batch=1320), dict(ko=2 * FAKE, k_head=72)):
        assert call(**bad) == -2, bad
    for name in ("q", "k", "table", "qo", "ko"):
        assert call(**{name: None}) == -1
    assert call(batch=0, q=None, qo=None) == 0 and call(tokens=0, q=None, k=None, qo=None, ko=None, table=None) == 0
    assert call(tokens=0, heads=4, kv_heads=0, k=None, ko=None) == 0


def packed_shape(**over):
    s = dict(samples=3, q_tokens=50, kv_tokens=50, heads=4, kv_heads=2, head_dim=64, dtype=1, own_offsets=0, causal=0, frame=1, scale=0.125, cap=0.0, q_token=256, q_head=64,
             k_token=128, k_head=64, v_token=128, v_head=64, o_token=256, o_head=64)
    s.update(over)
    return B._PackedShape(**s)


def call_packed(shape, q=FAKE, k=2 * FAKE, v=3 * FAKE, qo=4 * FAKE, ko=None, prefix=None, slopes=None, o=5 * FAKE, ws=None, nb=0):
    return B.lib().packed_attn(q, k, v, qo, ko, prefix, slopes, o, C.byref(shape) if shape else None, ws, nb, None)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=2), -3), (dict(head_dim=48), -2), (dict(samples=-1), -2), (dict(q_tokens=-1), -2), (dict(kv_tokens=-1), -2), (dict(heads=0), -2), (dict(kv_heads=0), -2),
    (dict(kv_heads=3), -2), (dict(samples=65536), -2), (dict(heads=65536), -2), (dict(q_tokens=(1 << 24) + 1), -2), (dict(kv_tokens=(1 << 24) + 1, own_offsets=1), -2),
    (dict(own_offsets=2), -2), (dict(kv_tokens=51), -2), (dict(causal=2), -2), (dict(frame=0), -2), (dict(frame=-5), -2), (dict(scale=0.0), -2), (dict(scale=-1.0), -2),
    (dict(scale=float("nan")), -2), (dict(scale=3e38), -2), (dict(cap=-1.0), -2), (dict(cap=float("nan")), -2), (dict(cap=float("inf")), -2), (dict(cap=1e-39, scale=1.0), -2),
    (dict(cap=3e38), -2), (dict(q_token=252), -2), (dict(q_head=-64), -2), (dict(k_token=100), -2), (dict(v_token=1 << 41), -2), (dict(o_token=0), -2), (dict(o_head=32), -2),
    (dict(q_tokens=1 << 24, kv_tokens=1 << 24, heads=256, kv_heads=1, q_token=16384, o_token=16384), -2),
    (dict(q_tokens=1 << 24, kv_tokens=1 << 24, heads=128, kv_heads=128, q_token=8192, o_token=8192), -2),
    (dict(samples=65535, q_tokens=50, heads=300, kv_heads=300, q_token=19200, o_token=19200, k_token=19200, v_token=19200), -2)])
def test_packed_attention_refuses(over, status):
    assert call_packed(packed_shape(**over)) == status
    assert B.lib().packed_attn_workspace_bytes(C.byref(packed_shape(**over))) == 0


def test_packed_attention_refuses_pointers():
    ok = packed_shape()
    assert call_packed(None) == -1 and B.lib().packed_attn_workspace_bytes(None) == 0
    for name in ("q", "k", "v", "qo", "o"):
        assert call_packed(ok, **{name: None}) == -1
        assert call_packed(ok, **{name: 6 * FAKE + 2}) == -2
    assert call_packed(ok, prefix=FAKE + 2) == -2 and call_packed(ok, slopes=FAKE + 2) == -2
    assert call_packed(ok, ko=7 * FAKE) == -2                            # offsets that the shape does not have
    assert call_packed(packed_shape(own_offsets=1)) == -1
    for same in (FAKE, 2 * FAKE, 3 * FAKE):
        assert call_packed(ok, o=same) == -2
    assert call_packed(packed_shape(samples=0), q=None, k=None, v=None, qo=None, o=None) == 0
    assert call_packed(packed_shape(q_tokens=0, kv_tokens=0), q=None, k=None, v=None, qo=None, o=None) == 0


def test_packed_attention_workspace():
    """Keys with offsets of their own may be divided, and more than 64 samples need a table; a missing, small or misaligned workspace is refused."""
    bytes_of = lambda **kw: B.lib().packed_attn_workspace_bytes(C.byref(packed_shape(**kw)))  # noqa: E731
    assert bytes_of() == 0 and bytes_of(q_tokens=17776, kv_tokens=17776) == 0 and bytes_of(samples=64) == 0
    table = bytes_of(samples=65)
    assert table >= 66 * 8 and table % 256 == 0
    one = dict(samples=1, q_tokens=1, kv_tokens=17776, own_offsets=1)
    n = bytes_of(**one)
    assert n >= 17 * 2 * 2 * 68 * 4 and n % 256 == 0                     # 17 pieces of two query heads for each of two key heads
    assert bytes_of(**dict(one, kv_tokens=1279)) == 0
    s = packed_shape(**one)
    assert call_packed(s, ko=6 * FAKE) == -4 and call_packed(s, ko=6 * FAKE, ws=7 * FAKE, nb=n - 1) == -4 and call_packed(s, ko=6 * FAKE, ws=7 * FAKE + 128, nb=n) == -4
    assert call_packed(packed_shape(samples=65)) == -4 and call_packed(packed_shape(samples=65), ws=7 * FAKE, nb=table - 256) == -4


RULES = """
#include "plan.h"
extern "C" int pieces(int rows, int keys, int kv_heads) { return ps::packed_pieces(rows, keys, kv_heads); }
extern "C" void plan(int bf16, int own, int samples, int rows, int kv_tokens, int kv_heads, int head_dim, long* out) {
    const ps::PackedPlan p = ps::packed_plan(bf16 != 0, own != 0, samples, rows, kv_tokens, kv_heads, head_dim, 256);
    out[0] = p.block; out[1] = p.slots; out[2] = p.part_rows; out[3] = (long)p.table_bytes; out[4] = (long)p.part_bytes; out[5] = ps::packed_workgroups(p.slots, kv_heads);
}
extern "C" void fp4(int m, int n, int blocks, int split, int* out) {
    const ps::Fp4Plan p = ps::fp4_plan(m, n, blocks, split != 0, 256);
    out[0] = p.tile; out[1] = p.pieces; out[2] = ps::kFp4Tiles[p.tile].bm; out[3] = ps::kFp4Tiles[p.tile].bn;
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("packed_rules")
    src, lib = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
    with open(src, "w") as f:
        f.write(RULES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, src, "-o", lib], check=True)
    return C.CDLL(lib)


def test_packed_attention_slots_hold_every_block_and_piece(rules):
    """Samples of any lengths have slots enough, scratch for each, and launches below 2^32 threads; pieces are not empty."""
    r = random.Random(1)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))  # noqa: E731
    out = (C.c_long * 6)()
    for _ in range(4000):
        kv_heads, share = r.choice([1, 2, 6, 30, 64, 200, 600]), r.choice([1, 1, 5, 8])
        n = r.choice([1, 1, 2, 8, 70, 300])
        own = r.random() < 0.7
        q = [log(1, 30000) if r.random() < 0.3 else r.randint(0, 40) for _ in range(n)]
        k = [log(1, 60000) if r.random() < 0.6 else r.randint(0, 2000) for _ in range(n)] if own else q
        rows, kv = sum(q) * share, sum(k)
        if (rows // 64 + n) * kv_heads > (1 << 19 if own else 1 << 23):
            continue
        for bf16, d in ((1, 64), (1, 128), (0, 32)):
            rules.plan(bf16, own, n, rows, kv, kv_heads, d, out)
            block, slots, part_rows, table, part, wgs = list(out)
            used = 0
            for a, b in zip(q, k):
                p = rules.pieces(a * share, b, kv_heads) if own else 1
                assert 1 <= p and (p == 1 or (b >= 1280 and p <= b // 256 and part > 0))
                used += -(-a * share // block) * p
            assert used <= slots and part_rows == min(rows, block)
            assert wgs >= slots * kv_heads and wgs < 1 << 24
            assert table >= (8 * (slots + 1) if n > 64 else 0) and table % 256 == 0
            assert part == (slots * kv_heads * part_rows * (d + 4) * 4 if own and kv >= 1280 else 0)


def test_packed_attention_launches_are_below_the_limit(rules):
    """The largest calls that are not refused: samples of 1280 keys each, or rows without end."""
    out = (C.c_long * 6)()
    for kv_heads in (1, 2, 8, 64, 512):
        for n in (1, 100, 13107, 65535):
            for own in (0, 1):
                rows = min(64 * (((1 << 19) if own else (1 << 23)) // kv_heads - n), 1 << 30)
                if rows < 1:
                    continue
                for bf16 in (0, 1):
                    rules.plan(bf16, own, n, rows, 1 << 24, kv_heads, 16, out)
                    assert out[5] < 1 << 24, (kv_heads, n, own, bf16)


def test_packed_attention_places_cover_every_head_and_slot():
    """Workgroup id -> (key head, slot), as the kernel computes it: every pair once, whatever the number of heads."""
    for kv_heads in (1, 2, 6, 7, 8, 9, 30, 64, 100):
        for slots in (8, 16, 72):
            seen = set()
            for wg in range(slots * kv_heads):
                x, n, own, rest = wg & 7, wg >> 3, kv_heads // 8, kv_heads % 8
                period, i = divmod(n, kv_heads)
                if i < 8 * own:
                    seen.add((x * own + i % own, period * 8 + i // own))
                else:
                    u = (period * rest + i - 8 * own) * 8 + x
                    seen.add((8 * own + u % rest, u // rest))
            assert seen == {(g, s) for g in range(kv_heads) for s in range(slots)}


def test_4_bit_product_plans(rules):
    r = random.Random(2)
    out = (C.c_int * 4)()
    sizes = [(1, 1, 1), (112, 7680, 15), (17776, 5760, 15), (1 << 24, 64, 1), (1, 1 << 24, 4), (60, 100, 32768)]
    sizes += [(int(2 ** r.uniform(0, 16)), int(2 ** r.uniform(0, 14)), int(2 ** r.uniform(0, 10))) for _ in range(4000)]
    for m, n, blocks in sizes:
        for split in (0, 1):
            rules.fp4(m, n, blocks, split, out)
            tile, pieces, bm, bn = list(out)
            assert 0 <= tile < 5 and 1 <= pieces and bm <= 256 and bn <= 256
            if pieces > 1:                                               # 4 stages of 256 at least, a round of workgroups at most
                assert split and 8 * pieces <= blocks and -(-m // bm) * -(-n // bn) * pieces <= 512


def test_binding_refuses_tensors():
    """Wrong types, shapes, strides and places raise before the library is called."""
    x, q4 = torch.zeros(4, 128), torch.zeros(4, 64, dtype=torch.uint8)
    s4 = torch.zeros(4, 16, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    bias = torch.zeros(4)
    q, k, t = torch.zeros(2, 5, 4, 64), torch.zeros(2, 5, 2, 64), torch.zeros(5, 32, 2)
    pq, pk, off = torch.zeros(50, 4, 64), torch.zeros(50, 2, 64), torch.zeros(4, dtype=torch.int32)
    shape, dtype = -2, -3
    calls = [
        (lambda: B.fp4_quantize(x[0]), shape), (lambda: B.fp4_quantize(x.half()), dtype), (lambda: B.fp4_quantize(x.t()), shape), (lambda: B.fp4_quantize(x), shape),
        (lambda: B.fp4_dequantize(q4.int(), s4), dtype), (lambda: B.fp4_dequantize(q4, s4.view(torch.uint8)), dtype), (lambda: B.fp4_dequantize(q4[:, :32], s4), shape),
        (lambda: B.fp4_dequantize(q4, s4[:2]), shape), (lambda: B.fp4_dequantize(q4, s4, cols=0), shape), (lambda: B.fp4_dequantize(q4, s4, cols=129), shape),
        (lambda: B.fp4_dequantize(q4, s4, dtype=torch.float16), dtype), (lambda: B.fp4_dequantize(q4, s4, out=torch.zeros(4, 127)), shape), (lambda: B.fp4_dequantize(q4, s4), shape),
        (lambda: B.dit_linear_fp4(x, s4, q4, s4, bias), shape), (lambda: B.dit_linear_fp4(q4.int(), s4, q4, s4, bias), dtype), (lambda: B.dit_linear_fp4(q4, s4.view(torch.uint8), q4, s4, bias), dtype),
        (lambda: B.dit_linear_fp4(q4[:, :32], s4, q4[:, :32], s4, bias), shape), (lambda: B.dit_linear_fp4(q4, s4[:, :4], q4, s4, bias), shape), (lambda: B.dit_linear_fp4(q4, s4, q4, s4, bias[:3]), shape),
        (lambda: B.dit_linear_fp4(q4, s4, q4, s4, bias.double()), dtype), (lambda: B.dit_linear_fp4(q4, s4, q4, s4, bias, act=2), shape), (lambda: B.dit_linear_fp4(q4, s4, q4, s4, bias), shape),
        (lambda: B.dit_linear_fp4(q4, s4, q4, s4, bias, out=torch.zeros(4, 4)), dtype),
        (lambda: B.rope_table(torch.zeros(5, 2), (16,)), shape), (lambda: B.rope_table(torch.zeros(5, 2).double(), (16, 16)), dtype), (lambda: B.rope_table(torch.zeros(5, 2), (16, 15)), shape),
        (lambda: B.rope_table(torch.zeros(5, 2), (16, 16), [1e4]), shape), (lambda: B.rope_table(torch.zeros(5, 5), (2,) * 5), shape), (lambda: B.rope_table(torch.zeros(5, 2), (16, 16)), shape),
        (lambda: B.rope_table(torch.zeros(5, 2), (16, 16), out=torch.zeros(5, 8, 2)), shape),
        (lambda: B.qk_norm_rope(q[0], k, t), shape), (lambda: B.qk_norm_rope(q, k[:, :4], t), shape), (lambda: B.qk_norm_rope(q, k.bfloat16(), t), dtype), (lambda: B.qk_norm_rope(q.half(), k.half(), t), dtype),
        (lambda: B.qk_norm_rope(q, k, t.double()), dtype), (lambda: B.qk_norm_rope(q, k, t[:4]), shape), (lambda: B.qk_norm_rope(q, k, t[:, ::2]), shape), (lambda: B.qk_norm_rope(q, k, t, bias), shape),
        (lambda: B.qk_norm_rope(q, k, t, torch.zeros(64).double()), dtype), (lambda: B.qk_norm_rope(q, k, t, norm=3), shape), (lambda: B.qk_norm_rope(q, k, t, q_out=q[:1]), shape),
        (lambda: B.qk_norm_rope(q, None, t, k_out=k), shape), (lambda: B.qk_norm_rope(q, k, t), shape), (lambda: B.qk_norm_rope(q, k, t, q_out=torch.zeros(2, 5, 64, 4).transpose(2, 3)), shape),
        (lambda: B.packed_attn(pq[0], pk, pk, 1.0, off), shape), (lambda: B.packed_attn(pq, pk, pk[:49], 1.0, off), shape), (lambda: B.packed_attn(pq, pk[:49], pk[:49], 1.0, off), shape),
        (lambda: B.packed_attn(pq, pk, pk.bfloat16(), 1.0, off), dtype), (lambda: B.packed_attn(pq.half(), pk.half(), pk.half(), 1.0, off), dtype), (lambda: B.packed_attn(pq, pk[..., :32], pk[..., :32], 1.0, off), shape),
        (lambda: B.packed_attn(pq, pk, pk, 1.0, off.long()), dtype), (lambda: B.packed_attn(pq, pk, pk, 1.0, off[:0]), shape), (lambda: B.packed_attn(pq, pk, pk, 1.0, off, kv_offsets=off[:3]), shape),
        (lambda: B.packed_attn(pq, pk, pk, 1.0, off, prefix_lens=off), shape), (lambda: B.packed_attn(pq, pk, pk, 1.0, off, prefix_lens=off[:3].float()), dtype),
        (lambda: B.packed_attn(pq, pk, pk, 1.0, off, slopes=torch.zeros(3)), shape), (lambda: B.packed_attn(pq, pk, pk, 1.0, off, slopes=torch.zeros(4).double()), dtype),
        (lambda: B.packed_attn(pq, pk, pk, 1.0, off, out=pq[:40]), shape), (lambda: B.packed_attn(pq, pk, pk, 1.0, off, out=pq.bfloat16()), dtype), (lambda: B.packed_attn(pq, pk, pk, 1.0, off), shape),
        (lambda: B.packed_attn(pq, pk, pk, 1.0, torch.zeros(8, dtype=torch.int32)[::2]), shape)]
    for i, (call, status) in enumerate(calls):
        with pytest.raises(B.PsError) as e:
            call()
        assert e.value.status == status, i
