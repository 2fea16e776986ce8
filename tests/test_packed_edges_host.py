"""Operators of self-attention on packed samples: what a call reserves and launches, by the rules that divide its work."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2505_14741_amd import binding as B
from paper_2505_14741_amd import build

# 12 samples of 32 key heads: enough workgroups for blocks of 256 rows; each of them alone is not
WIDE_HEADS = 32
WIDE_LENS = [1, 5, 300, 64, 0, 257, 513, 700, 31, 255, 130, 66]
WIDE_KEYS = [9, 1500, 2000, 64, 700, 1300, 513, 2500, 3000, 200, 5000, 1281]
# rows, outputs, k: every tile of the 4-bit product (in the order of plan.h), an even and an odd number of blocks of 128, whole and ragged sizes
PRODUCTS = [((2, 190, 1000), 0), ((190, 188, 300), 0), ((3585, 576, 2048), 1), ((3585, 578, 1900), 1), ((3601, 573, 2500), 1), ((3585, 1150, 1900), 2), ((3585, 1152, 2048), 2),
            ((4516, 1920, 7680), 3), ((3585, 1150, 7780), 3), ((4500, 1906, 7800), 3), ((3585, 1150, 7600), 3), ((3585, 2304, 1900), 4), ((3585, 2303, 2048), 4), ((3585, 2304, 100), 4),
            ((3585, 2304, 129), 4), ((3585, 2304, 300), 4)]
RULES = """
#include "plan.h"
extern "C" int pieces(int rows, int keys, int kv_heads) { return ps::packed_pieces(rows, keys, kv_heads); }
extern "C" long part_rows(int own, int samples, int rows, int kv_tokens, int kv_heads) { return ps::packed_part_rows(own != 0, samples, rows, kv_tokens, kv_heads); }
extern "C" int product_tile(int m, int n, int blocks, int split) { return ps::fp4_plan(m, n, blocks, split != 0, 256).tile; }
extern "C" void plan(int bf16, int own, int samples, int rows, int kv_tokens, int kv_heads, int head_dim, int most, long* out) {
    const ps::PackedPlan p = ps::packed_plan(bf16 != 0, own != 0, samples, rows, kv_tokens, kv_heads, head_dim, 256, most);
    out[0] = p.block; out[1] = p.slots; out[2] = p.part_rows; out[3] = (long)p.table_bytes; out[4] = (long)p.part_bytes; out[5] = ps::packed_workgroups(p.slots, kv_heads);
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("packed_edges")
    src, lib = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
    with open(src, "w") as f:
        f.write(RULES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, src, "-o", lib], check=True)
    r = C.CDLL(lib)
    r.part_rows.restype = C.c_long
    return r


def workspace(samples, q_tokens, kv_tokens, heads, kv_heads, d, dtype=1):
    s = B._PackedShape(samples, q_tokens, kv_tokens, heads, kv_heads, d, dtype, 1, 1, 1, 0.125, 0.0, heads * d, d, kv_heads * d, d, kv_heads * d, d, heads * d, d)
    return B.lib().packed_attn_workspace_bytes(C.byref(s))


# A token of 32 heads over 8 for each sample of 4096 keys: 4 pieces of 4 rows for each key head.  The bound holds for any samples of these sums: rows that lie in a
# few of them with all the keys have 64 pieces each, so 16 times what is used here.
@pytest.mark.parametrize("samples", [1, 8, 64, 65, 256, 1024])
def test_a_token_for_each_of_many_samples_reserves_little(rules, samples):
    used = samples * 4 * 4 * 8 * 132 * 4
    out = (C.c_long * 6)()
    rules.plan(1, 1, samples, 4 * samples, 4096 * samples, 8, 128, 256, out)
    assert used <= workspace(samples, samples, 4096 * samples, 32, 8, 128) <= 16 * used + 16 * out[1] + 4 * samples
    assert out[5] <= 4 * (samples * 4 * 8) + 64                          # workgroups: four times those that have work, at most


def test_rows_that_are_never_divided_reserve_little(rules):
    """17776 queries of 30 heads against as many keys: a sample of that size is not divided.  One of up to 4352 rows may be, in 4 pieces."""
    assert rules.pieces(17776, 17776, 30) == 1
    assert workspace(1, 17776, 17776, 30, 30, 64) <= 4 * 34 * 128 * 30 * 68 * 4 + 512
    out = (C.c_long * 6)()
    rules.plan(1, 1, 1, 17776, 17776, 30, 64, 256, out)
    assert out[1] <= 2 * 70


def test_rows_of_partial_sums_have_a_place(rules):
    """Samples of any lengths: their rows in all pieces are within what is reserved, and slots hold every block in every piece, whatever the block."""
    r = random.Random(3)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))  # noqa: E731
    out = (C.c_long * 6)()
    for _ in range(6000):
        kv_heads, share = r.choice([1, 2, 3, 6, 8, 30, 43, 64, 127, 128, 129, 200, 341, 512, 513, 600, 1023, 1024]), r.choice([1, 1, 4, 8, 33])
        n = r.choice([1, 1, 2, 8, 30, 70, 300])
        kind = r.choice(["any", "few", "units", "equal"])
        if kind == "few":
            q = [r.randint(0, 40 // share + 1) for _ in range(n)]
        elif kind == "units":
            q = [r.choice([1, 32, 33, 127, 128, 129, 256, 257, 1024, 2049]) for _ in range(n)]
        elif kind == "equal":
            q = [log(1, 5000)] * n
        else:
            q = [log(1, 30000) if r.random() < 0.3 else r.randint(0, 40) for _ in range(n)]
        top = r.choice([3000, 20000, 200000])
        k = [log(1, top) if r.random() < 0.6 else r.choice([0, 1279, 1280, 1281, 1536, 2047, 2048, 2560]) for _ in range(n)]
        rows, kv = sum(q) * share, sum(k)
        if rows == 0 or kv > 1 << 24 or (rows // 64 + n) * kv_heads > 1 << 19:
            continue
        total = sum(a * share * rules.pieces(a * share, b, kv_heads) for a, b in zip(q, k) if rules.pieces(a * share, b, kv_heads) > 1)
        assert total <= rules.part_rows(1, n, rows, kv, kv_heads) < 1 << 31, (q, k, kv_heads, share)
        for bf16, d, most in ((1, 64, 256), (1, 64, 128), (0, 32, 256)):
            rules.plan(bf16, 1, n, rows, kv, kv_heads, d, most, out)
            block, slots, part_rows, table, part, _ = list(out)
            assert block <= most
            assert sum(-(-a * share // block) * rules.pieces(a * share, b, kv_heads) for a, b in zip(q, k)) <= slots, (q, k, kv_heads, share, block)
            assert total * kv_heads * (d + 4) * 4 <= part or total == 0
            assert table >= (8 * (slots + 1) + 4 * n if n > 64 else 0)


def test_the_largest_calls_count_below_31_bits(rules):
    out = (C.c_long * 6)()
    for kv_heads in (1, 2, 8, 64, 512, 1024):
        for n in (1, 100, 13107, 65535):
            for rows in (n, 33 * n, 129 * n, 64 * ((1 << 19) // kv_heads - n)):
                if rows < 1 or (rows // 64 + n) * kv_heads > 1 << 19:
                    continue
                assert rules.part_rows(1, n, rows, 1 << 24, kv_heads) < 1 << 30
                for bf16 in (0, 1):
                    rules.plan(bf16, 1, n, rows, 1 << 24, kv_heads, 16, 256, out)
                    assert out[5] < 1 << 24


def test_blocks_of_256_rows_are_taken_where_their_tests_expect_them(rules):
    out = (C.c_long * 6)()
    for d in (16, 32, 64):
        rules.plan(1, 0, 12, sum(WIDE_LENS), sum(WIDE_LENS), WIDE_HEADS, d, 256, out)
        assert out[0] == 256
        rules.plan(1, 1, 12, sum(WIDE_LENS), sum(WIDE_KEYS), WIDE_HEADS, d, 256, out)
        assert out[0] == 256
        for n in WIDE_LENS:
            rules.plan(1, 1, 1, n, max(WIDE_KEYS), WIDE_HEADS, d, 256, out)
            assert out[0] == 128
    divided = {rules.pieces(a, b, WIDE_HEADS) for a, b in zip(WIDE_LENS, WIDE_KEYS)}
    assert 1 in divided and divided & {2, 3, 4} and max(divided) > 4


def test_products_take_the_tiles_their_tests_expect(rules):
    for (m, n, k), tile in PRODUCTS:
        for split in (0, 1):
            assert rules.product_tile(m, n, (k + 127) // 128, split) == tile, (m, n, k)
    for tile in range(5):
        assert {(k + 127) // 128 % 2 for (_, _, k), t in PRODUCTS if t == tile} == {0, 1}
