"""Rules of the block operators (csrc/plan.h) on the CPU: every position, row and key is somebody's, scratch and LDS are what the kernels have."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2505_14741_amd import build

WRAPPERS = """
#include "plan.h"
extern "C" void gnorm(int positions, int channels, int groups, int bytes, int* out) {
    const ps::GroupNormPlan p = ps::group_norm_plan(positions, channels, groups, bytes);
    out[0] = p.cpg; out[1] = p.slice_groups; out[2] = p.slices; out[3] = p.chunks; out[4] = p.per;
}
extern "C" void cross(int bf16, int rows, int kv_len, int kv_heads, int head_dim, int* out) {
    const ps::CrossPlan p = ps::cross_plan(bf16 != 0, rows, kv_len, kv_heads, head_dim, 256);
    out[0] = p.block; out[1] = p.nsplit; out[2] = p.resident; out[3] = ps::cross_resident_key_bytes(head_dim); out[4] = ps::cross_v_pitch(head_dim);
}
extern "C" void fp8(int m, int n, int blocks, int split, int* out) {
    const ps::Fp8Plan p = ps::fp8_plan(m, n, blocks, split != 0, 256);
    out[0] = p.tile; out[1] = p.pieces; out[2] = ps::kFp8Tiles[p.tile].bm; out[3] = ps::kFp8Tiles[p.tile].bn;
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("block_rules")
    src, lib = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
    with open(src, "w") as f:
        f.write(WRAPPERS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, src, "-o", lib], check=True)
    return C.CDLL(lib)


def ask(fn, *a):
    out = (C.c_int * 5)()
    fn(*a, out)
    return list(out)


def log(r, lo, hi):
    return int(round(lo * (hi / lo) ** r.random()))


def test_group_norm_chunks_and_slices_cover_everything(rules):
    r = random.Random(1)
    sizes = [(1, 1, 1), (1 << 24, 65536, 1), (1 << 24, 65536, 65536), (1 << 24, 1, 1), (3, 65536, 32)]
    for _ in range(4000):
        groups = log(r, 1, 1024)
        sizes.append((log(r, 1, 1 << 24), groups * log(r, 1, 65536 // groups), groups))
    for positions, channels, groups in sizes:
        for size in (2, 4):
            cpg, slice_groups, slices, chunks, per = ask(rules.gnorm, positions, channels, groups, size)
            assert cpg * groups == channels and 1 <= slice_groups <= min(groups, 256)
            assert (slices - 1) * slice_groups < groups <= slices * slice_groups
            assert 1 <= chunks and (chunks - 1) * per < positions <= chunks * per     # no chunk is empty
            assert chunks == 1 or slices * chunks <= 512
            # the launcher: threads of a position, positions at a time, threads per group, partial moments in LDS
            for width in (1, 4, 8):
                if slice_groups * cpg % width:
                    continue
                for threads in ((1024,) if chunks == 1 else (256,)):
                    lanes = min(slice_groups * cpg // width, threads)
                    rows, fill = threads // lanes, 16 if lanes * width % 32 == 0 and lanes >= 8 else 0
                    assert (rows - 1) * (lanes * width + fill) + lanes * width <= threads * width + 2 * threads
                    inv = ((1 << 20) + lanes - 1) // lanes
                    assert all((t * inv & 0xFFFFFFFF) >> 20 == t // lanes and t * inv < 1 << 32 for t in (0, 1, lanes - 1, lanes, threads // 2, threads - 1))


def test_cross_attention_plans(rules):
    r = random.Random(2)
    cases = [(1, 1, 1), (1 << 30, 1 << 24, 1), (1, 1 << 24, 65535), (17550, 226, 30), (160, 17776, 6), (300, 0, 4)]
    cases += [(log(r, 1, 1 << 24), log(r, 1, 1 << 24), log(r, 1, 64)) for _ in range(4000)]
    for rows, kv_len, kv_heads in cases:
        for bf16 in (0, 1):
            for d in (16, 32, 64, 128):
                block, nsplit, resident, key_bytes, pitch = ask(rules.cross, bf16, rows, kv_len, kv_heads, d)
                assert block in ((64, 128, 192) if bf16 and d < 128 else (64,))
                tiles = (kv_len + 63) // 64
                assert nsplit == 1 or nsplit * 4 <= tiles                    # a piece has 4 tiles at least
                assert nsplit == 1 or nsplit * kv_heads * -(-rows // block) <= 2 * 256
                assert key_bytes == 2 * (d + 8 + pitch) + 4 and pitch >= d and pitch % 8 == 0
                if resident:
                    assert bf16 and d <= 64 and nsplit == 1 and rows >= 256
                    assert 2 * tiles * 64 * key_bytes <= 160 * 1024 and tiles <= 32      # two workgroups per compute unit; tiles fit a mask of 32


def test_products_of_blocks(rules):
    r = random.Random(3)
    cases = [(1, 1, 1), (1 << 24, 64, 1), (1, 1 << 24, 32768), (17776, 5760, 15), (4516, 1920, 60), (112, 7680, 15)]
    cases += [(log(r, 1, 1 << 20), log(r, 1, 1 << 16), log(r, 1, 32768)) for _ in range(4000)]
    for m, n, blocks in cases:
        whole, split = ask(rules.fp8, m, n, blocks, 0), ask(rules.fp8, m, n, blocks, 1)
        assert whole[1] == 1 and whole[0] == split[0]                        # pieces of the same tile
        if split[1] > 1:
            assert split[0] == 0 and split[1] >= 3 and blocks >= 8 * split[1] and split[1] * -(-m // 64) * -(-n // 64) <= 2 * 256
    # measured: the fastest tile or within a tenth of it
    picks = {(112, 7680, 15): (64, 64), (448, 7680, 15): (128, 128), (1100, 1920, 60): (128, 128), (1100, 5760, 15): (192, 192),
             (4516, 1920, 60): (192, 192), (4516, 7680, 15): (192, 256), (17776, 5760, 15): (192, 256), (17776, 1920, 60): (192, 256)}
    for shape, tile in picks.items():
        assert tuple(ask(rules.fp8, *shape, 0)[2:4]) == tile, shape
