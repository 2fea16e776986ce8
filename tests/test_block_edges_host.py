"""Operators of a conditioned predictor block, without a GPU: what the compiler is told of addresses, limits of launches, what is refused at the
ends of the ranges."""
import ctypes as C
import os
import random
import re
import subprocess

import pytest

from paper_2505_14741_amd import binding as B
from paper_2505_14741_amd import build

FAKE = 0x10000                                                   # never dereferenced: what is called with it is refused
# 8-bit products (rows, columns, k) for each tile: last tiles that are partial in either direction, columns that no 16-byte store divides, one
# block of k, two, three, a last one that is partial, and many.  test_gpu_block_edges.py computes them.
PRODUCTS = {
    (64, 64): [(1, 65, 100), (70, 1004, 129), (129, 257, 300), (112, 2050, 1920), (33, 130, 7680)],
    (128, 128): [(1100, 1920, 100), (1100, 1921, 129), (4600, 516, 300), (1037, 1924, 1920), (1100, 1920, 7680)],
    (192, 192): [(2500, 2052, 100), (2500, 2050, 129), (4600, 1920, 300), (4516, 1917, 1920), (4600, 1908, 7680)],
    (192, 256): [(4600, 2052, 100), (4600, 2300, 129), (4600, 2052, 256), (4600, 2301, 300), (4600, 2300, 500), (3500, 5760, 1920), (9000, 1003, 1920)],
}
WRAPPERS = """
#include "plan.h"
extern "C" long quantize_workgroups(int rows, int cols) { return ps::quantize_workgroups(rows, cols); }
extern "C" bool cross_rows_fit(int batch, long rows, int kv_heads) { return ps::cross_rows_fit(batch, rows, kv_heads); }
extern "C" void cross(int rows, int kv_len, int kv_heads, int head_dim, int* out) {
    out[0] = ps::cross_plan(true, rows, kv_len, kv_heads, head_dim, 256).block;
}
extern "C" long cross_x(int bf16, int rows, int kv_len, int kv_heads, int head_dim) {
    const ps::CrossPlan p = ps::cross_plan(bf16 != 0, rows, kv_len, kv_heads, head_dim, 256);
    return (long)kv_heads * p.nsplit * ((rows + (long)p.block - 1) / p.block);
}
extern "C" void fp8(int m, int n, int blocks, int* out) {
    const ps::Fp8Plan p = ps::fp8_plan(m, n, blocks, false, 256);
    out[0] = ps::kFp8Tiles[p.tile].bm; out[1] = ps::kFp8Tiles[p.tile].bn;
}
extern "C" int fp8_tiles() { return ps::FP8_TILES; }
extern "C" bool pieces_meet(long a, long n, long b, long m, long width) { return ps::pieces_meet(a, n, b, m, width); }
extern "C" bool grid_fits(long workgroups, int threads) { return ps::grid_fits(workgroups, threads); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("edge_rules")
    src, lib = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
    with open(src, "w") as f:
        f.write(WRAPPERS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, src, "-o", lib], check=True)
    r = C.CDLL(lib)
    r.quantize_workgroups.restype, r.grid_fits.restype, r.grid_fits.argtypes = C.c_long, C.c_bool, [C.c_long, C.c_int]
    r.cross_rows_fit.restype, r.cross_rows_fit.argtypes, r.cross_x.restype = C.c_bool, [C.c_int, C.c_long, C.c_int], C.c_long
    r.pieces_meet.restype, r.pieces_meet.argtypes = C.c_bool, [C.c_long] * 5
    return r


def test_group_norm_accesses_promise_no_alignment_beyond_an_element():
    """x, out, gamma and beta may lie at any element's address: wide loads and stores of them, kept in L2 or not, must say so to the compiler."""
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm", os.path.join(build.CSRC, "group_norm.hip"), "-o", "-"],
                       capture_output=True, text=True, check=True)
    size = {"bfloat": 2, "float": 4}
    seen = set()
    for line in r.stdout.splitlines():
        for kind, pattern in (("store", r"store <(\d+) x (\w+)> [^,]*, (?:ptr|ptr addrspace\(1\)) \S+, align (\d+)"),
                              ("load", r"load <(\d+) x (\w+)>, (?:ptr|ptr addrspace\(1\)) \S+, align (\d+)")):
            m = re.search(pattern, line)
            if m and m.group(2) in size:
                assert int(m.group(3)) == size[m.group(2)], line
                seen.add((kind, m.group(1), m.group(2), "nontemporal" in line))
    for kind, count, elem, streamed in [(k, n, e, s) for n, e in (("8", "bfloat"), ("4", "bfloat"), ("4", "float"))
                                        for k, s in (("load", False), ("store", False), ("store", True))]:
        assert (kind, count, elem, streamed) in seen


def test_quantizer_launches_fit(rules):
    """Blocks are rounded up to whole workgroups of 16; their threads stay below 2^32, the sizes that would not are refused."""
    fits = lambda rows, blocks: rules.grid_fits(rules.quantize_workgroups(rows, blocks * 128), 256)  # noqa: E731
    assert rules.quantize_workgroups(1, 1) == 1 and rules.quantize_workgroups(16, 128) == 1 and rules.quantize_workgroups(17, 128) == 2
    assert rules.quantize_workgroups((1 << 24) - 1, 2048) * 256 == (1 << 32) - 256
    for rows, blocks, ok in (((1 << 24) - 1, 16, True), (1 << 24, 15, True), (16384, 16383, True), (16385, 16383, False), (1 << 24, 16, False)):
        assert fits(rows, blocks) == ok
        if not ok:
            assert B.lib().fp8_quantize(FAKE, 2 * FAKE, 3 * FAKE, rows, blocks * 128, blocks * 128, 1, None) == -2


def test_cross_attention_launches_fit(rules):
    """Every shape that is accepted has fewer than 2^32 threads in x, and at most 65535 samples in z; the last accepted and first refused."""
    r = random.Random(4)
    for batch, rows, kv_heads, ok in ((512, 1, 65535, True), (513, 1, 65535, False), (1, 1 << 29, 1, True), (1, (1 << 29) + 1, 1, False), (1, 8192, 65535, True),
                                      (1, 8193, 65535, False), (65535, 1, 512, True), (65535, 16, 512, True), (65535, 17, 512, False)):
        assert rules.cross_rows_fit(batch, rows, kv_heads) == ok
        if not ok and rows < 1 << 24:
            width = kv_heads * 16
            s = B._CrossShape(batch=batch, q_len=rows, kv_len=1, heads=kv_heads, kv_heads=kv_heads, head_dim=16, dtype=1, scale=1.0, q_batch=rows * width,
                              q_token=width, q_head=16, k_batch=width, k_token=width, k_head=16, v_batch=width, v_token=width, v_head=16, o_batch=rows * width,
                              o_token=width, o_head=16)
            assert B.lib().cross_attn(FAKE, 2 * FAKE, 3 * FAKE, None, None, 4 * FAKE, C.byref(s), None, 0, None) == -2
    tried = 0
    while tried < 3000:
        kv_heads, batch = int(2 ** r.uniform(0, 16)) & 65535 or 1, int(2 ** r.uniform(0, 10))
        rows = max(1, int((1 << 29) / kv_heads / batch * 2 ** r.uniform(-1, 0.1))) if r.random() < 0.5 else int(2 ** r.uniform(0, 30))
        if not rules.cross_rows_fit(batch, rows, kv_heads):
            continue
        tried += 1
        for bf16 in (0, 1):
            for d in (16, 64, 128):
                kv_len = int(2 ** r.uniform(0, 24))
                assert rules.grid_fits(rules.cross_x(bf16, rows, kv_len, kv_heads, d), 256), (rows, kv_heads, kv_len, d)


def test_the_library_holds_the_attention_kernels_that_the_rule_picks(rules):
    """Rows per workgroup of the bf16 kernel by head size, over all sizes: each one's kernel is built, and no other."""
    out, picked = (C.c_int * 5)(), set()
    for d in (16, 32, 64, 128):
        for rows in list(range(1, 800)) + [1 << n for n in range(10, 30)]:
            for kv_len in (64, 4096):
                rules.cross(rows, kv_len, 30, d, out)
                picked.add((d, out[0] // 64))
    with open(build.LIB, "rb") as f:
        lib = f.read()
    for d in (16, 32, 64, 128):
        for tiles in (1, 2, 3, 4):
            assert (b"cross_bf16_kernelILi%dELi%dEE" % (d, tiles) in lib) == ((d, tiles) in picked), (d, tiles)


def test_tested_products_take_every_tile(rules):
    assert len(PRODUCTS) == rules.fp8_tiles()
    out = (C.c_int * 2)()
    for tile, shapes in PRODUCTS.items():
        for m, n, k in shapes:
            rules.fp8(m, n, (k + 127) // 128, out)
            assert tuple(out) == tile, (m, n, k)


def test_pieces_that_meet(rules):
    """Against the pieces counted one by one; and at extents and strides as large as they may be, which take no time."""
    r = random.Random(5)
    met = 0
    for _ in range(20000):
        width, n, m = r.randint(1, 6), r.randint(1, 7), r.randint(1, 7)
        a, b = r.randint(0, 40), r.randint(0, 40)
        at = sorted(i * a + j * b for i in range(n) for j in range(m))
        want = any(y - x < width for x, y in zip(at, at[1:]))
        met += want
        assert rules.pieces_meet(a, n, b, m, width) == want, (a, n, b, m, width)
    assert 2000 < met < 18000
    far = 1 << 40
    for a, n, b, m, width, want in ((far, 65535, 64, 1 << 24, 64, False), (far, 65535, far, 1 << 24, 64, True), (far, 65535, far - 64, 1 << 24, 128, True),
                                    (64, 65535, 64 * 65535, 1 << 24, 64, False), (64, 65535, 64 * 65534, 1 << 24, 64, True)):
        assert rules.pieces_meet(a, n, b, m, width) == want and rules.pieces_meet(b, m, a, n, width) == want


@pytest.mark.parametrize("over", [dict(o_head=32), dict(o_token=128), dict(o_token=64, o_head=64), dict(o_batch=256, o_token=256), dict(o_batch=64),
                                  dict(o_batch=128, o_token=640, o_head=160), dict(q_len=1, o_batch=192)])
def test_cross_attention_refuses_an_output_whose_heads_overlap(over):
    s = dict(batch=2, q_len=5, kv_len=7, heads=4, kv_heads=2, head_dim=64, dtype=1, scale=0.125, q_batch=1280, q_token=256, q_head=64, k_batch=896, k_token=128, k_head=64,
             v_batch=896, v_token=128, v_head=64, o_batch=1280, o_token=256, o_head=64)
    s.update(over)
    assert B.lib().cross_attn(FAKE, 2 * FAKE, 3 * FAKE, None, None, 4 * FAKE, C.byref(B._CrossShape(**s)), None, 0, None) == -2


@pytest.mark.parametrize("over", [dict(out_batch=64), dict(out_batch=128, out_position=64), dict(out_batch=64, out_position=64), dict(out_batch=128, out_position=160)])
def test_group_norm_refuses_an_output_whose_positions_overlap(over):
    s = dict(batch=2, positions=5, channels=64, groups=8, act=0, dtype=1, eps=1e-5, x_batch=320, x_position=64, out_batch=320, out_position=64)
    s.update(over)
    assert B.lib().group_norm(FAKE, None, None, 2 * FAKE, C.byref(B._GroupNormShape(**s)), None, 0, None) == -2


def test_binding_refuses_sizes_that_do_not_fit_the_library():
    """Extents, groups and activations of 2^31 and more, which ctypes would cut to 32 bits (tensors without memory)."""
    import torch
    far = (1 << 32) + 5
    meta = lambda *s, dtype=torch.bfloat16: torch.empty(1, dtype=dtype, device="meta").as_strided(s, (8 * far,) * (len(s) - 1) + (1,))  # noqa: E731
    q, x, bias = meta(1, 4, 2, 64), torch.empty(1, 4, 64, device="meta"), torch.empty(4, device="meta")
    e4, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    q8 = lambda rows, k: (torch.empty(rows, k, dtype=e4, device="meta"), torch.empty(k // 128, (rows + 15) // 16 * 16, dtype=e8, device="meta"))  # noqa: E731
    calls = [(lambda: B.cross_attn(q, meta(1, far, 2, 64), meta(1, far, 2, 64), 1.0), "2\\^31"),
             (lambda: B.cross_attn(meta(1, far, 2, 64), q, q, 1.0), "2\\^31"),
             (lambda: B.fp8_quantize(meta(1, far)), "2\\^31"), (lambda: B.fp8_quantize(meta(far, 64)), "2\\^31"),
             (lambda: B.dit_linear_fp8(*q8(4, 1 << 33), *q8(4, 1 << 33), bias), "2\\^31"),
             (lambda: B.dit_linear_fp8(*q8(1 << 32, 128), *q8(4, 128), bias), "2\\^31"),
             (lambda: B.dit_linear_fp8(*q8(4, 128), *q8(4, 128), bias, act=1 << 32), "act"),
             (lambda: B.group_norm(torch.empty(1, far, 64, device="meta"), 8), "2\\^31"),
             (lambda: B.group_norm(x, (1 << 32) + 8), "groups"), (lambda: B.group_norm(x, 8, act=1 << 32), "act")]
    for i, (call, why) in enumerate(calls):
        with pytest.raises(B.PsError, match=why) as e:
            call()
        assert e.value.status == -2, i


def test_cross_attention_scale():
    """A scale is refused from where its product with log2(e) is not finite in fp32: a score of zero would be NaN under it."""
    s = lambda scale: B._CrossShape(batch=1, q_len=1, kv_len=100000, heads=1, kv_heads=1, head_dim=64, dtype=1, scale=scale, q_batch=64, q_token=64, q_head=64,  # noqa: E731
                                    k_batch=64, k_token=64, k_head=64, v_batch=64, v_token=64, v_head=64, o_batch=64, o_token=64, o_head=64)
    for scale, ok in ((2.0 ** -149, True), (2.358e38, True), (2.359e38, False), (3.4e38, False)):
        assert (B.lib().cross_attn_workspace_bytes(C.byref(s(scale))) > 0) == ok, scale
        assert B.lib().cross_attn(FAKE, 2 * FAKE, 3 * FAKE, None, None, 4 * FAKE, C.byref(s(scale)), None, 0, None) == (-4 if ok else -2)
