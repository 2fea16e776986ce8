// Rules that say which thread or workgroup computes what: plain arithmetic on sizes, without device code, so that a host
// program can evaluate them at sizes no test can run.  (constexpr functions are callable from kernels as they are.)
#pragma once

#include <stddef.h>

namespace ps {

// ---- merge of attention's key pieces: 16 threads per query row, 16 rows per workgroup of 256
struct MergeRow { int item, row, d4; };              // split item (over all samples), its row, group of 4 outputs
// Counted in rows: a launch holds fewer than 2^32 threads, i.e. fewer than 2^28 rows, so a row index fits 32 bits where a
// thread index does not (524800 items of 256 rows are 2^31 + 2 * 10^6 threads).
constexpr MergeRow merge_row(int block, int thread, int bq) {
    const int rowid = block * 16 + (thread >> 4);
    return MergeRow{rowid / bq, rowid % bq, thread & 15};
}

// ---- bf16 attention of samples whose items of 256 queries do not fill the chip: whether workgroups of 128 queries, alone, are
// faster than workgroups of 256 and the launch that looks their results through.  `bh`: (batch, head) pairs.
// Measured us per tile of 64 keys: 512 workgroups of 128 queries 1.25, up to 256 of them 0.98; of 256 queries 2.27 and 1.29; a
// single round that puts two on some compute units only is between them, nearer the full one.  A launch more costs 4 us; over
// several rounds the narrow ones, which read K and V twice as often, lose another 6 %.  Whole calls, narrow / wide us: 30 heads,
// 1000 keys, 4 and 8 samples 46.8 / 48.5 and 87.7 / 85.2, 2608 keys 88 / 90, two samples 131 / 130, four 245 / 243, 3600 keys 135 / 117;
// 16 heads, 3000 keys 59 / 60, 4200 keys 127 / 119; 4 heads, 6000 keys 84 / 107, 17776 keys 503 / 461.
// (On 278 shapes of 32 to 17776 keys and 1 to 3200 (batch, head) pairs the one picked is 3.2 % slower than the other at most.)
constexpr bool attn_narrow_items(long bh, int seq, int cus) {
    const long slots = 2L * cus, narrow = bh * ((seq + 127) / 128), wide = bh * ((seq + 255) / 256);
    const auto rounds = [slots, cus](long n, float full, float half) {
        const long tail = n % slots;
        if (n < slots && tail > cus) return full * (0.92f + 0.08f * (float)(tail - cus) / cus);
        return (float)(n / slots) * full + (tail == 0 ? 0.f : tail <= cus ? half : full);
    };
    const float tiles = (float)((seq + 63) / 64);
    const float a = tiles * rounds(narrow, 1.25f, 0.98f) * (narrow > 2 * slots ? 1.06f : 1.f);
    return a <= tiles * rounds(wide, 2.27f, 1.29f) + 4.f;
}

// Split plan of the bf16 head-dim-64 kernels: per sample, how many work items of 256 queries run whole and how many ways the
// rest is split along the keys.
struct AttnPlan { int qblocks, items_ps, full_ps, tail_ps, nsplit, bq; };
constexpr AttnPlan attention_plan(int seq, int heads, int cus) {
    constexpr int KV = 64;
    AttnPlan p{};
    p.bq = 256;
    p.qblocks = (seq + p.bq - 1) / p.bq;
    p.items_ps = p.qblocks * heads;
    const int slots = cus * 2;                           // two resident workgroups per CU
    const int tail = p.items_ps % slots;
    const int ntiles = (seq + KV - 1) / KV;
    // Fewer items than slots are never split: the plan must not depend on the batch, and a batch that fills the chip by
    // itself pays 70 KB of partial sums per piece for nothing.  (4 heads x 4096 keys in two pieces: 74 -> 49 us alone, but
    // 80 -> 94 for four samples and 256 -> 330 for sixteen; 16 heads x 1000 keys, four samples: 30 -> 50.)
    int ns = tail > 0 ? slots / tail : 1;
    if (ns > 8) ns = 8;
    if (ns > ntiles / 2) ns = ntiles / 2;
    if (tail == 0 || p.items_ps < slots || ns < 2) { p.full_ps = p.items_ps; p.tail_ps = 0; p.nsplit = 1; }
    else { p.full_ps = p.items_ps - tail; p.tail_ps = tail; p.nsplit = ns; }
    return p;
}

// Which kernels a bf16 head-dim-64 call takes.
//   ATTN_BY_128   attn_sp_kernel alone, 128 queries per workgroup, which redoes its own failures
//   ATTN_BY_256   attn_sp_kernel with 256 queries per workgroup, then attn_redo_kernel
//   ATTN_FLAGS    attn_sp_kernel marks the (batch, head) pairs it could not do, attn_mfma_kernel redoes those; key pieces
//   ATTN_TRACKED  attn_mfma_kernel for every head
// Samples whose items do not fill the chip take one of the first two: no split, no flags; the values of the two are the same,
// so the whole batch may decide between them.  Which samples these are must not depend on the batch, and a large batch of short
// ones is slower so than it was on attn_mfma_kernel alone: 30 heads x 512 keys, 16 samples 49.2 -> 51.4 us, 200 keys 22.5 ->
// 23.9 (one sample 17.7 -> 12.6 and 12.1 -> 8.7).
// Samples of 512 items and more (256 heads and more) of up to 512 keys: the second launch of ATTN_FLAGS costs more than the
// faster loop gains.
// path: kernel path (low byte 3: ATTN_TRACKED always).
enum AttnRoute { ATTN_BY_128, ATTN_BY_256, ATTN_FLAGS, ATTN_TRACKED };
constexpr AttnRoute attention_route(int batch, int seq, int heads, int path, int cus) {
    if ((path & 0xff) == 3) return ATTN_TRACKED;
    if (attention_plan(seq, heads, cus).items_ps < cus * 2)
        return attn_narrow_items((long)batch * heads, seq, cus) ? ATTN_BY_128 : ATTN_BY_256;
    return seq > 512 ? ATTN_FLAGS : ATTN_TRACKED;
}

// ---- projections: C[rows, Nn] = A[rows, K] * W[Nn, K]^T, rows = all samples of the batch
// Output tiles of the matrix kernels: gemm_few.hip (any K pieces; fp32 and bf16) and gemm_mfma.hip (bf16).
enum TileId { FEW_64x64, FEW_128x64, FEW_128x128, FEW_192x128, FEW_256x128, FEW_192x192, FEW_TILE_KINDS,
              WIDE_256x256 = FEW_TILE_KINDS, WIDE_128x128, WIDE_192x256, WIDE_192x128, TILE_KINDS };
// Us of a round of workgroups, one tile each: fixed + stages of 64 k * stage.  per_cu = 2: two workgroups share a CU; `half`: a
// round that leaves at most one to each.  (Fitted to bf16, operands that change from call to call, 32 to 9000 rows x 1920 to 7680
// columns x K = 1920 and 7680, with loops that had branches in a stage: all tiles are 2 to 13 % faster now, in the same order.)
// gated: what an epilogue that reads and writes an fp32 residual adds to a round (17776 rows x 1920, K = 1920, then 184, 170,
// 164 and 168 us on the tiles of gemm_mfma.hip in their order below, now 184, 162, 160 and 170).
struct Tile { int bm, bn, per_cu; float half_fixed, half_stage, fixed, stage, gated; };
constexpr Tile kTiles[TILE_KINDS] = {
    {64, 64, 2, 3.0f, 0.235f, 4.5f, 0.40f, 1.9f},        // 8 waves of 16 x 32
    {128, 64, 1, 0.f, 0.f, 4.0f, 0.30f, 1.9f},           // 8 waves of 32 x 32
    {128, 128, 1, 0.f, 0.f, 6.0f, 0.47f, 3.8f},          // 8 waves of 32 x 64
    {192, 128, 1, 0.f, 0.f, 7.0f, 0.60f, 5.7f},          // 8 waves of 48 x 64
    {256, 128, 1, 0.f, 0.f, 8.7f, 0.76f, 7.5f},          // 8 waves of 64 x 64
    {192, 192, 1, 0.f, 0.f, 10.f, 0.90f, 7.5f},          // 8 waves of 48 x 96
    {256, 256, 1, 0.f, 0.f, 7.3f, 1.34f, 15.f},          // gemm_mfma.hip: 8 waves of 128 x 64
    {128, 128, 2, 2.0f, 0.80f, 4.0f, 0.92f, 7.5f},       // 4 waves of 64 x 64
    {192, 256, 1, 0.f, 0.f, 5.4f, 1.14f, 14.6f},         // 8 waves of 96 x 64
    {192, 128, 2, 4.2f, 0.88f, 6.0f, 1.34f, 13.f},       // 4 waves of 96 x 64
};
constexpr long tile_count(int id, long rows, int Nn) {
    return (rows + kTiles[id].bm - 1) / kTiles[id].bm * ((Nn + kTiles[id].bn - 1) / kTiles[id].bn);
}
// Estimated us of `wgs` workgroups of `stages` stages each on `cus` compute units (without what launching takes).
constexpr float tile_time(int id, long wgs, float stages, bool gated, int cus) {
    const Tile& t = kTiles[id];
    const long slots = (long)cus * t.per_cu, tail = wgs % slots;
    const float epi = gated ? t.gated : 0.f;
    // (gemm_few.hip over more than two rounds: the chip at its power limit, and its smaller wave tiles read more LDS per
    // product: 41728 rows, 1920 x 7680 on 256 x 128 tiles 1323 us, on 192 x 256 of gemm_mfma.hip 1229)
    const float many = id < FEW_TILE_KINDS && wgs > 2 * slots ? 1.15f : 1.f;
    const float full = many * (t.fixed + stages * t.stage) + epi;
    const float half = t.half_fixed + stages * t.half_stage + 0.5f * epi;
    float last = tail == 0 ? 0.f : full;
    if (t.per_cu == 2 && tail > 0) {                     // two per CU do not start a last round together
        const float share = (float)(tail <= cus ? tail : tail - cus) / cus;
        if (wgs < slots) last = tail <= cus ? half : 0.9f * full;
        else last = tail <= cus ? half * (0.5f + 0.5f * share) : half + (full - half) * share;
    }
    return (float)(wgs / slots) * full + last;
}
// The bf16 tile with the least estimated time: `pieces` workgroups per tile along K; [first, last]: the kinds to choose from.
// Inside the network, 28 token counts from 64 to 33976 x the four projections of a layer, those that are not cut into pieces, the
// one picked is 0.8 % slower than the fastest on average, and 6 % at most but for QKV and fc1 at 1024 tokens (128 x 128 of
// gemm_mfma.hip 41.0 and 39.6 us, 256 x 128 here 35.9 and 32.3).
constexpr int best_tile(int first, int last, long rows, int Nn, int K, int pieces, bool gated, int cus) {
    int best = first;
    float least = 0.f;
    for (int id = first; id <= last; ++id) {
        const float t = tile_time(id, tile_count(id, rows, Nn) * pieces, (float)(K / 64) / pieces, gated, cus);
        if (id == first || t < least) { best = id; least = t; }
    }
    return best;
}

// ---- bf16 projections on the tiles of gemm_mfma.hip
// How a sample's [tokens, Nn] output is spread over the chip: which tile, how many tiles run whole and how the rest is
// split along K.  A function of the sample's shape only (never of the batch): see gemm_mfma_kernel.
struct GemmPlan { int tile, tiles_m, tiles_n, full, tail, nsplit; size_t ws_bytes_per_sample; };

// the K split of the last partial round: pieces per tail tile (1: none)
constexpr int gemm_tail_split(long tiles, long slots, int K, bool allow_split) {
    const long tail = tiles % slots, nk = K / 64;
    if (!allow_split || K < 4096 || tail == 0) return 1;
    long ns = slots / tail;
    if (ns > 8) ns = 8;
    if (ns > nk / 2) ns = nk / 2;
    return ns >= 2 ? (int)ns : 1;
}

// pieces > 0: every tile is summed in that many K pieces (1: whole), which the caller has fixed for the sample's shape.
constexpr GemmPlan gemm_plan(int tokens, int Nn, int K, bool allow_split, int forced_variant, int pieces, int cus) {
    GemmPlan p{};
    const auto slots_of = [cus](int tile) { return (long)cus * kTiles[tile].per_cu; };
    if (forced_variant >= 1 && forced_variant <= 4) {
        p.tile = WIDE_256x256 + forced_variant - 1;
    } else {
        // (for the kind of epilogue that follows a long K, whichever the call's is: the plan belongs to the shape)
        p.tile = best_tile(0, TILE_KINDS - 1, tokens, Nn, K, 1, true, cus);
        float best = tile_time(p.tile, tile_count(p.tile, tokens, Nn), (float)(K / 64), true, cus);
        // The last partial round of a long K in pieces, which count as 1/pieces of a round plus a third of one for the
        // partial sums (two passes over tile-size fp32 per piece) and the second launch -- measured at 17776 tokens: worth
        // it with a long K (1920 x 7680: 0.62 -> 0.57 ms on 128 x 128 tiles), not with K = 1920 (0.188 -> 0.196 ms); 1920 x
        // 7680 at 13000 rows: 192 x 256 tiles in two rounds and 32 tiles of 8 pieces 351 us, 192 x 128 whole 332
        bool split = false;
        for (int id = WIDE_256x256; id < TILE_KINDS && pieces == 0; ++id) {
            const long tiles = tile_count(id, tokens, Nn), slots = slots_of(id);
            const int ns = gemm_tail_split(tiles, slots, K, allow_split);
            if (ns == 1 || tiles < slots) continue;
            const float t = tile_time(id, slots, (float)(K / 64), true, cus) * (tiles / slots + 1.0f / ns + 0.35f);
            if (t < best) { best = t; p.tile = id; split = true; }
        }
        allow_split = split;
    }
    const Tile& t = kTiles[p.tile];
    p.tiles_m = (tokens + t.bm - 1) / t.bm;
    p.tiles_n = (Nn + t.bn - 1) / t.bn;
    const int tiles = p.tiles_m * p.tiles_n;
    p.nsplit = pieces > 0 ? pieces : gemm_tail_split(tiles, slots_of(p.tile), K, allow_split);
    p.tail = p.nsplit == 1 ? 0 : pieces > 0 ? tiles : (int)(tiles % slots_of(p.tile));
    p.full = tiles - p.tail;
    p.ws_bytes_per_sample = (size_t)p.tail * p.nsplit * t.bm * t.bn * sizeof(float);
    return p;
}

// The stages of a tile of gemm_mfma.hip are compiled in forms, one per number of stages that are left behind them; the largest
// form is the steady state and serves every larger number.  strips: the tile requests its residual ahead, strip 0 with two
// stages left and strip 1 with one, so the form of two must be the third-last stage alone.  (With rings of two stages and the
// form of two as the steady state, strip 0 was read again in every stage, as many bytes as both operands.  1920 x 1920 gated on
// 128 x 128 tiles inside the network, us, so / now: 3400 tokens 53.3 / 36.4, 8400 102 / 72.6, 17000 211 / 147, 33976 424 / 297.)
constexpr int steady_form(int deep, bool strips) { return strips && deep < 3 ? 3 : deep; }
constexpr int strip_of_form(int form) { return form == 2 ? 0 : form == 1 ? 1 : -1; }

// Longest operand rows of the matrix kernels.  A load's offset inside a tile's rows is 32 bits: 256 rows at most, and 64 on the
// 64 x 64 tile of gemm_few.hip, which takes the rows that are longer than the others do.  (Bases of eight rows, which any
// tile could use, cost 0.4 to 1 % of every forward.  64 rows x 64 columns, K = 2^22 + 64 in bf16 2.4 ms, 480 on the FMA kernel.)
constexpr long ANY_TILE_ROW_BYTES = 1L << 23, TILE_64_ROW_BYTES = 1L << 26;

// ---- projections of few tokens and of fp32 operands (gemm_few.hip)
constexpr int FEW_ROW_BYTES = 128;                       // bytes of an operand row per stage: 64 bf16 or 32 fp32

// Whether `pieces` workgroups per tile are one round, a compute unit each, on some tile of gemm_few.hip.
constexpr int FEW_CUS = 256;                             // (a plan must not depend on the device's count)
constexpr bool few_one_round(long rows, int Nn, int pieces) {
    for (int id = 0; id < FEW_TILE_KINDS; ++id)
        if (tile_count(id, rows, Nn) * pieces <= FEW_CUS) return true;
    return false;
}
// K pieces of a sample of more than 128 tokens and a long K (bf16): 4 or 3, whichever is estimated faster, where that is one
// round; 3 on 192 x 192 tiles excepted.  1920 x 7680, weights from memory, us apart / one workgroup per tile: 450 tokens 27.6 /
// 36.1, 768 35.7 / 49.2, 800 39.0 / 42.6, 960 42.5 / 44.4, 1024 42.7 / 49.5, 1100 45.0 / 65, 1200 49.8 / 62, 1280 49.6 / 68.5.
// From 1281 tokens on (3 pieces, 192 x 192: 1400 53.2 / 68) a batch would lose more than that: its pieces stay on tiles of
// gemm_few.hip, four samples of 1500 168 us, on wider tiles whole 146.  (Up to there it loses little: a layer of one sample
// of 1104 / 1264 tokens, whole and in pieces, 212 -> 188 / 225 -> 201 us, of four 475 -> 478 / 557 -> 569, of six 722 -> 740
// / 761 -> 779; two layers of twelve of 1264 3150 -> 3340, of sixteen 4210 -> 4330.)
constexpr int few_long_pieces(int tokens, int Nn, int nk) {
    int best = 1;
    float least = 0.f;
    for (int n = 4; n >= 3; --n)
        for (int id = 0; id < (n == 4 ? (int)FEW_TILE_KINDS : (int)FEW_192x192); ++id) {
            const long wgs = tile_count(id, tokens, Nn) * n;
            if (wgs > FEW_CUS) continue;
            const float t = tile_time(id, wgs, (float)nk / n, false, FEW_CUS);
            if (best == 1 || t < least) { best = n; least = t; }
        }
    return best;
}

// A sample's plan: a function of the sample's shape alone, so that its result does not depend on the batch.  tiles_m x
// tiles_n tiles of 64 x 64.
//   bf16: up to 640 of them, 512 with K >= 4096, where a sample is cut into K pieces that wider tiles would also need, and
//     beyond as long as it is cut, or its operand rows are longer than wider tiles take.
//   fp32: every size (the matrix instructions bind, 32 cycles per 2048 operations, not the LDS reads).
// K pieces, short K: as many as bring the workgroups to 256 (one per compute unit), 8 at most (fp32 16) and each at least 5
// stages.  1920 x 1920 bf16 at 112 tokens (60 tiles), without / with the launch that adds them: 1 piece 10.3 us, 4 pieces
// 5.8 / 9.7, 8 pieces 6.2 / 11.1.
// Long K (60 stages and more), fp32 and up to 128 tokens: to 512.  1920 x 7680 bf16 at 112 tokens: 8 pieces (128 x 64
// tiles) 15.2, 4 pieces 16.1, 3 pieces 18.9.  More tokens: few_long_pieces().
// path: kernel path (low byte 1: generic kernels, 4: no K pieces).
struct FewPlan { bool use; int tiles_m, tiles_n, nsplit; };
constexpr FewPlan few_plan(bool bf16, int tokens, int Nn, int K, int path) {
    FewPlan p{false, 0, 0, 1};
    const long row_bytes = (long)K * (bf16 ? 2 : 4);
    if ((path & 0xff) == 1 || row_bytes % FEW_ROW_BYTES != 0 || row_bytes > TILE_64_ROW_BYTES || Nn % 4 != 0 || tokens < 1) return p;
    p.tiles_m = (tokens + 63) / 64;
    p.tiles_n = (Nn + 63) / 64;
    const long tiles = (long)p.tiles_m * p.tiles_n, nk = row_bytes / FEW_ROW_BYTES;
    if (bf16 && Nn < 64) return p;
    const long most = bf16 ? 8 : 16;
    long ns = (nk >= 60 ? 512 : 256) / tiles;
    if (bf16 && nk >= 60 && tokens > 128) ns = few_long_pieces(tokens, Nn, (int)nk);
    if ((path & 0xff) == 4) ns = 1;
    if (bf16 && ns <= 1 && tiles > (K >= 4096 ? 512 : 640) && row_bytes <= ANY_TILE_ROW_BYTES) return p;
    p.use = true;
    ns = ns < most ? ns : most;
    ns = ns < nk / 5 ? ns : nk / 5;
    p.nsplit = ns > 1 ? (int)ns : 1;
    return p;
}

// What runs a batch of samples of one plan.  It counts the tiles of the whole batch; the values are the same either way (same
// instruction, same order of k, pieces added in the same order, same epilogue).
//   FEW_PIECES  a workgroup per tile and K piece; the pieces pass through memory
//   FEW_INREG   a workgroup per tile, which adds its pieces in registers
//   FEW_TILES   the same, and where there is one piece (bf16) the tiles of gemm_mfma.hip are candidates too
// Pieces of their own pay until the tiles alone occupy the chip: with a short K up to 256 tiles of 64 x 64, with a long one as
// long as the pieces are one round; a single sample's always are (its plan counts the same tiles).  Layer with cold weights,
// us, pieces apart / in registers: 1920 x 1920 and the LayerNorm that adds the pieces, 112 tokens: 3 samples (180 tiles) 19.3 /
// 21.5, 4 (240) 23.1 / 22.0, 8 (480) 37.1 / 26.3; 1920 x 7680 in 8 pieces, 112 tokens: 4 samples 28.8 / 37.6, 5 32.4 / 42.7,
// 6 (no longer one round) 47.9 / 42.1, 8 55.0 / 49.4; in 4 pieces 1040 rows 43.2 / 58.7, 1200 62.2 / 61.2, 1350 68.0 / 63.7.
// fp32 is bound by the matrix instructions and takes finer pieces longer: 1920 x 7680 at 320 tokens, 4 samples (600 tiles)
// 358 / 393, 8 (1200) 674 / 654.
// The tiles of gemm_mfma.hip are never the fastest up to 768 tiles of 64 x 64 (5760 x 1920, 512 rows).
enum FewHow { FEW_PIECES, FEW_INREG, FEW_TILES };
constexpr FewHow few_how(bool bf16, const FewPlan& p, int batch, int tokens, int Nn, int K) {
    const long tiles = (long)batch * p.tiles_m * p.tiles_n;
    if (p.nsplit > 1 && (bf16 && K >= 60 * 64 ? few_one_round((long)batch * tokens, Nn, p.nsplit) : tiles < (bf16 ? 256 : 640)))
        return FEW_PIECES;
    return bf16 && tiles > 768 && p.tiles_m > 1 && K * 2L <= ANY_TILE_ROW_BYTES ? FEW_TILES : FEW_INREG;
}

// scratch for the K pieces, [piece][row][column] in fp32, of the largest batch up to `batch` whose pieces pass through memory
constexpr size_t few_workspace_bytes(bool bf16, const FewPlan& p, int batch, int tokens, int Nn, int K) {
    while (batch > 0 && few_how(bf16, p, batch, tokens, Nn, K) != FEW_PIECES) --batch;
    return (size_t)p.nsplit * batch * tokens * Nn * sizeof(float);
}

// Results larger than the L2 caches of the 8 XCDs together are stored without keeping a place there for them: whoever reads them next finds
// them further away in any case, and what the launch reads again stays (8-bit product of 17776 x 5760, 205 MB: 202 -> 195 us; group norm of
// 70200 x 512, 72 MB, which reads its input twice: 43 -> 39; attention of 8 x 1350 x 30 heads of 64, 41 MB: 31 -> 30).
constexpr size_t STREAM_BYTES = (size_t)32 << 20;

// Threads of a launch in each dimension of its grid stay below 2^32.
constexpr bool grid_fits(long workgroups, int threads) { return workgroups * threads < (1L << 32); }

// Whether pieces of `width` elements at i * a + j * b, 0 <= i < n, 0 <= j < m, overlap (an extent of one has no stride; one of n and m is at most
// 65536, strides at most 2^40).
constexpr bool pieces_meet(long a, long n, long b, long m, long width) {
    if (n > m) { const long s = a, e = n; a = b; n = m; b = s; m = e; }
    if ((n > 1 && a < width) || (m > 1 && b < width)) return true;
    if (n < 2 || (n - 1) * a + width <= b) return false;         // (all of i between two neighbours of j)
    for (long i = 1; i < n; ++i) {
        const long p = i * a, j = p / b, r = p - j * b;          // the neighbours of p among j * b are j and j + 1
        if (j > m) return false;
        if (j < m && r < width) return true;
        if (j + 1 < m && b - r < width) return true;
    }
    return false;
}

// ---- quantizer (gemm_fp8.hip): a workgroup of 256 threads takes 16 blocks
constexpr long quantize_workgroups(int rows, int cols) { return ((long)rows * ((cols + 127) / 128) + 15) / 16; }

// ---- 8-bit products (gemm_fp8.hip): which tile, and how many pieces of k
// Us of a round of workgroups: fixed + blocks of 128 k * stage; `lone`: up to one workgroup per compute unit where two fit.
// Measured, us on 64 x 64 / 128 x 128 / 192 x 192 / 192 x 256 tiles (operands that change from call to call): 448 rows x 7680, k = 1920
// 15.9 / 12.0 / 17.9 / 19.9; 1100 x 5760 27.2 / 22.0 / 19.6 / 20.7; 1100 x 1920, k = 7680 39 / 31 / 48 / 58; 4516 x 1920, k = 7680 111 / 92 /
// 58 / 63, behind the quantization of its rows, from memory, 115 / 95 / 61 / 76 (the third stage); 17776 x 5760, k = 1920 338 / 249 / 210 / 197;
// 17776 x 1920, k = 7680 430 / 305 / 245 / 239.  (256 x 256: 195 and 263 on the last two, 79 at 4516 rows.)
enum Fp8TileId { FP8_64x64, FP8_128x128, FP8_192x192, FP8_192x256, FP8_TILES };
struct Fp8Tile { int bm, bn, per_cu; float fixed, stage, lone_fixed, lone_stage; };
constexpr Fp8Tile kFp8Tiles[FP8_TILES] = {
    {64, 64, 2, 3.0f, 0.39f, 4.0f, 0.15f},               // 4 waves of 32 x 32
    {128, 128, 1, 4.0f, 0.44f, 4.0f, 0.44f},             // 8 waves of 32 x 64
    {192, 192, 1, 4.0f, 0.95f, 4.0f, 0.95f},             // 8 waves of 96 x 48, three stages
    {192, 256, 1, 5.5f, 1.1f, 5.5f, 1.1f},               // 8 waves of 96 x 64, two stages
};
struct Fp8Plan { int tile, pieces; };
constexpr long fp8_tile_count(int id, int m, int n_out) {
    return ((long)m + kFp8Tiles[id].bm - 1) / kFp8Tiles[id].bm * (((long)n_out + kFp8Tiles[id].bn - 1) / kFp8Tiles[id].bn);
}
constexpr Fp8Plan fp8_plan(int m, int n_out, int blocks, bool split, int cus) {
    Fp8Plan p{};
    float best = 0.f;
    for (int id = 0; id < FP8_TILES; ++id) {
        const Fp8Tile& t = kFp8Tiles[id];
        const long n = fp8_tile_count(id, m, n_out), slots = (long)t.per_cu * cus;
        const float rounds = n > 4 * slots ? (float)n / slots : (float)((n + slots - 1) / slots);    // (many rounds drift apart)
        const float us = n <= cus ? t.lone_fixed + blocks * t.lone_stage : rounds * (t.fixed + blocks * t.stage);
        if (id == 0 || us < best) { best = us; p.tile = id; }
    }
    p.pieces = 1;
    if (split && p.tile == FP8_64x64) {
        // tiles that leave compute units idle: pieces of 8 blocks at least, and three of them, to be worth the second launch (1920 columns,
        // k = 7680, us whole / split: 1 to 112 rows 16 / 13.5 in 7 pieces, 200 16.4 / 14.8 in 4, 448 in two 16.7 / 19.6)
        long n = 2L * cus / fp8_tile_count(FP8_64x64, m, n_out);
        if (n > blocks / 8) n = blocks / 8;
        if (n >= 3) p.pieces = (int)n;
    }
    return p;
}

// ---- 4-bit blocks (gemm_fp4.hip): a workgroup of the quantizer, or of reading back, takes 16 rows x 512 columns
constexpr long fp4_workgroups(int rows, int cols) { return (((long)rows + 15) / 16) * (((long)cols + 511) / 512); }

// ---- 4-bit products (gemm_fp4.hip): which tile, and how many pieces of k
// Us of a round of workgroups: fixed + stages of 256 k * stage; `lone`: up to one workgroup per compute unit.
// Measured, us on 64 x 64 / 128 x 128 of 8 waves / 128 x 128 of 4, two to a unit / 192 x 192 / 192 x 256 tiles (operands that change from call to call):
// 112 rows x 7680, k = 1920 5.7 / 8.4 / 10.0 / 12.2 / 14.1; 448 x 7680 13.5 / 10.0 / 11.3 / 14.9 / 16.3; 1100 x 5760 20.2 / 16.4 / 14.8 / 15.4 / 16.9;
// 4516 x 5760 62 / 53 / 43 / 54 / 49; 4516 x 1920, k = 7680 64 / 60 / 57 / 39 / 42; 17776 x 5760, k = 1920 258 / 188 / 150 / 202 / 147; 17776 x 1920,
// k = 7680 239 / 187 / 167 / 170 / 147, k = 256 36 / 31 / 25 / 47 / 26.  (256 x 256: 181, 183 and 46 on the last three.)
enum Fp4TileId { FP4_64x64, FP4_128x128, FP4_128x128_PAIR, FP4_192x192, FP4_192x256, FP4_TILES };
struct Fp4Tile { int bm, bn, per_cu; float fixed, stage, lone_fixed, lone_stage; };
constexpr Fp4Tile kFp4Tiles[FP4_TILES] = {
    {64, 64, 2, 2.3f, 0.42f, 3.7f, 0.27f},               // 4 waves of 32 x 32
    {128, 128, 1, 2.6f, 0.68f, 4.8f, 0.60f},             // 8 waves of 32 x 64
    {128, 128, 2, 2.6f, 1.28f, 5.0f, 0.67f},             // 4 waves of 64 x 64
    {192, 192, 1, 10.6f, 1.06f, 6.0f, 1.09f},            // 8 waves of 96 x 48, three stages
    {192, 256, 1, 5.4f, 1.45f, 4.9f, 1.22f},             // 8 waves of 96 x 64, two stages
};
struct Fp4Plan { int tile, pieces; };
constexpr long fp4_tile_count(int id, int m, int n_out) {
    return ((long)m + kFp4Tiles[id].bm - 1) / kFp4Tiles[id].bm * (((long)n_out + kFp4Tiles[id].bn - 1) / kFp4Tiles[id].bn);
}
constexpr Fp4Plan fp4_plan(int m, int n_out, int blocks, bool split, int cus) {
    Fp4Plan p{};
    float best = 0.f;
    const float stages = 0.5f * blocks;
    for (int id = 0; id < FP4_TILES; ++id) {
        const Fp4Tile& t = kFp4Tiles[id];
        const long n = fp4_tile_count(id, m, n_out), slots = (long)t.per_cu * cus;
        const float rounds = n > 4 * slots ? (float)n / slots : (float)((n + slots - 1) / slots);    // (many rounds drift apart)
        const float us = n <= cus ? t.lone_fixed + stages * t.lone_stage : rounds * (t.fixed + stages * t.stage);
        if (id == 0 || us < best) { best = us; p.tile = id; }
    }
    p.pieces = 1;
    if (split && p.tile == FP4_64x64) {
        // tiles that leave compute units idle: pieces of 4 stages at least, and three of them, to be worth the second launch
        long n = 2L * cus / fp4_tile_count(FP4_64x64, m, n_out);
        if (n > blocks / 8) n = blocks / 8;
        if (n >= 3) p.pieces = (int)n;
    }
    return p;
}

// ---- cross attention: query rows per workgroup, and pieces of the keys.  A function of the sample's shape only, never of the batch.
// resident: all keys in LDS (bf16), which has to hold two such workgroups.
struct CrossPlan { int block, nsplit; bool resident; };
// Pitches of K and V rows in LDS (64 banks of 4 bytes).  A K fragment is 16-byte reads of 16 rows: an odd number of 16 bytes apart, they
// fall into different banks.  A V fragment is 8-byte reads of 8 rows x 32 bytes: an odd number of 32 bytes apart (heads of 16: of 16).
constexpr int cross_v_pitch(int head_dim) { return head_dim == 16 ? 24 : head_dim + 16; }
constexpr int cross_resident_key_bytes(int head_dim) { return 2 * (head_dim + 8 + cross_v_pitch(head_dim)) + 4; }

// The most rows: 2^25 times 16 over all samples and key heads.  The grid is key heads x blocks of 64 rows at least in x (x pieces where that is
// not much) and samples in z; each dimension's threads stay below 2^32, and a launch may have more of them in all.  In x: heads of up to 64
// rows are at most 65535 workgroups; of n > 1 started blocks, 2.5 n times 16 rows at least, so at most 2^25 / 2.5.  (512 samples x 65535 heads
// of one row, 2^33 threads, 52 ms.)
constexpr bool cross_rows_fit(int batch, long rows, int kv_heads) {
    return rows <= (1L << 30) && (rows + 15) / 16 * batch * kv_heads <= (1L << 25);
}

constexpr CrossPlan cross_plan(bool bf16, int rows, int kv_len, int kv_heads, int head_dim, int cus) {
    CrossPlan p{};
    // bf16: 64, 128 or 192 rows, whichever of the last two wastes less; more registers than heads of 128 leave spill (16 heads, 4290 rows x 512
    // keys: 64 rows 49 us, 128 85).
    const auto filled = [rows](int block) { return ((long)rows + block - 1) / block * block; };
    p.block = !bf16 || rows <= 64 || head_dim == 128 ? 64 : rows > 128 && filled(192) <= filled(128) ? 192 : 128;
    // Pieces of 256 keys at least, as many as there are compute units, twice as many for few rows, whose partial sums are small (us at one /
    // two per unit: a token of 30 heads, 17776 keys 55 / 35, 60 tokens 57 / 38; 32 tokens of 30 heads over 6 key heads 29 / 36).
    const long items = (filled(p.block) / p.block) * kv_heads, tiles = (kv_len + 63) / 64;
    long n = (rows <= 64 ? 2L : 1L) * cus / items;
    if (n > tiles / 4) n = tiles / 4;
    p.nsplit = n < 2 ? 1 : (int)n;
    p.resident = bf16 && head_dim <= 64 && p.nsplit == 1 && rows >= 256 && tiles * 64 * cross_resident_key_bytes(head_dim) <= 80 * 1024;
    return p;
}

// ---- attention of packed samples (packed_attention.hip): a sample's blocks of rows and pieces of its keys are found on the GPU; the host knows the sums
// over all samples only.
constexpr int PACKED_SEARCH = 64;                        // most samples that a workgroup looks through itself; more: a table
constexpr int PACKED_KEYS = 1280;                        // least keys of a sample that is divided
// (us with rows apart / keys apart: a token of 30 heads over 6, 17776 keys 22.3 / 21.7, 6 tokens, 1000 keys 19.6 / 14.7; 32 tokens of 30 heads, 17776 keys 41 / 37)
constexpr int PACKED_FEW_ROWS = 32;                      // rows up to which a workgroup's waves take keys apart instead of rows
constexpr int PACKED_FEW_KEYS = 1024;                    // least keys of a piece there
constexpr int PACKED_FEW_MIN = 128;                      // keys from which they do
constexpr int PACKED_PIECES = 512;                       // workgroups of a round, two per compute unit of 256
constexpr int PACKED_UNIT = 128;                         // rows by which pieces are counted
// Pieces of a sample's keys (calls whose keys have offsets of their own), a function of the sample alone.  items: workgroups without.  Few rows: pieces of
// PACKED_FEW_KEYS keys, one round at most.  Else pieces of 256 keys at least: one round of them where items are a quarter of one; up to two rounds of items, in up to 4
// pieces, as many as need the least rounds * tiles, a piece's partial sums counted as 8 tiles of 64 keys (1350 rows of 30 heads, 17776
// keys: whole 516 us, in 3 pieces 297; in 2 pieces of blocks of 256 rows 355).
constexpr int packed_pieces(int rows, int keys, int kv_heads) {
    if (keys < PACKED_KEYS || rows < 1) return 1;
    const int items = (rows + PACKED_UNIT - 1) / PACKED_UNIT * kv_heads;
    if (rows <= PACKED_FEW_ROWS || items <= PACKED_PIECES / 4) {
        const int n = PACKED_PIECES / items, most = keys / (rows <= PACKED_FEW_ROWS ? PACKED_FEW_KEYS : 256);
        return n < most ? (n < 1 ? 1 : n) : most < 1 ? 1 : most;
    }
    if (items >= 2 * PACKED_PIECES) return 1;
    const int tiles = (keys + 63) / 64;
    int best = 1, least = (items + PACKED_PIECES - 1) / PACKED_PIECES * tiles;
    for (int n = 2; n <= 4; ++n) {
        const int cost = (items * n + PACKED_PIECES - 1) / PACKED_PIECES * ((tiles + n - 1) / n + 8);
        if (cost < least) { least = cost; best = n; }
    }
    return best;
}
// block: rows of a workgroup (bf16, heads up to 64: 256 where that leaves three workgroups for two compute units; a row's result does not depend on it; us at 128 / 256 rows,
// one sample: 2926 tokens of 30 heads 102 / 112, 3400 155 / 134, 4276 218 / 225, 5600 325 / 291, 8326 640 / 557, 17776 of 6 heads 665 / 537); slots:
// the most workgroups of a key head; table_bytes: the table of the slots and, for each sample, of the rows of partial sums in front of it; part_bytes: partial sums, a block
// for each slot and key head
struct PackedPlan { int block, slots, part_rows; size_t table_bytes, part_bytes; };
// What the sums over all samples say of those that can be divided, by the three branches of packed_pieces(): few rows; up to a quarter of a round of items; up to two
// rounds, in 4 pieces at most.
struct PackedDivided {
    int samples, round;                                  // that have PACKED_KEYS keys; most pieces of a unit of rows
    int mid, mid_units, wide, wide_units;                // samples of the second and third branch, and the units of rows of one
};
constexpr PackedDivided packed_divided(int samples, int rows, int kv_tokens, int kv_heads) {
    PackedDivided d{};
    d.samples = samples < kv_tokens / PACKED_KEYS ? samples : kv_tokens / PACKED_KEYS;
    d.round = PACKED_PIECES / kv_heads;
    d.mid_units = PACKED_PIECES / 4 / kv_heads;
    d.mid = d.mid_units < 1 ? 0 : rows / (PACKED_FEW_ROWS + 1);
    if (d.mid > d.samples) d.mid = d.samples;
    d.wide_units = (2 * PACKED_PIECES - 1) / kv_heads;
    const int least = PACKED_UNIT * d.mid_units;         // such a sample has more rows
    d.wide = d.wide_units < 1 ? 0 : rows / ((least > PACKED_FEW_ROWS ? least : PACKED_FEW_ROWS) + 1);
    if (d.wide > d.samples) d.wide = d.samples;
    return d;
}
constexpr long packed_least(long a, long b) { return a < b ? a : b; }
constexpr long packed_most(long a, long b) { return a > b ? a : b; }
// the most workgroups of a key head: a block each, and what pieces add
constexpr long packed_slots(bool own, int samples, int rows, int kv_tokens, int kv_heads, int block) {
    const long blocks = rows / block + samples;
    if (!own || kv_tokens < PACKED_KEYS) return blocks;
    const PackedDivided d = packed_divided(samples, rows, kv_tokens, kv_heads);
    const long unit = PACKED_UNIT > block ? PACKED_UNIT / block : 1;                     // blocks of a unit of rows
    const long mid_blocks = packed_least(((long)rows + block - 1) / block, ((long)d.mid_units * PACKED_UNIT + block - 1) / block);
    const long wide_blocks = ((long)d.wide_units * PACKED_UNIT + block - 1) / block;
    const long few = packed_least((long)d.samples * d.round, kv_tokens / PACKED_FEW_KEYS);
    const long mid = packed_least(d.mid * d.round * unit, mid_blocks * (kv_tokens / 256));
    const long wide = 3 * packed_least(d.wide ? rows / block + d.wide : 0, d.wide * wide_blocks);
    const long more = packed_least(packed_least(few + mid, d.samples * d.round * unit) + wide, d.samples * packed_most(d.round * unit, 3 * wide_blocks));
    return blocks + more;
}
// the most rows of partial sums of a key head: those of every divided sample, in each of its pieces.  (1024 samples of a token, 4096 keys each, 4 query heads to
// each of 8 key heads: 262144, of which 16384 are used; a block for each slot would be 1.7 million.)
constexpr long packed_part_rows(bool own, int samples, int rows, int kv_tokens, int kv_heads) {
    if (!own || kv_tokens < PACKED_KEYS) return 0;
    const PackedDivided d = packed_divided(samples, rows, kv_tokens, kv_heads);
    const long few_rows = packed_least(rows, PACKED_FEW_ROWS), mid_rows = packed_least(rows, (long)d.mid_units * PACKED_UNIT);
    const long few = few_rows * packed_least((long)d.samples * d.round, kv_tokens / PACKED_FEW_KEYS);
    const long mid = packed_least((long)d.mid * d.round * PACKED_UNIT, mid_rows * (kv_tokens / 256));
    const long wide = 4 * packed_least(d.wide ? rows : 0, (long)d.wide * d.wide_units * PACKED_UNIT);
    const long each = packed_most(packed_most(few_rows * d.round, packed_least((long)d.round * PACKED_UNIT, mid_rows * (kv_tokens / 256))), 4 * packed_least(rows, (long)d.wide_units * PACKED_UNIT));
    return packed_least(packed_least(few + mid + wide, rows * packed_most(d.round, 4)), d.samples * each);
}
// a workgroup for each slot, up to a multiple of 8, and key head
constexpr long packed_workgroups(long slots, int kv_heads) { return (slots + 7) / 8 * 8 * kv_heads; }
// (most: 128 if there is no kernel for more)
constexpr PackedPlan packed_plan(bool bf16, bool own, int samples, int rows, int kv_tokens, int kv_heads, int head_dim, int cus, int most = 256) {
    PackedPlan p{};
    p.block = !bf16 ? 64 : most >= 256 && head_dim <= 64 && ((long)rows / 256 + samples) * kv_heads >= 3L * cus / 2 ? 256 : 128;
    p.slots = (int)packed_slots(own, samples, rows, kv_tokens, kv_heads, p.block);
    p.part_rows = rows < p.block ? rows : p.block;
    if (samples > PACKED_SEARCH) p.table_bytes = (((size_t)p.slots + 1) * 8 + (size_t)samples * 4) / 256 * 256 + 256;
    if (own && kv_tokens >= PACKED_KEYS) p.part_bytes = (size_t)p.slots * kv_heads * p.part_rows * (head_dim + 4) * sizeof(float);
    return p;
}

// ---- group norm: `slices` slices of slice_groups whole groups (the last may have fewer), each over `chunks` chunks of positions.
// A function of the sample's shape only, never of the batch.
constexpr int GROUP_NORM_SLICE_GROUPS = 256;             // most groups of a slice: one thread each
struct GroupNormPlan {
    int cpg, slice_groups, slices, chunks, per;          // per: positions of a chunk (the last may have fewer)
    int lanes, rows, team, fill;                         // threads of a position, positions at a time, threads per group (set by the launcher)
    unsigned lanes_inv;
};
constexpr GroupNormPlan group_norm_plan(int positions, int channels, int groups, int elem_bytes) {
    const int cpg = channels / groups;
    const long bytes = (long)cpg * elem_bytes;
    // a cache line of a position at least, and channels that 16-byte loads divide if a few groups more give them
    long k = (127 + bytes) / bytes;
    for (int more = 0; more < 8; ++more)
        if ((k + more) * bytes % 16 == 0) { k += more; break; }
    if (k > GROUP_NORM_SLICE_GROUPS) k = GROUP_NORM_SLICE_GROUPS;
    if (k > groups) k = groups;
    GroupNormPlan p{};
    p.slice_groups = (int)k;
    p.slices = (groups + p.slice_groups - 1) / p.slice_groups;
    const long of_slice = (long)positions * p.slice_groups * bytes;
    // 32 KB a chunk at least (16 KB: 70200 x 128 31 us, 64 KB 24; 2000 x 320 13.2 and 15.5, so 25 and 12.4), 512 workgroups at most: more read x
    // no faster and leave more moments to unite (512 / 1024 / 2048: 70200 x 512 41 / 42 / 46 us, 17550 x 1280 29 / 29 / 39)
    long chunks = of_slice / 32768, most = 512 / p.slices;
    if (chunks > most) chunks = most;
    if (chunks > positions) chunks = positions;
    p.cpg = cpg;
    p.per = (int)((positions + (chunks < 1 ? 0 : chunks - 1)) / (chunks < 1 ? 1 : chunks));
    p.chunks = (positions + p.per - 1) / p.per;
    return p;
}

}  // namespace ps
