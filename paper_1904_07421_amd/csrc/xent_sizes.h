// Which kernels a loss takes, and in what pieces: rules on sizes alone, in plain C++ (the device uses them too).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "jitdb.h"
#include "rounding.h"

namespace jitdb {
namespace {

// ---- few classes: everything in one pass, the class weights in LDS -----------------------------------------
constexpr int kFewRows = 64;             // rows a block works on at once
// classes in sixteens, features in blocks of what four waves cover with one load of 16 bytes a lane: in LDS, K in steps of four loads
constexpr size_t few_table_bytes(int ct, int nb) {
    return (size_t)ct * (nb * 16) * 4 * 17 * 16 + ct * 64;
}
// 128 registers of sums a lane; weights and two sets of g in LDS
constexpr bool few_variant(int element, int ct, int nb) {
    return ct * nb * (16 / element) <= 32 && few_table_bytes(ct, nb) + 2 * kFewRows * (ct * 64 + 4) <= 160 * 1024;
}
struct FewSizes { int ct, nb; };         // 0: no variant
// Taken wherever one fits (forward and backward of 100 k rows with fp32 gradients, the last size that fits and the next: fp32 150 x 64
// 215 us, 150 x 65 609; 512 x 32 327, 512 x 48 1234; bf16 512 x 64 445, 512 x 65 741).
constexpr FewSizes few_sizes(int element, int H, int C) {
    const int blocks = (int)ceil_div(H, 64 * (16 / element));
    const int ct = C <= 16 ? 1 : C <= 32 ? 2 : C <= 64 ? 4 : 0, nb = blocks <= 1 ? 1 : blocks <= 2 ? 2 : blocks <= 4 ? 4 : blocks <= 8 ? 8 : 0;
    if (ct == 0 || nb == 0 || !few_variant(element, ct, nb)) return {0, 0};
    return {ct, nb};
}
constexpr bool few_fits(int H, int C, jitdb_dtype dtype) { return few_sizes(dtype == JITDB_F32 ? 4 : 2, H, C).ct > 0; }

// ---- many classes, states of ordinary width: one operand resident ------------------------------------------
constexpr int kResRows = 256;            // resident rows of a block
constexpr int kResTile = 32;             // rows of the other operand in a tile
// A block's range is no shorter; where it makes further rounds of blocks, 8.  (Statistics and g with 8 everywhere and with 2: fp32 2304 x 150
// x 2003 30 + 43 us, 20 + 25; bf16 2000 x 512 x 2000 21 + 28, 16 + 16; with 2 everywhere fp32 4608 x 150 x 10007 79 + 113, 82 + 136.)
constexpr int kResMinTiles = 2, kResRoundTiles = 8;
constexpr int kResBlocks = 1024;         // ranges make no more blocks than this
// Ranges for `blocks` blocks of resident rows on a chip that holds `places` at once, `tiles` tiles to walk over: more of them where
// that leaves fewer places idle in the last round, by more than 1 / 64.
constexpr int res_ranges(int blocks, int tiles, int places) {
    if (blocks * 32 < places) {          // few rows: fill the chip
        const int fill = places / (blocks > 0 ? blocks : 1), most = tiles / kResMinTiles;
        return fill < most ? fill : most > 1 ? most : 1;
    }
    int best = 1, best_rounds = (blocks + places - 1) / places;
    for (int s = 2; s <= 32 && blocks * s <= kResBlocks && tiles >= s * (blocks * s <= places ? kResMinTiles : kResRoundTiles); ++s) {
        const int rounds = (blocks * s + places - 1) / places;
        if (rounds * best * 64 < best_rounds * s * 63) { best = s; best_rounds = rounds; }
    }
    return best;
}
// one wave a SIMD and two sets of accumulators, or two waves and one set
constexpr bool res_alone(int fragments, bool g) { return fragments > (g ? 8 : 16); }
constexpr int res_places(int fragments, bool g) { return res_alone(fragments, g) ? 256 : 512; }

// ---- tiles of two streaming operands: the gradients' products, and logits of wide states ------------------------
constexpr int kTileB = 256;                           // rows of B in a tile
template <int WM> constexpr int kTileA = WM * 64;     // rows of A; WM: 64-row waves along A (5: four waves along B with all 160)
template <> constexpr int kTileA<5> = 160;
template <int WM> constexpr int kTilePlaces = WM == 4 ? 256 : 512;      // blocks for each of the two products: half of what the chip holds at once
constexpr uint32_t kLongRange = 1200;      // stages
constexpr uint32_t kMinStages = 8;       // a range is no shorter
struct GradPlan {
    uint32_t b_tiles, nk, stages;   // stages of a part product, of a tile
    uint32_t total, per, ranges;    // (a stage stands for 8192 elements of g, six times at most: of a chunk of rows far below 2^32)
};
constexpr int grad_ranges(int places, int a_tiles) { return places > a_tiles ? places / a_tiles : 1; }      // at most
constexpr GradPlan make_plan(uint32_t b_tiles, uint32_t nk, uint32_t pairs, int places, int a_tiles) {
    GradPlan g = {b_tiles, nk, nk * pairs, b_tiles * nk * pairs, 0, 0};
    // Ranges: dh's and dV's together are as many blocks as the chip holds.  Long ones of several tiles of A are faster one product after
    // the other, on all of it (both products with joining, bf16 32768 x 512 x 32000 2.15 ms against 2.25; but 16384 rows 1.17 against
    // 1.15, 8192 x 512 x 16000 305 us against 286, 65536 x 256 x 32000 2.28 ms against 2.16, fp32 3000 x 256 x 8000 194 us against 163).
    const uint32_t half = grad_ranges(places / 2, a_tiles);
    const uint32_t most = a_tiles > 1 && g.total / half > kLongRange ? grad_ranges(places, a_tiles) : half;
    const uint32_t per = (g.total + most - 1) / most;
    g.per = per > kMinStages ? per : kMinStages;
    g.ranges = (g.total + g.per - 1) / g.per;
    return g;
}

constexpr int kBand = 8;                 // logits of wide states: row tiles that the blocks of an XCD work on side by side

// ---- a call -------------------------------------------------------------------------------------------------
constexpr int kMaxClasses = 1 << 22;
constexpr int kMaxWidth = 1 << 14;
constexpr int kLabelBlock = 1024, kLabelBlocks = 2048;     // labels of a block of the listing kernels at least, most blocks of them
constexpr int64_t kStatBytes = 512ll << 20;   // of tile statistics of wide states kept at once (forward) ...
constexpr int64_t kGradBytes = 4ll << 30;     // ... and of g (backward): rows beyond come in further chunks, of 256 rows at least
struct Sizes {
    int64_t n, n_pad;          // rows at most, and rounded up to whole tiles
    int H, C, Hk, Hf, Cp;      // widths: of K (states), of the turned states' rows, classes in whole tiles
    int wm, tile_a, a_tiles, places;      // of the gradients' products: variant, features of a tile, tiles, blocks on the chip
    int parts, g_parts;        // of the operands, of g
    int label_per, label_blocks;
    int res, class_tiles;      // resident_kernel: K in steps of 16 (0: not for this width), tiles of 32 classes
    int stat_rows, grad_rows;  // rows of a chunk
};
bool known(jitdb_dtype t) { return t == JITDB_F32 || t == JITDB_BF16; }
// K in steps of 16 of the variant of resident_kernel for this width: the fragments of 64 rows in up to 256 registers.  (bf16 32768 x 512
// x 50021: statistics 1.48 ms, g 1.83; with both operands streaming, as wider states have them, 1.78 and 2.83.)
int res_steps(int H, jitdb_dtype dtype) {
    if (dtype == JITDB_F32) return H <= 128 ? 8 : H <= 160 ? 10 : 0;
    return H <= 128 ? 8 : H <= 256 ? 16 : H <= 384 ? 24 : H <= 512 ? 32 : 0;
}
bool make_sizes(int64_t n, int32_t H, int32_t C, jitdb_dtype dtype, jitdb_dtype grad, Sizes &s) {
    if (n < 0 || n > JITDB_MAX_NODES || H < 1 || H > kMaxWidth || C < 1 || C > kMaxClasses || !known(dtype) || !known(grad)) return false;
    if (dtype == JITDB_F32 && grad == JITDB_BF16) return false;       // gradients are not rounded below their operands
    s.n = n; s.H = H; s.C = C;
    s.n_pad = round_up(n > 0 ? n : 1, 256);
    s.res = res_steps(H, dtype);
    s.Hk = s.res ? s.res * 16 : (int)round_up(H, 32);
    // The tile height that pads the features least, of equals the highest.  Both gradients' products: bf16 65536 x 150 x 32000 in tiles of
    // 160 features 1.70 ms, of 256 2.18; fp32 30000 x 300 x 8000 of 160 2.08, of 128 2.34; 30000 x 450 x 8000 of 160 3.21, of 256 3.32.
    auto take_tile = [&](auto wm) {
        constexpr int WM = decltype(wm)::value, A = kTileA<WM>;
        if (s.wm && round_up(H, A) >= (int64_t)s.tile_a * s.a_tiles) return;
        s.wm = WM; s.tile_a = A; s.a_tiles = (int)ceil_div(H, A); s.places = kTilePlaces<WM>;
    };
    s.wm = 0;
    take_tile(std::integral_constant<int, 4>());
    take_tile(std::integral_constant<int, 5>());
    take_tile(std::integral_constant<int, 2>());
    s.Hf = (int)round_up((int64_t)s.tile_a * s.a_tiles, 64);
    s.Cp = (int)round_up(C, 256);
    s.class_tiles = (int)ceil_div(C, kResTile);
    s.parts = dtype == JITDB_F32 ? 3 : 1;
    s.g_parts = grad == JITDB_F32 ? 3 : 1;
    s.label_per = kLabelBlock * (int)ceil_div(n > 0 ? n : 1, (int64_t)kLabelBlock * kLabelBlocks);
    s.label_blocks = (int)ceil_div(n > 0 ? n : 1, s.label_per);
    auto chunk = [&](int64_t bytes_a_row, int64_t budget) {
        const int64_t rows = budget / bytes_a_row / 256 * 256;
        return (int)(rows < 256 ? 256 : rows < s.n_pad ? rows : s.n_pad);
    };
    s.stat_rows = s.res ? (int)s.n_pad : chunk((int64_t)s.Cp / 64 * 8, kStatBytes);
    s.grad_rows = chunk((int64_t)s.Cp * 2 * s.g_parts, kGradBytes);
    return true;
}
// most blocks of resident_kernel with at most `blocks` blocks of resident rows and `tiles` tiles to walk over (res_ranges)
int64_t res_most(int64_t blocks, int64_t tiles) {
    const int64_t ranges = tiles / kResMinTiles > 1 ? tiles / kResMinTiles : 1, most = blocks > kResBlocks ? blocks : kResBlocks;
    return blocks * ranges < most ? blocks * ranges : most;
}
// sets of statistics, if every row has a label
int stat_sets(const Sizes &s) {
    return s.res ? res_ranges((int)(s.n_pad / kResRows), s.class_tiles, res_places(s.parts * s.res, false)) : s.Cp / 64;
}
// Many take sixteen waves (800 rows, 938 sets: 141 -> 52 us), few four (4608 rows, 28 sets: 14 -> 8 us).
constexpr int join_waves(int sets) { return sets > 64 ? 16 : 4; }
// most shares of tiles (grad_plan): of every tile of A, a tile of B more than ranges
int64_t grad_parts(const Sizes &s, int64_t b_tiles, int64_t nk, int pairs) {
    const int64_t most = grad_ranges(s.places, s.a_tiles), ranges = ceil_div(b_tiles * nk * pairs, kMinStages);
    return s.a_tiles * (b_tiles + (ranges < most ? ranges : most));
}
int pair_count(int a, int b) { return a == 3 && b == 3 ? 6 : a * b; }        // (one part and three: three products)

}  // namespace
}  // namespace jitdb
