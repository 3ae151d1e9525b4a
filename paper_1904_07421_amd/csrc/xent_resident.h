// The logits of many classes for states of ordinary width: one operand stays in registers while the other streams past.
//
// Two kernels in one skeleton.  Statistics (G = 0) keep the states: a lane has a row, and maximum and sum run over classes in its
// registers.  Derivatives (G > 0) keep the class weights: a lane has a class, and the bias' gradient runs over rows in its registers.
// A wave keeps the fragments of 64 rows of the resident operand (two MFMA tiles of 32) for all of K in registers, up to 256 of them; a
// block of four waves, 256 rows, walks over a range of the other operand, 32 rows at a time.  Those come straight into LDS, three
// buffers deep, and every wave reads each fragment once for its two products: half the LDS traffic of a tile whose operands both come
// from LDS.  One barrier a tile.
// The vector unit works on a tile of logits beside the matrix cores: where the resident fragments leave one wave a SIMD, on the tile
// before, in a second set of accumulators, a few instructions behind every product (measured: two are free, more cost what they
// take alone); where two waves fit, each takes the matrix cores while the other computes.
// bf16 32768 x 512 x 50021: statistics 1.48 ms (1.13 PFLOP/s), g 1.83 ms; without any work on the logits the loop takes 0.89.
// Lane l holds row l % 32 of both resident tiles and, of the 32 rows that stream past, 8 q + 4 (l / 32) + e (q, e < 4).
#pragma once

#include "level_common.h"
#include "xent_sizes.h"

#include <utility>

namespace jitdb {
namespace {

constexpr int kResT = 256;
constexpr int kResBufs = 3;
constexpr int kResInAcc = 44;            // resident fragments that are kept in accumulation registers, of 64 at most
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f, kLn2Low = (float)(0.69314718055994530942 - (double)kLn2);

struct ResArgs {
    const char *res; int64_t res_slab;   // the resident operand, K-blocked, the parts' slabs behind one another
    const char *str; int64_t str_slab;   // the other one
    const float *side;                   // what comes with 32 streaming rows.  G = 0: their bias (a float each; -inf behind the last class);
                                         // G > 0: 128 words, log-sum-exp, weight, label (as they are needed, weights over the scale of g) and 32 unused
    const int32_t *n_rows;
    int row0, max_rows;                  // the chunk: rows row0 .. row0 + max_rows of the list
    int class_tiles;                     // G = 0: the walk
    float2 *stat;                        // [ranges][256 row blocks]: reference m, sum of exp(z - m)
    int class_blocks;                    // G > 0: the resident classes
    const float *bias;                   // padded with -inf to whole blocks
    char *g; int64_t g_slab, g_part;     // g of the chunk, K-blocked with K = row: slab of 32 rows, class, 64 bytes
    float *db_part;                      // [ranges, at most kResBlocks / class_blocks or so][256 class_blocks]
};
template <typename F, int... I>
__device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void static_for(F &&f) { static_for_impl(f, std::make_integer_sequence<int, N>()); }

// e^x: the hardware's 2^t, good to a unit in the last place, with t = x log2 e rounded, times 1 + c, c = x - t ln 2: what the rounding
// of t and of log2 e itself left out.  ln 2 in two words: of one, t 1.9e-9 would stay, always in the same direction (as the lower word
// of log2 e did while c was computed from the upper: 2.3e-7 at -17, 1.2e-6 at -80).  (Not of -inf itself, whose c would be NaN.)
__device__ __forceinline__ float exp_close(float x) {
    x = x < -200.0f ? -200.0f : x;
    const float t = x * kLog2e, p = __builtin_amdgcn_exp2f(t);
    return fmaf(p, fmaf(-t, kLn2Low, fmaf(-t, kLn2, x)), p);
}

// e^(x - top) for a largest x of `top`: of +inf only the largest themselves count (inf - inf is no number)
__device__ __forceinline__ float exp_below(float x, float top) { return x == INFINITY ? 1.0f : expf(x - top); }

// A read of LDS that the compiler does not wait for: it would make it wait for every direct-to-LDS load in flight.
template <int OFFSET>
__device__ __forceinline__ void lds_read16(u32x4 &to, uint32_t at) { asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(to) : "v"(at), "n"(OFFSET) : "memory"); }

template <int OFFSET>                    // 16 lanes read 4 rows of 16 columns, transposed: a lane gets its column's four
__device__ __forceinline__ void lds_read8_turned(u32x2 &to, uint32_t at) { asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(to) : "v"(at), "n"(OFFSET) : "memory"); }
__device__ __forceinline__ void lds_read4(int32_t &to, uint32_t at) { asm volatile("ds_read_b32 %0, %1" : "=v"(to) : "v"(at) : "memory"); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// two values rounded to bf16 in one word
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// products (for both resident tiles) of a tile's first fragments
template <int PARTS>
constexpr int res_products(int fragments) { return PARTS == 3 ? fragments / 3 * 12 + (fragments % 3 == 0 ? 0 : fragments % 3 == 1 ? 2 : 6) : fragments * 2; }

// PARTS: bf16 parts of both operands; KS: K in steps of 16; G: 0 = statistics, else g in that many parts.
template <int PARTS, int KS, int G>
__global__ void __launch_bounds__(kResT, res_alone(PARTS * KS, G > 0) ? 1 : 2)
resident_kernel(const ResArgs a) {
    constexpr int NF = PARTS * KS;                       // fragments of a tile, 1 KB each
    constexpr int NG = NF / 2;                           // groups of two
    constexpr int RING = NG % 3 == 0 ? 3 : 4;            // groups of fragments in registers: one multiplied, two on their way
    constexpr int SIDE = G == 0 ? 1 : 2;                 // loads of what comes with a tile, 256 bytes each, a copy for each wave
    constexpr int LOADS = (NF + 3) / 4 + SIDE;           // per wave and tile
    constexpr int BUF = NF * 1024 + 4 * SIDE * 256;
    constexpr int PRODUCTS = PARTS == 3 ? KS * 12 : KS * 2;       // of a tile and wave
    // of those, the ones that work is dealt out over: for g, those in front of the last three groups, in which the next rows' values come
    constexpr int EARLY = (NG - 3) * 2;                  // fragments
    constexpr int SLOTS = G == 0 || !res_alone(NF, G > 0) ? PRODUCTS : res_products<PARTS>(EARLY);
    constexpr bool ALONE = res_alone(NF, G > 0);
    constexpr bool CLOSE = PARTS == 3 || G == 3;         // fp32 results: exponentials good to two roundings
    __shared__ __attribute__((aligned(1024))) char lds[kResBufs * BUF];
    const int left = *a.n_rows - a.row0, rows = left < 0 ? 0 : left < a.max_rows ? left : a.max_rows;
    const int blocks = G == 0 ? (rows + kResRows - 1) / kResRows : a.class_blocks;
    const int tiles = G == 0 ? a.class_tiles : (rows + 63) / 64 * 2;
    if (rows == 0) return;
    const int ranges = res_ranges(blocks, tiles, res_places(NF, G > 0));
    // neighbours on an XCD share their range
    const int total = blocks * ranges, per_xcd = (total + 7) / 8, place = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || place >= total) return;
    const int range = place / blocks, rb = place % blocks;
    const int t0 = (int)((int64_t)tiles * range / ranges), t1 = (int)((int64_t)tiles * (range + 1) / ranges), n_tiles = t1 - t0;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hf = lane >> 5, l32 = lane & 31;
    const int r0 = rb * kResRows + wave * 64;            // the wave's first resident row
    // ---- movers: 1 KB units of 16 rows of a slab, piece p of row r in slot p ^ ((r >> 2) & 3)
    // (scalar addresses and one offset for every lane: no vector instruction is spent on them)
    const uint32_t str_lane = (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 4) & 3)) * 16), side_lane = lane * 4;
    auto issue_one = [&](int tile, int buf, int i) __attribute__((always_inline)) {
        char *dst = lds + buf * BUF;
        if (i < LOADS - SIDE) {
            int u = wave + 4 * i;
            if (NF % 4 != 0 && u >= NF) u = NF - 1;      // the same bytes to the same place once more: every wave issues as many
            const char *at = a.str + (int64_t)(u >> 1) * a.str_slab + (int64_t)tile * 2048 + (u & 1) * 1024;
            __builtin_amdgcn_global_load_lds(JITDB_GLOBAL_PTR(at + str_lane), JITDB_LDS_PTR(dst + u * 1024), 16, 0, 0);
        } else {
            const char *at = reinterpret_cast<const char *>(a.side) + (int64_t)tile * (G == 0 ? 128 : 512) + (i - (LOADS - SIDE)) * 256;
            __builtin_amdgcn_global_load_lds(JITDB_GLOBAL_PTR(at + side_lane), JITDB_LDS_PTR(dst + NF * 1024 + (wave * SIDE + i - (LOADS - SIDE)) * 256), 4, 0, 0);
        }
    };
    auto issue = [&](int tile, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) issue_one(tile, buf, i);
    };
    auto wait_barrier = [&](auto n) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(n)::value) : "memory");
    };
    // ---- the resident fragments
    u32x4 hb[PARTS][2][KS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                hb[p][j][k] = *reinterpret_cast<const u32x4 *>(a.res + (int64_t)(p * (KS / 2) + k / 2) * a.res_slab + (int64_t)(r0 + j * 32 + l32) * 64 + (k & 1) * 32 + hf * 16);
    // Most of them in accumulation registers, from where the matrix instructions take them as well: left to itself the compiler moves
    // them there and back.
    if constexpr (ALONE)
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    if ((p * 2 + j) * KS + k < kResInAcc) asm volatile("" : "+a"(hb[p][j][k]));
    float own_bias[2] = {0.0f, 0.0f};
    if constexpr (G != 0) {
        own_bias[0] = a.bias[r0 + l32];
        own_bias[1] = a.bias[r0 + 32 + l32];
    }
    // nothing of the above may still be on its way when loads are counted
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int b = 0; b < kResBufs; ++b) issue(t0 + (b < n_tiles ? b : n_tiles - 1), b);

    // ---- fragments of the tile
    const uint32_t lds_base = (uint32_t)(uintptr_t)JITDB_LDS_PTR(lds);
    uint32_t rd[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) rd[k] = lds_base + l32 * 64 + (((2 * k + hf) ^ ((l32 >> 2) & 3)) * 16);
    const uint32_t rd_side = lds_base + NF * 1024 + wave * SIDE * 256 + hf * 16, rd_label = rd_side - hf * 16 + 256 + l32 * 4;
    u32x4 fa[RING][2], side[4];                            // side: G = 0, the bias of the next tile's 16 classes of this lane
    u32x4 lse_w[2][4];                                   // G > 0: log-sum-exp and weight of 16 rows of the tile that is worked on
    int32_t label = -1;                                  // ... label of row l32
    // fragment f of a tile: K step f / PARTS, part PARTS - 1 - f % PARTS (the smallest first)
    auto read_group = [&](auto g_tag, uint32_t at, u32x4 (&f)[2]) __attribute__((always_inline)) {
        constexpr int GI = decltype(g_tag)::value;
        static_for<2>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int F = GI * 2 + decltype(i_tag)::value, K = F / PARTS, P = PARTS - 1 - F % PARTS;
            lds_read16<(P * (KS / 2) + K / 2) * 2048>(f[decltype(i_tag)::value], rd[K & 1] + at);
        });
    };
    auto read_bias = [&](uint32_t at) __attribute__((always_inline)) {
        static_for<4>([&](auto i_tag) __attribute__((always_inline)) { lds_read16<decltype(i_tag)::value * 32>(side[decltype(i_tag)::value], rd_side + at); });
    };
    auto read_rows = [&](uint32_t at) __attribute__((always_inline)) {
        static_for<8>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int I = decltype(i_tag)::value;
            lds_read16<(I / 4) * 128 + (I % 4) * 32>(lse_w[I / 4][I % 4], rd_side + at);
        });
        lds_read4(label, rd_label + at);
    };
    // at most `later` reads asked for after these are still on their way
    auto reads_done = [&](auto later, u32x4 (&f)[2]) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(f[0]), "+v"(f[1]) : "n"(decltype(later)::value));
    };
    auto four_done = [&](u32x4 (&f)[4]) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]));
    };
    auto rows_done = [&]() __attribute__((always_inline)) {
        four_done(lse_w[0]);
        four_done(lse_w[1]);
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(label));
    };

    // ---- what happens to a tile of logits, dealt out over the products
    // Statistics: sums of exp(z - ref).  The reference is the maximum of the tiles up to the last one that left the range of fp32
    // (the first does): only then is a maximum taken and the sum so far scaled.
    // (A tile's sum is added to the others' as a whole: one chain over all classes would lose more to rounding.)
    float ref[2] = {-INFINITY, -INFINITY}, ref_l[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f}, kept[2] = {0.0f, 0.0f};
    float late[2] = {0.0f, 0.0f}, arg = 0.0f;            // an exponential is added when the tile's next is asked for
    // Derivatives
    float colsum[2] = {0.0f, 0.0f}, tile_sum[2] = {0.0f, 0.0f};      // of the tiles before, of this one (as for the statistics)
    uint32_t words[G > 0 ? G : 1][2][2];                 // [part][q & 1][pair]
    float d[4];
    const int own_class = rb * kResRows + wave * 64 + l32;
    char *g_lane = a.g + (int64_t)(r0 + l32) * 64 + hf * 16;

    auto statistics = [&](auto s_tag, floatx16 (&z)[2]) __attribute__((always_inline)) {
        constexpr int S = decltype(s_tag)::value;
        // step 2 e fetches and scales element e, step 2 e + 1 asks for its exponential and adds the one before
        constexpr int E0 = S * 64 / SLOTS, E1 = (S + 1) * 64 / SLOTS;
        static_for<E1 - E0>([&](auto e_tag) __attribute__((always_inline)) {
            constexpr int E = (E0 + decltype(e_tag)::value) >> 1, J = E & 1, V = E >> 1;
            if constexpr ((E0 + decltype(e_tag)::value) % 2 == 0) {
                if constexpr (ALONE) asm volatile("" : "+a"(z[J]));      // the accumulator is fetched here, not all of them in front of the tile
                arg = CLOSE ? z[J][V] - ref[J] : fmaf(z[J][V], kLog2e, -ref_l[J]);
            } else {
                sum[J] += late[J];
                late[J] = CLOSE ? exp_close(arg) : __builtin_amdgcn_exp2f(arg);
            }
        });
    };
    auto statistics_end = [&](floatx16 (&z)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sum[j] = kept[j] + (sum[j] + late[j]);
            late[j] = 0.0f;
        }
        // (behind the branch accumulators may be moved: the last products are through by then, which the compiler does not see to there)
        asm volatile("s_nop 15" ::: "memory");
        if (__any(!(sum[0] < 1e30f && sum[1] < 1e30f)))
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bool out = !(sum[j] < 1e30f);                      // taken by the lanes concerned alone: a row's result is its own
                float m = ref[j];
#pragma unroll
                for (int v = 0; v < 16; ++v) m = fmaxf(m, z[j][v]);
                const float from = m == -INFINITY ? 0.0f : m;            // nothing but masked classes so far
                float again = kept[j] * exp_below(ref[j], from);
#pragma unroll
                for (int v = 0; v < 16; ++v) again += exp_below(z[j][v], from);
                sum[j] = out ? again : sum[j];
                ref[j] = out ? m : ref[j];                               // (stays -inf until a class is not masked)
                ref_l[j] = ref[j] * kLog2e;
            }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            kept[j] = sum[j];
            sum[j] = 0.0f;
        }
    };
    // g of element v of resident tile j; after every second quad 16 bytes a lane go out, the wave's halves having exchanged quads
    auto derivatives = [&](auto s_tag, floatx16 (&z)[2], int tile) __attribute__((always_inline)) {
        constexpr int S = decltype(s_tag)::value, E0 = (S * 32 + SLOTS - 1) / SLOTS, E1 = ((S + 1) * 32 + SLOTS - 1) / SLOTS;
        static_for<E1 - E0>([&](auto e_tag) __attribute__((always_inline)) {
            constexpr int E = E0 + decltype(e_tag)::value, J = E / 16, V = E % 16, Q = V / 4;
            if constexpr (ALONE) asm volatile("" : "+a"(z[J]));
            const float x = z[J][V], lse = __uint_as_float(lse_w[0][Q][V % 4]), w = __uint_as_float(lse_w[1][Q][V % 4]);
            const float p = CLOSE ? exp_close(x - lse) : __builtin_amdgcn_exp2f(fmaf(x, kLog2e, -lse));
            d[V % 4] = p * w;
            if constexpr (V == 0) {
                colsum[J] += tile_sum[J];
                tile_sum[J] = d[0];
            } else {
                tile_sum[J] += d[V % 4];
            }
            if constexpr (V % 4 == 3) {
#pragma unroll
                for (int i = 0; i < G; ++i) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t y = pack_bf16(d[2 * k], d[2 * k + 1]);
                        words[i][Q & 1][k] = y;
                        if (i + 1 < G) { d[2 * k] -= low_bf16(y); d[2 * k + 1] -= high_bf16(y); }
                    }
                    if constexpr (Q & 1) {
                        u32x4 out;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const auto s = __builtin_amdgcn_permlane32_swap(words[i][0][k], words[i][1][k], false, false);
                            out[k] = s[0];
                            out[2 + k] = s[1];
                        }
                        *reinterpret_cast<u32x4 *>(g_lane + i * a.g_part + (int64_t)tile * a.g_slab + J * 2048 + (Q >> 1) * 32) = out;
                    }
                }
            }
        });
    };
    // Labels among the wave's classes, seldom: the derivative of a label's own logit goes out once more, after the others (a wave's
    // stores to one place take effect in order).
    auto derivatives_end = [&](floatx16 (&z)[2], int tile) __attribute__((always_inline)) {
        const int first = rb * kResRows + wave * 64;
        uint64_t hits = __ballot(label >= first && label < first + 64) & 0xFFFFFFFFull;      // (both halves hold all 32)
        while (hits) {
            const int row = __builtin_ctzll(hits);
            hits &= hits - 1;
            const int which = __builtin_amdgcn_readlane(label, row) - first, rel = row - hf * 4;
            float x = 0.0f, lse = 0.0f, w = 0.0f;
            bool mine = false;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const bool here = rel == (v >> 2) * 8 + (v & 3);
                x = here ? which < 32 ? z[0][v] : z[1][v] : x;
                lse = here ? __uint_as_float(lse_w[0][v >> 2][v & 3]) : lse;
                w = here ? __uint_as_float(lse_w[1][v >> 2][v & 3]) : w;
                mine |= here;
            }
            if (mine && (which & 31) == l32) {
                const float p = CLOSE ? exp_close(x - lse) : __builtin_amdgcn_exp2f(fmaf(x, kLog2e, -lse));
                float y = (p - 1.0f) * w;
                if (which < 32) tile_sum[0] -= w;
                else tile_sum[1] -= w;
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const uint32_t b = pack_bf16(y, 0.0f);
                    *reinterpret_cast<bf16_t *>(a.g + i * a.g_part + (int64_t)tile * a.g_slab + (int64_t)(first + which) * 64 + row * 2) = (bf16_t)b;
                    y -= low_bf16(b);
                }
            }
        }
    };

    // ---- the walk
    floatx16 za[2], zb[2];
    const std::integral_constant<int, (kResBufs - 2) * LOADS> younger;           // loads of the tiles behind the next (stores only make the wait longer)
    const std::integral_constant<int, (kResBufs - 1) * LOADS> younger_first;
    int buf = 0;
    wait_barrier(younger_first);
    read_group(std::integral_constant<int, 0>(), 0, fa[0]);
    read_group(std::integral_constant<int, 1>(), 0, fa[1]);
    if constexpr (G == 0 && ALONE) {
        read_bias(0);
        four_done(side);
    }
    reads_done(std::integral_constant<int, 0>(), fa[0]);
    // One tile: its products into `now`; the tile before, in `before`, is worked on between them if EARLIER
    auto walk = [&](auto turn_tag, auto earlier_tag, int i, floatx16 (&now)[2], floatx16 (&before)[2]) __attribute__((always_inline)) {
        constexpr int TURN = decltype(turn_tag)::value;
        constexpr bool EARLIER = decltype(earlier_tag)::value;
        const uint32_t at = buf * BUF;
        const int next_buf = buf == kResBufs - 1 ? 0 : buf + 1;
        const int ahead = t0 + (i + kResBufs < n_tiles ? i + kResBufs : n_tiles - 1);
        floatx16 start;
        if constexpr (G == 0 && !ALONE) {                // (the other wave has the SIMD meanwhile)
            const uint32_t from = rd_side + at;
            asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:32\n\tds_read_b128 %2, %4 offset:64\n\tds_read_b128 %3, %4 offset:96\n\t"
                         "s_waitcnt lgkmcnt(0)" : "=&v"(side[0]), "=&v"(side[1]), "=&v"(side[2]), "=&v"(side[3]) : "v"(from) : "memory");
        }
        if constexpr (G == 0)
#pragma unroll
            for (int v = 0; v < 16; ++v) start[v] = __uint_as_float(side[v >> 2][v & 3]);
        static_for<NG>([&](auto g_tag) __attribute__((always_inline)) {
            constexpr int GI = decltype(g_tag)::value, COUNT = TURN * NG + GI, CUR = COUNT % RING, NEXT = (COUNT + 1) % RING, AFTER = (COUNT + 2) % RING;
            if constexpr (G != 0 && GI == NG - 3) {
                if constexpr (ALONE && EARLIER) derivatives_end(before, t0 + i - 1);
                read_rows(at);
            }
            if constexpr (GI == NG - 2) {
                // this tile's buffer has been read: it takes the tile three on; the next tile is there
                wait_barrier(younger);
                if constexpr (G != 0) rows_done();
                if constexpr (G == 0 && ALONE) read_bias(next_buf * BUF);
            }
            if constexpr (GI < NG - 2) read_group(std::integral_constant<int, GI + 2>(), at, fa[AFTER]);
            else read_group(std::integral_constant<int, GI + 2 - NG>(), next_buf * BUF, fa[AFTER]);
            __builtin_amdgcn_sched_barrier(0);
            static_for<2>([&](auto f_tag) __attribute__((always_inline)) {
                constexpr int F = GI * 2 + decltype(f_tag)::value, K = F / PARTS, P = PARTS - 1 - F % PARTS;
                static_for<(PARTS - P) * 2>([&](auto m_tag) __attribute__((always_inline)) {
                    constexpr int M = decltype(m_tag)::value, J = M & 1, PB = PARTS - 1 - P - M / 2;
                    constexpr int S = PARTS == 3 ? K * 12 + (P == 2 ? 0 : P == 1 ? 2 : 6) + M : F * 2 + M;
                    if constexpr (S < 2 && G == 0) now[J] = start;
                    if constexpr (S < 2 && G != 0)
#pragma unroll
                        for (int v = 0; v < 16; ++v) now[J][v] = own_bias[J];
                    mfma_step<bf16_t>(fa[CUR][decltype(f_tag)::value], hb[PB][J][K], now[J]);
                    __builtin_amdgcn_sched_barrier(0);
                    // the requests go out between the last products, not in one burst
                    constexpr int LAST = PRODUCTS - res_products<PARTS>((NG - 2) * 2), L0 = PRODUCTS - LAST, FROM = (S - L0) * LOADS / LAST, TO = (S - L0 + 1) * LOADS / LAST;
                    if constexpr (S >= L0)
#pragma unroll
                        for (int l = FROM; l < TO; ++l) issue_one(ahead, buf, l);
                    if constexpr (ALONE && EARLIER && S < SLOTS) {
                        if constexpr (G == 0) statistics(std::integral_constant<int, S>(), before);
                        else derivatives(std::integral_constant<int, S>(), before, t0 + i - 1);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            // the next group is there (behind it at most the one after, and the rows' values)
            if constexpr (GI == NG - 3 && G != 0) reads_done(std::integral_constant<int, 11>(), fa[NEXT]);
            else reads_done(std::integral_constant<int, 2>(), fa[NEXT]);
            if constexpr (G == 0 && ALONE && GI == NG - 1) four_done(side);
        });
        buf = next_buf;
        if constexpr (ALONE && EARLIER && G == 0) statistics_end(before);
    };
    auto finish = [&](floatx16 (&last)[2], int tile) __attribute__((always_inline)) {
        static_for<SLOTS>([&](auto s_tag) __attribute__((always_inline)) {
            if constexpr (G == 0) statistics(s_tag, last);
            else derivatives(s_tag, last, tile);
            if constexpr (!ALONE && decltype(s_tag)::value % 2 == 1) __builtin_amdgcn_sched_barrier(0);       // (in turn: side by side they take registers)
        });
        if constexpr (G == 0) statistics_end(last);
        else derivatives_end(last, tile);
    };
    // The fragments that were asked for behind the last tile arrive before their registers are anybody else's.
    auto drain = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < RING; ++r) reads_done(std::integral_constant<int, 0>(), fa[r]);
        if constexpr (G == 0 && ALONE) four_done(side);
    };
    const std::integral_constant<int, 0> turn0;
    const std::integral_constant<int, 1> turn1;
    if constexpr (ALONE) {
        walk(turn0, std::false_type(), 0, za, zb);
        int i = 1;
        for (; i + 2 <= n_tiles; i += 2) {
            walk(turn1, std::true_type(), i, zb, za);
            walk(turn0, std::true_type(), i + 1, za, zb);
        }
        if (i < n_tiles) {
            walk(turn1, std::true_type(), i, zb, za);
            drain();
            finish(zb, t1 - 1);
        } else {
            drain();
            finish(za, t1 - 1);
        }
    } else {
        static_assert(ALONE || NG % RING == 0, "the fragments of the next tile's first group end up where it starts");
    static_assert(2 * NG % RING == 0, "... of the tile after the next");
        for (int i = 0; i < n_tiles; ++i) {
            walk(turn0, std::false_type(), i, za, za);
            finish(za, t0 + i);
        }
        drain();
    }
    if constexpr (G == 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {        // the two lanes of a row
            const float ref2 = __shfl_xor(ref[j], 32), sum2 = __shfl_xor(kept[j], 32), top = fmaxf(ref[j], ref2), m = top == -INFINITY ? 0.0f : top;
            const float s = kept[j] * exp_below(ref[j], m) + sum2 * exp_below(ref2, m);
            if (hf == 0) a.stat[((int64_t)range * blocks + rb) * kResRows + wave * 64 + j * 32 + l32] = make_float2(m, s);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {        // ... of a class
            const float own = colsum[j] + tile_sum[j], s = own + __shfl_xor(own, 32);
            if (hf == 0) a.db_part[(int64_t)range * blocks * kResRows + own_class + j * 32] = s;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // no load is on its way into LDS that is somebody else's by then
}

}  // namespace
}  // namespace jitdb
