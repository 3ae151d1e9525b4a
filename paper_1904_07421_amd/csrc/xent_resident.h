// The logits of many classes for states of ordinary width: the states stay in registers, the class weights stream past.
//
// A wave keeps the fragments of 64 rows (two MFMA tiles of 32) for all of K in registers, up to 256 of them; a block of four waves, 256
// rows, walks over a range of classes, 32 at a time.  The weights of 32 classes come straight into LDS, three buffers deep, and every
// wave reads each fragment once for its two products: half the LDS traffic of a tile whose two operands both come from LDS.
// One barrier a class tile.  What is done with a tile of logits (statistics, or the derivatives g) runs on the vector unit
// while the matrix cores multiply the next tile: two sets of accumulators take turns, and the work on the one is dealt out between the
// products of the other.
// Lane l holds row l % 32 of both tiles and, of the 32 classes, 8 q + 4 (l / 32) + e (q, e < 4): statistics are running
// maxima and sums in a lane's registers, put together once at the end.
#pragma once

#include "level_common.h"

#include <utility>

namespace jitdb {
namespace {

constexpr int kResT = 256;
constexpr int kResRows = 256;            // rows of a block
constexpr int kResClasses = 32;          // classes of a tile
constexpr int kResBufs = 3;
constexpr int kResPlaces = 256;          // a block a CU: its waves take more than half of the registers
constexpr int kResMinTiles = 8;          // a block's range of classes is no shorter
constexpr int kResBlocks = 1024;         // ranges of classes make no more blocks than this
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct ResArgs {
    const char *V; int64_t v_slab;       // class weights, K-blocked, the parts' slabs behind one another
    const char *h; int64_t h_slab;       // states, the same, from the chunk's first row on
    const float *bias;                   // padded with -inf to the last tile and 64 floats more
    int class_tiles;
    const int32_t *n_rows;
    int row0, max_rows;                  // the chunk: rows row0 .. row0 + max_rows of the list
    float2 *stat;                        // [splits][256 row blocks]: maximum, sum of exp(z - maximum)
    const int32_t *label_of;             // of the whole list
    const float *lse_of, *w_of;
    char *g; int64_t g_slab, g_part;     // g of the chunk, K-blocked with K = class
    float *db_part;                      // [4 row blocks of the chunk][32 class_tiles]
};
// Ranges of classes for `row_blocks` blocks of rows on a chip that holds `places` at once: more of them where that
// leaves fewer places idle in the last round, by more than 1 / 64.
__host__ __device__ inline int res_splits(int row_blocks, int class_tiles, int places) {
    if (row_blocks * 32 < places) {      // few rows: fill the chip
        const int fill = places / (row_blocks > 0 ? row_blocks : 1), most = class_tiles / kResMinTiles;
        return fill < most ? fill : most > 1 ? most : 1;
    }
    int best = 1, best_rounds = (row_blocks + places - 1) / places;
    for (int s = 2; s <= 32 && row_blocks * s <= kResBlocks && class_tiles >= s * kResMinTiles; ++s) {
        const int rounds = (row_blocks * s + places - 1) / places;
        if (rounds * best * 64 < best_rounds * s * 63) { best = s; best_rounds = rounds; }
    }
    return best;
}

template <typename F, int... I>
__device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void static_for(F &&f) { static_for_impl(f, std::make_integer_sequence<int, N>()); }

// e^x: the hardware's 2^t, corrected for the rounding of t = x log2 e.  (Not of -inf itself, whose correction would be NaN.)
__device__ __forceinline__ float exp_close(float x) {
    x = x < -200.0f ? -200.0f : x;
    const float t = x * kLog2e, p = __builtin_amdgcn_exp2f(t);
    return fmaf(p, kLn2 * fmaf(x, kLog2e, -t), p);
}

// A read of LDS that the compiler does not wait for: it would make it wait for every direct-to-LDS load in flight.
template <int OFFSET>
__device__ __forceinline__ void lds_read16(u32x4 &to, uint32_t at) { asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(to) : "v"(at), "n"(OFFSET) : "memory"); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// two values rounded to bf16 in one word
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// sum over the lane's row of 16, in every lane of it
__device__ __forceinline__ float row16_sum(float v) {
    v = dpp_add<0xB1>(v);                // lanes ^ 1
    v = dpp_add<0x4E>(v);                // lanes ^ 2
    v = dpp_add<0x141>(v);               // the other quad of eight
    return dpp_add<0x140>(v);            // the other eight of sixteen
}

// PARTS: bf16 parts of both operands; KS: K in steps of 16; G: 0 = statistics, else g in that many parts.
template <int PARTS, int KS, int G>
__global__ void __launch_bounds__(kResT, 1)
resident_logits_kernel(const ResArgs a) {
    constexpr int NF = PARTS * KS;                       // fragments of a class tile, 1 KB each
    constexpr int NG = (NF + 3) / 4;                     // groups of four
    constexpr int LOADS = (NF + 3) / 4;                  // per wave and tile; then the bias
    constexpr int BUF = NF * 1024 + 4 * 256;             // a copy of the bias for each wave
    constexpr bool CLOSE = PARTS == 3 || G == 3;         // fp32 results: exponentials good to a rounding
    __shared__ __attribute__((aligned(1024))) char lds[kResBufs * BUF];
    const int left = *a.n_rows - a.row0, rows = left < 0 ? 0 : left < a.max_rows ? left : a.max_rows;
    const int row_blocks = (rows + kResRows - 1) / kResRows;
    if (row_blocks == 0) return;
    const int splits = res_splits(row_blocks, a.class_tiles, kResPlaces);
    // neighbours on an XCD share their range of classes
    const int total = row_blocks * splits, per_xcd = (total + 7) / 8, place = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || place >= total) return;
    const int split = place / row_blocks, rb = place % row_blocks;
    const int t0 = (int)((int64_t)a.class_tiles * split / splits), t1 = (int)((int64_t)a.class_tiles * (split + 1) / splits);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hf = lane >> 5, l32 = lane & 31;
    const int r0 = rb * kResRows + wave * 64;            // of the wave, in the chunk
    // ---- movers: 1 KB units of 16 rows of a slab, piece p of row r in slot p ^ ((r >> 2) & 3)
    const char *v_lane = a.V + (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 4) & 3)) * 16);
    const float *b_lane = a.bias + lane;
    auto issue = [&](int tile, int buf) __attribute__((always_inline)) {
        char *dst = lds + buf * BUF;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int u = wave + 4 * i;
            if (NF % 4 != 0 && u >= NF) u = NF - 1;      // the same bytes to the same place once more: every wave issues as many
            __builtin_amdgcn_global_load_lds(JITDB_GLOBAL_PTR(v_lane + (int64_t)(u >> 1) * a.v_slab + (int64_t)tile * 2048 + (u & 1) * 1024),
                                             JITDB_LDS_PTR(dst + u * 1024), 16, 0, 0);
        }
        __builtin_amdgcn_global_load_lds(JITDB_GLOBAL_PTR(b_lane + tile * kResClasses), JITDB_LDS_PTR(dst + NF * 1024 + wave * 256), 4, 0, 0);
    };
    auto wait_barrier = [&](auto n) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(n)::value) : "memory");
    };
    // ---- the states
    u32x4 hb[PARTS][2][KS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                hb[p][j][k] = *reinterpret_cast<const u32x4 *>(a.h + (int64_t)(p * (KS / 2) + k / 2) * a.h_slab + (int64_t)(r0 + j * 32 + l32) * 64 + (k & 1) * 32 + hf * 16);
    float lse[2], w[2];
    int label[2];
    if constexpr (G != 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = r0 + j * 32 + l32;
            const bool in = r < rows;                    // rows behind the last: exp(z - inf) = 0
            lse[j] = in ? a.lse_of[a.row0 + r] : INFINITY;
            w[j] = in ? a.w_of[a.row0 + r] : 0.0f;
            label[j] = in ? a.label_of[a.row0 + r] : -1;
            if (!CLOSE) lse[j] *= kLog2e;
        }
    }
    // nothing of the above may still be on its way when loads are counted
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const int n_tiles = t1 - t0;
#pragma unroll
    for (int b = 0; b < kResBufs; ++b) issue(t0 + (b < n_tiles ? b : n_tiles - 1), b);

    // ---- fragments
    const uint32_t lds_base = (uint32_t)(uintptr_t)JITDB_LDS_PTR(lds);
    uint32_t rd[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) rd[k] = lds_base + l32 * 64 + (((2 * k + hf) ^ ((l32 >> 2) & 3)) * 16);
    const uint32_t rd_bias = lds_base + NF * 1024 + wave * 256 + hf * 16;
    u32x4 fa[2][4], bias[4];
    // fragment f of a tile: K step f / PARTS, part PARTS - 1 - f % PARTS (the smallest first)
    auto read_group = [&](auto g_tag, uint32_t at, u32x4 (&f)[4]) __attribute__((always_inline)) {
        constexpr int GI = decltype(g_tag)::value;
        static_for<4>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int F = GI * 4 + decltype(i_tag)::value;
            if constexpr (F < NF) {
                constexpr int K = F / PARTS, P = PARTS - 1 - F % PARTS;
                lds_read16<(P * (KS / 2) + K / 2) * 2048>(f[decltype(i_tag)::value], rd[K & 1] + at);
            }
        });
    };
    auto read_bias = [&](uint32_t at) __attribute__((always_inline)) {
        static_for<4>([&](auto i_tag) __attribute__((always_inline)) {
            lds_read16<decltype(i_tag)::value * 32>(bias[decltype(i_tag)::value], rd_bias + at);
        });
    };
    auto reads_done = [&](u32x4 (&f)[4]) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]), "+v"(bias[0]), "+v"(bias[1]), "+v"(bias[2]), "+v"(bias[3]));
    };

    // ---- what happens to a tile of logits, in NG pieces
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f}, part[2] = {0.0f, 0.0f};
    float colsum[16], mine = 0.0f;
    uint32_t words[G > 0 ? G : 1][2][2];                 // [part][q & 1][pair]
    char *g_lane = a.g + (int64_t)(r0 + l32) * 64 + hf * 16;
    auto statistics = [&](auto g_tag, floatx16 (&z)[2]) __attribute__((always_inline)) {
        constexpr int GI = decltype(g_tag)::value, MAXES = (NG + 2) / 4;         // the first quarter: maxima
        if constexpr (GI < MAXES) {
            constexpr int E0 = GI * 16 / MAXES, E1 = (GI + 1) * 16 / MAXES;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float m = z[j][E0];
#pragma unroll
                for (int v = E0 + 1; v < E1; ++v) m = fmaxf(m, z[j][v]);
                part[j] = GI == 0 ? m : fmaxf(part[j], m);
                if constexpr (GI == MAXES - 1) {
                    const float next = fmaxf(top[j], part[j]), from = next == -INFINITY ? 0.0f : next;   // nothing but masked classes so far
                    sum[j] *= CLOSE ? exp_close(top[j] - from) : __builtin_amdgcn_exp2f((top[j] - from) * kLog2e);
                    top[j] = next;
                    part[j] = CLOSE ? from : from * kLog2e;
                }
            }
        } else {
            constexpr int E0 = (GI - MAXES) * 16 / (NG - MAXES), E1 = (GI - MAXES + 1) * 16 / (NG - MAXES);
#pragma unroll
            for (int v = E0; v < E1; ++v)
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[j] += CLOSE ? exp_close(z[j][v] - part[j]) : __builtin_amdgcn_exp2f(fmaf(z[j][v], kLog2e, -part[j]));
        }
    };
    auto derivatives = [&](auto g_tag, floatx16 (&z)[2], int tile) __attribute__((always_inline)) {
        constexpr int GI = decltype(g_tag)::value, Q0 = GI * 8 / NG, Q1 = (GI + 1) * 8 / NG;     // quads of four classes, four of each row tile
        static_for<Q1 - Q0>([&](auto q_tag) __attribute__((always_inline)) {
            constexpr int J = (Q0 + decltype(q_tag)::value) / 4, Q = (Q0 + decltype(q_tag)::value) % 4;
            const int rel = label[J] - tile * kResClasses - hf * 4;
            float d[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = z[J][4 * Q + e];
                const float p = CLOSE ? exp_close(v - lse[J]) : __builtin_amdgcn_exp2f(fmaf(v, kLog2e, -lse[J]));
                d[e] = CLOSE ? (p - (rel == 8 * Q + e ? 1.0f : 0.0f)) * w[J] : fmaf(p, w[J], rel == 8 * Q + e ? -w[J] : 0.0f);
                colsum[4 * Q + e] = J == 0 ? d[e] : colsum[4 * Q + e] + d[e];
            }
#pragma unroll
            for (int i = 0; i < G; ++i) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t x = pack_bf16(d[2 * k], d[2 * k + 1]);
                    words[i][Q & 1][k] = x;
                    if (i + 1 < G) { d[2 * k] -= low_bf16(x); d[2 * k + 1] -= high_bf16(x); }
                }
                if constexpr (Q & 1) {
                    // the halves of the wave exchange quads: eight classes of a row side by side in a lane
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
            // the bias' gradient: over the wave's 64 rows; lane i of each sixteen keeps value i
            if constexpr (J == 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float s = row16_sum(colsum[4 * Q + e]);
                    mine = (lane & 15) == 4 * Q + e ? s : mine;
                }
                if constexpr (Q == 3) {
                    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(mine), __float_as_uint(mine), false, false);
                    mine = __uint_as_float(s[0]) + __uint_as_float(s[1]);
                    if ((lane & 16) == 0)
                        a.db_part[((int64_t)(rb * 4 + wave) * a.class_tiles + tile) * kResClasses + ((lane & 15) >> 2) * 8 + hf * 4 + (lane & 3)] = mine;
                }
            }
        });
    };

    // ---- the walk: a tile of logits grows in one set of accumulators while the tile before it is worked on in the other
    floatx16 za[2], zb[2];
    const std::integral_constant<int, (kResBufs - 2) * (LOADS + 1)> younger;     // loads of the tiles behind the next (stores only make the wait longer)
    const std::integral_constant<int, (kResBufs - 1) * (LOADS + 1)> younger_first;
    int buf = 0;
    wait_barrier(younger_first);
    read_bias(0);
    read_group(std::integral_constant<int, 0>(), 0, fa[0]);
    reads_done(fa[0]);
    auto walk = [&](auto turn_tag, auto first_tag, int i, floatx16 (&now)[2], floatx16 (&before)[2]) __attribute__((always_inline)) {
        constexpr int TURN = decltype(turn_tag)::value;
        constexpr bool FIRST = decltype(first_tag)::value;
        const uint32_t at = buf * BUF;
        const int next_buf = buf == kResBufs - 1 ? 0 : buf + 1;
        static_for<NG>([&](auto g_tag) __attribute__((always_inline)) {
            constexpr int GI = decltype(g_tag)::value, CUR = (TURN * NG + GI) & 1;
            if constexpr (GI == 0) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) now[0][4 * q + e] = now[1][4 * q + e] = __uint_as_float(bias[q][e]);
            }
            if constexpr (GI == NG - 1) {
                // this tile's buffer has been read: it takes the tile three on; the next tile is there
                wait_barrier(younger);
                issue(t0 + (i + kResBufs < n_tiles ? i + kResBufs : n_tiles - 1), buf);
                read_bias(next_buf * BUF);
                read_group(std::integral_constant<int, 0>(), next_buf * BUF, fa[CUR ^ 1]);
            } else {
                read_group(std::integral_constant<int, GI + 1>(), at, fa[CUR ^ 1]);
            }
            __builtin_amdgcn_sched_barrier(0);
            static_for<4>([&](auto f_tag) __attribute__((always_inline)) {
                constexpr int F = GI * 4 + decltype(f_tag)::value;
                if constexpr (F < NF) {
                    constexpr int K = F / PARTS, P = PARTS - 1 - F % PARTS;
#pragma unroll
                    for (int p = PARTS - 1 - P; p >= 0; --p)
#pragma unroll
                        for (int j = 0; j < 2; ++j) mfma_step<bf16_t>(fa[CUR][decltype(f_tag)::value], hb[p][j][K], now[j]);
                }
            });
            if constexpr (!FIRST) {
                if constexpr (G == 0) statistics(g_tag, before);
                else derivatives(g_tag, before, t0 + i - 1);
                // one product, then its share of the other work
#pragma unroll
                for (int k = 0; k < (PARTS == 3 ? 16 : 8); ++k) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, G == 0 ? 4 : 8, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            reads_done(fa[CUR ^ 1]);
        });
        buf = next_buf;
    };
    auto finish = [&](floatx16 (&last)[2]) __attribute__((always_inline)) {
        static_for<NG>([&](auto g_tag) __attribute__((always_inline)) {
            if constexpr (G == 0) statistics(g_tag, last);
            else derivatives(g_tag, last, t1 - 1);
        });
    };
    walk(std::integral_constant<int, 0>(), std::true_type(), 0, za, zb);
    int i = 1;
    for (; i + 2 <= n_tiles; i += 2) {
        walk(std::integral_constant<int, 1>(), std::false_type(), i, zb, za);
        walk(std::integral_constant<int, 0>(), std::false_type(), i + 1, za, zb);
    }
    if (i < n_tiles) {
        walk(std::integral_constant<int, 1>(), std::false_type(), i, zb, za);
        finish(zb);
    } else {
        finish(za);
    }
    if constexpr (G == 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {        // the two lanes of a row
            const float top2 = __shfl_xor(top[j], 32), sum2 = __shfl_xor(sum[j], 32), m = fmaxf(top[j], top2), from = m == -INFINITY ? 0.0f : m;
            const float s = sum[j] * expf(top[j] - from) + sum2 * expf(top2 - from);
            if (hf == 0) a.stat[((int64_t)split * row_blocks + rb) * kResRows + wave * 64 + j * 32 + l32] = make_float2(m, s);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // no load is on its way into LDS that is somebody else's by then
}

}  // namespace
}  // namespace jitdb
