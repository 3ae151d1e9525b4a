// C = A^T B or A B^T in tiles, both operands streaming through LDS: the gradients' products, and logits of wide states.
//
// A block multiplies a tile of kTileA rows of A (128, 160 or 256) and 256 rows of B; each wave TM x TN MFMA tiles of 32 x 32.  In such a
// tile lane l holds row l % 32 of B and rows 8 q + 4 (l / 32) + e of A (q, e < 4).  K runs over stages of 64 bytes a row (32 bf16) that
// travel straight into LDS, one barrier a stage.  K_ROWS: the reduction runs over the operands' rows instead (32 a stage; a tile takes
// slabs of 32 columns each), transposed on the way out of LDS.  Two waves share a SIMD: eight of a block of 256 rows, else of two blocks of
// four.  (Four waves of twice the size, alone on their SIMDs, read less LDS and were no faster.)
// A direct load writes the 64 lanes' pieces to 1024 consecutive LDS bytes, 16 rows of 64: piece p of row r is kept in slot
// p ^ ((r >> 2) & 3), so that a fragment read of 16 rows touches 16 distinct 16-byte columns.
#pragma once

#include "xent_resident.h"

namespace jitdb {
namespace {

constexpr int kT = 256;                               // threads of the small kernels
template <int WM> constexpr int kTM = WM == 5 ? 5 : 2;
template <int WM> constexpr int kTN = WM == 5 ? 2 : 4;
template <int WM> constexpr int kTileT = WM == 4 ? 512 : 256;           // threads
template <int WM> constexpr int kTileBufs = WM == 4 ? 4 : 3;
template <int WM> constexpr int kTileBuf = (kTileA<WM> + kTileB) * 64;
template <int WM> constexpr int kTileWaves = WM == 4 ? 1 : 2;           // blocks on a CU

// Operands are K-blocked as in operand_offset, in one to three bf16 parts: part p, slab s (32 elements of K), row r
// at + p * part + s * slab + r * 64.
struct Operand {
    char *at;
    int64_t slab, part;
};
// The part products of one product, smallest first: four bits each, which part of A and of B.
struct Pairs {
    uint32_t code;
    int n;
};
inline Pairs make_pairs(int parts_a, int parts_b) {
    Pairs p = {};
    for (int w = 2; w >= 0; --w)
        for (int i = 0; i <= w; ++i)
            if (i < parts_a && w - i < parts_b) p.code |= (uint32_t)(i | (w - i) << 2) << (4 * p.n++);
    return p;
}
struct Product {
    Operand A, B;
    Pairs pairs;
    int a_slabs, b_slabs;           // K_ROWS: slabs there are; what lies behind the last is never read
};

// acc += stages s0 .. s0 + n_stages (n_stages >= 1); a0, b0: the tile's first row of each operand (K_ROWS: first slab).  The part products
// of 32 elements of K follow one another, so that each part comes from memory once and from L2 after that (both gradients' products, fp32
// 8192 x 160 x 10000: 338 us; with one part product behind the other, which read g twice as often, 426)
template <bool K_ROWS, int WM>
__device__ __forceinline__ void multiply_tile(const Product &p, int64_t a0, int64_t b0, int s0, int n_stages, char *lds, floatx16 (&acc)[kTM<WM>][kTN<WM>]) {
    constexpr int TM = kTM<WM>, TN = kTN<WM>, WAVES = kTileT<WM> / 64, WAVES_N = kTileB / (32 * TN);
    constexpr int A_UNITS = kTileA<WM> / 16, UNITS = A_UNITS + kTileB / 16, LOADS = (UNITS + WAVES - 1) / WAVES, BUFS = kTileBufs<WM>, BUF = kTileBuf<WM>, B_AT = A_UNITS * 1024;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WAVES_N, wn = wave % WAVES_N, hf = lane >> 5, l32 = lane & 31, lrow = lane >> 2;
    // movers: 1 KB units of 16 rows of a slab, those of A in front of those of B, LOADS a wave (scalar addresses and one offset for
    // every lane: no vector instruction is spent on them)
    const uint32_t lane_off = lrow * 64 + (K_ROWS ? lane & 3 : (lane & 3) ^ ((lane >> 4) & 3)) * 16;
    const char *from[LOADS];
    auto unit = [&](int i) __attribute__((always_inline)) {         // (the last wave's last may come twice: every wave issues as many)
        const int u = wave * LOADS + i;
        return UNITS % WAVES == 0 || u < UNITS ? u : UNITS - 1;
    };
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int u = unit(i), v = u < A_UNITS ? u : u - A_UNITS;
        const Operand &o = u < A_UNITS ? p.A : p.B;
        const int64_t first = u < A_UNITS ? a0 : b0;
        if constexpr (K_ROWS) {
            const int n_slabs = u < A_UNITS ? p.a_slabs : p.b_slabs;
            const int64_t s = first + (v >> 1) < n_slabs ? first + (v >> 1) : n_slabs - 1;
            from[i] = o.at + s * o.slab + (v & 1) * 1024;
        } else {
            from[i] = o.at + (first + v * 16) * 64;
        }
    }
    const int64_t a_stage = K_ROWS ? 32 * 64 : p.A.slab, b_stage = K_ROWS ? 32 * 64 : p.B.slab;
    int k = s0 / p.pairs.n, q = s0 - k * p.pairs.n, issued = 0;
    int64_t a_at = k * a_stage, b_at = k * b_stage, a_off, b_off;
    auto take_part = [&]() __attribute__((always_inline)) {
        const uint32_t i = p.pairs.code >> (4 * q) & 3, j = p.pairs.code >> (4 * q + 2) & 3;
        a_off = a_at + (i == 0 ? 0 : i == 1 ? p.A.part : 2 * p.A.part);
        b_off = b_at + (j == 0 ? 0 : j == 1 ? p.B.part : 2 * p.B.part);
    };
    take_part();
    auto issue_one = [&](int buf, int i) __attribute__((always_inline)) {
        const int u = unit(i);
        const char *at = from[i] + (u < A_UNITS ? a_off : b_off);
        __builtin_amdgcn_global_load_lds(JITDB_GLOBAL_PTR(at + lane_off), JITDB_LDS_PTR(lds + buf * BUF + u * 1024), 16, 0, 0);
    };
    auto advance = [&]() __attribute__((always_inline)) {        // behind the last stage the last one is asked for again: the waits count on it
        if (++issued >= n_stages) return;
        if (++q == p.pairs.n) {
            q = 0;
            a_at += a_stage;
            b_at += b_stage;
        }
        take_part();
    };
    int a_rd[2], b_rd[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (K_ROWS) {
            const int at = h * 1024 + (hf * 4 + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
            a_rd[h] = wm * TM * 2048 + at;
            b_rd[h] = B_AT + wn * TN * 2048 + at;
        } else {
            const int slot16 = ((2 * h + hf) ^ ((l32 >> 2) & 3)) * 16;
            a_rd[h] = wm * TM * 2048 + l32 * 64 + slot16;
            b_rd[h] = B_AT + wn * TN * 2048 + l32 * 64 + slot16;
        }
    }
    const uint32_t lds_base = (uint32_t)(uintptr_t)JITDB_LDS_PTR(lds);
    struct Frags {
        u32x4 a[TM], b[TN];
    };
    // tiles of 32 rows lie 2048 bytes apart in either layout
    auto read_one = [&](auto tile, uint32_t at, u32x4 &f) __attribute__((always_inline)) {
        constexpr int I = decltype(tile)::value;
        if constexpr (K_ROWS) {
            u32x2 lo, hi;
            lds_read8_turned<I * 2048>(lo, at);
            lds_read8_turned<I * 2048 + 512>(hi, at);
            f = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
        } else {
            lds_read16<I * 2048>(f, at);
        }
    };
    auto read_group = [&](int buf, int h, Frags &f) __attribute__((always_inline)) {
        const uint32_t aa = lds_base + buf * BUF + a_rd[h], bb = lds_base + buf * BUF + b_rd[h];
        static_for<(TM > TN ? TM : TN)>([&](auto i) __attribute__((always_inline)) {
            if constexpr (decltype(i)::value < TM) read_one(i, aa, f.a[decltype(i)::value]);
            if constexpr (decltype(i)::value < TN) read_one(i, bb, f.b[decltype(i)::value]);
        });
    };
    auto reads_done = [&](Frags &f) __attribute__((always_inline)) {
        if constexpr (TM == 2)
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f.a[0]), "+v"(f.a[1]), "+v"(f.b[0]), "+v"(f.b[1]), "+v"(f.b[2]), "+v"(f.b[3]));
        else
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f.a[0]), "+v"(f.a[1]), "+v"(f.a[2]), "+v"(f.a[3]), "+v"(f.a[4]), "+v"(f.b[0]), "+v"(f.b[1]));
    };
    auto multiply = [&](const Frags &f) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < TM * TN; ++m) mfma_step<bf16_t>(f.a[m / TN], f.b[m % TN], acc[m / TN][m % TN]);
    };
    // the next requests are dealt out between the MFMAs: a burst of them would hold the wave back until the memory pipeline took them
    auto multiply_and_issue = [&](const Frags &f, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < TM * TN; ++m) {
            mfma_step<bf16_t>(f.a[m / TN], f.b[m % TN], acc[m / TN][m % TN]);
            __builtin_amdgcn_sched_barrier(0);
            if (m < LOADS) issue_one(buf, m);
            __builtin_amdgcn_sched_barrier(0);
        }
        advance();
    };
    auto wait_barrier = [&](auto n) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(n)::value) : "memory");
    };
    const std::integral_constant<int, (BUFS - 1) * LOADS> first_left;    // loads of younger stages that may stay in flight
    const std::integral_constant<int, (BUFS - 2) * LOADS> next_left;
    const std::integral_constant<int, 0> none_left;
#pragma unroll
    for (int b = 0; b < BUFS; ++b) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) issue_one(b, i);
        advance();
    }
    Frags P, Q;
    int cur = 0;
    wait_barrier(first_left);
    read_group(0, 0, P);
    reads_done(P);
    // P holds the first half of stage g (buffer cur), whose buffer is free for stage g + BUFS behind the barrier
    for (int g = 0; g < n_stages; ++g) {
        const int next = cur == BUFS - 1 ? 0 : cur + 1;
        read_group(cur, 1, Q);
        __builtin_amdgcn_sched_barrier(0);
        multiply(P);
        __builtin_amdgcn_sched_barrier(0);
        reads_done(Q);
        wait_barrier(next_left);
        read_group(next, 0, P);
        __builtin_amdgcn_sched_barrier(0);
        multiply_and_issue(Q, cur);
        __builtin_amdgcn_sched_barrier(0);
        reads_done(P);
        cur = next;
    }
    wait_barrier(none_left);             // nothing is on its way into the buffers, and every wave is done with them
}

template <int TM, int TN>
__device__ __forceinline__ void clear_tile(floatx16 (&acc)[TM][TN]) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int g = 0; g < TN; ++g)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][g][v] = 0.0f;
}

// Blocks are dealt round-robin to the 8 XCDs, each with an L2 of its own: XCD x takes the x-th eighth of the places in order.
__device__ __forceinline__ int64_t xcd_order(int64_t total, int block) {
    const int64_t per = (total + 7) / 8, i = (int64_t)(block & 7) * per + (block >> 3);
    return (block >> 3) < per && i < total ? i : -1;
}
__device__ __forceinline__ int chunk_rows(const int32_t *n_rows, int row0, int max_rows) {
    const int left = *n_rows - row0;
    return left < 0 ? 0 : left < max_rows ? left : max_rows;
}

// ---- the two products with g -------------------------------------------------------------------------
// dh^T = V^T g^T: A = class weights, B = g, K = classes: the rows of both.  dV^T = h^T g: A = turned states, B = g, K = rows.  A's
// rows (columns) are features in either, so that a lane ends with four features of a row or class side by side.
// The stages of all tiles of B together are cut into equal ranges, as many as fill the chip, whatever the number of rows turns out to
// be; the blocks of a range, one for each tile of A, run side by side on an XCD and read the same g at the same time.  A block leaves its
// share of a tile in register order, grad_finish_kernel adds a tile's shares in order.
struct GradArgs {
    Product p;
    int a_tiles;
    const int32_t *n_rows;
    int row0, max_rows;
    int C;
    float *part;
    const int32_t *row_of;
    int H;
    void *out;
    float *acc;                     // dV over several chunks of rows
    const float *scale;             // what g was divided by (gradients in bf16)
};
template <bool WEIGHTS, int WM>
__device__ __forceinline__ GradPlan grad_plan(const GradArgs &a) {
    const int rows = chunk_rows(a.n_rows, a.row0, a.max_rows);
    return make_plan(WEIGHTS ? (a.C + kTileB - 1) / kTileB : (rows + kTileB - 1) / kTileB, WEIGHTS ? (rows + 31) / 32 : (a.C + 31) / 32,
                     a.p.pairs.n, kTilePlaces<WM>, a.a_tiles);
}
template <bool WEIGHTS, int WM>
__device__ __forceinline__ void grad_product(const GradArgs &a, char *lds, int block) {
    const GradPlan g = grad_plan<WEIGHTS, WM>(a);
    const int64_t place = xcd_order((int64_t)g.ranges * a.a_tiles, block);
    if (place < 0) return;
    const uint32_t range = (uint32_t)place / (uint32_t)a.a_tiles, at = (uint32_t)place - range * a.a_tiles;
    uint32_t s = range * g.per;
    const uint32_t end = s + g.per < g.total ? s + g.per : g.total;
    while (s < end) {
        const uint32_t bt = s / g.stages, s0 = s - bt * g.stages, n = end - s < g.stages - s0 ? end - s : g.stages - s0;
        floatx16 acc[kTM<WM>][kTN<WM>];
        clear_tile(acc);
        if constexpr (WEIGHTS) multiply_tile<false, WM>(a.p, (int64_t)at * kTileA<WM>, (int64_t)bt * kTileB, s0, n, lds, acc);
        else multiply_tile<true, WM>(a.p, (int64_t)at * (kTileA<WM> / 32), (int64_t)bt * (kTileB / 32), s0, n, lds, acc);
        float4 *out = reinterpret_cast<float4 *>(a.part + ((int64_t)(bt + range) * a.a_tiles + at) * (kTileA<WM> * kTileB)) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < kTM<WM>; ++i)
#pragma unroll
            for (int j = 0; j < kTN<WM>; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    out[((i * kTN<WM> + j) * 4 + v) * kTileT<WM>] = make_float4(acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]);
        s += n;
    }
}
// The first `half` blocks (a multiple of 8) compute dh, as many more dV: where one leaves places on the chip, the other takes them.
// 32768 x 512 x 50021 bf16: 3.24 ms, 1.04 PFLOP/s, of 1.54 that a large library product reaches; the clock falls to 1.6 - 1.85 GHz under it.
template <int WM>
__global__ void __launch_bounds__(kTileT<WM>, kTileWaves<WM>)
grad_product_kernel(const GradArgs h, const GradArgs v, int half) {
    __shared__ __attribute__((aligned(1024))) char lds[kTileBufs<WM> * kTileBuf<WM>];
    if ((int)blockIdx.x < half) grad_product<false, WM>(h, lds, blockIdx.x);
    else grad_product<true, WM>(v, lds, blockIdx.x - half);
}
// A tile's shares are put together in a piece for each of a wave's MFMA tiles; a lane writes 32 features of its row or class, the wave's
// halves taking every other four, so that a block writes at least half a line of a row (32768 x 512 x 50021 bf16: 81 us; in pieces of
// four features, whose lines several XCDs share, 127).
template <bool WEIGHTS, int WM, typename O>
__device__ __forceinline__ void grad_finish(const GradArgs &a, const GradPlan &g, int64_t piece) {
    constexpr int TM = kTM<WM>, TN = kTN<WM>, WAVES_N = kTileB / (32 * TN);
    const int t = threadIdx.x;
    const uint32_t tile = (uint32_t)piece / (TM * TN), ij = (uint32_t)piece % (TM * TN), i = ij / TN, j = ij % TN, bt = tile / (uint32_t)a.a_tiles, at = tile - bt * a.a_tiles;
    const int lane = t & 63, wave = t >> 6;
    const int m0 = at * kTileA<WM> + wave / WAVES_N * (TM * 32) + i * 32 + (lane >> 5) * 4;                // first feature, and 8, 16, 24 on
    const int n = bt * kTileB + wave % WAVES_N * (TN * 32) + j * 32 + (lane & 31);                          // row or class
    if (m0 >= a.H || n >= (WEIGHTS ? a.C : chunk_rows(a.n_rows, a.row0, a.max_rows))) return;
    float s[4][4] = {};
    if (g.stages > 0) {
        const uint32_t first = bt * g.stages / g.per, last = ((bt + 1) * g.stages - 1) / g.per;
        const float4 *in = reinterpret_cast<const float4 *>(a.part + ((int64_t)(bt + first) * a.a_tiles + at) * (kTileA<WM> * kTileB)) + ij * 4 * kTileT<WM> + t;
#pragma unroll 2
        for (uint32_t k = first; k <= last; ++k) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float4 p = in[v * kTileT<WM>];
                s[v][0] += p.x; s[v][1] += p.y; s[v][2] += p.z; s[v][3] += p.w;
            }
            in += (int64_t)a.a_tiles * (kTileA<WM> * kTileB / 4);
        }
    }
    const int64_t row = (WEIGHTS ? (int64_t)n : (int64_t)a.row_of[a.row0 + n]) * a.H;
    const bool more = WEIGHTS && *a.n_rows - a.row0 > a.max_rows;       // chunks to come
    const float scale = sizeof(O) == 2 ? *a.scale : 1.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int m = m0 + v * 8, left = a.H - m < 4 ? a.H - m : 4;
        if (left <= 0) break;
        const int64_t to = row + m;
        if (WEIGHTS && a.row0 > 0)
            for (int k = 0; k < left; ++k) s[v][k] += a.acc[to + k];
        if (more) {
            for (int k = 0; k < left; ++k) a.acc[to + k] = s[v][k];
            continue;
        }
        O e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = from_f32<O>(s[v][k] * scale);
        O *o = static_cast<O *>(a.out) + to;
        if (left == 4) {
            __builtin_memcpy(o, e, sizeof(e));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < left) o[k] = e[k];
        }
    }
}

// db: 64 classes a block; its waves take the sums there are (4 of each 256 rows, or, places > 0, one of each range of resident_kernel's)
// in turn, each in order
struct BiasArgs {
    const float *part;
    float *db;
    const float *scale;             // nullptr: 1
    int width, places;              // classes in whole blocks; resident_kernel's places
};
template <int WAVES>
__device__ __forceinline__ void bias_finish(const BiasArgs &b, const GradArgs &a, int rows, int c0, float (&sums)[WAVES][64]) {
    const int n = rows == 0 ? 0 : b.places > 0 ? res_ranges(b.width / kResRows, (rows + 63) / 64 * 2, b.places) : (rows + 255) / 256 * 4;
    const int l = threadIdx.x & 63, q = threadIdx.x >> 6, c = c0 + l;
    float s = 0.0f;
    if (c < a.C)
#pragma unroll 4
        for (int p = q; p < n; p += WAVES) s += b.part[(int64_t)p * b.width + c];
    __syncthreads();                    // (the sums of the 64 classes before have been read)
    sums[q][l] = s;
    __syncthreads();
    if (q || c >= a.C) return;
#pragma unroll
    for (int k = 1; k < WAVES; ++k) s += sums[k][l];
    if (b.scale) s *= *b.scale;
    b.db[c] = a.row0 > 0 ? b.db[c] + s : s;
}
// Blocks take pieces in turn: how many there are depends on the number of rows, which the host does not know.
template <int WM, typename O>
__global__ void __launch_bounds__(kTileT<WM>)
grad_finish_kernel(const GradArgs h, const GradArgs v, const BiasArgs bias) {
    constexpr int WAVES = kTileT<WM> / 64, PIECES = kTM<WM> * kTN<WM>;
    __shared__ float sums[WAVES][64];
    const int rows = chunk_rows(h.n_rows, h.row0, h.max_rows);
    if (rows == 0 && h.row0 > 0) return;                         // the chunks before have had all rows
    const GradPlan gh = grad_plan<false, WM>(h), gv = grad_plan<true, WM>(v);
    const int64_t n_h = (int64_t)gh.b_tiles * h.a_tiles * PIECES, n_v = (int64_t)gv.b_tiles * v.a_tiles * PIECES, n = n_h + n_v + (v.C + 63) / 64;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        if (i < n_h) grad_finish<false, WM, O>(h, gh, i);
        else if (i < n_h + n_v) grad_finish<true, WM, O>(v, gv, i - n_h);
        else bias_finish<WAVES>(bias, v, rows, (int)(i - n_h - n_v) * 64, sums);
    }
}

// ---- logits of wide states: both operands stream ---------------------------------------------------------
// G = 0: A = class weights, B = states; statistics of every 64 classes.  G > 0: A = states, B = class weights; g.
struct LogitArgs {
    Product p;
    int nk, a_tiles, b_tiles;       // (those of the rows are known on the device)
    const int32_t *n_rows;
    int row0, max_rows;
    const float *bias;              // padded with -inf
    float2 *stat;                   // [2 a_tiles][max_rows]
    const float *side;              // the rows' records, as in ResArgs
    char *g; int64_t g_slab, g_part;
    float *db_part;                 // [2 row tiles][256 b_tiles]
};
template <int G, bool CLOSE>
__global__ void __launch_bounds__(kTileT<2>, 2)
wide_logits_kernel(const LogitArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[kTileBufs<2> * kTileBuf<2>];
    const int rows = chunk_rows(a.n_rows, a.row0, a.max_rows);
    const int row_tiles = (rows + 255) / 256 * (G == 0 ? 1 : 2), class_tiles = G == 0 ? a.a_tiles : a.b_tiles;
    const int64_t i = xcd_order((int64_t)row_tiles * class_tiles, (int)blockIdx.x);
    if (i < 0) return;
    // bands of row tiles, class tiles one after another inside a band: the blocks of an XCD share them in its L2
    const int band = (int)(i / (kBand * (int64_t)class_tiles)), rem = (int)(i - (int64_t)band * kBand * class_tiles);
    const int left = row_tiles - band * kBand, width = left < kBand ? left : kBand;
    const int ct = rem / width, rt = band * kBand + rem % width;
    floatx16 acc[2][4];
    clear_tile(acc);
    const int n_stages = a.nk * a.p.pairs.n;
    multiply_tile<false, 2>(a.p, (int64_t)(G == 0 ? ct : rt) * 128, (int64_t)(G == 0 ? rt : ct) * 256, 0, n_stages, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, hf = lane >> 5, l32 = lane & 31;
    if constexpr (G == 0) {
        const int c0 = ct * 128 + wm * 64;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 b = *reinterpret_cast<const float4 *>(a.bias + c0 + t * 32 + q * 8 + hf * 4);
                const float e[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[t][j][4 * q + k] += e[k];
            }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = rt * 256 + wn * 128 + j * 32 + l32;
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v) top = fmaxf(top, acc[t][j][v]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float from = top == -INFINITY ? 0.0f : top;       // every class masked: the sum is 0, not NaN
            float s = 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v) s += CLOSE ? exp_close(acc[t][j][v] - from) : __expf(acc[t][j][v] - from);
            if (top == INFINITY) {                                  // (inf - inf is no number)
                s = 1.0f;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (acc[t][j][v] != acc[t][j][v]) s = acc[t][j][v];
            }
            s += __shfl_xor(s, 32);
            if (hf == 0) a.stat[(int64_t)(2 * ct + wm) * a.max_rows + r] = make_float2(from, s);
        }
    } else {
        const int c0 = ct * 256 + wn * 128 + l32, r0 = rt * 128 + wm * 64;
        float colsum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        float own_bias[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) own_bias[j] = a.bias[c0 + j * 32];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int qq = 0; qq < 2; ++qq) {             // two quads of rows: the wave's halves exchange them for stores of 16 bytes
                const float *rec = a.side + (int64_t)(r0 / 32 + t) * 128 + qq * 16 + hf * 4;
                float lse[2][4], w[2][4];
                int label[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    __builtin_memcpy(lse[i], rec + i * 8, 16);
                    __builtin_memcpy(w[i], rec + i * 8 + 32, 16);
                    __builtin_memcpy(label[i], rec + i * 8 + 64, 16);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t words[G][2][2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float d[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float z = acc[t][j][4 * (2 * qq + i) + e] + own_bias[j];
                            const float p = CLOSE ? exp_close(z - lse[i][e]) : __builtin_amdgcn_exp2f(fmaf(z, kLog2e, -lse[i][e]));
                            d[e] = (p - (label[i][e] == c0 + j * 32 ? 1.0f : 0.0f)) * w[i][e];
                            colsum[j] += d[e];
                        }
#pragma unroll
                        for (int k = 0; k < G; ++k)
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const uint32_t y = pack_bf16(d[2 * m], d[2 * m + 1]);
                                words[k][i][m] = y;
                                d[2 * m] -= low_bf16(y);
                                d[2 * m + 1] -= high_bf16(y);
                            }
                    }
#pragma unroll
                    for (int k = 0; k < G; ++k) {
                        u32x4 out;
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const auto s = __builtin_amdgcn_permlane32_swap(words[k][0][m], words[k][1][m], false, false);
                            out[m] = s[0];
                            out[2 + m] = s[1];
                        }
                        *reinterpret_cast<u32x4 *>(a.g + k * a.g_part + (int64_t)(r0 / 32 + t) * a.g_slab + (int64_t)(c0 + j * 32) * 64 + qq * 32 + hf * 16) = out;
                    }
                }
            }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float s = colsum[j] + __shfl_xor(colsum[j], 32);
            if (hf == 0) a.db_part[((int64_t)(rt * 2 + wm) * a.b_tiles) * 256 + c0 + j * 32] = s;
        }
    }
}

}  // namespace
}  // namespace jitdb
