// Softmax cross entropy over classes or words: loss of every labelled node and the gradients of states, class weights and bias,
// without the logits of the batch ever being kept.  (Few classes take the kernels of xent_few.h.)
//
//     z_nc = <h_n, V_c> + b_c     lse_n = log sum_c exp z_nc     loss_n = lse_n - z_n,label(n)
//     g_nc = gloss_n (exp(z_nc - lse_n) - [c = label(n)])
//     dh_n = sum_c g_nc V_c       dV_c = sum_n g_nc h_n          db_c = sum_n g_nc
//
// Only nodes with a label are multiplied: label_rows_kernel lists them (their number stays on the device, and every later kernel
// reads it there), and their states are laid out for the matrix cores.  Forward: the logits go through the matrix cores and leave
// maximum and sum of exponentials of a range of classes for each row; join_kernel puts those together.  Backward: the same logits
// become g, which is kept for a bounded chunk of rows; two products with it give the gradients.
//
// Everything is multiplied on the bf16 matrix cores with fp32 accumulators.  An fp32 operand is the sum of three bf16 parts
// (8 mantissa bits each, 24 in all) and a product of two of them is the six part products of weight 2^-16 and more; what is left out
// is about 2^-23 of the product at most, two roundings of an fp32 multiplication, at 2.5 times the rate of the fp32 matrix instructions.
// g, computed in fp32, is multiplied as one bf16 part where the gradients leave in bf16 (a rounding of 2^-8 on terms of a sum that
// is itself rounded to 2^-8: norm-wise up to 2.4e-3 of the gradients, of which rounding them alone is 1.7e-3), in three parts where they leave
// in fp32 (two would leave 2.5e-6 of them, as a norm: more than the fp32 sums do).  The bias' gradient sums fp32 values.
// Of a likely label's competitors g is small, its own is nearly -gloss: where that is rounded, all of the row's gradient is off by as much,
// and where every gloss is the same (a mean), all gradients in the same direction.  So the one part is of g / m, m the significand of the
// largest |gloss|: weights that are alike are powers of two then, and m is multiplied into the sums, in fp32.

#include "xent_few.h"
#include "xent_tile.h"

namespace jitdb {
namespace {

constexpr float kMaxBf16 = 0x1.FEp127f;

// ---- the labelled rows -----------------------------------------------------------------------------
struct RowList {
    const int32_t *label;       // [N], -1: none
    const float *lse, *gloss;   // [N] (backward); gloss may be nullptr
    int64_t n;
    int C, per_block;           // labels of a block
    float lse_scale;            // of the records' log-sum-exp
    int32_t *counts;            // labelled rows of each block of labels
    int32_t *n_rows;            // how many there are
    int32_t *row_of;            // [N + pad]
    int32_t *label_of;          // forward: the same rows' labels (-1: names no class)
    float *side;                // backward: records of 32 rows, as in ResArgs
    float *big, *scale;         // gradients in bf16: largest |gloss| of each block of labels; its significand over all of them
    float *loss_out, *lse_out;  // forward: 0 for rows without a label
};
// what a row adds to the largest |gloss|
__device__ __forceinline__ float weight_size(float w, int32_t label) { return label != -1 && fabsf(w) < INFINITY ? fabsf(w) : 0.0f; }
// in [1, 2); 1 where there is none (0, and what is below the normal range)
__device__ __forceinline__ float significand(float v) {
    const uint32_t u = __float_as_uint(v);
    return u >> 23 ? __uint_as_float((u & 0x7FFFFFu) | 0x3F800000u) : 1.0f;
}
// sum and maximum over a block
__device__ __forceinline__ void block_sum_max(int &c, float &big, int32_t (&red)[kT / 64], float (&red_big)[kT / 64]) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        c += __shfl_xor(c, m);
        big = fmaxf(big, __shfl_xor(big, m));
    }
    if ((threadIdx.x & 63) == 0) {
        red[threadIdx.x >> 6] = c;
        red_big[threadIdx.x >> 6] = big;
    }
    __syncthreads();
    c = red[0] + red[1] + red[2] + red[3];
    big = fmaxf(fmaxf(red_big[0], red_big[1]), fmaxf(red_big[2], red_big[3]));
}
__device__ __forceinline__ void count_labels(const RowList &a, int block) {
    __shared__ int32_t red[kT / 64];
    __shared__ float red_big[kT / 64];
    int c = 0;
    float big = 0.0f;
    const bool weights = a.scale && a.gloss;
    const int64_t at = (int64_t)block * a.per_block;
    for (int i0 = 0; i0 < a.per_block; i0 += kLabelBlock) {     // (all loads of a turn on their way at once)
        constexpr int TURN = kLabelBlock / kT;
        int32_t label[TURN];
        float w[TURN];
#pragma unroll
        for (int u = 0; u < TURN; ++u) {
            const int64_t i = at + i0 + u * kT + threadIdx.x;
            label[u] = i < a.n ? a.label[i] : -1;
            w[u] = weights && i < a.n ? a.gloss[i] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < TURN; ++u) {
            c += label[u] != -1;
            big = fmaxf(big, weight_size(w[u], label[u]));
        }
    }
    block_sum_max(c, big, red, red_big);
    if (threadIdx.x == 0) {
        a.counts[block] = c;
        if (weights) a.big[block] = big;
    }
}
// Lists the rows in ascending order.  The last block also knows their number, and fills the last 256 rows' records.
__global__ void __launch_bounds__(kT)
label_rows_kernel(const RowList a) {
    __shared__ int32_t red[kT / 64];
    __shared__ float red_big[kT / 64];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const bool weights = a.scale && a.gloss;
    int base = 0;
    float big = 0.0f;
    for (int i = t; i < (int)gridDim.x && gridDim.x > 1; i += kT) {
        base += i < (int)blockIdx.x ? a.counts[i] : 0;
        if (weights) big = fmaxf(big, a.big[i]);
    }
    if (weights && gridDim.x == 1)                              // (a single block is not asked before)
        for (int i = t; i < a.n; i += kT) big = fmaxf(big, weight_size(a.gloss[i], a.label[i]));
    block_sum_max(base, big, red, red_big);
    const float scale = significand(big);
    auto record = [&](int at, float lse, float w, int32_t label) {
        float *rec = a.side + (int64_t)(at >> 5) * 128 + (at & 31);
        rec[0] = lse;
        rec[32] = w;
        rec[64] = __int_as_float(label);
    };
    for (int i0 = 0; i0 < a.per_block; i0 += kT) {
        const int64_t i = (int64_t)blockIdx.x * a.per_block + i0 + t;
        const int32_t label = i < a.n ? a.label[i] : -1;
        const bool has = label != -1;
        const uint64_t votes = __ballot(has);
        __syncthreads();
        if (lane == 0) red[wave] = __popcll(votes);
        __syncthreads();
        int at = base + __popcll(votes & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) at += red[w];
        if (has) {
            const bool known = label >= 0 && label < a.C;           // a label that names no class makes its row NaN
            a.row_of[at] = (int32_t)i;
            if (a.side) record(at, a.lse[i] * a.lse_scale, !known ? __builtin_nanf("") : a.gloss ? a.gloss[i] / scale : 1.0f, known ? label : -1);
            else a.label_of[at] = known ? label : -1;
        } else if (i < a.n && a.loss_out) {
            a.loss_out[i] = 0.0f;
            a.lse_out[i] = 0.0f;
        }
        base += red[0] + red[1] + red[2] + red[3];
    }
    if (blockIdx.x != gridDim.x - 1) return;
    if (t == 0) {
        *a.n_rows = base;
        if (a.scale) *a.scale = scale;
    }
    if (a.side && base + t < (base + 255) / 256 * 256) record(base + t, INFINITY, 0.0f, -1);       // exp(z - inf) = 0
}

// ---- packing ---------------------------------------------------------------------------------------
// bf16 parts of eight values: v = sum of parts, exactly for three of them (down to the smallest bf16).  The first is held at the largest
// bf16, which fp32 goes beyond by up to half its step.
template <typename T, int PARTS>
__device__ __forceinline__ void store_parts(const T (&e)[8], char *to, int64_t part) {
    if constexpr (sizeof(T) == 2) {
        __builtin_memcpy(to, e, 16);
    } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e[j];
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (i == 0) w[j] = pack_bf16(__builtin_amdgcn_fmed3f(v[2 * j], -kMaxBf16, kMaxBf16), __builtin_amdgcn_fmed3f(v[2 * j + 1], -kMaxBf16, kMaxBf16));
                else w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
                v[2 * j] -= low_bf16(w[j]);
                v[2 * j + 1] -= high_bf16(w[j]);
            }
            *reinterpret_cast<u32x4 *>(to + i * part) = w;
        }
    }
}
// Eight elements a thread; rows past the last one up to a multiple of 256 are zero.  map: row r of the operand is row map[r] of src.
template <typename T, int PARTS>
__device__ __forceinline__ void pack_rows(const T *__restrict__ src, const int32_t *__restrict__ map, int64_t n, int width, int slabs,
                                          const Operand &o, int block, int n_blocks) {
    const uint32_t pieces = (uint32_t)slabs * 4;
    const int64_t total = (n + 255) / 256 * 256 * pieces;
    for (int64_t q = (int64_t)block * kT + threadIdx.x; q < total; q += (int64_t)n_blocks * kT) {
        const int64_t r = total >> 32 ? q / pieces : (int64_t)((uint32_t)q / pieces);
        const int piece = (int)(q - r * pieces), k = piece * 8;
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = T(0);
        if (r < n && k < width) {
            const T *p = src + (map ? (int64_t)map[r] : r) * width + k;
            if (k + 8 <= width) {
                __builtin_memcpy(e, p, sizeof(e));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j < width) e[j] = p[j];
            }
        }
        store_parts<T, PARTS>(e, o.at + (piece >> 2) * o.slab + r * 64 + (piece & 3) * 16, o.part);
    }
}
// The turned states: row f = feature (f_rows of them, zero behind the last), K = row of the list, up to a multiple of 64.  A block
// turns 32 rows x 64 features through LDS.
template <typename T, int PARTS>
__device__ __forceinline__ void pack_turned(const T *__restrict__ src, const int32_t *__restrict__ map, int n, int H, int f_rows, const Operand &o,
                                            int block, int n_blocks) {
    __shared__ T tile[32][65];
    const int t = threadIdx.x, f_blocks = f_rows / 64, r_blocks = (n + 63) / 64 * 2;
    for (int64_t q = block; q < (int64_t)f_blocks * r_blocks; q += n_blocks) {
        const int rb = (int)(q / f_blocks), r0 = rb * 32, f0 = (int)(q - (int64_t)rb * f_blocks) * 64;
        for (int i = t >> 6; i < 32; i += 4) {
            const int f = f0 + (t & 63);
            tile[i][t & 63] = r0 + i < n && f < H ? src[(int64_t)map[r0 + i] * H + f] : T(0);
        }
        __syncthreads();
        const int f = t >> 2, piece = t & 3;
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = tile[piece * 8 + j][f];
        store_parts<T, PARTS>(e, o.at + rb * o.slab + (int64_t)(f0 + f) * 64 + piece * 16, o.part);
        __syncthreads();
    }
}

// z of the label itself, in fp32: a wave a row
template <typename T>
__device__ __forceinline__ void label_logits(const T *__restrict__ h, const T *__restrict__ V, const float *__restrict__ b, int n,
                                             const int32_t *__restrict__ row_of, const int32_t *__restrict__ label_of, int H, float *__restrict__ out,
                                             int block, int n_blocks) {
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)block * 4 + (threadIdx.x >> 6); r < n; r += (int64_t)n_blocks * 4) {
        const int c = label_of[r];
        float s = 0.0f;
        if (c >= 0) {
            const T *x = h + (int64_t)row_of[r] * H, *v = V + (int64_t)c * H;
#pragma unroll 4
            for (int k = lane; k < H; k += 64) s = fmaf(to_f32<T>(x[k]), to_f32<T>(v[k]), s);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
        if (lane == 0) out[r] = c >= 0 ? s + (b ? b[c] : 0.0f) : __builtin_nanf("");
    }
}
// rows without a label have no gradient
template <typename O>
__device__ __forceinline__ void clear_rows(const int32_t *__restrict__ label, int64_t n, int H, O *__restrict__ dh, int block, int n_blocks) {
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)block * 4 + (threadIdx.x >> 6); r < n; r += (int64_t)n_blocks * 4)
        if (label[r] == -1)
            for (int k = lane; k < H; k += 64) dh[r * H + k] = O(0);
}

// ---- the two launches around the listing of the rows: work that does not depend on one another shares each
struct PrepArgs {
    RowList list;
    const void *h, *V;
    const float *b;
    int H, C, Hf, slabs, n_bias;
    Operand h_op, v_op, ht;
    float *bias, *label_z;
    void *dh;
    int blocks[3];              // of each piece of work
};
// Counts the labels, packs the class weights, pads the bias.
template <typename T, int PARTS>
__global__ void __launch_bounds__(kT)
before_rows_kernel(const PrepArgs a) {
    int b = blockIdx.x;
    if (b < a.blocks[0]) { count_labels(a.list, b); return; }
    b -= a.blocks[0];
    if (b < a.blocks[1]) { pack_rows<T, PARTS>(static_cast<const T *>(a.V), nullptr, a.C, a.H, a.slabs, a.v_op, b, a.blocks[1]); return; }
    b -= a.blocks[1];
    for (int c = b * kT + threadIdx.x; c < a.n_bias; c += a.blocks[2] * kT) a.bias[c] = c >= a.C ? -INFINITY : a.b ? a.b[c] : 0.0f;
}
// Packs the rows' states; forward: the labels' own logits; backward: the turned states, zeros for the rows without a label.
template <typename T, int PARTS, bool BACKWARD, typename O>
__global__ void __launch_bounds__(kT)
after_rows_kernel(const PrepArgs a) {
    int b = blockIdx.x;
    const int n = *a.list.n_rows;
    if (b < a.blocks[0]) { pack_rows<T, PARTS>(static_cast<const T *>(a.h), a.list.row_of, n, a.H, a.slabs, a.h_op, b, a.blocks[0]); return; }
    b -= a.blocks[0];
    if constexpr (!BACKWARD) {
        label_logits<T>(static_cast<const T *>(a.h), static_cast<const T *>(a.V), a.b, n, a.list.row_of, a.list.label_of, a.H, a.label_z, b, a.blocks[1]);
    } else {
        if (b < a.blocks[1]) { pack_turned<T, PARTS>(static_cast<const T *>(a.h), a.list.row_of, n, a.H, a.Hf, a.ht, b, a.blocks[1]); return; }
        b -= a.blocks[1];
        clear_rows<O>(a.list.label, a.list.n, a.H, static_cast<O *>(a.dh), b, a.blocks[2]);
    }
}

// 64 rows a block; each of WAVES waves takes every WAVES-th set of statistics, then theirs are put together.
struct JoinArgs {
    const float2 *stat;
    int n_stat;                     // sets of max_rows rows; of resident_kernel's (class_tiles > 0): as many as it made
    int class_tiles, places;
    int row0, max_rows;
    const int32_t *n_rows, *row_of;
    const float *label_z;
    float *loss, *lse;
};
template <int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
join_kernel(const JoinArgs a) {
    __shared__ float2 red[WAVES][64];
    const int rows = chunk_rows(a.n_rows, a.row0, a.max_rows);
    if ((int)blockIdx.x * 64 >= rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.x * 64 + lane;
    int n_stat = a.n_stat;
    int64_t stride = a.max_rows;
    if (a.class_tiles > 0) {
        const int blocks = (rows + kResRows - 1) / kResRows;
        n_stat = res_ranges(blocks, a.class_tiles, a.places);
        stride = (int64_t)blocks * kResRows;
    }
    float top = -INFINITY, s = 0.0f;
    auto add = [&](float2 p) {
        if (p.y == 0.0f) return;                     // nothing but masked classes
        const float m = fmaxf(top, p.x);
        s = s * exp_below(top, m) + p.y * exp_below(p.x, m);
        top = m;
    };
    if (r < rows)
#pragma unroll 4
        for (int k = wave; k < n_stat; k += WAVES) add(a.stat[k * stride + r]);
    red[wave][lane] = make_float2(top, s);
    __syncthreads();
    if (wave || r >= rows) return;
    for (int w = 1; w < WAVES; ++w) add(red[w][lane]);
    const float v = top + logf(s);
    const int64_t at = a.row_of[a.row0 + r];
    a.lse[at] = v;
    a.loss[at] = v - a.label_z[a.row0 + r];
}

template <typename O>
__global__ void __launch_bounds__(kT)
clear_kernel(O *__restrict__ p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * kT + threadIdx.x; i < n; i += (int64_t)gridDim.x * kT) p[i] = O(0);
}

// ---- workspaces ----------------------------------------------------------------------------------------
struct Space {
    int32_t *counts, *n_rows, *row_of, *label_of;
    float *big, *scale, *side, *label_z, *bias, *db_part, *part_h, *part_v, *acc_v;
    float2 *stat;
    Operand h, v, ht, g;
    size_t bytes;
};
Operand take_operand(Carver &c, int parts, int64_t slabs, int64_t rows) {
    Operand o;
    o.slab = rows * 64;
    o.part = slabs * o.slab;
    o.at = c.take<char>((size_t)(parts * o.part));
    return o;
}
Space carve(const Sizes &s, bool backward, void *base) {
    Space w = {};
    Carver c(base);
    w.counts = c.take<int32_t>(s.label_blocks);
    w.n_rows = c.take<int32_t>(1);
    w.row_of = c.take<int32_t>(s.n_pad);
    w.bias = c.take<float>(s.Cp + 64);
    w.h = take_operand(c, s.parts, s.Hk / 32, s.n_pad);
    w.v = take_operand(c, s.parts, s.Hk / 32, s.Cp);
    if (!backward) {
        w.label_of = c.take<int32_t>(s.n_pad);
        w.label_z = c.take<float>(s.n_pad);
        w.stat = c.take<float2>(s.res ? (size_t)res_most(s.n_pad / kResRows, s.class_tiles) * kResRows : (size_t)(s.Cp / 64) * s.stat_rows);
    } else {
        w.side = c.take<float>((size_t)s.n_pad * 4);
        if (s.g_parts == 1) {
            w.big = c.take<float>(s.label_blocks);
            w.scale = c.take<float>(1);
        }
        w.ht = take_operand(c, s.parts, s.n_pad / 32, s.Hf);
        w.g = take_operand(c, s.g_parts, s.grad_rows / 32, s.Cp);
        w.db_part = c.take<float>(s.res ? (size_t)res_most(s.Cp / kResRows, s.grad_rows / kResTile) * kResRows : (size_t)(s.grad_rows / 64) * s.Cp);
        const int pairs = pair_count(s.parts, s.g_parts), tile = s.tile_a * kTileB;
        w.part_h = c.take<float>((size_t)(grad_parts(s, s.grad_rows / kTileB, ceil_div(s.C, 32), pairs) * tile));
        w.part_v = c.take<float>((size_t)(grad_parts(s, ceil_div(s.C, kTileB), s.grad_rows / 32, pairs) * tile));
        if (s.grad_rows < s.n) w.acc_v = c.take<float>((size_t)s.C * s.H);
    }
    w.bytes = c.off;
    return w;
}

unsigned grid_of(int64_t work) {        // grid of a kernel that loops: enough blocks to fill the chip
    const int64_t b = ceil_div(work, kT);
    return (unsigned)(b < 1 ? 1 : b < 4096 ? b : 4096);
}
unsigned xcd_grid(int64_t blocks) { return (unsigned)(8 * ceil_div(blocks, 8)); }

template <typename T, bool BACKWARD, typename O>
int prepare(const T *h, const T *V, const float *b, const RowList &list, const Sizes &s, const Space &w, O *dh, hipStream_t st) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    PrepArgs a = {};
    a.list = list; a.list.per_block = s.label_per;
    a.h = h; a.V = V; a.b = b; a.H = s.H; a.C = s.C; a.Hf = s.Hf; a.slabs = s.Hk / 32; a.n_bias = s.Cp + 64;
    a.h_op = w.h; a.v_op = w.v; a.ht = w.ht; a.bias = w.bias; a.label_z = w.label_z; a.dh = dh;
    a.blocks[0] = s.label_blocks > 1 ? s.label_blocks : 0;          // (nobody asks a single block how many stand in front of it)
    a.blocks[1] = (int)grid_of((int64_t)s.Cp * (s.Hk / 8));
    a.blocks[2] = (int)(ceil_div(a.n_bias, kT) < 64 ? ceil_div(a.n_bias, kT) : 64);
    before_rows_kernel<T, PARTS><<<(unsigned)(a.blocks[0] + a.blocks[1] + a.blocks[2]), kT, 0, st>>>(a);
    JITDB_LAUNCH_CHECK();
    label_rows_kernel<<<(unsigned)s.label_blocks, kT, 0, st>>>(a.list);
    JITDB_LAUNCH_CHECK();
    a.blocks[0] = (int)grid_of(s.n_pad * (s.Hk / 8));
    const int64_t waves = ceil_div(s.n, 4), turned = s.n_pad / 32 * (s.Hf / 64);
    a.blocks[1] = (int)(BACKWARD ? (turned < 4096 ? turned : 4096) : (waves < 4096 ? waves : 4096));
    a.blocks[2] = BACKWARD ? (int)(waves < 2048 ? waves : 2048) : 0;
    after_rows_kernel<T, PARTS, BACKWARD, O><<<(unsigned)(a.blocks[0] + a.blocks[1] + a.blocks[2]), kT, 0, st>>>(a);
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}
template <typename T, int G>
int launch_resident(int steps, int64_t blocks, const ResArgs &a, hipStream_t st) {
    const unsigned grid = xcd_grid(blocks);
    if constexpr (sizeof(T) == 4) {
        if (steps == 8) resident_kernel<3, 8, G><<<grid, kResT, 0, st>>>(a);
        else resident_kernel<3, 10, G><<<grid, kResT, 0, st>>>(a);
    } else {
        if (steps == 8) resident_kernel<1, 8, G><<<grid, kResT, 0, st>>>(a);
        else if (steps == 16) resident_kernel<1, 16, G><<<grid, kResT, 0, st>>>(a);
        else if (steps == 24) resident_kernel<1, 24, G><<<grid, kResT, 0, st>>>(a);
        else resident_kernel<1, 32, G><<<grid, kResT, 0, st>>>(a);
    }
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}

int launch_join(const JoinArgs &a, const Sizes &s, int64_t rows, hipStream_t st) {
    const unsigned blocks = (unsigned)ceil_div(rows, 64);
    if (join_waves(stat_sets(s)) == 16) join_kernel<16><<<blocks, 64 * 16, 0, st>>>(a);
    else join_kernel<4><<<blocks, 64 * 4, 0, st>>>(a);
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}
template <typename T>
int run_forward_xent(const T *h, const T *V, const float *b, const RowList &list, const Sizes &s, const Space &w,
                     float *loss, float *lse, hipStream_t st) {
    int rc = prepare<T, false, T>(h, V, b, list, s, w, nullptr, st);
    if (rc != JITDB_OK) return rc;
    JoinArgs j = {};
    j.stat = w.stat; j.n_rows = w.n_rows; j.row_of = w.row_of; j.label_z = w.label_z; j.loss = loss; j.lse = lse;
    if (s.res) {
        ResArgs a = {};
        a.res = w.h.at; a.res_slab = w.h.slab; a.str = w.v.at; a.str_slab = w.v.slab; a.side = w.bias;
        a.n_rows = w.n_rows; a.max_rows = (int)s.n_pad; a.class_tiles = s.class_tiles; a.stat = w.stat;
        if ((rc = launch_resident<T, 0>(s.res, res_most(s.n_pad / kResRows, s.class_tiles), a, st)) != JITDB_OK) return rc;
        j.class_tiles = s.class_tiles; j.places = res_places(s.parts * s.res, false); j.max_rows = a.max_rows;
        return launch_join(j, s, s.n, st);
    }
    LogitArgs a = {};
    a.p.A = w.v; a.p.B = w.h; a.p.pairs = make_pairs(s.parts, s.parts);
    a.nk = s.Hk / 32; a.a_tiles = s.Cp / 128; a.n_rows = w.n_rows; a.bias = w.bias; a.stat = w.stat;
    a.max_rows = j.max_rows = s.stat_rows; j.n_stat = stat_sets(s);
    for (int64_t r0 = 0; r0 < s.n; r0 += s.stat_rows) {
        a.row0 = (int)r0;
        a.p.B.at = w.h.at + r0 * 64;
        const int64_t rows = s.n - r0 < s.stat_rows ? s.n - r0 : s.stat_rows;
        wide_logits_kernel<0, sizeof(T) == 4><<<xcd_grid(ceil_div(rows, 256) * a.a_tiles), kTileT<2>, 0, st>>>(a);
        JITDB_LAUNCH_CHECK();
        j.row0 = a.row0;
        if ((rc = launch_join(j, s, rows, st)) != JITDB_OK) return rc;
    }
    return JITDB_OK;
}

// dh, dV and db of one chunk of rows
template <int WM, typename O>
int run_grad_products(int64_t row_tiles, const GradArgs &gh, const GradArgs &gv, BiasArgs bias, hipStream_t st) {
    const int64_t ranges = grad_ranges(kTilePlaces<WM>, gh.a_tiles), pieces = gh.a_tiles * (row_tiles + ceil_div(gv.C, kTileB)) * (kTM<WM> * kTN<WM>) + ceil_div(gv.C, 64);
    const unsigned half = xcd_grid(ranges * gh.a_tiles);
    grad_product_kernel<WM><<<2 * half, kTileT<WM>, 0, st>>>(gh, gv, (int)half);
    JITDB_LAUNCH_CHECK();
    grad_finish_kernel<WM, O><<<(unsigned)(pieces < 4096 ? pieces : 4096), kTileT<WM>, 0, st>>>(gh, gv, bias);
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}

template <typename T, typename O>
int run_backward_xent(const T *h, const T *V, const float *b, const RowList &list, const Sizes &s, const Space &w,
                      O *dh, O *dV, float *db, hipStream_t st) {
    constexpr int G_PARTS = sizeof(O) == 4 ? 3 : 1;
    int rc = prepare<T, true, O>(h, V, b, list, s, w, dh, st);
    if (rc != JITDB_OK) return rc;
    ResArgs ra = {};
    ra.res = w.v.at; ra.res_slab = w.v.slab; ra.str_slab = w.h.slab; ra.n_rows = w.n_rows; ra.max_rows = s.grad_rows;
    ra.class_blocks = s.Cp / kResRows; ra.bias = w.bias; ra.g = w.g.at; ra.g_slab = w.g.slab; ra.g_part = w.g.part; ra.db_part = w.db_part;
    LogitArgs a = {};
    a.p.A = w.h; a.p.B = w.v; a.p.pairs = make_pairs(s.parts, s.parts);
    a.nk = s.Hk / 32; a.b_tiles = s.Cp / 256; a.n_rows = w.n_rows; a.max_rows = s.grad_rows; a.bias = w.bias;
    a.g = w.g.at; a.g_slab = w.g.slab; a.g_part = w.g.part; a.db_part = w.db_part;
    GradArgs gh = {}, gv = {};
    gh.p.A = w.v; gh.p.B = w.g; gh.p.pairs = make_pairs(s.parts, s.g_parts); gh.p.a_slabs = s.Hk / 32; gh.p.b_slabs = s.grad_rows / 32;
    gh.part = w.part_h; gh.out = dh; gh.row_of = w.row_of;
    gv.p.A = w.ht; gv.p.B = w.g; gv.p.pairs = make_pairs(s.parts, s.g_parts);
    gv.part = w.part_v; gv.out = dV; gv.acc = w.acc_v;
    for (GradArgs *g : {&gh, &gv}) { g->scale = w.scale; g->a_tiles = s.a_tiles; g->n_rows = w.n_rows; g->max_rows = s.grad_rows; g->H = s.H; g->C = s.C; }
    for (int64_t r0 = 0; r0 < s.n; r0 += s.grad_rows) {
        const int64_t rows = s.n - r0 < s.grad_rows ? s.n - r0 : s.grad_rows, row_tiles = ceil_div(rows, 256);
        ra.row0 = a.row0 = gh.row0 = gv.row0 = (int)r0;
        if (s.res) {
            ra.str = w.h.at + r0 * 64;
            ra.side = w.side + r0 * 4;
            if ((rc = launch_resident<T, G_PARTS>(s.res, res_most(ra.class_blocks, row_tiles * (256 / kResTile)), ra, st)) != JITDB_OK) return rc;
        } else {
            a.p.A.at = w.h.at + r0 * 64;
            a.side = w.side + r0 * 4;
            wide_logits_kernel<G_PARTS, G_PARTS == 3><<<xcd_grid(2 * row_tiles * a.b_tiles), kTileT<2>, 0, st>>>(a);
            JITDB_LAUNCH_CHECK();
        }
        gv.p.A.at = w.ht.at + r0 / 32 * w.ht.slab;
        const BiasArgs bias = {w.db_part, db, w.scale, s.Cp, s.res ? res_places(s.parts * s.res, true) : 0};
        rc = s.wm == 4 ? run_grad_products<4, O>(row_tiles, gh, gv, bias, st) : s.wm == 5 ? run_grad_products<5, O>(row_tiles, gh, gv, bias, st)
                                                                                          : run_grad_products<2, O>(row_tiles, gh, gv, bias, st);
        if (rc != JITDB_OK) return rc;
    }
    return JITDB_OK;
}

// ---- few classes ---------------------------------------------------------------------------------------
// Of the backward pass, each of which leaves a set of sums.  A single block writes the gradients itself, a launch less (62 rows of 160,
// 5 classes, fp32: 12.1 -> 10.3 us in a graph; two turns of a single block lose: 128 rows 16.6 us, with two blocks 12.1).
int few_blocks(int64_t n) {
    const int64_t b = ceil_div(n, kFewRows);
    return (int)(b < 1024 ? b : 1024);
}
size_t few_part_bytes(int64_t n, int H, int C) {
    Carver c(nullptr);
    c.take<float>((size_t)few_blocks(n > 0 ? n : 1) * ((size_t)C * H + C));
    return c.off;
}
template <typename T>
int run_few_forward(const FewArgs &a, hipStream_t st) {
    const int64_t b = ceil_div(a.n, kFewRows);
    const unsigned blocks = (unsigned)(b < 2048 ? b : 2048);
    for_few<T>(a.H, a.C, [&](auto c, auto nb) { few_forward_kernel<T, decltype(c)::value, decltype(nb)::value><<<blocks, kFewT, 0, st>>>(a); });
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}
template <typename T, typename O>
int run_few_backward(FewArgs &a, O *dV, float *db, hipStream_t st) {
    const int blocks = few_blocks(a.n);
    if (blocks == 1) { a.dV = dV; a.db = db; }
    for_few<T>(a.H, a.C, [&](auto c, auto nb) { few_backward_kernel<T, O, decltype(c)::value, decltype(nb)::value><<<blocks, kFewT, 0, st>>>(a); });
    JITDB_LAUNCH_CHECK();
    if (blocks == 1) return JITDB_OK;
    few_reduce_kernel<O><<<(unsigned)ceil_div((int64_t)a.C * a.H + a.C, 64), 1024, 0, st>>>(a.part, blocks, a.H, a.C, dV, db);
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}

bool off_type(const void *p, jitdb_dtype t) { return reinterpret_cast<uintptr_t>(p) & (t == JITDB_F32 ? 3 : 1); }
bool off_word(const void *p) { return reinterpret_cast<uintptr_t>(p) & 3; }

}  // namespace
}  // namespace jitdb

using namespace jitdb;

extern "C" size_t jitdb_softmax_xent_workspace_bytes(int64_t n_rows, int32_t H, int32_t n_classes, jitdb_dtype dtype) {
    Sizes s;
    if (!make_sizes(n_rows, H, n_classes, dtype, dtype, s)) return 0;
    return few_fits(H, n_classes, dtype) ? 256 : carve(s, false, nullptr).bytes;      // (few classes need none: never 0, which is an error)
}
extern "C" size_t jitdb_softmax_xent_backward_workspace_bytes(int64_t n_rows, int32_t H, int32_t n_classes, jitdb_dtype dtype,
                                                              jitdb_dtype grad_dtype) {
    Sizes s;
    if (!make_sizes(n_rows, H, n_classes, dtype, grad_dtype, s)) return 0;
    return few_fits(H, n_classes, dtype) ? few_part_bytes(n_rows, H, n_classes) : carve(s, true, nullptr).bytes;
}

extern "C" int jitdb_softmax_xent_forward(const void *h, const void *V, const float *b, const int32_t *label,
                                          int64_t n_rows, int32_t H, int32_t n_classes, jitdb_dtype dtype,
                                          float *loss, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
    drop_stale_hip_error();
    Sizes s;
    if (!make_sizes(n_rows, H, n_classes, dtype, dtype, s)) return JITDB_E_BADARG;
    if (n_rows == 0) return JITDB_OK;
    if (!h || !V || !label || !loss || !lse || !workspace) return JITDB_E_NULL;
    if (off_type(h, dtype) || off_type(V, dtype) || off_word(b) || off_word(label) || off_word(loss) || off_word(lse) ||
        (reinterpret_cast<uintptr_t>(workspace) & 255))
        return JITDB_E_BADARG;
    if (workspace_bytes < jitdb_softmax_xent_workspace_bytes(n_rows, H, n_classes, dtype)) return JITDB_E_WORKSPACE;
    if (few_fits(H, n_classes, dtype)) {
        FewArgs a = {};
        a.h = h; a.V = V; a.b = b; a.label = label; a.n = n_rows; a.H = H; a.C = n_classes; a.loss = loss; a.lse = lse;
        return dtype == JITDB_F32 ? run_few_forward<float>(a, (hipStream_t)hip_stream) : run_few_forward<bf16_t>(a, (hipStream_t)hip_stream);
    }
    const Space w = carve(s, false, workspace);
    RowList list = {};
    list.label = label; list.n = n_rows; list.C = n_classes; list.counts = w.counts; list.n_rows = w.n_rows;
    list.row_of = w.row_of; list.label_of = w.label_of; list.loss_out = loss; list.lse_out = lse;
    hipStream_t st = (hipStream_t)hip_stream;
    if (dtype == JITDB_F32)
        return run_forward_xent<float>(static_cast<const float *>(h), static_cast<const float *>(V), b, list, s, w, loss, lse, st);
    return run_forward_xent<bf16_t>(static_cast<const bf16_t *>(h), static_cast<const bf16_t *>(V), b, list, s, w, loss, lse, st);
}

extern "C" int jitdb_softmax_xent_backward(const void *h, const void *V, const float *b, const int32_t *label, const float *lse,
                                           const float *gloss, int64_t n_rows, int32_t H, int32_t n_classes, jitdb_dtype dtype,
                                           jitdb_dtype grad_dtype, void *dh, void *dV, float *db,
                                           void *workspace, size_t workspace_bytes, void *hip_stream) {
    drop_stale_hip_error();
    Sizes s;
    if (!make_sizes(n_rows, H, n_classes, dtype, grad_dtype, s)) return JITDB_E_BADARG;
    if (!dV || !db) return JITDB_E_NULL;
    if (off_type(dV, grad_dtype) || off_word(db)) return JITDB_E_BADARG;
    hipStream_t st = (hipStream_t)hip_stream;
    if (n_rows == 0) {
        const int64_t weights = (int64_t)n_classes * H;
        if (grad_dtype == JITDB_F32) clear_kernel<float><<<grid_of(weights), kT, 0, st>>>(static_cast<float *>(dV), weights);
        else clear_kernel<bf16_t><<<grid_of(weights), kT, 0, st>>>(static_cast<bf16_t *>(dV), weights);
        JITDB_LAUNCH_CHECK();
        clear_kernel<float><<<grid_of(n_classes), kT, 0, st>>>(db, n_classes);
        JITDB_LAUNCH_CHECK();
        return JITDB_OK;
    }
    if (!h || !V || !label || !lse || !dh || !workspace) return JITDB_E_NULL;
    if (off_type(h, dtype) || off_type(V, dtype) || off_word(b) || off_word(label) || off_word(lse) || off_word(gloss) ||
        off_type(dh, grad_dtype) || (reinterpret_cast<uintptr_t>(workspace) & 255))
        return JITDB_E_BADARG;
    if (workspace_bytes < jitdb_softmax_xent_backward_workspace_bytes(n_rows, H, n_classes, dtype, grad_dtype)) return JITDB_E_WORKSPACE;
    if (few_fits(H, n_classes, dtype)) {
        FewArgs a = {};
        a.h = h; a.V = V; a.b = b; a.label = label; a.n = n_rows; a.H = H; a.C = n_classes; a.lse_in = lse; a.gloss = gloss;
        a.dh = dh; a.part = static_cast<float *>(workspace);
        if (dtype == JITDB_F32) return run_few_backward<float, float>(a, static_cast<float *>(dV), db, st);
        if (grad_dtype == JITDB_F32) return run_few_backward<bf16_t, float>(a, static_cast<float *>(dV), db, st);
        return run_few_backward<bf16_t, bf16_t>(a, static_cast<bf16_t *>(dV), db, st);
    }
    const Space w = carve(s, true, workspace);
    RowList list = {};
    list.label = label; list.lse = lse; list.gloss = gloss; list.n = n_rows; list.C = n_classes; list.counts = w.counts;
    list.n_rows = w.n_rows; list.row_of = w.row_of; list.side = w.side; list.big = w.big; list.scale = w.scale;
    list.lse_scale = grad_dtype == JITDB_F32 ? 1.0f : kLog2e;          // as the kernels' exponentials want it
    if (dtype == JITDB_F32)
        return run_backward_xent<float, float>(static_cast<const float *>(h), static_cast<const float *>(V), b, list, s, w,
                                               static_cast<float *>(dh), static_cast<float *>(dV), db, st);
    if (grad_dtype == JITDB_F32)
        return run_backward_xent<bf16_t, float>(static_cast<const bf16_t *>(h), static_cast<const bf16_t *>(V), b, list, s, w,
                                                static_cast<float *>(dh), static_cast<float *>(dV), db, st);
    return run_backward_xent<bf16_t, bf16_t>(static_cast<const bf16_t *>(h), static_cast<const bf16_t *>(V), b, list, s, w,
                                             static_cast<bf16_t *>(dh), static_cast<bf16_t *>(dV), db, st);
}
