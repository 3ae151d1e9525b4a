// Softmax cross entropy over classes or words: loss of every labelled node and the gradients of states, class weights and bias,
// without the logits of the batch ever being kept.  (Few classes take the kernels of xent_few.h.)
//
//     z_nc = <h_n, V_c> + b_c     lse_n = log sum_c exp z_nc     loss_n = lse_n - z_n,label(n)
//     g_nc = gloss_n (exp(z_nc - lse_n) - [c = label(n)])
//     dh_n = sum_c g_nc V_c       dV_c = sum_n g_nc h_n          db_c = sum_n g_nc
//
// Only nodes with a label are multiplied: label_rows_kernel lists them (their number stays on the device, and every later kernel
// reads it there), pack_rows_kernel gathers their states.  Forward: tiles of 128 classes x 256 rows of the product go through the
// matrix cores and leave maximum and sum of exponentials of their classes for each row; join_kernel puts those together.
// Backward: the same tiles become g, which is kept for a bounded chunk of rows; two products with it give the gradients.
//
// Everything is multiplied on the bf16 matrix cores with fp32 accumulators.  An fp32 operand is the sum of three bf16 parts
// (8 mantissa bits each, 24 in all) and a product of two of them is the six part products of weight 2^-16 and more; what is left out
// is below 2^-23 of the product, less than an fp32 multiplication rounds away, at 2.5 times the rate of the fp32 matrix instructions.
// g, computed in fp32, is multiplied as one bf16 part where the gradients leave in bf16 (a rounding of 2^-8 on terms of a sum that
// is itself rounded to 2^-8), in three parts where they leave in fp32 (two would leave 2.5e-6 of them, as a norm: more than the fp32
// sums do).  The bias' gradient sums fp32 values.

#include "xent_few.h"
#include "xent_resident.h"

namespace jitdb {
namespace {

constexpr int kT = 256;
constexpr int kTileA = 128, kTileB = 256;     // rows of the two operands in a tile: classes x nodes, features x nodes, classes x features
constexpr int kStageBytes = 64;               // of K per row and pipeline stage: 32 bf16
constexpr int kBufBytes = (kTileA + kTileB) * kStageBytes;
constexpr int kMaxPairs = 6;
constexpr int kMaxClasses = 1 << 22;
constexpr int kMaxWidth = 1 << 14;
constexpr int kLabelBlock = 4096;             // labels of a block of the two listing kernels
constexpr int kSlots = 512;                   // blocks the chip holds at once: two a CU
constexpr int64_t kStatBytes = 512ll << 20;   // of tile statistics kept at once (forward) ...
constexpr int64_t kGradBytes = 4ll << 30;     // ... and of g (backward): rows beyond come in further chunks

// ---- operands: K-blocked as in operand_offset, in one to three bf16 parts ------------------------
// Part p, slab s (32 elements of K), row r: at + p * part + s * slab + r * 64.
struct Operand {
    char *at;
    int64_t slab, part;
};
// The part products of one product, smallest first: where the parts lie behind each operand's first.  (Whole words: the
// compiler reads them with scalar loads, which the K loop's hand-counted waits for vector memory do not see.)
struct Pairs {
    int64_t a[kMaxPairs], b[kMaxPairs];
    int n;
};
Pairs make_pairs(const Operand &a, int parts_a, const Operand &b, int parts_b) {
    Pairs p = {};
    for (int w = 2; w >= 0; --w)
        for (int i = 0; i <= w; ++i)
            if (i < parts_a && w - i < parts_b) { p.a[p.n] = i * a.part; p.b[p.n] = (w - i) * b.part; ++p.n; }
    return p;
}
// bf16 parts of an fp32 value: v = sum of parts, exactly for three of them (down to the smallest bf16)
template <int PARTS>
__device__ __forceinline__ void split_parts(float v, bf16_t (&p)[PARTS]) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        p[i] = f32_to_bf16(v);
        v -= bf16_to_f32(p[i]);
    }
}

// ---- the labelled rows -----------------------------------------------------------------------------
struct RowList {
    const int32_t *label;       // [N], -1: none
    const float *lse, *gloss;   // [N] (backward); gloss may be nullptr
    int64_t n;
    int C;
    int32_t *counts;            // labelled rows of each block of labels
    int32_t *n_rows;            // how many there are
    int32_t *row_of;            // [N + pad]
    int32_t *label_of;          // the same rows' labels (-1: names no class), log-sum-exps and weights
    float *lse_of, *w_of;
    float *loss_out, *lse_out;  // forward: 0 for rows without a label
};
__global__ void __launch_bounds__(kT)
label_count_kernel(const RowList a) {
    __shared__ int32_t red[kT / 64];
    int c = 0;
    const int64_t at = (int64_t)blockIdx.x * kLabelBlock;
    for (int i = threadIdx.x; i < kLabelBlock; i += kT) c += at + i < a.n && a.label[at + i] != -1;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) c += __shfl_xor(c, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0) a.counts[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}
// Lists the rows in ascending order.  The last block also knows their number.
__global__ void __launch_bounds__(kT)
label_rows_kernel(const RowList a) {
    __shared__ int32_t red[kT / 64];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    int before = 0;
    for (int i = t; i < (int)blockIdx.x; i += kT) before += a.counts[i];
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) before += __shfl_xor(before, m);
    if (lane == 0) red[wave] = before;
    __syncthreads();
    int base = red[0] + red[1] + red[2] + red[3];
    for (int i0 = 0; i0 < kLabelBlock; i0 += kT) {
        const int64_t i = (int64_t)blockIdx.x * kLabelBlock + i0 + t;
        const int32_t label = i < a.n ? a.label[i] : -1;
        const bool has = label != -1;
        const uint64_t votes = __ballot(has);
        __syncthreads();
        if (lane == 0) red[wave] = __popcll(votes);
        __syncthreads();
        int at = base + __popcll(votes & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) at += red[w];
        if (has) {
            a.row_of[at] = (int32_t)i;
            const bool known = label >= 0 && label < a.C;           // a label that names no class makes its row NaN
            a.label_of[at] = known ? label : -1;
            if (a.lse) {
                a.lse_of[at] = a.lse[i];
                a.w_of[at] = !known ? __builtin_nanf("") : a.gloss ? a.gloss[i] : 1.0f;
            }
        } else if (i < a.n && a.loss_out) {
            a.loss_out[i] = 0.0f;
            a.lse_out[i] = 0.0f;
        }
        base += red[0] + red[1] + red[2] + red[3];
    }
    if (t == 0 && blockIdx.x == gridDim.x - 1) *a.n_rows = base;
}

// ---- packing ---------------------------------------------------------------------------------------
// Eight elements a thread; rows past the last one up to a multiple of a tile are zero.  map: row r of the operand is row map[r] of src.
template <typename T, int PARTS>
__global__ void __launch_bounds__(kT)
pack_rows_kernel(const T *__restrict__ src, const int32_t *__restrict__ map, const int32_t *__restrict__ n_dev, int64_t n_host, int width,
                 int slabs, int pad, Operand o) {
    const int64_t n = n_dev ? *n_dev : n_host, rows = (n + pad - 1) / pad * pad;
    const int pieces = slabs * 4;
    const int64_t total = rows * pieces;
    for (int64_t q = (int64_t)blockIdx.x * kT + threadIdx.x; q < total; q += (int64_t)gridDim.x * kT) {
        const int64_t r = q / pieces;
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
        bf16_t part[PARTS][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            bf16_t one[PARTS];
            if constexpr (sizeof(T) == 2) one[0] = e[j];
            else split_parts<PARTS>(e[j], one);
#pragma unroll
            for (int i = 0; i < PARTS; ++i) part[i][j] = one[i];
        }
#pragma unroll
        for (int i = 0; i < PARTS; ++i)
            __builtin_memcpy(o.at + i * o.part + (piece >> 2) * o.slab + r * 64 + (piece & 3) * 16, part[i], 16);
    }
}
// The transposed operand: row f = feature, K = class.  Blocks of 32 classes x 64 features turn through LDS.
template <typename T, int PARTS>
__global__ void __launch_bounds__(kT)
pack_turned_kernel(const T *__restrict__ V, int C, int H, int f_rows, Operand o) {
    __shared__ T tile[32][65];
    const int c0 = blockIdx.x * 32, f0 = blockIdx.y * 64, t = threadIdx.x;
    for (int i = t >> 6; i < 32; i += 4) {
        const int f = f0 + (t & 63);
        tile[i][t & 63] = c0 + i < C && f < H ? V[(int64_t)(c0 + i) * H + f] : T(0);
    }
    __syncthreads();
    const int f = t >> 2, piece = t & 3;
    if (f0 + f >= f_rows) return;
    bf16_t part[PARTS][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        bf16_t one[PARTS];
        if constexpr (sizeof(T) == 2) one[0] = tile[piece * 8 + j][f];
        else split_parts<PARTS>(tile[piece * 8 + j][f], one);
#pragma unroll
        for (int i = 0; i < PARTS; ++i) part[i][j] = one[i];
    }
#pragma unroll
    for (int i = 0; i < PARTS; ++i)
        __builtin_memcpy(o.at + i * o.part + blockIdx.x * o.slab + (int64_t)(f0 + f) * 64 + piece * 16, part[i], 16);
}
__global__ void __launch_bounds__(kT)
pad_bias_kernel(const float *__restrict__ b, int C, int n, float *__restrict__ out) {
    for (int c = blockIdx.x * kT + threadIdx.x; c < n; c += gridDim.x * kT) out[c] = c >= C ? -INFINITY : b ? b[c] : 0.0f;
}

// ---- the tiled product -------------------------------------------------------------------------------
// Four waves multiply a tile of 128 rows of A and 256 rows of B; each a 64 x 128 piece, 2 x 4 MFMA tiles of 32 x 32.  In a 32 x 32
// tile lane l holds row l % 32 of B and rows 8 q + 4 (l / 32) + e of A (q, e < 4).  K runs over stages of 64 bytes a row that
// travel straight into LDS, three buffers deep, one barrier a stage; two blocks share a CU, so that the start-up and the
// epilogue of one leave the matrix cores to the other.  K_ROWS: the reduction runs over the operands' rows instead (32 a stage; a
// tile takes 4 and 8 slabs of columns), transposed on the way out of LDS.
// A direct load writes the 64 lanes' pieces to 1024 consecutive LDS bytes, 16 rows of 64: piece p of row r is kept in slot
// p ^ ((r >> 2) & 3), so that a fragment read of 16 rows touches 16 distinct 16-byte columns.
template <bool K_ROWS>
struct Movers {
    const char *a[2], *b[4];
    // first row of the tile in each operand (K_ROWS: first slab, of n_slabs: what lies behind the last one is never read)
    __device__ __forceinline__ Movers(const Operand &A, int64_t a0, int a_slabs, const Operand &B, int64_t b0, int b_slabs) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lrow = lane >> 2;
        if constexpr (K_ROWS) {
            auto unit = [&](const Operand &o, int64_t s0, int n_slabs, int u) -> const char * {
                const int64_t s = s0 + (u >> 1) < n_slabs ? s0 + (u >> 1) : n_slabs - 1;
                return o.at + s * o.slab + ((u & 1) * 16 + lrow) * 64 + (lane & 3) * 16;
            };
#pragma unroll
            for (int i = 0; i < 2; ++i) a[i] = unit(A, a0, a_slabs, wave + 4 * i);
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = unit(B, b0, b_slabs, wave * 4 + i);
        } else {
            const int piece16 = ((lane & 3) ^ ((lane >> 4) & 3)) * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) a[i] = A.at + (a0 + (wave + 4 * i) * 16 + lrow) * 64 + piece16;
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = B.at + (b0 + (wave * 4 + i) * 16 + lrow) * 64 + piece16;
        }
    }
};

struct Product {
    Operand A, B;
    Pairs pairs;
};

// acc += over stages k0 .. k0 + nk of every part product (nk >= 2)
template <bool K_ROWS>
__device__ __forceinline__ void multiply_tile(const Product &p, const Movers<K_ROWS> &mv, int k0, int nk, char *lds, floatx16 (&acc)[2][4]) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, hf = lane >> 5, l32 = lane & 31;
    const int64_t a_stage = K_ROWS ? 32 * 64 : p.A.slab, b_stage = K_ROWS ? 32 * 64 : p.B.slab;
    const int n_stages = p.pairs.n * nk;
    int q = 0, k = 0;
    int64_t a_off = p.pairs.a[0] + k0 * a_stage, b_off = p.pairs.b[0] + k0 * b_stage;
    auto issue_one = [&](int buf, int i) __attribute__((always_inline)) {
        char *dst = lds + buf * kBufBytes;
        if (i < 2) __builtin_amdgcn_global_load_lds(JITDB_GLOBAL_PTR(mv.a[i] + a_off), JITDB_LDS_PTR(dst + (wave + 4 * i) * 1024), 16, 0, 0);
        else __builtin_amdgcn_global_load_lds(JITDB_GLOBAL_PTR(mv.b[i - 2] + b_off), JITDB_LDS_PTR(dst + (8 + wave * 4 + i - 2) * 1024), 16, 0, 0);
    };
    auto advance = [&]() __attribute__((always_inline)) {
        a_off += a_stage;
        b_off += b_stage;
        if (++k == nk) {
            k = 0;
            q = q + 1 < p.pairs.n ? q + 1 : 0;
            a_off = p.pairs.a[q] + k0 * a_stage;
            b_off = p.pairs.b[q] + k0 * b_stage;
        }
    };
    int a_rd[2], b_rd[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (K_ROWS) {
            const int at = h * 1024 + (hf * 4 + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
            a_rd[h] = wm * 4096 + at;
            b_rd[h] = 8192 + wn * 8192 + at;
        } else {
            const int slot16 = ((2 * h + hf) ^ ((l32 >> 2) & 3)) * 16;
            a_rd[h] = (wm * 64 + l32) * kStageBytes + slot16;
            b_rd[h] = (kTileA + wn * 128 + l32) * kStageBytes + slot16;
        }
    }
    const uint32_t lds_base = (uint32_t)(uintptr_t)JITDB_LDS_PTR(lds);
    struct Frags {
        u32x4 a[2], b[4];
    };
    // The reads are asm, because the compiler would make every LDS read wait for all direct-to-LDS loads in flight; the
    // waits are placed by hand as well.  Tiles of 32 rows lie 2048 bytes apart in either layout.
    auto turned = [&](uint32_t at, auto tile, u32x4 &f) __attribute__((always_inline)) {
        constexpr int I = decltype(tile)::value;
        u32x2 lo, hi;
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(lo) : "v"(at), "n"(I * 2048) : "memory");
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(hi) : "v"(at), "n"(I * 2048 + 512) : "memory");
        f = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
    };
    auto read_group = [&](int buf, int h, Frags &f) __attribute__((always_inline)) {
        const uint32_t aa = lds_base + buf * kBufBytes + a_rd[h], bb = lds_base + buf * kBufBytes + b_rd[h];
        if constexpr (K_ROWS) {
            turned(aa, std::integral_constant<int, 0>(), f.a[0]);
            turned(bb, std::integral_constant<int, 0>(), f.b[0]);
            turned(aa, std::integral_constant<int, 1>(), f.a[1]);
            turned(bb, std::integral_constant<int, 1>(), f.b[1]);
            turned(bb, std::integral_constant<int, 2>(), f.b[2]);
            turned(bb, std::integral_constant<int, 3>(), f.b[3]);
        } else {
            asm volatile("ds_read_b128 %0, %1" : "=v"(f.a[0]) : "v"(aa) : "memory");
            asm volatile("ds_read_b128 %0, %1" : "=v"(f.b[0]) : "v"(bb) : "memory");
            asm volatile("ds_read_b128 %0, %1 offset:2048" : "=v"(f.a[1]) : "v"(aa) : "memory");
            asm volatile("ds_read_b128 %0, %1 offset:2048" : "=v"(f.b[1]) : "v"(bb) : "memory");
            asm volatile("ds_read_b128 %0, %1 offset:4096" : "=v"(f.b[2]) : "v"(bb) : "memory");
            asm volatile("ds_read_b128 %0, %1 offset:6144" : "=v"(f.b[3]) : "v"(bb) : "memory");
        }
    };
    auto reads_done = [&](Frags &f) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f.a[0]), "+v"(f.a[1]), "+v"(f.b[0]), "+v"(f.b[1]), "+v"(f.b[2]), "+v"(f.b[3]));
    };
    auto multiply = [&](const Frags &f) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 8; ++m) mfma_step<bf16_t>(f.a[m / 4], f.b[m % 4], acc[m / 4][m % 4]);
    };
    // the next requests are dealt out between the MFMAs: a burst of them would hold the wave back until the memory pipeline took them
    auto multiply_and_issue = [&](const Frags &f, int buf, bool wanted) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            mfma_step<bf16_t>(f.a[m / 4], f.b[m % 4], acc[m / 4][m % 4]);
            __builtin_amdgcn_sched_barrier(0);
            if (m < 6 && wanted) issue_one(buf, m);
            __builtin_amdgcn_sched_barrier(0);
        }
        advance();
    };
    auto wait_barrier = [&](auto n) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(n)::value) : "memory");
    };
    auto issue = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 6; ++i) issue_one(buf, i);
        advance();
    };
    const std::integral_constant<int, 12> two_left;      // loads of younger stages that may stay in flight
    const std::integral_constant<int, 6> one_left;
    const std::integral_constant<int, 0> none_left;
    Frags P, Q;
    int cur = 0;
    auto next_buf = [&]() __attribute__((always_inline)) { return cur == 2 ? 0 : cur + 1; };
    // On entry P holds the first half of stage g (buffer cur), whose buffer is free for stage g + 3 behind the barrier.
    auto step = [&](int g, auto left) __attribute__((always_inline)) {
        read_group(cur, 1, Q);
        __builtin_amdgcn_sched_barrier(0);
        multiply(P);
        __builtin_amdgcn_sched_barrier(0);
        reads_done(Q);
        wait_barrier(left);
        read_group(next_buf(), 0, P);
        __builtin_amdgcn_sched_barrier(0);
        multiply_and_issue(Q, cur, g + 3 < n_stages);
        __builtin_amdgcn_sched_barrier(0);
        reads_done(P);
        cur = next_buf();
    };
    issue(0);
    issue(1);
    if (n_stages > 2) {
        issue(2);
        wait_barrier(two_left);
    } else {
        wait_barrier(one_left);
    }
    read_group(0, 0, P);
    reads_done(P);
    int g = 0;
    for (; g < n_stages - 2; ++g) step(g, one_left);
    step(g, none_left);
    read_group(cur, 1, Q);
    multiply(P);
    reads_done(Q);
    multiply(Q);
    __builtin_amdgcn_sched_barrier(0);
    wait_barrier(none_left);             // every wave is done with the stage buffers
}

__device__ __forceinline__ void clear_tile(floatx16 (&acc)[2][4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][g][v] = 0.0f;
}

// Blocks are dealt round-robin to the 8 XCDs, each with an L2 of its own: XCD x takes the x-th eighth of the tiles in order.
__device__ __forceinline__ int64_t xcd_order(int64_t total) {
    const int64_t per = (total + 7) / 8, i = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
    return (blockIdx.x >> 3) < per && i < total ? i : -1;
}

// ---- logits: their statistics, or g --------------------------------------------------------------------
struct LogitArgs {
    Product p;                      // A: class weights, B: states
    int nk, n_class_tiles;
    const int32_t *n_rows;
    int row0, max_rows;             // the chunk: rows row0 .. row0 + max_rows of the list
    const float *bias;              // padded with -inf
    float2 *stat;                   // [2 n_class_tiles][max_rows]: maximum, sum of exp(z - maximum) over 64 classes
    const int32_t *label_of;
    const float *lse_of, *w_of;
    Operand g;                      // rows: of the chunk, K = class
    float *db_part;                 // [row tiles of the chunk][classes]
};
__device__ __forceinline__ int chunk_rows(const int32_t *n_rows, int row0, int max_rows) {
    const int left = *n_rows - row0;
    return left < 0 ? 0 : left < max_rows ? left : max_rows;
}
// Bands of eight row tiles, class tiles one after another inside a band: the 64 blocks of an XCD share 8 x 8 tiles in its L2.
__device__ __forceinline__ bool logit_tile(int row_tiles, int class_tiles, int &rt, int &ct) {
    const int64_t i = xcd_order((int64_t)row_tiles * class_tiles);
    if (i < 0) return false;
    const int band = (int)(i / (8 * (int64_t)class_tiles)), rem = (int)(i - (int64_t)band * 8 * class_tiles);
    const int left = row_tiles - band * 8, width = left < 8 ? left : 8;
    ct = rem / width;
    rt = band * 8 + rem % width;
    return true;
}

// PARTS 0: statistics; else g in that many parts.  ACCURATE: expf instead of the hardware's exponential of a rounded product.
template <int PARTS, bool ACCURATE>
__global__ void __launch_bounds__(kT, 2)
logits_kernel(const LogitArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[3 * kBufBytes];
    const int rows = chunk_rows(a.n_rows, a.row0, a.max_rows);
    int rt, ct;
    if (!logit_tile((rows + kTileB - 1) / kTileB, a.n_class_tiles, rt, ct)) return;
    floatx16 acc[2][4];
    clear_tile(acc);
    const Movers<false> mv(a.p.A, (int64_t)ct * kTileA, 0, a.p.B, (int64_t)a.row0 + (int64_t)rt * kTileB, 0);
    multiply_tile<false>(a.p, mv, 0, a.nk, lds, acc);
    auto exp_of = [](float v) { return ACCURATE ? expf(v) : __expf(v); };

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, hf = lane >> 5, l32 = lane & 31;
    const int c0 = ct * kTileA + wm * 64;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 b = *reinterpret_cast<const float4 *>(a.bias + c0 + i * 32 + q * 8 + hf * 4);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                acc[i][g][4 * q] += b.x;
                acc[i][g][4 * q + 1] += b.y;
                acc[i][g][4 * q + 2] += b.z;
                acc[i][g][4 * q + 3] += b.w;
            }
        }
    if constexpr (PARTS == 0) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int r = rt * kTileB + wn * 128 + g * 32 + l32;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) top = fmaxf(top, acc[i][g][v]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float from = top == -INFINITY ? 0.0f : top;       // every class masked: the sum is 0, not NaN
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) s += exp_of(acc[i][g][v] - from);
            s += __shfl_xor(s, 32);
            if (hf == 0 && r < a.max_rows) a.stat[(int64_t)(2 * ct + wm) * a.max_rows + r] = make_float2(top, s);
        }
    } else {
        float sums[2][16];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) sums[i][v] = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int r = rt * kTileB + wn * 128 + g * 32 + l32;
            const bool in = r < rows;
            const float lse = in ? a.lse_of[a.row0 + r] : 0.0f, w = in ? a.w_of[a.row0 + r] : 0.0f;
            const int label = (in ? a.label_of[a.row0 + r] : -1) - c0 - hf * 4;     // in the order of this lane's classes
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    bf16_t part[PARTS][4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int v = 4 * q + e;
                        float d = exp_of(acc[i][g][v] - lse);
                        if (label == i * 32 + q * 8 + e) d -= 1.0f;
                        d = in ? d * w : 0.0f;
                        sums[i][v] += d;
                        bf16_t one[PARTS];
                        split_parts<PARTS>(d, one);
#pragma unroll
                        for (int k = 0; k < PARTS; ++k) part[k][e] = one[k];
                    }
#pragma unroll
                    for (int k = 0; k < PARTS; ++k)
                        __builtin_memcpy(a.g.at + k * a.g.part + (int64_t)(c0 / 32 + i) * a.g.slab + (int64_t)r * 64 + q * 16 + hf * 8, part[k], 8);
                }
        }
        // sums over the wave's 128 rows, then over the two waves that share the classes
        float *red = reinterpret_cast<float *>(lds);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                float s = sums[i][v];
#pragma unroll
                for (int m = 1; m < 32; m <<= 1) s += __shfl_xor(s, m);
                if (l32 == 0) red[wn * 128 + wm * 64 + i * 32 + (v >> 2) * 8 + hf * 4 + (v & 3)] = s;
            }
        __syncthreads();
        if (threadIdx.x < kTileA)
            a.db_part[((int64_t)rt * a.n_class_tiles + ct) * kTileA + threadIdx.x] = red[threadIdx.x] + red[kTileA + threadIdx.x];
    }
}

// z of the label itself, in fp32: a wave a row
template <typename T>
__global__ void __launch_bounds__(kT)
label_logit_kernel(const T *__restrict__ h, const T *__restrict__ V, const float *__restrict__ b, const int32_t *__restrict__ n_rows,
                   const int32_t *__restrict__ row_of, const int32_t *__restrict__ label_of, int H, float *__restrict__ out) {
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < *n_rows; r += (int64_t)gridDim.x * 4) {
        const int c = label_of[r];
        float s = 0.0f;
        if (c >= 0) {
            const T *x = h + (int64_t)row_of[r] * H, *v = V + (int64_t)c * H;
            for (int k = lane; k < H; k += 64) s = fmaf(to_f32<T>(x[k]), to_f32<T>(v[k]), s);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
        if (lane == 0) out[r] = c >= 0 ? s + (b ? b[c] : 0.0f) : __builtin_nanf("");
    }
}

// 64 rows a block; wave w takes every fourth set of statistics, then the four are put together.  The sets are `n_stat` of max_rows
// rows, or, class_tiles > 0, those that resident_logits_kernel left.
__global__ void __launch_bounds__(kT)
join_kernel(const float2 *__restrict__ stat, int n_stat, int class_tiles, int row0, int max_rows, const int32_t *__restrict__ n_rows,
            const int32_t *__restrict__ row_of, const float *__restrict__ label_z, float *__restrict__ loss, float *__restrict__ lse) {
    __shared__ float2 red[4][64];
    const int rows = chunk_rows(n_rows, row0, max_rows);
    if ((int)blockIdx.x * 64 >= rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.x * 64 + lane;
    int64_t stride = max_rows;
    if (class_tiles > 0) {
        const int blocks = (rows + kResRows - 1) / kResRows;
        n_stat = res_splits(blocks, class_tiles, kResPlaces);
        stride = (int64_t)blocks * kResRows;
    }
    float top = -INFINITY, s = 0.0f;
    auto add = [&](float2 p) {
        if (p.y == 0.0f) return;                     // nothing but masked classes
        const float m = fmaxf(top, p.x);
        s = s * expf(top - m) + p.y * expf(p.x - m);
        top = m;
    };
    if (r < rows)
#pragma unroll 4
        for (int k = wave; k < n_stat; k += 4) add(stat[k * stride + r]);
    red[wave][lane] = make_float2(top, s);
    __syncthreads();
    if (wave || r >= rows) return;
    for (int w = 1; w < 4; ++w) add(red[w][lane]);
    const float v = top + logf(s);
    const int64_t at = row_of[row0 + r];
    lse[at] = v;
    loss[at] = v - label_z[row0 + r];
}

// ---- the two products with g ---------------------------------------------------------------------------
// dh: A = turned class weights (features), B = g (rows), K = classes.  dV: A = g (classes), B = states (features), K = rows.
// Tiles are left in register order, one per range of K; the ranges are as many as fill the chip with the rows there are.
struct GradArgs {
    Product p;
    int a_tiles, a_slabs, b_slabs;
    const int32_t *n_rows;
    int row0, max_rows;
    int class_stages;               // K of dh in stages
    int tiles_most;                 // dV: its tiles
    float *part;
    // results
    const int32_t *row_of;
    int H, C;
    void *out;
    float *acc;                     // dV over several chunks of rows
    int first, last;
};
constexpr int kMinStages = 8;       // a range of K is no shorter
template <bool WEIGHTS>
__device__ __forceinline__ void grad_shape(const GradArgs &a, int rows, int &tiles, int &stages, int &splits, int &per) {
    tiles = WEIGHTS ? a.tiles_most : a.a_tiles * ((rows + kTileB - 1) / kTileB);
    stages = WEIGHTS ? (rows + 63) / 64 * 2 : a.class_stages;
    splits = 0;
    per = 0;
    if (tiles == 0 || stages == 0) return;
    const int want = kSlots / tiles, most = stages / kMinStages;
    splits = want < most ? want : most;
    if (splits < 1) splits = 1;
    per = ((stages + splits - 1) / splits + 1) & ~1;
    splits = (stages + per - 1) / per;
}
template <bool WEIGHTS>
__global__ void __launch_bounds__(kT, 2)
grad_product_kernel(const GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[3 * kBufBytes];
    const int rows = chunk_rows(a.n_rows, a.row0, a.max_rows);
    int tiles, stages, splits, per;
    grad_shape<WEIGHTS>(a, rows, tiles, stages, splits, per);
    const int64_t i = xcd_order((int64_t)tiles * splits);
    if (i < 0) return;
    const int split = (int)(i / tiles), tile = (int)(i - (int64_t)split * tiles);
    const int k0 = split * per, nk = k0 + per < stages ? per : stages - k0;
    floatx16 acc[2][4];
    clear_tile(acc);
    if constexpr (WEIGHTS) {        // neighbours share the classes' g
        const int n_bt = a.tiles_most / a.a_tiles, at = tile / n_bt, bt = tile % n_bt;
        const Movers<true> mv(a.p.A, at * 4, a.a_slabs, a.p.B, bt * 8, a.b_slabs);
        multiply_tile<true>(a.p, mv, k0, nk, lds, acc);
    } else {                        // neighbours share the rows' g
        const int bt = tile / a.a_tiles, at = tile % a.a_tiles;
        const Movers<false> mv(a.p.A, (int64_t)at * kTileA, 0, a.p.B, (int64_t)bt * kTileB, 0);
        multiply_tile<false>(a.p, mv, k0, nk, lds, acc);
    }
    float4 *out = reinterpret_cast<float4 *>(a.part + i * (kTileA * kTileB)) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                out[((i * 4 + g) * 4 + v) * kT] = make_float4(acc[i][g][4 * v], acc[i][g][4 * v + 1], acc[i][g][4 * v + 2], acc[i][g][4 * v + 3]);
}
// Sixteen blocks a tile: the ranges of K in order, then the place of the value.
template <bool WEIGHTS, typename O>
__global__ void __launch_bounds__(kT)
grad_finish_kernel(const GradArgs a) {
    const int rows = chunk_rows(a.n_rows, a.row0, a.max_rows);
    int tiles, stages, splits, per;
    grad_shape<WEIGHTS>(a, rows, tiles, stages, splits, per);
    const int tile = blockIdx.x >> 5, rest = blockIdx.x & 31, t = threadIdx.x;
    if (tile >= tiles) return;
    const int lane = t & 63, wave = t >> 6, i = rest >> 4, g = (rest >> 2) & 3, v = rest & 3;
    const int n_bt = WEIGHTS ? a.tiles_most / a.a_tiles : 1;
    const int at = WEIGHTS ? tile / n_bt : tile % a.a_tiles, bt = WEIGHTS ? tile % n_bt : tile / a.a_tiles;
    const int m = at * kTileA + (wave >> 1) * 64 + i * 32 + v * 8 + (lane >> 5) * 4;      // first of four rows of A
    const int n = bt * kTileB + (wave & 1) * 128 + g * 32 + (lane & 31);                  // row of B
    if (WEIGHTS ? m >= a.C || n >= a.H : m >= a.H || n >= rows) return;
    const float4 *in = reinterpret_cast<const float4 *>(a.part + (int64_t)tile * (kTileA * kTileB)) + rest * kT + t;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
        const float4 p = in[(int64_t)k * tiles * (kTileA * kTileB / 4)];
        s[0] += p.x; s[1] += p.y; s[2] += p.z; s[3] += p.w;
    }
    if constexpr (WEIGHTS) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (m + e >= a.C) break;
            const int64_t q = (int64_t)(m + e) * a.H + n;
            if (!a.first) s[e] += a.acc[q];
            if (a.last) static_cast<O *>(a.out)[q] = from_f32<O>(s[e]);
            else a.acc[q] = s[e];
        }
    } else {
        O *o = static_cast<O *>(a.out) + (int64_t)a.row_of[a.row0 + n] * a.H + m;
        O e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = from_f32<O>(s[k]);
        if (m + 4 <= a.H) {
            __builtin_memcpy(o, e, sizeof(e));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (m + k < a.H) o[k] = e[k];
        }
    }
}
// 64 classes a block; sixteen waves take every sixteenth of the sums that `per` of each 256 rows left, in order
__global__ void __launch_bounds__(1024)
bias_grad_kernel(const float *__restrict__ part, int n_classes_pad, int per, int C, const int32_t *__restrict__ n_rows, int row0, int max_rows,
                 int first, float *__restrict__ db) {
    __shared__ float sums[16][64];
    const int tiles = (chunk_rows(n_rows, row0, max_rows) + kTileB - 1) / kTileB * per;
    const int l = threadIdx.x & 63, q = threadIdx.x >> 6, c = blockIdx.x * 64 + l;
    float s = 0.0f;
    if (c < C)
#pragma unroll 4
        for (int p = q; p < tiles; p += 16) s += part[(int64_t)p * n_classes_pad + c];
    sums[q][l] = s;
    __syncthreads();
    if (q || c >= C) return;
    for (int k = 1; k < 16; ++k) s += sums[k][l];
    db[c] = first ? s : db[c] + s;
}
// rows without a label have no gradient
template <typename O>
__global__ void __launch_bounds__(kT)
clear_rows_kernel(const int32_t *__restrict__ label, int64_t n, int H, O *__restrict__ dh) {
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < n; r += (int64_t)gridDim.x * 4)
        if (label[r] == -1)
            for (int k = lane; k < H; k += 64) dh[r * H + k] = O(0);
}
template <typename O>
__global__ void __launch_bounds__(kT)
clear_kernel(O *__restrict__ p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * kT + threadIdx.x; i < n; i += (int64_t)gridDim.x * kT) p[i] = O(0);
}

// ---- sizes and workspaces ------------------------------------------------------------------------------
struct Sizes {
    int64_t n, n_pad;          // rows at most, and rounded up to whole tiles
    int H, C, Hk, Hf, Cp;      // widths: of K (states), of the turned weights' rows, classes in whole tiles
    int parts, g_parts;        // of the operands, of g
    int label_blocks;
    int res, class_tiles;      // resident_logits_kernel: K in steps of 16 (0: not for this width), tiles of 32 classes (an even number)
    int stat_rows, grad_rows;  // rows of a chunk
};
bool known(jitdb_dtype t) { return t == JITDB_F32 || t == JITDB_BF16; }
// K in steps of 16 of the variant of resident_logits_kernel for this width: the states of 64 rows in up to 256 registers
int res_steps(int H, jitdb_dtype dtype) {
    if (dtype == JITDB_F32) return H <= 64 ? 4 : H <= 128 ? 8 : H <= 160 ? 10 : 0;
    return H <= 128 ? 8 : H <= 256 ? 16 : H <= 384 ? 24 : H <= 512 ? 32 : 0;
}
bool make_sizes(int64_t n, int32_t H, int32_t C, jitdb_dtype dtype, jitdb_dtype grad, Sizes &s) {
    if (n < 0 || n > JITDB_MAX_NODES || H < 1 || H > kMaxWidth || C < 1 || C > kMaxClasses || !known(dtype) || !known(grad)) return false;
    if (dtype == JITDB_F32 && grad == JITDB_BF16) return false;       // gradients are not rounded below their operands
    s.n = n; s.H = H; s.C = C;
    s.n_pad = round_up(n > 0 ? n : 1, kTileB);
    s.res = res_steps(H, dtype);
    s.class_tiles = (int)round_up(C, 64) / kResClasses;
    s.Hk = s.res ? s.res * 16 : (int)round_up(H, 64);
    s.Hf = (int)round_up(H, kTileA);
    s.Cp = (int)round_up(C, kTileA);
    s.parts = dtype == JITDB_F32 ? 3 : 1;
    s.g_parts = grad == JITDB_F32 ? 3 : 1;
    s.label_blocks = (int)ceil_div(n > 0 ? n : 1, kLabelBlock);
    auto chunk = [&](int64_t bytes_a_row, int64_t budget) {
        const int64_t rows = budget / bytes_a_row / kTileB * kTileB;
        return (int)(rows < kTileB ? kTileB : rows < s.n_pad ? rows : s.n_pad);
    };
    s.stat_rows = s.res ? (int)s.n_pad : chunk((int64_t)s.Cp / 64 * 8, kStatBytes);
    s.grad_rows = chunk((int64_t)s.Cp * 2 * s.g_parts, kGradBytes);
    return true;
}
// most tiles x ranges of a product with `tiles` tiles at most and `stages` stages at most (grad_shape, whatever the rows)
int64_t grad_parts(int64_t tiles, int64_t stages) {
    const int64_t ranges = stages / kMinStages > 1 ? stages / kMinStages : 1;
    const int64_t filled = tiles * ranges < kSlots ? tiles * ranges : kSlots;
    return tiles > filled ? tiles : filled;
}
// most blocks of resident_logits_kernel, whatever the rows (res_splits)
int64_t res_blocks(int64_t rows, int class_tiles) {
    const int64_t rb = ceil_div(rows, kResRows), ranges = class_tiles / kResMinTiles > 1 ? class_tiles / kResMinTiles : 1;
    const int64_t most = rb > kResBlocks ? rb : kResBlocks;
    return rb * ranges < most ? rb * ranges : most;
}
struct Space {
    int32_t *counts, *n_rows, *row_of, *label_of;
    float *lse_of, *w_of, *label_z, *bias, *db_part, *part_h, *part_v, *acc_v;
    float2 *stat;
    Operand h, v, vt, g;
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
    w.label_of = c.take<int32_t>(s.n_pad);
    w.bias = c.take<float>(s.Cp + 64);
    w.h = take_operand(c, s.parts, s.Hk / 32, s.n_pad);
    w.v = take_operand(c, s.parts, s.Hk / 32, s.Cp);
    if (!backward) {
        w.label_z = c.take<float>(s.n_pad);
        w.stat = c.take<float2>(s.res ? (size_t)res_blocks(s.n_pad, s.class_tiles) * kResRows : (size_t)(s.Cp / 64) * s.stat_rows);
    } else {
        w.lse_of = c.take<float>(s.n_pad);
        w.w_of = c.take<float>(s.n_pad);
        w.vt = take_operand(c, s.parts, s.Cp / 32, s.Hf);
        w.g = take_operand(c, s.g_parts, s.Cp / 32, s.grad_rows);
        w.db_part = c.take<float>((size_t)(s.grad_rows / kTileB) * (s.res ? 4 : 1) * s.Cp);
        w.part_h = c.take<float>((size_t)(grad_parts((int64_t)s.Hf / kTileA * (s.grad_rows / kTileB), s.Cp / 32) * kTileA * kTileB));
        w.part_v = c.take<float>((size_t)(grad_parts((int64_t)s.Cp / kTileA * ceil_div(s.H, kTileB), s.grad_rows / 32) * kTileA * kTileB));
        if (s.grad_rows < s.n) w.acc_v = c.take<float>((size_t)s.C * s.H);
    }
    w.bytes = c.off;
    return w;
}

unsigned grid_of(int64_t work) {        // grid of a kernel that loops: enough blocks to fill the chip
    const int64_t b = ceil_div(work, kT);
    return (unsigned)(b < 1 ? 1 : b < 4096 ? b : 4096);
}
unsigned tile_grid(int64_t tiles) { return (unsigned)(8 * ceil_div(tiles, 8)); }

template <typename T>
int prepare(const T *h, const T *V, const float *b, const RowList &list, const Sizes &s, const Space &w, hipStream_t st) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    label_count_kernel<<<s.label_blocks, kT, 0, st>>>(list);
    JITDB_LAUNCH_CHECK();
    label_rows_kernel<<<s.label_blocks, kT, 0, st>>>(list);
    JITDB_LAUNCH_CHECK();
    pack_rows_kernel<T, PARTS><<<grid_of(s.n_pad * (s.Hk / 8)), kT, 0, st>>>(h, w.row_of, w.n_rows, 0, s.H, s.Hk / 32, kTileB, w.h);
    JITDB_LAUNCH_CHECK();
    pack_rows_kernel<T, PARTS><<<grid_of((int64_t)s.Cp * (s.Hk / 8)), kT, 0, st>>>(V, nullptr, nullptr, s.C, s.H, s.Hk / 32, kTileA, w.v);
    JITDB_LAUNCH_CHECK();
    pad_bias_kernel<<<grid_of(s.Cp + 64), kT, 0, st>>>(b, s.C, s.Cp + 64, w.bias);
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}
LogitArgs logit_args(const Sizes &s, const Space &w) {
    LogitArgs a = {};
    a.p.A = w.v; a.p.B = w.h; a.p.pairs = make_pairs(w.v, s.parts, w.h, s.parts);
    a.nk = s.Hk / 32; a.n_class_tiles = s.Cp / kTileA;
    a.n_rows = w.n_rows; a.bias = w.bias;
    return a;
}

ResArgs res_args(const Sizes &s, const Space &w) {
    ResArgs a = {};
    a.V = w.v.at; a.v_slab = w.v.slab; a.h = w.h.at; a.h_slab = w.h.slab;
    a.bias = w.bias; a.class_tiles = s.class_tiles; a.n_rows = w.n_rows;
    a.label_of = w.label_of; a.lse_of = w.lse_of; a.w_of = w.w_of;
    a.g = w.g.at; a.g_slab = w.g.slab; a.g_part = w.g.part; a.db_part = w.db_part;
    return a;
}
template <typename T, int G>
int launch_resident(int steps, int64_t rows, const ResArgs &a, hipStream_t st) {
    const unsigned grid = tile_grid(res_blocks(rows, a.class_tiles));
    if constexpr (sizeof(T) == 4) {
        if (steps == 4) resident_logits_kernel<3, 4, G><<<grid, kResT, 0, st>>>(a);
        else if (steps == 8) resident_logits_kernel<3, 8, G><<<grid, kResT, 0, st>>>(a);
        else resident_logits_kernel<3, 10, G><<<grid, kResT, 0, st>>>(a);
    } else {
        if (steps == 8) resident_logits_kernel<1, 8, G><<<grid, kResT, 0, st>>>(a);
        else if (steps == 16) resident_logits_kernel<1, 16, G><<<grid, kResT, 0, st>>>(a);
        else if (steps == 24) resident_logits_kernel<1, 24, G><<<grid, kResT, 0, st>>>(a);
        else resident_logits_kernel<1, 32, G><<<grid, kResT, 0, st>>>(a);
    }
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}

template <typename T>
int run_forward_xent(const T *h, const T *V, const float *b, const RowList &list, const Sizes &s, const Space &w,
                     float *loss, float *lse, hipStream_t st) {
    int rc = prepare<T>(h, V, b, list, s, w, st);
    if (rc != JITDB_OK) return rc;
    const int64_t label_blocks = ceil_div(s.n, 4);
    label_logit_kernel<T><<<(unsigned)(label_blocks < 8192 ? label_blocks : 8192), kT, 0, st>>>(h, V, b, w.n_rows, w.row_of, w.label_of, s.H, w.label_z);
    JITDB_LAUNCH_CHECK();
    if (s.res) {
        ResArgs a = res_args(s, w);
        a.stat = w.stat;
        a.max_rows = (int)s.n_pad;
        if ((rc = launch_resident<T, 0>(s.res, s.n, a, st)) != JITDB_OK) return rc;
        join_kernel<<<(unsigned)ceil_div(s.n, 64), kT, 0, st>>>(w.stat, 0, s.class_tiles, 0, a.max_rows, w.n_rows, w.row_of, w.label_z, loss, lse);
        JITDB_LAUNCH_CHECK();
        return JITDB_OK;
    }
    LogitArgs a = logit_args(s, w);
    a.stat = w.stat;
    a.max_rows = s.stat_rows;
    for (int64_t r0 = 0; r0 < s.n; r0 += s.stat_rows) {
        a.row0 = (int)r0;
        const int64_t rows = s.n - r0 < s.stat_rows ? s.n - r0 : s.stat_rows;
        logits_kernel<0, sizeof(T) == 4><<<tile_grid(ceil_div(rows, kTileB) * a.n_class_tiles), kT, 0, st>>>(a);
        JITDB_LAUNCH_CHECK();
        join_kernel<<<(unsigned)ceil_div(rows, 64), kT, 0, st>>>(w.stat, 2 * a.n_class_tiles, 0, a.row0, a.max_rows, w.n_rows, w.row_of, w.label_z, loss, lse);
        JITDB_LAUNCH_CHECK();
    }
    return JITDB_OK;
}

template <typename T, typename O>
int run_backward_xent(const T *h, const T *V, const float *b, const RowList &list, const Sizes &s, const Space &w,
                      O *dh, O *dV, float *db, hipStream_t st) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, G_PARTS = sizeof(O) == 4 ? 3 : 1;
    int rc = prepare<T>(h, V, b, list, s, w, st);
    if (rc != JITDB_OK) return rc;
    pack_turned_kernel<T, PARTS><<<dim3((unsigned)(s.Cp / 32), (unsigned)ceil_div(s.Hf, 64)), kT, 0, st>>>(V, s.C, s.H, s.Hf, w.vt);
    JITDB_LAUNCH_CHECK();
    const int64_t clear_blocks = ceil_div(s.n, 4);
    clear_rows_kernel<O><<<(unsigned)(clear_blocks < 4096 ? clear_blocks : 4096), kT, 0, st>>>(list.label, s.n, s.H, dh);
    JITDB_LAUNCH_CHECK();
    LogitArgs a = logit_args(s, w);
    a.label_of = w.label_of; a.lse_of = w.lse_of; a.w_of = w.w_of; a.g = w.g; a.db_part = w.db_part;
    a.max_rows = s.grad_rows;
    ResArgs ra = res_args(s, w);
    ra.max_rows = s.grad_rows;
    GradArgs gh = {}, gv = {};
    gh.p.A = w.vt; gh.p.B = w.g; gh.p.pairs = make_pairs(w.vt, s.parts, w.g, s.g_parts);
    gh.a_tiles = s.Hf / kTileA; gh.class_stages = s.class_tiles; gh.part = w.part_h; gh.out = dh; gh.row_of = w.row_of;
    gv.p.A = w.g; gv.p.B = w.h; gv.p.pairs = make_pairs(w.g, s.g_parts, w.h, s.parts);
    gv.a_tiles = s.Cp / kTileA; gv.a_slabs = s.class_tiles; gv.b_slabs = s.Hk / 32;
    gv.tiles_most = gv.a_tiles * (int)ceil_div(s.H, kTileB); gv.part = w.part_v; gv.out = dV; gv.acc = w.acc_v;
    for (GradArgs *g : {&gh, &gv}) { g->n_rows = w.n_rows; g->max_rows = s.grad_rows; g->H = s.H; g->C = s.C; }
    for (int64_t r0 = 0; r0 < s.n; r0 += s.grad_rows) {
        const int64_t rows = s.n - r0 < s.grad_rows ? s.n - r0 : s.grad_rows, row_tiles = ceil_div(rows, kTileB);
        a.row0 = gh.row0 = gv.row0 = (int)r0;
        gv.first = r0 == 0; gv.last = r0 + s.grad_rows >= s.n;
        if (s.res) {
            ra.row0 = (int)r0;
            ra.h = w.h.at + r0 * 64;
            if ((rc = launch_resident<T, G_PARTS>(s.res, rows, ra, st)) != JITDB_OK) return rc;
        } else {
            logits_kernel<G_PARTS, sizeof(T) == 4><<<tile_grid(row_tiles * a.n_class_tiles), kT, 0, st>>>(a);
            JITDB_LAUNCH_CHECK();
        }
        bias_grad_kernel<<<(unsigned)ceil_div(s.C, 64), 1024, 0, st>>>(w.db_part, s.res ? s.class_tiles * kResClasses : s.Cp, s.res ? 4 : 1, s.C, w.n_rows, a.row0, a.max_rows, gv.first, db);
        JITDB_LAUNCH_CHECK();
        const int64_t h_tiles = gh.a_tiles * row_tiles;
        gv.p.B.at = w.h.at + r0 * 64;
        grad_product_kernel<false><<<tile_grid(grad_parts(h_tiles, gh.class_stages)), kT, 0, st>>>(gh);
        JITDB_LAUNCH_CHECK();
        grad_finish_kernel<false, O><<<(unsigned)(h_tiles * 32), kT, 0, st>>>(gh);
        JITDB_LAUNCH_CHECK();
        grad_product_kernel<true><<<tile_grid(grad_parts(gv.tiles_most, row_tiles * (kTileB / 32))), kT, 0, st>>>(gv);
        JITDB_LAUNCH_CHECK();
        grad_finish_kernel<true, O><<<(unsigned)gv.tiles_most * 32u, kT, 0, st>>>(gv);
        JITDB_LAUNCH_CHECK();
    }
    return JITDB_OK;
}

// ---- few classes ---------------------------------------------------------------------------------------
// Is there a variant for these sizes?
bool few_fits(int H, int C, jitdb_dtype dtype) {
    auto any = [](auto, auto) {};
    return dtype == JITDB_F32 ? for_few<float>(H, C, any) : for_few<bf16_t>(H, C, any);
}
int few_blocks(int64_t n) {              // of the backward pass: each leaves a set of sums
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
int run_few_backward(const FewArgs &a, O *dV, float *db, hipStream_t st) {
    const int blocks = few_blocks(a.n);
    for_few<T>(a.H, a.C, [&](auto c, auto nb) { few_backward_kernel<T, O, decltype(c)::value, decltype(nb)::value><<<blocks, kFewT, 0, st>>>(a); });
    JITDB_LAUNCH_CHECK();
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
    list.n_rows = w.n_rows; list.row_of = w.row_of; list.label_of = w.label_of; list.lse_of = w.lse_of; list.w_of = w.w_of;
    if (dtype == JITDB_F32)
        return run_backward_xent<float, float>(static_cast<const float *>(h), static_cast<const float *>(V), b, list, s, w,
                                               static_cast<float *>(dh), static_cast<float *>(dV), db, st);
    if (grad_dtype == JITDB_F32)
        return run_backward_xent<bf16_t, float>(static_cast<const bf16_t *>(h), static_cast<const bf16_t *>(V), b, list, s, w,
                                                static_cast<float *>(dh), static_cast<float *>(dV), db, st);
    return run_backward_xent<bf16_t, bf16_t>(static_cast<const bf16_t *>(h), static_cast<const bf16_t *>(V), b, list, s, w,
                                             static_cast<bf16_t *>(dh), static_cast<bf16_t *>(dV), db, st);
}
