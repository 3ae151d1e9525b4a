// What stands on either side of the node states in a training step, one pass over memory each: layer norm with its backward
// pass, and dropout from a counter-based generator.
//
// Layer norm of a row x of H values:  mean = sum x / H,  rstd = 1 / sqrt(sum (x - mean)^2 / H + eps),
//     xhat = (x - mean) rstd,  y = D(xhat gamma + beta)            D: dropout, where asked for
// and for a cotangent gy of y, with g = D(gy) and a = g gamma:
//     dx = rstd (a - sum a / H - xhat sum (a xhat) / H),  dgamma = sum over rows of g xhat,  dbeta = sum over rows of g.
// A row stays in the registers of the lanes that share it (16 to 64 of a wave, or a block of 512 for long rows) between its sums and
// its result, so x is read once and the variance is that of the centred values; everything is fp32.  A mean m0 from a sum in fp32 is
// off by more than a rounding, which rows far from zero show (30000.1 in every column: by 0.002, and y would be 0.5 instead of beta):
// what is left of it is the mean of x - m0, summed beside the squares, and comes off both,
//     c = sum (x - m0) / H,  mean = m0 + c,  sum (x - mean)^2 = sum (x - m0)^2 - c sum (x - m0).
//
// Dropout keeps element i of a call (rows one after another) where half i % 2 (low half first) of the 64-bit word
//     mix64(mix64(seed) + (first + i / 2) golden)                  (SplitMix64 with a mixed key; seed, first: state[0], state[1])
// is at least p 2^32.  The mask is a function of i: the backward pass computes it again and nothing is stored.
//
// All kernels are bound by memory (copies reach 4.5 to 5.4 TB/s, by their shape).  1.18 M rows of 512, bf16: forward 510 us (4.7 TB/s), with
// dropout 591, backward 1068 (4.5 TB/s; fp32 dx out); dropout of 1.18 M x 300 bf16 258 us (5.5 TB/s).

#include "common.h"

#include <type_traits>

namespace jitdb {
namespace {

constexpr int kT = 256;
constexpr int kWide = 512;               // threads that share a row of more than kWaveMax values: the variant of kMaxWidth, whatever its length
constexpr int kWaveMax = 2048;           // (fp32 forward and backward: 120000 x 2048 350 and 568 us, 100000 x 2049 1226 and 2491, 16000 x 16384 490 and 708)
constexpr int kMaxWidth = 1 << 14;
constexpr int kForwardBlocks = 8192;     // of the forward pass (2048 take 10 to 15 % longer on a million rows)
constexpr int kMaxParts = 1024;          // partial sums of the weight gradients: blocks of the backward pass
constexpr float kFar = 16.0f;            // |mean| / spread up to which the rounding of a mean (2^-20 of the spread) stays in the backward pass
constexpr int kChain = 16, kWideChain = 32;       // rows whose terms are added in a row

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Drop {
    const uint64_t *state;               // nullptr: nothing is dropped
    uint32_t limit, all;                 // a half below limit is dropped; all: every one is
    float scale;
};
// p is in [0, 1]: p 2^32 fits 33 bits, and 2^32 itself (p = 1) is told apart by `all`
Drop make_drop(float p, const uint64_t *state) {
    Drop d = {};
    const double limit = (double)p * 4294967296.0;
    d.state = state;
    d.all = limit >= 4294967296.0;
    d.limit = d.all ? 0xFFFFFFFFu : (uint32_t)limit;
    d.scale = d.all ? 0.0f : 1.0f / (1.0f - p);
    return d;
}
__device__ __forceinline__ uint64_t drop_start(const Drop &d) { return mix64(d.state[0]) + d.state[1] * kGolden; }

// v[k] = value k of elements at .. at + N of the stream, scaled, or 0 where dropped (whatever it was)
template <int N>
__device__ __forceinline__ void apply_drop(const Drop &d, uint64_t start, uint64_t at, float (&v)[N]) {
    uint32_t u[N + 2];
    const uint64_t w = start + (at >> 1) * kGolden;
#pragma unroll
    for (int j = 0; j < (N + 1) / 2; ++j) {
        const uint64_t z = mix64(w + j * kGolden);
        u[2 * j] = (uint32_t)z;
        u[2 * j + 1] = (uint32_t)(z >> 32);
    }
    if (at & 1) {
        const uint64_t z = mix64(w + (N / 2) * kGolden);
        u[N / 2 * 2] = (uint32_t)z;
        u[N / 2 * 2 + 1] = (uint32_t)(z >> 32);
#pragma unroll
        for (int k = 0; k < N; ++k) u[k] = u[k + 1];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = u[k] >= d.limit && !d.all ? v[k] * d.scale : 0.0f;
}

// Sixteen bytes of a row, from any element boundary; only the first `left` elements exist.  Loads stay packed until they are used,
// so that several are on their way; what is written is not read again soon and goes past the caches.
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);
typedef u32x4 __attribute__((aligned(2))) any4;
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T *p, int left) {
    constexpr int N = kVec<T>;
    u32x4 w = {0u, 0u, 0u, 0u};
    if (left >= N) {
        __builtin_memcpy(&w, p, 16);
    } else {
        T e[N];
#pragma unroll
        for (int k = 0; k < N; ++k) e[k] = k < left ? p[k] : T(0);
        __builtin_memcpy(&w, e, 16);
    }
    return w;
}
template <typename E, int N> struct Piece { uint32_t w[N * (int)sizeof(E) / 4]; };
template <typename E, int N>
__device__ __forceinline__ Piece<E, N> load_row(const E *p, int left) {
    Piece<E, N> r = {};
    if (left >= N) {
        __builtin_memcpy(&r, p, sizeof(r));
    } else {
        E e[N];
#pragma unroll
        for (int k = 0; k < N; ++k) e[k] = k < left ? p[k] : E(0);
        __builtin_memcpy(&r, e, sizeof(r));
    }
    return r;
}
template <typename E, int N>
__device__ __forceinline__ void unpack(const Piece<E, N> &r, float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if constexpr (sizeof(E) == 4) v[k] = __uint_as_float(r.w[k]);
        else v[k] = __uint_as_float(k & 1 ? r.w[k >> 1] & 0xFFFF0000u : r.w[k >> 1] << 16);
    }
}
template <typename T>
__device__ __forceinline__ float element(const u32x4 &w, int k) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
    else return __uint_as_float(k & 1 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16);
}
template <typename T, int N>
__device__ __forceinline__ void store_row_piece(T *p, int left, const float (&v)[N]) {
    T e[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if constexpr (sizeof(T) == 4) e[k] = v[k];
        else e[k] = __builtin_bit_cast(bf16_t, (__bf16)v[k]);          // (the hardware's rounding, two a instruction)
    }
    if (left >= N) {
        if constexpr (N == kVec<T>) {
            u32x4 w;
            __builtin_memcpy(&w, e, 16);
            __builtin_nontemporal_store(w, reinterpret_cast<any4 *>(p));
        } else {                         // (in two halves or quarters: the caches make whole lines of them; past them, dx takes 16 % longer)
            __builtin_memcpy(p, e, sizeof(e));
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < left) p[k] = e[k];
    }
}

// ---- dropout ---------------------------------------------------------------------------------
// Four pieces a thread and turn.
template <typename T>
__global__ void __launch_bounds__(kT)
dropout_kernel(const T *x, int64_t n, const Drop d, T *y) {
    constexpr int V = kVec<T>, TURN = 4;
    const uint64_t start = drop_start(d);
    const int64_t step = (int64_t)gridDim.x * kT * V * TURN;
    for (int64_t i0 = ((int64_t)blockIdx.x * kT * TURN + threadIdx.x) * V; i0 < n; i0 += step) {
        u32x4 w[TURN];
#pragma unroll
        for (int u = 0; u < TURN; ++u) {
            const int64_t i = i0 + (int64_t)u * kT * V;
            w[u] = load_piece<T>(x + i, n - i >= V ? V : n > i ? (int)(n - i) : 0);
        }
#pragma unroll
        for (int u = 0; u < TURN; ++u) {
            const int64_t i = i0 + (int64_t)u * kT * V;
            if (i >= n) break;
            float v[V];
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = element<T>(w[u], k);
            apply_drop<V>(d, start, (uint64_t)i, v);
            store_row_piece<T, V>(y + i, n - i < V ? (int)(n - i) : V, v);
        }
    }
}

// ---- sums over the lanes that share a row ------------------------------------------------------
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int m = 1; m < G; m <<= 1) v += __shfl_xor(v, m);
    return v;
}
// G <= 64: lanes of a wave.  G = kWide: the block; `red` holds one float per wave, and two sums in a row need two of them.
template <int G>
__device__ __forceinline__ float row_sum(float v, float *red) {
    if constexpr (G <= 64) {
        return lanes_sum<G>(v);
    } else {
        v = lanes_sum<64>(v);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < G / 64; ++w) s += red[w];
        return s;
    }
}

// two at once; `red` holds two floats per wave
template <int G>
__device__ __forceinline__ void row_sums(float &v, float &w, float *red) {
    v = lanes_sum<(G <= 64 ? G : 64)>(v);
    w = lanes_sum<(G <= 64 ? G : 64)>(w);
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) {
            red[threadIdx.x >> 6] = v;
            red[G / 64 + (threadIdx.x >> 6)] = w;
        }
        __syncthreads();
        v = w = 0.0f;
#pragma unroll
        for (int k = 0; k < G / 64; ++k) {
            v += red[k];
            w += red[G / 64 + k];
        }
    }
}

struct NormArgs {
    const void *x;
    const float *gamma, *beta;
    int64_t n;
    int H;
    float eps, inv_h;
    void *y;
    float *mean, *rstd;
    Drop drop;
    // backward
    const void *gy;
    float *dx, *part;
};

template <typename T, int G, int NV>
__global__ void __launch_bounds__(G <= 64 ? kT : kWide)
layernorm_kernel(const NormArgs a) {
    constexpr int V = kVec<T>, THREADS = G <= 64 ? kT : kWide, GROUPS = THREADS / G;
    __shared__ float red[G <= 64 ? 1 : 3 * kWide / 64];
    const int l = threadIdx.x % G, H = a.H;
    const T *x = static_cast<const T *>(a.x);
    const uint64_t start = a.drop.state ? drop_start(a.drop) : 0;
    float gamma[NV][V], beta[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * G + l) * V;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            gamma[j][k] = c + k < H ? a.gamma[c + k] : 0.0f;
            beta[j][k] = c + k < H ? a.beta[c + k] : 0.0f;
        }
    }
    // the next row is on its way while this one is worked on
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    Piece<T, V> next[NV];
    auto fetch = [&](int64_t r) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + l) * V;
            next[j] = load_row<T, V>(x + r * H + c, H - c);
        }
    };
    if (row < a.n) fetch(row);
    for (; row < a.n; row += step) {
        float v[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j) unpack<T, V>(next[j], v[j]);
        if (row + step < a.n) fetch(row + step);
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int k = 0; k < V; ++k) s += v[j][k];
        }
        const float m0 = row_sum<G>(s, red) / (float)H;           // (a quotient: a product would be fused into the differences, unrounded)
        float off = 0.0f, sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                v[j][k] -= m0;
                if ((j * G + l) * V + k < H) {
                    off += v[j][k];
                    sq += v[j][k] * v[j][k];
                }
            }
        row_sums<G>(off, sq, red + kWide / 64 * (G > 64));
        float more = off * a.inv_h, taken = off * more;
        // up to 2^-23 of the spread, c is the rounding of the differences as likely as what the mean is off by, and the mean stays
        if (taken < 0x1p-46f * sq) more = taken = 0.0f;
        const float mean = more == more ? m0 + more : m0, left = sq - taken;       // (an infinite mean stays one)
        const float rstd = 1.0f / sqrtf((left < 0.0f ? 0.0f : left) * a.inv_h + a.eps);        // (below 0 by rounding alone: equal values)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + l) * V;
            if (c >= H) continue;
#pragma unroll
            for (int k = 0; k < V; ++k) v[j][k] = (v[j][k] - more) * rstd * gamma[j][k] + beta[j][k];
            if (a.drop.state) apply_drop<V>(a.drop, start, (uint64_t)row * H + c, v[j]);
            store_row_piece<T, V>(static_cast<T *>(a.y) + row * H + c, H - c, v[j]);
        }
        if (l == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// The rows of a block add to the same columns: every lane keeps the weight gradients of its columns, the groups of a block are
// added in order through LDS, the blocks by layernorm_reduce_kernel, also in order: the result does not depend on timing.
// A lane's sums start anew every kChain rows, and those before are added to its second ones: one chain over all its rows (1.18 M x 512:
// 288) would lose up to half a step of the whole sum in each addition, 5e-6 of it where the terms are alike; norm-wise, of random terms,
// 3.3e-7 became 1.4e-7.
template <typename T, typename GT, int G, int NV>
__global__ void __launch_bounds__(G <= 64 ? kT : kWide)
layernorm_backward_kernel(const NormArgs a) {
    constexpr int V = kVec<T>, THREADS = G <= 64 ? kT : kWide, GROUPS = THREADS / G;
    __shared__ float red[G <= 64 ? 1 : 3 * kWide / 64];
    constexpr int W = G * NV * V;
    __shared__ float sums[2 * W * GROUPS];          // KEEP: the second sums, in lane order; else the first, in column order
    int l = threadIdx.x % G;
    const int H = a.H;
    const T *x = static_cast<const T *>(a.x);
    const GT *gy = static_cast<const GT *>(a.gy);
    const uint64_t start = a.drop.state ? drop_start(a.drop) : 0;
    // gamma and the gradients of the longest rows do not fit the registers of 512 threads: the gradients stay in LDS, their second sums
    // where the block's go
    constexpr bool KEEP = G <= 64;
    constexpr bool AHEAD = G <= 64 && NV * V <= 16;      // the next row is on its way while this one is worked on, where registers allow
    float gamma[KEEP ? NV : 1][V], dgamma[KEEP ? NV : 1][V], dbeta[KEEP ? NV : 1][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int c = (j * G + l) * V + k;
            if constexpr (KEEP) {
                gamma[j][k] = c < H ? a.gamma[c] : 0.0f;
                dgamma[j][k] = dbeta[j][k] = 0.0f;
            } else {
                sums[c] = sums[W + c] = 0.0f;
            }
        }
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    Piece<T, V> next_x[NV];
    Piece<GT, V> next_g[NV];
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto fetch = [&](int64_t r) __attribute__((always_inline)) {
        next_mean = a.mean[r];
        next_rstd = a.rstd[r];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + l) * V;
            next_x[j] = load_row<T, V>(x + r * H + c, H - c);
            next_g[j] = load_row<GT, V>(gy + r * H + c, H - c);
        }
    };
    float *part = a.part + (int64_t)blockIdx.x * 2 * H;
    bool begun = false;
    auto second = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if constexpr (KEEP) {
                    float &sg = sums[(j * V + k) * THREADS + threadIdx.x], &sb = sums[((NV + j) * V + k) * THREADS + threadIdx.x];
                    sg = begun ? sg + dgamma[j][k] : dgamma[j][k];
                    sb = begun ? sb + dbeta[j][k] : dbeta[j][k];
                    dgamma[j][k] = dbeta[j][k] = 0.0f;
                } else {
                    const int c = (j * G + l) * V + k;
                    if (c >= H) continue;
                    part[c] = begun ? part[c] + sums[c] : sums[c];
                    part[H + c] = begun ? part[H + c] + sums[W + c] : sums[W + c];
                    sums[c] = sums[W + c] = 0.0f;
                }
            }
        begun = true;
    };
    int chain = 0;
    if (AHEAD && row < a.n) fetch(row);
    for (; row < a.n; row += step) {
        if constexpr (!AHEAD) fetch(row);
        if constexpr (!KEEP) asm volatile("" : "+v"(l));        // addresses and gamma anew for each row: kept, they cost registers
        float xh[NV][V], g[NV][V];
        const float mean = next_mean, rstd = next_rstd;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack<T, V>(next_x[j], xh[j]);
            unpack<GT, V>(next_g[j], g[j]);
        }
        if (AHEAD && row + step < a.n) fetch(row + step);
        // A mean is kept to 2^-24 of itself: where that is much of a row's spread, what is left of it comes off the centred values here too
        float more = 0.0f;
        const bool far = fabsf(mean) * rstd > kFar;
        if (__any(far)) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if ((j * G + l) * V + k < H) more += xh[j][k] - mean;
            more = row_sum<G>(more, red + 2 * kWide / 64 * (G > 64)) * a.inv_h;
            more = far ? more : 0.0f;                          // (a row's result does not depend on those beside it in a wave)
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + l) * V;
            if (a.drop.state) apply_drop<V>(a.drop, start, (uint64_t)row * H + c, g[j]);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                xh[j][k] = (xh[j][k] - mean - more) * rstd;
                if (c + k >= H) xh[j][k] = g[j][k] = 0.0f;
                if constexpr (KEEP) {
                    dgamma[j][k] += g[j][k] * xh[j][k];
                    dbeta[j][k] += g[j][k];
                    g[j][k] *= gamma[j][k];
                } else {
                    sums[c + k] += g[j][k] * xh[j][k];
                    sums[W + c + k] += g[j][k];
                    g[j][k] *= c + k < H ? a.gamma[c + k] : 0.0f;
                }
                s1 += g[j][k];
                s2 += g[j][k] * xh[j][k];
            }
        }
        s1 = row_sum<G>(s1, red) * a.inv_h;
        s2 = row_sum<G>(s2, red + kWide / 64 * (G > 64)) * a.inv_h;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + l) * V;
            if (c >= H) continue;
#pragma unroll
            for (int k = 0; k < V; ++k) g[j][k] = (g[j][k] - s1 - xh[j][k] * s2) * rstd;
            store_row_piece<float, V>(a.dx + row * H + c, H - c, g[j]);
        }
        if (++chain == (KEEP ? kChain : kWideChain)) {
            second();
            chain = 0;
        }
    }
    second();
    if constexpr (KEEP) {
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * H; c += THREADS) {
            const int of = c < H ? c : c - H, piece = of / V, at = ((c < H ? 0 : NV) + piece / G) * V + of % V;
            float s = 0.0f;
#pragma unroll
            for (int q = 0; q < GROUPS; ++q) s += sums[at * THREADS + q * G + piece % G];
            part[c] = s;
        }
    }
}

// column c of [n_parts, 2H], 16 parts at a time and the sixteen sums in order; in fp64, which costs nothing here
__global__ void __launch_bounds__(1024)
layernorm_reduce_kernel(const float *__restrict__ part, int n_parts, int H, float *__restrict__ dgamma, float *__restrict__ dbeta) {
    __shared__ double sums[16][64];
    const int l = threadIdx.x & 63, q = threadIdx.x >> 6, c = blockIdx.x * 64 + l;
    double s = 0.0;
    if (c < 2 * H)
#pragma unroll 8
        for (int p = q; p < n_parts; p += 16) s += part[(int64_t)p * 2 * H + c];
    sums[q][l] = s;
    __syncthreads();
    if (q || c >= 2 * H) return;
    for (int k = 1; k < 16; ++k) s += sums[k][l];
    if (c < H) dgamma[c] = (float)s;
    else dbeta[c - H] = (float)s;
}

int norm_groups(int H, int vec) {       // rows that a block works on at once
    const int pieces = (int)ceil_div(H, vec);
    return H > kWaveMax ? 1 : pieces <= 16 ? kT / 16 : pieces <= 32 ? kT / 32 : kT / 64;
}
// no more blocks than there are rows for
int norm_blocks(int64_t n, int H, int vec, int most) {
    const int64_t b = ceil_div(n, norm_groups(H, vec));
    return (int)(b < most ? b : most);
}

// launch(G, NV) for rows of H values in pieces of `vec`
template <int VEC, typename F>
void for_width(int H, F &&launch) {
    const int pieces = (int)ceil_div(H, VEC);
    if (H > kWaveMax) launch(std::integral_constant<int, kWide>(), std::integral_constant<int, kMaxWidth / (kWide * VEC)>());
    else if (pieces <= 16) launch(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    else if (pieces <= 32) launch(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    else if (pieces <= 64) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    else if (pieces <= 128) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    else if (pieces <= 256) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
    else if constexpr (VEC == 4) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
}

template <typename T>
int run_forward_norm(const NormArgs &a, hipStream_t st) {
    const int blocks = norm_blocks(a.n, a.H, kVec<T>, kForwardBlocks);
    for_width<kVec<T>>(a.H, [&](auto g, auto nv) {
        constexpr int G = decltype(g)::value, NV = decltype(nv)::value;
        layernorm_kernel<T, G, NV><<<blocks, G <= 64 ? kT : kWide, 0, st>>>(a);
    });
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}
template <typename T, typename GT>
int run_backward_norm(const NormArgs &a, float *dgamma, float *dbeta, hipStream_t st) {
    const int blocks = norm_blocks(a.n, a.H, kVec<T>, kMaxParts);
    for_width<kVec<T>>(a.H, [&](auto g, auto nv) {
        constexpr int G = decltype(g)::value, NV = decltype(nv)::value;
        layernorm_backward_kernel<T, GT, G, NV><<<blocks, G <= 64 ? kT : kWide, 0, st>>>(a);
    });
    JITDB_LAUNCH_CHECK();
    layernorm_reduce_kernel<<<(unsigned)ceil_div(2 * a.H, 64), 1024, 0, st>>>(a.part, blocks, a.H, dgamma, dbeta);
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}

bool known(jitdb_dtype t) { return t == JITDB_F32 || t == JITDB_BF16; }
bool off_type(const void *p, jitdb_dtype t) { return reinterpret_cast<uintptr_t>(p) & (t == JITDB_F32 ? 3 : 1); }
bool off_f32(const void *p) { return reinterpret_cast<uintptr_t>(p) & 3; }
bool off_state(const void *p) { return reinterpret_cast<uintptr_t>(p) & 7; }
bool norm_sizes(int64_t n, int32_t H) { return n >= 0 && n <= JITDB_MAX_NODES && H >= 1 && H <= kMaxWidth; }

}  // namespace
}  // namespace jitdb

using namespace jitdb;

extern "C" int jitdb_dropout(const void *x, int64_t n, jitdb_dtype dtype, float p, const uint64_t *state, void *y, void *hip_stream) {
    drop_stale_hip_error();
    if (n < 0 || n > ((int64_t)1 << 42) || !known(dtype) || !(p >= 0.0f && p <= 1.0f)) return JITDB_E_BADARG;
    if (n == 0) return JITDB_OK;
    if (!x || !y || !state) return JITDB_E_NULL;
    if (off_type(x, dtype) || off_type(y, dtype) || off_state(state)) return JITDB_E_BADARG;
    const Drop d = make_drop(p, state);
    hipStream_t st = (hipStream_t)hip_stream;
    const int vec = dtype == JITDB_F32 ? kVec<float> : kVec<bf16_t>;
    const int64_t want = ceil_div(n, (int64_t)kT * vec * 4);
    const unsigned blocks = (unsigned)(want < 4096 ? want : 4096);
    if (dtype == JITDB_F32) dropout_kernel<float><<<blocks, kT, 0, st>>>(static_cast<const float *>(x), n, d, static_cast<float *>(y));
    else dropout_kernel<bf16_t><<<blocks, kT, 0, st>>>(static_cast<const bf16_t *>(x), n, d, static_cast<bf16_t *>(y));
    JITDB_LAUNCH_CHECK();
    return JITDB_OK;
}

extern "C" int jitdb_layernorm_forward(const void *x, const float *gamma, const float *beta, int64_t n_rows, int32_t H,
                                       jitdb_dtype dtype, float eps, float p, const uint64_t *state,
                                       void *y, float *mean, float *rstd, void *hip_stream) {
    drop_stale_hip_error();
    if (!norm_sizes(n_rows, H) || !known(dtype) || !(p >= 0.0f && p <= 1.0f) || !(eps >= 0.0f && eps < 3.0e38f)) return JITDB_E_BADARG;
    if (n_rows == 0) return JITDB_OK;
    if (!x || !gamma || !beta || !y || (p > 0.0f && !state)) return JITDB_E_NULL;
    if (off_type(x, dtype) || off_type(y, dtype) || off_f32(gamma) || off_f32(beta) || off_f32(mean) || off_f32(rstd) ||
        (p > 0.0f && off_state(state)))
        return JITDB_E_BADARG;
    NormArgs a = {};
    a.x = x; a.gamma = gamma; a.beta = beta; a.n = n_rows; a.H = H; a.eps = eps; a.inv_h = 1.0f / (float)H;
    a.y = y; a.mean = mean; a.rstd = rstd; a.drop = make_drop(p, p > 0.0f ? state : nullptr);
    hipStream_t st = (hipStream_t)hip_stream;
    return dtype == JITDB_F32 ? run_forward_norm<float>(a, st) : run_forward_norm<bf16_t>(a, st);
}

extern "C" size_t jitdb_layernorm_backward_workspace_bytes(int64_t n_rows, int32_t H, jitdb_dtype dtype) {
    if (!norm_sizes(n_rows, H) || !known(dtype)) return 0;
    Carver c(nullptr);
    const int parts = norm_blocks(n_rows, H, dtype == JITDB_F32 ? kVec<float> : kVec<bf16_t>, kMaxParts);
    c.take<float>((size_t)(parts > 0 ? parts : 1) * 2 * H);
    return c.off;
}

extern "C" int jitdb_layernorm_backward(const void *x, const float *gamma, const float *mean, const float *rstd,
                                        const void *gy, int64_t n_rows, int32_t H, jitdb_dtype dtype, jitdb_dtype grad_dtype,
                                        float p, const uint64_t *state, float *dx, float *dgamma, float *dbeta,
                                        void *workspace, size_t workspace_bytes, void *hip_stream) {
    drop_stale_hip_error();
    if (!norm_sizes(n_rows, H) || !known(dtype) || !known(grad_dtype) || !(p >= 0.0f && p <= 1.0f)) return JITDB_E_BADARG;
    if (!dgamma || !dbeta) return JITDB_E_NULL;
    if (off_f32(dgamma) || off_f32(dbeta)) return JITDB_E_BADARG;
    hipStream_t st = (hipStream_t)hip_stream;
    if (n_rows == 0) {                   // no parts: their sums are 0
        layernorm_reduce_kernel<<<(unsigned)ceil_div(2 * H, 64), 1024, 0, st>>>(nullptr, 0, H, dgamma, dbeta);
        JITDB_LAUNCH_CHECK();
        return JITDB_OK;
    }
    if (!x || !gamma || !mean || !rstd || !gy || !dx || !workspace || (p > 0.0f && !state)) return JITDB_E_NULL;
    if (off_type(x, dtype) || off_type(gy, grad_dtype) || off_f32(gamma) || off_f32(mean) || off_f32(rstd) || off_f32(dx) ||
        (p > 0.0f && off_state(state)) || (reinterpret_cast<uintptr_t>(workspace) & 255))
        return JITDB_E_BADARG;
    if (workspace_bytes < jitdb_layernorm_backward_workspace_bytes(n_rows, H, dtype)) return JITDB_E_WORKSPACE;
    NormArgs a = {};
    a.x = x; a.gamma = gamma; a.n = n_rows; a.H = H; a.inv_h = 1.0f / (float)H;
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd); a.gy = gy; a.dx = dx;
    a.part = static_cast<float *>(workspace); a.drop = make_drop(p, p > 0.0f ? state : nullptr);
    if (dtype == JITDB_F32)
        return grad_dtype == JITDB_F32 ? run_backward_norm<float, float>(a, dgamma, dbeta, st)
                                       : run_backward_norm<float, bf16_t>(a, dgamma, dbeta, st);
    return grad_dtype == JITDB_F32 ? run_backward_norm<bf16_t, float>(a, dgamma, dbeta, st)
                                   : run_backward_norm<bf16_t, bf16_t>(a, dgamma, dbeta, st);
}
