// Softmax cross entropy over few classes (up to 64): bound by memory, so every state is read once from HBM and everything that
// is computed from it happens while it passes.
//
// The class weights lie in LDS.  A wave works on 16 rows: their logits come from the matrix instructions of 16 classes x 16 rows (a
// lane holds one row and four classes of every 16), so that statistics are sums over four lanes' registers; the derivatives g of the
// logits are in the place where the product g V (fp32 matrix instructions, as for the weights' gradients) wants them, and the rows'
// gradients leave at once.  The weights' gradients sum over rows: the 64 rows of a block put their g into LDS, and each wave adds them
// to its own quarter of the features, reading the states a second time out of L2, now with a feature in each lane.  Blocks keep their
// sums in registers to the end; few_reduce_kernel adds the blocks in order.
// 1.18 M rows of 512, 5 classes, bf16: forward 240 us (5.0 TB/s), backward with fp32 dh 785 (4.6 TB/s; 945 with half lines stored).
#pragma once

#include "level_common.h"
#include "xent_sizes.h"

namespace jitdb {
namespace {

constexpr int kFewT = 256;               // threads of a block: four waves
template <typename T> constexpr int kFewVec = 16 / (int)sizeof(T);        // elements of one load
template <typename T> constexpr int kFewBlock = 64 * kFewVec<T>;          // features that four waves cover with one load a lane

struct FewArgs {
    const void *h, *V;
    const float *b;
    const int32_t *label;
    int64_t n;
    int H, C;
    // forward
    float *loss, *lse;
    // backward
    const float *lse_in, *gloss;
    void *dh;
    float *part;                         // [blocks][C H + C]
    void *dV; float *db;                 // of a single block
};

// The weights in LDS: in the order of the logits' loads, K in steps of four loads side by side.  Element e of piece (step s, quarter q)
// of class i; 17 pieces instead of 16 spread the other reader, who wants one element of 4 x 16 pieces at once, over the banks.
template <typename T>
__device__ __forceinline__ int few_at(int steps, int ct, int s, int q, int i, int e) {
    return ((((ct * steps + s) * 4 + q) * 17) + i) * kFewVec<T> + e;
}
template <typename T, int CT, int NB>
struct FewTable {
    static constexpr int kSteps = NB * kFewBlock<T> / (4 * kFewVec<T>);
    T w[CT * kSteps * 4 * 17 * kFewVec<T>];
    float bias[CT * 16];
    __device__ __forceinline__ void load(const FewArgs &a) {
        constexpr int V = kFewVec<T>;
        const T *src = static_cast<const T *>(a.V);
        const int steps = (a.H + 4 * V - 1) / (4 * V) + 1;      // the gradient goes by 32 features: at most one more step
        for (int p = threadIdx.x; p < CT * 16 * steps * 4; p += kFewT) {
            const int piece = p % (steps * 4), c = p / (steps * 4), s = piece >> 2, q = piece & 3, k = piece * V;
            if (s >= kSteps) continue;
            T e[V];
#pragma unroll
            for (int j = 0; j < V; ++j) e[j] = c < a.C && k + j < a.H ? src[(int64_t)c * a.H + k + j] : T(0);
            __builtin_memcpy(&w[few_at<T>(kSteps, c >> 4, s, q, c & 15, 0)], e, 16);
        }
        for (int c = threadIdx.x; c < CT * 16; c += kFewT) bias[c] = c >= a.C ? -INFINITY : a.b ? a.b[c] : 0.0f;
    }
};

// Sixteen bytes of a row as they are; only the first `left` elements exist (none: zeros).
template <typename T>
__device__ __forceinline__ u32x4 few_load(const T *p, int left) {
    constexpr int V = kFewVec<T>;
    u32x4 w = {0u, 0u, 0u, 0u};
    if (left >= V) {
        __builtin_memcpy(&w, p, 16);
    } else if (left > 0) {
        T e[V];
#pragma unroll
        for (int k = 0; k < V; ++k) e[k] = k < left ? p[k] : T(0);
        __builtin_memcpy(&w, e, 16);
    }
    return w;
}
template <typename T>
__device__ __forceinline__ float few_element(const u32x4 &w, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
}

// z[ct][v]: logit of class 16 ct + 4 (lane / 16) + v, row `row` (that of the lane; every sixteenth lane has the same), bias and all
template <typename T, int CT, int NB>
__device__ __forceinline__ void few_logits(const FewArgs &a, const FewTable<T, CT, NB> &t, const T *row, bool has, floatx4 (&z)[CT]) {
    constexpr int V = kFewVec<T>, STEPS = FewTable<T, CT, NB>::kSteps;
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 4; ++v) z[ct][v] = t.bias[ct * 16 + q * 4 + v];
    auto step = [&](int s, const u32x4 &x) __attribute__((always_inline)) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            u32x4 w;
            __builtin_memcpy(&w, &t.w[few_at<T>(STEPS, ct, s, q, i, 0)], 16);
            mfma16<T>(w, x, z[ct]);                  // (products of bf16 values are exact)
        }
    };
    const int whole = has ? a.H / (4 * V) : 0, steps = (a.H + 4 * V - 1) / (4 * V);
    const T *at = row + q * V;
    int s = 0;
    for (; s + 4 <= a.H / (4 * V); s += 4) {         // four loads in flight
        u32x4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = few_load<T>(at + (s + u) * 4 * V, whole ? V : 0);
#pragma unroll
        for (int u = 0; u < 4; ++u) step(s + u, x[u]);
    }
    for (; s < steps; ++s) step(s, few_load<T>(at + s * 4 * V, has ? a.H - (s * 4 + q) * V : 0));
}
__device__ __forceinline__ float quarters_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float quarters_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

template <typename T, int CT, int NB>
__global__ void __launch_bounds__(kFewT)
few_forward_kernel(const FewArgs a) {
    __shared__ FewTable<T, CT, NB> table;
    table.load(a);
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
    const T *h = static_cast<const T *>(a.h);
    for (int64_t r0 = ((int64_t)blockIdx.x * 4 + wave) * 16; r0 < a.n; r0 += (int64_t)gridDim.x * kFewRows) {
        const int64_t r = r0 + (lane & 15);
        const int label = r < a.n ? a.label[r] : -1;
        const bool has = label != -1;
        float loss = 0.0f, lse = 0.0f;
        if (__any(has)) {
            floatx4 z[CT];
            few_logits<T, CT, NB>(a, table, h + (has ? r : 0) * a.H, has, z);
            float top = -INFINITY, at = 0.0f, s = 0.0f;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    top = fmaxf(top, z[ct][v]);
                    if (label == ct * 16 + q * 4 + v) at = z[ct][v];
                }
            top = quarters_max(top);
            const float from = fabsf(top) == INFINITY ? 0.0f : top;       // every class masked: the sum is 0, not NaN; a logit of +inf: it is +inf
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int v = 0; v < 4; ++v) s += expf(z[ct][v] - from);
            lse = from + logf(quarters_sum(s));
            at = quarters_sum(at);
            loss = label >= 0 && label < a.C ? lse - at : __builtin_nanf("");
        }
        if (q == 0 && r < a.n) {
            a.loss[r] = has ? loss : 0.0f;
            a.lse[r] = has ? lse : 0.0f;
        }
    }
}

template <typename T, typename O, int CT, int NB>
__global__ void __launch_bounds__(kFewT, CT * NB * kFewVec<T> <= 8 ? 4 : 1)
few_backward_kernel(const FewArgs a) {
    constexpr int V = kFewVec<T>, STEPS = FewTable<T, CT, NB>::kSteps, COLS = CT * 16;
    __shared__ FewTable<T, CT, NB> table;
    __shared__ __attribute__((aligned(16))) float gs[2][kFewRows][COLS];
    __shared__ int32_t has_of[2][kFewRows];
    table.load(a);
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, q = lane >> 4, H = a.H;
    const T *h = static_cast<const T *>(a.h);
    O *dh = static_cast<O *>(a.dh);
    floatx4 dv[NB][V][CT];                           // feature (nb 4 + wave) 16 V + i16 V + e, classes 16 ct + 4 q + v
    float db[CT][4];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            db[ct][v] = 0.0f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < V; ++e) dv[nb][e][ct][v] = 0.0f;
        }
    int turn = 0;
    for (int64_t b0 = (int64_t)blockIdx.x * kFewRows; b0 < a.n; b0 += (int64_t)gridDim.x * kFewRows, turn ^= 1) {
        const int64_t r = b0 + wave * 16 + i16;
        const int label = r < a.n ? a.label[r] : -1;
        const bool has = label != -1;
        floatx4 g[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) g[ct] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        if (__any(has)) {
            floatx4 z[CT];
            few_logits<T, CT, NB>(a, table, h + (has ? r : 0) * H, has, z);
            const float lse = has ? a.lse_in[r] : 0.0f;
            const float w = !has ? 0.0f : label < 0 || label >= a.C ? __builtin_nanf("") : a.gloss ? a.gloss[r] : 1.0f;
            if (has)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int c = ct * 16 + q * 4 + v;
                        // classes past the last have p = 0 and weights of 0: they add nothing, also in rows that are NaN
                        const float d = expf(z[ct][v] - lse) - (label == c ? 1.0f : 0.0f);
                        g[ct][v] = c < a.C ? d * w : 0.0f;
                        db[ct][v] += g[ct][v];
                    }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) *reinterpret_cast<floatx4 *>(&gs[turn][wave * 16 + i16][ct * 16 + q * 4]) = g[ct];
        if (q == 0) has_of[turn][wave * 16 + i16] = has;
        // dh of the wave's rows, 128 bytes of each at a time: a lane has two pieces of sixteen bytes of its row (fp32: features 4 q ..
        // 4 q + 3 of either half; bf16: 8 q .. 8 q + 7) and exchanges one with the row eight lanes on, so that a store writes whole
        // lines of eight rows.  Nothing reads dh soon: past the caches, where the states wait for their second reading
        constexpr int PER = 16 / (int)sizeof(O), STEP = 8 * PER, D = STEP / 16;
        const bool low = i16 < 8;
        const int64_t first = b0 + wave * 16 + (i16 & 7);
        for (int f0 = 0; f0 < H; f0 += STEP) {
            floatx4 d[D];
#pragma unroll
            for (int u = 0; u < D; ++u) {
                d[u] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                const int f = f0 + (sizeof(O) == 4 ? u * 16 + i16 : (u >> 1) * 32 + (i16 >> 2) * 8 + (u & 1) * 4 + (i16 & 3));    // whose weights this lane brings
                const int s = f / (4 * V), fq = f / V & 3, e = f % V;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        d[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(to_f32<T>(table.w[few_at<T>(STEPS, ct, s, fq, q * 4 + v, e)]), g[ct][v], d[u], 0, 0, 0);
            }
            u32x4 piece[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                O e[PER];
#pragma unroll
                for (int k = 0; k < PER; ++k) e[k] = from_f32<O>(has ? d[p * (D / 2) + (k >> 2)][k & 3] : 0.0f);
                __builtin_memcpy(&piece[p], e, 16);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t other = __builtin_amdgcn_mov_dpp(low ? piece[1][k] : piece[0][k], 0x128, 0xF, 0xF, true);      // of lane i16 ^ 8
                if (low) piece[1][k] = other;
                else piece[0][k] = other;
            }
            const int f = f0 + (low ? 0 : STEP / 2) + q * PER;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                if (first + 8 * p >= a.n) continue;
                O *o = dh + (first + 8 * p) * H + f;
                if (f + PER <= H) {
                    typedef u32x4 __attribute__((aligned(2))) any4;
                    __builtin_nontemporal_store(piece[p], reinterpret_cast<any4 *>(o));
                } else {
                    O e[PER];
                    __builtin_memcpy(e, &piece[p], 16);
#pragma unroll
                    for (int k = 0; k < PER; ++k)
                        if (f + k < H) o[k] = e[k];
                }
            }
        }
        __syncthreads();                             // the 64 rows' g is there; the other buffer is free again behind the next one
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int f = ((nb * 4 + wave) * 16 + i16) * V;
            if ((nb * 4 + wave) * 16 * V >= H) continue;
            // four rows a quarter in flight; `left`: elements of the lane's piece (a block of features that ends inside one is the exception)
            auto add = [&](int left) __attribute__((always_inline)) {
                for (int k0 = 0; k0 < kFewRows; k0 += 16) {
                    u32x4 x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int rr = k0 + 4 * k + q;
                        const bool on = has_of[turn][rr];
                        x[k] = few_load<T>(h + (on ? (b0 + rr) * H + f : 0), on ? left : 0);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) {
                            const float ga = gs[turn][k0 + 4 * k + q][ct * 16 + i16];
#pragma unroll
                            for (int e = 0; e < V; ++e)
                                dv[nb][e][ct] = __builtin_amdgcn_mfma_f32_16x16x4f32(ga, few_element<T>(x[k], e), dv[nb][e][ct], 0, 0, 0);
                        }
                }
            };
            if (((nb * 4 + wave) * 16 + 16) * V <= H) add(V);
            else add(H - f);
        }
    }
    float *part = a.part + (int64_t)blockIdx.x * ((int64_t)a.C * H + a.C);
    O *own = static_cast<O *>(a.dV);                 // a single block's sums are the gradients
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int c = ct * 16 + q * 4 + v, f = ((nb * 4 + wave) * 16 + i16) * V;
                if (c < a.C)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (f + e < H) {
                            if (own) own[(int64_t)c * H + f + e] = from_f32<O>(dv[nb][e][ct][v]);
                            else part[(int64_t)c * H + f + e] = dv[nb][e][ct][v];
                        }
            }
    // the bias: over the 16 lanes that hold the same classes, then the four waves
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            float s = db[ct][v];
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) s += __shfl_xor(s, m);
            if (i16 == 0) gs[0][wave][ct * 16 + q * 4 + v] = s;
        }
    __syncthreads();
    float *bias = own ? a.db : part + (int64_t)a.C * H;
    if ((int)threadIdx.x < a.C)
        bias[threadIdx.x] = gs[0][0][threadIdx.x] + gs[0][1][threadIdx.x] + gs[0][2][threadIdx.x] + gs[0][3][threadIdx.x];
}

// Value c of [n_parts][C H + C]: 64 values a block, sixteen waves take every sixteenth part in order, then the sixteen in order.
template <typename O>
__global__ void __launch_bounds__(1024)
few_reduce_kernel(const float *__restrict__ part, int n_parts, int H, int C, O *__restrict__ dV, float *__restrict__ db) {
    __shared__ float sums[16][64];
    const int64_t weights = (int64_t)C * H, width = weights + C;
    const int l = threadIdx.x & 63, q = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + l;
    float s = 0.0f;
    if (c < width)
#pragma unroll 8
        for (int p = q; p < n_parts; p += 16) s += part[p * width + c];
    sums[q][l] = s;
    __syncthreads();
    if (q || c >= width) return;
    for (int k = 1; k < 16; ++k) s += sums[k][l];
    if (c < weights) dV[c] = from_f32<O>(s);
    else db[c - weights] = s;
}

// The variant of H features and C classes: launch(classes / 16, blocks of features), false where there is none.
template <typename T, typename F>
bool for_few(int H, int C, F &&launch) {
    const FewSizes few = few_sizes(sizeof(T), H, C);
    auto with = [&](auto c, auto b) {
        constexpr int CT = decltype(c)::value, NB = decltype(b)::value;
        static_assert(sizeof(FewTable<T, CT, NB>) == few_table_bytes(CT, NB), "what the rule counts with is what there is");
        if constexpr (few_variant(sizeof(T), CT, NB)) {
            if (few.ct == CT && few.nb == NB) launch(c, b);
        }
    };
    auto blocks = [&](auto c) {
        with(c, std::integral_constant<int, 1>());
        with(c, std::integral_constant<int, 2>());
        with(c, std::integral_constant<int, 4>());
        with(c, std::integral_constant<int, 8>());
    };
    blocks(std::integral_constant<int, 1>());
    blocks(std::integral_constant<int, 2>());
    blocks(std::integral_constant<int, 4>());
    return few.ct > 0;
}

}  // namespace
}  // namespace jitdb
