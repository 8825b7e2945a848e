// Top-k router with balance and z loss: one pass over the logits forward, one backward.
//
// Forward: softmax, choice and weights are local to a token; the losses need the sums over tokens of p_te, of lse^2 and
// the counts.  Every thread (up to 32 experts) or lane (more) keeps the sums of its own experts in registers over all
// its tokens, the block adds them up in a fixed order and leaves one partial row in the workspace, and the block that
// finishes last adds the rows, again in a fixed order.  One launch, and no floating-point atomics.
// Backward: with the counts known the gradient of a token's logits is local to the token again; it is recomputed from
// the logits, which are the only thing both passes have to read.
#include "layer_common.h"

namespace loco_layer {

constexpr int kRouterThreads = 256;
constexpr int kRouterWarps = kRouterThreads / 32;
constexpr int kMaxExperts = 512;
constexpr int kMaxChoice = 16;
constexpr int kBlocksPerSm = 2;
constexpr int kMaxBlocks = 512;                     // partial rows the workspace holds
constexpr unsigned kAll = 0xffffffffu;

struct RouterParams {
    const void *logits;
    int64_t row_stride;
    const uint8_t *mask;
    int32_t *index;
    float *weight;
    int32_t *counts;
    float *mean, *losses;
    unsigned *ticket;                                // zero between calls
    float *part;                                     // [block][2 E + 2]: sums of p, counts (as integers), sum of lse^2, active tokens
    // backward
    const int32_t *in_index, *in_counts;
    const float *dlosses, *dweight;
    void *dlogits;
    int64_t drow_stride;
    int64_t tokens;
    int32_t experts, top_k, normalize;
    float balance_coef, z_coef;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}

// Order of the choice as unsigned integers: larger logit first, NaN before all.  -inf maps to 0x007fffff; 0 is free.
__device__ __forceinline__ unsigned order_key(float z) {
    const unsigned u = __float_as_uint(z);
    const unsigned k = u & 0x80000000u ? ~u : u | 0x80000000u;
    return z != z ? 0xffffffffu : (z == 0.0f ? 0x80000000u : k);
}
constexpr unsigned kKeyMinusInf = 0x007fffffu;

// A row of up to N logits, -inf where there is none.
template <typename T, int N, bool kWide> __device__ __forceinline__ void load_row(const T *row, int experts, float *z) {
    constexpr int kV = 16 / sizeof(T);
    if constexpr (kWide) {
#pragma unroll
        for (int i = 0; i < N / kV; ++i) {
            if (i * kV < experts) {
                const Pack<T, kV> p = *reinterpret_cast<const Pack<T, kV> *>(row + i * kV);
#pragma unroll
                for (int j = 0; j < kV; ++j) z[i * kV + j] = to_f32(p.v[j]);
            } else {
#pragma unroll
                for (int j = 0; j < kV; ++j) z[i * kV + j] = -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = i < experts ? to_f32(row[i]) : -INFINITY;
    }
}

// Adds the blocks' partial rows once all of them are written; called by every thread with the block's own row in shared
// memory: sums[E], tally[E], extra = {sum of lse^2, active tokens}.
__device__ void finish(const RouterParams &P, const float *sums, const int *tally, float zsq, int active) {
    __shared__ bool last;
    __shared__ double fold[kRouterThreads];
    __shared__ int ifold[kRouterThreads];
    __shared__ float mean[kMaxExperts];
    __shared__ int count[kMaxExperts];
    const int E = P.experts, width = 2 * E + 2, tid = threadIdx.x;
    const int blocks = static_cast<int>(gridDim.x);
    float *mine = P.part + static_cast<int64_t>(blockIdx.x) * width;
    for (int e = tid; e < E; e += kRouterThreads) {
        mine[e] = sums[e];
        mine[E + e] = __int_as_float(tally[e]);
    }
    if (tid == 0) {
        mine[2 * E] = zsq;
        mine[2 * E + 1] = __int_as_float(active);
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(P.ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (tid == 0) *P.ticket = 0;
    // slices of blocks per column, so that few experts still use all threads
    int slices = 1;
    while (slices * 2 * (E + 1) <= kRouterThreads && slices < blocks) slices *= 2;
    double zz = 0.0;
    int n = 0;
    const int columns = E + 1;                        // the last one: lse^2 and active tokens
    for (int c0 = 0; c0 < columns; c0 += kRouterThreads / slices) {
        const int c = c0 + tid / slices, s = tid % slices;
        double a = 0.0;
        int k = 0;
        if (c < columns) {
            const int fa = c < E ? c : 2 * E, ia = c < E ? E + c : 2 * E + 1;
#pragma unroll 8
            for (int b = s; b < blocks; b += slices) {
                const float *row = P.part + static_cast<int64_t>(b) * width;
                a += static_cast<double>(__ldcg(row + fa));
                k += __float_as_int(__ldcg(row + ia));
            }
        }
        fold[tid] = a;
        ifold[tid] = k;
        __syncthreads();
        if (s == 0 && c < columns) {
            for (int i = 1; i < slices; ++i) {
                a += fold[tid + i];
                k += ifold[tid + i];
            }
            if (c < E) {
                mean[c] = static_cast<float>(a);      // still the sum
                count[c] = k;
            } else {
                fold[tid] = a;
                ifold[tid] = k;
            }
        }
        __syncthreads();
        if (c0 + kRouterThreads / slices >= columns) {
            zz = fold[(columns - 1 - c0) * slices];
            n = ifold[(columns - 1 - c0) * slices];
        }
        __syncthreads();
    }
    const double per = n > 0 ? 1.0 / n : 0.0;
    double load = 0.0;
    for (int e = tid; e < E; e += kRouterThreads) {
        const float m = static_cast<float>(mean[e] * per);
        P.mean[e] = m;
        P.counts[e] = count[e];
        load += static_cast<double>(count[e]) * (mean[e] * per);
    }
    load = warp_sum(load);
    if (tid % 32 == 0) fold[tid / 32] = load;
    __syncthreads();
    if (tid == 0) {
        double all = 0.0;
        for (int w = 0; w < kRouterWarps; ++w) all += fold[w];
        P.counts[E] = n;
        P.losses[0] = static_cast<float>(static_cast<double>(P.balance_coef) * E * all * per / P.top_k);
        P.losses[1] = static_cast<float>(static_cast<double>(P.z_coef) * zz * per);
    }
}

// Softmax of a row kept by one thread: z becomes exp(z - max); false where no expert is available.
template <int N> __device__ __forceinline__ bool row_softmax(float *z, float &total, float &lse) {
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        top = fmaxf(top, z[i]);
        nan |= z[i] != z[i];
    }
    if (top == -INFINITY && !nan) return false;
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        z[i] = z[i] == -INFINITY ? 0.0f : expf(z[i] - top);
        total += z[i];
    }
    lse = logf(total) + top;
    return true;
}

// Up to 32 experts: a thread per token.
template <typename T, int N, bool kWide>
__global__ void __launch_bounds__(kRouterThreads) router_forward_thread(const __grid_constant__ RouterParams P) {
    __shared__ float sums[kRouterWarps][N];
    __shared__ int tally[kRouterWarps][N];
    __shared__ float extra[kRouterWarps];
    __shared__ int active[kRouterWarps];
    const int E = P.experts, tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    float sum[N], zsq = 0.0f;
    int cnt[N], act = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) { sum[i] = 0.0f; cnt[i] = 0; }
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRouterThreads + tid; t < P.tokens; t += static_cast<int64_t>(gridDim.x) * kRouterThreads) {
        float z[N];
        load_row<T, N, kWide>(static_cast<const T *>(P.logits) + t * P.row_stride, E, z);
        if (P.mask && P.mask[t] == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = -INFINITY;
        }
        unsigned key[N];
#pragma unroll
        for (int i = 0; i < N; ++i) key[i] = order_key(z[i]);
        float total = 1.0f, lse = 0.0f;
        const bool some = row_softmax<N>(z, total, lse);
        const float inv = some ? 1.0f / total : 0.0f;
        float share = 0.0f;
        int pick[kMaxChoice];
        float w[kMaxChoice];
#pragma unroll
        for (int j = 0; j < kMaxChoice; ++j) {
            if (j < P.top_k) {
                unsigned best = kKeyMinusInf;
                int at = -1;
                float p = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (key[i] > best) { best = key[i]; at = i; p = z[i]; }
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i == at) { key[i] = 0; ++cnt[i]; }
                pick[j] = some ? at : -1;
                w[j] = some && at >= 0 ? p * inv : 0.0f;
                share += w[j];
            }
        }
        const float norm = P.normalize ? (share != 0.0f ? share : 1.0f) : 1.0f;
#pragma unroll
        for (int j = 0; j < kMaxChoice; ++j)
            if (j < P.top_k) {
                P.index[t * P.top_k + j] = pick[j];
                P.weight[t * P.top_k + j] = w[j] / norm;
            }
        if (some) {
            ++act;
            zsq = fmaf(lse, lse, zsq);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = fmaf(z[i], inv, sum[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float s = warp_sum(sum[i]);
        const int c = __reduce_add_sync(kAll, cnt[i]);
        if (lane == 0) { sums[warp][i] = s; tally[warp][i] = c; }
    }
    zsq = warp_sum(zsq);
    act = __reduce_add_sync(kAll, act);
    if (lane == 0) { extra[warp] = zsq; active[warp] = act; }
    __syncthreads();
    if (tid < N) {
        for (int w = 1; w < kRouterWarps; ++w) { sums[0][tid] += sums[w][tid]; tally[0][tid] += tally[w][tid]; }
    }
    zsq = 0.0f;
    act = 0;
    for (int w = 0; w < kRouterWarps; ++w) { zsq += extra[w]; act += active[w]; }
    __syncthreads();
    finish(P, sums[0], tally[0], zsq, act);
}

// More experts: a warp per token, expert i * 32 + lane in the lane's i-th place.
template <int N> struct WarpRow {
    float z[N];              // logits, then exp(z - max)
    float total, lse, top;
    bool some;
};

template <typename T, int N> __device__ __forceinline__ void load_warp_row(const RouterParams &P, int64_t t, int lane, float *z) {
    const T *row = static_cast<const T *>(P.logits) + t * P.row_stride;
    const bool on = !P.mask || P.mask[t] != 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * 32 + lane;
        z[i] = on && e < P.experts ? to_f32(row[e]) : -INFINITY;
    }
}

template <int N> __device__ __forceinline__ void warp_softmax(WarpRow<N> &r) {
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        top = fmaxf(top, r.z[i]);
        nan |= r.z[i] != r.z[i];
    }
    const unsigned k = __reduce_max_sync(kAll, order_key(top));
    r.some = k > kKeyMinusInf || __any_sync(kAll, nan);
    // back from the ordered integer to the float
    r.top = k <= kKeyMinusInf ? 0.0f : __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        r.z[i] = r.z[i] == -INFINITY ? 0.0f : expf(r.z[i] - r.top);
        total += r.z[i];
    }
    r.total = warp_sum(total);
    r.lse = logf(r.total) + r.top;
}

template <typename T, int N>
__global__ void __launch_bounds__(kRouterThreads) router_forward_warp(const __grid_constant__ RouterParams P) {
    __shared__ float sums[kRouterWarps][N * 32];
    __shared__ int tally[kRouterWarps][N * 32];
    __shared__ float extra[kRouterWarps];
    __shared__ int active[kRouterWarps];
    const int E = P.experts, tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    float sum[N], zsq = 0.0f;
    int cnt[N], act = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) { sum[i] = 0.0f; cnt[i] = 0; }
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRouterWarps;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRouterWarps + warp; t < P.tokens; t += step) {
        WarpRow<N> r;
        load_warp_row<T, N>(P, t, lane, r.z);
        unsigned key[N];
#pragma unroll
        for (int i = 0; i < N; ++i) key[i] = order_key(r.z[i]);
        warp_softmax<N>(r);
        const float inv = r.some ? 1.0f / r.total : 0.0f;
        float share = 0.0f, w = 0.0f;
        int pick = -1;
        for (int j = 0; j < P.top_k; ++j) {
            unsigned best = 0;
            int at = N;
            float p = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (key[i] > best) { best = key[i]; at = i; p = r.z[i]; }
            const unsigned all = __reduce_max_sync(kAll, best);
            if (all <= kKeyMinusInf) break;
            const int e = static_cast<int>(__reduce_min_sync(kAll, best == all ? static_cast<unsigned>(at * 32 + lane) : 0xffffffffu));
            const float pe = __shfl_sync(kAll, p, e % 32) * inv;
            share += pe;
            if (lane == e % 32) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i == at) { key[i] = 0; ++cnt[i]; }
            }
            if (lane == j) { pick = e; w = pe; }
        }
        const float norm = P.normalize ? (share != 0.0f ? share : 1.0f) : 1.0f;
        if (lane < P.top_k) {
            P.index[t * P.top_k + lane] = pick;
            P.weight[t * P.top_k + lane] = w / norm;
        }
        if (r.some) {
            ++act;
            zsq = fmaf(r.lse, r.lse, zsq);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = fmaf(r.z[i], inv, sum[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) { sums[warp][i * 32 + lane] = sum[i]; tally[warp][i * 32 + lane] = cnt[i]; }
    if (lane == 0) { extra[warp] = zsq; active[warp] = act; }
    __syncthreads();
    for (int e = tid; e < E; e += kRouterThreads)
        for (int w = 1; w < kRouterWarps; ++w) { sums[0][e] += sums[w][e]; tally[0][e] += tally[w][e]; }
    zsq = 0.0f;
    act = 0;
    for (int w = 0; w < kRouterWarps; ++w) { zsq += extra[w]; act += active[w]; }
    __syncthreads();
    finish(P, sums[0], tally[0], zsq, act);
}

// dz_e = p_e (g_e - sum_j p_j g_j) + zc lse p_e + [chosen] weight gradient, g_e = d balance / d p_e

__device__ __forceinline__ float expert_gradient(const RouterParams &P, int e) {
    const int n = P.in_counts[P.experts];
    if (n <= 0 || !P.dlosses) return 0.0f;
    const float load = static_cast<float>(P.in_counts[e]) / (static_cast<float>(n) * static_cast<float>(P.top_k));
    return P.dlosses[0] * P.balance_coef * static_cast<float>(P.experts) * load / static_cast<float>(n);
}

template <typename T, int N, bool kWide>
__global__ void __launch_bounds__(kRouterThreads) router_backward_thread(const __grid_constant__ RouterParams P) {
    const int E = P.experts;
    float g[N];
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = i < E ? expert_gradient(P, i) : 0.0f;
    const int n = P.in_counts[E];
    const float zc = P.dlosses && n > 0 ? P.dlosses[1] * P.z_coef * 2.0f / static_cast<float>(n) : 0.0f;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRouterThreads + threadIdx.x; t < P.tokens; t += static_cast<int64_t>(gridDim.x) * kRouterThreads) {
        float z[N], d[N];
        load_row<T, N, kWide>(static_cast<const T *>(P.logits) + t * P.row_stride, E, z);
        float total = 1.0f, lse = 0.0f;
        const bool some = row_softmax<N>(z, total, lse) && (!P.mask || P.mask[t] != 0);
        if (some) {
            const float inv = 1.0f / total;
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                z[i] *= inv;
                dot = fmaf(z[i], g[i], dot);
            }
            if (P.dweight) {
                float share = 0.0f, wd = 0.0f;                    // sum of the chosen p, and of p * dweight
                float dw[N];
                unsigned chosen = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) dw[i] = 0.0f;
                for (int j = 0; j < P.top_k; ++j) {
                    const int e = P.in_index[t * P.top_k + j];
                    const float x = P.dweight[t * P.top_k + j];
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (i == e) {
                            dw[i] = x;
                            share += z[i];
                            wd = fmaf(z[i], x, wd);
                            chosen |= 1u << i;
                        }
                }
                const float norm = share != 0.0f ? 1.0f / share : 1.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float own = P.normalize ? ((chosen >> i) & 1 ? z[i] * norm * (dw[i] - wd * norm) : 0.0f) : z[i] * (dw[i] - wd);
                    d[i] = z[i] * (g[i] - dot + zc * lse) + own;
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] = z[i] * (g[i] - dot + zc * lse);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = 0.0f;
        }
        T *out = static_cast<T *>(P.dlogits) + t * P.drow_stride;
        if constexpr (kWide) {
            constexpr int kV = 16 / sizeof(T);
#pragma unroll
            for (int i = 0; i < N / kV; ++i)
                if (i * kV < E) {
                    Pack<T, kV> p;
#pragma unroll
                    for (int j = 0; j < kV; ++j) p.v[j] = from_f32<T>(d[i * kV + j]);
                    *reinterpret_cast<Pack<T, kV> *>(out + i * kV) = p;
                }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < E) out[i] = from_f32<T>(d[i]);
        }
    }
}

template <typename T, int N>
__global__ void __launch_bounds__(kRouterThreads) router_backward_warp(const __grid_constant__ RouterParams P) {
    const int E = P.experts, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    float g[N];
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = i * 32 + lane < E ? expert_gradient(P, i * 32 + lane) : 0.0f;
    const int n = P.in_counts[E];
    const float zc = P.dlosses && n > 0 ? P.dlosses[1] * P.z_coef * 2.0f / static_cast<float>(n) : 0.0f;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRouterWarps;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRouterWarps + warp; t < P.tokens; t += step) {
        WarpRow<N> r;
        load_warp_row<T, N>(P, t, lane, r.z);
        warp_softmax<N>(r);
        const float inv = r.some ? 1.0f / r.total : 0.0f;
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            r.z[i] *= inv;
            dot = fmaf(r.z[i], g[i], dot);
        }
        dot = warp_sum(dot);
        const float common = r.some ? zc * r.lse - dot : 0.0f;
        float add[N], wd = 0.0f, share = 1.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) add[i] = 0.0f;
        if (P.dweight && r.some) {
            // the lane's own choice, for the two sums
            const int e = lane < P.top_k ? P.in_index[t * P.top_k + lane] : -1;
            const float x = e >= 0 ? P.dweight[t * P.top_k + lane] : 0.0f;
            share = 0.0f;
            for (int j = 0; j < P.top_k; ++j) {
                const int ej = __shfl_sync(kAll, e, j);
                const float xj = __shfl_sync(kAll, x, j);
                if (ej >= 0 && lane == ej % 32) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (i == ej / 32) {
                            add[i] = xj;
                            share += r.z[i];
                            wd = fmaf(r.z[i], xj, wd);
                        }
                }
            }
            share = warp_sum(share);
            wd = warp_sum(wd);
            const float norm = share != 0.0f ? 1.0f / share : 1.0f;
            if (P.normalize) {
                for (int j = 0; j < P.top_k; ++j) {
                    const int ej = __shfl_sync(kAll, e, j);
                    if (ej >= 0 && lane == ej % 32) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (i == ej / 32) add[i] = r.z[i] * norm * (add[i] - wd * norm);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) add[i] = r.z[i] * (add[i] - wd);
            }
        }
        T *out = static_cast<T *>(P.dlogits) + t * P.drow_stride;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * 32 + lane < E) out[i * 32 + lane] = from_f32<T>(r.z[i] * (g[i] + common) + add[i]);
    }
}

template <typename T> void launch_forward(const RouterParams &P, unsigned blocks, bool wide, cudaStream_t s) {
    const int E = P.experts;
    if (E <= 8) wide ? router_forward_thread<T, 8, true><<<blocks, kRouterThreads, 0, s>>>(P) : router_forward_thread<T, 8, false><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 16) wide ? router_forward_thread<T, 16, true><<<blocks, kRouterThreads, 0, s>>>(P) : router_forward_thread<T, 16, false><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 64) router_forward_warp<T, 2><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 128) router_forward_warp<T, 4><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 192) router_forward_warp<T, 6><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 256) router_forward_warp<T, 8><<<blocks, kRouterThreads, 0, s>>>(P);
    else router_forward_warp<T, 16><<<blocks, kRouterThreads, 0, s>>>(P);
}

template <typename T> void launch_backward(const RouterParams &P, unsigned blocks, bool wide, cudaStream_t s) {
    const int E = P.experts;
    if (E <= 8) wide ? router_backward_thread<T, 8, true><<<blocks, kRouterThreads, 0, s>>>(P) : router_backward_thread<T, 8, false><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 16) wide ? router_backward_thread<T, 16, true><<<blocks, kRouterThreads, 0, s>>>(P) : router_backward_thread<T, 16, false><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 64) router_backward_warp<T, 2><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 128) router_backward_warp<T, 4><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 192) router_backward_warp<T, 6><<<blocks, kRouterThreads, 0, s>>>(P);
    else if (E <= 256) router_backward_warp<T, 8><<<blocks, kRouterThreads, 0, s>>>(P);
    else router_backward_warp<T, 16><<<blocks, kRouterThreads, 0, s>>>(P);
}

int check_router(const loco_router_t *c) {
    if (!c) return LOCO_ERR_ARG;
    if (c->dtype != LOCO_F32 && c->dtype != LOCO_BF16) return LOCO_ERR_ARG;
    if (c->experts < 1 || c->experts > kMaxExperts) return LOCO_ERR_ARG;
    if (c->top_k < 1 || c->top_k > kMaxChoice || c->top_k > c->experts) return LOCO_ERR_ARG;
    if (!std::isfinite(c->balance_coef) || !std::isfinite(c->z_coef)) return LOCO_ERR_ARG;
    return LOCO_OK;
}

// Blocks of a launch: tokens per block of the kernel the number of experts selects, at most what the machine holds.
int64_t router_blocks(const loco_router_t *c, int64_t tokens, int most) {
    const int64_t per = c->experts <= 16 ? kRouterThreads : kRouterWarps;
    const int64_t need = (tokens + per - 1) / per;
    return need < most ? (need < 1 ? 1 : need) : most;
}

}  // namespace loco_layer

using namespace loco_layer;

extern "C" {

uint64_t loco_router_workspace_bytes(const loco_router_t *c) {
    if (check_router(c) != LOCO_OK) return 0;
    return 256 + static_cast<uint64_t>(kMaxBlocks) * (2 * c->experts + 2) * 4;
}

int loco_router_forward(const loco_router_t *c, int64_t tokens, const void *d_logits, int64_t row_stride, const uint8_t *d_mask,
                        int32_t *d_index, float *d_weight, int32_t *d_counts, float *d_mean, float *d_losses, void *d_work,
                        uint64_t d_work_bytes, void *stream) {
    const int rc = check_router(c);
    if (rc != LOCO_OK) return rc;
    if (tokens < 0 || tokens * c->top_k > 0x7fffffff) return LOCO_ERR_ARG;
    if (!d_counts || !d_mean || !d_losses || !d_work || (tokens > 0 && (!d_logits || !d_index || !d_weight))) return LOCO_ERR_ARG;
    const uintptr_t size = c->dtype == LOCO_BF16 ? 2 : 4;
    if (!aligned(d_logits, size) || !aligned(d_index, 4) || !aligned(d_weight, 4) || !aligned(d_counts, 4) || !aligned(d_mean, 4) ||
        !aligned(d_losses, 4) || !aligned(d_work, 16)) return LOCO_ERR_ALIGN;
    if (d_work_bytes < loco_router_workspace_bytes(c)) return LOCO_ERR_SIZE;
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    RouterParams P{};
    P.logits = d_logits;
    P.row_stride = row_stride;
    P.mask = d_mask;
    P.index = d_index;
    P.weight = d_weight;
    P.counts = d_counts;
    P.mean = d_mean;
    P.losses = d_losses;
    P.ticket = static_cast<unsigned *>(d_work);
    P.part = reinterpret_cast<float *>(static_cast<uint8_t *>(d_work) + 256);
    P.tokens = tokens;
    P.experts = c->experts;
    P.top_k = c->top_k;
    P.normalize = c->normalize;
    P.balance_coef = c->balance_coef;
    P.z_coef = c->z_coef;
    const int most = sms * kBlocksPerSm < kMaxBlocks ? sms * kBlocksPerSm : kMaxBlocks;
    const unsigned blocks = static_cast<unsigned>(router_blocks(c, tokens, most));
    // rows that are whole 16-byte vectors on 16-byte boundaries are read as such
    const int vec = 16 / static_cast<int>(size);
    const bool wide = aligned(d_logits, 16) && row_stride % vec == 0 && c->experts % vec == 0;
    if (c->dtype == LOCO_BF16) launch_forward<__nv_bfloat16>(P, blocks, wide, static_cast<cudaStream_t>(stream));
    else launch_forward<float>(P, blocks, wide, static_cast<cudaStream_t>(stream));
    return launched();
}

int loco_router_backward(const loco_router_t *c, int64_t tokens, const void *d_logits, int64_t row_stride, const uint8_t *d_mask,
                         const int32_t *d_index, const int32_t *d_counts, const float *d_dlosses, const float *d_dweight,
                         void *d_dlogits, int64_t drow_stride, void *stream) {
    const int rc = check_router(c);
    if (rc != LOCO_OK) return rc;
    if (tokens < 0 || tokens * c->top_k > 0x7fffffff) return LOCO_ERR_ARG;
    if (tokens == 0) return LOCO_OK;
    if (!d_logits || !d_index || !d_counts || !d_dlogits) return LOCO_ERR_ARG;
    const uintptr_t size = c->dtype == LOCO_BF16 ? 2 : 4;
    if (!aligned(d_logits, size) || !aligned(d_dlogits, size) || !aligned(d_index, 4) || !aligned(d_counts, 4) ||
        !aligned(d_dlosses, 4) || !aligned(d_dweight, 4)) return LOCO_ERR_ALIGN;
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    RouterParams P{};
    P.logits = d_logits;
    P.row_stride = row_stride;
    P.mask = d_mask;
    P.in_index = d_index;
    P.in_counts = d_counts;
    P.dlosses = d_dlosses;
    P.dweight = d_dweight;
    P.dlogits = d_dlogits;
    P.drow_stride = drow_stride;
    P.tokens = tokens;
    P.experts = c->experts;
    P.top_k = c->top_k;
    P.normalize = c->normalize;
    P.balance_coef = c->balance_coef;
    P.z_coef = c->z_coef;
    const int vec = 16 / static_cast<int>(size);
    const bool wide = aligned(d_logits, 16) && aligned(d_dlogits, 16) && row_stride % vec == 0 && drow_stride % vec == 0 && c->experts % vec == 0;
    const unsigned blocks = static_cast<unsigned>(router_blocks(c, tokens, sms * 8));
    if (c->dtype == LOCO_BF16) launch_backward<__nv_bfloat16>(P, blocks, wide, static_cast<cudaStream_t>(stream));
    else launch_backward<float>(P, blocks, wide, static_cast<cudaStream_t>(stream));
    return launched();
}

}  // extern "C"
