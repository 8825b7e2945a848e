// Attention, one warp per row: every sum in fp32, four dimensions of the head per lane.
#include "layer_attention.h"

namespace loco_layer {

constexpr int kAttnWarps = 8;

__device__ __forceinline__ float warp_total(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

struct Four { float v[4]; };
__device__ __forceinline__ Four load4(const __nv_bfloat16 *row, int lane, int d) {
    Four f{{0.0f, 0.0f, 0.0f, 0.0f}};
    if (lane * 4 < d) {
        const Pack<__nv_bfloat16, 4> p = *reinterpret_cast<const Pack<__nv_bfloat16, 4> *>(row + lane * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) f.v[i] = __bfloat162float(p.v[i]);
    }
    return f;
}
__device__ __forceinline__ void store4(__nv_bfloat16 *row, int lane, int d, const Four &f) {
    if (lane * 4 < d) {
        Pack<__nv_bfloat16, 4> p;
#pragma unroll
        for (int i = 0; i < 4; ++i) p.v[i] = __float2bfloat16_rn(f.v[i]);
        *reinterpret_cast<Pack<__nv_bfloat16, 4> *>(row + lane * 4) = p;
    }
}
__device__ __forceinline__ float dot4(const Four &a, const Four &b) {
    return warp_total(a.v[0] * b.v[0] + a.v[1] * b.v[1] + a.v[2] * b.v[2] + a.v[3] * b.v[3]);
}
__device__ __forceinline__ void add4(Four &a, float w, const Four &b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a.v[i] = fmaf(w, b.v[i], a.v[i]);
}

struct Place { int b, h, i; };
__device__ __forceinline__ Place place(int rows, int heads) {
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kAttnWarps + threadIdx.x / 32;
    const int64_t bh = r / rows;
    return Place{static_cast<int>(bh / heads), static_cast<int>(bh % heads), static_cast<int>(r - bh * rows)};
}

__global__ void __launch_bounds__(kAttnWarps * 32) attention_forward_rows(const __grid_constant__ AttentionParams P) {
    const Place at = place(P.max_q, P.heads_q);
    if (at.b >= P.batch) return;
    const int lane = threadIdx.x % 32, d = P.head_dim;
    const Rows Q = query_rows(P, at.b), K = key_rows(P, at.b);
    if (at.i >= Q.n && P.packed) return;
    const int see = at.i >= Q.n ? 0 : (P.causal ? min(K.n, at.i + K.n - Q.n + 1) : K.n);
    Four o{{0.0f, 0.0f, 0.0f, 0.0f}};
    float top = -INFINITY, total = 0.0f;
    if (see > 0) {
        const Four q = load4(row_of(P.q, Q, at.i, at.h), lane, d);
        for (int j = 0; j < see; ++j) {
            const float s = dot4(q, load4(row_of(P.k, K, j, at.h / P.group), lane, d)) * P.scale;
            const float next = fmaxf(top, s), fade = top == -INFINITY ? 0.0f : expf(top - next), p = expf(s - next);
            total = fmaf(total, fade, p);
#pragma unroll
            for (int i = 0; i < 4; ++i) o.v[i] *= fade;
            add4(o, p, load4(row_of(P.v, K, j, at.h / P.group), lane, d));
            top = next;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o.v[i] /= total;
    }
    store4(row_of(P.o, Q, at.i, at.h), lane, d, o);
    if (lane == 0) P.lse[stat_at(P, Q, at.i, at.h)] = see > 0 ? logf(total) + top : -INFINITY;
}

__global__ void __launch_bounds__(kAttnWarps * 32) attention_backward_queries(const __grid_constant__ AttentionParams P) {
    const Place at = place(P.max_q, P.heads_q);
    if (at.b >= P.batch) return;
    const int lane = threadIdx.x % 32, d = P.head_dim;
    const Rows Q = query_rows(P, at.b), K = key_rows(P, at.b);
    if (at.i >= Q.n && P.packed) return;
    const int see = at.i >= Q.n ? 0 : (P.causal ? min(K.n, at.i + K.n - Q.n + 1) : K.n);
    Four dq{{0.0f, 0.0f, 0.0f, 0.0f}};
    float dot = 0.0f;
    if (see > 0) {
        const Four q = load4(row_of(P.q, Q, at.i, at.h), lane, d), go = load4(row_of(P.d_o, Q, at.i, at.h), lane, d);
        dot = dot4(go, load4(row_of(P.o, Q, at.i, at.h), lane, d));
        const float lse = P.lse[stat_at(P, Q, at.i, at.h)];
        for (int j = 0; j < see; ++j) {
            const Four k = load4(row_of(P.k, K, j, at.h / P.group), lane, d);
            const float p = expf(dot4(q, k) * P.scale - lse);
            add4(dq, p * (dot4(go, load4(row_of(P.v, K, j, at.h / P.group), lane, d)) - dot), k);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) dq.v[i] *= P.scale;
    }
    store4(row_of(P.dq, Q, at.i, at.h), lane, d, dq);
    if (lane == 0) P.row_dot[stat_at(P, Q, at.i, at.h)] = dot;
}

__global__ void __launch_bounds__(kAttnWarps * 32) attention_backward_keys(const __grid_constant__ AttentionParams P) {
    const Place at = place(P.max_k, P.heads_kv);
    if (at.b >= P.batch) return;
    const int lane = threadIdx.x % 32, d = P.head_dim;
    const Rows Q = query_rows(P, at.b), K = key_rows(P, at.b);
    if (at.i >= K.n && P.packed) return;
    Four dk{{0.0f, 0.0f, 0.0f, 0.0f}}, dv = dk;
    if (at.i < K.n) {
        const Four k = load4(row_of(P.k, K, at.i, at.h), lane, d), v = load4(row_of(P.v, K, at.i, at.h), lane, d);
        const int from = P.causal ? max(0, at.i - (K.n - Q.n)) : 0;
        for (int g = 0; g < P.group; ++g) {
            const int h = at.h * P.group + g;
            for (int i = from; i < Q.n; ++i) {
                const Four q = load4(row_of(P.q, Q, i, h), lane, d), go = load4(row_of(P.d_o, Q, i, h), lane, d);
                const int64_t s = stat_at(P, Q, i, h);
                const float p = expf(dot4(q, k) * P.scale - P.lse[s]);
                add4(dv, p, go);
                add4(dk, p * (dot4(go, v) - P.row_dot[s]), q);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) dk.v[i] *= P.scale;
    }
    store4(row_of(P.dk, K, at.i, at.h), lane, d, dk);
    store4(row_of(P.dv, K, at.i, at.h), lane, d, dv);
}

static unsigned row_blocks(int64_t batch, int64_t heads, int64_t rows) {
    const int64_t n = (batch * heads * rows + kAttnWarps - 1) / kAttnWarps;
    return n > 0x7fffffff ? 0u : static_cast<unsigned>(n);
}

int launch_attention_forward(const AttentionParams &P, cudaStream_t stream) {
    if (P.max_q == 0) return LOCO_OK;
    const unsigned n = row_blocks(P.batch, P.heads_q, P.max_q);
    if (!n) return LOCO_ERR_UNSUPPORTED;
    attention_forward_rows<<<n, kAttnWarps * 32, 0, stream>>>(P);
    return launched();
}

int launch_attention_backward(const AttentionParams &P, cudaStream_t stream) {
    if (P.max_q > 0) {
        const unsigned n = row_blocks(P.batch, P.heads_q, P.max_q);
        if (!n) return LOCO_ERR_UNSUPPORTED;
        attention_backward_queries<<<n, kAttnWarps * 32, 0, stream>>>(P);
        const int rc = launched();
        if (rc != LOCO_OK) return rc;
    }
    if (P.max_k > 0) {
        const unsigned n = row_blocks(P.batch, P.heads_kv, P.max_k);
        if (!n) return LOCO_ERR_UNSUPPORTED;
        attention_backward_keys<<<n, kAttnWarps * 32, 0, stream>>>(P);
        return launched();
    }
    return LOCO_OK;
}

}  // namespace loco_layer
