// Rotary positions: one streaming pass over query and key heads.
//
// y_a = x_a c - x_b s, y_b = x_b c + x_a s: three operations per element read and written, so the bound is HBM.  A thread
// owns one vector of pairs of a token and walks over `kHeads` heads with the pairs' cosines and sines in registers: the
// table is then read once per token and head group (from L2) instead of once per head, and the loads of all heads are in
// flight together.
#include "layer_common.h"

namespace loco_layer {

std::atomic<uint64_t> g_launches{0};

int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return 0;
    }
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
            cudaGetLastError();
            return 0;
        }
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

struct RotaryTensor {
    const void *x;
    void *y;
    int64_t xb, xr, xh, yb, yr, yh;
    uint32_t heads, groups;
};

struct RotaryParams {
    RotaryTensor t[2];
    const float *table;
    const void *positions;
    int64_t items;
    uint32_t seq, vecs, vecs_turned, groups;
    int32_t rotary_dim, rows, wide_positions;
    float sign;                            // of the sine: -1 for the transposed rotation
};

constexpr int kRotaryThreads = 256;

// By ordinary loads: the launch before, which may have written the table, need not have ended when this one starts.
template <int N> __device__ __forceinline__ void load_floats(const float *p, float *out) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 f = reinterpret_cast<const float4 *>(p)[i];
            out[4 * i] = f.x; out[4 * i + 1] = f.y; out[4 * i + 2] = f.z; out[4 * i + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = p[i];
    }
}

// kVec elements of T per access (1: no alignment needed), kHeads heads per thread.
template <typename T, bool kHalf, int kVec, int kHeads>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const __grid_constant__ RotaryParams P) {
    wait_for_previous();
    let_next_start();
    const int64_t item64 = static_cast<int64_t>(blockIdx.x) * kRotaryThreads + threadIdx.x;
    if (item64 >= P.items) return;
    const uint32_t per_token = P.vecs * P.groups;
    const uint32_t token = static_cast<uint32_t>(P.items <= 0xffffffffll ? static_cast<uint32_t>(item64) / per_token
                                                                         : item64 / per_token);
    const uint32_t rest = static_cast<uint32_t>(item64 - static_cast<int64_t>(token) * per_token);
    uint32_t group = rest / P.vecs;
    const uint32_t vec = rest - group * P.vecs;
    const uint32_t b = token / P.seq, row = token - b * P.seq;
    const RotaryTensor &t = group < P.t[0].groups ? P.t[0] : P.t[1];
    if (group >= P.t[0].groups) group -= P.t[0].groups;
    const uint32_t h0 = group * kHeads;
    const T *x = static_cast<const T *>(t.x) + b * t.xb + row * t.xr + h0 * t.xh;
    T *y = static_cast<T *>(t.y) + b * t.yb + row * t.yr + h0 * t.yh;
    const int heads = min(kHeads, static_cast<int>(t.heads - h0));
    using V = Pack<T, kVec>;
    if (vec >= P.vecs_turned) {            // dimensions that are not rotated
        if (x == y) return;
        const int at = P.rotary_dim + static_cast<int>(vec - P.vecs_turned) * kVec;
        V in[kHeads];
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
            if (h < heads) in[h] = *reinterpret_cast<const V *>(x + h * t.xh + at);
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
            if (h < heads) *reinterpret_cast<V *>(y + h * t.yh + at) = in[h];
        return;
    }
    int64_t pos = row;
    if (P.positions)
        pos = P.wide_positions ? static_cast<const int64_t *>(P.positions)[token] : static_cast<const int32_t *>(P.positions)[token];
    const bool inside = pos >= 0 && pos < P.rows;
    const int half = P.rotary_dim / 2;
    // the pairs of this thread: in the half layout vectors at `at` and `at + half`, else neighbours within one or two vectors
    constexpr int kPairs = kHalf ? kVec : (kVec > 1 ? kVec / 2 : 1);
    constexpr bool kTwo = kHalf || kVec == 1;
    const int pair = static_cast<int>(vec) * kPairs;
    const int at = kHalf ? pair : 2 * pair;
    const int second = kHalf ? half : 1;
    float c[kPairs], s[kPairs];
    const float *table = P.table + (inside ? pos : 0) * P.rotary_dim + pair;
    load_floats<kPairs>(table, c);
    load_floats<kPairs>(table + half, s);
    const float bad = __int_as_float(0x7fffffff);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        c[i] = inside ? c[i] : bad;
        s[i] = inside ? s[i] * P.sign : bad;
    }
    V in[kHeads][kTwo ? 2 : 1];
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
        if (h < heads) {
            in[h][0] = *reinterpret_cast<const V *>(x + h * t.xh + at);
            if constexpr (kTwo) in[h][1] = *reinterpret_cast<const V *>(x + h * t.xh + at + second);
        }
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
        if (h < heads) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                T &pa = kTwo ? in[h][0].v[i] : in[h][0].v[(2 * i) % kVec];
                T &pb = kTwo ? in[h][kTwo ? 1 : 0].v[i] : in[h][0].v[(2 * i + 1) % kVec];
                const float a = to_f32(pa), bb = to_f32(pb);
                pa = from_f32<T>(a * c[i] - bb * s[i]);
                pb = from_f32<T>(bb * c[i] + a * s[i]);
            }
            *reinterpret_cast<V *>(y + h * t.yh + at) = in[h][0];
            if constexpr (kTwo) *reinterpret_cast<V *>(y + h * t.yh + at + second) = in[h][1];
        }
}

// cos and sin of p w_j in 64 bits; a row per p.
__global__ void rotary_table_kernel(float *table, const loco_rotary_table_t c) {
    wait_for_previous();
    let_next_start();
    const int half = c.rotary_dim / 2;
    const int64_t n = static_cast<int64_t>(c.positions) * half;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const int64_t p = i / half;
        const int j = static_cast<int>(i - p * half);
        double w = pow(static_cast<double>(c.base), -2.0 * j / c.rotary_dim);
        if (c.scaling == LOCO_ROTARY_LINEAR) {
            w /= c.factor;
        } else if (c.scaling == LOCO_ROTARY_PARTS) {
            const double turns = c.trained * w / 6.283185307179586476925286766559;
            const double keep = fmin(fmax((turns - c.slow) / (static_cast<double>(c.fast) - c.slow), 0.0), 1.0);
            w = w / c.factor * (1.0 - keep) + w * keep;
        }
        double s, co;
        sincos(static_cast<double>(p) * w, &s, &co);
        table[p * c.rotary_dim + j] = static_cast<float>(co * c.magnitude);
        table[p * c.rotary_dim + half + j] = static_cast<float>(s * c.magnitude);
    }
}

template <typename T, bool kHalf, int kVec>
int launch_rotary(RotaryParams &P, int64_t tokens, void *stream) {
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    const auto fill = [&](uint32_t per) {
        for (auto &t : P.t) t.groups = (t.heads + per - 1) / per;
        P.groups = P.t[0].groups + P.t[1].groups;
        P.items = tokens * P.vecs * P.groups;
    };
    // Several heads per thread only where that still leaves every SM its 2048 threads.
    fill(4);
    const bool many = P.items >= static_cast<int64_t>(sms) * 2048;
    if (!many) fill(1);
    const int64_t blocks = (P.items + kRotaryThreads - 1) / kRotaryThreads;
    if (blocks > 0x7fffffff) return LOCO_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(blocks));
    return launch_kernel(many ? rotary_kernel<T, kHalf, kVec, 4> : rotary_kernel<T, kHalf, kVec, 1>, grid, kRotaryThreads, 0, stream, P);
}

}  // namespace loco_layer

using namespace loco_layer;

extern "C" {

uint64_t loco_layer_launch_count(void) { return g_launches.load(); }

int loco_rotary_table(const loco_rotary_table_t *c, float *d_table, void *stream) {
    if (!c || !d_table) return LOCO_ERR_ARG;
    if (c->rotary_dim < 2 || c->rotary_dim > 1024 || c->rotary_dim % 2 || c->positions < 1) return LOCO_ERR_ARG;
    if (c->scaling < LOCO_ROTARY_PLAIN || c->scaling > LOCO_ROTARY_PARTS) return LOCO_ERR_ARG;
    if (!(c->base > 0.0f) || !std::isfinite(c->base) || !std::isfinite(c->magnitude)) return LOCO_ERR_ARG;
    if (c->scaling != LOCO_ROTARY_PLAIN && (!(c->factor > 0.0f) || !std::isfinite(c->factor))) return LOCO_ERR_ARG;
    if (c->scaling == LOCO_ROTARY_PARTS && (!(c->trained > 0.0f) || !std::isfinite(c->trained) || !(c->slow >= 0.0f) ||
                                            !(c->fast > c->slow) || !std::isfinite(c->fast))) return LOCO_ERR_ARG;
    if (!aligned(d_table, 16)) return LOCO_ERR_ALIGN;
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    const int64_t n = static_cast<int64_t>(c->positions) * (c->rotary_dim / 2);
    const int64_t blocks = (n + 255) / 256;
    return launch_kernel(rotary_table_kernel, dim3(static_cast<unsigned>(blocks < sms * 8 ? blocks : sms * 8)), 256, 0, stream, d_table, *c);
}

int loco_rotary_apply(const loco_rotary_t *c, const float *d_table, const void *d_positions, const loco_heads_t *x,
                      const loco_heads_t *y, const int32_t *heads, int32_t count, void *stream) {
    if (!c || count < 1 || count > 2 || !x || !y || !heads) return LOCO_ERR_ARG;
    if (c->dtype != LOCO_F32 && c->dtype != LOCO_BF16) return LOCO_ERR_ARG;
    if (c->layout != LOCO_ROTARY_HALF && c->layout != LOCO_ROTARY_INTERLEAVED) return LOCO_ERR_ARG;
    if (c->head_dim < 1 || c->head_dim > 1024 || c->rotary_dim < 2 || c->rotary_dim > c->head_dim || c->rotary_dim % 2)
        return LOCO_ERR_ARG;
    if (c->batch < 0 || c->seq < 0 || c->positions < 1) return LOCO_ERR_ARG;
    if (d_positions && c->position_bytes != 4 && c->position_bytes != 8) return LOCO_ERR_ARG;
    if (!d_positions && c->seq > c->positions) return LOCO_ERR_ARG;
    const int64_t tokens = static_cast<int64_t>(c->batch) * c->seq;
    if (tokens > 0x7fffffff) return LOCO_ERR_ARG;
    for (int i = 0; i < count; ++i)
        if (heads[i] < 0 || heads[i] > 65536) return LOCO_ERR_ARG;
    if (tokens == 0 || (heads[0] == 0 && (count == 1 || heads[1] == 0))) return LOCO_OK;
    if (!d_table) return LOCO_ERR_ARG;
    if (!aligned(d_table, 16) || (d_positions && !aligned(d_positions, static_cast<uintptr_t>(c->position_bytes)))) return LOCO_ERR_ALIGN;
    const int size = c->dtype == LOCO_BF16 ? 2 : 4, vec = 16 / size;
    const bool half = c->layout == LOCO_ROTARY_HALF;
    // 16-byte accesses where every vector of every head starts on a 16-byte boundary and none straddles the two halves
    // or the end of the rotated part; element accesses otherwise.
    bool wide = (half ? c->rotary_dim / 2 : c->rotary_dim) % vec == 0 && c->head_dim % vec == 0 && c->rotary_dim % vec == 0;
    RotaryParams P{};
    for (int i = 0; i < count; ++i) {
        if (heads[i] == 0) continue;
        if (!x[i].ptr || !y[i].ptr) return LOCO_ERR_ARG;
        if (!aligned(x[i].ptr, static_cast<uintptr_t>(size)) || !aligned(y[i].ptr, static_cast<uintptr_t>(size))) return LOCO_ERR_ALIGN;
        RotaryTensor &t = P.t[i];
        t = RotaryTensor{x[i].ptr, y[i].ptr, x[i].batch_stride, x[i].row_stride, x[i].head_stride,
                         y[i].batch_stride, y[i].row_stride, y[i].head_stride, static_cast<uint32_t>(heads[i]), 0};
        if (c->batch == 1) t.xb = t.yb = 0;              // the stride of a dimension of extent one means nothing
        if (c->seq == 1) t.xr = t.yr = 0;
        if (heads[i] == 1) t.xh = t.yh = 0;
        // zero strides repeat what is read; nothing that is written may be repeated
        if ((c->batch > 1 && t.yb == 0) || (c->seq > 1 && t.yr == 0) || (heads[i] > 1 && t.yh == 0)) return LOCO_ERR_ARG;
        wide = wide && aligned(t.x, 16) && aligned(t.y, 16);
        for (int64_t s : {t.xb, t.xr, t.xh, t.yb, t.yr, t.yh}) wide = wide && s % vec == 0;
    }
    P.table = d_table;
    P.positions = d_positions;
    P.seq = static_cast<uint32_t>(c->seq);
    P.rotary_dim = c->rotary_dim;
    P.rows = c->positions;
    P.wide_positions = c->position_bytes == 8;
    P.sign = c->inverse ? -1.0f : 1.0f;
    const int v = wide ? vec : 1;
    P.vecs_turned = static_cast<uint32_t>(half || !wide ? c->rotary_dim / 2 / v : c->rotary_dim / v);
    P.vecs = P.vecs_turned + static_cast<uint32_t>((c->head_dim - c->rotary_dim) / v);
    if (c->dtype == LOCO_BF16) {
        if (half) return wide ? launch_rotary<__nv_bfloat16, true, 8>(P, tokens, stream) : launch_rotary<__nv_bfloat16, true, 1>(P, tokens, stream);
        return wide ? launch_rotary<__nv_bfloat16, false, 8>(P, tokens, stream) : launch_rotary<__nv_bfloat16, false, 1>(P, tokens, stream);
    }
    if (half) return wide ? launch_rotary<float, true, 4>(P, tokens, stream) : launch_rotary<float, true, 1>(P, tokens, stream);
    return wide ? launch_rotary<float, false, 4>(P, tokens, stream) : launch_rotary<float, false, 1>(P, tokens, stream);
}

}  // extern "C"
