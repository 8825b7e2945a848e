// Arguments of the attention kernels and the geometry of a sample.
#pragma once
#include "layer_common.h"

namespace loco_layer {

struct Heads {
    __nv_bfloat16 *ptr;
    int64_t batch_stride, row_stride, head_stride;
};

struct AttentionParams {
    Heads q, k, v, o, d_o, dq, dk, dv;
    float *lse;
    float *row_dot;                   // D_i, laid out as lse
    const int32_t *len_q, *len_k;
    int32_t batch, heads_q, heads_kv, group, head_dim, packed, seq_q, seq_k, max_q, max_k, causal;
    int32_t span;                     // heads (of samples) whose blocks come together
    float scale;
};

// One sample's rows: `first` + i inside the tensor's rows of batch `at`; n of them take part.
struct Rows {
    int at, first, n;
};

__device__ __forceinline__ Rows sample_rows(const int32_t *len, int packed, int seq, int most, int b) {
    if (packed) {                     // offsets are clamped to the tensor, whatever they hold
        const int lo = min(max(len[b], 0), seq), hi = min(max(len[b + 1], lo), seq);
        return Rows{0, lo, min(hi - lo, most)};
    }
    return Rows{b, 0, len ? min(max(len[b], 0), seq) : seq};
}
__device__ __forceinline__ Rows query_rows(const AttentionParams &P, int b) { return sample_rows(P.len_q, P.packed, P.seq_q, P.max_q, b); }
__device__ __forceinline__ Rows key_rows(const AttentionParams &P, int b) { return sample_rows(P.len_k, P.packed, P.seq_k, P.max_k, b); }

__device__ __forceinline__ __nv_bfloat16 *row_of(const Heads &t, const Rows &r, int i, int h) {
    return t.ptr + r.at * t.batch_stride + (static_cast<int64_t>(r.first) + i) * t.row_stride + h * t.head_stride;
}
// Where row i of head h has its log-sum-exp.
__device__ __forceinline__ int64_t stat_at(const AttentionParams &P, const Rows &r, int i, int h) {
    return (static_cast<int64_t>(r.at) * P.heads_q + h) * P.seq_q + r.first + i;
}

int launch_attention_forward(const AttentionParams &P, cudaStream_t stream);
int launch_attention_backward(const AttentionParams &P, cudaStream_t stream);

}  // namespace loco_layer
