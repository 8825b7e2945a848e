// C ABI of the attention operators: checks of the arguments, then one or two launches.
#include "layer_attention.h"

using namespace loco_layer;

namespace {

int check_attention(const loco_attention_t *c) {
    if (!c) return LOCO_ERR_ARG;
    if (c->batch < 0 || c->heads_q < 1 || c->heads_kv < 1 || c->heads_q % c->heads_kv) return LOCO_ERR_ARG;
    if (c->head_dim < 1 || c->seq_q < 0 || c->seq_k < 0 || !std::isfinite(c->scale)) return LOCO_ERR_ARG;
    if (c->packed && (c->max_q < 0 || c->max_k < 0 || c->max_q > c->seq_q || c->max_k > c->seq_k || !c->d_len_q || !c->d_len_k))
        return LOCO_ERR_ARG;
    if (c->head_dim > 128 || c->head_dim % 8) return LOCO_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(c->batch) * c->heads_q > 0x7fffffff) return LOCO_ERR_UNSUPPORTED;      // blocks and rows stay within 64 bits
    if (!aligned(c->d_len_q, 4) || !aligned(c->d_len_k, 4)) return LOCO_ERR_ALIGN;
    return LOCO_OK;
}

// An operand with rows: present, on 16-byte boundaries, strides of whole 16-byte units and none negative.  The stride of a
// dimension of extent one means nothing.  Zero strides repeat what is read; nothing that is written may be repeated.
int take(const loco_attention_t *c, const loco_heads_t *t, int32_t heads, int32_t rows, Heads &out, bool written = false) {
    if (!t) return LOCO_ERR_ARG;
    const int64_t b = c->packed || c->batch <= 1 ? 0 : t->batch_stride, r = rows <= 1 ? 0 : t->row_stride, h = heads <= 1 ? 0 : t->head_stride;
    out = Heads{static_cast<__nv_bfloat16 *>(t->ptr), b, r, h};
    if (rows == 0 || c->batch == 0) return LOCO_OK;
    if (!t->ptr || b < 0 || r < 0 || h < 0) return LOCO_ERR_ARG;
    if (written && ((!c->packed && c->batch > 1 && b == 0) || (rows > 1 && r == 0) || (heads > 1 && h == 0))) return LOCO_ERR_ARG;
    if (!aligned(t->ptr, 16) || b % 8 || r % 8 || h % 8) return LOCO_ERR_ALIGN;
    return LOCO_OK;
}

int fill(const loco_attention_t *c, AttentionParams &P) {
    const int rc = check_attention(c);
    if (rc != LOCO_OK) return rc;
    P.len_q = c->d_len_q;
    P.len_k = c->d_len_k;
    P.batch = c->batch;
    P.heads_q = c->heads_q;
    P.heads_kv = c->heads_kv;
    P.group = c->heads_q / c->heads_kv;
    P.head_dim = c->head_dim;
    P.packed = c->packed != 0;
    P.seq_q = c->seq_q;
    P.seq_k = c->seq_k;
    P.max_q = c->packed ? c->max_q : c->seq_q;
    P.max_k = c->packed ? c->max_k : c->seq_k;
    P.causal = c->causal != 0;
    P.scale = c->scale;
    return LOCO_OK;
}

int64_t rows_of(const loco_attention_t *c, int32_t seq) { return static_cast<int64_t>(c->packed ? (c->batch > 0) : c->batch) * seq; }

}  // namespace

extern "C" {

int loco_attention_forward(const loco_attention_t *c, const loco_heads_t *q, const loco_heads_t *k, const loco_heads_t *v,
                           const loco_heads_t *o, float *d_lse, void *stream) {
    AttentionParams P{};
    int rc = fill(c, P);
    const int64_t nq = rc == LOCO_OK ? rows_of(c, c->seq_q) : 0, nk = rc == LOCO_OK ? rows_of(c, c->seq_k) : 0;
    if (rc == LOCO_OK) rc = take(c, q, c->heads_q, c->seq_q, P.q);
    if (rc == LOCO_OK) rc = take(c, k, c->heads_kv, c->seq_k, P.k);
    if (rc == LOCO_OK) rc = take(c, v, c->heads_kv, c->seq_k, P.v);
    if (rc == LOCO_OK) rc = take(c, o, c->heads_q, c->seq_q, P.o, true);
    if (rc != LOCO_OK) return rc;
    if (nq == 0) return LOCO_OK;
    if (!d_lse) return LOCO_ERR_ARG;
    if (!aligned(d_lse, 4)) return LOCO_ERR_ALIGN;
    P.lse = d_lse;
    return launch_attention_forward(P, static_cast<cudaStream_t>(stream));
}

uint64_t loco_attention_backward_workspace_bytes(const loco_attention_t *c) {
    if (check_attention(c) != LOCO_OK) return 0;
    return static_cast<uint64_t>(rows_of(c, c->seq_q)) * c->heads_q * 4 + 256;
}

int loco_attention_backward(const loco_attention_t *c, const loco_heads_t *q, const loco_heads_t *k, const loco_heads_t *v,
                            const loco_heads_t *o, const float *d_lse, const loco_heads_t *d_o, const loco_heads_t *dq,
                            const loco_heads_t *dk, const loco_heads_t *dv, void *d_work, uint64_t d_work_bytes, void *stream) {
    AttentionParams P{};
    int rc = fill(c, P);
    const int64_t nq = rc == LOCO_OK ? rows_of(c, c->seq_q) : 0, nk = rc == LOCO_OK ? rows_of(c, c->seq_k) : 0;
    if (rc == LOCO_OK) rc = take(c, q, c->heads_q, c->seq_q, P.q);
    if (rc == LOCO_OK) rc = take(c, k, c->heads_kv, c->seq_k, P.k);
    if (rc == LOCO_OK) rc = take(c, v, c->heads_kv, c->seq_k, P.v);
    if (rc == LOCO_OK) rc = take(c, o, c->heads_q, c->seq_q, P.o);
    if (rc == LOCO_OK) rc = take(c, d_o, c->heads_q, c->seq_q, P.d_o);
    if (rc == LOCO_OK) rc = take(c, dq, c->heads_q, c->seq_q, P.dq, true);
    if (rc == LOCO_OK) rc = take(c, dk, c->heads_kv, c->seq_k, P.dk, true);
    if (rc == LOCO_OK) rc = take(c, dv, c->heads_kv, c->seq_k, P.dv, true);
    if (rc != LOCO_OK) return rc;
    if (nq == 0 && nk == 0) return LOCO_OK;
    if (!d_work || (nq > 0 && !d_lse)) return LOCO_ERR_ARG;
    if (!aligned(d_work, 16) || !aligned(d_lse, 4)) return LOCO_ERR_ALIGN;
    if (d_work_bytes < loco_attention_backward_workspace_bytes(c)) return LOCO_ERR_SIZE;
    P.lse = const_cast<float *>(d_lse);
    P.row_dot = static_cast<float *>(d_work);
    return launch_attention_backward(P, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
