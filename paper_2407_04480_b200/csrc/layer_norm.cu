// Root-mean-square norm with the residual's addition, and its gradient: a row is read once into registers by a team of
// threads, summed over the team and written.
//
// Some ten operations per element read, so the bound is HBM.  A team is 4 to 32 lanes for rows of up to 512 elements, several
// teams to a block, and a whole block above; the weight stays in registers from row to row.
#include <cuda_fp8.h>

#include "layer_common.h"

namespace loco_layer {

constexpr int kMaxDim = 16384;
constexpr int kNormThreads = 512;                // most threads of a block
constexpr int kSmallBlock = 256;                 // threads of a block of several teams
constexpr int kPartials = 444;                   // most blocks of the backward kernel, each leaves a partial row of dw
constexpr int kScaleBlock = 128;
constexpr float kLargestE4m3 = 448.0f, kLeastScale = 1.17549435e-38f;
constexpr unsigned kAll = 0xffffffffu;

struct NormParams {
    const void *x, *r, *w, *dy, *dt;             // x: h in the backward pass
    void *h, *y, *dx;
    float *scale, *part;
    int64_t xs, rs, hs, ys, dys, dts, dxs, rows;
    int32_t dim, team, block, groups, wanted;
    float eps, over_dim;
};

template <typename T, int V> __device__ __forceinline__ void unpack(const Pack<T, V> &p, float *out) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = to_f32(p.v[i]);
}

// Sum over the team, the same in every lane of it; a team above a warp is the block, whose every thread calls.
__device__ __forceinline__ float2 team_sum(float2 s, int team, float2 *fold) {
    for (int o = (team < 32 ? team : 32) / 2; o; o >>= 1) {
        s.x += __shfl_xor_sync(kAll, s.x, o);
        s.y += __shfl_xor_sync(kAll, s.y, o);
    }
    if (team > 32) {
        const int warps = team / 32;
        __syncthreads();                         // what the call before left has been read
        if (threadIdx.x % 32 == 0) fold[threadIdx.x / 32] = s;
        __syncthreads();
        s = make_float2(0.0f, 0.0f);
        for (int i = 0; i < warps; ++i) {
            s.x += fold[i].x;
            s.y += fold[i].y;
        }
    }
    return s;
}
// Largest of the bits of values without a sign: their order is that of the values, NaN above infinity.
__device__ __forceinline__ unsigned team_max(unsigned m, int team, unsigned *fold) {
    for (int o = (team < 32 ? team : 32) / 2; o; o >>= 1) m = max(m, __shfl_xor_sync(kAll, m, o));
    if (team > 32) {
        const int warps = team / 32;
        __syncthreads();
        if (threadIdx.x % 32 == 0) fold[threadIdx.x / 32] = m;
        __syncthreads();
        m = 0;
        for (int i = 0; i < warps; ++i) m = max(m, fold[i]);
    }
    return m;
}
__device__ __forceinline__ float scale_of(unsigned largest) {
    const float m = __uint_as_float(largest);
    return m != m ? m : fmaxf(m / kLargestE4m3, kLeastScale);
}

template <typename T, int V, int kMine, bool kBits8> __global__ void __launch_bounds__(kNormThreads) norm_forward_kernel(const __grid_constant__ NormParams P) {
    wait_for_previous();
    let_next_start();
    constexpr int kVecs = kMine / V;
    using Vec = Pack<T, V>;
    __shared__ float2 fold[kNormThreads / 32];
    __shared__ unsigned most[kBits8 ? 256 : 1];  // a row's or several rows' runs of 128 columns: threads * kMine / 128 of them at most
    const int team = P.team, lane = static_cast<int>(threadIdx.x) % team, mine = static_cast<int>(threadIdx.x) / team, teams = static_cast<int>(blockDim.x) / team;
    Vec w[kVecs];
    if (P.w) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (i * team + lane) * V;
            if (at < P.dim) w[i] = *reinterpret_cast<const Vec *>(static_cast<const T *>(P.w) + at);
        }
    }
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * teams; first < P.rows; first += static_cast<int64_t>(gridDim.x) * teams) {
        const int64_t row = first + mine;
        const bool there = row < P.rows;
        const T *x = static_cast<const T *>(P.x) + row * P.xs, *r = static_cast<const T *>(P.r) + row * P.rs;
        Vec a[kVecs], b[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (i * team + lane) * V;
            if (there && at < P.dim) {
                a[i] = *reinterpret_cast<const Vec *>(x + at);
                if (P.r) b[i] = *reinterpret_cast<const Vec *>(r + at);
            }
        }
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (i * team + lane) * V;
            if (there && at < P.dim) {
                if (P.r) {
#pragma unroll
                    for (int j = 0; j < V; ++j) a[i].v[j] = from_f32<T>(to_f32(a[i].v[j]) + to_f32(b[i].v[j]));
                    *reinterpret_cast<Vec *>(static_cast<T *>(P.h) + row * P.hs + at) = a[i];
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float f = to_f32(a[i].v[j]);
                    sum.x = fmaf(f, f, sum.x);
                }
            }
        }
        const float by = rsqrtf(team_sum(sum, team, fold).x * P.over_dim + P.eps);
        if constexpr (!kBits8) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const int at = (i * team + lane) * V;
                if (there && at < P.dim) {
#pragma unroll
                    for (int j = 0; j < V; ++j) a[i].v[j] = from_f32<T>(to_f32(a[i].v[j]) * by * (P.w ? to_f32(w[i].v[j]) : 1.0f));
                    *reinterpret_cast<Vec *>(static_cast<T *>(P.y) + row * P.ys + at) = a[i];
                }
            }
        } else {
            float y[kVecs][V];
            unsigned m[kVecs];
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const int at = (i * team + lane) * V;
                m[i] = 0;
                if (there && at < P.dim) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        y[i][j] = to_f32(a[i].v[j]) * by * (P.w ? to_f32(w[i].v[j]) : 1.0f);
                        m[i] = max(m[i], __float_as_uint(y[i][j]) & 0x7fffffffu);
                    }
                }
            }
            unsigned all = 0;
            if (P.block == 0) {
#pragma unroll
                for (int i = 0; i < kVecs; ++i) all = max(all, m[i]);
                all = team_max(all, team, reinterpret_cast<unsigned *>(fold));
                if (there && lane == 0) P.scale[row] = scale_of(all);
            } else {
                __syncthreads();                 // what the row before left has been read
                for (int i = threadIdx.x; i < teams * P.groups; i += blockDim.x) most[i] = 0;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    const int at = (i * team + lane) * V;
                    if (there && at < P.dim) atomicMax(&most[mine * P.groups + at / kScaleBlock], m[i]);
                }
                __syncthreads();
                for (int i = lane; i < P.groups && there; i += team) P.scale[row * P.groups + i] = scale_of(most[mine * P.groups + i]);
            }
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const int at = (i * team + lane) * V;
                if (there && at < P.dim) {
                    const float over = 1.0f / scale_of(P.block == 0 ? all : most[mine * P.groups + at / kScaleBlock]);
                    Pack<__nv_fp8_storage_t, V> q;
#pragma unroll
                    for (int j = 0; j < V; ++j) q.v[j] = __nv_cvt_float_to_fp8(y[i][j] * over, __NV_SATFINITE, __NV_E4M3);
                    *reinterpret_cast<Pack<__nv_fp8_storage_t, V> *>(static_cast<__nv_fp8_storage_t *>(P.y) + row * P.ys + at) = q;
                }
            }
        }
    }
}

// dx of every row, and over the block's rows the sums of dy n, each thread its own columns'.
template <typename T, int V, int kMine> __global__ void __launch_bounds__(kNormThreads) norm_backward_kernel(const __grid_constant__ NormParams P) {
    wait_for_previous();
    let_next_start();
    constexpr int kVecs = kMine / V;
    using Vec = Pack<T, V>;
    __shared__ float2 fold[kNormThreads / 32];
    extern __shared__ float sums[];              // of a block of several teams: dw of each
    const int team = P.team, lane = static_cast<int>(threadIdx.x) % team, mine = static_cast<int>(threadIdx.x) / team, teams = static_cast<int>(blockDim.x) / team;
    Vec w[kVecs];
    float dw[kVecs][V];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int at = (i * team + lane) * V;
        if (P.w && at < P.dim) w[i] = *reinterpret_cast<const Vec *>(static_cast<const T *>(P.w) + at);
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = 0.0f;
    }
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * teams; first < P.rows; first += static_cast<int64_t>(gridDim.x) * teams) {
        const int64_t row = first + mine;
        const bool there = row < P.rows;
        const T *h = static_cast<const T *>(P.x) + row * P.xs, *dy = static_cast<const T *>(P.dy) + row * P.dys, *dt = static_cast<const T *>(P.dt) + row * P.dts;
        Vec a[kVecs], d[kVecs], t[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (i * team + lane) * V;
            if (there && at < P.dim) {
                a[i] = *reinterpret_cast<const Vec *>(h + at);
                d[i] = *reinterpret_cast<const Vec *>(dy + at);
                if (P.dt) t[i] = *reinterpret_cast<const Vec *>(dt + at);
            }
        }
        float2 sum = make_float2(0.0f, 0.0f);    // of h^2 and of dy w h
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (i * team + lane) * V;
            if (there && at < P.dim) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float f = to_f32(a[i].v[j]), g = to_f32(d[i].v[j]) * (P.w ? to_f32(w[i].v[j]) : 1.0f);
                    sum.x = fmaf(f, f, sum.x);
                    sum.y = fmaf(f, g, sum.y);
                }
            }
        }
        sum = team_sum(sum, team, fold);
        const float by = rsqrtf(sum.x * P.over_dim + P.eps), pull = sum.y * P.over_dim * by * by;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (i * team + lane) * V;
            if (there && at < P.dim) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float f = to_f32(a[i].v[j]), e = to_f32(d[i].v[j]);
                    const float g = e * (P.w ? to_f32(w[i].v[j]) : 1.0f);
                    dw[i][j] = fmaf(e, f * by, dw[i][j]);
                    float out = by * (g - f * pull);
                    if (P.dt) out += to_f32(t[i].v[j]);
                    a[i].v[j] = from_f32<T>(out);
                }
                *reinterpret_cast<Vec *>(static_cast<T *>(P.dx) + row * P.dxs + at) = a[i];
            }
        }
    }
    if (!P.wanted) return;
    float *const part = P.part + static_cast<int64_t>(blockIdx.x) * P.dim;
    if (teams == 1) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (i * team + lane) * V;
            if (at < P.dim) *reinterpret_cast<Pack<float, V> *>(part + at) = *reinterpret_cast<Pack<float, V> *>(dw[i]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int at = (i * team + lane) * V;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (at < P.dim) sums[mine * P.dim + at + j] = dw[i][j];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < P.dim; c += blockDim.x) {
        float s = 0.0f;
        for (int i = 0; i < teams; ++i) s += sums[i * P.dim + c];
        part[c] = s;
    }
}

// The blocks' partial rows added in their order: 32 columns to a block, eight warps that each take an eighth of the rows.
template <typename T> __global__ void __launch_bounds__(256) norm_weight_kernel(const float *part, int blocks, int dim, T *dw) {
    wait_for_previous();
    let_next_start();
    __shared__ float fold[8][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = static_cast<int>(blockIdx.x) * 32 + lane;
    const int per = (blocks + 7) / 8, from = warp * per, until = min(from + per, blocks);
    float s = 0.0f;
    if (c < dim)
#pragma unroll 8
        for (int b = from; b < until; ++b) s += part[static_cast<int64_t>(b) * dim + c];
    fold[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < dim) {
        s = 0.0f;
        for (int i = 0; i < 8; ++i) s += fold[i][lane];
        dw[c] = from_f32<T>(s);
    }
}

namespace {

using NormKernel = void (*)(const NormParams);

template <typename T, int V, int kMine> NormKernel pick_norm(bool backward, bool bits8) {
    if (backward) return norm_backward_kernel<T, V, kMine>;
    return bits8 ? norm_forward_kernel<T, V, kMine, true> : norm_forward_kernel<T, V, kMine, false>;
}
template <typename T, int V> NormKernel pick_norm(int dim, bool backward, bool bits8) {
    return dim <= 8192 ? pick_norm<T, V, 16>(backward, bits8) : pick_norm<T, V, 32>(backward, bits8);
}

int check_norm(const loco_norm_t *c) {
    if (!c) return LOCO_ERR_ARG;
    if (c->dtype != LOCO_F32 && c->dtype != LOCO_BF16) return LOCO_ERR_ARG;
    if (c->dim < 1 || !(c->eps >= 0.0f) || !std::isfinite(c->eps)) return LOCO_ERR_ARG;
    if (c->bits8 && c->block != 0 && c->block != kScaleBlock) return LOCO_ERR_ARG;
    return c->dim > kMaxDim ? LOCO_ERR_UNSUPPORTED : LOCO_OK;
}

// What the vector accesses of a call have to keep to: `vec` elements of every row and of the weight together.
struct Widths {
    int vec;
    int64_t rows;
    void narrow(int to) { vec = to < vec ? to : vec; }
    void take(const void *at, int64_t stride, int size, int64_t dim) {
        int v = vec;
        while (v > 1 && (!aligned(at, static_cast<uintptr_t>(v * size)) || (rows > 1 && stride % v != 0) || dim % v != 0)) v /= 2;
        narrow(v);
    }
};

// A tensor of rows: present where it has to be, aligned to its elements; an output's rows do not overlap.
int take_rows(const loco_rows_t *t, int64_t rows, int dim, int size, bool written, Widths &W, int64_t &stride) {
    if (!t || !t->ptr) return LOCO_ERR_ARG;
    stride = rows > 1 ? t->row_stride : 0;
    if (stride < 0 || (written && rows > 1 && stride < dim)) return LOCO_ERR_ARG;
    if (!aligned(t->ptr, static_cast<uintptr_t>(size))) return LOCO_ERR_ALIGN;
    W.take(t->ptr, stride, size, dim);
    return LOCO_OK;
}

// Threads of a row, and blocks; 16 elements a thread, 32 above 8192.
int launch_norm(NormParams &P, const loco_norm_t *c, bool backward, int vec, void *stream, int &blocks) {
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    const int mine = c->dim <= 8192 ? 16 : 32, lanes = (c->dim + mine - 1) / mine;
    int team = 4;
    while (team < 32 && team < lanes) team *= 2;
    if (lanes > 32) team = (lanes + 31) / 32 * 32;
    const int threads = team > 32 ? team : kSmallBlock, teams = threads / team;
    const int64_t all = (P.rows + teams - 1) / teams, most = backward ? (3 * sms < kPartials ? 3 * sms : kPartials) : static_cast<int64_t>(sms) * (2048 / threads);
    blocks = static_cast<int>(all < most ? all : most);
    P.team = team;
    P.dim = c->dim;
    P.block = c->block;
    P.groups = (c->dim + kScaleBlock - 1) / kScaleBlock;
    P.eps = c->eps;
    P.over_dim = 1.0f / static_cast<float>(c->dim);
    NormKernel fn;
    if (c->dtype == LOCO_BF16) {
        fn = vec >= 8 ? pick_norm<__nv_bfloat16, 8>(c->dim, backward, c->bits8) : vec >= 2 ? pick_norm<__nv_bfloat16, 2>(c->dim, backward, c->bits8)
                                                                                       : pick_norm<__nv_bfloat16, 1>(c->dim, backward, c->bits8);
    } else {
        fn = vec >= 4 ? pick_norm<float, 4>(c->dim, backward, c->bits8) : pick_norm<float, 1>(c->dim, backward, c->bits8);
    }
    const size_t shared = backward && teams > 1 && P.wanted ? static_cast<size_t>(teams) * c->dim * sizeof(float) : 0;
    return launch_kernel(fn, dim3(static_cast<unsigned>(blocks)), static_cast<unsigned>(threads), shared, stream, P);
}

}  // namespace

}  // namespace loco_layer

using namespace loco_layer;

extern "C" {

int loco_norm_forward(const loco_norm_t *c, int64_t rows, const loco_rows_t *x, const loco_rows_t *residual, const void *d_weight,
                      const loco_rows_t *total, const loco_rows_t *y, float *d_scale, void *stream) {
    int rc = check_norm(c);
    if (rc != LOCO_OK) return rc;
    if (rows < 0 || (residual != nullptr) != (total != nullptr)) return LOCO_ERR_ARG;
    if (rows == 0) return LOCO_OK;
    const int size = c->dtype == LOCO_BF16 ? 2 : 4;
    NormParams P{};
    P.rows = rows;
    Widths W{16 / size, rows};
    if ((rc = take_rows(x, rows, c->dim, size, false, W, P.xs)) != LOCO_OK) return rc;
    if (residual && (rc = take_rows(residual, rows, c->dim, size, false, W, P.rs)) != LOCO_OK) return rc;
    if (total && (rc = take_rows(total, rows, c->dim, size, true, W, P.hs)) != LOCO_OK) return rc;
    if ((rc = take_rows(y, rows, c->dim, c->bits8 ? 1 : size, true, W, P.ys)) != LOCO_OK) return rc;
    if (c->bits8 && !d_scale) return LOCO_ERR_ARG;
    if (!aligned(d_weight, static_cast<uintptr_t>(size)) || !aligned(d_scale, 4)) return LOCO_ERR_ALIGN;
    if (d_weight) W.take(d_weight, 0, size, c->dim);
    P.x = x->ptr;
    P.r = residual ? residual->ptr : nullptr;
    P.h = total ? total->ptr : nullptr;
    P.y = y->ptr;
    P.w = d_weight;
    P.scale = d_scale;
    int blocks;
    return launch_norm(P, c, false, W.vec, stream, blocks);
}

uint64_t loco_norm_backward_workspace_bytes(const loco_norm_t *c) {
    return check_norm(c) == LOCO_OK ? static_cast<uint64_t>(kPartials) * c->dim * sizeof(float) : 0;
}

int loco_norm_backward(const loco_norm_t *c, int64_t rows, const loco_rows_t *h, const loco_rows_t *dy, const void *d_weight,
                       const loco_rows_t *dtotal, const loco_rows_t *dx, void *d_dweight, void *d_work, uint64_t d_work_bytes, void *stream) {
    int rc = check_norm(c);
    if (rc != LOCO_OK) return rc;
    if (rows < 0 || c->bits8) return LOCO_ERR_ARG;
    const int size = c->dtype == LOCO_BF16 ? 2 : 4;
    NormParams P{};
    P.rows = rows;
    P.wanted = d_dweight != nullptr;
    if (P.wanted) {
        if (!d_work) return LOCO_ERR_ARG;
        if (!aligned(d_work, 16) || !aligned(d_dweight, static_cast<uintptr_t>(size))) return LOCO_ERR_ALIGN;
        if (d_work_bytes < loco_norm_backward_workspace_bytes(c)) return LOCO_ERR_SIZE;
    }
    if (rows == 0 && !P.wanted) return LOCO_OK;
    int blocks = 0;
    P.part = static_cast<float *>(d_work);
    if (rows > 0) {
        Widths W{16 / size, rows};
        if ((rc = take_rows(h, rows, c->dim, size, false, W, P.xs)) != LOCO_OK) return rc;
        if ((rc = take_rows(dy, rows, c->dim, size, false, W, P.dys)) != LOCO_OK) return rc;
        if (dtotal && (rc = take_rows(dtotal, rows, c->dim, size, false, W, P.dts)) != LOCO_OK) return rc;
        if ((rc = take_rows(dx, rows, c->dim, size, true, W, P.dxs)) != LOCO_OK) return rc;
        if (!aligned(d_weight, static_cast<uintptr_t>(size))) return LOCO_ERR_ALIGN;
        if (d_weight) W.take(d_weight, 0, size, c->dim);
        P.x = h->ptr;
        P.dy = dy->ptr;
        P.dt = dtotal ? dtotal->ptr : nullptr;
        P.dx = dx->ptr;
        P.w = d_weight;
        rc = launch_norm(P, c, true, W.vec, stream, blocks);
        if (rc != LOCO_OK || !P.wanted) return rc;
    }
    const dim3 grid(static_cast<unsigned>((c->dim + 31) / 32));
    if (c->dtype == LOCO_BF16) return launch_kernel(norm_weight_kernel<__nv_bfloat16>, grid, 256, 0, stream, P.part, blocks, c->dim, static_cast<__nv_bfloat16 *>(d_dweight));
    return launch_kernel(norm_weight_kernel<float>, grid, 256, 0, stream, P.part, blocks, c->dim, static_cast<float *>(d_dweight));
}

}  // extern "C"
