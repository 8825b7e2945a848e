// Choices sorted by expert, tokens laid out in that order and summed back with their weights, and the gradients.
//
// Sorting is a counting sort: every warp counts the experts of its own run of choices, the counts before it (of the block's
// warps, and of the blocks before) give the warp's first row of every expert, and the lanes that hold the same expert take
// rows in their order.  So the order is that of expert, token, slot, and no atomic decides it.
// The other passes move rows: a team of threads has a token, reads its row once and writes it to all of its places, or
// reads them all and writes the sum.  One or two operations an element, so HBM bounds them.
#include "layer_common.h"
#include "layer_tc.cuh"

namespace loco_layer {

using namespace tc;

constexpr int kMostExperts = 512;
constexpr int kMostChoices = 16;
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortBlocks = 148;                 // most blocks, each leaves its counts to the others
constexpr int kSortEach = 2048;                  // choices a block is worth starting for
constexpr int kMoveThreads = 256;
constexpr int kMostDim = 1 << 30;               // of a row: places in it are counted in 32 bits, some of them past its end
constexpr unsigned kAll = 0xffffffffu;

struct SortParams {
    const int32_t *index;
    int32_t *offsets, *place, *counts;           // counts: [block][expert]
    int64_t choices, each;                       // choices of a block, a multiple of kSortThreads
    int32_t experts;
};

// Counts of each warp's own run of choices, in shared memory.
__device__ __forceinline__ void count_run(const SortParams &P, int *mine, int64_t from, int64_t until, int lane) {
#pragma unroll 8
    for (int64_t i = from + lane; i < until; i += 32) {
        const int e = P.index[i];
        if (static_cast<unsigned>(e) < static_cast<unsigned>(P.experts)) atomicAdd(&mine[e], 1);
    }
}
// The warp's run: choices are dealt to blocks, then warps, in runs.
__device__ __forceinline__ void run_of(const SortParams &P, int warp, int64_t &from, int64_t &until) {
    const int64_t each = P.each / kSortWarps;
    from = static_cast<int64_t>(blockIdx.x) * P.each + warp * each;
    until = min(from + each, P.choices);
}

__global__ void __launch_bounds__(kSortThreads) experts_count_kernel(const SortParams P) {
    wait_for_previous();
    let_next_start();
    __shared__ int count[kMostExperts];
    for (int e = threadIdx.x; e < P.experts; e += kSortThreads) count[e] = 0;
    __syncthreads();
    int64_t from, until;
    run_of(P, threadIdx.x / 32, from, until);
    count_run(P, count, from, until, threadIdx.x % 32);
    __syncthreads();
    for (int e = threadIdx.x; e < P.experts; e += kSortThreads) P.counts[static_cast<int64_t>(blockIdx.x) * P.experts + e] = count[e];
}

// Sum of the values of the threads before, over the block; `total` is the sum of all.
__device__ __forceinline__ int before_in_block(int x, int *fold, int &total) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int s = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kAll, s, o);
        s += lane >= o ? y : 0;
    }
    if (lane == 31) fold[warp] = s;
    __syncthreads();
    int sum = 0;
    total = 0;
    for (int w = 0; w < kSortWarps; ++w) {
        sum += w < warp ? fold[w] : 0;
        total += fold[w];
    }
    return sum + s - x;
}

__global__ void __launch_bounds__(kSortThreads) experts_place_kernel(const SortParams P) {
    wait_for_previous();
    let_next_start();
    extern __shared__ int next[];                // [warp][expert]: counts, then the warp's next row of the expert
    __shared__ int fold[kSortWarps];
    __shared__ int2 counted[kSortThreads];
    static_assert(kMostExperts <= kSortThreads, "one expert a thread");
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, E = P.experts, blocks = static_cast<int>(gridDim.x);
    for (int i = threadIdx.x; i < kSortWarps * E; i += kSortThreads) next[i] = 0;
    __syncthreads();
    int64_t from, until;
    run_of(P, warp, from, until);
    count_run(P, next + warp * E, from, until, lane);
    __syncthreads();
    const int e = threadIdx.x;
    int all = 0, before = 0;                     // of the expert: choices of all blocks, of the blocks before this one
    if (blocks == 1) {
        if (e < E)
            for (int w = 0; w < kSortWarps; ++w) all += next[w * E + e];
    } else {                                     // the blocks' counts are dealt to as many threads for each expert as there are
        const int parts = kSortThreads / E, part = e / E, mine = e % E;
        if (part < parts) {
#pragma unroll 8
            for (int b = part; b < blocks; b += parts) {
                const int n = __ldcg(P.counts + static_cast<int64_t>(b) * E + mine);
                all += n;
                before += b < static_cast<int>(blockIdx.x) ? n : 0;
            }
        }
        counted[e] = make_int2(all, before);
        __syncthreads();
        all = before = 0;
        if (e < E)
            for (int p = 0; p < parts; ++p) {
                all += counted[p * E + e].x;
                before += counted[p * E + e].y;
            }
    }
    int total;
    const int first = before_in_block(all, fold, total);
    if (e < E) {
        if (blockIdx.x == 0) {
            P.offsets[e] = first;
            if (e == 0) P.offsets[E] = total;
        }
        int row = first + before;
        for (int w = 0; w < kSortWarps; ++w) {
            const int n = next[w * E + e];
            next[w * E + e] = row;
            row += n;
        }
    }
    __syncthreads();
    int *const mine = next + warp * E;
    constexpr int kAtOnce = 8;                   // of the warp's loads: one by one they are what a long run waits for
    for (int64_t i = from; i < until; i += 32 * kAtOnce) {
        int chosen[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) chosen[u] = i + u * 32 + lane < until ? P.index[i + u * 32 + lane] : -1;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t at = i + u * 32 + lane;
            const bool some = static_cast<unsigned>(chosen[u]) < static_cast<unsigned>(E);
            const unsigned same = __match_any_sync(kAll, some ? chosen[u] : -1);
            const int row = some ? mine[chosen[u]] : 0;
            __syncwarp();
            if (some && lane == __ffs(same) - 1) mine[chosen[u]] = row + __popc(same);
            __syncwarp();
            if (at < until) P.place[at] = some ? row + __popc(same & ((1u << lane) - 1)) : -1;
        }
    }
}

struct MoveParams {
    const void *in, *rows;                       // tokens read (x, dy), sorted rows read
    void *out, *rows_out;                        // tokens written, sorted rows written
    const int32_t *place;
    const float *weight;
    float *dweight;
    int64_t in_stride, out_stride, rows_stride, rows_out_stride, tokens, row_count;
    int32_t dim, top_k, team;
};

// Token and lane of a thread: a team of threads to a token, several teams to a block.
struct Seat {
    int64_t token;
    int lane;
};
__device__ __forceinline__ Seat seat(int team) {
    return Seat{static_cast<int64_t>(blockIdx.x) * (kMoveThreads / team) + static_cast<int>(threadIdx.x) / team, static_cast<int>(threadIdx.x) % team};
}

template <typename T, int V> __global__ void __launch_bounds__(kMoveThreads) experts_dispatch_kernel(const __grid_constant__ MoveParams P) {
    wait_for_previous();
    let_next_start();
    using Vec = Pack<T, V>;
    const Seat s = seat(P.team);
    if (s.token >= P.tokens) return;
    const T *x = static_cast<const T *>(P.in) + s.token * P.in_stride;
    const int32_t *place = P.place + s.token * P.top_k;
    for (int c = s.lane * V; c < P.dim; c += P.team * V) {
        const Vec v = *reinterpret_cast<const Vec *>(x + c);
        for (int j = 0; j < P.top_k; ++j) {
            const int p = place[j];
            if (p >= 0 && p < P.row_count) *reinterpret_cast<Vec *>(static_cast<T *>(P.rows_out) + p * P.rows_out_stride + c) = v;
        }
    }
}

// The choices j0 .. j0 + kRows - 1 of a token: their rows (-1: none) and weights.  Read again where they are needed again, from
// L1: kept for all choices they cost the registers that keep enough threads at work (six choices: 46 us against 30).  By ordinary loads: the launch
// before, which may have written them, need not have ended when this one starts, so that they are not constant over its lifetime.
template <int kRows> __device__ __forceinline__ void choices_at(const MoveParams &P, int64_t token, int j0, int (&p)[kRows], float (&w)[kRows]) {
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
        p[j] = -1;
        w[j] = 0.0f;
        if (j0 + j < P.top_k) {
            const int at = P.place[token * P.top_k + j0 + j];
            p[j] = at < P.row_count ? at : -1;
            w[j] = P.weight ? P.weight[token * P.top_k + j0 + j] : 1.0f;
        }
    }
}

// A thread asks for kRows * kPlaces vectors before it uses the first.  kEvery: kRows are all choices of a token; else four at a
// time, at one place.
template <typename T, int V, int kRows, int kPlaces, bool kEvery>
__global__ void __launch_bounds__(kMoveThreads, 4) experts_combine_kernel(const __grid_constant__ MoveParams P) {
    wait_for_previous();
    let_next_start();
    static_assert(kEvery || kPlaces == 1, "sums of one place are kept");
    using Vec = Pack<T, V>;
    constexpr int kPairs = (V + 1) / 2;
    const Seat s = seat(P.team);
    if (s.token >= P.tokens) return;
    T *const y = static_cast<T *>(P.out) + s.token * P.out_stride;
    const int step = P.team * V;
    int p[kRows];
    float w[kRows];
    if (kEvery) choices_at<kRows>(P, s.token, 0, p, w);
#pragma unroll 1
    for (int c = s.lane * V; c < P.dim; c += kPlaces * step) {
        float2 sum[kPairs];
#pragma unroll
        for (int q = 0; q < kPairs; ++q) sum[q] = make_float2(0.0f, 0.0f);
#pragma unroll 1
        for (int j0 = 0; j0 < (kEvery ? 1 : P.top_k); j0 += kRows) {
            if (!kEvery) choices_at<kRows>(P, s.token, j0, p, w);
            Vec v[kPlaces][kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const T *const row = static_cast<const T *>(P.rows) + p[j] * P.rows_stride + c;
#pragma unroll
                for (int u = 0; u < kPlaces; ++u)
                    if (p[j] >= 0 && c + u * step < P.dim) v[u][j] = *reinterpret_cast<const Vec *>(row + u * step);
            }
#pragma unroll
            for (int u = 0; u < kPlaces; ++u) {
#pragma unroll
                for (int j = 0; j < kRows; ++j)
                    if (p[j] >= 0)
#pragma unroll
                        for (int q = 0; q < kPairs; ++q) sum[q] = fma2(make_float2(w[j], w[j]), pair_of(v[u][j], q), sum[q]);
                if (kEvery && c + u * step < P.dim) {
                    Vec out;
#pragma unroll
                    for (int q = 0; q < kPairs; ++q) {
                        set_pair(out, q, sum[q]);
                        sum[q] = make_float2(0.0f, 0.0f);
                    }
                    *reinterpret_cast<Vec *>(y + c + u * step) = out;
                }
            }
        }
        if (!kEvery) {
            Vec out;
#pragma unroll
            for (int q = 0; q < kPairs; ++q) set_pair(out, q, sum[q]);
            *reinterpret_cast<Vec *>(y + c) = out;
        }
    }
}

// Sums of kN values over aligned groups of `width` lanes.  Lanes first share out the values (a step halves what each holds), so
// that eight values over a warp take 7 + 2 exchanges instead of 40; value j ends in the lanes whose low bits are j.
template <int kN> __device__ __forceinline__ float shared_sum(float (&x)[kN], int lane, int width) {
    int o = 1;
#pragma unroll
    for (int n = kN / 2; n; n /= 2) {
        const bool upper = lane & o;
#pragma unroll
        for (int j = 0; j < n; ++j) {                // values j and j + n: the lane's bit says which it keeps
            const float give = upper ? x[2 * j] : x[2 * j + 1], keep = upper ? x[2 * j + 1] : x[2 * j];
            x[j] = keep + __shfl_xor_sync(kAll, give, o);
        }
        o <<= 1;
    }
    float s = x[0];
    for (; o < width; o <<= 1) s += __shfl_xor_sync(kAll, s, o);
    return s;
}

// kRows choices at a time, at kPlaces places; dy is read again, from L1 or L2, for the next ones.
template <typename T, int V, int kRows, int kPlaces>
__global__ void __launch_bounds__(kMoveThreads, kRows > 4 ? 3 : 4) experts_backward_kernel(const __grid_constant__ MoveParams P) {
    wait_for_previous();
    let_next_start();
    using Vec = Pack<T, V>;
    __shared__ float fold[2][kMoveThreads / 32][kRows];
    const Seat s = seat(P.team);
    const bool there = s.token < P.tokens;
    const int64_t token = there ? s.token : 0;
    const T *const dy = static_cast<const T *>(P.in) + token * P.in_stride;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, width = P.team < 32 ? P.team : 32, step = P.team * V;
    int side = 0;
#pragma unroll 1
    for (int j0 = 0; j0 < P.top_k; j0 += kRows) {
        int p[kRows];
        float w[kRows], dot[kRows];
        choices_at<kRows>(P, token, j0, p, w);
#pragma unroll
        for (int j = 0; j < kRows; ++j) dot[j] = 0.0f;
#pragma unroll 1
        for (int c = s.lane * V; c < P.dim && there; c += kPlaces * step) {
            Vec d[kPlaces], r[kPlaces][kRows];
#pragma unroll
            for (int u = 0; u < kPlaces; ++u)
                if (c + u * step < P.dim) d[u] = *reinterpret_cast<const Vec *>(dy + c + u * step);
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const T *const row = static_cast<const T *>(P.rows) + p[j] * P.rows_stride + c;
#pragma unroll
                for (int u = 0; u < kPlaces; ++u)
                    if (p[j] >= 0 && c + u * step < P.dim) r[u][j] = *reinterpret_cast<const Vec *>(row + u * step);
            }
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                T *const row = static_cast<T *>(P.rows_out) + p[j] * P.rows_out_stride + c;
#pragma unroll
                for (int u = 0; u < kPlaces; ++u)
                    if (p[j] >= 0 && c + u * step < P.dim) {
                        Vec out;
#pragma unroll
                        for (int q = 0; q < (V + 1) / 2; ++q) {
                            const float2 f = pair_of(d[u], q), g = pair_of(r[u][j], q);
                            dot[j] = fmaf(f.x, g.x, fmaf(f.y, g.y, dot[j]));
                            set_pair(out, q, mul2(make_float2(w[j], w[j]), f));
                        }
                        *reinterpret_cast<Vec *>(row + u * step) = out;
                    }
            }
        }
        float sum = shared_sum<kRows>(dot, lane, width);
        float *const dw = P.dweight + token * P.top_k + j0;
        if (P.team <= 32) {
            if (there && s.lane < kRows && j0 + s.lane < P.top_k) dw[s.lane] = sum;
        } else {                                     // two sides: the next ones' sums go to the other
            if (lane < kRows) fold[side][warp][lane] = sum;
            __syncthreads();
            if (there && s.lane < kRows && j0 + s.lane < P.top_k) {
                sum = 0.0f;
                for (int i = 0; i < P.team / 32; ++i) sum += fold[side][warp + i][s.lane];
                dw[s.lane] = sum;
            }
            side ^= 1;
        }
    }
}

// ---- rows that do not share their 16-byte boundaries -----------------------------------------

// Rows of an odd width lie each at a distance of its own from the boundaries.  What is written is then cut into the aligned vectors of
// its own row, but for the ends; what is read comes as the two aligned vectors that hold its 16 bytes, slid together.  Every
// tensor begins on a boundary.  In single elements 30,000 tokens of 1367, two choices, bfloat16, are laid out in 123 us.
template <typename T> struct Slide {
    static constexpr int kV = 16 / sizeof(T);
    const T *row;
    int64_t left;                                // elements from `row` to the end of the tensor
    struct Two {
        uint4 lo, hi;
    };
    __device__ __forceinline__ unsigned off(int c) const { return static_cast<unsigned>(reinterpret_cast<uintptr_t>(row + c)) & 15u; }
    // The vectors that hold elements c .. c + kV - 1 of the row, all of them the row's.
    __device__ __forceinline__ Two ask(int c) const {
        const unsigned o = off(c);
        const uint4 *const from = reinterpret_cast<const uint4 *>(reinterpret_cast<const uint8_t *>(row + c) - o);
        Two t{from[0], make_uint4(0, 0, 0, 0)};
        const int have = o / sizeof(T);          // elements in the second one
        if (have && c + 2 * kV - have <= left) {
            t.hi = from[1];
        } else if (have) {                       // past the tensor's end there may be nothing: what is the row's, one by one
#pragma unroll
            for (int j = 0; j < kV; ++j)
                if (j < have) {
                    const T *const at = row + c + kV - have + j;
                    const uint32_t bits = sizeof(T) == 2 ? *reinterpret_cast<const uint16_t *>(at) : *reinterpret_cast<const uint32_t *>(at);
                    (&t.hi.x)[j * sizeof(T) / 4] |= bits << (j * sizeof(T) % 4 * 8);
                }
        }
        return t;
    }
    __device__ __forceinline__ Pack<T, kV> join(const Two &t, int c) const {
        const unsigned o = off(c);
        uint32_t w[8] = {t.lo.x, t.lo.y, t.lo.z, t.lo.w, t.hi.x, t.hi.y, t.hi.z, t.hi.w};
#pragma unroll
        for (int k = 0; k < 6; ++k) w[k] = o & 8u ? w[k + 2] : w[k];
#pragma unroll
        for (int k = 0; k < 5; ++k) w[k] = o & 4u ? w[k + 1] : w[k];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], o & 2u ? 16 : 0);
        Pack<T, kV> v;
        memcpy(&v, w, 16);
        return v;
    }
};
template <typename T> __device__ __forceinline__ Slide<T> slide(const void *base, int64_t row, int64_t stride, int64_t rows, int dim) {
    return Slide<T>{static_cast<const T *>(base) + row * stride, (rows - 1 - row) * stride + dim};
}
// A row that is written: its vectors begin this many elements ahead of it.
template <typename T> __device__ __forceinline__ int shift_of(const T *row) { return static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T)); }
// The 16 bytes within the row that hold what vector c has of it: the vector itself, or at the row's ends the first or the last ones.
template <int kV> __device__ __forceinline__ int within_row(int c, int dim) { return min(max(c, 0), dim - kV); }
// Vector c of a row, of which `v` holds the elements from `at` on; element by element at the row's ends.
template <typename T, int kV> __device__ __forceinline__ void put(T *row, int c, int at, int dim, const Pack<T, kV> &v) {
    if (c == at) {
        *reinterpret_cast<Pack<T, kV> *>(row + c) = v;
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (at + i >= c && at + i < c + kV) row[at + i] = v.v[i];
    }
}

// Both of a thread's vectors are asked for before the first is written: loads are not moved over stores.
template <typename T> __global__ void __launch_bounds__(kMoveThreads) experts_dispatch_slide_kernel(const __grid_constant__ MoveParams P) {
    wait_for_previous();
    let_next_start();
    constexpr int kV = 16 / sizeof(T);
    const Seat s = seat(P.team);
    if (s.token >= P.tokens) return;
    const Slide<T> x = slide<T>(P.in, s.token, P.in_stride, P.tokens, P.dim);
    const int step = P.team * kV;
    for (int j = 0; j < P.top_k; ++j) {
        const int p = P.place[s.token * P.top_k + j];
        if (p < 0 || p >= P.row_count) continue;
        T *const row = static_cast<T *>(P.rows_out) + p * P.rows_out_stride;
        for (int c0 = s.lane * kV - shift_of(row); c0 < P.dim; c0 += 2 * step) {
            typename Slide<T>::Two t[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (c0 + u * step < P.dim) t[u] = x.ask(within_row<kV>(c0 + u * step, P.dim));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int c = c0 + u * step, at = within_row<kV>(c, P.dim);
                if (c < P.dim) put<T, kV>(row, c, at, P.dim, x.join(t[u], at));
            }
        }
    }
}

// kRows choices at a time, all asked for before the first is used.
template <typename T, int kRows> __global__ void __launch_bounds__(kMoveThreads, 4) experts_combine_slide_kernel(const __grid_constant__ MoveParams P) {
    wait_for_previous();
    let_next_start();
    constexpr int kV = 16 / sizeof(T);
    const Seat s = seat(P.team);
    if (s.token >= P.tokens) return;
    T *const y = static_cast<T *>(P.out) + s.token * P.out_stride;
#pragma unroll 1
    for (int c = s.lane * kV - shift_of(y); c < P.dim; c += P.team * kV) {
        const int at = within_row<kV>(c, P.dim);
        float2 sum[kV / 2];
#pragma unroll
        for (int q = 0; q < kV / 2; ++q) sum[q] = make_float2(0.0f, 0.0f);
#pragma unroll 1
        for (int j0 = 0; j0 < P.top_k; j0 += kRows) {
            int p[kRows];
            float w[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                p[j] = j0 + j < P.top_k ? P.place[s.token * P.top_k + j0 + j] : -1;
                if (p[j] >= P.row_count) p[j] = -1;
            }
            typename Slide<T>::Two t[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j)
                if (p[j] >= 0) t[j] = slide<T>(P.rows, p[j], P.rows_stride, P.row_count, P.dim).ask(at);
#pragma unroll
            for (int j = 0; j < kRows; ++j)                              // behind what takes longer: 9000 x 1367, six choices, 55 us against 70
                w[j] = j0 + j >= P.top_k ? 0.0f : P.weight ? P.weight[s.token * P.top_k + j0 + j] : 1.0f;
#pragma unroll
            for (int j = 0; j < kRows; ++j)
                if (p[j] >= 0) {
                    const Pack<T, kV> v = slide<T>(P.rows, p[j], P.rows_stride, P.row_count, P.dim).join(t[j], at);
#pragma unroll
                    for (int q = 0; q < kV / 2; ++q) sum[q] = fma2(make_float2(w[j], w[j]), pair_of(v, q), sum[q]);
                }
        }
        Pack<T, kV> out;
#pragma unroll
        for (int q = 0; q < kV / 2; ++q) set_pair(out, q, sum[q]);
        put<T, kV>(y, c, at, P.dim, out);
    }
}

// One choice after the other, each in its own row's vectors, two at a time.
template <typename T> __global__ void __launch_bounds__(kMoveThreads, 4) experts_backward_slide_kernel(const __grid_constant__ MoveParams P) {
    wait_for_previous();
    let_next_start();
    constexpr int kV = 16 / sizeof(T);
    __shared__ float fold[2][kMoveThreads / 32];
    const Seat s = seat(P.team);
    const bool there = s.token < P.tokens;
    const int64_t token = there ? s.token : 0;
    const Slide<T> dy = slide<T>(P.in, token, P.in_stride, P.tokens, P.dim);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, width = P.team < 32 ? P.team : 32, step = P.team * kV;
#pragma unroll 1
    for (int j = 0; j < P.top_k; ++j) {
        const int place = there ? P.place[token * P.top_k + j] : -1, p = place < P.row_count ? place : -1;
        float dot = 0.0f;
        if (p >= 0) {
            const float w = P.weight[token * P.top_k + j];
            const Slide<T> r = slide<T>(P.rows, p, P.rows_stride, P.row_count, P.dim);
            T *const row = static_cast<T *>(P.rows_out) + p * P.rows_out_stride;
#pragma unroll 1
            for (int c0 = s.lane * kV - shift_of(row); c0 < P.dim; c0 += 2 * step) {
                typename Slide<T>::Two a[2], b[2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    if (c0 + u * step < P.dim) {
                        const int at = within_row<kV>(c0 + u * step, P.dim);
                        a[u] = dy.ask(at);
                        b[u] = r.ask(at);
                    }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int c = c0 + u * step, at = within_row<kV>(c, P.dim);
                    if (c < P.dim) {
                        const Pack<T, kV> d = dy.join(a[u], at), f = r.join(b[u], at);
                        Pack<T, kV> out;
                        const int from = max(c, 0) - at, until = min(c + kV, P.dim) - at;      // what of it is this vector's
#pragma unroll
                        for (int q = 0; q < kV / 2; ++q) {
                            const float2 x = pair_of(d, q), y = pair_of(f, q);
                            dot = 2 * q >= from && 2 * q < until ? fmaf(x.x, y.x, dot) : dot;
                            dot = 2 * q + 1 >= from && 2 * q + 1 < until ? fmaf(x.y, y.y, dot) : dot;
                            set_pair(out, q, mul2(make_float2(w, w), x));
                        }
                        put<T, kV>(row, c, at, P.dim, out);
                    }
                }
            }
        }
        for (int o = width / 2; o; o >>= 1) dot += __shfl_xor_sync(kAll, dot, o);
        float *const dw = P.dweight + token * P.top_k + j;
        if (P.team <= 32) {
            if (there && s.lane == 0) *dw = dot;
        } else {                                     // two sides: the next choice's sums go to the other
            if (lane == 0) fold[j & 1][warp] = dot;
            __syncthreads();
            if (there && s.lane == 0) {
                dot = 0.0f;
                for (int i = 0; i < P.team / 32; ++i) dot += fold[j & 1][warp + i];
                *dw = dot;
            }
        }
    }
}

// Rows from the last offset on, or (kOthers) all that no expert has as the products read the offsets: ahead of the first, and from the
// largest on.  Nothing to write, as a rule.
template <typename T, bool kOthers>
__global__ void __launch_bounds__(kMoveThreads) experts_clear_kernel(T *rows, int64_t stride, int64_t count, int dim, const int32_t *offsets, int experts) {
    wait_for_previous();
    let_next_start();
    int64_t ahead = 0;
    int end = kOthers ? 0 : max(offsets[experts], 0);
    if constexpr (kOthers) {
        for (int e = threadIdx.x % 32; e <= experts; e += 32) end = max(end, offsets[e]);
        end = __reduce_max_sync(kAll, end);
        ahead = min(static_cast<int64_t>(max(offsets[0], 0)), count);
    }
    const int64_t none = ahead + max(count - end, static_cast<int64_t>(0));
    for (int64_t i = blockIdx.x; i < none; i += gridDim.x) {
        T *const row = rows + (i < ahead ? i : i - ahead + end) * stride;
        for (int c = threadIdx.x; c < dim; c += kMoveThreads) row[c] = from_f32<T>(0.0f);
    }
}

namespace {

using MoveKernel = void (*)(const MoveParams);
enum Move { kDispatch, kCombine, kBackward };
template <typename T, int V> MoveKernel pick_move(Move m, int k, int places) {
    if (m == kDispatch) return experts_dispatch_kernel<T, V>;
    // Combine, two choices, at one, two, four places: 16384 x 4096: 68, 71, 60 us; 700,000 x 64: 60, 53, 58; 30,000 x 1367 in single elements:
    // 121, 86, 141.  At two, four: 70,001 x 768 68, 54; 300,001 x 150 in words 121, 130; fp32 in words 20,000 x 1367 69, 57.
    // A single choice, four places, against the kernels for two choices: 40 million elements in rows of 1024, fp32, combine 52, 50 us, backward
    // 82, 72; bfloat16 30, 28 and 43, 39; in words 67, 46 and 86, 67.
    if (m == kCombine)
        return k == 1 ? experts_combine_kernel<T, V, 1, 4, true> : k <= 2 ? (places > 2 ? experts_combine_kernel<T, V, 2, 4, true> : experts_combine_kernel<T, V, 2, 2, true>)
               : k <= 4 ? experts_combine_kernel<T, V, 4, 2, true> : experts_combine_kernel<T, V, 4, 1, false>;
    return k == 1 ? experts_backward_kernel<T, V, 1, 4> : k <= 2 ? experts_backward_kernel<T, V, 2, 2> : k <= 4 ? experts_backward_kernel<T, V, 4, 1> : experts_backward_kernel<T, V, 8, 1>;
}

template <typename T> MoveKernel pick_slide(Move m) {
    return m == kDispatch ? experts_dispatch_slide_kernel<T> : m == kCombine ? experts_combine_slide_kernel<T, 4> : experts_backward_slide_kernel<T>;
}

int check_experts(const loco_experts_t *c) {
    if (!c) return LOCO_ERR_ARG;
    if (c->dtype != LOCO_F32 && c->dtype != LOCO_BF16) return LOCO_ERR_ARG;
    if (c->dim < 1 || c->top_k < 1 || c->top_k > kMostChoices) return LOCO_ERR_ARG;
    if (c->tokens < 0 || c->tokens > 0x7fffffff / c->top_k || c->rows < 0 || c->rows > 0x7fffffff) return LOCO_ERR_ARG;
    return c->dim > kMostDim ? LOCO_ERR_UNSUPPORTED : LOCO_OK;
}

// What the accesses of a call can be: all rows on 16-byte boundaries, or on those of four, or every tensor on the former at least.
struct Vectors {
    bool rows = true, words = true, tensors = true;
};
// A tensor of rows: present, aligned to its elements; an output's rows do not overlap.
int take_rows(const loco_experts_t *c, const loco_rows_t *t, int64_t rows, bool written, Vectors &V, int64_t &stride) {
    if (!t) return LOCO_ERR_ARG;
    stride = rows > 1 ? t->row_stride : 0;
    if (rows == 0) return LOCO_OK;
    const int size = c->dtype == LOCO_BF16 ? 2 : 4;
    if (!t->ptr || stride < 0 || (written && rows > 1 && stride < c->dim)) return LOCO_ERR_ARG;
    if (!aligned(t->ptr, static_cast<uintptr_t>(size))) return LOCO_ERR_ALIGN;
    V.tensors = V.tensors && aligned(t->ptr, 16);
    V.rows = V.rows && V.tensors && stride * size % 16 == 0 && c->dim * size % 16 == 0;
    V.words = V.words && aligned(t->ptr, 4) && stride * size % 4 == 0 && c->dim * size % 4 == 0;
    return LOCO_OK;
}

int launch_move(Move m, MoveParams &P, const loco_experts_t *c, const Vectors &V, void *stream) {
    P.tokens = c->tokens;
    P.row_count = c->rows;
    P.dim = c->dim;
    P.top_k = c->top_k;
    // Off the boundaries rows are slid together where single elements would be moved one by one, or rows are short: 30,000 x 1367, bfloat16, two
    // choices, in elements or sliding: laid out 123, 64 us, backward 171, 167; 9000 x 1367, six, 166, 132; 399,644 x 101, fp32, one, 189, 159.
    // Long rows of words are faster word by word, but laid out: 40 million elements in rows of 1002, two choices, bfloat16, in words or sliding: backward
    // 64, 67 us, in rows of 2502 53, 84, fp32 100, 111; 20,000 x 1004, four, laid out 52, 44.  Sums slide from five choices on: 20,000 x
    // 1004, four, 53, 57; 30,000 x 1367, two, 69, 89; 9000 x 1367, six, 162, 54.
    const bool bf16 = c->dtype == LOCO_BF16;
    const int k = c->top_k;
    const bool slides = V.tensors && !V.rows && c->dim >= (bf16 ? 8 : 4) && (m == kDispatch || (m == kCombine ? k > 4 : (bf16 && !V.words) || c->dim < 128));
    const int v = slides || V.rows ? (bf16 ? 8 : 4) : bf16 && V.words ? 2 : 1;
    // places in a row that a thread takes at once
    const bool four = k == 1 || (m == kCombine && k == 2 && (bf16 ? v > 1 : true) && c->dim >= (bf16 && v == 2 ? 128 : 64) * v);
    const int places = slides ? (m == kCombine ? 1 : 2) : m == kDispatch ? 1 : four ? 4 : k <= (m == kCombine ? 4 : 2) ? 2 : 1;
    const MoveKernel fn = slides ? (bf16 ? pick_slide<__nv_bfloat16>(m) : pick_slide<float>(m))
                          : bf16 ? (v == 8   ? pick_move<__nv_bfloat16, 8>(m, k, places)
                                    : v == 2 ? pick_move<__nv_bfloat16, 2>(m, k, places)
                                             : pick_move<__nv_bfloat16, 1>(m, k, places))
                                 : (v == 4 ? pick_move<float, 4>(m, k, places) : pick_move<float, 1>(m, k, places));
    const int least = m == kBackward && k > 4 ? 8 : 4;               // lanes that end with a choice's sum each
    int team = least;
    while (team < kMoveThreads && team * places * v < c->dim) team *= 2;
    // With enough tokens a thread goes round twice (four times over single elements), so that the wait for the places and the sums over
    // the team come to less: 5021 x 2040, six choices, backward once, twice, four times: 46.6, 42.4, 41.3 us, combine 29.1, 28.3, 31.4.
    if (!slides && (m == kBackward || (m == kCombine && (k > 2 || v == 1))))
        for (int turns = 1; turns < (v == 1 ? 4 : 2) && team > 32 && c->tokens * (team / 2) >= sm_count() * 2048ll; turns *= 2) team /= 2;
    P.team = team;
    const int64_t blocks = (c->tokens + kMoveThreads / team - 1) / (kMoveThreads / team);
    return launch_kernel(fn, dim3(static_cast<unsigned>(blocks)), kMoveThreads, 0, stream, P);
}

template <bool kOthers> int clear(int32_t dtype, int32_t dim, int64_t rows_count, const loco_rows_t *rows, int32_t experts, const int32_t *d_offsets, void *stream) {
    const loco_experts_t c{dtype, dim, 1, 0, rows_count};
    int rc = check_experts(&c);
    if (rc != LOCO_OK) return rc;
    if (experts < 1 || experts > kMostExperts || !d_offsets) return LOCO_ERR_ARG;
    Vectors V;
    int64_t stride;
    if ((rc = take_rows(&c, rows, rows_count, true, V, stride)) != LOCO_OK) return rc;
    if (!aligned(d_offsets, 4)) return LOCO_ERR_ALIGN;
    if (rows_count == 0) return LOCO_OK;
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    const dim3 grid(static_cast<unsigned>(rows_count < sms * 4 ? rows_count : sms * 4));
    if (dtype == LOCO_BF16)
        return launch_kernel(experts_clear_kernel<__nv_bfloat16, kOthers>, grid, kMoveThreads, 0, stream, static_cast<__nv_bfloat16 *>(rows->ptr), stride, rows_count, dim, d_offsets, experts);
    return launch_kernel(experts_clear_kernel<float, kOthers>, grid, kMoveThreads, 0, stream, static_cast<float *>(rows->ptr), stride, rows_count, dim, d_offsets, experts);
}

int start(const loco_experts_t *c, const int32_t *place, const float *weight) {
    const int rc = check_experts(c);
    if (rc != LOCO_OK || c->tokens == 0) return rc;
    if (!place) return LOCO_ERR_ARG;
    return aligned(place, 4) && aligned(weight, 4) ? LOCO_OK : LOCO_ERR_ALIGN;
}

}  // namespace

}  // namespace loco_layer

using namespace loco_layer;

extern "C" {

uint64_t loco_experts_sort_workspace_bytes(int32_t experts) {
    return experts < 1 || experts > kMostExperts ? 0 : static_cast<uint64_t>(kSortBlocks) * experts * sizeof(int32_t);
}

int loco_experts_sort(int32_t experts, int64_t tokens, int32_t top_k, const int32_t *d_index, int32_t *d_offsets, int32_t *d_place,
                      void *d_work, uint64_t d_work_bytes, void *stream) {
    if (experts < 1 || experts > kMostExperts || top_k < 1 || top_k > kMostChoices || tokens < 0 || tokens > 0x7fffffff / top_k) return LOCO_ERR_ARG;
    if (!d_offsets || !d_work || (tokens > 0 && (!d_index || !d_place))) return LOCO_ERR_ARG;
    if (!aligned(d_index, 4) || !aligned(d_offsets, 4) || !aligned(d_place, 4) || !aligned(d_work, 16)) return LOCO_ERR_ALIGN;
    if (d_work_bytes < loco_experts_sort_workspace_bytes(experts)) return LOCO_ERR_SIZE;
    SortParams P{};
    P.index = d_index;
    P.offsets = d_offsets;
    P.place = d_place;
    P.counts = static_cast<int32_t *>(d_work);
    P.choices = tokens * top_k;
    P.experts = experts;
    int64_t blocks = (P.choices + kSortEach - 1) / kSortEach;
    blocks = blocks < 1 ? 1 : blocks > kSortBlocks ? kSortBlocks : blocks;
    P.each = ((P.choices + blocks - 1) / blocks + kSortThreads - 1) / kSortThreads * kSortThreads;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (blocks > 1) {
        const int rc = launch_kernel(experts_count_kernel, grid, kSortThreads, 0, stream, P);
        if (rc != LOCO_OK) return rc;
    }
    return launch_kernel(experts_place_kernel, grid, kSortThreads, static_cast<size_t>(kSortWarps) * experts * sizeof(int), stream, P);
}

int loco_experts_clear(int32_t dtype, int32_t dim, int64_t rows_count, const loco_rows_t *rows, int32_t experts, const int32_t *d_offsets, void *stream) {
    return clear<false>(dtype, dim, rows_count, rows, experts, d_offsets, stream);
}

int loco_experts_clear_others(int32_t dtype, int32_t dim, int64_t rows_count, const loco_rows_t *rows, int32_t experts, const int32_t *d_offsets, void *stream) {
    return clear<true>(dtype, dim, rows_count, rows, experts, d_offsets, stream);
}

int loco_experts_dispatch(const loco_experts_t *c, const loco_rows_t *x, const int32_t *d_place, const loco_rows_t *rows, void *stream) {
    int rc = start(c, d_place, nullptr);
    if (rc != LOCO_OK || c->tokens == 0) return rc;
    MoveParams P{};
    Vectors V;
    if ((rc = take_rows(c, x, c->tokens, false, V, P.in_stride)) != LOCO_OK) return rc;
    if ((rc = take_rows(c, rows, c->rows, true, V, P.rows_out_stride)) != LOCO_OK) return rc;
    if (c->rows == 0) return LOCO_OK;
    P.in = x->ptr;
    P.rows_out = rows->ptr;
    P.place = d_place;
    return launch_move(kDispatch, P, c, V, stream);
}

int loco_experts_combine(const loco_experts_t *c, const loco_rows_t *rows, const int32_t *d_place, const float *d_weight,
                         const loco_rows_t *y, void *stream) {
    int rc = start(c, d_place, d_weight);
    if (rc != LOCO_OK || c->tokens == 0) return rc;
    MoveParams P{};
    Vectors V;
    if ((rc = take_rows(c, rows, c->rows, false, V, P.rows_stride)) != LOCO_OK) return rc;
    if ((rc = take_rows(c, y, c->tokens, true, V, P.out_stride)) != LOCO_OK) return rc;
    P.rows = rows->ptr;
    P.out = y->ptr;
    P.place = d_place;
    P.weight = d_weight;
    return launch_move(kCombine, P, c, V, stream);
}

int loco_experts_combine_backward(const loco_experts_t *c, const loco_rows_t *dy, const loco_rows_t *rows, const int32_t *d_place,
                                  const float *d_weight, const loco_rows_t *drows, float *d_dweight, void *stream) {
    int rc = start(c, d_place, d_weight);
    if (rc != LOCO_OK || c->tokens == 0) return rc;
    if (!d_weight || !d_dweight) return LOCO_ERR_ARG;
    if (!aligned(d_dweight, 4)) return LOCO_ERR_ALIGN;
    MoveParams P{};
    Vectors V;
    if ((rc = take_rows(c, dy, c->tokens, false, V, P.in_stride)) != LOCO_OK) return rc;
    if ((rc = take_rows(c, rows, c->rows, false, V, P.rows_stride)) != LOCO_OK) return rc;
    if ((rc = take_rows(c, drows, c->rows, true, V, P.rows_out_stride)) != LOCO_OK) return rc;
    P.in = dy->ptr;
    P.rows = rows->ptr;
    P.rows_out = drows->ptr;
    P.place = d_place;
    P.weight = d_weight;
    P.dweight = d_dweight;
    return launch_move(kBackward, P, c, V, stream);
}

}  // extern "C"
