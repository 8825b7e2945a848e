// Sum of squares over a list of gradients, and the list scaled down to a largest norm.
//
// The list travels in the kernel's parameters.  It is cut into chunks; every block takes a run of consecutive chunks, finds
// the first by bisection and walks on from there.  HBM bounds both passes.  The second walks its run backwards, from what
// the first has read last, which L2 still holds; a list that fits there is read from HBM once.
#include <type_traits>

#include "layer_common.h"

namespace loco_layer {

constexpr int kListThreads = 512;
constexpr int kMostSpans = 768;                  // of a launch: 21 KB of parameters
constexpr int kFewSpans = 128;                   // 3.6 KB: a short list's launch costs less
constexpr int kChunkBytes = 32768;
constexpr int kMostRuns = 1024;                  // blocks whose sums the workspace holds
constexpr uint64_t kTicketBytes = 256;
constexpr unsigned kAll = 0xffffffffu;

template <int kMost> struct ListParams {
    static constexpr int kSpans = kMost;
    const void *x[kMost];
    void *y[kMost];
    uint64_t n[kMost];
    uint32_t first[kMost + 1];                   // chunk
    uint8_t type[kMost];
    uint32_t chunks;
    int32_t count, begin, end;                   // the list's first and last launch
    double max_norm;
    double *squares, *running, *part;
    const double *in;
    unsigned *ticket;
    float *norm;
};

// Elements of a span before the first 16-byte boundary of x.
template <typename T> __device__ __forceinline__ uint32_t head_of(const void *x, uint64_t n) {
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T), head = off ? 16 / sizeof(T) - off : 0;
    return head < n ? head : static_cast<uint32_t>(n);
}

// Sum of squares of a few values, in 64 bits: formed in fp32 unless that leaves its range (values above 1e19 or below 1e-15;
// zeros, of which an idle expert's gradient consists, are told apart).
template <int V> __device__ __forceinline__ double squares_of(const float *f) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) s = fmaf(f[i], f[i], s);
    if (s > 1e-30f && s < 3e38f) return s;
    bool some = false;
#pragma unroll
    for (int i = 0; i < V; ++i) some = some || f[i] != 0.0f;
    if (!some) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) d = fma(static_cast<double>(f[i]), static_cast<double>(f[i]), d);
    return d;
}

// The chunk's part of a span: vectors of 16 bytes from `head` on; the first chunk has the head too, the last one the rest.
struct Piece {
    uint64_t from, until;                        // elements, multiples of the vector from `head`
    bool head, tail;
};
template <typename T> __device__ __forceinline__ Piece piece_of(uint64_t n, uint32_t head, uint32_t chunk, uint32_t chunks) {
    constexpr uint64_t kEach = kChunkBytes / sizeof(T), kV = 16 / sizeof(T);
    const uint64_t body = (n - head) / kV * kV, from = min(chunk * kEach, body), until = chunk + 1 == chunks ? body : min(from + kEach, body);
    return Piece{head + from, head + until, chunk == 0, chunk + 1 == chunks};
}

template <typename T> __device__ __forceinline__ double square_piece(const T *x, uint64_t n, uint32_t chunk, uint32_t chunks) {
    constexpr int kV = 16 / sizeof(T);
    const uint32_t head = head_of<T>(x, n);
    const Piece p = piece_of<T>(n, head, chunk, chunks);
    double sum = 0.0;
#pragma unroll 4
    for (uint64_t i = p.from + threadIdx.x * kV; i < p.until; i += kListThreads * kV) {
        const Pack<T, kV> v = *reinterpret_cast<const Pack<T, kV> *>(x + i);
        float f[kV];
#pragma unroll
        for (int j = 0; j < kV; ++j) f[j] = to_f32(v.v[j]);
        sum += squares_of<kV>(f);
    }
    if (p.head && threadIdx.x < head) {
        const float f = to_f32(x[threadIdx.x]);
        sum += squares_of<1>(&f);
    }
    if (p.tail && threadIdx.x < n - p.until) {
        const float f = to_f32(x[p.until + threadIdx.x]);
        sum += squares_of<1>(&f);
    }
    return sum;
}

template <typename T> __device__ __forceinline__ void scale_piece(const T *x, T *y, uint64_t n, uint32_t chunk, uint32_t chunks, float by) {
    constexpr int kV = 16 / sizeof(T);
    const uint32_t head = head_of<T>(x, n);
    const Piece p = piece_of<T>(n, head, chunk, chunks);
    if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15u) == 0) {
#pragma unroll 4
        for (uint64_t i = p.from + threadIdx.x * kV; i < p.until; i += kListThreads * kV) {
            Pack<T, kV> v = *reinterpret_cast<const Pack<T, kV> *>(x + i);
#pragma unroll
            for (int j = 0; j < kV; ++j) v.v[j] = from_f32<T>(to_f32(v.v[j]) * by);
            *reinterpret_cast<Pack<T, kV> *>(y + i) = v;
        }
    } else {                                     // the two do not meet 16-byte boundaries together
#pragma unroll 4
        for (uint64_t i = p.from + threadIdx.x; i < p.until; i += kListThreads) y[i] = from_f32<T>(to_f32(x[i]) * by);
    }
    if (p.head && threadIdx.x < head) y[threadIdx.x] = from_f32<T>(to_f32(x[threadIdx.x]) * by);
    if (p.tail && threadIdx.x < n - p.until) y[p.until + threadIdx.x] = from_f32<T>(to_f32(x[p.until + threadIdx.x]) * by);
}

// The block's run of chunks, and the span that holds the first of them.
template <int kMost> struct Run {
    uint32_t at, until;
    int span;
    __device__ __forceinline__ explicit Run(const ListParams<kMost> &P) {
        at = static_cast<uint32_t>(static_cast<uint64_t>(P.chunks) * blockIdx.x / gridDim.x);
        until = static_cast<uint32_t>(static_cast<uint64_t>(P.chunks) * (blockIdx.x + 1) / gridDim.x);
    }
    __device__ __forceinline__ void find(const ListParams<kMost> &P, uint32_t chunk) {   // the last span that starts at or before it
        int lo = 0, hi = P.count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (P.first[mid] <= chunk) lo = mid;
            else hi = mid - 1;
        }
        span = lo;
    }
};

// Adds the blocks' sums, in their order, when all are there; fp64 of the block's own sum in every thread of the first warp.
template <int kMost> __global__ void __launch_bounds__(kListThreads) gradient_squares_kernel(const __grid_constant__ ListParams<kMost> P) {
    wait_for_previous();
    let_next_start();
    __shared__ double fold[kListThreads / 32];
    __shared__ bool last;
    Run<kMost> r(P);
    double sum = 0.0;
    if (r.at < r.until) r.find(P, r.at);
    for (; r.at < r.until; ++r.at) {
        while (r.at >= P.first[r.span + 1]) ++r.span;
        const uint32_t chunk = r.at - P.first[r.span], chunks = P.first[r.span + 1] - P.first[r.span];
        if (P.type[r.span] == LOCO_BF16) sum += square_piece(static_cast<const __nv_bfloat16 *>(P.x[r.span]), P.n[r.span], chunk, chunks);
        else sum += square_piece(static_cast<const float *>(P.x[r.span]), P.n[r.span], chunk, chunks);
    }
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    if (lane == 0) fold[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = lane < kListThreads / 32 ? fold[lane] : 0.0;
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    }
    if (threadIdx.x == 0) {
        P.part[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(P.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last || warp != 0) return;
    __threadfence();
    sum = 0.0;
    for (unsigned i = lane; i < gridDim.x; i += 32) sum += __ldcg(P.part + i);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    if (lane == 0) {
        if (!P.begin) sum += *P.running;
        if (P.end) *P.squares = sum;
        else *P.running = sum;
        *P.ticket = 0;
    }
}

template <int kMost> __global__ void __launch_bounds__(kListThreads) gradient_clip_kernel(const __grid_constant__ ListParams<kMost> P) {
    wait_for_previous();
    let_next_start();
    const double norm = sqrt(*P.in);
    if (P.begin && blockIdx.x == 0 && threadIdx.x == 0 && P.norm) *P.norm = static_cast<float>(norm);
    const float by = norm <= P.max_norm ? 1.0f : static_cast<float>(P.max_norm / norm);
    Run<kMost> r(P);
    if (r.at >= r.until) return;
    r.find(P, r.until - 1);
    for (uint32_t c = r.until; c-- > r.at;) {
        while (c < P.first[r.span]) --r.span;
        if (by == 1.0f && P.x[r.span] == P.y[r.span]) continue;
        const uint32_t chunk = c - P.first[r.span], chunks = P.first[r.span + 1] - P.first[r.span];
        if (P.type[r.span] == LOCO_BF16)
            scale_piece(static_cast<const __nv_bfloat16 *>(P.x[r.span]), static_cast<__nv_bfloat16 *>(P.y[r.span]), P.n[r.span], chunk, chunks, by);
        else scale_piece(static_cast<const float *>(P.x[r.span]), static_cast<float *>(P.y[r.span]), P.n[r.span], chunk, chunks, by);
    }
}

namespace {

int check_list(const loco_span_t *s, int32_t count, bool outputs) {
    if (count < 0 || (count > 0 && !s)) return LOCO_ERR_ARG;
    for (int32_t i = 0; i < count; ++i) {
        if (s[i].dtype != LOCO_F32 && s[i].dtype != LOCO_BF16) return LOCO_ERR_ARG;
        if (s[i].n > (1ull << 44)) return LOCO_ERR_ARG;
        if (s[i].n == 0) continue;
        if (!s[i].x || (outputs && !s[i].y)) return LOCO_ERR_ARG;
        const uintptr_t size = s[i].dtype == LOCO_BF16 ? 2 : 4;
        if (!aligned(s[i].x, size) || (outputs && !aligned(s[i].y, size))) return LOCO_ERR_ALIGN;
    }
    return LOCO_OK;
}

// Fills P with spans from `at` on; returns the first one that found no place.
template <int kMost> int32_t fill_list(ListParams<kMost> &P, const loco_span_t *s, int32_t count, int32_t at) {
    uint64_t chunks = 0;
    P.begin = at == 0;
    P.count = 0;
    for (; at < count && P.count < kMost; ++at) {
        if (s[at].n == 0) continue;
        const uint64_t bytes = s[at].n * (s[at].dtype == LOCO_BF16 ? 2 : 4), more = (bytes + kChunkBytes - 1) / kChunkBytes;
        if (chunks + more > 0xffffffffull) break;                    // 128 TB
        P.x[P.count] = s[at].x;
        P.y[P.count] = s[at].y;
        P.n[P.count] = s[at].n;
        P.type[P.count] = static_cast<uint8_t>(s[at].dtype);
        P.first[P.count++] = static_cast<uint32_t>(chunks);
        chunks += more;
    }
    P.first[P.count] = P.chunks = static_cast<uint32_t>(chunks);
    P.end = at == count;
    return at;
}

// One launch for as many spans as fit, in order.
template <int kMost, bool kClip> int launch_list(const loco_span_t *s, int32_t count, ListParams<kMost> &P, void *stream) {
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    int32_t at = 0;
    do {
        at = fill_list(P, s, count, at);
        const int64_t most = sms * 4 < kMostRuns ? sms * 4 : kMostRuns;
        const unsigned blocks = P.chunks < 1 ? 1 : P.chunks > most ? static_cast<unsigned>(most) : P.chunks;
        const int rc = launch_kernel(kClip ? gradient_clip_kernel<kMost> : gradient_squares_kernel<kMost>, dim3(blocks), kListThreads, 0, stream, P);
        if (rc != LOCO_OK) return rc;
    } while (at < count);
    return LOCO_OK;
}
template <bool kClip> int run_list(const loco_span_t *s, int32_t count, double max_norm, const double *in, double *squares, void *work, float *norm, void *stream) {
    const auto go = [&](auto &P) {
        P.max_norm = max_norm;
        P.in = in;
        P.squares = squares;
        P.ticket = static_cast<unsigned *>(work);
        P.running = reinterpret_cast<double *>(static_cast<uint8_t *>(work) + kTicketBytes);
        P.part = P.running + 1;
        P.norm = norm;
        return launch_list<std::decay_t<decltype(P)>::kSpans, kClip>(s, count, P, stream);
    };
    if (count <= kFewSpans) {
        ListParams<kFewSpans> P;
        return go(P);
    }
    ListParams<kMostSpans> P;
    return go(P);
}

}  // namespace

}  // namespace loco_layer

using namespace loco_layer;

extern "C" {

uint64_t loco_gradient_squares_workspace_bytes(void) { return kTicketBytes + (kMostRuns + 1) * sizeof(double); }

int loco_gradient_squares(const loco_span_t *spans, int32_t count, double *d_squares, void *d_work, uint64_t d_work_bytes, void *stream) {
    const int rc = check_list(spans, count, false);
    if (rc != LOCO_OK) return rc;
    if (!d_squares || !d_work) return LOCO_ERR_ARG;
    if (!aligned(d_squares, 8) || !aligned(d_work, 16)) return LOCO_ERR_ALIGN;
    if (d_work_bytes < loco_gradient_squares_workspace_bytes()) return LOCO_ERR_SIZE;
    return run_list<false>(spans, count, 0.0, nullptr, d_squares, d_work, nullptr, stream);
}

int loco_gradient_clip(const loco_span_t *spans, int32_t count, const double *d_squares, double max_norm, float *d_norm, void *stream) {
    const int rc = check_list(spans, count, true);
    if (rc != LOCO_OK) return rc;
    if (!d_squares || !(max_norm >= 0.0)) return LOCO_ERR_ARG;
    if (!aligned(d_squares, 8) || !aligned(d_norm, 4)) return LOCO_ERR_ALIGN;
    return run_list<true>(spans, count, max_norm, d_squares, nullptr, nullptr, d_norm, stream);
}

}  // extern "C"
