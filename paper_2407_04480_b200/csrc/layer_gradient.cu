// Sum of squares over a list of gradients, and the list scaled down to a largest norm.
//
// The list travels in the kernel's parameters.  It is cut into chunks; every block takes a run of consecutive chunks, finds
// the first by bisection and walks on from there.  HBM bounds both passes; the next chunks are on their way to shared memory
// (cp.async, every thread its own vectors, so that no barrier is needed) while one is worked on.  The second walks the list backwards, from
// what the first has read last, which L2 still holds; a list that fits there is read from HBM once.
#include <type_traits>

#include "layer_common.h"
#include "layer_tc.cuh"

namespace loco_layer {

constexpr int kListThreads = 512;
constexpr int kMostSpans = 768;                  // of a launch: 21 KB of parameters
constexpr int kFewSpans = 128;                   // 3.6 KB: a short list's launch costs less
constexpr int kChunkBytes = 32768;
constexpr int kAtOnce = kChunkBytes / 16 / kListThreads;             // vectors of a thread
constexpr int kAhead = 3;                        // chunks on their way, the one at work among them
constexpr size_t kListShared = static_cast<size_t>(kAhead) * kChunkBytes;
constexpr int kMostRuns = 4096;                  // blocks whose sums the workspace holds
// Chunks of a run: more blocks than run at once, of which the SMs that are nearer to memory take more, against what a block costs to
// start.  842 million bfloat16 elements, runs of 8, 16, 32: squares 308, 307, 290 us, scaling 537, 544, 567.
template <bool kClip> constexpr int kRunChunks = kClip ? 8 : 32;
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

// A chunk of a span: `count` vectors of 16 bytes from `at` on.  The elements before the first 16-byte boundary of x belong to the
// first chunk, those behind the last whole vector to the last.
template <typename T> struct Piece {
    static constexpr int kV = 16 / sizeof(T), kEach = kChunkBytes / 16;
    using Vec = Pack<T, kV>;
    uint64_t at;                                 // element
    int count, head, tail;
    uint64_t rest;                               // where the tail begins
    __host__ __device__ __forceinline__ Piece(const void *x, uint64_t n, uint32_t chunk, uint32_t chunks) {
        const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T);
        const uint64_t to_boundary = off ? kV - off : 0, before = to_boundary < n ? to_boundary : n;
        const uint64_t vectors = (n - before) / kV, skipped = static_cast<uint64_t>(chunk) * kEach, first = skipped < vectors ? skipped : vectors;
        at = before + first * kV;
        count = static_cast<int>(vectors - first < kEach ? vectors - first : kEach);
        head = chunk == 0 ? static_cast<int>(before) : 0;
        rest = before + vectors * kV;
        tail = chunk + 1 == chunks ? static_cast<int>(n - rest) : 0;
    }
    // What the copy of vector i names.  Past the vectors nothing is read, but an address has to be a boundary all the same: the one
    // at or before the span, which need not have a vector at all.
    __host__ __device__ __forceinline__ const uint4 *vector(const void *x, int i) const {
        return reinterpret_cast<const uint4 *>(i < count ? reinterpret_cast<uintptr_t>(static_cast<const T *>(x) + at) + i * 16ull : reinterpret_cast<uintptr_t>(x) & ~uintptr_t{15});
    }
};

// Chunks on their way: [chunk][vector][thread] of shared memory.  What lies past a chunk's vectors reads as zeros.
struct Ahead {
    uint4 *const at;
    int put = 0, got = 0;
    __device__ __forceinline__ explicit Ahead(void *shared) : at(static_cast<uint4 *>(shared) + threadIdx.x) {}
    template <typename T> __device__ __forceinline__ void send(const void *x, const Piece<T> &p) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = static_cast<int>(threadIdx.x) + u * kListThreads;
            const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(at + (put * kAtOnce + u) * kListThreads));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(p.vector(x, i)), "r"(i < p.count ? 16 : 0) : "memory");
        }
        if (++put == kAhead) put = 0;
    }
    // Of the chunks sent (none, too, counts as one) the oldest is there.
    __device__ __forceinline__ void wait() const { asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory"); }
    __device__ __forceinline__ static void sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    __device__ __forceinline__ uint4 operator[](int u) const { return at[(got * kAtOnce + u) * kListThreads]; }
    __device__ __forceinline__ void next() {
        if (++got == kAhead) got = 0;
    }
};

// Sum of squares of a vector in fp32, and whether there is anything in it but zeros.
template <typename T> __device__ __forceinline__ float squares_of(const uint4 &v, bool &some) {
    some = some || ((v.x | v.y | v.z | v.w) & (sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu)) != 0;
    float2 s = make_float2(0.0f, 0.0f);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w = (&v.x)[k];
            const float2 f = make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
            s = tc::fma2(f, f, s);
        }
    } else {
        const float2 f = make_float2(__uint_as_float(v.x), __uint_as_float(v.y)), g = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
        s = tc::fma2(g, g, tc::mul2(f, f));
    }
    return s.x + s.y;
}
template <typename T> __device__ __forceinline__ double square(T x) { return static_cast<double>(to_f32(x)) * static_cast<double>(to_f32(x)); }

template <typename T> __device__ __forceinline__ double square_piece(const T *x, const Piece<T> &p, const Ahead &ahead) {
    const int tid = threadIdx.x;
    // A thread's 32 (fp32: 16) squares are added in fp32, seven roundings in a row at most, and only then in 64 bits: a conversion and an
    // addition a vector kept the issue slots 78% busy.  Where the sum leaves fp32's range (values above 1e19 or below 1e-15) all
    // of it is done in 64 bits; zeros, of which an idle expert's gradient consists, are told apart.
    bool some = false;
    float group[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) group[u] = squares_of<T>(ahead[u], some);
    static_assert(kAtOnce == 4, "a tree of four");
    const float all = (group[0] + group[1]) + (group[2] + group[3]);
    double sum = static_cast<double>(all);
    if (some && !(all > 1e-30f && all < 3e38f)) {
        sum = 0.0;
#pragma unroll 1
        for (int i = tid; i < p.count; i += kListThreads)
#pragma unroll 1
            for (int j = 0; j < Piece<T>::kV; ++j) sum += square(x[p.at + static_cast<uint64_t>(i) * Piece<T>::kV + j]);
    }
    if (tid < p.head) sum += square(x[tid]);
    if (tid < p.tail) sum += square(x[p.rest + tid]);
    return sum;
}

template <typename T> __device__ __forceinline__ void scale_piece(const T *x, T *y, const Piece<T> &p, const Ahead &ahead, float by) {
    const int tid = threadIdx.x;
    if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15u) == 0) {
        uint4 *const to = reinterpret_cast<uint4 *>(y + p.at);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (tid + u * kListThreads < p.count) {
                uint4 v = ahead[u];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t &w = (&v.x)[k];
                    w = sizeof(T) == 2 ? tc::pack_bf16(__uint_as_float(w << 16) * by, __uint_as_float(w & 0xffff0000u) * by)
                                       : __float_as_uint(__uint_as_float(w) * by);
                }
                to[tid + u * kListThreads] = v;
            }
    } else {                                     // the two do not meet 16-byte boundaries together
#pragma unroll 4
        for (int i = tid; i < p.count * Piece<T>::kV; i += kListThreads) y[p.at + i] = from_f32<T>(to_f32(x[p.at + i]) * by);
    }
    if (tid < p.head) y[tid] = from_f32<T>(to_f32(x[tid]) * by);
    if (tid < p.tail) y[p.rest + tid] = from_f32<T>(to_f32(x[p.rest + tid]) * by);
}

// The block's run of chunks, and a place in it: a chunk and the span that holds it.
template <int kMost> struct Run {
    uint32_t first, until;
    __device__ __forceinline__ Run(const ListParams<kMost> &P, uint32_t which) {
        first = static_cast<uint32_t>(static_cast<uint64_t>(P.chunks) * which / gridDim.x);
        until = static_cast<uint32_t>(static_cast<uint64_t>(P.chunks) * (which + 1) / gridDim.x);
    }
};
template <int kMost> __device__ __forceinline__ int span_of(const ListParams<kMost> &P, uint32_t chunk) {      // the last span that starts at or before it
    int lo = 0, hi = P.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (P.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
template <typename T, int kMost> __device__ __forceinline__ Piece<T> piece_at(const ListParams<kMost> &P, int span, uint32_t chunk) {
    return Piece<T>(P.x[span], P.n[span], chunk - P.first[span], P.first[span + 1] - P.first[span]);
}
template <int kMost> __device__ __forceinline__ void send_chunk(const ListParams<kMost> &P, int span, uint32_t chunk, Ahead &ahead) {
    if (P.type[span] == LOCO_BF16) ahead.send(P.x[span], piece_at<__nv_bfloat16>(P, span, chunk));
    else ahead.send(P.x[span], piece_at<float>(P, span, chunk));
}

// Adds the blocks' sums, in their order, when all are there; fp64 of the block's own sum in every thread of the first warp.
template <int kMost> __global__ void __launch_bounds__(kListThreads, 2) gradient_squares_kernel(const __grid_constant__ ListParams<kMost> P) {
    wait_for_previous();
    let_next_start();
    __shared__ double fold[kListThreads / 32];
    __shared__ bool last;
    extern __shared__ __align__(16) uint8_t shared[];
    const Run<kMost> run(P, blockIdx.x);
    Ahead ahead(shared);
    double sum = 0.0;
    int span = run.first < run.until ? span_of(P, run.first) : 0, next_span = span;
    uint32_t next = run.first;
    const auto send = [&] {
        if (next < run.until) {
            while (next >= P.first[next_span + 1]) ++next_span;
            send_chunk(P, next_span, next++, ahead);
        }
        ahead.sent();
    };
    for (int i = 1; i < kAhead; ++i) send();
    for (uint32_t c = run.first; c < run.until; ++c) {
        while (c >= P.first[span + 1]) ++span;
        send();
        ahead.wait();
        if (P.type[span] == LOCO_BF16) sum += square_piece(static_cast<const __nv_bfloat16 *>(P.x[span]), piece_at<__nv_bfloat16>(P, span, c), ahead);
        else sum += square_piece(static_cast<const float *>(P.x[span]), piece_at<float>(P, span, c), ahead);
        ahead.next();
    }
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    if (lane == 0) fold[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = lane < kListThreads / 32 ? fold[lane] : 0.0;
#pragma unroll
        for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    }
    if (threadIdx.x == 0) {
        P.part[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(P.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kListThreads) sum += __ldcg(P.part + i);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    if (lane == 0) fold[warp] = sum;
    __syncthreads();
    if (warp != 0) return;
    sum = lane < kListThreads / 32 ? fold[lane] : 0.0;
#pragma unroll
    for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    if (lane == 0) {
        if (!P.begin) sum += *P.running;
        if (P.end) *P.squares = sum;
        else *P.running = sum;
        *P.ticket = 0;
    }
}

template <int kMost> __global__ void __launch_bounds__(kListThreads, 2) gradient_clip_kernel(const __grid_constant__ ListParams<kMost> P) {
    wait_for_previous();
    let_next_start();
    const double norm = sqrt(*P.in);
    if (P.begin && blockIdx.x == 0 && threadIdx.x == 0 && P.norm) *P.norm = static_cast<float>(norm);
    const float by = norm <= P.max_norm ? 1.0f : static_cast<float>(P.max_norm / norm);
    extern __shared__ __align__(16) uint8_t shared[];
    const Run<kMost> run(P, gridDim.x - 1 - blockIdx.x);
    if (run.first >= run.until) return;
    Ahead ahead(shared);
    int span = span_of(P, run.until - 1), next_span = span;
    uint32_t next = run.until;
    const auto kept = [&](int span) { return by == 1.0f && P.x[span] == P.y[span]; };
    const auto send = [&] {
        if (next > run.first) {
            --next;
            while (next < P.first[next_span]) --next_span;
            if (!kept(next_span)) send_chunk(P, next_span, next, ahead);
        }
        ahead.sent();
    };
    for (int i = 1; i < kAhead; ++i) send();
    for (uint32_t c = run.until; c-- > run.first;) {
        while (c < P.first[span]) --span;
        send();
        if (kept(span)) continue;
        ahead.wait();
        if (P.type[span] == LOCO_BF16)
            scale_piece(static_cast<const __nv_bfloat16 *>(P.x[span]), static_cast<__nv_bfloat16 *>(P.y[span]), piece_at<__nv_bfloat16>(P, span, c), ahead, by);
        else scale_piece(static_cast<const float *>(P.x[span]), static_cast<float *>(P.y[span]), piece_at<float>(P, span, c), ahead, by);
        ahead.next();
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

// Shared memory above the default limit, set once per device and kernel.
template <int kMost, bool kClip> bool allow() {
    static std::atomic<bool> set[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return false;
    }
    if (set[dev].load(std::memory_order_acquire)) return true;
    const auto fn = kClip ? gradient_clip_kernel<kMost> : gradient_squares_kernel<kMost>;
    if (cudaFuncSetAttribute(reinterpret_cast<const void *>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kListShared)) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    set[dev].store(true, std::memory_order_release);
    return true;
}

// One launch for as many spans as fit, in order.
template <int kMost, bool kClip> int launch_list(const loco_span_t *s, int32_t count, ListParams<kMost> &P, void *stream) {
    const int sms = sm_count();
    if (sms == 0 || !allow<kMost, kClip>()) return LOCO_ERR_CUDA;
    int32_t at = 0;
    do {
        at = fill_list(P, s, count, at);
        const int64_t few = sms * 2, runs = P.chunks <= few ? P.chunks : P.chunks / kRunChunks<kClip> < few ? few : P.chunks / kRunChunks<kClip>;
        const unsigned blocks = runs < 1 ? 1 : runs > kMostRuns ? kMostRuns : static_cast<unsigned>(runs);
        const int rc = launch_kernel(kClip ? gradient_clip_kernel<kMost> : gradient_squares_kernel<kMost>, dim3(blocks), kListThreads, kListShared, stream, P);
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
