// Root-mean-square norm with the residual's addition, and its gradient: a row is read once into registers by a team of
// threads, summed over the team and written.
//
// Some ten operations per element read, so the bound is HBM.  A team is 4 to 32 lanes for short rows and up to a block's 1024
// threads for long ones; a block holds as many teams as fit, its blocks go round the rows, and the weight stays in registers
// from row to row.  The next row is on its way while one is worked on: every thread copies its own part of it to shared
// memory (cp.async) and reads nobody else's, so the copies need no barrier.  With the next row in registers instead the
// backward kernel spilled what it waited for: 8192 rows of 4096, bfloat16, 99 us.
//
// bfloat16 with residual, 16384 x 5120: 105 us, 6.4 TB/s; 300,000 x 128: 50 us, 6.1 TB/s; 50,003 x 1367, whose rows begin anywhere,
// 109 us, 5.0 TB/s; 16384 x 4096 to 8 bits 96 us, 4.9 TB/s: there the instructions bound it, some thirty for two elements.  Backward 8192 x 4096:
// 45 us, 6.0 TB/s, and 6 for the sum of the blocks' parts of dw; 20,000 x 4096 in fp32 193 us, 6.8 TB/s.
#include <cuda_fp8.h>

#include <cstring>

#include "layer_common.h"
#include "layer_tc.cuh"

namespace loco_layer {

constexpr int kMaxDim = 16384;
constexpr int kNormThreads = 1024;               // most threads of a block, and threads of an SM
constexpr int kBlockThreads = 512;               // of a block of several teams
constexpr int kPartials = 444;                   // most blocks of the backward kernel, each leaves a partial row of dw
constexpr int kScaleBlock = 128;
constexpr int kRingBytes = 200 * 1024;           // shared memory of an SM for rows on their way
constexpr float kLargestE4m3 = 448.0f, kLeastScale = 1.17549435e-38f;
constexpr unsigned kAll = 0xffffffffu;

struct NormParams {
    const void *x, *r, *w, *dy, *dt;             // x: h in the backward pass
    void *h, *y, *dx;
    float *scale, *part;
    int64_t xs, rs, hs, ys, dys, dts, dxs, rows;
    int32_t dim, team, block, groups, wanted, depth;
    float eps, over_dim;
};

// The threads that share a row: a part of a warp, or several warps, which then have a barrier of their own.
struct Team {
    int size, lane, mine, all;                   // threads, this one's place; the team's place in the block, teams
    int shift;                                   // elements between the 16-byte boundary before a row and the row, the same for all of the team's
    __device__ __forceinline__ Team(const NormParams &P, int vec)
        : size(P.team), lane(static_cast<int>(threadIdx.x) % P.team), mine(static_cast<int>(threadIdx.x) / P.team), all(static_cast<int>(blockDim.x) / P.team),
          shift(static_cast<int>((static_cast<int64_t>(blockIdx.x) * all + mine) * P.xs % vec)) {}
    __device__ __forceinline__ void sync() const {
        if (size > 32) asm volatile("bar.sync %0, %1;" ::"r"(mine + 1), "r"(size) : "memory");
        else __syncwarp();
    }
};

// Sums over the team, the same in every lane of it.  `fold` has a place for every warp of the block, twice: a row's sums go to the
// one side, the next row's to the other, so that one barrier a row will do.
__device__ __forceinline__ float2 team_sum(float2 s, const Team &t, float2 *fold) {
    for (int o = (t.size < 32 ? t.size : 32) / 2; o; o >>= 1) {
        s.x += __shfl_xor_sync(kAll, s.x, o);
        s.y += __shfl_xor_sync(kAll, s.y, o);
    }
    if (t.size > 32) {
        const int warps = t.size / 32, first = t.mine * warps;
        if (threadIdx.x % 32 == 0) fold[threadIdx.x / 32] = s;
        t.sync();
        s = threadIdx.x % 32 < warps ? fold[first + threadIdx.x % 32] : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            s.x += __shfl_xor_sync(kAll, s.x, o);
            s.y += __shfl_xor_sync(kAll, s.y, o);
        }
    }
    return s;
}
__device__ __forceinline__ float team_sum(float s, const Team &t, float2 *fold) {
    for (int o = (t.size < 32 ? t.size : 32) / 2; o; o >>= 1) s += __shfl_xor_sync(kAll, s, o);
    if (t.size > 32) {
        const int warps = t.size / 32, first = t.mine * warps;
        if (threadIdx.x % 32 == 0) fold[threadIdx.x / 32].x = s;
        t.sync();
        s = threadIdx.x % 32 < warps ? fold[first + threadIdx.x % 32].x : 0.0f;
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kAll, s, o);
    }
    return s;
}
// Largest of the bits of values without a sign: their order is that of the values, NaN above infinity.  Between two calls there
// is a barrier of the team, that of the row's sum.
__device__ __forceinline__ unsigned team_max(unsigned m, const Team &t, unsigned *fold) {
    for (int o = (t.size < 32 ? t.size : 32) / 2; o; o >>= 1) m = max(m, __shfl_xor_sync(kAll, m, o));
    if (t.size > 32) {
        const int warps = t.size / 32, first = t.mine * warps;
        if (threadIdx.x % 32 == 0) fold[threadIdx.x / 32] = m;
        t.sync();
        m = threadIdx.x % 32 < warps ? fold[first + threadIdx.x % 32] : 0;
#pragma unroll
        for (int o = 16; o; o >>= 1) m = max(m, __shfl_xor_sync(kAll, m, o));
    }
    return m;
}
// An 8-bit scale from the largest |h w| of its columns and the row's r: max |y| / 448.  y / scale is then (h w) (448 / max |h w|), r
// leaves it, and h w of bfloat16 is exact in fp32: with 448 / max in two fp32 (`over`, `rest`) the value is rounded once before it
// is rounded to 8 bits, and falls on the wrong side of a step where the exact one is within 2^-24 of it.
struct Scale {
    float scale, over, rest, then;               // then: 1, what `over` is off by, or, where the scale is its least value, over it
    __device__ __forceinline__ Scale(unsigned largest, float r) {
        const float m = __uint_as_float(largest), s = m * r / kLargestE4m3;
        if (s > kLeastScale) {
            // below 1.3e-36 the quotient leaves fp32's range, though a large r keeps the scale above its least value: there both are 2^64 off
            const float up = m < 0x1p-64f ? 0x1p64f : 1.0f, n = m * up;
            scale = s;
            over = kLargestE4m3 / n;
            rest = fmaf(-over, n, kLargestE4m3) / n;
            then = up;
        } else {                                 // nothing there, or NaN
            scale = s != s ? s : kLeastScale;
            over = r;
            rest = 0.0f;
            then = 1.0f / kLeastScale;
        }
    }
    // y / scale; fp32: what h w was rounded by is taken along
    template <typename T> __device__ __forceinline__ float2 apply(float2 h, float2 w) const {
        const float2 p = tc::mul2(h, w), o = make_float2(over, over);
        float2 low = tc::mul2(p, make_float2(rest, rest));
        if constexpr (sizeof(T) == 4) low = tc::fma2(tc::fma2(h, w, make_float2(-p.x, -p.y)), o, low);
        return tc::mul2(tc::fma2(p, o, low), make_float2(then, then));
    }
};

// A thread's part of a row: kMine elements in vectors of V, dealt to the team in turn.  Vectors lie on the tensors' 16-byte
// boundaries, so that rows of any width are read and written in whole vectors but for the two that hold a row's ends (kShift;
// without, every row begins and ends on a boundary).
// Elements are taken two at a time: bfloat16 is converted in pairs, and the sums and products are two to an instruction.
template <typename T, int V, int kMine, bool kShift> struct Part {
    static constexpr int kVecs = kMine / V, kPairs = kMine / 2;
    using Vec = Pack<T, V>;
    Vec v[kVecs];
    __device__ __forceinline__ static int column(const Team &t, int i) { return (i * t.size + t.lane) * V - (kShift ? t.shift : 0); }
    __device__ __forceinline__ static bool inside(const Team &t, int i, int dim) { return column(t, i) < dim; }         // a part of it at least
    __device__ __forceinline__ static bool whole(const Team &t, int i, int dim) { return !kShift || (column(t, i) >= 0 && column(t, i) + V <= dim); }
    __device__ __forceinline__ void fill(float x) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) v[i].v[j] = from_f32<T>(x);
    }
    // element by element where the row's ends are; columns past the row keep what they were filled with
    __device__ __forceinline__ void load(const T *row, const Team &t, int dim, bool vectors) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (inside(t, i, dim)) {
                if (vectors && whole(t, i, dim)) {
                    v[i] = *reinterpret_cast<const Vec *>(row + column(t, i));
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (static_cast<unsigned>(column(t, i) + j) < static_cast<unsigned>(dim)) v[i].v[j] = row[column(t, i) + j];
                }
            }
    }
    __device__ __forceinline__ void store(T *row, const Team &t, int dim) const {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (inside(t, i, dim)) {
                if (whole(t, i, dim)) {
                    *reinterpret_cast<Vec *>(row + column(t, i)) = v[i];
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (static_cast<unsigned>(column(t, i) + j) < static_cast<unsigned>(dim)) row[column(t, i) + j] = v[i].v[j];
                }
            }
    }
    // zeros where a vector reaches past the row's ends
    __device__ __forceinline__ void trim(const Team &t, int dim) {
        if constexpr (kShift)
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
                if (!whole(t, i, dim))
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (static_cast<unsigned>(column(t, i) + j) >= static_cast<unsigned>(dim)) v[i].v[j] = from_f32<T>(0.0f);
    }
    __device__ __forceinline__ float2 operator[](int q) const {
        if constexpr (V > 1 && sizeof(T) == 2) {
            uint32_t w;
            memcpy(&w, &v[2 * q / V].v[2 * q % V], 4);
            return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        } else {
            return make_float2(to_f32(v[2 * q / V].v[2 * q % V]), to_f32(v[(2 * q + 1) / V].v[(2 * q + 1) % V]));
        }
    }
    // Keeps pairs of bfloat16 as they are: what is converted before is converted again after, and holds no registers between.
    __device__ __forceinline__ void keep() {
        if constexpr (V > 1 && sizeof(T) == 2)
#pragma unroll
            for (int q = 0; q < kPairs; ++q) {
                uint32_t w;
                memcpy(&w, &v[2 * q / V].v[2 * q % V], 4);
                asm volatile("" : "+r"(w));
                memcpy(&v[2 * q / V].v[2 * q % V], &w, 4);
            }
    }
    __device__ __forceinline__ void set(int q, float2 f) {
        if constexpr (V > 1 && sizeof(T) == 2) {
            const uint32_t w = tc::pack_bf16(f.x, f.y);
            memcpy(&v[2 * q / V].v[2 * q % V], &w, 4);
        } else {
            v[2 * q / V].v[2 * q % V] = from_f32<T>(f.x);
            v[(2 * q + 1) / V].v[(2 * q + 1) % V] = from_f32<T>(f.y);
        }
    }
};
template <typename T> __device__ __forceinline__ const T *row_at(const void *p, int64_t row, int64_t stride) { return static_cast<const T *>(p) + row * stride; }
template <typename T> __device__ __forceinline__ T *row_at(void *p, int64_t row, int64_t stride) { return static_cast<T *>(p) + row * stride; }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// The rows on their way: for each of `depth` of them the thread's vectors of kTensors tensors, [row][tensor][vector][thread].
// Single elements (tensors that do not share their boundaries) are read where they are needed instead.
template <typename T, int V, int kMine, bool kShift, int kTensors> struct Ring {
    using Row = Part<T, V, kMine, kShift>;
    using Vec = typename Row::Vec;
    static constexpr bool kCopies = V > 1;
    Vec *const at;
    const int depth;
    int put = 0, got = 0;
    __device__ __forceinline__ Ring(void *shared, int rows) : at(static_cast<Vec *>(shared) + threadIdx.x), depth(rows) {}
    __device__ __forceinline__ Vec *place(int slot, int tensor, int i) const { return at + ((slot * kTensors + tensor) * Row::kVecs + i) * static_cast<int>(blockDim.x); }
    // A vector with the row's begin has the end of the row before in it (the first row of a tensor begins on a boundary); of the
    // one with its end only what is the row's is read.
    __device__ __forceinline__ void copy(int tensor, const T *row, const Team &t, int dim, bool there) {
        if constexpr (kCopies) {
#pragma unroll
            for (int i = 0; i < Row::kVecs; ++i) {
                const int left = there ? (dim - Row::column(t, i)) * static_cast<int>(sizeof(T)) : 0, bytes = left < 0 ? 0 : left > 16 ? 16 : left;
                const T *from = bytes ? row + Row::column(t, i) : none;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_addr(place(put, tensor, i))), "l"(from), "r"(bytes) : "memory");
            }
        }
    }
    const T *none;                               // any address that may be named; nothing is read there
    __device__ __forceinline__ void sent() {
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++put == depth) put = 0;
    }
    // the oldest row is there; `depth` rows have been sent
    __device__ __forceinline__ void wait() const {
        if (depth == 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
        else if (depth == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 2;" ::: "memory");
    }
    __device__ __forceinline__ void next() {
        if (++got == depth) got = 0;
    }
    __device__ __forceinline__ void read(Row &r, int tensor) const {
#pragma unroll
        for (int i = 0; i < Row::kVecs; ++i) r.v[i] = *place(got, tensor, i);
    }
};

template <typename T, int V, int kMine, bool kShift, bool kBits8>
__global__ void __launch_bounds__(kNormThreads) norm_forward_kernel(const __grid_constant__ NormParams P) {
    wait_for_previous();
    let_next_start();
    using Row = Part<T, V, kMine, kShift>;
    extern __shared__ __align__(16) uint8_t shared[];
    __shared__ float2 fold[2][kNormThreads / 32];
    __shared__ unsigned tops[kBits8 ? kNormThreads / 32 : 1];        // not `fold`, which another team may be at
    __shared__ unsigned most[kBits8 ? 256 : 1];  // a row's or several rows' runs of 128 columns: threads * kMine / 128 of them at most
    const Team t(P, V);
    Ring<T, V, kMine, kShift, 2> ring(shared, P.depth);
    ring.none = static_cast<const T *>(P.x);
    Row w;
    w.fill(1.0f);
    if (P.w) w.load(static_cast<const T *>(P.w), t, P.dim, t.shift == 0);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * t.all, mine = static_cast<int64_t>(blockIdx.x) * t.all + t.mine;
    int64_t ahead = mine;
    const auto send = [&]() {
        ring.copy(0, row_at<T>(P.x, ahead, P.xs), t, P.dim, ahead < P.rows);
        if (P.r) ring.copy(1, row_at<T>(P.r, ahead, P.rs), t, P.dim, ahead < P.rows);
        ring.sent();
        ahead += stride;
    };
    for (int i = 1; i < P.depth; ++i) send();
    int64_t row = mine;
    int side = 0;
    for (int64_t first = row - t.mine; first < P.rows; first += stride, row += stride, side ^= 1) {
        const bool there = row < P.rows;
        send();
        Row h;
        if constexpr (Ring<T, V, kMine, kShift, 2>::kCopies) {
            ring.wait();
            ring.read(h, 0);
            h.trim(t, P.dim);
        } else {
            h.fill(0.0f);
            if (there) h.load(row_at<T>(P.x, row, P.xs), t, P.dim, true);
        }
        if (P.r) {
            Row r;
            if constexpr (Ring<T, V, kMine, kShift, 2>::kCopies) {
                ring.read(r, 1);
                r.trim(t, P.dim);
            } else {
                r.fill(0.0f);
                if (there) r.load(row_at<T>(P.r, row, P.rs), t, P.dim, true);
            }
#pragma unroll
            for (int q = 0; q < Row::kPairs; ++q) h.set(q, tc::add2(h[q], r[q]));
            if (there) h.store(row_at<T>(P.h, row, P.hs), t, P.dim);
        }
        ring.next();
        float2 sum = both(0.0f);
#pragma unroll
        for (int q = 0; q < Row::kPairs; ++q) sum = tc::fma2(h[q], h[q], sum);
        h.keep();
        const float by = rsqrtf(team_sum(sum.x + sum.y, t, fold[side]) * P.over_dim + P.eps);
        h.keep();
        w.keep();
        if constexpr (!kBits8) {
#pragma unroll
            for (int q = 0; q < Row::kPairs; ++q) h.set(q, tc::mul2(tc::mul2(h[q], both(by)), w[q]));
            if (there) h.store(row_at<T>(P.y, row, P.ys), t, P.dim);
        } else {
            const auto y = [&](int q) { return tc::mul2(h[q], w[q]); };          // but for r
            uint32_t out[kMine / 4] = {};        // a byte an element
            const auto pack = [&](int q, float2 f) {
                const uint32_t e = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
                out[q / 2] = q % 2 ? out[q / 2] | e << 16 : e;
            };
            // the largest of the row, or of each run of 128 columns: 16 lanes' vectors where rows begin on the boundaries
            constexpr bool kLanes = V == 8 && !kShift;
            const bool lanes = kLanes && t.size >= 32;
            if (P.block == 0 || lanes) {
                unsigned m[Row::kVecs], all = 0;
#pragma unroll
                for (int i = 0; i < Row::kVecs; ++i) {
                    float x = 0.0f;                                  // NaN where one is
                    if constexpr (V == 1) {
                        const float2 f = y(i / 2);
                        x = fabsf(i % 2 ? f.y : f.x);
                    } else {
#pragma unroll
                        for (int q = i * V / 2; q < (i + 1) * V / 2; ++q) {
                            const float2 f = y(q);
                            x = tc::max3(x, fabsf(f.x), fabsf(f.y));
                        }
                    }
                    m[i] = __float_as_uint(x);
                }
                if (P.block == 0) {
#pragma unroll
                    for (int i = 0; i < Row::kVecs; ++i) all = max(all, m[i]);
                    const Scale s(team_max(all, t, tops), by);
                    if (there && t.lane == 0) P.scale[row] = s.scale;
#pragma unroll
                    for (int q = 0; q < Row::kPairs; ++q) pack(q, s.apply<T>(h[q], w[q]));
                } else if constexpr (kLanes) {
#pragma unroll
                    for (int i = 0; i < Row::kVecs; ++i) {
#pragma unroll
                        for (int o = 8; o; o >>= 1) m[i] = max(m[i], __shfl_xor_sync(kAll, m[i], o));
                        const Scale s(m[i], by);
                        if (there && threadIdx.x % 16 == 0 && Row::inside(t, i, P.dim)) P.scale[row * P.groups + Row::column(t, i) / kScaleBlock] = s.scale;
#pragma unroll
                        for (int q = i * V / 2; q < (i + 1) * V / 2; ++q) pack(q, s.apply<T>(h[q], w[q]));
                    }
                }
            } else {
                unsigned *const mine = most + t.mine * P.groups;
                const auto run = [&](int i, int j) { return min(max(Row::column(t, i) + j, 0) / kScaleBlock, P.groups - 1); };
                if (t.size <= 32) __syncwarp();  // what the row before left has been read; larger teams know from the sum's barrier
                for (int i = t.lane; i < P.groups; i += t.size) mine[i] = 0;
                t.sync();
#pragma unroll
                for (int q = 0; q < Row::kPairs; ++q) {              // past the row there are zeros
                    const float2 f = y(q);
                    atomicMax(&mine[run(2 * q / V, 2 * q % V)], __float_as_uint(f.x) & 0x7fffffffu);
                    atomicMax(&mine[run((2 * q + 1) / V, (2 * q + 1) % V)], __float_as_uint(f.y) & 0x7fffffffu);
                }
                t.sync();
                for (int i = t.lane; i < P.groups && there; i += t.size) P.scale[row * P.groups + i] = Scale(mine[i], by).scale;
#pragma unroll
                for (int q = 0; q < Row::kPairs; ++q) {
                    const Scale a(mine[run(2 * q / V, 2 * q % V)], by), b(mine[run((2 * q + 1) / V, (2 * q + 1) % V)], by);
                    pack(q, make_float2(a.apply<T>(h[q], w[q]).x, b.apply<T>(h[q], w[q]).y));
                }
            }
            if (there) {
                uint8_t *const to = row_at<uint8_t>(P.y, row, P.ys);
#pragma unroll
                for (int i = 0; i < Row::kVecs; ++i)
                    if (Row::inside(t, i, P.dim)) {
                        if (V > 1 && Row::whole(t, i, P.dim)) {
                            if constexpr (V == 8) *reinterpret_cast<uint2 *>(to + Row::column(t, i)) = make_uint2(out[2 * i], out[2 * i + 1]);
                            else if constexpr (V == 4) *reinterpret_cast<uint32_t *>(to + Row::column(t, i)) = out[i];
                        } else {
#pragma unroll
                            for (int j = 0; j < V; ++j)
                                if (static_cast<unsigned>(Row::column(t, i) + j) < static_cast<unsigned>(P.dim))
                                    to[Row::column(t, i) + j] = static_cast<uint8_t>(out[(i * V + j) / 4] >> (i * V + j) % 4 * 8);
                        }
                    }
            }
        }
    }
}

// dx of every row, and over the block's rows the sums of dy n, each thread its own columns'.
template <typename T, int V, int kMine, bool kShift> __global__ void __launch_bounds__(kNormThreads) norm_backward_kernel(const __grid_constant__ NormParams P) {
    wait_for_previous();
    let_next_start();
    using Row = Part<T, V, kMine, kShift>;
    using Rows = Ring<T, V, kMine, kShift, 3>;           // what the norm was of, its output's gradient, the one past it
    extern __shared__ __align__(16) uint8_t shared[];
    __shared__ float2 fold[2][kNormThreads / 32];
    const Team t(P, V);
    Rows ring(shared, P.depth);
    ring.none = static_cast<const T *>(P.x);
    Row w;
    w.fill(1.0f);
    if (P.w) w.load(static_cast<const T *>(P.w), t, P.dim, t.shift == 0);
    float2 dw[Row::kPairs];
#pragma unroll
    for (int q = 0; q < Row::kPairs; ++q) dw[q] = both(0.0f);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * t.all, mine = static_cast<int64_t>(blockIdx.x) * t.all + t.mine;
    int64_t ahead = mine;
    const auto send = [&]() {
        ring.copy(0, row_at<T>(P.x, ahead, P.xs), t, P.dim, ahead < P.rows);
        ring.copy(1, row_at<T>(P.dy, ahead, P.dys), t, P.dim, ahead < P.rows);
        if (P.dt) ring.copy(2, row_at<T>(P.dt, ahead, P.dts), t, P.dim, ahead < P.rows);
        ring.sent();
        ahead += stride;
    };
    for (int i = 1; i < P.depth; ++i) send();
    int64_t row = mine;
    int side = 0;
    for (int64_t first = row - t.mine; first < P.rows; first += stride, row += stride) {
        const bool there = row < P.rows;
        send();
        Row f, e, out;
        if constexpr (Rows::kCopies) {
            ring.wait();
            ring.read(f, 0);
            ring.read(e, 1);
            f.trim(t, P.dim);
            e.trim(t, P.dim);
        } else {
            f.fill(0.0f);
            e.fill(0.0f);
            if (there) {
                f.load(row_at<T>(P.x, row, P.xs), t, P.dim, true);
                e.load(row_at<T>(P.dy, row, P.dys), t, P.dim, true);
            }
        }
        float2 squares = both(0.0f), dots = both(0.0f);              // of h^2 and of dy w h
#pragma unroll
        for (int q = 0; q < Row::kPairs; ++q) {
            squares = tc::fma2(f[q], f[q], squares);
            dots = tc::fma2(f[q], tc::mul2(e[q], w[q]), dots);
        }
        f.keep();
        e.keep();
        w.keep();
        // fp32 has no register to spare for the side, and takes a barrier more: 20000 x 4096, 198 us against 203; bfloat16, 4000 x 16384: 112, 109.
        if constexpr (sizeof(T) == 4) t.sync();
        const float2 sum = team_sum(make_float2(squares.x + squares.y, dots.x + dots.y), t, fold[side]);
        if constexpr (sizeof(T) == 2) side ^= 1;
        const float by = rsqrtf(sum.x * P.over_dim + P.eps), pull = -sum.y * P.over_dim * by * by;
        out.fill(0.0f);
        if (P.dt) {
            if constexpr (Rows::kCopies) ring.read(out, 2);
            else if (there) out.load(row_at<T>(P.dt, row, P.dts), t, P.dim, true);
        }
        if (there) {
#pragma unroll
            for (int q = 0; q < Row::kPairs; ++q) {
                dw[q] = tc::fma2(e[q], tc::mul2(f[q], both(by)), dw[q]);
                out.set(q, tc::fma2(tc::fma2(f[q], both(pull), tc::mul2(e[q], w[q])), both(by), out[q]));
            }
            out.store(row_at<T>(P.dx, row, P.dxs), t, P.dim);
        }
        ring.next();
    }
    if (!P.wanted) return;
    float *const part = P.part + static_cast<int64_t>(blockIdx.x) * P.dim, *const sums = reinterpret_cast<float *>(shared);
    float *const to = t.all == 1 ? part : sums + t.mine * P.dim;
    asm volatile("cp.async.wait_group 0;" ::: "memory");             // the ring's memory holds the teams' sums now
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = Row::column(t, i / V) + i % V;
        if (static_cast<unsigned>(at) < static_cast<unsigned>(P.dim)) to[at] = i % 2 ? dw[i / 2].y : dw[i / 2].x;
    }
    if (t.all == 1) return;
    __syncthreads();
    for (int c = threadIdx.x; c < P.dim; c += blockDim.x) {
        float s = 0.0f;
        for (int i = 0; i < t.all; ++i) s += sums[i * P.dim + c];
        part[c] = s;
    }
}

// The blocks' partial rows added in their order: 32 columns to a block, 16 warps that each take a part of the rows, five of them asked
// for at once and none left over (by a loop unrolled ten times with a rest both gradients of 300,000 x 128 took 60.4 us, so 57.8; by 32 warps 57.4, but
// 64 x 4096 9.6 against 7.2).
constexpr int kWeightWarps = 16, kWeightRows = 5;
template <typename T> __global__ void __launch_bounds__(kWeightWarps * 32) norm_weight_kernel(const float *part, int blocks, int dim, T *dw) {
    wait_for_previous();
    let_next_start();
    __shared__ float fold[kWeightWarps][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = static_cast<int>(blockIdx.x) * 32 + lane;
    const int per = (blocks + kWeightWarps - 1) / kWeightWarps, from = warp * per, until = min(from + per, blocks);
    float s = 0.0f;
    if (c < dim)
        for (int b = from; b < until; b += kWeightRows) {
            float x[kWeightRows];
#pragma unroll
            for (int u = 0; u < kWeightRows; ++u) x[u] = b + u < until ? part[static_cast<int64_t>(b + u) * dim + c] : 0.0f;
#pragma unroll
            for (int u = 0; u < kWeightRows; ++u) s += x[u];
        }
    fold[warp][lane] = s;
    __syncthreads();
    s = fold[lane % kWeightWarps][warp * 2 + lane / kWeightWarps];   // warp w adds columns 2w and 2w + 1
#pragma unroll
    for (int o = kWeightWarps / 2; o; o >>= 1) s += __shfl_xor_sync(kAll, s, o);
    const int column = static_cast<int>(blockIdx.x) * 32 + warp * 2 + lane / kWeightWarps;
    if (lane % kWeightWarps == 0 && column < dim) dw[column] = from_f32<T>(s);
}

namespace {

using NormKernel = void (*)(const NormParams);

template <typename T, int V, int kMine, bool kShift> NormKernel pick_norm(bool backward, bool bits8) {
    if (backward) return norm_backward_kernel<T, V, kMine, kShift>;
    return bits8 ? norm_forward_kernel<T, V, kMine, kShift, true> : norm_forward_kernel<T, V, kMine, kShift, false>;
}
template <typename T, int V> NormKernel pick_norm(int mine, bool shift, bool backward, bool bits8) {
    if constexpr (V > 1) {
        if constexpr (sizeof(T) == 4)
            if (mine == 8) return shift ? pick_norm<T, V, 8, true>(backward, bits8) : pick_norm<T, V, 8, false>(backward, bits8);
        return shift ? pick_norm<T, V, 16, true>(backward, bits8) : pick_norm<T, V, 16, false>(backward, bits8);
    } else {
        if constexpr (sizeof(T) == 4)
            if (mine == 8) return pick_norm<T, V, 8, false>(backward, bits8);
        return pick_norm<T, V, 16, false>(backward, bits8);
    }
}

int check_norm(const loco_norm_t *c) {
    if (!c) return LOCO_ERR_ARG;
    if (c->dtype != LOCO_F32 && c->dtype != LOCO_BF16) return LOCO_ERR_ARG;
    if (c->dim < 1 || !(c->eps >= 0.0f) || !std::isfinite(c->eps)) return LOCO_ERR_ARG;
    if (c->bits8 && c->block != 0 && c->block != kScaleBlock) return LOCO_ERR_ARG;
    return c->dim > kMaxDim ? LOCO_ERR_UNSUPPORTED : LOCO_OK;
}

// Whether a call's rows can be taken in 16-byte vectors: every tensor begins on a boundary, and its rows keep the same distance
// from one as those of the first.
struct Vectors {
    int64_t rows, stride = -1;
    int vec;
    bool fit = true;
    void take(const void *at, int64_t row_stride, int size) {
        if (stride < 0) stride = row_stride;
        fit = fit && aligned(at, static_cast<uintptr_t>(vec * size)) && (row_stride - stride) % vec == 0;
    }
};

// A tensor of rows: present where it has to be, aligned to its elements; an output's rows do not overlap.
int take_rows(const loco_rows_t *t, int dim, int size, bool written, Vectors &V, int64_t &stride) {
    if (!t || !t->ptr) return LOCO_ERR_ARG;
    stride = V.rows > 1 ? t->row_stride : 0;
    if (stride < 0 || (written && V.rows > 1 && stride < dim)) return LOCO_ERR_ARG;
    if (!aligned(t->ptr, static_cast<uintptr_t>(size))) return LOCO_ERR_ALIGN;
    V.take(t->ptr, stride, size);
    return LOCO_OK;
}

// Shared memory above the default limit, set once per device.
bool allow(NormKernel fn, int which) {
    static std::atomic<bool> set[64][48];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return false;
    }
    if (set[dev][which].load(std::memory_order_acquire)) return true;
    if (cudaFuncSetAttribute(reinterpret_cast<const void *>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    set[dev][which].store(true, std::memory_order_release);
    return true;
}

// Threads of a row, teams of a block, and blocks: as many as run at once, fewer teams where the rows would not fill the SMs.
int launch_norm(NormParams &P, const loco_norm_t *c, bool backward, const Vectors &V, void *stream, int &blocks) {
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    // elements of a thread: 32 bytes of them, 64 where a row of fp32 needs more than a block
    const int size = c->dtype == LOCO_BF16 ? 2 : 4;
    int vec = V.fit ? V.vec : 1, columns = c->dim + (P.xs % vec ? vec - 1 : 0);      // a row and what lies before it up to a boundary
    if (columns > 16 * kNormThreads) {
        vec = 1;
        columns = c->dim;
    }
    const int mine = size == 2 || columns > 8 * kNormThreads ? 16 : 8, lanes = (columns + mine - 1) / mine;
    int team = 4;
    while (team < 32 && team < lanes) team *= 2;
    if (lanes > 32) team = (lanes + 31) / 32 * 32;
    // Backward with long rows one block an SM: half the partial rows of dw (8192 x 4096 bfloat16 53.4 -> 51.3 us; shorter rows lose 1 to 2).
    int teams = (backward && team >= 256 ? kNormThreads : kBlockThreads) / team;
    const int least = team < 32 ? 32 / team : 1;
    const int64_t spread = P.rows / (2 * sms);
    if (spread < teams) teams = static_cast<int>(spread) / least * least;
    if (teams < least) teams = least;
    const int threads = team * teams, tensors = backward ? 3 : 2;
    // rows on their way: as many as the shared memory of the blocks that run at once holds, three at most
    const int together = kNormThreads / threads, each = threads * mine * size * tensors;
    int depth = kRingBytes / (together * each + 2048 * together);
    depth = depth < 1 ? 1 : depth > 3 ? 3 : depth;
    // Forward with a residual a block has 256 KB to move, and there are more than run at once: the SMs are not equally far from
    // memory, and those that are done first take more of them.  16384 x 5120, bfloat16 with residual, 1, 2, 4, 8 times as many as run at once: 123, 111, 105,
    // 103 us; without, 1, 2, 4 times: 59, 59, 60.  Backward every block costs a partial row: 47.5 us with one time, 56 with 1.5.
    const int64_t all = (P.rows + teams - 1) / teams, once = static_cast<int64_t>(sms) * together;
    const int64_t more = P.r ? P.rows * c->dim * size * 4 / (once * (256 << 10)) : 1;
    int64_t most = backward || more < 1 ? once : once * more;
    if (backward && most > kPartials) most = kPartials;
    blocks = static_cast<int>(all < most ? all : most);
    if (all > most)                              // the rows of a team, blocks * teams apart, have one distance from the boundaries
        while (static_cast<int64_t>(blocks) * teams % vec * (P.xs % vec) % vec != 0) --blocks;
    P.team = team;
    P.depth = depth;
    P.dim = c->dim;
    P.block = c->block;
    P.groups = (c->dim + kScaleBlock - 1) / kScaleBlock;
    P.eps = c->eps;
    P.over_dim = 1.0f / static_cast<float>(c->dim);
    const bool shift = P.xs % vec != 0 || c->dim % vec != 0;
    const NormKernel fn = size == 2 ? (vec > 1 ? pick_norm<__nv_bfloat16, 8>(mine, shift, backward, c->bits8) : pick_norm<__nv_bfloat16, 1>(mine, shift, backward, c->bits8))
                                    : (vec > 1 ? pick_norm<float, 4>(mine, shift, backward, c->bits8) : pick_norm<float, 1>(mine, shift, backward, c->bits8));
    const size_t ring = static_cast<size_t>(depth) * each;
    if (!allow(fn, ((((size == 4) * 2 + (vec > 1)) * 2 + (mine * size > 32)) * 2 + shift) * 3 + (backward ? 2 : c->bits8 ? 1 : 0))) return LOCO_ERR_CUDA;
    return launch_kernel(fn, dim3(static_cast<unsigned>(blocks)), static_cast<unsigned>(threads), ring, stream, P);
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
    Vectors V{rows};
    V.vec = 16 / size;
    if ((rc = take_rows(x, c->dim, size, false, V, P.xs)) != LOCO_OK) return rc;
    if (residual && (rc = take_rows(residual, c->dim, size, false, V, P.rs)) != LOCO_OK) return rc;
    if (total && (rc = take_rows(total, c->dim, size, true, V, P.hs)) != LOCO_OK) return rc;
    if ((rc = take_rows(y, c->dim, c->bits8 ? 1 : size, true, V, P.ys)) != LOCO_OK) return rc;
    if (c->bits8 && !d_scale) return LOCO_ERR_ARG;
    if (!aligned(d_weight, static_cast<uintptr_t>(size)) || !aligned(d_scale, 4)) return LOCO_ERR_ALIGN;
    if (!aligned(d_weight, 16)) V.fit = false;
    P.x = x->ptr;
    P.r = residual ? residual->ptr : nullptr;
    P.h = total ? total->ptr : nullptr;
    P.y = y->ptr;
    P.w = d_weight;
    P.scale = d_scale;
    int blocks;
    return launch_norm(P, c, false, V, stream, blocks);
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
        Vectors V{rows};
        V.vec = 16 / size;
        if ((rc = take_rows(h, c->dim, size, false, V, P.xs)) != LOCO_OK) return rc;
        if ((rc = take_rows(dy, c->dim, size, false, V, P.dys)) != LOCO_OK) return rc;
        if (dtotal && (rc = take_rows(dtotal, c->dim, size, false, V, P.dts)) != LOCO_OK) return rc;
        if ((rc = take_rows(dx, c->dim, size, true, V, P.dxs)) != LOCO_OK) return rc;
        if (!aligned(d_weight, static_cast<uintptr_t>(size))) return LOCO_ERR_ALIGN;
        if (!aligned(d_weight, 16)) V.fit = false;
        P.x = h->ptr;
        P.dy = dy->ptr;
        P.dt = dtotal ? dtotal->ptr : nullptr;
        P.dx = dx->ptr;
        P.w = d_weight;
        rc = launch_norm(P, c, true, V, stream, blocks);
        if (rc != LOCO_OK || !P.wanted) return rc;
    }
    const dim3 grid(static_cast<unsigned>((c->dim + 31) / 32));
    if (c->dtype == LOCO_BF16) return launch_kernel(norm_weight_kernel<__nv_bfloat16>, grid, kWeightWarps * 32, 0, stream, P.part, blocks, c->dim, static_cast<__nv_bfloat16 *>(d_dweight));
    return launch_kernel(norm_weight_kernel<float>, grid, kWeightWarps * 32, 0, stream, P.part, blocks, c->dim, static_cast<float *>(d_dweight));
}

}  // extern "C"
