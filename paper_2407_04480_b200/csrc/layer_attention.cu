// Attention on the tensor cores: tiles of 128 rows that stay, tiles of 80, 96 or 128 that stream, products accumulated in
// tensor memory (TMEM).  1 x 4096 tokens, 32 heads of 128, not causal, calls in a row: forward 233 us (1180 TFLOP/s),
// backward 713 us (the seven products it executes: 1350 TFLOP/s); the tensor pipe, 68 to 72% busy while an SM is active,
// bounds each.
//
// All three kernels have the same parts.  One warp copies tiles to shared memory (TMA, 128-byte swizzle), one thread issues
// the products, two groups of four warps turn scores into probabilities (a thread per TMEM lane, i.e. per row), and one warp
// zeroes what a copy brought in from past the end of a sample, so that whatever lies there (NaN included) meets a zero
// probability as a zero.  Probabilities and their gradients go back to TMEM as bfloat16 (P to a place of its own, dS over dP)
// and are the first operand of the second product from there: they never pass through shared memory.
//
//   forward           two tiles of 128 queries stay, keys and values stream; one warp group per query tile, so that one
//                     group's exponentials run under the other tile's products.  The running maximum is moved (and o
//                     rescaled) only when it grows by more than 2^8: until then exp2 stays inside the range of fp32 and
//                     bfloat16, and the final division by the sum takes the common factor out exactly.
//   backward queries  128 queries stay, keys and values stream: S, dP, then dq += dS K.  It also leaves D = do . o.
//   backward keys     128 keys and values stay, the queries of all heads that share them stream: the transposed scores,
//                     so that P^T and dS^T have the keys as rows: dv += P^T dO, dk += dS^T Q.  A shared head's gradient is
//                     summed in its accumulator, and no output needs an atomic: the price is seven products instead
//                     of the five that a single kernel with atomic dq would need.
#include <cuda.h>

#include "layer_attention.h"
#include "layer_tc.cuh"

namespace loco_layer {

using namespace tc;

constexpr int kTile = 128;                       // queries and keys of a tile
constexpr int kGroupWarps = 4;                   // warps of a softmax group: the 128 lanes of TMEM
constexpr int kThreads = 3 * kGroupWarps * 32;   // two softmax groups and one of single warps, the last of which idles
constexpr int kLoadWarp = 2 * kGroupWarps, kProductWarp = kLoadWarp + 1, kHelpWarp = kLoadWarp + 2;
// Of so many pairs of scores one goes through exp2_poly.  Forward with none, one in eight, in four, in three: 4 x 2048, 16
// heads of 64: 138, 139, 132, 143 us; 1 x 4096, 32 heads of 128: 231, 232, 233, 235.  Backward with none, one in eight, in
// four: 404, 392, 400 and 716, 713, 720 us.
constexpr int kPolyForward = 4, kPolyBackward = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ unsigned g_status;                    // LOCO_LAYER_FLAG_*

struct Maps { CUtensorMap q, k, v, d_o, o; };

// Shared memory: two tiles that stay, the ring of tiles that stream, then Shared.  Either head size fills the SM, so that no
// two blocks compete for its tensor memory.
template <int kDim> __host__ __device__ constexpr int tile_bytes() { return kTile * kDim * 2; }
template <int kDim> __host__ __device__ constexpr int stream_slots() { return kDim == 128 ? 5 : 10; }
constexpr int kMaxSlots = 12;
struct Shared {
    uint64_t full[kMaxSlots], empty[kMaxSlots];  // streaming tiles: copied, no longer read
    uint64_t stay, rows_in;                      // the tiles that stay are in shared memory, in TMEM
    uint64_t score[2], second[2];                // products ready: S per query tile; o per query tile (forward), dP and dv (backward)
    uint64_t read[2];                            // forward: S in registers
    uint64_t prob[2], grad;                      // P written to TMEM (forward: per query tile), S read (backward); dS written
    uint64_t last, clean;                        // a tile with rows past the end is copied; those rows are zero
    uint64_t stats[2], stats_free[2];            // backward keys: row statistics of a query tile
    uint64_t done, drain;
    uint32_t tmem, failed;
    alignas(16) float row[2][2][kTile];          // backward keys: -lse * log2(e), -D of the query tile; backward queries: D
};
template <int kDim> constexpr int shared_bytes() {
    return (2 + stream_slots<kDim>()) * tile_bytes<kDim>() + static_cast<int>(sizeof(Shared));
}
static_assert(shared_bytes<128>() <= 227 * 1024 && shared_bytes<64>() <= 227 * 1024, "shared memory of a block");

template <int kDim, int kRows = kTile>
__device__ __forceinline__ void load_tile(uint32_t to, const CUtensorMap *map, int row, int head, int batch, uint32_t bar) {
    bar_expect(bar, kRows * kDim * 2);
#pragma unroll
    for (int x = 0; x < kDim; x += 64) load_box(to + x / 64 * (kRows * 128), map, x, row, head, batch, bar);
}

// Zero the rows from `first` on of a tile, by one warp.
template <int kDim, int kRows = kTile> __device__ __forceinline__ void clean_tile(uint8_t *tile, int first, int lane) {
    for (int x = 0; x < kDim; x += 64)
        for (int i = first * 8 + lane; i < kRows * 8; i += 32)
            reinterpret_cast<uint4 *>(tile + x / 64 * (kRows * 128))[i] = make_uint4(0, 0, 0, 0);
}

// S (128 x kRows) = A B^T over kDim columns, both tiles in shared memory.
template <int kDim, int kRows = kTile> __device__ __forceinline__ void product_scores(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t word) {
    const uint32_t da = desc_along_columns(a), db = desc_along_columns(b);
#pragma unroll
    for (int x = 0; x < kDim; x += 16)
        mma_ss(lead, d, da + ((x / 64 * (kTile * 128) + x % 64 * 2) >> 4), db + ((x / 64 * (kRows * 128) + x % 64 * 2) >> 4), word, x > 0);
}
// The same with A in TMEM, two dimensions to a column.
template <int kDim> __device__ __forceinline__ void product_scores_tmem(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t word) {
    const uint32_t db = desc_along_columns(b);
#pragma unroll
    for (int x = 0; x < kDim; x += 16) mma_ts(lead, d, a + x / 2, db + ((x / 64 * (kTile * 128) + x % 64 * 2) >> 4), word, x > 0);
}
// d (128 x kDim) += A B: A (128 x kRows) in TMEM, its columns at `a0` (first half) and `a1`; B's rows are the tile's.
template <int kDim, int kRows = kTile>
__device__ __forceinline__ void product_apply(uint32_t lead, uint32_t d, uint32_t a0, uint32_t a1, uint32_t b, uint32_t accumulate) {
    constexpr uint32_t word = product(kDim, true);
    const uint32_t db = desc_along_rows(b, kRows * 128);
#pragma unroll
    for (int r = 0; r < kRows; r += 16)
        mma_ts(lead, d, r < kRows / 2 ? a0 + r / 2 : a1 + (r - kRows / 2) / 2, db + (r * 128 >> 4), word, accumulate | (r > 0));
}

// Sets up barriers and TMEM; returns the TMEM base.
template <int kColumns> __device__ __forceinline__ uint32_t begin_block(Shared &S, int slots, int last_arrivals, int prob_arrivals) {
    const int warp = threadIdx.x / 32;
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) {
            bar_init(smem_addr(&S.full[i]), 1);
            bar_init(smem_addr(&S.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_addr(&S.score[i]), 1);
            bar_init(smem_addr(&S.second[i]), 1);
            bar_init(smem_addr(&S.prob[i]), prob_arrivals);
            bar_init(smem_addr(&S.read[i]), prob_arrivals);
            bar_init(smem_addr(&S.stats[i]), 1);
            bar_init(smem_addr(&S.stats_free[i]), 2 * kGroupWarps);
        }
        bar_init(smem_addr(&S.grad), 2 * kGroupWarps);
        bar_init(smem_addr(&S.stay), 1);
        bar_init(smem_addr(&S.rows_in), 2 * kGroupWarps);
        bar_init(smem_addr(&S.last), last_arrivals);
        bar_init(smem_addr(&S.clean), 1);
        bar_init(smem_addr(&S.done), 1);
        bar_init(smem_addr(&S.drain), 1);
        S.failed = 0;
        fence_bar_init();
        fence_async_shared();
    }
    if (warp == kProductWarp) tmem_alloc<kColumns>(smem_addr(&S.tmem));
    fence_before();
    __syncthreads();
    fence_after();
    return S.tmem;
}
template <int kColumns> __device__ __forceinline__ void end_block(Shared &S, uint32_t tmem) {
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x / 32 == kProductWarp) tmem_free<kColumns>(tmem);
    if (threadIdx.x == 0 && S.failed) atomicOr(&g_status, LOCO_LAYER_FLAG_TIMEOUT);
}

// Registers: the block starts with 168 a thread (3 x 128 x 168 of the SM's 65536); the softmax groups, which hold rows of
// scores, take 208 each and the third group keeps 88: 2 x 208 + 88 = 3 x 168.
// Set at the head of each side's own code.
__device__ __forceinline__ void registers_many() { asm volatile("setmaxnreg.inc.sync.aligned.u32 208;"); }
__device__ __forceinline__ void registers_few() { asm volatile("setmaxnreg.dec.sync.aligned.u32 88;"); }

// A role that gave up still waits for the copies it started before the block's shared memory goes away.
__device__ __forceinline__ void settle(uint32_t bar, uint32_t parity) {
    const uint64_t begin = now_ns();
    while (!bar_test(bar, parity) && now_ns() - begin < kWaitLimitNs / 20) {}
}

// Ring of streaming tiles, seen by the thread that fills it and the one that empties it.
struct Ring {
    uint32_t slot = 0, phase = 0;
    template <int kSlots> __device__ __forceinline__ void next() {
        if (++slot == kSlots) {
            slot = 0;
            phase ^= 1;
        }
    }
};

// A warp's 32 rows of an accumulator leave through shared memory, so that its stores cover whole rows: a thread's own row
// of 16-byte pieces would touch 32 lines an instruction (measured: 2000 clocks a block more).  kCols columns a row; the
// pieces are permuted so that neither side meets a bank twice.
template <int kCols> __device__ __forceinline__ uint32_t piece_at(int row, int piece) {
    constexpr int kPieces = kCols / 8;
    return row * (kCols * 2) + ((piece ^ (kPieces >= 8 ? row & 7 : row >> 1 & 3)) << 4);
}
template <int kCols> __device__ __forceinline__ void stage_columns(uint8_t *stage, int row, const uint32_t (&r)[32], int first, float by, bool some) {
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (some) {
            w.x = pack_bf16(__uint_as_float(r[i]) * by, __uint_as_float(r[i + 1]) * by);
            w.y = pack_bf16(__uint_as_float(r[i + 2]) * by, __uint_as_float(r[i + 3]) * by);
            w.z = pack_bf16(__uint_as_float(r[i + 4]) * by, __uint_as_float(r[i + 5]) * by);
            w.w = pack_bf16(__uint_as_float(r[i + 6]) * by, __uint_as_float(r[i + 7]) * by);
        }
        *reinterpret_cast<uint4 *>(stage + piece_at<kCols>(row, (first + i) / 8)) = w;
    }
}
// kCols accumulator columns at `tmem` times `by` (zeros where not `some`), rows [i, i + 32) below `end` of a head, from
// dimension `x` on.  `filled` is false where the accumulator holds nothing.
template <int kCols>
__device__ __forceinline__ void store_rows(uint8_t *stage, uint32_t tmem, bool filled, float by, bool some, const Heads &t, const Rows &rows, int i, int end,
                                           int head, int x, int dim) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int c = 0; c < kCols; c += 32) {
        uint32_t r[32];
        if (filled) {
            load_columns(tmem + c, r);
            wait_loads();
            pin(r);
        }
        stage_columns<kCols>(stage, lane, r, c, by, some && filled);
    }
    __syncwarp();
    constexpr int kPieces = kCols / 8;
    const int piece = lane % kPieces;
    if (x + piece * 8 < dim)                     // dim is a multiple of 8
#pragma unroll 4
        for (int row = lane / kPieces; row < 32; row += 32 / kPieces)
            if (i + row < end)
                *reinterpret_cast<uint4 *>(row_of(t, rows, i + row, head) + x + piece * 8) = *reinterpret_cast<const uint4 *>(stage + piece_at<kCols>(row, piece));
}
// c + the product of two pairs of bfloat16
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
    c = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), c);
    return fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), c);
}
// Whether a streamed tile that holds the last of n rows also holds rows past them that are not the copy's zero fill.
__device__ __forceinline__ bool ends_inside(const Rows &r, int packed, int seq, int tile = kTile) { return r.n % tile != 0 && (packed || r.n != seq); }

// The block's place.  Heads come in spans; within a span the tiles are the slow index and `reverse` starts with the last one,
// which under a causal mask is the longest for queries.
struct BlockPlace { int tile, head, batch; };
__device__ __forceinline__ BlockPlace block_place(const AttentionParams &P, int heads, int tiles, bool reverse) {
    const int first = static_cast<int>(blockIdx.x) / (P.span * tiles) * P.span, size = min(P.span, heads * P.batch - first);
    const int r = static_cast<int>(blockIdx.x) - first * tiles, t = r / size, hb = first + r - t * size;
    return BlockPlace{reverse ? tiles - 1 - t : t, hb % heads, hb / heads};
}

// Whether a packed sample ends before row `first` of its queries or keys: most blocks of short samples, so it is asked
// before a block is set up.
template <typename RowsOf> __device__ __forceinline__ bool no_such_rows(const AttentionParams &P, const RowsOf &rows_of, int batch, int first) {
    wait_for_previous();
    return first >= rows_of(P, batch).n;
}

// Keys that query i sees: [0, limit).
__device__ __forceinline__ int key_limit(const Rows &Q, const Rows &K, int causal, int i) {
    if (i >= Q.n) return 0;
    return causal ? max(0, min(K.n, i + K.n - Q.n + 1)) : K.n;
}
// Key tiles that the queries [first, first + 128) need.
__device__ __forceinline__ int key_tiles(const Rows &Q, const Rows &K, int causal, int first, int tile = kTile) {
    if (first >= Q.n) return 0;
    return (key_limit(Q, K, causal, min(first + kTile, Q.n) - 1) + tile - 1) / tile;
}

__device__ __forceinline__ void mask_from(uint32_t (&s)[16], int left) {
#pragma unroll
    for (int x = 0; x < 16; ++x)
        if (x >= left) s[x] = 0xff800000u;       // -inf
}
__device__ __forceinline__ float row_max(const uint32_t (&s)[16]) {
    float m[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        const uint32_t *x = s + 8 * y;
        m[y] = max3(max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2])),
                    max3(__uint_as_float(x[3]), __uint_as_float(x[4]), __uint_as_float(x[5])),
                    max2(__uint_as_float(x[6]), __uint_as_float(x[7])));
    }
    return max2(m[0], m[1]);
}

// ------------------------------------------------------------------------------------------------ forward

// TMEM: o, S and P of both query tiles.  S is free again once its softmax group has it in registers, so that the next scores
// are computed under this tile's exponentials; with heads of 128 that takes key tiles of 80, as two tiles of 128 would fill
// TMEM without a place of its own for P, and the next scores would wait for the product with the values (measured at 4096,
// 32 heads: 252 us).
template <int kDim> __host__ __device__ constexpr int key_tile() { return kDim == 128 ? 80 : 128; }
constexpr int kForwardSlots = 8;
template <int kDim> constexpr int forward_bytes() {
    return 2 * tile_bytes<kDim>() + kForwardSlots * key_tile<kDim>() * kDim * 2 + static_cast<int>(sizeof(Shared));
}
static_assert(forward_bytes<128>() <= 227 * 1024 && forward_bytes<64>() <= 227 * 1024, "shared memory of a block");

template <int kDim>
__global__ void __launch_bounds__(kThreads, 1) attention_forward_kernel(const __grid_constant__ AttentionParams P, const __grid_constant__ Maps M) {
    constexpr int kSlots = kForwardSlots, kBytes = tile_bytes<kDim>(), kKeys = key_tile<kDim>(), kStep = kKeys * kDim * 2;
    extern __shared__ __align__(1024) uint8_t tiles[];
    Shared &S = *reinterpret_cast<Shared *>(tiles + 2 * kBytes + kSlots * kStep);
    const uint32_t base = smem_addr(tiles), ring = base + 2 * kBytes;
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) / 32, 0), lane = threadIdx.x % 32;
    const BlockPlace at = block_place(P, P.heads_q, (P.max_q + 2 * kTile - 1) / (2 * kTile), P.causal);
    if (P.packed && no_such_rows(P, query_rows, at.batch, at.tile * 2 * kTile)) return;
    const uint32_t tmem = begin_block<512>(S, kSlots, 1, kGroupWarps);
    wait_for_previous();
    let_next_start();
    const Rows Q = query_rows(P, at.batch), K = key_rows(P, at.batch);
    const int first = at.tile * 2 * kTile, head_kv = at.head / P.group;
    const int n0 = key_tiles(Q, K, P.causal, first, kKeys), n1 = key_tiles(Q, K, P.causal, first + kTile, kKeys), n = max(n0, n1);
    const bool ragged = ends_inside(K, P.packed, P.seq_k, kKeys) && n == K.n / kKeys + 1;
    volatile uint32_t *const failed = &S.failed;

    if (warp >= 2 * kGroupWarps) {
        registers_few();
        if (warp == kLoadWarp && lane == 0 && n > 0) {
            Ring r;
            bar_expect(smem_addr(&S.stay), (n0 > 0 ? kBytes : 0) + (n1 > 0 ? kBytes : 0));
            for (int t = 0; t < 2; ++t)
                if ((t ? n1 : n0) > 0)
#pragma unroll
                    for (int x = 0; x < kDim; x += 64)
                        load_box(base + t * kBytes + x / 64 * (kTile * 128), &M.q, x, Q.first + first + t * kTile, at.head, Q.at, smem_addr(&S.stay));
            int sent = 0;
            for (int j = 0; j < 2 * n; ++j) {
                bar_wait(smem_addr(&S.empty[r.slot]), r.phase ^ 1, failed);
                if (*failed) break;
                load_tile<kDim, kKeys>(ring + r.slot * kStep, j % 2 ? &M.v : &M.k, K.first + j / 2 * kKeys, head_kv, K.at,
                                       smem_addr(ragged && j >= 2 * n - 1 ? &S.last : &S.full[r.slot]));
                ++sent;
                r.next<kSlots>();
            }
            if (*failed) {
                settle(smem_addr(&S.stay), 0);
                for (int j = max(0, sent - kSlots); j < sent; ++j)
                    if (ragged && j >= 2 * n - 1) settle(smem_addr(&S.last), 0);
                    else settle(smem_addr(&S.full[j % kSlots]), j / kSlots & 1);
            }
        } else if (warp == kProductWarp && n > 0) {
            const uint32_t lead = elect_lane();
            const uint32_t scores = product(kKeys, false, P.scale < 0.0f);
            const uint32_t s_at = tmem + 2 * kDim, p_at = s_at + 2 * kKeys;
            bar_wait(smem_addr(&S.stay), 0, failed);
            bar_wait(smem_addr(&S.full[0]), 0, failed);
            for (int t = 0; t < 2; ++t)
                if ((t ? n1 : n0) > 0) {
                    product_scores<kDim, kKeys>(lead, s_at + t * kKeys, base + t * kBytes, ring, scores);
                    commit(lead, smem_addr(&S.score[t]));
                }
            commit(lead, smem_addr(&S.empty[0]));
            Ring v, k;                               // value tiles at odd places of the stream, key tiles at even ones
            v.next<kSlots>();
            k.next<kSlots>();
            k.next<kSlots>();
            for (int j = 0; j < n; ++j) {
                if (j + 1 < n) bar_wait(smem_addr(&S.full[k.slot]), k.phase, failed);
                for (int t = 0; t < 2; ++t) {
                    const int nt = t ? n1 : n0;
                    if (j + 1 < nt) {
                        bar_wait(smem_addr(&S.read[t]), j & 1, failed);
                        fence_after();
                        product_scores<kDim, kKeys>(lead, s_at + t * kKeys, base + t * kBytes, ring + k.slot * kStep, scores);
                        commit(lead, smem_addr(&S.score[t]));
                    }
                    if (j < nt) {
                        if (ragged && j == n - 1) bar_wait(smem_addr(&S.clean), 0, failed);
                        else bar_wait(smem_addr(&S.full[v.slot]), v.phase, failed);
                        bar_wait(smem_addr(&S.prob[t]), j & 1, failed);
                        fence_after();
                        const uint32_t p = p_at + t * (kKeys / 2);
                        product_apply<kDim, kKeys>(lead, tmem + t * kDim, p, p + kKeys / 4, ring + v.slot * kStep, j > 0);
                        commit(lead, smem_addr(&S.second[t]));
                    }
                }
                commit(lead, smem_addr(&S.empty[v.slot]));
                if (j + 1 < n) commit(lead, smem_addr(&S.empty[k.slot]));
                for (int i = 0; i < 2; ++i) {
                    v.next<kSlots>();
                    k.next<kSlots>();
                }
            }
            commit(lead, smem_addr(&S.drain));
            bar_wait(smem_addr(&S.drain), 0, failed);
            if (*failed) settle(smem_addr(&S.drain), 0);
        } else if (warp == kHelpWarp && ragged) {
            const int load = 2 * n - 1;              // the last value tile
            bar_wait(smem_addr(&S.last), 0, failed);
            clean_tile<kDim, kKeys>(tiles + 2 * kBytes + load % kSlots * kStep, K.n % kKeys, lane);
            fence_async_shared();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.clean));
        }
    } else {
        registers_many();
        constexpr int kParts = kKeys / 16;
        const int t = warp / kGroupWarps, i = first + t * kTile + threadIdx.x % kTile;
        const int nt = t ? n1 : n0, limit = key_limit(Q, K, P.causal, i);
        const uint32_t lanes = tmem + (static_cast<uint32_t>(warp % kGroupWarps * 32) << 16);
        const uint32_t o_at = lanes + t * kDim, s_at = lanes + 2 * kDim + t * kKeys, p_at = lanes + 2 * kDim + 2 * kKeys + t * (kKeys / 2);
        const float scale = fmaxf(fabsf(P.scale), 1e-30f) * kLog2e;
        const float room = 8.0f / scale;         // how far the maximum may grow before o is rescaled
        float top = -INFINITY, total = 0.0f;
        for (int j = 0; j < nt; ++j) {
            bar_wait(smem_addr(&S.score[t]), j & 1, failed);
            __syncwarp();
            fence_after();
            uint32_t s[kParts][16];
#pragma unroll
            for (int c = 0; c < kParts; ++c) load_columns(s_at + c * 16, s[c]);
            wait_loads();
#pragma unroll
            for (int c = 0; c < kParts; ++c) pin(s[c]);
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.read[t]));
            const int left = limit - j * kKeys;  // columns from here on are not seen
            if (__any_sync(0xffffffffu, left < kKeys)) {
#pragma unroll
                for (int c = 0; c < kParts; ++c) mask_from(s[c], left - c * 16);
            }
            float most = row_max(s[0]);
#pragma unroll
            for (int c = 1; c < kParts; c += 2) most = c + 1 < kParts ? max3(most, row_max(s[c]), row_max(s[c + 1 < kParts ? c + 1 : c])) : max2(most, row_max(s[c]));
            if (j == 0) {
                top = most;
            } else {
                bar_wait(smem_addr(&S.second[t]), (j - 1) & 1, failed);      // o is complete so far, and P free
                __syncwarp();
                fence_after();
                if (__any_sync(0xffffffffu, !(most - top <= room))) {
                    const float next = max2(top, most);
                    const float fade = next == -INFINITY ? 1.0f : exp2_fast((top - next) * scale);
#pragma unroll
                    for (int c = 0; c < kDim / 16; ++c) {
                        uint32_t o[16];
                        load_columns(o_at + c * 16, o);
                        wait_loads();
                        pin(o);
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * fade);
                        store_columns(o_at + c * 16, o);
                    }
                    total *= fade;
                    top = next;
                }
            }
            const float shift = top == -INFINITY ? 0.0f : top * scale;
            const float2 by = make_float2(scale, scale), minus = make_float2(-shift, -shift);
#pragma unroll
            for (int c = 0; c < kParts; ++c) {
                uint32_t p[8];
#pragma unroll
                for (int x = 0; x < 16; x += 2) {
                    float2 e = fma2(make_float2(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1])), by, minus);
                    if (x / 2 % kPolyForward == kPolyForward - 1) {
                        e = exp2_poly(e);
                    } else {
                        e.x = exp2_fast(e.x);
                        e.y = exp2_fast(e.y);
                    }
                    s[c][x] = __float_as_uint(e.x);
                    s[c][x + 1] = __float_as_uint(e.y);
                    p[x / 2] = pack_bf16(e.x, e.y);
                }
                store_columns(p_at + c * 8, p);
            }
            wait_stores();
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.prob[t]));
            // the sum is nobody's wait: it is formed under the products
            float2 sum[2];
#pragma unroll
            for (int c = 0; c < kParts; ++c) {
                pin(s[c]);
#pragma unroll
                for (int x = 0; x < 16; x += 2) {
                    const float2 e = make_float2(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1]));
                    sum[x / 2 % 2] = c == 0 && x < 4 ? e : add2(sum[x / 2 % 2], e);
                }
            }
            sum[0] = add2(sum[0], sum[1]);
            total += sum[0].x + sum[0].y;
        }
        if (nt > 0) bar_wait(smem_addr(&S.second[t]), (nt - 1) & 1, failed);
        __syncwarp();
        fence_after();
        const int end = P.packed ? Q.n : P.seq_q;
        const bool some = limit > 0 && top != -INFINITY;           // a score above -infinity, or NaN
        // through this tile's queries, which no product reads any more
        store_rows<kDim>(tiles + t * kBytes + warp % kGroupWarps * (32 * kDim * 2), o_at, nt > 0, 1.0f / total, some, P.o, Q, i - lane, end, at.head, 0,
                         P.head_dim);
        if (i < end) P.lse[stat_at(P, Q, i, at.head)] = some ? (top == INFINITY ? INFINITY : (top * scale + log2f(total)) * kLn2) : -INFINITY;
    }
    __syncwarp();
    end_block<512>(S, tmem);
}

// ------------------------------------------------------------------------------------------------ backward: queries

// TMEM: S, dP, dq, and as bfloat16 the q and do that stay: read from there they leave shared memory to the stream (seven
// tiles of keys and values instead of five: with five the copies' latency showed) and halve what the score products read
// from it.  S is free again once the softmax groups have it in registers; dS goes over dP: columns 0-31 from the first
// group, 64-95 from the second.
template <int kDim>
__global__ void __launch_bounds__(kThreads, 1) attention_backward_queries_kernel(const __grid_constant__ AttentionParams P, const __grid_constant__ Maps M) {
    constexpr int kSlots = stream_slots<kDim>() + 2, kBytes = tile_bytes<kDim>();
    extern __shared__ __align__(1024) uint8_t tiles[];
    Shared &S = *reinterpret_cast<Shared *>(tiles + kSlots * kBytes);
    const uint32_t ring = smem_addr(tiles);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) / 32, 0), lane = threadIdx.x % 32;
    const BlockPlace at = block_place(P, P.heads_q, (P.max_q + kTile - 1) / kTile, P.causal);
    if (P.packed && no_such_rows(P, query_rows, at.batch, at.tile * kTile)) return;
    const uint32_t tmem = begin_block<512>(S, kSlots, 2, 2 * kGroupWarps);
    wait_for_previous();
    let_next_start();
    const Rows Q = query_rows(P, at.batch), K = key_rows(P, at.batch);
    const int first = at.tile * kTile, head_kv = at.head / P.group;
    const int n = key_tiles(Q, K, P.causal, first);
    const bool ragged = ends_inside(K, P.packed, P.seq_k) && n == K.n / kTile + 1;
    const uint32_t s_at = tmem, dp_at = tmem + kTile, dq_at = tmem + 2 * kTile, q_at = tmem + 3 * kTile, do_at = q_at + kDim / 2;
    volatile uint32_t *const failed = &S.failed;

    if (warp >= 2 * kGroupWarps) {
        registers_few();
        if (warp == kLoadWarp && lane == 0 && n > 0) {
            Ring r;
            // the last three places of the ring hold q, do and o until the softmax groups have read them
            bar_expect(smem_addr(&S.stay), 3 * kBytes);
            for (int x = 0; x < 3; ++x)
#pragma unroll
                for (int y = 0; y < kDim; y += 64)
                    load_box(ring + (kSlots - 3 + x) * kBytes + y / 64 * (kTile * 128), x == 0 ? &M.q : x == 1 ? &M.d_o : &M.o, y, Q.first + first, at.head, Q.at,
                             smem_addr(&S.stay));
            int sent = 0;
            for (int j = 0; j < 2 * n; ++j) {
                if (j == kSlots - 3) bar_wait(smem_addr(&S.rows_in), 0, failed);
                bar_wait(smem_addr(&S.empty[r.slot]), r.phase ^ 1, failed);
                if (*failed) break;
                load_tile<kDim>(ring + r.slot * kBytes, j % 2 ? &M.v : &M.k, K.first + j / 2 * kTile, head_kv, K.at,
                                smem_addr(ragged && j >= 2 * n - 2 ? &S.last : &S.full[r.slot]));
                ++sent;
                r.next<kSlots>();
            }
            if (*failed) {
                settle(smem_addr(&S.stay), 0);
                for (int j = max(0, sent - kSlots); j < sent; ++j)
                    if (ragged && j >= 2 * n - 2) settle(smem_addr(&S.last), 0);
                    else settle(smem_addr(&S.full[j % kSlots]), j / kSlots & 1);
            }
        } else if (warp == kProductWarp && n > 0) {
            const uint32_t lead = elect_lane();
            const uint32_t scores = product(kTile, false, P.scale < 0.0f), plain = product(kTile, false);
            // tile j: keys at place 2j of the ring, values at 2j + 1
            const auto slot = [](int load) { return load % kSlots; };
            const auto ready = [&](int load) {
                if (ragged && load >= 2 * n - 2) bar_wait(smem_addr(&S.clean), 0, failed);
                else bar_wait(smem_addr(&S.full[load % kSlots]), load / kSlots & 1, failed);
            };
            bar_wait(smem_addr(&S.rows_in), 0, failed);
            ready(0);
            fence_after();
            product_scores_tmem<kDim>(lead, s_at, q_at, ring, scores);
            commit(lead, smem_addr(&S.score[0]));
            ready(1);
            product_scores_tmem<kDim>(lead, dp_at, do_at, ring + kBytes, plain);
            commit(lead, smem_addr(&S.second[0]));
            commit(lead, smem_addr(&S.empty[1]));
            for (int j = 0; j < n; ++j) {
                if (j + 1 < n) {
                    bar_wait(smem_addr(&S.prob[0]), j & 1, failed);
                    ready(2 * j + 2);
                    fence_after();
                    product_scores_tmem<kDim>(lead, s_at, q_at, ring + slot(2 * j + 2) * kBytes, scores);
                    commit(lead, smem_addr(&S.score[0]));
                }
                bar_wait(smem_addr(&S.grad), j & 1, failed);
                fence_after();
                product_apply<kDim>(lead, dq_at, dp_at, dp_at + 64, ring + slot(2 * j) * kBytes, j > 0);
                commit(lead, smem_addr(&S.empty[slot(2 * j)]));
                if (j + 1 < n) {
                    ready(2 * j + 3);
                    product_scores_tmem<kDim>(lead, dp_at, do_at, ring + slot(2 * j + 3) * kBytes, plain);
                    commit(lead, smem_addr(&S.second[0]));
                    commit(lead, smem_addr(&S.empty[slot(2 * j + 3)]));
                }
            }
            commit(lead, smem_addr(&S.done));
            commit(lead, smem_addr(&S.drain));
            bar_wait(smem_addr(&S.drain), 0, failed);
            if (*failed) settle(smem_addr(&S.drain), 0);
        } else if (warp == kHelpWarp && ragged) {
            bar_wait(smem_addr(&S.last), 0, failed);
            for (int load = 2 * n - 2; load < 2 * n; ++load) clean_tile<kDim>(tiles + load % kSlots * kBytes, K.n % kTile, lane);
            fence_async_shared();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.clean));
        }
    } else {
        registers_many();
        const int t = warp / kGroupWarps, row = threadIdx.x % kTile, i = first + row;
        const int limit = key_limit(Q, K, P.causal, i);
        const uint32_t lanes = static_cast<uint32_t>(warp % kGroupWarps * 32) << 16;
        const float scale = fmaxf(fabsf(P.scale), 1e-30f) * kLog2e;
        const int end = P.packed ? Q.n : P.seq_q;
        // the first group moves its rows of q to TMEM, the second those of do, and forms D on the way
        float dot = 0.0f;
        if (n > 0) {
            bar_wait(smem_addr(&S.stay), 0, failed);
            __syncwarp();
#pragma unroll
            for (int c = 0; c < kDim / 64; ++c) {
                const uint8_t *from = tiles + (kSlots - 3 + t) * kBytes + c * (kTile * 128) + row * 128;
                uint32_t r[32];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int at_piece = (x ^ (row & 7)) * 16;           // the copy's swizzle
                    const uint4 w = *reinterpret_cast<const uint4 *>(from + at_piece);
                    r[4 * x] = w.x; r[4 * x + 1] = w.y; r[4 * x + 2] = w.z; r[4 * x + 3] = w.w;
                    if (t) {
                        const uint4 u = *reinterpret_cast<const uint4 *>(from + kBytes + at_piece);
                        dot = dot2(w.x, u.x, dot2(w.y, u.y, dot2(w.z, u.z, dot2(w.w, u.w, dot))));
                    }
                }
                store_columns((t ? do_at : q_at) + lanes + c * 32, r);
            }
        }
        wait_stores();
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(smem_addr(&S.rows_in));
        if (t) S.row[0][0][row] = dot;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        dot = limit > 0 ? S.row[0][0][row] : 0.0f;
        float shift = INFINITY;                  // a row that sees nothing has p = exp2(-inf) = 0
        if (limit > 0) {
            shift = P.lse[stat_at(P, Q, i, at.head)] * kLog2e;
            if (shift == -INFINITY) shift = INFINITY;
        }
        if (t == 0 && i < end) P.row_dot[stat_at(P, Q, i, at.head)] = dot;
        const float2 by = make_float2(scale, scale), minus = make_float2(-shift, -shift), less = make_float2(-dot, -dot);
        for (int j = 0; j < n; ++j) {
            bar_wait(smem_addr(&S.score[0]), j & 1, failed);
            __syncwarp();
            fence_after();
            uint32_t s[2][32], d[2][32];
#pragma unroll
            for (int c = 0; c < 2; ++c) load_columns(s_at + lanes + t * 64 + c * 32, s[c]);
            wait_loads();
#pragma unroll
            for (int c = 0; c < 2; ++c) pin(s[c]);
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.prob[0]));
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int x = 0; x < 32; x += 2) {
                    float2 e = fma2(make_float2(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1])), by, minus);
                    e = x / 2 % kPolyBackward == kPolyBackward - 1 ? exp2_poly(e) : make_float2(exp2_fast(e.x), exp2_fast(e.y));
                    s[c][x] = __float_as_uint(e.x);
                    s[c][x + 1] = __float_as_uint(e.y);
                }
            const int left = limit - j * kTile - t * 64;
            if (__any_sync(0xffffffffu, left < 64)) {
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int x = 0; x < 32; ++x)
                        if (c * 32 + x >= left) s[c][x] = 0;
            }
            bar_wait(smem_addr(&S.second[0]), j & 1, failed);
            __syncwarp();
            fence_after();
#pragma unroll
            for (int c = 0; c < 2; ++c) load_columns(dp_at + lanes + t * 64 + c * 32, d[c]);
            wait_loads();
#pragma unroll
            for (int c = 0; c < 2; ++c) pin(d[c]);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t w[16];
#pragma unroll
                for (int x = 0; x < 32; x += 2) {
                    const float2 e = mul2(make_float2(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1])),
                                          add2(make_float2(__uint_as_float(d[c][x]), __uint_as_float(d[c][x + 1])), less));
                    w[x / 2] = pack_bf16(e.x, e.y);
                }
                store_columns(dp_at + lanes + t * 64 + c * 16, w);
            }
            wait_stores();
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.grad));
        }
        if (n > 0) bar_wait(smem_addr(&S.done), 0, failed);
        __syncwarp();
        fence_after();
        store_rows<kDim / 2>(tiles + warp * (32 * kDim), dq_at + lanes + t * (kDim / 2), n > 0, P.scale, limit > 0, P.dq, Q, i - lane, end, at.head,
                             t * (kDim / 2), P.head_dim);
    }
    __syncwarp();
    end_block<512>(S, tmem);
}

// ------------------------------------------------------------------------------------------------ backward: keys

// TMEM: dv, dk, S^T, dP^T and P^T; dS^T goes over dP^T.  S^T is free again once the softmax groups have it in registers, so
// that the next scores are computed under this tile's exponentials.  With heads of 128 that takes query tiles of 96: 128 of
// them would fill TMEM without a place of its own for P^T, and the next scores would wait for dv (measured at 4096, 32
// heads: 472 us).  A group has half of the tile's queries, a thread one key's half row.
template <int kDim> __host__ __device__ constexpr int query_tile() { return kDim == 128 ? 96 : 128; }
template <int kDim> __host__ __device__ constexpr int query_slots() { return kDim == 128 ? 6 : 10; }
template <int kDim> constexpr int shared_bytes_keys() {
    return 2 * tile_bytes<kDim>() + query_slots<kDim>() * query_tile<kDim>() * kDim * 2 + static_cast<int>(sizeof(Shared));
}
static_assert(shared_bytes_keys<128>() <= 227 * 1024 && shared_bytes_keys<64>() <= 227 * 1024, "shared memory of a block");

template <int kDim>
__global__ void __launch_bounds__(kThreads, 1) attention_backward_keys_kernel(const __grid_constant__ AttentionParams P, const __grid_constant__ Maps M) {
    constexpr int kSlots = query_slots<kDim>(), kRows = query_tile<kDim>(), kBytes = tile_bytes<kDim>(), kStep = kRows * kDim * 2;
    constexpr int kHalf = kRows / 2;
    extern __shared__ __align__(1024) uint8_t tiles[];
    Shared &S = *reinterpret_cast<Shared *>(tiles + 2 * kBytes + kSlots * kStep);
    const uint32_t base = smem_addr(tiles), ring = base + 2 * kBytes;
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) / 32, 0), lane = threadIdx.x % 32;
    const BlockPlace at = block_place(P, P.heads_kv, (P.max_k + kTile - 1) / kTile, false);
    const int first = at.tile * kTile;
    // only the block's set-up runs under the kernel over queries: what that one waited for is visible to it, not to this one
    if (P.packed && no_such_rows(P, key_rows, at.batch, first)) return;
    const uint32_t tmem = begin_block<512>(S, kSlots, 1, 2 * kGroupWarps);
    wait_for_previous();
    let_next_start();
    const Rows Q = query_rows(P, at.batch), K = key_rows(P, at.batch);
    // query tiles [from, until) see this tile; the heads of the group one after the other
    const int off = K.n - Q.n;
    const int until = (Q.n + kRows - 1) / kRows, from = P.causal ? min(until, max(0, first - off) / kRows) : 0;
    const int per = first < K.n ? until - from : 0, n = per * P.group;
    const bool ragged = ends_inside(Q, P.packed, P.seq_q, kRows);
    const uint32_t dv_at = tmem, dk_at = tmem + kDim, s_at = tmem + 2 * kDim, dp_at = s_at + kRows, p_at = dp_at + kRows;
    volatile uint32_t *const failed = &S.failed;

    if (warp >= 2 * kGroupWarps) {
        registers_few();
        if (warp == kLoadWarp && lane == 0 && n > 0) {
            Ring r;
            bar_expect(smem_addr(&S.stay), 2 * kBytes);
#pragma unroll
            for (int x = 0; x < kDim; x += 64) {
                load_box(base + x / 64 * (kTile * 128), &M.k, x, K.first + first, at.head, K.at, smem_addr(&S.stay));
                load_box(base + kBytes + x / 64 * (kTile * 128), &M.v, x, K.first + first, at.head, K.at, smem_addr(&S.stay));
            }
            int sent = 0, g = 0, tile = from;
            for (int j = 0; j < n; ++j) {
                for (int x = 0; x < 2; ++x) {
                    bar_wait(smem_addr(&S.empty[r.slot]), r.phase ^ 1, failed);
                    if (*failed) break;
                    load_tile<kDim, kRows>(ring + r.slot * kStep, x ? &M.d_o : &M.q, Q.first + tile * kRows, at.head * P.group + g, Q.at, smem_addr(&S.full[r.slot]));
                    ++sent;
                    r.next<kSlots>();
                }
                if (*failed) break;
                if (++tile == until) {
                    tile = from;
                    ++g;
                }
            }
            if (*failed) {
                settle(smem_addr(&S.stay), 0);
                for (int j = max(0, sent - kSlots); j < sent; ++j) settle(smem_addr(&S.full[j % kSlots]), j / kSlots & 1);
            }
        } else if (warp == kProductWarp && n > 0) {
            const uint32_t lead = elect_lane();
            const uint32_t scores = product(kRows, false, P.scale < 0.0f), plain = product(kRows, false);
            const auto slot = [](int load) { return load % kSlots; };
            const auto ready = [&](int load) { bar_wait(smem_addr(&S.full[load % kSlots]), load / kSlots & 1, failed); };
            const auto whole = [&](int j) { bar_wait(smem_addr(&S.stats[j % 2]), j / 2 & 1, failed); };
            bar_wait(smem_addr(&S.stay), 0, failed);
            whole(0);
            ready(0);
            product_scores<kDim, kRows>(lead, s_at, base, ring, scores);
            commit(lead, smem_addr(&S.score[0]));
            ready(1);
            product_scores<kDim, kRows>(lead, dp_at, base + kBytes, ring + kStep, plain);
            commit(lead, smem_addr(&S.second[0]));
            for (int j = 0; j < n; ++j) {
                if (j + 1 < n) {
                    whole(j + 1);
                    ready(2 * j + 2);
                    bar_wait(smem_addr(&S.prob[1]), j & 1, failed);
                    fence_after();
                    product_scores<kDim, kRows>(lead, s_at, base, ring + slot(2 * j + 2) * kStep, scores);
                    commit(lead, smem_addr(&S.score[0]));
                }
                bar_wait(smem_addr(&S.prob[0]), j & 1, failed);
                fence_after();
                product_apply<kDim, kRows>(lead, dv_at, p_at, p_at + kHalf / 2, ring + slot(2 * j + 1) * kStep, j > 0);
                commit(lead, smem_addr(&S.second[1]));
                commit(lead, smem_addr(&S.empty[slot(2 * j + 1)]));
                bar_wait(smem_addr(&S.grad), j & 1, failed);
                fence_after();
                product_apply<kDim, kRows>(lead, dk_at, dp_at, dp_at + kHalf, ring + slot(2 * j) * kStep, j > 0);
                commit(lead, smem_addr(&S.empty[slot(2 * j)]));
                if (j + 1 < n) {
                    ready(2 * j + 3);
                    product_scores<kDim, kRows>(lead, dp_at, base + kBytes, ring + slot(2 * j + 3) * kStep, plain);
                    commit(lead, smem_addr(&S.second[0]));
                }
            }
            commit(lead, smem_addr(&S.done));
            commit(lead, smem_addr(&S.drain));
            bar_wait(smem_addr(&S.drain), 0, failed);
            if (*failed) settle(smem_addr(&S.drain), 0);
        } else if (warp == kHelpWarp) {
            // row statistics of each query tile, read one tile ahead, and zeros past the sample's end in the tile that holds it
            constexpr int kMine = kRows / 32;
            float l[kMine], d[kMine];
            int g = 0, tile = from;
            const auto read = [&]() {
#pragma unroll
                for (int x = 0; x < kMine; ++x) {
                    const int i = tile * kRows + x * 32 + lane;
                    l[x] = INFINITY;             // no such query, or one that sees nothing: p = exp2(-inf) = 0
                    d[x] = 0.0f;
                    if (i < Q.n) {
                        const int64_t s = stat_at(P, Q, i, at.head * P.group + g);
                        l[x] = P.lse[s];
                        d[x] = P.row_dot[s];
                    }
                }
            };
            if (n > 0) read();
            for (int j = 0; j < n; ++j) {
                const int b = j % 2;
                const bool clean = ragged && tile == until - 1;
                bar_wait(smem_addr(&S.stats_free[b]), (j / 2 & 1) ^ 1, failed);
#pragma unroll
                for (int x = 0; x < kMine; ++x) {
                    S.row[b][0][x * 32 + lane] = l[x] == -INFINITY ? -INFINITY : -l[x] * kLog2e;
                    S.row[b][1][x * 32 + lane] = -d[x];
                }
                if (++tile == until) {
                    tile = from;
                    ++g;
                }
                if (j + 1 < n) read();
                if (clean) {
                    for (int load = 2 * j; load < 2 * j + 2; ++load) {
                        bar_wait(smem_addr(&S.full[load % kSlots]), load / kSlots & 1, failed);
                        clean_tile<kDim, kRows>(tiles + 2 * kBytes + load % kSlots * kStep, Q.n % kRows, lane);
                    }
                    fence_async_shared();
                }
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&S.stats[b]));
            }
        }
    } else {
        registers_many();
        const int t = warp / kGroupWarps, key = first + threadIdx.x % kTile;
        const uint32_t lanes = static_cast<uint32_t>(warp % kGroupWarps * 32) << 16;
        const uint32_t my_s = s_at + lanes + t * kHalf, my_dp = dp_at + lanes + t * kHalf, my_p = p_at + lanes + t * (kHalf / 2);
        const float scale = fmaxf(fabsf(P.scale), 1e-30f) * kLog2e;
        const float2 by = make_float2(scale, scale);
        int tile = from;
        for (int j = 0; j < n; ++j) {
            const int b = j % 2;
            const float4 *lse = reinterpret_cast<const float4 *>(S.row[b][0] + t * kHalf), *dot = reinterpret_cast<const float4 *>(S.row[b][1] + t * kHalf);
            bar_wait(smem_addr(&S.stats[b]), j / 2 & 1, failed);
            bar_wait(smem_addr(&S.score[0]), j & 1, failed);
            __syncwarp();
            fence_after();
            uint32_t s[kHalf / 16][16], d[kHalf / 16][16];
#pragma unroll
            for (int c = 0; c < kHalf / 16; ++c) load_columns(my_s + c * 16, s[c]);
            wait_loads();
#pragma unroll
            for (int c = 0; c < kHalf / 16; ++c) pin(s[c]);
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.prob[1]));
#pragma unroll
            for (int c = 0; c < kHalf / 16; ++c)
#pragma unroll
                for (int x = 0; x < 16; x += 4) {
                    const float4 l = lse[c * 4 + x / 4];
                    float2 e = fma2(make_float2(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1])), by, make_float2(l.x, l.y));
                    float2 f = fma2(make_float2(__uint_as_float(s[c][x + 2]), __uint_as_float(s[c][x + 3])), by, make_float2(l.z, l.w));
                    e = make_float2(exp2_fast(e.x), exp2_fast(e.y));
                    f = x / 2 % kPolyBackward == kPolyBackward - 2 ? exp2_poly(f) : make_float2(exp2_fast(f.x), exp2_fast(f.y));
                    s[c][x] = __float_as_uint(e.x);
                    s[c][x + 1] = __float_as_uint(e.y);
                    s[c][x + 2] = __float_as_uint(f.x);
                    s[c][x + 3] = __float_as_uint(f.y);
                }
            // under the causal mask the queries before key - off do not see this key; nor do those past the sample's end, whose zeros
            // times an infinite key are NaN
            const int begin = P.causal ? key - off - tile * kRows - t * kHalf : 0, stop = Q.n - tile * kRows - t * kHalf;
            if (__any_sync(0xffffffffu, begin > 0 || stop < kHalf)) {
                const unsigned live = static_cast<unsigned>(max(stop - begin, 0));
#pragma unroll
                for (int c = 0; c < kHalf / 16; ++c)
#pragma unroll
                    for (int x = 0; x < 16; ++x)
                        if (static_cast<unsigned>(c * 16 + x - begin) >= live) s[c][x] = 0;
            }
            if (++tile == until) tile = from;
            if (j > 0) {                         // dv has read the previous P^T
                bar_wait(smem_addr(&S.second[1]), (j - 1) & 1, failed);
                __syncwarp();
                fence_after();
            }
#pragma unroll
            for (int c = 0; c < kHalf / 16; ++c) {
                uint32_t w[8];
#pragma unroll
                for (int x = 0; x < 16; x += 2) w[x / 2] = pack_bf16(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1]));
                store_columns(my_p + c * 8, w);
            }
            wait_stores();
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&S.prob[0]));
            bar_wait(smem_addr(&S.second[0]), j & 1, failed);
            __syncwarp();
            fence_after();
#pragma unroll
            for (int c = 0; c < kHalf / 16; ++c) load_columns(my_dp + c * 16, d[c]);
            wait_loads();
#pragma unroll
            for (int c = 0; c < kHalf / 16; ++c) pin(d[c]);
#pragma unroll
            for (int c = 0; c < kHalf / 16; ++c) {
                uint32_t w[8];
#pragma unroll
                for (int x = 0; x < 16; x += 4) {
                    const float4 e = dot[c * 4 + x / 4];
                    const float2 f = mul2(make_float2(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1])),
                                          add2(make_float2(__uint_as_float(d[c][x]), __uint_as_float(d[c][x + 1])), make_float2(e.x, e.y)));
                    const float2 h = mul2(make_float2(__uint_as_float(s[c][x + 2]), __uint_as_float(s[c][x + 3])),
                                          add2(make_float2(__uint_as_float(d[c][x + 2]), __uint_as_float(d[c][x + 3])), make_float2(e.z, e.w)));
                    w[x / 2] = pack_bf16(f.x, f.y);
                    w[x / 2 + 1] = pack_bf16(h.x, h.y);
                }
                store_columns(my_dp + c * 8, w);
            }
            wait_stores();
            fence_before();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(smem_addr(&S.grad));
                bar_arrive(smem_addr(&S.stats_free[b]));
            }
        }
        if (n > 0) bar_wait(smem_addr(&S.done), 0, failed);
        __syncwarp();
        fence_after();
        // the first group writes dv, the second dk, each through one of the tiles that stayed
        store_rows<kDim>(tiles + t * kBytes + warp % kGroupWarps * (32 * kDim * 2), (t ? dk_at : dv_at) + lanes, n > 0, t ? P.scale : 1.0f, key < K.n,
                         t ? P.dk : P.dv, K, key - lane, P.packed ? K.n : P.seq_k, at.head, 0, P.head_dim);
    }
    __syncwarp();
    end_block<512>(S, tmem);
}

// ------------------------------------------------------------------------------------------------ host

namespace {

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
    static std::atomic<EncodeFn> known{nullptr};
    EncodeFn f = known.load();
    if (!f) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        f = reinterpret_cast<EncodeFn>(p);
        known.store(f);
    }
    return f;
}

// Heads as [batch, head, row, dim] in boxes of `box_rows` rows by 64 dimensions; what lies past the tensor reads as zero.
bool make_map(CUtensorMap &map, const Heads &t, int batch, int heads, int rows, int dim, int box_rows, const void *stand_in) {
    const EncodeFn encode = encode_fn();
    if (!encode) return false;
    const bool none = rows == 0 || batch == 0;             // never read
    void *at = none ? const_cast<void *>(stand_in) : static_cast<void *>(t.ptr);
    const cuuint64_t size[4] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(none ? 1 : rows), static_cast<cuuint64_t>(heads),
                                static_cast<cuuint64_t>(none ? 1 : batch)};
    // the stride of a single row, head or sample means nothing, but has to be a valid one
    const auto stride = [&](int64_t s, cuuint64_t n) { return static_cast<cuuint64_t>(n == 1 ? 256 : s * 2); };
    const cuuint64_t strides[3] = {stride(t.row_stride, size[1]), stride(t.head_stride, size[2]), stride(t.batch_stride, size[3])};
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(box_rows), 1, 1}, step[4] = {1, 1, 1, 1};
    const auto made = [&] {
        return encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, at, size, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    if (made()) return true;
    // Unlike a launch the encoding binds no context to the calling thread, and needs one: a thread's first call binds it.
    int dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess) return made();
    cudaGetLastError();
    return false;
}

using Kernel = void (*)(const AttentionParams, const Maps);

// Shared-memory limit of a kernel, set once per device.
bool allow(Kernel fn, int which, int bytes) {
    static std::atomic<bool> set[64][6];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return false;
    }
    if (set[dev][which].load(std::memory_order_acquire)) return true;
    if (cudaFuncSetAttribute(reinterpret_cast<const void *>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    set[dev][which].store(true, std::memory_order_release);
    return true;
}

// Without a causal mask blocks are alike, and heads come in spans whose streams stay in L2 (126 MB, whose halves may hold the
// same lines): with all heads at once 4096 rows of 32 heads were read from HBM three times over.  Backward in spans of 20 MB,
// of 40 MB, all at once: 1 x 4096, 32 heads of 128: 706, 712, 747 us; 2 x 4096, 32 over 8 of 128: 1489, 1506, 1540; 8 x 2048,
// 16 of 64: 711, 702, 722; 1 x 16384, 16 of 64: 4008, 4010, 4090; 4 x 1536, 64 over 8 of 128: 922, 917, 940; spans of 5 MB
// stay within 2% of 20.  Under a causal mask the longest blocks of all heads have to come first: one span (1 x 8192, 32 heads,
// backward 1467 us; in spans of 20 MB 1565, the grid ending in long blocks).
constexpr int64_t kSpanBytes = 20ll << 20;

// A launch, checked as far as the host can: nothing of a call is launched before all of it is.  `stream_bytes`: what the blocks
// of one head and sample read again and again.
struct Launch {
    Kernel fn;
    int which, bytes;                // place in allow(), shared memory
    int64_t blocks;
    int32_t span;
    Maps maps;
    bool ready() const { return blocks == 0 || allow(fn, which, bytes); }
    int go(const AttentionParams &P, cudaStream_t stream) const {
        if (blocks == 0) return LOCO_OK;
        AttentionParams Q = P;
        Q.span = span;
        return launch_kernel(fn, dim3(static_cast<unsigned>(blocks)), kThreads, static_cast<size_t>(bytes), stream, Q, maps);
    }
};
constexpr int64_t kMostBlocks = 0x7fffffff;
Launch plan(Kernel fn, int which, int bytes, int64_t tiles, int64_t heads, int64_t stream_bytes, const AttentionParams &P) {
    const int64_t span = kSpanBytes / (stream_bytes > 0 ? stream_bytes : 1), all = heads * P.batch;
    return Launch{fn, which, bytes, tiles * all, static_cast<int32_t>(P.causal || span > all ? all : span < 1 ? 1 : span), {}};
}

// What each kernel reads, in boxes of its own tiles.
bool make_query_map(const AttentionParams &P, CUtensorMap &map, const Heads &t, int box_rows) {
    return make_map(map, t, P.packed ? 1 : P.batch, P.heads_q, P.seq_q, P.head_dim, box_rows, P.seq_q > 0 ? P.q.ptr : P.k.ptr);
}
bool make_key_map(const AttentionParams &P, CUtensorMap &map, const Heads &t, int box_rows) {
    return make_map(map, t, P.packed ? 1 : P.batch, P.heads_kv, P.seq_k, P.head_dim, box_rows, P.seq_q > 0 ? P.q.ptr : P.k.ptr);
}

// Keys and values per query head, queries and their gradients per key head, of one sample on average.
int64_t key_bytes(const AttentionParams &P) { return 4ll * P.head_dim * P.seq_k / P.group / (P.packed ? P.batch : 1); }
int64_t query_bytes(const AttentionParams &P) { return 4ll * P.head_dim * P.seq_q * P.group / (P.packed ? P.batch : 1); }

template <int kDim> int forward(const AttentionParams &P, cudaStream_t stream) {
    Launch f = plan(attention_forward_kernel<kDim>, kDim / 64 - 1, forward_bytes<kDim>(), (P.max_q + 2 * kTile - 1) / (2 * kTile), P.heads_q, key_bytes(P), P);
    if (f.blocks > kMostBlocks) return LOCO_ERR_UNSUPPORTED;
    if (!make_query_map(P, f.maps.q, P.q, kTile) || !make_key_map(P, f.maps.k, P.k, key_tile<kDim>()) || !make_key_map(P, f.maps.v, P.v, key_tile<kDim>()) ||
        !f.ready()) return LOCO_ERR_CUDA;
    return f.go(P, stream);
}
template <int kDim> int backward(const AttentionParams &P, cudaStream_t stream) {
    Launch q = plan(attention_backward_queries_kernel<kDim>, 2 + kDim / 64 - 1, shared_bytes<kDim>(), (P.max_q + kTile - 1) / kTile, P.heads_q, key_bytes(P), P);
    Launch k = plan(attention_backward_keys_kernel<kDim>, 4 + kDim / 64 - 1, shared_bytes_keys<kDim>(), (P.max_k + kTile - 1) / kTile, P.heads_kv, query_bytes(P), P);
    if (q.blocks > kMostBlocks || k.blocks > kMostBlocks) return LOCO_ERR_UNSUPPORTED;
    if (!make_query_map(P, q.maps.q, P.q, kTile) || !make_query_map(P, q.maps.d_o, P.d_o, kTile) || !make_query_map(P, q.maps.o, P.o, kTile) ||
        !make_key_map(P, q.maps.k, P.k, kTile) || !make_key_map(P, q.maps.v, P.v, kTile)) return LOCO_ERR_CUDA;
    k.maps = q.maps;
    if (query_tile<kDim>() != kTile && (!make_query_map(P, k.maps.q, P.q, query_tile<kDim>()) || !make_query_map(P, k.maps.d_o, P.d_o, query_tile<kDim>())))
        return LOCO_ERR_CUDA;
    if (!q.ready() || !k.ready()) return LOCO_ERR_CUDA;
    const int rc = q.go(P, stream);
    return rc == LOCO_OK ? k.go(P, stream) : rc;
}

}  // namespace

int launch_attention_forward(const AttentionParams &P, cudaStream_t stream) {
    return P.head_dim <= 64 ? forward<64>(P, stream) : forward<128>(P, stream);
}

int launch_attention_backward(const AttentionParams &P, cudaStream_t stream) {
    return P.head_dim <= 64 ? backward<64>(P, stream) : backward<128>(P, stream);
}

}  // namespace loco_layer

extern "C" int loco_layer_status(uint32_t *flags, void *stream) {
    if (!flags) return LOCO_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    unsigned host = 0;
    if (cudaMemcpyFromSymbolAsync(&host, loco_layer::g_status, sizeof(host), 0, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
        cudaStreamSynchronize(s) != cudaSuccess) {
        cudaGetLastError();
        return LOCO_ERR_CUDA;
    }
    *flags = host;
    return LOCO_OK;
}
