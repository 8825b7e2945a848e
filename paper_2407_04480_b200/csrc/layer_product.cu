// The products of every expert's rows with its matrix, and the gradient of the matrices, on the tensor cores.
//
// One block to an SM, or two that work together, take tiles of outputs one after the other, expert by expert; where an expert's
// rows begin is known on the device only.  One warp copies 64 of the contraction at a time to a ring in shared memory (TMA,
// 128-byte swizzle), one issues the products, eight write the accumulator out while the next tile's products run into the other
// half of TMEM.  Where there are few tiles, up to eight blocks share the contraction of each.
//   product   A, the 128 lanes of the accumulator, are columns of the expert's matrix, either way round, and B, its columns, are rows
//             of x: as many as the expert has left, rounded up to 16 (two blocks: 32), so that no product is spent on an
//             expert's ragged end.  Rows past it belong to the next expert (or are the copy's zero fill): what they give is in
//             accumulator columns that are not written.
//   weights   A and B are rows of a and b, contracted along the rows.  Rows past the expert's last are zeroed in shared memory
//             in both, so that whatever lies there (NaN included) adds nothing.
#include <cuda.h>

#include <type_traits>

#include "layer_maps.h"
#include "layer_tc.cuh"

namespace loco_layer {

using namespace tc;

constexpr int kMostExperts = 512;
constexpr int kMostColumns = 1 << 30;            // coordinates are 32 bits, some of them past the end
constexpr int kTileRows = 128;                   // of the accumulator
constexpr int kStep = 64;                        // of the contraction: a swizzled row of 128 bytes
constexpr int kProductThreads = 384;
constexpr int kLoadWarp = 0, kIssueWarp = 1, kCleanWarp = 2, kFirstWriter = 4, kWriteWarps = 8;        // lanes of TMEM go by the warp's number modulo 4

__device__ unsigned g_product_status;            // LOCO_LAYER_FLAG_*
// At a block's end: whether one of its waits has run out.
__device__ __forceinline__ void report(uint32_t failed) {
    if (threadIdx.x == 0 && failed) atomicOr(&g_product_status, LOCO_LAYER_FLAG_TIMEOUT);
}

struct ProductMaps { CUtensorMap a, b; };
struct ProductParams {
    const int32_t *offsets;
    __nv_bfloat16 *out;
    int64_t out_expert, out_row, rows;
    int32_t experts, deep, high, wide;           // contraction (product), rows of an output matrix (weights), columns of the output
    int32_t last;                                // experts' last tiles of rows, where they are not full, come after all full ones
};

constexpr int kMostStages = 12;
constexpr int kMostParts = 8;                    // SMs to the contraction of a tile
struct ProductShared {
    uint64_t full[kMostStages], edge[kMostStages], empty[kMostStages], clean[kMostStages], ready[2], written[2], drain;
    uint32_t tmem, failed;
    int32_t begin[kMostExperts], count[kMostExperts];                // rows of an expert
    int32_t first[kMostExperts + 1], ends[kMostExperts + 1];         // tiles of rows, and tiles that come last, before it
};
constexpr int kPiece = 32;                       // columns that a writing warp puts to shared memory at a time
constexpr int kPieceBytes = 32 * kPiece * 2;     // of its 32 rows
constexpr int kBesides = 1024 + kWriteWarps * kPieceBytes + static_cast<int>(sizeof(ProductShared));     // of shared memory besides the stages
// 128 of A and kN of B to a stage of one block.
template <int kN> __host__ __device__ constexpr int stage_bytes() { return (kTileRows + kN) * 128; }
template <int kN> __host__ __device__ constexpr int stages() {
    constexpr int n = (227 * 1024 - kBesides) / stage_bytes<kN>();
    return n < kMostStages ? n : kMostStages;
}
template <int kN> constexpr int product_bytes() { return kBesides + stages<kN>() * stage_bytes<kN>(); }

__device__ __forceinline__ void load_box3(uint32_t to, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// Where the tiles are.  `walk` goes on to the tile's expert; tiles only grow.
struct Tile {
    int expert, row, col, rows, steps;           // first row within the expert (product) or the matrix (weights), columns; rows of the expert, steps of the contraction
};
template <bool kWeights, int kRows, int kCols> struct Walk {
    int expert = 0;
    bool ends = false;
    __device__ __forceinline__ static int across(const ProductParams &P) { return (P.wide + kCols - 1) / kCols; }
    __device__ __forceinline__ static int tiles(const ProductShared &S, const ProductParams &P) {
        return (kWeights ? P.experts * ((P.high + kRows - 1) / kRows) : S.first[P.experts] + S.ends[P.experts]) * across(P);
    }
    __device__ __forceinline__ Tile at(const ProductShared &S, const ProductParams &P, int tile) {
        const int wide = across(P);
        if constexpr (kWeights) {
            const int down = (P.high + kRows - 1) / kRows, each = down * wide;
            expert = tile / each;
            const int r = tile - expert * each, n = S.count[expert];
            return Tile{expert, r % down * kRows, r / down * kCols, n, (n + kStep - 1) / kStep};
        } else {
            const int steps = (P.deep + kStep - 1) / kStep, full = S.first[P.experts] * wide;
            if (tile < full) {
                while (tile >= S.first[expert + 1] * wide) ++expert;
                const int down = S.first[expert + 1] - S.first[expert], r = tile - S.first[expert] * wide;
                // bands of eight tiles of rows, column by column, so that the blocks at work share rows and columns in L2
                const int band = r / (8 * wide), high = min(8, down - band * 8), q = r - band * 8 * wide;
                return Tile{expert, (band * 8 + q % high) * kRows, q / high * kCols, S.count[expert], steps};
            }
            if (!ends) expert = 0;
            ends = true;
            const int r = tile - full, end = r / wide;
            while (end >= S.ends[expert + 1]) ++expert;
            return Tile{expert, S.count[expert] / kRows * kRows, (r - end * wide) * kCols, S.count[expert], steps};
        }
    }
};

// Zeros in the rows from `left` on up to the next step of 16 in each of kBlocks blocks of 64 columns, by one warp.
template <int kBlocks> __device__ __forceinline__ void clean_rows(uint8_t *stage, int left, int lane) {
    const int end = (left + 15) / 16 * 16;
    for (int x = 0; x < kBlocks; ++x)
        for (int i = left * 8 + lane; i < end * 8; i += 32) reinterpret_cast<uint4 *>(stage + x * (kStep * 128))[i] = make_uint4(0, 0, 0, 0);
    fence_async_shared();
    __syncwarp();
}

// Rows of every expert, and the tiles of kRows rows before it, to shared memory.  Offsets are read as the largest so far, within the
// tensor, whatever they hold: experts' rows never overlap.
template <int kRows> __device__ __forceinline__ void find_rows(ProductShared &S, const ProductParams &P) {
    const int lane = threadIdx.x % 32;
    if (threadIdx.x >= 32) return;
    const auto offset = [&](int e) {
        const int64_t o = P.offsets[e < P.experts ? e : P.experts];
        return static_cast<int>(o < 0 ? 0 : o > P.rows ? P.rows : o);
    };
    int most = 0, before = 0, ended = 0;         // of the offsets, the tiles and the last tiles of the experts before
    for (int e0 = 0; e0 < P.experts; e0 += 32) {
        const int e = e0 + lane;
        int lo = max(offset(e), most);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, lo, o);
            lo = lane >= o ? max(lo, y) : lo;
        }
        const int hi = max(offset(e + 1), lo), rows = e < P.experts ? hi - lo : 0;
        int n = P.last ? rows / kRows : (rows + kRows - 1) / kRows;
        const unsigned ends = __ballot_sync(0xffffffffu, P.last && rows % kRows != 0);
        if (e < P.experts) {
            S.begin[e] = lo;
            S.count[e] = rows;
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, n, o);
            n += lane >= o ? y : 0;
        }
        if (e < P.experts) {
            S.first[e + 1] = before + n;
            S.ends[e + 1] = ended + __popc(ends & (0xffffffffu >> (31 - lane)));
        }
        before += __shfl_sync(0xffffffffu, n, 31);
        ended += __popc(ends);
        most = __shfl_sync(0xffffffffu, hi, 31);
    }
    if (lane == 0) S.first[0] = S.ends[0] = 0;
}

__device__ __forceinline__ void settle(uint32_t bar, uint32_t parity) {
    const uint64_t begin = now_ns();
    while (!bar_test(bar, parity) && now_ns() - begin < kWaitLimitNs / 20) {}
}

// A writing warp's part of the accumulator of a tile of dw: 32 rows of half the columns, `below` rows into the tile, through shared memory so
// that a store covers 64 bytes of a row.  (With copies of 64 columns by the copy engine instead of stores the gradient of 64
// matrices of 2048 x 1032 over 47 rows each took 102 us, 50634 rows of 256 through 3328 columns 171.)  `done` is called by one lane
// when the accumulator has been read.  Zeros for a tile without a contraction.
template <int kRows, int kCols, typename Done>
__device__ __forceinline__ void write_tile(const ProductShared &S, const ProductParams &P, const Tile &t, int below, uint32_t accumulator, uint8_t *staging,
                                           const Done &done) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32 - kFirstWriter, part = warp % 4, half = warp / 4 * (kCols / 2), first = t.row + below + part * 32;
    uint8_t *const stage = staging + warp * kPieceBytes;
    const int live = min(min(P.high, t.row + kRows) - first, 32), cols = P.wide - t.col - half;       // that are written
    __nv_bfloat16 *const out = P.out + t.expert * P.out_expert + first * P.out_row + t.col + half;
    const int piece = lane % 4, end = live > 0 ? min(kCols / 2, cols) : 0;
    const auto read = [&] {                      // ahead of the last stores, which the arrival need not wait for
        fence_before();
        __syncwarp();
        if (lane == 0) done();
    };
    if (t.steps > 0 && end <= 0) read();
#pragma unroll 1
    for (int c = 0; c < end; c += kPiece) {
        uint32_t r[32];
        if (t.steps > 0) {
            load_columns(accumulator + half + c + (static_cast<uint32_t>(part * 32) << 16), r);
            wait_loads();
            pin(r);
            if (c + kPiece >= end) read();
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = 0;
        }
#pragma unroll
        for (int i = 0; i < kPiece; i += 8) {
            uint4 w;
            w.x = pack_bf16(__uint_as_float(r[i]), __uint_as_float(r[i + 1]));
            w.y = pack_bf16(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
            w.z = pack_bf16(__uint_as_float(r[i + 4]), __uint_as_float(r[i + 5]));
            w.w = pack_bf16(__uint_as_float(r[i + 6]), __uint_as_float(r[i + 7]));
            *reinterpret_cast<uint4 *>(stage + lane * 64 + ((i / 8 ^ lane / 2 % 4) << 4)) = w;
        }
        __syncwarp();
        if (c + piece * 8 < cols)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = lane / 4 + i * 8;
                if (row < live)
                    *reinterpret_cast<uint4 *>(out + row * P.out_row + c + piece * 8) = *reinterpret_cast<const uint4 *>(stage + row * 64 + ((piece ^ row / 2 % 4) << 4));
            }
        __syncwarp();
    }
}

// The same of a product's tile: the warp's 32 lanes are columns of the output from `col` on, the accumulator's columns its rows.
// The two halves of the writing warps take 32 rows in turn.
// Where rows are many and the contraction short, stores bound a product: 55880 rows of 120 through 13,536 columns leave at 3.0 TB/s, where
// memory that is only written takes 3.9.
template <int kN, typename Done>
__device__ __forceinline__ void write_rows(const ProductShared &S, const ProductParams &P, const Tile &t, int col, uint32_t accumulator, uint8_t *staging,
                                           const Done &done) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32 - kFirstWriter, part = warp % 4, first = warp / 4 * 32;
    uint8_t *const stage = staging + warp * kPieceBytes;
    col += part * 32;
    const int piece = lane % 4, end = col < P.wide ? min(t.rows - t.row, kN) : 0;
    __nv_bfloat16 *const out = P.out + (S.begin[t.expert] + static_cast<int64_t>(t.row)) * P.out_row + col + piece * 8;
    const auto read = [&] {
        fence_before();
        __syncwarp();
        if (lane == 0) done();
    };
    if (first >= end) read();
#pragma unroll 1
    for (int j = first; j < end; j += 64) {
        uint32_t r[32];
        load_columns(accumulator + j + (static_cast<uint32_t>(part * 32) << 16), r);
        wait_loads();
        pin(r);
        if (j + 64 >= end) read();
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const uint32_t w = pack_bf16(__uint_as_float(r[i]), __uint_as_float(r[i + 1]));
            *reinterpret_cast<uint16_t *>(stage + i * 64 + lane * 2) = static_cast<uint16_t>(w);
            *reinterpret_cast<uint16_t *>(stage + i * 64 + 64 + lane * 2) = static_cast<uint16_t>(w >> 16);
        }
        __syncwarp();
        if (col + piece * 8 < P.wide)
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                const int row = lane / 4 + i;
                if (j + row < end) *reinterpret_cast<uint4 *>(out + (j + row) * P.out_row) = *reinterpret_cast<const uint4 *>(stage + row * 64 + piece * 16);
            }
        __syncwarp();
    }
}

// An instruction word's part for n columns of the accumulator.
__device__ __forceinline__ uint32_t columns_word(int n) { return static_cast<uint32_t>(n >> 3) << 17; }

// kDown: the matrices are [in, out], their rows are the contraction (and in weights a's and b's); else [out, in].
template <bool kWeights, bool kDown, int kN>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ ProductParams P, const __grid_constant__ ProductMaps M) {
    constexpr int kStages = stages<kN>(), kBytes = stage_bytes<kN>();
    constexpr int kRows = kWeights ? kTileRows : kN, kCols = kWeights ? kN : kTileRows;          // of the output's tile
    constexpr uint32_t kTmem = 2 * kN;
    extern __shared__ uint8_t raw[];
    uint8_t *const ring = raw + (1024 - smem_addr(raw) % 1024) % 1024;      // not by an integer, past which nobody knows that it is shared memory
    uint8_t *const staging = ring + kStages * kBytes;
    ProductShared &S = *reinterpret_cast<ProductShared *>(staging + kWriteWarps * kPieceBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile uint32_t *const failed = &S.failed;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            bar_init(smem_addr(&S.full[i]), 1);
            bar_init(smem_addr(&S.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_addr(&S.ready[i]), 1);
            bar_init(smem_addr(&S.written[i]), kWriteWarps);
        }
        bar_init(smem_addr(&S.drain), 1);
        S.failed = 0;
        fence_bar_init();
        fence_async_shared();
    }
    if (warp == kIssueWarp) tmem_alloc<kTmem>(smem_addr(&S.tmem));
    wait_for_previous();
    let_next_start();
    find_rows<kRows>(S, P);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = S.tmem;
    const int stride = static_cast<int>(gridDim.x);
    const uint32_t base = smem_addr(ring);
    Walk<kWeights, kRows, kCols> walk;
    const int tiles = walk.tiles(S, P);

    if (warp == kLoadWarp) {
        if (lane == 0) {
            int slot = 0, phase = 0, issued = 0;
            for (int tile = blockIdx.x; tile < tiles && !*failed; tile += stride) {
                const Tile t = walk.at(S, P, tile);
                const int begin = S.begin[t.expert];
                for (int k = 0; k < t.steps; ++k) {
                    bar_wait(smem_addr(&S.empty[slot]), phase ^ 1, failed);
                    if (*failed) break;
                    const uint32_t a = base + slot * kBytes, b = a + kTileRows * 128, bar = smem_addr(&S.full[slot]);
                    bar_expect(bar, kBytes);
                    if constexpr (kWeights) {
#pragma unroll
                        for (int x = 0; x < kTileRows; x += 64) load_box3(a + x * 128, &M.a, t.row + x, begin + k * kStep, 0, bar);
#pragma unroll
                        for (int x = 0; x < kN; x += 64) load_box3(b + x * 128, &M.b, t.col + x, begin + k * kStep, 0, bar);
                    } else {
                        if constexpr (kDown) {
#pragma unroll
                            for (int x = 0; x < kTileRows; x += 64) load_box3(a + x * 128, &M.a, t.col + x, k * kStep, t.expert, bar);
                        } else {
                            load_box3(a, &M.a, k * kStep, t.col, t.expert, bar);
                        }
                        load_box3(b, &M.b, k * kStep, begin + t.row, 0, bar);
                    }
                    ++issued;
                    if (++slot == kStages) {
                        slot = 0;
                        phase ^= 1;
                    }
                }
            }
            for (int i = 0, s = slot, p = phase; i < kStages && i < issued; ++i) {
                s = s ? s - 1 : kStages - 1;
                if (s == kStages - 1) p ^= 1;
                bar_wait(smem_addr(&S.empty[s]), p, failed);
            }
            if (*failed)                         // copies in flight end before the block's shared memory goes away
                for (int i = 0; i < kStages && i < issued; ++i) {
                    slot = slot ? slot - 1 : kStages - 1;
                    if (slot == kStages - 1) phase ^= 1;
                    settle(smem_addr(&S.full[slot]), phase);
                }
        }
    } else if (warp == kIssueWarp) {
        const uint32_t lead = elect_lane();
        constexpr uint32_t plain = product(0, kWeights) | (kDown ? 1u << 15 : 0u);
        int slot = 0, phase = 0, buffer = 0, turn = 0;
        for (int tile = blockIdx.x; tile < tiles; tile += stride) {
            const Tile t = walk.at(S, P, tile);
            if (t.steps == 0) continue;
            const uint32_t word = plain | columns_word(kWeights ? kN : min(kN, (t.rows - t.row + 15) / 16 * 16));
            bar_wait(smem_addr(&S.written[buffer]), turn ^ 1, failed);
            fence_after();
            for (int k = 0; k < t.steps; ++k) {
                bar_wait(smem_addr(&S.full[slot]), phase, failed);
                __syncwarp();
                const int left = kWeights ? t.rows - k * kStep : kStep;
                if (left < kStep) clean_rows<(kTileRows + kN) / 64>(ring + slot * kBytes, left, lane);
                fence_after();
                const uint32_t a = base + slot * kBytes, b = a + kTileRows * 128;
                const uint32_t da = kDown ? desc_along_rows(a, kStep * 128) : desc_along_columns(a);
                const uint32_t db = kWeights ? desc_along_rows(b, kStep * 128) : desc_along_columns(b);
#pragma unroll
                for (int x = 0; x < kStep; x += 16)
                    if (!kWeights || x < left)   // whole steps past the expert's last row are left out
                        mma_ss(lead, tmem + buffer * kN, da + (kDown ? x * 128 >> 4 : x * 2 >> 4), db + (kWeights ? x * 128 >> 4 : x * 2 >> 4), word, k > 0 || x > 0);
                commit(lead, smem_addr(&S.empty[slot]));
                if (++slot == kStages) {
                    slot = 0;
                    phase ^= 1;
                }
            }
            commit(lead, smem_addr(&S.ready[buffer]));
            buffer ^= 1;
            if (buffer == 0) turn ^= 1;
        }
        commit(lead, smem_addr(&S.drain));
        bar_wait(smem_addr(&S.drain), 0, failed);
        if (*failed) settle(smem_addr(&S.drain), 0);
    } else if (warp >= kFirstWriter) {
        int buffer = 0, turn = 0;
        for (int tile = blockIdx.x; tile < tiles; tile += stride) {
            const Tile t = walk.at(S, P, tile);
            if (t.steps > 0) {
                bar_wait(smem_addr(&S.ready[buffer]), turn, failed);
                __syncwarp();
                fence_after();
            }
            const auto done = [&] { bar_arrive(smem_addr(&S.written[buffer])); };
            if constexpr (kWeights) write_tile<kTileRows, kN>(S, P, t, 0, tmem + buffer * kN, staging, done);
            else write_rows<kN>(S, P, t, t.col, tmem + buffer * kN, staging, done);
            if (t.steps > 0) {
                buffer ^= 1;
                if (buffer == 0) turn ^= 1;
            }
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kIssueWarp) tmem_free<kTmem>(tmem);
    report(S.failed);
}

// ---- two SMs to a tile -----------------------------------------------------------------------

// Tiles of 256 x 256 by a cluster of two blocks: each holds 128 of A and 128 of B, and 128 lanes of the accumulator; the products,
// issued by the first, read both.  Against one SM's 128 x 256 each byte of B is copied to and read from shared memory half as
// often.
constexpr int kPairRows = 256, kPairCols = 256, kPairStage = 2 * kTileRows * 128;
constexpr int kPairStages = (227 * 1024 - kBesides) / kPairStage;
constexpr int kPairBytes = kBesides + kPairStages * kPairStage;
static_assert(kPairStages == 6, "shared memory of a block");

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The same place in the shared memory of block `rank` of the cluster.
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// In any block of the cluster, with what this thread wrote before...
__device__ __forceinline__ void bar_arrive_in(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// ... or without, where only an accumulator is handed back: its loads are complete, and the tcgen05 fences on both sides order what comes
// after.  A release to the cluster waits for the thread's stores to global memory (2600 tiles of 256 steps: 120 us with it).
__device__ __forceinline__ void bar_arrive_in_relaxed(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Once more, for what another block of the cluster did before it arrived.
__device__ __forceinline__ bool bar_test_cluster(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// A box to this block's shared memory; completes on a barrier of either block.
__device__ __forceinline__ void load_box3_pair(uint32_t to, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
template <int kColumns> __device__ __forceinline__ void tmem_alloc_pair(uint32_t to) {       // one warp of each block
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
template <int kColumns> __device__ __forceinline__ void tmem_free_pair(uint32_t at) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(kColumns) : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t word, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n mov.b64 a, {%1, %6};\n mov.b64 b, {%2, %6};\n setp.ne.u32 p, %4, 0;\n setp.ne.u32 q, %5, 0;\n"
                 " @q tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "r"(b), "r"(word), "r"(accumulate), "r"(lead), "r"(kDescHigh) : "memory");
}
// Arrives on the barrier of both blocks when every product issued is complete.
__device__ __forceinline__ void commit_pair(uint32_t lead, uint32_t bar) {
    asm volatile("{\n .reg .pred q;\n .reg .b16 m;\n setp.ne.u32 q, %1, 0;\n mov.b16 m, 3;\n"
                 " @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n}\n"
                 ::"r"(bar), "r"(lead) : "memory");
}

// Columns of a product's accumulator: the rows that the expert has left, half of them each block's.
__device__ __forceinline__ int pair_columns(const Tile &t) { return min(kPairRows, (t.rows - t.row + 31) / 32 * 32); }

template <bool kWeights, bool kDown>
__global__ void __launch_bounds__(kProductThreads, 1) product_pair_kernel(const __grid_constant__ ProductParams P, const __grid_constant__ ProductMaps M) {
    extern __shared__ uint8_t raw[];
    uint8_t *const ring = raw + (1024 - smem_addr(raw) % 1024) % 1024;      // not by an integer, past which nobody knows that it is shared memory
    uint8_t *const staging = ring + kPairStages * kPairStage;
    ProductShared &S = *reinterpret_cast<ProductShared *>(staging + kWriteWarps * kPieceBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    volatile uint32_t *const failed = &S.failed;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairStages; ++i) {
            bar_init(smem_addr(&S.full[i]), 1);                      // the first block's: both blocks' copies, but for those with rows past
            bar_init(smem_addr(&S.edge[i]), 1);                      // an expert's end in them, which each block has on its own `edge`
            bar_init(smem_addr(&S.empty[i]), 1);
            bar_init(smem_addr(&S.clean[i]), 2);                     // the first block's: those rows are zero in both
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_addr(&S.ready[i]), 1);
            bar_init(smem_addr(&S.written[i]), 2 * kWriteWarps);     // the first block's: both blocks' warps
        }
        bar_init(smem_addr(&S.drain), 1);
        S.failed = 0;
        fence_bar_init();
        fence_async_shared();
    }
    if (warp == kIssueWarp) tmem_alloc_pair<512>(smem_addr(&S.tmem));
    wait_for_previous();
    let_next_start();
    find_rows<kPairRows>(S, P);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = S.tmem;
    const int begin = static_cast<int>(blockIdx.x) / 2, stride = static_cast<int>(gridDim.x) / 2;
    const uint32_t base = smem_addr(ring);
    Walk<kWeights, kPairRows, kPairCols> walk;
    const int tiles = walk.tiles(S, P);

    if (warp == kLoadWarp) {
        if (lane == 0) {
            int slot = 0, phase = 0, issued = 0;
            for (int tile = begin; tile < tiles && !*failed; tile += stride) {
                const Tile t = walk.at(S, P, tile);
                const int first = S.begin[t.expert], row = t.row + rank * (kWeights ? kTileRows : pair_columns(t) / 2), col = t.col + rank * kTileRows;
                for (int k = 0; k < t.steps; ++k) {
                    bar_wait(smem_addr(&S.empty[slot]), phase ^ 1, failed);
                    if (*failed) break;
                    const bool ragged = kWeights && t.rows - k * kStep < kStep;
                    const uint32_t a = base + slot * kPairStage, b = a + kTileRows * 128;
                    const uint32_t own = smem_addr(ragged ? &S.edge[slot] : &S.full[slot]), bar = in_block(own, ragged ? rank : 0);
                    if (rank == 0 || ragged) bar_expect(own, ragged ? kPairStage : 2 * kPairStage);
                    if constexpr (kWeights) {
#pragma unroll
                        for (int x = 0; x < kTileRows; x += 64) {
                            load_box3_pair(a + x * 128, &M.a, row + x, first + k * kStep, 0, bar);
                            load_box3_pair(b + x * 128, &M.b, col + x, first + k * kStep, 0, bar);
                        }
                    } else {
                        if constexpr (kDown) {
#pragma unroll
                            for (int x = 0; x < kTileRows; x += 64) load_box3_pair(a + x * 128, &M.a, col + x, k * kStep, t.expert, bar);
                        } else {
                            load_box3_pair(a, &M.a, k * kStep, col, t.expert, bar);
                        }
                        load_box3_pair(b, &M.b, k * kStep, first + row, 0, bar);
                    }
                    ++issued;
                    if (++slot == kPairStages) {
                        slot = 0;
                        phase ^= 1;
                    }
                }
            }
            for (int i = 0; i < kPairStages && i < issued; ++i) {    // the first block's products say so in this one's memory
                slot = slot ? slot - 1 : kPairStages - 1;
                if (slot == kPairStages - 1) phase ^= 1;
                bar_wait(smem_addr(&S.empty[slot]), phase, failed);
            }
            if (rank == 1 && !*failed) bar_wait(smem_addr(&S.drain), 0, failed);      // the last arrival from there
            if (*failed && issued > 0) {         // copies in flight end before the blocks' shared memory goes away: nothing tells when, so
                const uint64_t from = now_ns();  // they get far more time than a copy takes
                while (now_ns() - from < 1000000ull) {}
            }
        }
    } else if (warp == kIssueWarp) {
        const uint32_t lead = elect_lane();
        constexpr uint32_t plain = (product(0, kWeights) & 0x00ffffffu) | (16u << 24) | (kDown ? 1u << 15 : 0u);       // 256 lanes
        int slot = 0, buffer = 0, turn = 0;
        uint32_t fulls = 0, ends = 0;            // by slot: the phases of `full`, and of `edge` and `clean`
        for (int tile = begin; tile < tiles && rank == 0; tile += stride) {
            const Tile t = walk.at(S, P, tile);
            if (t.steps == 0) continue;
            const uint32_t word = plain | columns_word(kWeights ? kPairCols : pair_columns(t));
            bar_wait(smem_addr(&S.written[buffer]), turn ^ 1, failed);
            for (int k = 0; k < t.steps; ++k) {
                const int left = kWeights ? t.rows - k * kStep : kStep;
                if (left < kStep) {
                    bar_wait(smem_addr(&S.edge[slot]), ends >> slot & 1, failed);
                    bar_wait(smem_addr(&S.clean[slot]), ends >> slot & 1, failed);
                    bar_test_cluster(smem_addr(&S.clean[slot]), ends >> slot & 1);     // what the other block did before it arrived is seen
                    ends ^= 1u << slot;
                } else {
                    bar_wait(smem_addr(&S.full[slot]), fulls >> slot & 1, failed);
                    fulls ^= 1u << slot;
                }
                __syncwarp();
                fence_after();
                const uint32_t a = base + slot * kPairStage, b = a + kTileRows * 128;
                const uint32_t da = kDown ? desc_along_rows(a, kStep * 128) : desc_along_columns(a);
                const uint32_t db = kWeights ? desc_along_rows(b, kStep * 128) : desc_along_columns(b);
#pragma unroll
                for (int x = 0; x < kStep; x += 16)
                    if (!kWeights || x < left)
                        mma_pair(lead, tmem + buffer * kPairCols, da + (kDown ? x * 128 >> 4 : x * 2 >> 4), db + (kWeights ? x * 128 >> 4 : x * 2 >> 4), word, k > 0 || x > 0);
                commit_pair(lead, smem_addr(&S.empty[slot]));
                if (++slot == kPairStages) slot = 0;
            }
            commit_pair(lead, smem_addr(&S.ready[buffer]));
            buffer ^= 1;
            if (buffer == 0) turn ^= 1;
        }
        if (rank == 0) {
            commit_pair(lead, smem_addr(&S.drain));
            bar_wait(smem_addr(&S.drain), 0, failed);
            if (*failed) settle(smem_addr(&S.drain), 0);
        }
    } else if (warp == kCleanWarp && kWeights) {
        // Zeros in the rows past an expert's last, in this block's part of the step that holds them.  A phase told by its parity has to be
        // the current one or the last: `edge` has such steps' phases alone, and their slots are filled again only after their products,
        // which wait for this warp's arrival.
        int slot = 0;
        uint32_t ends = 0;                       // by slot: the phase of `edge`
        for (int tile = begin; tile < tiles; tile += stride) {
            const Tile t = walk.at(S, P, tile);
            if (t.steps == 0) continue;
            slot = (slot + t.steps - 1) % kPairStages;               // of the tile's last step
            const int left = t.rows - (t.steps - 1) * kStep;
            if (left < kStep) {
                bar_wait(smem_addr(&S.edge[slot]), ends >> slot & 1, failed);
                ends ^= 1u << slot;
                __syncwarp();
                clean_rows<2 * kTileRows / 64>(ring + slot * kPairStage, left, lane);
                if (lane == 0) bar_arrive_in(in_block(smem_addr(&S.clean[slot]), 0));
            }
            slot = (slot + 1) % kPairStages;
        }
    } else if (warp >= kFirstWriter) {
        int buffer = 0, turn = 0;
        for (int tile = begin; tile < tiles; tile += stride) {
            const Tile t = walk.at(S, P, tile);
            if (t.steps > 0) {
                bar_wait(smem_addr(&S.ready[buffer]), turn, failed);
                __syncwarp();
                fence_after();
            }
            const auto done = [&] { bar_arrive_in_relaxed(in_block(smem_addr(&S.written[buffer]), 0)); };
            if constexpr (kWeights) write_tile<kPairRows, kPairCols>(S, P, t, rank * kTileRows, tmem + buffer * kPairCols, staging, done);
            else write_rows<kPairRows>(S, P, t, t.col + rank * kTileRows, tmem + buffer * kPairCols, staging, done);
            if (t.steps > 0) {
                buffer ^= 1;
                if (buffer == 0) turn ^= 1;
            }
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    cluster_sync();                              // neither block leaves while the other's products read it or its arrivals are under way
    fence_after();
    if (warp == kIssueWarp) tmem_free_pair<512>(tmem);
    report(S.failed);
}

// ---- several SMs to the contraction of a tile -------------------------------------------------

__device__ __forceinline__ uint32_t cluster_blocks() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float4 load_in_block(uint32_t at) {
    float4 f;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(at) : "memory");
    return f;
}

// Few tiles with a long contraction: the blocks of a cluster take a part of it each for one tile of kN rows by 128 columns, leave
// their sums in shared memory, and each adds up, in the blocks' order, and writes a part of the tile.
template <bool kDown, int kN>
__global__ void __launch_bounds__(kProductThreads, 1) product_split_kernel(const __grid_constant__ ProductParams P, const __grid_constant__ ProductMaps M) {
    constexpr int kStages = stages<kN>(), kBytes = stage_bytes<kN>();
    static_assert(kN * kTileRows * 4 <= kStages * kBytes, "the sums are left where the copies were");
    extern __shared__ uint8_t raw[];
    uint8_t *const ring = raw + (1024 - smem_addr(raw) % 1024) % 1024;
    ProductShared &S = *reinterpret_cast<ProductShared *>(ring + kStages * kBytes + kWriteWarps * kPieceBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rank = static_cast<int>(cluster_rank()), parts = static_cast<int>(cluster_blocks());
    volatile uint32_t *const failed = &S.failed;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            bar_init(smem_addr(&S.full[i]), 1);
            bar_init(smem_addr(&S.empty[i]), 1);
        }
        bar_init(smem_addr(&S.ready[0]), 1);
        S.failed = 0;
        fence_bar_init();
        fence_async_shared();
    }
    if (warp == kIssueWarp) tmem_alloc<kN>(smem_addr(&S.tmem));
    wait_for_previous();
    let_next_start();
    find_rows<kN>(S, P);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = S.tmem, base = smem_addr(ring);
    Walk<false, kN, kTileRows> walk;
    const int tile = static_cast<int>(blockIdx.x) / parts;
    const bool some = tile < walk.tiles(S, P);   // the same for all blocks of the cluster
    Tile t{};
    if (some) t = walk.at(S, P, tile);
    const int from = static_cast<int>(static_cast<int64_t>(t.steps) * rank / parts), until = static_cast<int>(static_cast<int64_t>(t.steps) * (rank + 1) / parts);
    const int rows = min(t.rows - t.row, kN);

    if (some && warp == kLoadWarp) {
        if (lane == 0) {
            int slot = 0, phase = 0, issued = 0;
            for (int k = from; k < until; ++k) {
                bar_wait(smem_addr(&S.empty[slot]), phase ^ 1, failed);
                if (*failed) break;
                const uint32_t a = base + slot * kBytes, b = a + kTileRows * 128, bar = smem_addr(&S.full[slot]);
                bar_expect(bar, kBytes);
                if constexpr (kDown) {
#pragma unroll
                    for (int x = 0; x < kTileRows; x += 64) load_box3(a + x * 128, &M.a, t.col + x, k * kStep, t.expert, bar);
                } else {
                    load_box3(a, &M.a, k * kStep, t.col, t.expert, bar);
                }
                load_box3(b, &M.b, k * kStep, S.begin[t.expert] + t.row, 0, bar);
                ++issued;
                if (++slot == kStages) {
                    slot = 0;
                    phase ^= 1;
                }
            }
            for (int i = 0, s = slot, p = phase; i < kStages && i < issued; ++i) {
                s = s ? s - 1 : kStages - 1;
                if (s == kStages - 1) p ^= 1;
                bar_wait(smem_addr(&S.empty[s]), p, failed);
            }
            if (*failed)                         // copies in flight end before the block's shared memory goes away
                for (int i = 0; i < kStages && i < issued; ++i) {
                    slot = slot ? slot - 1 : kStages - 1;
                    if (slot == kStages - 1) phase ^= 1;
                    settle(smem_addr(&S.full[slot]), phase);
                }
        }
    } else if (some && warp == kIssueWarp) {
        const uint32_t lead = elect_lane();
        const uint32_t word = product(0, false) | (kDown ? 1u << 15 : 0u) | columns_word((rows + 15) / 16 * 16);
        int slot = 0, phase = 0;
        for (int k = from; k < until; ++k) {
            bar_wait(smem_addr(&S.full[slot]), phase, failed);
            __syncwarp();
            fence_after();
            // within the block's own shared memory: above these bits an address says which block of the cluster is meant
            const uint32_t a = (base & 0x3ffffu) + slot * kBytes, b = a + kTileRows * 128;
            const uint32_t da = kDown ? desc_along_rows(a, kStep * 128) : desc_along_columns(a), db = desc_along_columns(b);
#pragma unroll
            for (int x = 0; x < kStep; x += 16) mma_ss(lead, tmem, da + (kDown ? x * 128 >> 4 : x * 2 >> 4), db + (x * 2 >> 4), word, k > from || x > 0);
            commit(lead, smem_addr(&S.empty[slot]));
            if (++slot == kStages) {
                slot = 0;
                phase ^= 1;
            }
        }
        commit(lead, smem_addr(&S.ready[0]));
        bar_wait(smem_addr(&S.ready[0]), 0, failed);
        if (*failed) settle(smem_addr(&S.ready[0]), 0);
    } else if (some && warp >= kFirstWriter) {
        const int part = warp % 4, first = (warp - kFirstWriter) / 4 * 32;
        if (first < kN) {
            bar_wait(smem_addr(&S.ready[0]), 0, failed);
            __syncwarp();
            fence_after();
            uint32_t r[32];
            load_columns(tmem + first + (static_cast<uint32_t>(part * 32) << 16), r);
            wait_loads();
            pin(r);
            float *const sums = reinterpret_cast<float *>(ring) + part * 32 + lane;              // [row][column]: every product that read the ring is done
#pragma unroll
            for (int i = 0; i < 32; ++i) sums[(first + i) * kTileRows] = __uint_as_float(r[i]);
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    cluster_sync();                              // all blocks' sums are there
    fence_after();
    if (warp == kIssueWarp) tmem_free<kN>(tmem);
    if (some) {
        __nv_bfloat16 *const out = P.out + (S.begin[t.expert] + static_cast<int64_t>(t.row)) * P.out_row + t.col;
        for (int u = rank * kProductThreads + static_cast<int>(threadIdx.x); u < rows * (kTileRows / 8); u += parts * kProductThreads) {
            const int row = u / (kTileRows / 8), c = u % (kTileRows / 8) * 8;
            if (t.col + c >= P.wide) continue;
            float4 lo = make_float4(0.0f, 0.0f, 0.0f, 0.0f), hi = lo;
            for (int b = 0; b < parts; ++b) {
                const uint32_t at = in_block(base + (row * kTileRows + c) * 4, b);
                const float4 x = load_in_block(at), y = load_in_block(at + 16);
                lo = make_float4(lo.x + x.x, lo.y + x.y, lo.z + x.z, lo.w + x.w);
                hi = make_float4(hi.x + y.x, hi.y + y.y, hi.z + y.z, hi.w + y.w);
            }
            *reinterpret_cast<uint4 *>(out + row * P.out_row + c) = make_uint4(pack_bf16(lo.x, lo.y), pack_bf16(lo.z, lo.w), pack_bf16(hi.x, hi.y), pack_bf16(hi.z, hi.w));
        }
    }
    __syncwarp();
    cluster_sync();                              // no block leaves while another reads its sums
    report(S.failed);
}

namespace {

using ProductKernel = void (*)(const ProductParams, const ProductMaps);

// Shared-memory limit of a kernel, set once per device.
bool allow(ProductKernel fn, int which, int bytes) {
    static std::atomic<bool> set[64][14];
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

// [slabs, rows, columns] in boxes of `box_rows` rows by 64 columns.
bool make_map(CUtensorMap &map, void *at, int64_t columns, int64_t rows, int64_t slabs, int64_t row_stride, int64_t slab_stride, int box_rows) {
    const cuuint64_t size[3] = {static_cast<cuuint64_t>(columns), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(slabs)};
    // the stride of a single row or matrix means nothing, but has to be a valid one
    const cuuint64_t strides[2] = {rows > 1 ? static_cast<cuuint64_t>(row_stride) * 2 : 256, slabs > 1 ? static_cast<cuuint64_t>(slab_stride) * 2 : 256};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_rows), 1};
    return encode_map(map, 3, at, size, strides, box);
}

int check_product(const loco_product_t *c, const int32_t *offsets) {
    if (!c) return LOCO_ERR_ARG;
    if (c->experts < 1 || c->experts > kMostExperts || c->rows < 0 || c->rows > 0x7fffffff || c->d_in < 1 || c->d_out < 1) return LOCO_ERR_ARG;
    if (c->d_in % 8 || c->d_out % 8 || c->d_in > kMostColumns || c->d_out > kMostColumns) return LOCO_ERR_UNSUPPORTED;
    if (!offsets) return LOCO_ERR_ARG;
    return aligned(offsets, 4) ? LOCO_OK : LOCO_ERR_ALIGN;
}

// Rows or matrices: present, on 16-byte boundaries, strides of whole 16-byte units below the copies' limit; an output's do not overlap.
constexpr int64_t kMostStride = 1ll << 38;
int check_rows(const loco_rows_t *t, int64_t rows, int64_t dim, bool written) {
    if (!t || !t->ptr) return LOCO_ERR_ARG;
    if (!aligned(t->ptr, 16)) return LOCO_ERR_ALIGN;
    if (rows <= 1) return LOCO_OK;
    if (t->row_stride < 0 || t->row_stride > kMostStride || (written && t->row_stride < dim)) return LOCO_ERR_ARG;
    return t->row_stride % 8 ? LOCO_ERR_ALIGN : LOCO_OK;
}
int check_matrices(const loco_matrices_t *t, int64_t experts, int64_t rows, int64_t columns, bool written) {
    if (!t || !t->ptr) return LOCO_ERR_ARG;
    if (!aligned(t->ptr, 16)) return LOCO_ERR_ALIGN;
    if (rows > 1) {
        if (t->row_stride < 0 || t->row_stride > kMostStride || (written && t->row_stride < columns)) return LOCO_ERR_ARG;
        if (t->row_stride % 8) return LOCO_ERR_ALIGN;
    }
    if (experts > 1) {
        const int64_t span = (rows > 1 ? (rows - 1) * t->row_stride : 0) + columns;
        if (t->expert_stride < 0 || t->expert_stride > kMostStride || (written && t->expert_stride < span)) return LOCO_ERR_ARG;
        if (t->expert_stride % 8) return LOCO_ERR_ALIGN;
    }
    return LOCO_OK;
}

template <bool kWeights, bool kDown, int kN> int launch_product(const ProductParams &P, const ProductMaps &M, int64_t tiles, int which, void *stream) {
    static_assert(product_bytes<kN>() <= 227 * 1024 && stages<kN>() >= 4, "shared memory of a block");
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    if (tiles > 0x7fffffff - sms) return LOCO_ERR_UNSUPPORTED;
    constexpr ProductKernel fn = product_kernel<kWeights, kDown, kN>;
    if (!allow(fn, which, product_bytes<kN>())) return LOCO_ERR_CUDA;
    return launch_kernel(fn, dim3(static_cast<unsigned>(tiles < sms ? tiles : sms)), kProductThreads, product_bytes<kN>(), stream, P, M);
}

template <bool kWeights, bool kDown> int launch_pair(const ProductParams &P, const ProductMaps &M, int64_t tiles, int which, void *stream) {
    const int pairs = sm_count() / 2;
    if (pairs == 0) return LOCO_ERR_CUDA;
    if (tiles > 0x7fffffff - pairs) return LOCO_ERR_UNSUPPORTED;
    constexpr ProductKernel fn = product_pair_kernel<kWeights, kDown>;
    if (!allow(fn, which, kPairBytes)) return LOCO_ERR_CUDA;
    return launch_clusters(fn, dim3(static_cast<unsigned>(2 * (tiles < pairs ? tiles : pairs))), kProductThreads, kPairBytes, stream, 2, P, M);
}

// Clusters of `parts` blocks that run at once, asked for once per device: fewer than the SMs there are would make, since a cluster's lie together.
template <bool kDown, int kN> int clusters_at_once(int parts, int which) {
    static std::atomic<int> known[64][kMostParts + 1];               // one more than the answer
    constexpr ProductKernel fn = product_split_kernel<kDown, kN>;
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return 0;
    }
    if ((n = known[dev][parts].load(std::memory_order_relaxed)) > 0) return n - 1;
    if (!allow(fn, which, product_bytes<kN>())) return 0;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3(static_cast<unsigned>(parts));
    how.blockDim = dim3(kProductThreads);
    how.dynamicSmemBytes = product_bytes<kN>();
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(parts);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    how.attrs = &attr;
    how.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, fn, &how) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
    }
    known[dev][parts].store(n + 1, std::memory_order_relaxed);
    return n;
}
// Blocks to a tile's contraction: as many as leave every tile its cluster at once and a block twelve steps.
template <bool kDown, int kN> int parts_of(int64_t tiles, int64_t steps, int which) {
    for (int parts = kMostParts; parts > 1; --parts)
        if (steps / parts >= 12 && tiles * parts <= sm_count() && tiles <= clusters_at_once<kDown, kN>(parts, which)) return parts;
    return 1;
}

template <bool kDown, int kN> int launch_split(const ProductParams &P, const ProductMaps &M, int64_t tiles, int parts, int which, void *stream) {
    constexpr ProductKernel fn = product_split_kernel<kDown, kN>;
    if (!allow(fn, which, product_bytes<kN>())) return LOCO_ERR_CUDA;
    return launch_clusters(fn, dim3(static_cast<unsigned>(tiles * parts)), kProductThreads, product_bytes<kN>(), stream, parts, P, M);
}

int64_t over(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

// Read by loco_layer_status, which is also built without this file.
int more_status(unsigned *flags, cudaStream_t stream) {
    return cudaMemcpyFromSymbolAsync(flags, g_product_status, sizeof(*flags), 0, cudaMemcpyDeviceToHost, stream) == cudaSuccess ? 0 : 1;
}

}  // namespace loco_layer

using namespace loco_layer;

extern "C" {

int loco_experts_product(const loco_product_t *c, const loco_rows_t *x, const loco_matrices_t *w, const int32_t *d_offsets, const loco_rows_t *y, void *stream) {
    int rc = check_product(c, d_offsets);
    if (rc != LOCO_OK || c->rows == 0) return rc;
    const bool turned = c->transposed != 0;
    const int64_t rows = turned ? c->d_out : c->d_in, columns = turned ? c->d_in : c->d_out;
    if ((rc = check_rows(x, c->rows, c->d_in, false)) != LOCO_OK || (rc = check_rows(y, c->rows, c->d_out, true)) != LOCO_OK ||
        (rc = check_matrices(w, c->experts, rows, columns, false)) != LOCO_OK) return rc;
    ProductParams P{d_offsets, static_cast<__nv_bfloat16 *>(y->ptr), 0, c->rows > 1 ? y->row_stride : 0, c->rows, c->experts, c->d_in, 0, c->d_out, 0};
    ProductMaps M;
    // Tiles by the rows an expert has on average (the counts are on the device; 1500 rows through 64 matrices of 4096 x 2048 take 173 us evenly, with 1200 of them on
    // one expert 221): 32 and 64 for few, which leave the more of shared memory to the matrices on their
    // way (10 and 8 stages), else 256 by pairs of SMs.  64 a pair's against 128 of one SM: 64 rows an expert, 4096 x 14336: 139, 147 us; pairs
    // against 64 for 47 rows an expert, 1032 x 2048: 62, 57 us.  A pair's tile has 256 columns; for 128 and fewer one SM takes 256 rows of
    // them: 55880 rows of 13536 through 120 columns, 128 experts, 452, 315 us, the matrices' gradient 489, 411.
    const int64_t each = c->rows / c->experts, ends = c->rows < c->experts ? c->rows : c->experts;           // every expert may end in a tile of its own
    const bool many = each >= 56, pair = many && c->d_out > kTileRows;
    // Where products bound the call, the tiles with less to do fill the last rounds (16384 rows of 14336 through 4096 columns, eight experts:
    // 1720 us expert by expert, 1635 so); where the matrices' reading does, an expert's tiles stay together (3001 rows, 64 experts: 57, 69).
    P.last = each >= 512;
    // Where tiles of up to 64 rows leave half of the SMs without one, two to eight SMs share each tile's contraction, twelve steps each at
    // least: one token's two experts of 14,336 x 4096 58.6, 39.0 us; 23 rows of 12,568 through 160 columns 48.0, 13.4; 300 rows of 8192 through 120
    // 50.2, 13.9; with eight steps each 100 rows of 1024 through 1024 take 9.5 instead of 8.4.  Clusters that have to wait for others are worse
    // than smaller ones: of eight SMs fifteen run at once, and one row of 14,336 through 1920 columns takes 14.4 us, but through 2048 27.3.
    const int few = each < 24 ? 32 : 64;
    const int64_t small = (c->rows / few + ends) * over(c->d_out, kTileRows), steps = over(c->d_in, kStep);
    const int parts = turned ? (few == 32 ? parts_of<false, 32>(small, steps, 10) : parts_of<false, 64>(small, steps, 11))
                             : (few == 32 ? parts_of<true, 32>(small, steps, 12) : parts_of<true, 64>(small, steps, 13));
    const int high = parts > 1 ? few : pair ? kTileRows : many ? 256 : few;
    const int64_t tiles = pair ? (c->rows / kPairRows + ends) * over(c->d_out, kPairCols) : (c->rows / high + ends) * over(c->d_out, kTileRows);
    if (!make_map(M.a, w->ptr, columns, rows, c->experts, w->row_stride, w->expert_stride, turned ? kTileRows : kStep) ||
        !make_map(M.b, x->ptr, c->d_in, c->rows, 1, x->row_stride, 0, high)) return LOCO_ERR_CUDA;
    const auto go = [&](auto down) {
        constexpr bool kDown = decltype(down)::value;
        constexpr int kFirst = kDown ? 4 : 0;
        if (parts > 1)
            return high == 32 ? launch_split<kDown, 32>(P, M, small, parts, kDown ? 12 : 10, stream) : launch_split<kDown, 64>(P, M, small, parts, kDown ? 13 : 11, stream);
        if (pair) return launch_pair<false, kDown>(P, M, tiles, kFirst, stream);
        if (many) return launch_product<false, kDown, 256>(P, M, tiles, kFirst + 3, stream);
        return high == 32 ? launch_product<false, kDown, 32>(P, M, tiles, kFirst + 1, stream) : launch_product<false, kDown, 64>(P, M, tiles, kFirst + 2, stream);
    };
    return turned ? go(std::false_type{}) : go(std::true_type{});
}

int loco_experts_product_weights(const loco_product_t *c, const loco_rows_t *a, const loco_rows_t *b, const int32_t *d_offsets, const loco_matrices_t *dw,
                                 void *stream) {
    int rc = check_product(c, d_offsets);
    if (rc != LOCO_OK) return rc;
    if ((rc = check_matrices(dw, c->experts, c->d_in, c->d_out, true)) != LOCO_OK) return rc;
    if (c->rows > 0 && ((rc = check_rows(a, c->rows, c->d_in, false)) != LOCO_OK || (rc = check_rows(b, c->rows, c->d_out, false)) != LOCO_OK)) return rc;
    ProductParams P{d_offsets, static_cast<__nv_bfloat16 *>(dw->ptr), c->experts > 1 ? dw->expert_stride : 0, c->d_in > 1 ? dw->row_stride : 0, c->rows, c->experts,
                    0, c->d_in, c->d_out, 0};
    ProductMaps M;
    // without rows nothing is read: the maps need a valid address all the same
    const bool none = c->rows == 0, pair = c->d_in > kTileRows && c->d_out > kTileRows;
    if (!make_map(M.a, none ? dw->ptr : a->ptr, c->d_in, none ? 1 : c->rows, 1, none ? 0 : a->row_stride, 0, kStep) ||
        !make_map(M.b, none ? dw->ptr : b->ptr, c->d_out, none ? 1 : c->rows, 1, none ? 0 : b->row_stride, 0, kStep)) return LOCO_ERR_CUDA;
    if (pair) return launch_pair<true, true>(P, M, c->experts * over(c->d_in, kPairRows) * over(c->d_out, kPairCols), 8, stream);
    return launch_product<true, true, 128>(P, M, c->experts * over(c->d_in, kTileRows) * over(c->d_out, 128), 9, stream);
}

}  // extern "C"
