// Thin wrappers over the sm_100a instructions of the attention and product kernels: mbarriers, tensor copies, tensor-core products
// with their accumulators in tensor memory, and small arithmetic that the other kernels use too.  Every wait is bounded.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cstring>

#include "layer_common.h"

namespace loco_layer {
namespace tc {

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// ---- mbarriers -------------------------------------------------------------------------------

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

constexpr uint64_t kWaitLimitNs = 2000000000ull;      // a wait longer than this gives up

// Waits for the phase.  Past the limit it raises `failed` and returns; from then on every wait of the block returns after one
// look at its barrier (0.14 us, measured), so that all roles walk to their ends (on meaningless values) in about the time
// that the block would have taken anyway.  Leaving their loops instead takes a vote of the warp a tile: 5 to 20% slower.
template <uint64_t kLimitNs = kWaitLimitNs> __device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *failed) {
    if (bar_test(bar, parity) || *failed) return;
    const uint64_t begin = now_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (bar_test(bar, parity)) return;
        if (*failed) return;
        if (now_ns() - begin > kLimitNs) {
            *failed = 1;
            return;
        }
    }
}

// Order generic writes to shared memory before reads of the tensor core and the copy engine.
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_bar_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

// ---- tensor copies ---------------------------------------------------------------------------

// A box of `map` at (x, row, head, batch) to shared memory; completes on `bar`.
__device__ __forceinline__ void load_box(uint32_t to, const CUtensorMap *map, int x, int row, int head, int batch, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(to), "l"(map), "r"(x), "r"(row), "r"(head), "r"(batch), "r"(bar) : "memory");
}

// ---- tensor memory ---------------------------------------------------------------------------

template <int kColumns> __device__ __forceinline__ void tmem_alloc(uint32_t to) {       // one warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int kColumns> __device__ __forceinline__ void tmem_free(uint32_t at) {         // the same warp
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(kColumns) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the thread's lane.  The values may be used only after wait_load() on them.
__device__ __forceinline__ void load_columns(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void load_columns(uint32_t at, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Ties the values to the wait before it: nothing that uses them is moved above.
template <int kN> __device__ __forceinline__ void pin(uint32_t (&r)[kN]) {
#pragma unroll
    for (int i = 0; i < kN; i += 8)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
__device__ __forceinline__ void store_columns(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
                 "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
                   "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
                   "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void store_columns(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void store_columns(uint32_t at, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- products --------------------------------------------------------------------------------

// Operand tiles are [columns / 64][rows][64] bfloat16 with the copy engine's 128-byte swizzle: rows of 128 bytes, groups of
// 8 rows of 1024.  Descriptor fields in 16-byte units: address 0-13, leading offset 16-29, stride 32-45, version 1 at 46,
// swizzle 128 B = 2 at 61.  Only the low word depends on the tile.
constexpr uint32_t kDescHigh = (1024 >> 4) | (1u << 14) | (2u << 29);
// contraction along the columns: 8-row groups 1024 bytes apart
__device__ __forceinline__ uint32_t desc_along_columns(uint32_t addr) { return (1u << 16) | (addr >> 4); }
// contraction along the rows: 8-row groups 1024 bytes apart, 64-column blocks `block` bytes apart
__device__ __forceinline__ uint32_t desc_along_rows(uint32_t addr, uint32_t block) { return ((block >> 4) << 16) | (addr >> 4); }

// Instruction word: fp32 accumulators, bfloat16 operands, 128 x n.
__host__ __device__ constexpr uint32_t product(int n, bool b_along_rows, bool negate = false) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (negate ? 1u << 13 : 0u) | (b_along_rows ? 1u << 16 : 0u) |
           (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}

// One lane of the warp.  The products' operands live in uniform registers: the whole warp runs the issuing code and the
// instruction itself is predicated, since in code that only one lane runs every operand would have to be moved there first.
__device__ __forceinline__ uint32_t elect_lane() {
    uint32_t r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
    return r;
}

// One 128 x n x 16 step, by the elected lane; both operands in shared memory, or A in tensor memory.
__device__ __forceinline__ void mma_ss(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t word, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n mov.b64 a, {%1, %6};\n mov.b64 b, {%2, %6};\n setp.ne.u32 p, %4, 0;\n setp.ne.u32 q, %5, 0;\n"
                 " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "r"(b), "r"(word), "r"(accumulate), "r"(lead), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t word, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p, q;\n .reg .b64 b;\n mov.b64 b, {%2, %6};\n setp.ne.u32 p, %4, 0;\n setp.ne.u32 q, %5, 0;\n"
                 " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "r"(b), "r"(word), "r"(accumulate), "r"(lead), "r"(kDescHigh) : "memory");
}
// Arrives on the barrier when every product the elected lane has issued is complete.
__device__ __forceinline__ void commit(uint32_t lead, uint32_t bar) {
    asm volatile("{\n .reg .pred q;\n setp.ne.u32 q, %1, 0;\n @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n"
                 ::"r"(bar), "r"(lead) : "memory");
}

// ---- small arithmetic ------------------------------------------------------------------------

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Two fp32 operations at a time.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// Elements 2q and 2q + 1 of a vector in fp32 (a vector of one: the element and 0), and back, rounded.  bfloat16 in pairs: a shift
// and a mask one way, one conversion the other.
template <typename T, int V> __device__ __forceinline__ float2 pair_of(const Pack<T, V> &p, int q) {
    if constexpr (V == 1) {
        return make_float2(to_f32(p.v[0]), 0.0f);
    } else if constexpr (sizeof(T) == 2) {
        uint32_t w;
        memcpy(&w, &p.v[2 * q], 4);
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    } else {
        return make_float2(to_f32(p.v[2 * q]), to_f32(p.v[2 * q + 1]));
    }
}
template <typename T, int V> __device__ __forceinline__ void set_pair(Pack<T, V> &p, int q, float2 f) {
    if constexpr (V == 1) {
        p.v[0] = from_f32<T>(f.x);
    } else if constexpr (sizeof(T) == 2) {
        const uint32_t w = pack_bf16(f.x, f.y);
        memcpy(&p.v[2 * q], &w, 4);
    } else {
        p.v[2 * q] = from_f32<T>(f.x);
        p.v[2 * q + 1] = from_f32<T>(f.y);
    }
}
// Largest of three or two, NaN if one is.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max2(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// 2^x without the special-function unit, whose 16 results a clock bound the softmax: x = n + f with |f| <= 1/2, 2^f by the
// polynomial of degree 4 with the least largest relative error there (2.7e-6; fitted by weighted least squares), times 2^n
// put together as its bits.  Below -127 and at -infinity the answer is 0 (as n + 127 is), for NaN it is NaN; x above 127 is
// not for this function.
__device__ __forceinline__ float2 exp2_poly(float2 x) {
    constexpr float kRound = 12582912.0f;          // 1.5 * 2^23: adding it leaves the nearest integer in the low bits
    x.x = max2(x.x, -127.0f);
    x.y = max2(x.y, -127.0f);
    const float2 t = add2(x, make_float2(kRound, kRound));
    const float2 f = fma2(add2(t, make_float2(-kRound, -kRound)), make_float2(-1.0f, -1.0f), x);
    float2 p = fma2(f, make_float2(0.00957007986f, 0.00957007986f), make_float2(0.0559178367f, 0.0559178367f));
    p = fma2(p, f, make_float2(0.240247443f, 0.240247443f));
    p = fma2(p, f, make_float2(0.693121791f, 0.693121791f));
    p = fma2(p, f, make_float2(0.999999285f, 0.999999285f));
    const auto power = [](float t) { return __uint_as_float((__float_as_uint(t) << 23) + 0x3f800000u); };
    return mul2(p, make_float2(power(t.x), power(t.y)));
}

}  // namespace tc
}  // namespace loco_layer
