// The addresses that the copies of a gradient's chunks name, found on the host: built and called by a test that needs no GPU.
#include "../paper_2407_04480_b200/csrc/layer_gradient.cu"

namespace loco_layer {
std::atomic<uint64_t> g_launches{0};
int sm_count() { return 0; }

// Whether every thread of every chunk of n elements at x names a boundary: of a vector that lies within the span where it reads one,
// else one whose 16 bytes hold the span's first element.  `read` counts the elements of the vectors, `rest` those of the ends.
template <typename T> int check(uintptr_t x, uint64_t n, uint64_t *read, uint64_t *rest) {
    const uint32_t chunks = static_cast<uint32_t>((n * sizeof(T) + kChunkBytes - 1) / kChunkBytes);
    const uintptr_t end = x + n * sizeof(T);
    *read = *rest = 0;
    for (uint32_t chunk = 0; chunk < chunks; ++chunk) {
        const Piece<T> p(reinterpret_cast<const void *>(x), n, chunk, chunks);
        for (int i = 0; i < kAtOnce * kListThreads; ++i) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p.vector(reinterpret_cast<const void *>(x), i));
            if (at % 16 != 0) return 1;
            if (i < p.count ? at < x || at + 16 > end : at > x || at + 16 <= x) return 2;
        }
        *read += static_cast<uint64_t>(p.count) * Piece<T>::kV;
        *rest += p.head + p.tail;
    }
    return 0;
}
}  // namespace loco_layer

extern "C" int check_addresses(int32_t dtype, uintptr_t x, uint64_t n, uint64_t *read, uint64_t *rest) {
    return dtype == LOCO_BF16 ? loco_layer::check<__nv_bfloat16>(x, n, read, rest) : loco_layer::check<float>(x, n, read, rest);
}
