// A block of the attention kernels whose wait runs out: one thread waits for a barrier that nothing arrives on, with a limit of
// 20 ms.  Nothing is in flight, the kernel returns, and the library's status shows the flag.  Built by the test that runs it.
#include "../paper_2407_04480_b200/csrc/layer_attention.cu"

namespace loco_layer {
std::atomic<uint64_t> g_launches{0};

__global__ void __launch_bounds__(kThreads, 1) wait_that_runs_out(uint64_t *ns, int waits_after) {
    __shared__ Shared S;
    const uint32_t tmem = begin_block<512>(S, 1, 1, kGroupWarps);
    volatile uint32_t *const failed = &S.failed;
    if (threadIdx.x == 0) {
        const uint64_t begin = now_ns();
        bar_wait<20000000ull>(smem_addr(&S.clean), 0, failed);
        const uint64_t first = now_ns();
        for (int i = 0; i < waits_after; ++i) bar_wait(smem_addr(&S.last), 0, failed);
        ns[0] = first - begin;
        ns[1] = now_ns() - first;
        ns[2] = S.failed;
    }
    end_block<512>(S, tmem);
}
}  // namespace loco_layer

// ns (device, three words): the wait that ran out, the waits after it, the block's word.
extern "C" int run_wait(uint64_t *ns, int waits_after, void *stream) {
    loco_layer::wait_that_runs_out<<<1, loco_layer::kThreads, 0, static_cast<cudaStream_t>(stream)>>>(ns, waits_after);
    return cudaGetLastError() == cudaSuccess ? 0 : 1;
}
