// A block of the product kernels whose wait runs out: one thread waits for a barrier that nothing arrives on, with a limit of 20 ms.
// Nothing is in flight, the kernel returns and raises the product kernels' flag, which the library's status has to show beside the
// attention kernels'.  Built, together with attention_wait.cu, by the test that runs it.
#include "../paper_2407_04480_b200/csrc/layer_product.cu"

namespace loco_layer {
int sm_count() { return 0; }

__global__ void __launch_bounds__(kProductThreads, 1) product_wait_that_runs_out(uint64_t *ns, int waits_after) {
    __shared__ uint64_t never;
    __shared__ uint32_t word;
    volatile uint32_t *const failed = &word;
    if (threadIdx.x == 0) {
        bar_init(smem_addr(&never), 1);
        word = 0;
        fence_bar_init();
        const uint64_t begin = now_ns();
        bar_wait<20000000ull>(smem_addr(&never), 0, failed);
        const uint64_t first = now_ns();
        for (int i = 0; i < waits_after; ++i) bar_wait(smem_addr(&never), 0, failed);
        ns[0] = first - begin;
        ns[1] = now_ns() - first;
        ns[2] = word;
    }
    __syncthreads();
    report(word);
}
}  // namespace loco_layer

// ns (device, three words): the wait that ran out, the waits after it, the block's word.
extern "C" int run_product_wait(uint64_t *ns, int waits_after, void *stream) {
    loco_layer::product_wait_that_runs_out<<<1, loco_layer::kProductThreads, 0, static_cast<cudaStream_t>(stream)>>>(ns, waits_after);
    return cudaGetLastError() == cudaSuccess ? 0 : 1;
}
