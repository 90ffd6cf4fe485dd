// Waits of stom_async.cuh on a barrier that nothing arrives at: a wait with a limit, one that another warp calls off, one
// that has been called off already, and one whose barrier is arrived at.  out: per wait 1 or 0 and what it took in ns (of the
// second: from the call-off on).
#include "stom_async.cuh"

using namespace stom;

__global__ void waits(unsigned long long limit_ns, unsigned long long off_after_ns, unsigned long long *out) {
    __shared__ uint64_t never, once;
    __shared__ uint32_t abort_word;
    __shared__ unsigned long long off_at;
    volatile uint32_t *abort_flag = &abort_word;
    const bool first = threadIdx.x == 0, other = threadIdx.x == 32;
    if (first) {
        mbar_init(smem_u32(&never), 1);
        mbar_init(smem_u32(&once), 1);
        abort_word = 0;
        mbar_init_fence();
    }
    __syncthreads();
    unsigned long long t = global_ns();
    if (first) {
        out[0] = mbar_wait_bounded(smem_u32(&never), 0, abort_flag, limit_ns);
        out[1] = global_ns() - t;
    }
    __syncthreads();
    t = global_ns();
    if (other) {
        while (global_ns() - t < off_after_ns) {}
        off_at = global_ns();
        *abort_flag = 1;
    }
    if (first) {
        out[2] = mbar_wait_bounded(smem_u32(&never), 0, abort_flag, 100 * off_after_ns);
        t = global_ns();
    }
    __syncthreads();
    if (first) {
        out[3] = t - off_at;
        t = global_ns();
        out[4] = mbar_wait_bounded(smem_u32(&never), 0, abort_flag, limit_ns);
        out[5] = global_ns() - t;
        mbar_arrive(smem_u32(&once));
        t = global_ns();
        out[6] = mbar_wait_bounded(smem_u32(&once), 0, abort_flag, limit_ns);
        out[7] = global_ns() - t;
    }
}

extern "C" int run_waits(unsigned long long limit_ns, unsigned long long off_after_ns, unsigned long long *host) {
    unsigned long long *dev = nullptr;
    cudaError_t e = cudaMalloc(&dev, 8 * sizeof(*dev));
    if (e == cudaSuccess) waits<<<1, 64>>>(limit_ns, off_after_ns, dev);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) e = cudaMemcpy(host, dev, 8 * sizeof(*dev), cudaMemcpyDeviceToHost);
    cudaFree(dev);
    return (int)e;
}
