// One warp runs one softmax step of the prefix kernel on given scores and accumulators.  The barrier for which the second half
// waits has completed, or (ready 0) nothing ever completes it.
#include "../paper_2609_00097_b200/csrc/ffd_prefix_step.cuh"

namespace {

using namespace ffd;

// scores, o_in, o_out: [32][128]; ml_out: [32][2]; arrived: [2], whether each half's weights were announced
template <int PIECES>
__global__ void __launch_bounds__(32) step_kernel(const float* scores, const float* o_in, float m, float l, int ready, float* o_out,
                                                  float* ml_out, int* arrived) {
    __shared__ __align__(8) uint64_t bars[3];
    __shared__ uint32_t tmem_base;
    const int lane = threadIdx.x;
    const uint32_t halves = smem_u32(bars), probs = halves + 8;
    if (lane == 0) {
        for (int i = 0; i < 3; ++i) mbar_init(halves + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t s_col = __shfl_sync(kFull, tmem_base, 0), o_col = s_col + 256;
    for (int c = 0; c < 128; c += 16) {
        uint32_t x[16], y[16];
        for (int i = 0; i < 16; ++i) {
            x[i] = __float_as_uint(scores[128 * lane + c + i]);
            y[i] = __float_as_uint(o_in[128 * lane + c + i]);
        }
        tmem_st16(s_col + c, x);
        tmem_st16(o_col + c, y);
    }
    tmem_wait_st();
    if (ready && lane == 0) mbar_arrive(halves);
    __syncwarp();
    const float2 ml = softmax_step<PIECES>(s_col, o_col, m, l, 1.f, 64, 64, true, probs, halves, 0u);
    __syncwarp();
    for (int c = 0; c < 128; c += 16) {
        float y[16];
        tmem_ld16(o_col + c, y);
        tmem_wait_ld();
        for (int i = 0; i < 16; ++i) o_out[128 * lane + c + i] = y[i];
    }
    ml_out[2 * lane] = ml.x;
    ml_out[2 * lane + 1] = ml.y;
    if (lane < 2) arrived[lane] = mbar_try(probs + 8 * lane, 0);
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(s_col) : "memory");
}

}  // namespace

extern "C" int run_step(int pieces, const float* scores, const float* o_in, float m, float l, int ready, float* o_out, float* ml_out,
                        int* arrived) {
    (pieces == 1 ? step_kernel<1> : step_kernel<2>)<<<1, 32>>>(scores, o_in, m, l, ready, o_out, ml_out, arrived);
    const cudaError_t launched = cudaGetLastError();
    return (int)(launched != cudaSuccess ? launched : cudaDeviceSynchronize());
}
