// A softmax step of the prefix kernel, and what it needs of tensor memory and barriers.
#pragma once
#include <math.h>
#include <stdint.h>

#include "ffd_paged.cuh"

namespace ffd {

// ---- tensor memory and barriers --------------------------------------------------------------------------------------------

__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float* x) {
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float* x) {
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st2(uint32_t addr, float a, float b) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};\n" ::"r"(addr), "r"(__float_as_uint(a)), "r"(__float_as_uint(b)) : "memory");
}
__device__ __forceinline__ void tmem_ld2(uint32_t addr, float* x) {
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];\n" : "=r"(r[0]), "=r"(r[1]) : "r"(addr));
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}

// ---- the step --------------------------------------------------------------------------------------------------------------

// a x b + c and a + b on two numbers at once
__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void pair_split(unsigned long long r, float& a, float& b) {
    asm("mov.b64 {%0, %1}, %2;\n" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ unsigned long long pair_fma(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long pair_add(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The weights of 64 scores s against the reference -shift, in bf16 pieces, and their sum and the scores' maximum
template <int PIECES>
__device__ __forceinline__ void weights_of(const float (&s)[64], float scale, float shift, uint32_t (&hi)[32],
                                           uint32_t (&lo)[PIECES == 2 ? 32 : 1], float& sum, float& top) {
    const unsigned long long scale2 = pair_of(scale, scale), shift2 = pair_of(shift, shift);
    unsigned long long sums[2] = {0ull, 0ull};
    float tops[2] = {s[0], s[1]};
#pragma unroll
    for (int x = 0; x < 32; ++x) {
        float a, b;
        pair_split(pair_fma(pair_of(s[2 * x], s[2 * x + 1]), scale2, shift2), a, b);
        const float p0 = fast_ex2(a), p1 = fast_ex2(b);
        tops[x & 1] = max3(tops[x & 1], s[2 * x], s[2 * x + 1]);
        sums[x & 1] = pair_add(sums[x & 1], pair_of(p0, p1));
        hi[x] = pack_bf16(p0, p1);
        if (PIECES == 2) lo[x] = pack_bf16(p0 - __uint_as_float(hi[x] << 16), p1 - __uint_as_float(hi[x] & 0xffff0000u));
    }
    float a, b;
    pair_split(pair_add(sums[0], sums[1]), a, b);
    sum = a + b;
    top = fmaxf(tops[0], tops[1]);
}

// A step of one softmax warpgroup: the weights of 128 tokens over their scores in TMEM, in two halves, of which the first is
// announced (probs) while the second is computed.  A thread has a row; (m, l) is its reference (log2) and sum, and the new ones
// are returned.  keep0, keep1: tokens of each half that have logits (keep0 below 0: a pass that works on whatever TMEM holds and
// changes nothing).  rescale: O holds earlier steps' products, which are complete; halves: completes with the first half's.
// Weights are computed against the reference as it stands, while the maximum is found; if a row exceeds the reference by 2^8
// (as its first tokens do), the reference is raised, O rescaled, and the half is computed again.  The second half's rescaling
// waits for the first half's product.  If that wait runs out, the whole warp gets NaN for m, which no logits make of it.
// Not inlined: this is the kernel's longest code, and it has to be fetched line by line when it first runs.  In the middle of
// the first loads that took 5 us; a pass ahead of them fetches it while nothing else is going on.
template <int PIECES>
__device__ __noinline__ float2 softmax_step(uint32_t s_col, uint32_t o_col, float m, float l, float scale, int keep0, int keep1,
                                            bool rescale, uint32_t probs, uint32_t halves, uint32_t parity) {
    constexpr bool kAhead = PIECES == 1;   // the second half's scores on their way while the first is computed, if registers allow
    const bool live = keep0 >= 0;
    float s[2][64];
    tmem_ld32(s_col, s[0]);
    tmem_ld32(s_col + 32, s[0] + 32);
    tmem_wait_ld();
    if (kAhead) {
        tmem_ld32(s_col + 64, s[1]);
        tmem_ld32(s_col + 96, s[1] + 32);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int keep = half ? keep1 : keep0;
        uint32_t hi[32], lo[PIECES == 2 ? 32 : 1];
        float sum, top;
        if (half && !kAhead) {
            tmem_ld32(s_col + 64, s[1]);
            tmem_ld32(s_col + 96, s[1] + 32);
        }
        if (half) tmem_wait_ld();
        for (;;) {
            if (live && keep < 64) {
#pragma unroll
                for (int x = 0; x < 64; ++x)
                    if (x >= keep) s[half][x] = -INFINITY;
            }
            weights_of<PIECES>(s[half], scale, m == -INFINITY ? 0.f : -m, hi, lo, sum, top);
            top *= scale;
            if (!__any_sync(kFull, top > m + 8.f) || !live) break;
            const float raised = fmaxf(m, top);
            const float alpha = raised == -INFINITY ? 1.f : fast_ex2(m - raised);
            m = raised;
            l *= alpha;
            if (rescale || half) {
                if (half) {
                    bool done = mbar_try(halves, parity);
                    for (const long long t0 = clock64(); !done && clock64() - t0 < kSpinCycles;) done = mbar_try(halves, parity);
                    // run out: the product may still be adding to O, so O is left alone and no weights are announced
                    if (!__all_sync(kFull, done)) return make_float2(NAN, l);
                    tmem_after_sync();
                }
#pragma unroll 1
                for (int c = 0; c < 8; ++c) {
                    float o[16];
                    tmem_ld16(o_col + 16 * c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[x] *= alpha;
                    tmem_st16(o_col + 16 * c, reinterpret_cast<const uint32_t*>(o));
                }
            }
            tmem_ld32(s_col + 64 * half, s[half]);
            tmem_ld32(s_col + 64 * half + 32, s[half] + 32);
            tmem_wait_ld();
        }
        l += sum;
        if (live) {
            tmem_st32(s_col + 64 * half, hi);      // over the half's own scores
            if (PIECES == 2) tmem_st32(s_col + 64 * half + 32, lo);
            tmem_wait_st();
            tmem_before_sync();
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbar_arrive(probs + 8 * half);
        }
    }
    return make_float2(m, l);
}

}  // namespace ffd
