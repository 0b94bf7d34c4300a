// What the kernels of the byte cache and of the shared prefix have in common: the formats, the parameters of an attention
// call, and the partition of ragged work over a fixed grid.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "ffd_kernels.cuh"

namespace ffd {

constexpr int kFmtInt8 = 0, kFmtE4m3 = 1, kFmtBf16 = 2;   // the first two are FFD_BYTE_INT8 and FFD_BYTE_E4M3
constexpr int kMaxGroup = 8;                              // query heads per KV head in the kernels of this header

// One attention call over the sequences' own pages, with the partial results of a shared prefix (prefix_splits > 0).
struct PagedParams {
    const __nv_bfloat16* q;        // [batch, Hq, 128]
    const unsigned char* k;        // [num_pages, Hkv, 64, 128] codes or bf16
    const unsigned char* v;
    const float* k_scale;          // [num_pages, Hkv, 64]; byte formats only
    const float* v_scale;
    const int32_t* block_table;    // [batch, max_blocks]; null: page b * max_blocks + blk
    const int32_t* seq_lens;
    int batch, Hq, Hkv, G, max_blocks, num_pages;
    float logit_scale;             // sm_scale * log2(e)
    uint32_t* status;
    // partial results.  A partial is the normalised attention over some of a unit's tokens and the log2 of its sum of
    // weights; -inf marks an empty one, whose channels are not read.
    float* part_out;               // own tokens: [units + parts][G][128], see paged_slot
    float* part_lse;               // [units + parts][G]
    int parts;                     // CTAs that share the own tokens
    const float* prefix_out;       // prefix: [Hkv][prefix_splits][batch * G][128]
    const float* prefix_lse;       // [Hkv][prefix_splits][batch * G]
    int prefix_splits;             // 0: no prefix
    void* out;                     // [batch, Hq, 128] bf16 or fp32
    float* lse;                    // nullable
    int out_fp32;
};

// The flattened list of a call's (sequence, KV head, block) items, ordered by sequence, then head, then block, is cut into
// P = min(parts, T) shares that differ by at most one item, whatever the lengths: part i takes items [i T / P, (i + 1) T / P),
// and no part in between is empty.
// The part of a unit (sequence, KV head) that falls into part c is stored in slot unit + c: along the list each new segment
// raises the unit or the part by at least one, so no two segments share a slot and `units + parts` slots are enough.
__device__ __forceinline__ long long paged_slot(int unit, int part) { return (long long)unit + part; }

struct Share {
    long long begin, end;   // items of this part
    long long off;          // first item of sequence b
    int b;                  // sequence of item `begin` (when begin < end)
};

__device__ __forceinline__ int paged_len(const int32_t* seq_lens, int b, int max_blocks, uint32_t* status) {
    const int n = seq_lens[b], cap = max_blocks * kBlk;
    if (n < 0 || n > cap) {
        atomicOr(status, kDevBadSeqLen);
        return n < 0 ? 0 : cap;
    }
    return n;
}

__device__ __forceinline__ int blocks_of(int n) { return (n >> 6) + ((n & 63) != 0); }

// Share `part` of `parts` over sequences with count(b) * heads items each.  Every thread of the CTA calls it (THREADS of
// them) and gets the same answer.  A thread sums a run of consecutive sequences, a scan places the runs, and the thread
// whose run holds the share's first item walks it: one pass over the lengths.
template <int THREADS, typename Count>
__device__ __forceinline__ Share find_share(int batch, int heads, int part, int parts, Count count) {
    __shared__ long long warp_sum[THREADS / 32];
    __shared__ long long found_off;
    __shared__ int found_b;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int run = (batch + THREADS - 1) / THREADS;
    const int lo = min(batch, tid * run), hi = min(batch, lo + run);
    long long sum = 0;
    for (int b = lo; b < hi; ++b) sum += count(b);
    long long scan = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(kFull, scan, o);
        if (lane >= o) scan += x;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    long long before = scan - sum, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += warp_sum[w];
        total += warp_sum[w];
    }
    Share s;
    total *= heads;
    const long long p = min((long long)parts, total);
    s.begin = s.end = 0;
    if (part < p) {
        s.begin = total * part / p;
        s.end = total * (part + 1) / p;
    }
    long long off = before * heads;
    if (s.begin < s.end && off <= s.begin && s.begin < off + sum * heads) {
        int b = lo;
        for (long long c; s.begin >= off + (c = (long long)count(b) * heads); ++b) off += c;
        found_b = b;
        found_off = off;
    }
    __syncthreads();
    s.b = found_b;
    s.off = found_off;
    return s;
}

// part that holds item x of `total`: the largest i with i * total / P <= x
__device__ __forceinline__ int part_of(long long x, long long total, int parts) {
    return (int)(((x + 1) * min((long long)parts, total) - 1) / total);
}

}  // namespace ffd
