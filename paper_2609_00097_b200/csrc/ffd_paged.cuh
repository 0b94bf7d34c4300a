// What the kernels of the byte cache and of the shared prefix have in common: the formats, the parameters of an attention
// call, and the partition of ragged work over a fixed grid.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "ffd_kernels.cuh"

namespace ffd {

constexpr int kFmtInt8 = 0, kFmtE4m3 = 1, kFmtBf16 = 2;   // the first two are FFD_BYTE_INT8 and FFD_BYTE_E4M3
constexpr int kMaxGroup = 8;                              // query heads per KV head in the kernels of this header

// One attention call over the sequences' own pages, with the partial results of a shared prefix if there is one.
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
    // weights; -inf marks an empty one, whose channels are not used.
    float* part_out;               // own tokens: [units + parts][G][128], see paged_slot
    float* part_lse;               // [units + parts][G]
    long long* offsets;            // [batch + 1] items of the sequences before each, per KV head: attention -> merge
    struct Shares* shares;         // their partition: attention -> merge
    const float* prefix_out;       // prefix: [Hkv][prefix_stride][batch * G][128], the first Shares::chunks of each head
    const float* prefix_lse;       // [Hkv][prefix_stride][batch * G]
    int prefix_stride;
    void* out;                     // [batch, Hq, 128] bf16 or fp32
    float* lse;                    // nullable
    int out_fp32;
};

__device__ __forceinline__ float fast_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}

// a / b and a % b; the 64-bit division, ten times as long, only where 32 bits are not enough
__device__ __forceinline__ long long quick_div(long long a, int b) {
    return (unsigned long long)a >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}

// The flattened list of a call's items (runs of 16 or 32 tokens of one sequence and KV head; a sequence's last may be
// shorter), ordered by sequence, then head, then token, is cut into `parts` shares that differ by at most one item, whatever
// the lengths: the first `more` have each + 1 items, the others `each`.  All parts of the launch take one, but none gets fewer
// than about 32 tokens, so that short calls are not all merging.  The part of a unit (sequence, KV head) that falls into part
// c is stored in slot unit + c: along the list each new segment raises the unit or the part by at least one, so no two
// segments share a slot, and `units + parts` slots are enough.
struct Shares {
    long long each;
    int parts, more;
    int chunks;   // partial results of the prefix per row

    __device__ __forceinline__ static Shares of(long long items, int most, int min_shift, int prefix_chunks) {
        Shares s;
        s.chunks = prefix_chunks;
        s.parts = (int)min((long long)most, (items + (1 << min_shift) - 1) >> min_shift);
        s.each = s.parts ? quick_div(items, s.parts) : 0;
        s.more = (int)(items - s.each * s.parts);
        return s;
    }
    __device__ __forceinline__ long long begin(int part) const { return part * each + min(part, more); }
    __device__ __forceinline__ int part_of(long long item) const {
        const long long first = more * (each + 1);   // items of the larger shares
        return item < first ? (int)quick_div(item, (int)each + 1) : more + (int)quick_div(item - first, (int)each);
    }
};
__device__ __forceinline__ long long paged_slot(int unit, int part) { return (long long)unit + part; }

__device__ __forceinline__ int paged_len(const int32_t* seq_lens, int b, int max_blocks, uint32_t* status) {
    const int n = seq_lens[b], cap = max_blocks * kBlk;
    if (n < 0 || n > cap) {
        atomicOr(status, kDevBadSeqLen);
        return n < 0 ? 0 : cap;
    }
    return n;
}

__device__ __forceinline__ int ceil_shift(int n, int shift) { return (n >> shift) + ((n & ((1 << shift) - 1)) != 0); }
__device__ __forceinline__ int blocks_of(int n) { return ceil_shift(n, 6); }

// Prefix sums of count(b) over the sequences, by every warp for itself (by all threads together, with barriers, a call on one 4 K
// sequence took 0.7 us longer): lane x sums the x-th of 32 runs of sequences, and a scan places the runs.
template <typename Count>
struct WarpScan {
    int lo, hi;
    long long before, sum, total;
    Count count;

    __device__ __forceinline__ WarpScan(int batch, Count c, int lane) : count(c) {
        const int run = (batch + 31) >> 5;
        lo = min(batch, lane * run);
        hi = min(batch, lo + run);
        sum = 0;
        for (int b = lo; b < hi; ++b) sum += count(b);
        long long scan = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(kFull, scan, o);
            if (lane >= o) scan += x;
        }
        before = scan - sum;
        total = __shfl_sync(kFull, scan, 31);
    }
    // the sequence whose items (heads * count) hold item x, 0 <= x < total * heads, and the items before it
    __device__ __forceinline__ void find(long long x, int heads, int& b, long long& off) const {
        off = before * heads;
        b = lo;
        const bool here = x >= off && x < off + sum * heads;
        if (here && hi - lo > 1)
            for (long long c; x >= off + (c = (long long)count(b) * heads); ++b) off += c;
        const int from = __ffs(__ballot_sync(kFull, here)) - 1;
        b = __shfl_sync(kFull, b, from);
        off = __shfl_sync(kFull, off, from);
    }
};

// The last sequence whose rows start at or before `row`, by a search in which the 32 lanes probe at once: two rounds for
// up to 1024 sequences.  -1: none.
__device__ __forceinline__ int sequence_of_row(const int32_t* row_start, int batch, int row, int lane) {
    int lo = -1, hi = batch;   // row_start[lo] <= row (lo >= 0), row_start[hi] > row (hi < batch)
    while (hi - lo > 1) {
        const int step = (hi - lo - 1 + 31) / 32;
        const int at = lo + 1 + lane * step;
        const bool below = at < hi && row_start[at] <= row;
        const int below_count = __popc(__ballot_sync(kFull, below));
        if (below_count == 0) {
            hi = lo + 1;
        } else {
            lo += 1 + (below_count - 1) * step;
            hi = min(hi, lo + step);
        }
    }
    return lo;
}

}  // namespace ffd
