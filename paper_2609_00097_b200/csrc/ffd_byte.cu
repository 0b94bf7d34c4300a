// The byte cache: K and V with one byte per element (int8 or e4m3) and one binary32 scale for each token and KV head.
// Kernels that write it, read it back into 16-bit pages and attend to it, and the merge of partial attention results.
#include <cuda_runtime.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "../../include/ffd.h"
#include "ffd_host.cuh"
#include "ffd_own.cuh"
#include "ffd_prefix.cuh"

namespace ffd {

// ---- writing ------------------------------------------------------------------------------------------------------

// below this a row is stored as zeros: L / absmax would leave binary32
constexpr float kTinyRow = 7.888609052210118e-31f;   // 2^-100

struct WriteParams {
    const __nv_bfloat16* k_new;   // [num_rows][Hkv][128], rows row_stride elements apart
    const __nv_bfloat16* v_new;
    long long row_stride;
    const int32_t* row_start;     // [batch], null: row b is the last token of sequence b
    const int32_t* first_token;
    const int32_t* seq_lens;
    const int32_t* block_table;
    unsigned char* k;
    unsigned char* v;
    float* k_scale;
    float* v_scale;
    uint32_t* status;
    int num_rows, batch, Hkv, max_blocks, num_pages;
};

// largest magnitude of eight bf16 numbers, as a 16-bit integer (the order of bf16 magnitudes)
__device__ __forceinline__ uint32_t top_of(const uint4& x) {
    const uint32_t m = __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16);
}

// NaN becomes 0 and an infinity the largest finite bf16, so that one bad element cannot spoil its row's neighbours
__device__ __forceinline__ uint32_t finite_pair(uint32_t x) {
    uint32_t r = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t e = x >> (16 * h) & 0xffffu, mag = e & 0x7fffu;
        r |= (mag > 0x7f80u ? 0u : mag == 0x7f80u ? (e & 0x8000u) | 0x7f7fu : e) << (16 * h);
    }
    return r;
}

template <int FMT>
__device__ __forceinline__ uint2 codes_of(const uint4& x, float inv) {
    const float2 a = bf16x2_to_float2(x.x), b = bf16x2_to_float2(x.y), c = bf16x2_to_float2(x.z), d = bf16x2_to_float2(x.w);
    return make_uint2(floats_to_codes<FMT>(__fmul_rn(a.x, inv), __fmul_rn(a.y, inv), __fmul_rn(b.x, inv), __fmul_rn(b.y, inv)),
                      floats_to_codes<FMT>(__fmul_rn(c.x, inv), __fmul_rn(c.y, inv), __fmul_rn(d.x, inv), __fmul_rn(d.y, inv)));
}

// N head pairs of a row: lane 16 y + s has elements 8 s .. 8 s + 7 of heads head0 + 2 i + y, K and V.  Rows go to `at` =
// page * Hkv * 64 + row of the page.  The arithmetic costs as much as the memory traffic if it is not shared out: K's and V's
// maxima travel in one register, and of the 4 N quotients of a head (L / absmax and absmax / L, IEEE divisions of twenty
// instructions) every lane computes one.
template <int FMT, int N>   // N: 1 or 4
__device__ __forceinline__ void store_heads(const WriteParams& p, long long at, int head0, int lane, uint4 (&k)[N], uint4 (&v)[N]) {
    const int s = lane & 15, y = lane >> 4;
    uint32_t top[N];   // K's in the upper half
#pragma unroll
    for (int i = 0; i < N; ++i) top[i] = top_of(k[i]) << 16 | top_of(v[i]);
    uint32_t high = top[0];
#pragma unroll
    for (int i = 1; i < N; ++i) high = __vmaxu2(high, top[i]);
    if (__any_sync(kFull, high >= 0x7f800000u || (high & 0xffffu) >= 0x7f80u)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            k[i] = make_uint4(finite_pair(k[i].x), finite_pair(k[i].y), finite_pair(k[i].z), finite_pair(k[i].w));
            v[i] = make_uint4(finite_pair(v[i].x), finite_pair(v[i].y), finite_pair(v[i].z), finite_pair(v[i].w));
            top[i] = top_of(k[i]) << 16 | top_of(v[i]);
        }
    }
#pragma unroll
    for (int o = 8; o; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) top[i] = __vmaxu2(top[i], __shfl_xor_sync(kFull, top[i], o));
    // lane s: pair s / 4, quotient s % 4: 0 L / absmax(K), 1 absmax(K) / L, 2 and 3 the same of V
    const uint32_t even = s & 4 ? top[N > 1 ? 1 : 0] : top[0], odd = s & 4 ? top[N - 1] : top[N > 2 ? 2 : 0], mine = s & 8 ? odd : even;
    const float absmax = __uint_as_float(s & 2 ? mine << 16 : mine & 0xffff0000u);
    const bool tiny = absmax < kTinyRow;
    const float limit = code_limit<FMT>(), over = s & 1 ? absmax : limit, under = s & 1 ? limit : absmax;
    const float quotient = tiny ? 0.f : __fdiv_rn(over, tiny ? 1.f : under);
    if ((s & 1) && (s >> 2) < N && head0 + 2 * (s >> 2) + y < p.Hkv) {
        const long long to = at + (long long)(head0 + 2 * (s >> 2) + y) * kBlk;
        if (s & 2) p.v_scale[to] = quotient;
        else p.k_scale[to] = quotient;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float ki = __shfl_sync(kFull, quotient, (lane & 16) + 4 * i), vi = __shfl_sync(kFull, quotient, (lane & 16) + 4 * i + 2);
        const uint2 kc = codes_of<FMT>(k[i], ki), vc = codes_of<FMT>(v[i], vi);
        const int head = head0 + 2 * i + y;
        if (head < p.Hkv) {
            const size_t to = ((size_t)at + (size_t)head * kBlk) * kD + 8 * s;
            *reinterpret_cast<uint2*>(p.k + to) = kc;
            *reinterpret_cast<uint2*>(p.v + to) = vc;
        }
    }
}

// the page of block blk of sequence b; -1: none
__device__ __forceinline__ long long write_page(const WriteParams& p, int b, int blk, int lane) {
    const long long index = (long long)b * p.max_blocks + blk, page = p.block_table ? p.block_table[index] : index;
    if (page >= 0 && page < p.num_pages) return page;
    if (lane == 0) atomicOr(p.status, kDevBadPage);
    return -1;
}

constexpr int kWriteFewWarps = 8;

// Few rows: a warp for two heads of a row, so that a step's handful of tokens is spread over the card; the time is the latency of
// the loads, and those of K and V do not wait for the token's place.
template <int FMT>
__global__ void __launch_bounds__(kWriteFewWarps * 32) write_few_kernel(WriteParams p) {
    const int lane = threadIdx.x & 31, pairs = (p.Hkv + 1) / 2;
    const long long task = (long long)blockIdx.x * kWriteFewWarps + (threadIdx.x >> 5);
    pdl_launch_dependents();
    pdl_wait();
    if (task >= (long long)p.num_rows * pairs) return;
    const int row = (int)quick_div(task, pairs), head0 = 2 * (int)(task - (long long)row * pairs);
    uint4 k[1] = {make_uint4(0u, 0u, 0u, 0u)}, v[1] = {make_uint4(0u, 0u, 0u, 0u)};
    if (head0 + (lane >> 4) < p.Hkv) {
        const size_t at = (size_t)row * p.row_stride + (size_t)(head0 + (lane >> 4)) * kD + 8 * (lane & 15);
        k[0] = ldg_plain(reinterpret_cast<const uint4*>(p.k_new + at));
        v[0] = ldg_plain(reinterpret_cast<const uint4*>(p.v_new + at));
    }
    int b = row;
    long long token = 0;
    if (p.row_start) {
        b = sequence_of_row(p.row_start, p.batch, row, lane);
        if (b < 0) return;
        token = (long long)p.first_token[b] + row - p.row_start[b];
    }
    const int n = paged_len(p.seq_lens, b, p.max_blocks, p.status);
    if (!p.row_start) token = n - 1;
    if (token < 0 || token >= n) return;   // a row behind its sequence's new tokens
    const long long page = write_page(p, b, (int)(token >> 6), lane);
    if (page >= 0) store_heads<FMT, 1>(p, page * p.Hkv * kBlk + (token & 63), head0, lane, k, v);
}

// Many rows: a CTA takes an equal share of consecutive (row, eight heads) units, its warps in turn, so that neighbouring tokens are
// written at about the same time.  A warp keeps the copies of its next unit in flight in its own ring (a lane reads back what it
// copied itself, so nothing is waited for but the copies); its sequence and page are looked up again only when a row leaves them.
// Bound by memory: 512 bytes read and 264 written for each head (32 K rows of eight heads: 36 to 38 us, 5.4 to 5.6 TB/s).  A row per
// warp, its loads in registers, waited for the look-ups row by row: 42 us.
constexpr int kWriteWarps = 4, kWriteStages = 2, kWriteStage = 2 * 8 * kD * 2, kWriteCtasPerSm = 5;
constexpr int kWriteSmem = kWriteWarps * kWriteStages * kWriteStage;

template <int FMT>
__global__ void __launch_bounds__(kWriteWarps * 32, kWriteCtasPerSm) write_many_kernel(WriteParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunks = (p.Hkv + 7) / 8;
    const long long units = (long long)p.num_rows * chunks, first_unit = units * blockIdx.x / gridDim.x;
    const int cta_units = (int)(units * (blockIdx.x + 1) / gridDim.x - first_unit);
    const int count = (cta_units - warp + kWriteWarps - 1) / kWriteWarps;   // units first_unit + warp, + kWriteWarps, ...
    const uint32_t ring = smem_u32(smem) + warp * kWriteStages * kWriteStage + 16 * lane;
    pdl_launch_dependents();
    pdl_wait();
    if (count <= 0) return;
    int row = (int)quick_div(first_unit + warp, chunks), chunk = (int)(first_unit + warp - (long long)row * chunks);   // of the next unit
    auto advance = [&](int& r, int& c) {
        c += kWriteWarps;
        while (c >= chunks) {
            c -= chunks;
            ++r;
        }
    };
    int load_row = row, load_chunk = chunk, loaded = 0;
    auto issue = [&]() {
        if (loaded < count) {
            const uint32_t stage = ring + (loaded % kWriteStages) * kWriteStage;
            const size_t at = (size_t)load_row * p.row_stride + (size_t)load_chunk * 8 * kD + 8 * lane;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (8 * load_chunk + 2 * i + (lane >> 4) < p.Hkv) {
                    cp_async16(stage + 512 * i, p.k_new + at + 256 * i);
                    cp_async16(stage + 2048 + 512 * i, p.v_new + at + 256 * i);
                }
            ++loaded;
            advance(load_row, load_chunk);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kWriteStages - 1; ++i) issue();
    int b = -1, n = 0, blk = -1, next = row;   // the sequence's rows end in front of `next`
    long long first = 0, page = -1;            // row 0 would be token `first` of the sequence
    for (int it = 0; it < count; ++it) {
        if (row >= next) {
            if (p.row_start) {
                b = sequence_of_row(p.row_start, p.batch, row, lane);
                next = b + 1 < p.batch ? p.row_start[b + 1] : 0x7fffffff;
                first = b >= 0 ? (long long)p.first_token[b] - p.row_start[b] : -0x80000000LL;   // (in front of all: nowhere)
                n = b >= 0 ? paged_len(p.seq_lens, b, p.max_blocks, p.status) : 0;
            } else {
                b = row;
                next = row + 1;
                n = paged_len(p.seq_lens, b, p.max_blocks, p.status);
                first = (long long)n - 1 - row;
            }
            blk = -1;
        }
        const long long token = first + row;
        const bool in = token >= 0 && token < n;   // else a row behind its sequence's new tokens
        if (in && blk != (int)(token >> 6)) {
            blk = (int)(token >> 6);
            page = write_page(p, b, blk, lane);
        }
        cp_async_wait<kWriteStages - 2>();
        issue();
        if (in && page >= 0) {
            const uint32_t stage = ring + (it % kWriteStages) * kWriteStage;
            uint4 k[4], v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
                if (8 * chunk + 2 * i + (lane >> 4) < p.Hkv) {
                    k[i] = lds128(stage + 512 * i);
                    v[i] = lds128(stage + 2048 + 512 * i);
                }
            }
            store_heads<FMT, 4>(p, page * p.Hkv * kBlk + (token & 63), 8 * chunk, lane, k, v);
        }
        advance(row, chunk);
    }
}

// ---- reading back ---------------------------------------------------------------------------------------------------

struct ReadParams {
    const unsigned char* k;
    const unsigned char* v;
    const float* k_scale;
    const float* v_scale;
    const int32_t* block_table;
    const int32_t* first_token;   // null: 0
    const int32_t* seq_lens;
    __nv_bfloat16* k_out;
    __nv_bfloat16* v_out;
    const int32_t* out_table;
    uint32_t* status;
    int batch, Hkv, max_blocks, num_pages, num_out_pages;
};

constexpr int kReadThreads = 256;

template <int FMT>
__device__ __forceinline__ uint4 codes_to_bf16(uint2 c, float scale) {
    uint32_t h[4];
    codes_to_f16<FMT>(c.x, h[0], h[1]);
    codes_to_f16<FMT>(c.y, h[2], h[3]);
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = f16x2_to_float2(h[i]);
        r[i] = pack_bf16(__fmul_rn(x.x, scale), __fmul_rn(x.y, scale));   // the one rounding to bf16
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// A CTA takes an equal share of all (sequence, block, KV head) tiles; a tile is 64 rows of K and of V.  A lane turns 8
// codes into 16 bytes, so that a warp reads 256 and writes 512 consecutive bytes.  Bound by memory.
template <int FMT>
__global__ void __launch_bounds__(kReadThreads) read_byte_kernel(ReadParams p) {
    pdl_launch_dependents();
    pdl_wait();
    auto first_of = [&](int b) { return p.first_token ? max(p.first_token[b], 0) : 0; };
    auto count = [&](int b) {
        const int n = paged_len(p.seq_lens, b, p.max_blocks, p.status), first = first_of(b);
        return first < n ? blocks_of(n) - (first >> 6) : 0;
    };
    const WarpScan<decltype(count)> scan(p.batch, count, threadIdx.x & 31);
    const long long total = scan.total * p.Hkv, begin = total * blockIdx.x / gridDim.x, end = total * (blockIdx.x + 1) / gridDim.x;
    if (begin >= end) return;
    int b;
    long long off;
    scan.find(begin, p.Hkv, b, off);
    int n = paged_len(p.seq_lens, b, p.max_blocks, p.status), first = first_of(b);
    long long items = (long long)count(b) * p.Hkv;
    for (long long x = begin; x < end; ++x) {
        while (x >= off + items) {   // ends: x < end <= the total of all sequences
            off += items;
            ++b;
            n = paged_len(p.seq_lens, b, p.max_blocks, p.status);
            first = first_of(b);
            items = (long long)count(b) * p.Hkv;
        }
        const int row_blk = (int)quick_div(x - off, p.Hkv), blk = (first >> 6) + row_blk, g = (int)(x - off - (long long)row_blk * p.Hkv);
        const size_t at = (size_t)b * p.max_blocks + blk;
        const long long from = p.block_table ? p.block_table[at] : (long long)at;
        const long long to = p.out_table ? p.out_table[at] : (long long)at;
        if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_out_pages) {
            if (threadIdx.x == 0) atomicOr(p.status, kDevBadPage);
            continue;
        }
        const size_t src = ((size_t)from * p.Hkv + g) * kBlk, dst = ((size_t)to * p.Hkv + g) * kBlk;
        const int row_lo = first - blk * kBlk, row_hi = n - blk * kBlk;
        constexpr int kPer = kBlk * kD / 8 / kReadThreads;   // 8-code vectors of K (and of V) per thread
        uint2 kc[kPer], vc[kPer];
        float ks[kPer], vs[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int vec = i * kReadThreads + threadIdx.x, row = vec >> 4;
            if (row >= row_lo && row < row_hi) {
                kc[i] = *reinterpret_cast<const uint2*>(p.k + src * kD + (size_t)vec * 8);
                vc[i] = *reinterpret_cast<const uint2*>(p.v + src * kD + (size_t)vec * 8);
                ks[i] = p.k_scale[src + row];
                vs[i] = p.v_scale[src + row];
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int vec = i * kReadThreads + threadIdx.x, row = vec >> 4;
            if (row >= row_lo && row < row_hi) {
                *reinterpret_cast<uint4*>(p.k_out + dst * kD + (size_t)vec * 8) = codes_to_bf16<FMT>(kc[i], ks[i]);
                *reinterpret_cast<uint4*>(p.v_out + dst * kD + (size_t)vec * 8) = codes_to_bf16<FMT>(vc[i], vs[i]);
            }
        }
    }
}

// ---- attention over the byte cache ----------------------------------------------------------------------------------

template <int FMT, int NH>
__global__ void __launch_bounds__(Paged<FMT>::kWarps * 32, kPagedCtasPerSm) paged_attention_kernel(PagedParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TeamShared sh;
    pdl_launch_dependents();
    pdl_wait();
    attend_own<FMT, NH>(p, gridDim.x * Paged<FMT>::kWarps, 0, smem, sh, blockIdx.x, threadIdx.x, [] { __syncthreads(); });
}

// ---- merge of the partials --------------------------------------------------------------------------------------------

// warps of a CTA.  16 for one warp per head: half as many CTAs to start (8192 heads: 3 us less); 8 where they are enough for all
// of a head, the CTAs being few then (8 heads: 0.3 us less)
__host__ __device__ constexpr int merge_cta(int warps) { return warps == 1 || warps == 16 ? 16 : 8; }

// WARPS warps per (sequence, query head): weights 2^(lse_i - max), then the weighted mean of the partials; a
// lane has four channels.  The weights of up to 32 WARPS partials are found at once, a lane each, while the first channels are
// already being read.
template <int WARPS>
__global__ void __launch_bounds__(merge_cta(WARPS) * 32) merge_partials_kernel(PagedParams p) {
    constexpr int kMergeWarps = merge_cta(WARPS), kHeads = kMergeWarps / WARPS, kAhead = 4;
    __shared__ float s_max[kMergeWarps], s_weight[kMergeWarps][32], s_total[kMergeWarps];
    __shared__ float4 s_acc[kMergeWarps][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp % WARPS;
    const long long head = (long long)blockIdx.x * kHeads + warp / WARPS;   // b * Hq + h
    // No early launch of the next call's kernel from here: its CTAs would take their places while these still hold some SMs'
    // shared memory at this kernel's size, and an SM that got fewer of them would stay short for the whole pass (measured on
    // the ragged batch: 217 us a pass without, 303 us with).
    pdl_wait();
    const bool live = head < (long long)p.batch * p.Hq;
    if (WARPS == 1 && !live) return;
    const int b = live ? (int)quick_div(head, p.Hq) : 0, h = live ? (int)(head - (long long)b * p.Hq) : 0, g = h / p.G, hl = h - g * p.G;
    const long long before = p.offsets[b], mine = p.offsets[b + 1] - before;
    // The unit's parts c0 .. c1.  CTAs whose four parts lie wholly inside the unit, k0 .. k1, left one partial, at their first
    // part's slot: partial i is part c0 + i in front of them, then one in four, then one by one again.
    constexpr int kCta = Paged<kFmtInt8>::kWarps;
    int c0 = 0, own = 0, single = 0x7fffffff, merged = 0;
    const Shares shares = *p.shares;
    if (mine > 0) {
        const long long off = before * p.Hkv + g * mine;
        c0 = shares.part_of(off);
        const int c1 = shares.part_of(off + mine - 1);
        int k0 = c0 / kCta, k1 = (c1 + 1) / kCta - 1;
        if (shares.begin(k0 * kCta) < off) ++k0;
        if ((c1 + 1) % kCta == 0 && shares.begin(c1 + 1) > off + mine) --k1;
        own = c1 - c0 + 1;
        if (k1 >= k0) {
            single = k0 * kCta - c0;
            merged = k1 - k0 + 1;
            own -= (kCta - 1) * merged;
        }
    }
    const int n = own + shares.chunks;
    // rows of partials: fewer than 65536 units and 2^16 parts of up to eight heads, so that 32 bits are enough
    const unsigned own_row = (unsigned)paged_slot(b * p.Hkv + g, c0) * p.G + hl;       // part c0 + i: + i * G
    const unsigned rows = p.batch * p.G;
    const unsigned pre_row = (unsigned)g * p.prefix_stride * rows + b * p.G + hl;      // prefix partial i: + i * rows
    auto row_of = [&](int i) {
        return i < own ? own_row + (i + (kCta - 1) * min(max(i - single, 0), merged)) * p.G : pre_row + (i - own) * rows;
    };
    auto out_of = [&](int i) {
        return *reinterpret_cast<const float4*>((i < own ? p.part_out : p.prefix_out) + (size_t)row_of(i) * kD + 4 * lane);
    };
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f, top = -INFINITY;
    for (int base = 0; base < n; base += 32 * WARPS) {   // each warp its run of up to 32
        const int run = (min(n - base, 32 * WARPS) + WARPS - 1) / WARPS, first = base + run * w, mine_n = min(run, n - first);
        float4 ahead[kAhead];
#pragma unroll
        for (int x = 0; x < kAhead; ++x)
            if (x < mine_n) ahead[x] = out_of(first + x);
        const float lse = lane < mine_n ? (first + lane < own ? p.part_lse : p.prefix_lse)[row_of(first + lane)] : -INFINITY;
        float high = lse;
#pragma unroll
        for (int o = 16; o; o >>= 1) high = fmaxf(high, __shfl_xor_sync(kFull, high, o));
        high = fmaxf(high, top);
        if (__all_sync(kFull, lse == -INFINITY) && top == -INFINITY) continue;   // nothing so far
        const float use = high == -INFINITY ? 0.f : high;   // (a NaN is no maximum, but makes the sum one)
        const float scale = fast_ex2(top - use), weight = fast_ex2(lse - use);
        top = high;
        s_weight[warp][lane] = weight;
        __syncwarp();
        sum = sum * scale + weight;                  // this lane's share
        acc.x *= scale; acc.y *= scale; acc.z *= scale; acc.w *= scale;
        auto add = [&](int x, const float4& y) {
            const float f = s_weight[warp][x];
            if (f != 0.f) {   // an empty partial's channels may hold anything
                acc.x += f * y.x; acc.y += f * y.y; acc.z += f * y.z; acc.w += f * y.w;
            }
        };
#pragma unroll
        for (int x = 0; x < kAhead; ++x)
            if (x < mine_n) add(x, ahead[x]);
#pragma unroll 4
        for (int x = kAhead; x < mine_n; ++x) add(x, out_of(first + x));
        __syncwarp();
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
    if (WARPS > 1) {
        s_acc[warp][lane] = acc;
        if (lane == 0) { s_total[warp] = sum; s_max[warp] = top; }
        __syncthreads();
        if (w > 0 || !live) return;
#pragma unroll
        for (int x = 1; x < WARPS; ++x) top = fmaxf(top, s_max[warp + x]);
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
        sum = 0.f;
        const float use = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
            const float4 y = s_acc[warp + x][lane];
            const float f = fast_ex2(s_max[warp + x] - use);
            sum += f * s_total[warp + x];
            acc.x += f * y.x; acc.y += f * y.y; acc.z += f * y.z; acc.w += f * y.w;
        }
    }
    const float norm = sum != 0.f ? 1.f / sum : 0.f;
    acc.x *= norm; acc.y *= norm; acc.z *= norm; acc.w *= norm;
    const size_t at = (size_t)head * kD + 4 * lane;
    if (p.out_fp32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = acc;
    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at) = make_uint2(pack_bf16(acc.x, acc.y), pack_bf16(acc.z, acc.w));
    if (lane == 0 && p.lse) p.lse[head] = sum != 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

// ---- host side ----------------------------------------------------------------------------------------------------------

// Workspace of the calls in this file: header, partials of the own tokens, partials of the prefix.  A pure function of its
// arguments, so that ffd_workspace_bytes_prefix and the launch agree.
struct PagedPlan {
    int parts;
    PrefixGeometry geo;   // with a prefix; chunks 0: none
    size_t off_offsets, off_shares, off_lse, off_out, off_plse, off_pout, total;
};

static PagedPlan make_paged_plan(const ffd_config* cfg, int batch, int max_blocks, int max_prefix_blocks, int sms) {
    PagedPlan pl;
    const int G = cfg->num_q_heads / cfg->num_kv_heads;
    const long long units = (long long)batch * cfg->num_kv_heads, blocks = units * max_blocks;
    if (max_prefix_blocks > 0) {
        pl.geo = prefix_geometry(batch * G, cfg->num_kv_heads, max_prefix_blocks, sms);
        pl.parts = pl.geo.parts;
    } else {
        // a warp for every resident slot, but none with fewer than 64 tokens if all sequences are as long as they can be
        const int warps = Paged<kFmtInt8>::kWarps;
        pl.geo = PrefixGeometry{};
        pl.parts = (int)min((blocks + warps - 1) / warps, (long long)kPagedCtasPerSm * sms) * warps;
    }
    // the sizes are bounds that grow with each argument, so that a workspace for the largest call serves the smaller ones
    const size_t rows = (size_t)(units + (max_prefix_blocks > 0 ? (long long)kPrefixCtaParts * sms : pl.parts)) * G;
    const size_t prows = prefix_slots(batch * G, cfg->num_kv_heads, max_prefix_blocks, sms);
    pl.off_offsets = align_up(kInitBytes, 256);
    pl.off_shares = align_up(pl.off_offsets + ((size_t)batch + 1) * sizeof(long long), 256);
    pl.off_lse = pl.off_shares + 256;
    pl.off_out = align_up(pl.off_lse + rows * sizeof(float), 256);
    pl.off_plse = align_up(pl.off_out + rows * kD * sizeof(float), 256);
    pl.off_pout = align_up(pl.off_plse + prows * sizeof(float), 256);
    pl.total = align_up(pl.off_pout + prows * kD * sizeof(float), 256);
    return pl;
}

static ffd_status check_paged(const ffd_config* cfg, int format, int batch, int max_blocks, int num_pages) {
    ffd_status st = check_paged_config(cfg);
    if (st) return st;
    if (format != kFmtInt8 && format != kFmtE4m3 && format != kFmtBf16) return FFD_ERR_UNSUPPORTED;
    st = check_geometry(batch, max_blocks, num_pages);
    if (st) return st;
    if ((long)batch * cfg->num_kv_heads >= 65536L) return FFD_ERR_SHAPE;
    if ((double)num_pages * cfg->num_kv_heads * kBlk >= 2147483648.0 * kBlk) return FFD_ERR_SHAPE;
    return FFD_OK;
}

// The second kernel of a call: as many warps per head as the card has room for, but at least two partials for each if the
// lengths are about equal.  The lengths themselves are on the device.  Where one sequence has most of the tokens, its heads have
// most of the partials and only the average's warps: the merge then takes longer than the attention (9000 tokens beside 63
// sequences of one, 32 query and 8 KV heads: 32 us a call; as single launches 26 us of merge after 12 of attention).
static ffd_status launch_merge(const PagedParams& p, int parts, int sms, cudaStream_t s) {
    const long long heads = (long long)p.batch * p.Hq;
    const long long expected = p.prefix_stride + parts / Paged<kFmtInt8>::kWarps / ((long long)p.batch * p.Hkv) + 2;
    int warps = 16;
    while (warps > 1 && (heads * warps > 64LL * sms || 2 * warps > expected)) warps /= 2;
    void (*kernel)(PagedParams) = warps == 16 ? merge_partials_kernel<16> : warps == 8 ? merge_partials_kernel<8>
                                  : warps == 4 ? merge_partials_kernel<4>
                                  : warps == 2 ? merge_partials_kernel<2> : merge_partials_kernel<1>;
    const int cta = merge_cta(warps), per_cta = cta / warps;
    launch_pdl(kernel, dim3((unsigned)((heads + per_cta - 1) / per_cta)), dim3(cta * 32), 0, s, p);
    return launch_status();
}

struct OwnTokens {   // the sequences' own cache of an attention call
    int format;
    const void *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *block_table, *seq_lens;
    int batch, max_blocks, num_pages;
};

struct SharedTokens {   // the prefix; max_blocks 0: none
    const void *k, *v;
    const int32_t *table, *len;
    int max_blocks, num_pages;
};

static ffd_status run_attention(const ffd_config* cfg, const void* q, const OwnTokens& own, const SharedTokens& pre, void* out,
                                float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    ffd_status st = check_paged(cfg, own.format, own.batch, own.max_blocks, own.num_pages);
    if (st) return st;
    if (!q || !own.k || !own.v || !own.seq_lens || !out || !workspace) return FFD_ERR_NULL;
    if (own.format != kFmtBf16 && (!own.k_scale || !own.v_scale)) return FFD_ERR_NULL;
    if (any_misaligned(q, own.k, own.v, own.k_scale, own.v_scale, own.block_table, own.seq_lens, out, lse, workspace))
        return FFD_ERR_ALIGN;
    if (pre.max_blocks) {
        if (!pre.k || !pre.v || !pre.table || !pre.len) return FFD_ERR_NULL;
        if (pre.max_blocks < 0 || pre.num_pages <= 0 || (long)pre.max_blocks * kBlk > 0x7fffffffL) return FFD_ERR_SHAPE;
        if ((double)pre.num_pages * cfg->num_kv_heads * kBlk >= 2147483648.0) return FFD_ERR_SHAPE;   // a TMA row coordinate
        if (any_misaligned(pre.k, pre.v, pre.table, pre.len)) return FFD_ERR_ALIGN;
    }
    const int sms = device_sms();
    const PagedPlan pl = make_paged_plan(cfg, own.batch, own.max_blocks, pre.max_blocks, sms);
    if (workspace_bytes < pl.total) return FFD_ERR_WORKSPACE;
    PagedParams p;
    memset(&p, 0, sizeof p);
    char* ws = static_cast<char*>(workspace);
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const unsigned char*>(own.k);
    p.v = static_cast<const unsigned char*>(own.v);
    p.k_scale = own.k_scale;
    p.v_scale = own.v_scale;
    p.block_table = own.block_table;
    p.seq_lens = own.seq_lens;
    p.batch = own.batch;
    p.Hq = cfg->num_q_heads;
    p.Hkv = cfg->num_kv_heads;
    p.G = p.Hq / p.Hkv;
    p.max_blocks = own.max_blocks;
    p.num_pages = own.num_pages;
    p.logit_scale = (cfg->sm_scale > 0.f ? cfg->sm_scale : 1.0f / sqrtf((float)kD)) * kLog2e;
    p.status = reinterpret_cast<uint32_t*>(ws);
    p.part_lse = reinterpret_cast<float*>(ws + pl.off_lse);
    p.part_out = reinterpret_cast<float*>(ws + pl.off_out);
    p.offsets = reinterpret_cast<long long*>(ws + pl.off_offsets);
    p.shares = reinterpret_cast<Shares*>(ws + pl.off_shares);
    p.prefix_lse = reinterpret_cast<const float*>(ws + pl.off_plse);
    p.prefix_out = reinterpret_cast<const float*>(ws + pl.off_pout);
    p.prefix_stride = pl.geo.chunks;
    p.out = out;
    p.lse = lse;
    p.out_fp32 = cfg->out_dtype;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (pre.max_blocks) {
        PrefixParams pp;
        memset(&pp, 0, sizeof pp);
        pp.q = p.q;
        pp.table = pre.table;
        pp.len = pre.len;
        pp.batch = p.batch;
        pp.Hq = p.Hq;
        pp.Hkv = p.Hkv;
        pp.G = p.G;
        pp.max_blocks = pre.max_blocks;
        pp.num_pages = pre.num_pages;
        pp.groups = pl.geo.groups;
        pp.chunks = pl.geo.chunks;
        pp.logit_scale = p.logit_scale;
        pp.out = reinterpret_cast<float*>(ws + pl.off_pout);
        pp.lse = reinterpret_cast<float*>(ws + pl.off_plse);
        pp.status = p.status;
        pp.query_copy = kPrefixRows % p.G == 0;
        pp.two_piece = cfg->out_dtype == 1;
        st = launch_prefix(pp, pl.geo, pre.k, pre.v, own.format, p, s);
        if (st) return st;
    } else {   // (the byte formats only)
        const bool wide = p.G > 4;   // two tiles of four heads
        void (*kernel)(PagedParams) =
            own.format == kFmtInt8 ? (wide ? paged_attention_kernel<kFmtInt8, 2> : paged_attention_kernel<kFmtInt8, 1>)
                                   : (wide ? paged_attention_kernel<kFmtE4m3, 2> : paged_attention_kernel<kFmtE4m3, 1>);
        constexpr int kWarps = Paged<kFmtInt8>::kWarps, kSmem = Paged<kFmtInt8>::kSmem;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return FFD_ERR_CUDA;
        launch_pdl(kernel, dim3(pl.parts / kWarps), dim3(kWarps * 32), kSmem, s, p);
        st = launch_status();   // without its partition in the workspace the merge would read anywhere
        if (st) return st;
    }
    return launch_merge(p, pl.parts, sms, s);
}

}  // namespace ffd

using namespace ffd;

extern "C" {

ffd_status ffd_workspace_bytes_prefix(const ffd_config* cfg, int32_t batch, int32_t max_blocks_per_seq,
                                      int32_t max_prefix_blocks, size_t* bytes) {
    ffd_status st = check_paged(cfg, kFmtInt8, batch, max_blocks_per_seq, 1);
    if (st) return st;
    if (!bytes) return FFD_ERR_NULL;
    if (max_prefix_blocks < 0 || (long)max_prefix_blocks * kBlk > 0x7fffffffL) return FFD_ERR_SHAPE;
    *bytes = make_paged_plan(cfg, batch, max_blocks_per_seq, max_prefix_blocks, device_sms()).total;
    return FFD_OK;
}

ffd_status ffd_write_kv_byte(const ffd_config* cfg, int32_t format, const void* k_new, const void* v_new, int64_t row_stride,
                             int32_t num_rows, const int32_t* row_start, void* k_byte, void* v_byte, float* k_scale,
                             float* v_scale, const int32_t* block_table, const int32_t* first_token, const int32_t* seq_lens,
                             int32_t batch, int32_t max_blocks_per_seq, int32_t num_pages, void* workspace,
                             size_t workspace_bytes, void* stream) {
    ffd_status st = check_paged(cfg, format, batch, max_blocks_per_seq, num_pages);
    if (st) return st;
    if (format == kFmtBf16) return FFD_ERR_UNSUPPORTED;
    if (!k_new || !v_new || !k_byte || !v_byte || !k_scale || !v_scale || !seq_lens || !workspace) return FFD_ERR_NULL;
    if ((row_start == nullptr) != (first_token == nullptr)) return FFD_ERR_NULL;
    if (num_rows <= 0 || (!row_start && num_rows != batch)) return FFD_ERR_SHAPE;
    const int64_t width = (int64_t)cfg->num_kv_heads * kD;
    if (row_stride < width || row_stride % 8) return FFD_ERR_SHAPE;
    if (workspace_bytes < kHeaderBytes) return FFD_ERR_WORKSPACE;
    if (any_misaligned(k_new, v_new, row_start, k_byte, v_byte, k_scale, v_scale, block_table, first_token, seq_lens, workspace))
        return FFD_ERR_ALIGN;
    WriteParams p{static_cast<const __nv_bfloat16*>(k_new), static_cast<const __nv_bfloat16*>(v_new), row_stride, row_start,
                  first_token, seq_lens, block_table, static_cast<unsigned char*>(k_byte), static_cast<unsigned char*>(v_byte),
                  k_scale, v_scale, static_cast<uint32_t*>(workspace), num_rows, batch, cfg->num_kv_heads, max_blocks_per_seq,
                  num_pages};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // a warp for every two heads of a row while that fills the card once
    const long long few = (long long)num_rows * ((p.Hkv + 1) / 2);
    const int sms = device_sms();
    if (few <= 64LL * sms) {
        launch_pdl(format == kFmtInt8 ? write_few_kernel<kFmtInt8> : write_few_kernel<kFmtE4m3>,
                   dim3((unsigned)((few + kWriteFewWarps - 1) / kWriteFewWarps)), dim3(kWriteFewWarps * 32), 0, s, p);
    } else {
        void (*kernel)(WriteParams) = format == kFmtInt8 ? write_many_kernel<kFmtInt8> : write_many_kernel<kFmtE4m3>;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWriteSmem) != cudaSuccess) return FFD_ERR_CUDA;
        launch_pdl(kernel, dim3(4 * kWriteCtasPerSm * sms), dim3(kWriteWarps * 32), kWriteSmem, s, p);   // (four rounds: shorter shares)
    }
    return launch_status();
}

ffd_status ffd_read_kv_byte(const ffd_config* cfg, int32_t format, const void* k_byte, const void* v_byte, const float* k_scale,
                            const float* v_scale, const int32_t* block_table, const int32_t* first_token,
                            const int32_t* seq_lens, int32_t batch, int32_t max_blocks_per_seq, int32_t num_pages,
                            void* k_cache, void* v_cache, const int32_t* cache_table, int32_t num_cache_pages, void* workspace,
                            size_t workspace_bytes, void* stream) {
    ffd_status st = check_paged(cfg, format, batch, max_blocks_per_seq, num_pages);
    if (st) return st;
    if (format == kFmtBf16) return FFD_ERR_UNSUPPORTED;
    if (!k_byte || !v_byte || !k_scale || !v_scale || !seq_lens || !k_cache || !v_cache || !workspace) return FFD_ERR_NULL;
    if (num_cache_pages <= 0) return FFD_ERR_SHAPE;
    if (workspace_bytes < kHeaderBytes) return FFD_ERR_WORKSPACE;
    if (any_misaligned(k_byte, v_byte, k_scale, v_scale, block_table, first_token, seq_lens, k_cache, v_cache, cache_table, workspace))
        return FFD_ERR_ALIGN;
    ReadParams p{static_cast<const unsigned char*>(k_byte), static_cast<const unsigned char*>(v_byte), k_scale, v_scale,
                 block_table, first_token, seq_lens, static_cast<__nv_bfloat16*>(k_cache), static_cast<__nv_bfloat16*>(v_cache),
                 cache_table, static_cast<uint32_t*>(workspace), batch, cfg->num_kv_heads, max_blocks_per_seq, num_pages,
                 num_cache_pages};
    const long long items = (long long)batch * cfg->num_kv_heads * max_blocks_per_seq;
    const unsigned grid = (unsigned)min(items, 64LL * device_sms());   // short shares: 8 CTAs per SM took a tenth longer
    launch_pdl(format == kFmtInt8 ? read_byte_kernel<kFmtInt8> : read_byte_kernel<kFmtE4m3>, dim3(grid), dim3(kReadThreads), 0,
               static_cast<cudaStream_t>(stream), p);
    return launch_status();
}

ffd_status ffd_decode_byte(const ffd_config* cfg, int32_t format, const void* q, const void* k_byte, const void* v_byte,
                           const float* k_scale, const float* v_scale, const int32_t* block_table, const int32_t* seq_lens,
                           int32_t batch, int32_t max_blocks_per_seq, int32_t num_pages, void* out, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
    if (format != FFD_BYTE_INT8 && format != FFD_BYTE_E4M3) return cfg ? FFD_ERR_UNSUPPORTED : FFD_ERR_NULL;
    const OwnTokens own{format, k_byte, v_byte, k_scale, v_scale, block_table, seq_lens, batch, max_blocks_per_seq, num_pages};
    return run_attention(cfg, q, own, SharedTokens{}, out, lse, workspace, workspace_bytes, stream);
}

ffd_status ffd_decode_prefix(const ffd_config* cfg, const void* q, const void* k_cache, const void* v_cache,
                             const int32_t* prefix_table, const int32_t* prefix_len, int32_t max_prefix_blocks,
                             const int32_t* block_table, const int32_t* seq_lens, int32_t batch, int32_t max_blocks_per_seq,
                             int32_t num_pages, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (max_prefix_blocks <= 0) return cfg ? FFD_ERR_SHAPE : FFD_ERR_NULL;
    const OwnTokens own{kFmtBf16, k_cache, v_cache, nullptr, nullptr, block_table, seq_lens, batch, max_blocks_per_seq, num_pages};
    const SharedTokens pre{k_cache, v_cache, prefix_table, prefix_len, max_prefix_blocks, num_pages};
    return run_attention(cfg, q, own, pre, out, lse, workspace, workspace_bytes, stream);
}

ffd_status ffd_decode_prefix_byte(const ffd_config* cfg, int32_t format, const void* q, const void* k_cache, const void* v_cache,
                                  const int32_t* prefix_table, const int32_t* prefix_len, int32_t max_prefix_blocks,
                                  int32_t num_prefix_pages, const void* k_byte, const void* v_byte, const float* k_scale,
                                  const float* v_scale, const int32_t* block_table, const int32_t* seq_lens, int32_t batch,
                                  int32_t max_blocks_per_seq, int32_t num_pages, void* out, float* lse, void* workspace,
                                  size_t workspace_bytes, void* stream) {
    if (format != FFD_BYTE_INT8 && format != FFD_BYTE_E4M3) return cfg ? FFD_ERR_UNSUPPORTED : FFD_ERR_NULL;
    if (max_prefix_blocks <= 0) return cfg ? FFD_ERR_SHAPE : FFD_ERR_NULL;
    const OwnTokens own{format, k_byte, v_byte, k_scale, v_scale, block_table, seq_lens, batch, max_blocks_per_seq, num_pages};
    const SharedTokens pre{k_cache, v_cache, prefix_table, prefix_len, max_prefix_blocks, num_prefix_pages};
    return run_attention(cfg, q, own, pre, out, lse, workspace, workspace_bytes, stream);
}

}  // extern "C"
