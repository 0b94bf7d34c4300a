// The byte cache: K and V with one byte per element (int8 or e4m3) and one binary32 scale for each token and KV head.
// Kernels that write it, read it back into 16-bit pages and attend to it, and the merge of partial attention results.
#include <cuda_runtime.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "../../include/ffd.h"
#include "ffd_host.cuh"
#include "ffd_paged.cuh"
#include "ffd_prefix.cuh"

namespace ffd {

// ---- conversions ------------------------------------------------------------------------------------------------

template <int FMT>
__device__ __forceinline__ constexpr float code_limit() { return FMT == kFmtInt8 ? 127.f : 448.f; }

// below this a row is stored as zeros: L / absmax would leave binary32
constexpr float kTinyRow = 7.888609052210118e-31f;   // 2^-100

// four codes (bytes c0 c1 c2 c3) -> f16 pairs (c0, c1) and (c2, c3), exactly
template <int FMT>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if constexpr (FMT == kFmtInt8) {
        // 0x6400 | u is the f16 number 1024 + u for a byte u; u = code + 128
        const uint32_t u = w ^ 0x80808080u;
        const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), bias);
        const __half2 y = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
        lo = *reinterpret_cast<const uint32_t*>(&x);
        hi = *reinterpret_cast<const uint32_t*>(&y);
    } else {
        asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
            : "=r"(lo), "=r"(hi)
            : "r"(w));
    }
}

__device__ __forceinline__ float2 f16x2_to_float2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

__device__ __forceinline__ float2 bf16x2_to_float2(uint32_t x) {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}

// four scaled values -> four codes.  int8: adding 1.5 * 2^23 rounds to the nearest integer (ties to even) and leaves its
// two's complement in the low byte; |y| <= 127 (1 + 2^-22) rounds to at most 127.
template <int FMT>
__device__ __forceinline__ uint32_t floats_to_codes(float y0, float y1, float y2, float y3) {
    if constexpr (FMT == kFmtInt8) {
        const float magic = 12582912.f;
        const uint32_t a = __float_as_uint(__fadd_rn(y0, magic)), b = __float_as_uint(__fadd_rn(y1, magic));
        const uint32_t c = __float_as_uint(__fadd_rn(y2, magic)), d = __float_as_uint(__fadd_rn(y3, magic));
        return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
    } else {
        uint32_t r;
        asm("{\n .reg .b16 a, b;\n cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n mov.b32 %0, {a, b};\n}\n"
            : "=r"(r)
            : "f"(y0), "f"(y1), "f"(y2), "f"(y3));
        return r;
    }
}

// ---- writing ------------------------------------------------------------------------------------------------------

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
    int chunks;                   // tasks per row: ceil(Hkv / (2 * PAIRS))
};

// Eight elements (16 bytes of a row) per lane, 16 lanes per head: absmax over the 16 lanes, scale, codes.
// NaN becomes 0 and an infinity the largest finite bf16, so that one bad element cannot spoil its row's neighbours.
template <int FMT>
__device__ __forceinline__ uint2 quantise_lane(uint4 x, float& scale) {
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t top2 = 0;   // magnitudes as 16-bit integers: the order of bf16 numbers
#pragma unroll
    for (int i = 0; i < 4; ++i) top2 = __vmaxu2(top2, w[i] & 0x7fff7fffu);
    uint32_t top = max(top2 & 0xffffu, top2 >> 16);
    if (__any_sync(kFull, top >= 0x7f80u)) {
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t e = (w[i / 2] >> (16 * (i & 1))) & 0xffffu;
            const uint32_t mag = e & 0x7fffu;
            e = mag > 0x7f80u ? 0u : mag == 0x7f80u ? (e & 0x8000u) | 0x7f7fu : e;
            w[i / 2] = (i & 1) ? (w[i / 2] & 0xffffu) | (e << 16) : (w[i / 2] & 0xffff0000u) | e;
            top = max(top, e & 0x7fffu);
        }
    }
#pragma unroll
    for (int o = 8; o; o >>= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
    const float absmax = __uint_as_float(top << 16);
    const bool tiny = absmax < kTinyRow;
    const float inv = tiny ? 0.f : __fdiv_rn(code_limit<FMT>(), absmax);
    scale = tiny ? 0.f : __fdiv_rn(absmax, code_limit<FMT>());
    uint2 codes;
    const float2 a = bf16x2_to_float2(w[0]), b = bf16x2_to_float2(w[1]), c = bf16x2_to_float2(w[2]), d = bf16x2_to_float2(w[3]);
    codes.x = floats_to_codes<FMT>(__fmul_rn(a.x, inv), __fmul_rn(a.y, inv), __fmul_rn(b.x, inv), __fmul_rn(b.y, inv));
    codes.y = floats_to_codes<FMT>(__fmul_rn(c.x, inv), __fmul_rn(c.y, inv), __fmul_rn(d.x, inv), __fmul_rn(d.y, inv));
    return codes;
}

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

constexpr int kWriteWarps = 8;

// A warp takes one row (a new token) and 2 * PAIRS of its KV heads: a 512-byte load holds two heads, and all loads of K and
// V are in flight before the token's place is looked up.  Bound by memory: 512 bytes read and 264 written for each head.
template <int FMT, int PAIRS>
__global__ void __launch_bounds__(kWriteWarps * 32) write_byte_kernel(WriteParams p) {
    const int lane = threadIdx.x & 31;
    pdl_launch_dependents();
    pdl_wait();
    const long long tasks = (long long)p.num_rows * p.chunks;
    for (long long task = (long long)blockIdx.x * kWriteWarps + (threadIdx.x >> 5); task < tasks;
         task += (long long)gridDim.x * kWriteWarps) {
        const int row = (int)(task / p.chunks), head0 = (int)(task % p.chunks) * 2 * PAIRS;
        const int sub = lane & 15;
        uint4 kx[PAIRS], vx[PAIRS];
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const int head = head0 + 2 * i + (lane >> 4);
            kx[i] = vx[i] = make_uint4(0u, 0u, 0u, 0u);
            if (head < p.Hkv) {
                const size_t at = (size_t)row * p.row_stride + (size_t)head * kD + 8 * sub;
                kx[i] = ldg_plain(reinterpret_cast<const uint4*>(p.k_new + at));
                vx[i] = ldg_plain(reinterpret_cast<const uint4*>(p.v_new + at));
            }
        }
        int b, token, n;
        if (p.row_start) {
            b = sequence_of_row(p.row_start, p.batch, row, lane);
            if (b < 0) continue;
            n = paged_len(p.seq_lens, b, p.max_blocks, p.status);
            const long long t = (long long)p.first_token[b] + row - p.row_start[b];
            if (t < 0 || t >= n) continue;   // a row behind its sequence's new tokens
            token = (int)t;
        } else {
            b = row;
            n = paged_len(p.seq_lens, b, p.max_blocks, p.status);
            token = n - 1;
            if (token < 0) continue;
        }
        const int blk = token >> 6;
        const int page = p.block_table ? p.block_table[(size_t)b * p.max_blocks + blk] : b * p.max_blocks + blk;
        if (page < 0 || page >= p.num_pages) {
            if (lane == 0) atomicOr(p.status, kDevBadPage);
            continue;
        }
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            if (head0 + 2 * i >= p.Hkv) break;   // uniform over the warp
            const int head = head0 + 2 * i + (lane >> 4);
            float ks, vs;
            const uint2 kc = quantise_lane<FMT>(kx[i], ks), vc = quantise_lane<FMT>(vx[i], vs);
            if (head < p.Hkv) {
                const size_t at = ((size_t)page * p.Hkv + head) * kBlk + (token & 63);
                *reinterpret_cast<uint2*>(p.k + at * kD + 8 * sub) = kc;
                *reinterpret_cast<uint2*>(p.v + at * kD + 8 * sub) = vc;
                if (sub == 0) {
                    p.k_scale[at] = ks;
                    p.v_scale[at] = vs;
                }
            }
        }
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
    __shared__ long long s_off;
    __shared__ int s_b;
    const ItemScan<kReadThreads, decltype(count)> scan(p.batch, count);
    const long long total = scan.total * p.Hkv, begin = total * blockIdx.x / gridDim.x, end = total * (blockIdx.x + 1) / gridDim.x;
    int b;
    long long off;
    if (begin < end && scan.find(begin, p.Hkv, b, off)) {
        s_b = b;
        s_off = off;
    }
    __syncthreads();
    if (begin >= end) return;
    b = s_b;
    off = s_off;
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

// ---- attention over the sequences' own pages ----------------------------------------------------------------------
//
// A warp works alone on an equal share of all items (kTokens tokens of one sequence and KV head) with mma.sync:
//   S = Q K^T : rows = query heads (0..7) and, in rows 8..15, what a second piece of Q holds; columns = tokens, tiles of 8
//   O = P V   : rows 0..7 = P rounded to 16 bits, rows 8..15 = what the rounding left, so that P keeps 22 (16) bits at no cost
// Token 16 u + 4 j + 2 i + x of an item sits in tile 2 u + i, column 2 j + x: the lane that holds S for columns 2 j, 2 j + 1
// holds it for tokens 4 j .. 4 j + 3 of each 16, whose scales are one 16-byte read, and the accumulator fragment of S is the
// A fragment of P.  The order of the channels inside a contraction is permuted so that every shared-memory read is 16 bytes of
// one row.
//
// Byte formats.  K meets the tensor cores as it is stored, with no conversion:
//   e4m3: q, scaled by a power of two per head to below 256, is the sum of two e4m3 numbers (4 bits each of its 8; elements
//         2^-10 below the head's largest lose bits, under 2^-17 of it), one m16n8k32 per 32 channels and 8 tokens
//   int8: q = qmax / 127 (d0 + d1 / 254 + d2 / 254^2) with integers |d| <= 127 (24 bits), two m16n8k32
// V becomes f16 exactly and the tokens' scales stay outside the products:
//   t = (q . code) * k_scale * logit_scale,   o += 2^(t + log2 v_scale - m') code_v,   l += 2^(t - m)
// with separate running references m' and m: the weights that meet the codes lie in [0, 2^8] whatever the scales are.
// 16-bit format: bf16 products, P in two bf16 pieces, m' = m.
//
// The unpacking of V (byte permutes and conversions at half rate) and the bookkeeping bound the instruction issue at about the
// rate at which memory delivers, so both are kept small: 32 tokens per pass share one maximum, one vote and one ring slot.
// The next item's copies (cp.async, 16 bytes a lane, into the warp's own ring) are in flight during each pass, also across the
// ends of sequences.

template <int FMT>
struct Paged {
    static constexpr int kWarps = 4;
    static constexpr int kShift = FMT == kFmtBf16 ? 4 : 5;
    static constexpr int kTokens = 1 << kShift;                                // of an item
    static constexpr int kRow = FMT == kFmtBf16 ? 2 * kD : kD;                 // bytes of a token's key
    static constexpr int kScaleBytes = FMT == kFmtBf16 ? 0 : kTokens * 4;
    static constexpr int kStage = 2 * kTokens * kRow + 2 * kScaleBytes;
    static constexpr int kStages = 2;
    static constexpr int kSmem = kWarps * kStages * kStage;
};
constexpr int kPagedCtasPerSm = 3;
constexpr int kPagedMinShift = 6;   // log2 of the tokens that a part has at least

constexpr float kLazyMax = 8.f;   // a reference is raised when a logit exceeds it by this many powers of two

// place in the flattened list
struct Cursor {
    int b, g, item, n, items;
};

template <int SHIFT>
__device__ __forceinline__ void cursor_next(Cursor& c, const PagedParams& p) {
    if (++c.item < c.items) return;
    c.item = 0;
    if (++c.g < p.Hkv) return;
    c.g = 0;
    do {
        if (++c.b >= p.batch) {   // behind the last item: never used
            c.n = c.items = 0;
            return;
        }
        c.n = paged_len(p.seq_lens, c.b, p.max_blocks, p.status);
        c.items = ceil_shift(c.n, SHIFT);
    } while (c.items == 0);
}

template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float fast_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor_sync(kFull, x, 1));
    return fmaxf(x, __shfl_xor_sync(kFull, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(kFull, x, 1);
    return x + __shfl_xor_sync(kFull, x, 2);
}

// A warp's attention state for one unit: row r = lane / 4 is head r of the group
template <int FMT>
struct WarpState {
    // A fragments of Q.  bf16: 8 k-steps of two registers (rows 0..7 only); bytes: register w of a piece covers channels
    // 64 (w / 4) + 16 j + 4 (w % 4) .. + 3, pieces at 0, 8 and (int8) 16
    uint32_t qa[FMT == kFmtInt8 ? 24 : 16];
    float q_scale;       // logit_scale and what was taken out of q
    float m, mp, l;      // references (log2) of l and of acc; l is this lane's share
    float acc[16][4];
};

template <int FMT>
__device__ __forceinline__ void state_begin(WarpState<FMT>& st, const PagedParams& p, int b, int g, int lane) {
    const int r = lane >> 2, j = lane & 3;
    const __nv_bfloat16* q = p.q + ((size_t)b * p.Hq + (size_t)g * p.G + r) * kD;
    if constexpr (FMT == kFmtBf16) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (r < p.G) x = *reinterpret_cast<const uint4*>(q + 32 * h + 8 * j);
            st.qa[4 * h] = x.x; st.qa[4 * h + 1] = x.y; st.qa[4 * h + 2] = x.z; st.qa[4 * h + 3] = x.w;
        }
        st.q_scale = p.logit_scale;
    } else {
        uint32_t raw[16];   // raw[2 w], raw[2 w + 1]: the four channels of register w
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                uint4 x = make_uint4(0u, 0u, 0u, 0u);
                if (r < p.G) x = *reinterpret_cast<const uint4*>(q + 64 * h + 16 * j + 8 * y);
                uint32_t* to = raw + 8 * h + 4 * y;
                to[0] = x.x; to[1] = x.y; to[2] = x.z; to[3] = x.w;
            }
        uint32_t top2 = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) top2 = __vmaxu2(top2, raw[i] & 0x7fff7fffu);
        uint32_t top = max(top2 & 0xffffu, top2 >> 16);
        top = max(top, __shfl_xor_sync(kFull, top, 1));
        top = max(top, __shfl_xor_sync(kFull, top, 2));
        // 2^(e - 127) <= largest < 2^(e - 126): scaled by 2^(127 - e) it is in [1, 2)
        const int e = min(max((int)(top >> 7), 1), 253);
        const float down = __uint_as_float((uint32_t)(254 - e) << 23), up = __uint_as_float((uint32_t)e << 23);
        if constexpr (FMT == kFmtE4m3) {
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const float2 a = bf16x2_to_float2(raw[2 * w]), c = bf16x2_to_float2(raw[2 * w + 1]);
                const float x0 = a.x * down * 128.f, x1 = a.y * down * 128.f, x2 = c.x * down * 128.f, x3 = c.y * down * 128.f;
                const uint32_t hi = floats_to_codes<kFmtE4m3>(x0, x1, x2, x3);
                uint32_t h0, h1;
                codes_to_f16<kFmtE4m3>(hi, h0, h1);
                const float2 f0 = f16x2_to_float2(h0), f1 = f16x2_to_float2(h1);
                st.qa[w] = hi;
                st.qa[8 + w] = floats_to_codes<kFmtE4m3>(x0 - f0.x, x1 - f0.y, x2 - f1.x, x3 - f1.y);
            }
            st.q_scale = p.logit_scale * up * 0.0078125f;
        } else {
            const float big = fmaxf(__uint_as_float(top << 16) * down, 1e-30f);   // in [1, 2), or q is zero
            const float unit = big / 127.f, inv = 127.f / big;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const float2 a = bf16x2_to_float2(raw[2 * w]), c = bf16x2_to_float2(raw[2 * w + 1]);
                float d[3][4];
                const float x[4] = {a.x * down, a.y * down, c.x * down, c.y * down};
#pragma unroll
                for (int y = 0; y < 4; ++y) {   // digits of x / unit; each remainder is at most half of its digit's unit
                    const float v = x[y] * inv;
                    d[0][y] = fminf(fmaxf(rintf(v), -127.f), 127.f);
                    const float v1 = fmaf(-d[0][y], unit, x[y]) * inv * 254.f;
                    d[1][y] = fminf(fmaxf(rintf(v1), -127.f), 127.f);
                    d[2][y] = fminf(fmaxf(rintf((v1 - d[1][y]) * 254.f), -127.f), 127.f);
                }
#pragma unroll
                for (int k = 0; k < 3; ++k) st.qa[8 * k + w] = floats_to_codes<kFmtInt8>(d[k][0], d[k][1], d[k][2], d[k][3]);
            }
            st.q_scale = p.logit_scale * up * unit;
        }
    }
    st.m = st.mp = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) st.acc[i][0] = st.acc[i][1] = st.acc[i][2] = st.acc[i][3] = 0.f;
}

// An item in a stage of shared memory: the first `rows` (1 .. kTokens) of its tokens are the sequence's
template <int FMT>
__device__ __forceinline__ void state_item(WarpState<FMT>& st, uint32_t stage, int rows, int lane) {
    using P = Paged<FMT>;
    constexpr int kRow = P::kRow, kTok = P::kTokens, kSets = kTok / 16;   // sets of 16 tokens
    const int r = lane >> 2, j = lane & 3;
    float t[kSets][4];   // q . k of tokens 16 u + 4 j + y, then the logits
#pragma unroll
    for (int u = 0; u < kSets; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t row = stage + (16 * u + 4 * (r >> 1) + 2 * i + (r & 1)) * kRow;
            const uint32_t swizzle = (r & 1) << 2;   // odd rows have their chunks XOR 4: eight rows' reads miss each other
            if constexpr (FMT == kFmtBf16) {
                float c0 = 0.f, c1 = 0.f;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const uint4 x = lds128(row + (((4 * h + j) ^ swizzle) << 4));
                    mma_bf16_top(c0, c1, st.qa[4 * h], st.qa[4 * h + 1], x.x, x.y);
                    mma_bf16_top(c0, c1, st.qa[4 * h + 2], st.qa[4 * h + 3], x.z, x.w);
                }
                t[u][2 * i] = c0;
                t[u][2 * i + 1] = c1;
            } else if constexpr (FMT == kFmtE4m3) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 x = lds128(row + (((4 * h + j) ^ swizzle) << 4));
                    mma_e4m3(c, st.qa[4 * h], st.qa[8 + 4 * h], st.qa[4 * h + 1], st.qa[8 + 4 * h + 1], x.x, x.y);
                    mma_e4m3(c, st.qa[4 * h + 2], st.qa[8 + 4 * h + 2], st.qa[4 * h + 3], st.qa[8 + 4 * h + 3], x.z, x.w);
                }
                t[u][2 * i] = c[0] + c[2];
                t[u][2 * i + 1] = c[1] + c[3];
            } else {
                int c[4] = {0, 0, 0, 0}, d[4] = {0, 0, 0, 0};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 x = lds128(row + (((4 * h + j) ^ swizzle) << 4));
                    mma_s8(c, st.qa[4 * h], st.qa[8 + 4 * h], st.qa[4 * h + 1], st.qa[8 + 4 * h + 1], x.x, x.y);
                    mma_s8(d, st.qa[16 + 4 * h], 0u, st.qa[16 + 4 * h + 1], 0u, x.x, x.y);
                    mma_s8(c, st.qa[4 * h + 2], st.qa[8 + 4 * h + 2], st.qa[4 * h + 3], st.qa[8 + 4 * h + 3], x.z, x.w);
                    mma_s8(d, st.qa[16 + 4 * h + 2], 0u, st.qa[16 + 4 * h + 3], 0u, x.z, x.w);
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    t[u][2 * i + x] = (float)c[x] + ((float)c[x + 2] + (float)d[x] * (1.f / 254.f)) * (1.f / 254.f);
            }
        }
    float tv[kSets][4];   // with log2 of the values' scales
    float top = -INFINITY, topv = -INFINITY;
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        if constexpr (FMT != kFmtBf16) {
            const uint4 a = lds128(stage + 2 * kTok * kRow + 64 * u + 16 * j);
            const uint4 b = lds128(stage + 2 * kTok * kRow + P::kScaleBytes + 64 * u + 16 * j);
            const uint32_t au[4] = {a.x, a.y, a.z, a.w}, bu[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                t[u][y] *= __uint_as_float(au[y]) * st.q_scale;
                tv[u][y] = t[u][y] + fast_lg2(__uint_as_float(bu[y]));   // a zero row: -inf, weight 0
            }
        } else {
#pragma unroll
            for (int y = 0; y < 4; ++y) t[u][y] *= st.q_scale;
        }
        if (rows < kTok) {   // uniform: the sequence's last item
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (16 * u + 4 * j + y >= rows) t[u][y] = tv[u][y] = -INFINITY;
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            top = fmaxf(top, t[u][y]);
            if (FMT != kFmtBf16) topv = fmaxf(topv, tv[u][y]);
        }
    }
    const bool raise = top > st.m + kLazyMax || (FMT != kFmtBf16 && topv > st.mp + kLazyMax);
    if (__any_sync(kFull, raise)) {   // always for the first tokens: -inf + 8 is -inf
        const float m = fmaxf(st.m, quad_max(top));
        const float use = m == -INFINITY ? 0.f : m;
        float alpha = fast_ex2(st.m - use);
        st.l *= alpha;
        st.m = m;
        if constexpr (FMT != kFmtBf16) {
            const float mp = fmaxf(st.mp, quad_max(topv));
            alpha = mp == -INFINITY ? 1.f : fast_ex2(st.mp - mp);
            st.mp = mp;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) st.acc[i][x] *= alpha;
    }
    const float use = st.m == -INFINITY ? 0.f : st.m, usep = st.mp == -INFINITY ? 0.f : st.mp;
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        float hi[4], lo[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const float e = fast_ex2(t[u][y] - use);
            st.l += e;
            if constexpr (FMT == kFmtBf16) {
                hi[y] = bf16_round(e);
                lo[y] = e - hi[y];
            } else {
                const float w = fast_ex2(tv[u][y] - usep);
                hi[y] = __half2float(__float2half_rn(w));
                lo[y] = (w - hi[y]) * 2048.f;   // 11 bits further down: the remainder of a small weight stays normal in f16
            }
        }
        const uint32_t a0 = FMT == kFmtBf16 ? pack_bf16(hi[0], hi[1]) : pack_f16(hi[0], hi[1]);
        const uint32_t a2 = FMT == kFmtBf16 ? pack_bf16(hi[2], hi[3]) : pack_f16(hi[2], hi[3]);
        const uint32_t a1 = FMT == kFmtBf16 ? pack_bf16(lo[0], lo[1]) : pack_f16(lo[0], lo[1]);
        const uint32_t a3 = FMT == kFmtBf16 ? pack_bf16(lo[2], lo[3]) : pack_f16(lo[2], lo[3]);
#pragma unroll
        for (int hf = 0; hf < kRow / 128; ++hf) {
            uint32_t v[4][4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const uint4 x = lds128(stage + (kTok + 16 * u + 4 * j + y) * kRow + (((8 * hf + r) ^ (j << 1)) << 4));
                v[y][0] = x.x; v[y][1] = x.y; v[y][2] = x.z; v[y][3] = x.w;
            }
            if (rows < kTok) {   // rows that are not the sequence's may hold NaN, which weight 0 would not silence
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    if (16 * u + 4 * j + y >= rows) v[y][0] = v[y][1] = v[y][2] = v[y][3] = 0u;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if constexpr (FMT == kFmtBf16) {
                    const int i = 8 * hf + 2 * c;
                    mma_bf16(st.acc[i], a0, a1, a2, a3, __byte_perm(v[0][c], v[1][c], 0x5410), __byte_perm(v[2][c], v[3][c], 0x5410));
                    mma_bf16(st.acc[i + 1], a0, a1, a2, a3, __byte_perm(v[0][c], v[1][c], 0x7632), __byte_perm(v[2][c], v[3][c], 0x7632));
                } else {
                    uint32_t x0, x1, x2, x3, y0, y1, y2, y3;
                    codes_to_f16<FMT>(__byte_perm(v[0][c], v[1][c], 0x5140), x0, x1);
                    codes_to_f16<FMT>(__byte_perm(v[0][c], v[1][c], 0x7362), x2, x3);
                    codes_to_f16<FMT>(__byte_perm(v[2][c], v[3][c], 0x5140), y0, y1);
                    codes_to_f16<FMT>(__byte_perm(v[2][c], v[3][c], 0x7362), y2, y3);
                    mma_f16(st.acc[4 * c], a0, a1, a2, a3, x0, y0);
                    mma_f16(st.acc[4 * c + 1], a0, a1, a2, a3, x1, y1);
                    mma_f16(st.acc[4 * c + 2], a0, a1, a2, a3, x2, y2);
                    mma_f16(st.acc[4 * c + 3], a0, a1, a2, a3, x3, y3);
                }
            }
        }
    }
}

// The segment's partial, [G] and [G][128]: acc / l in the reference of acc, 2^(m' - m) / l, with the remainder rows folded onto
// the rounded ones
template <int FMT>
__device__ __forceinline__ void state_end(WarpState<FMT>& st, int G, float* lse, float* out, int lane) {
    const int r = lane >> 2, j = lane & 3;
    const float l = quad_sum(st.l);
    const bool some = l > 0.f;
    const float norm = some ? (FMT == kFmtBf16 ? 1.f : fast_ex2(fmaxf(st.mp - st.m, -200.f))) / l : 0.f;
    const float rest = FMT == kFmtBf16 ? 1.f : 1.f / 2048.f;
    if (r >= G) return;
    if (j == 0) lse[r] = some ? st.m + log2f(l) : -INFINITY;
    float* to = out + r * kD;
    constexpr int kRun = FMT == kFmtBf16 ? 8 : 16;   // channels that accumulators i .. i + kRun - 1 hold side by side
#pragma unroll
    for (int i = 0; i < 16; i += 4)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int c = (FMT == kFmtBf16 ? 64 * (i >> 3) : 0) + kRun * (2 * j + x) + (i % kRun);
            float4 v;
            v.x = (st.acc[i][x] + st.acc[i][x + 2] * rest) * norm;
            v.y = (st.acc[i + 1][x] + st.acc[i + 1][x + 2] * rest) * norm;
            v.z = (st.acc[i + 2][x] + st.acc[i + 2][x + 2] * rest) * norm;
            v.w = (st.acc[i + 3][x] + st.acc[i + 3][x + 2] * rest) * norm;
            *reinterpret_cast<float4*>(to + c) = v;
        }
}

template <int FMT>
__global__ void __launch_bounds__(Paged<FMT>::kWarps * 32, kPagedCtasPerSm) paged_attention_kernel(PagedParams p) {
    using P = Paged<FMT>;
    constexpr int kBlockShift = 6 - P::kShift;   // log2 of a block's items
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int s_rows[P::kWarps][P::kStages];
    __shared__ long long s_off[P::kWarps];
    __shared__ int s_b[P::kWarps];
    __shared__ int s_left;
    __shared__ float s_lse[P::kWarps][kMaxGroup];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    pdl_wait();
    auto items_of = [&](int b) { return ceil_shift(paged_len(p.seq_lens, b, p.max_blocks, p.status), P::kShift); };
    const ItemScan<P::kWarps * 32, decltype(items_of)> scan(p.batch, items_of);
    const Shares shares = Shares::of(scan.total * p.Hkv, p.parts, kPagedMinShift - P::kShift);
    const int part0 = blockIdx.x * P::kWarps, part = part0 + warp;
    if (part0 >= shares.parts && blockIdx.x > 0) return;
    if (blockIdx.x == 0) {   // for the merge
        long long before = scan.before;
        for (int b = scan.lo; b < scan.hi; ++b) {
            p.offsets[b] = before;
            before += items_of(b);
        }
        if (scan.lo < scan.hi && scan.hi == p.batch) {
            p.offsets[p.batch] = before;
            *p.shares = shares;
        }
    }
#pragma unroll 1
    for (int w = 0; w < P::kWarps; ++w) {
        int b;
        long long off;
        if (part0 + w < shares.parts && scan.find(shares.begin(part0 + w), p.Hkv, b, off)) {
            s_b[w] = b;
            s_off[w] = off;
            if (w == 0) {   // items of the unit from the CTA's first on
                const int items = items_of(b);
                const long long at = shares.begin(part0) - off;
                s_left = items - (int)(at - quick_div(at, items) * items);
            }
        }
    }
    __syncthreads();
    if (part >= shares.parts) return;
    const long long begin = shares.begin(part);
    const int count = (int)(shares.begin(part + 1) - begin);
    Cursor load;
    load.b = s_b[warp];
    load.n = paged_len(p.seq_lens, load.b, p.max_blocks, p.status);
    load.items = ceil_shift(load.n, P::kShift);
    load.g = (int)quick_div(begin - s_off[warp], load.items);
    load.item = (int)(begin - s_off[warp] - (long long)load.g * load.items);
    Cursor now = load;
    // one partial for the CTA if all its items are of one unit
    const bool whole = part0 + P::kWarps <= shares.parts && shares.begin(part0 + P::kWarps) - shares.begin(part0) <= s_left;
    const uint32_t ring = smem_u32(smem) + warp * P::kStages * P::kStage;
    // pages of the loading cursor's blocks: lane x has block pages_from + x of sequence pages_b
    int pages = 0, pages_b = -1, pages_from = 0;
    int loaded = 0;
    auto issue = [&]() {   // the copies of one item (or none), always one commit group
        if (loaded < count) {
            const int slot = loaded % P::kStages, blk = load.item >> kBlockShift;
            if (load.b != pages_b || blk < pages_from || blk >= pages_from + 32) {
                pages_b = load.b;
                pages_from = blk;
                const long long at = (long long)load.b * p.max_blocks + blk + lane;
                pages = (blk + lane) * kBlk >= load.n ? -1 : p.block_table ? p.block_table[at] : at < p.num_pages ? (int)at : -1;
            }
            const int page = __shfl_sync(kFull, pages, blk - pages_from);
            const bool good = page >= 0 && page < p.num_pages;
            if (!good && lane == 0) atomicOr(p.status, kDevBadPage);
            const int rows = good ? min(P::kTokens, load.n - load.item * P::kTokens) : 0;
            if (lane == 0) s_rows[warp][slot] = rows;
            if (rows > 0) {
                const size_t token0 = ((size_t)page * p.Hkv + load.g) * kBlk + (load.item & ((1 << kBlockShift) - 1)) * P::kTokens;
                const uint32_t stage = ring + slot * P::kStage;
                constexpr int kChunks = P::kRow / 16;                  // 16-byte chunks of a row
                constexpr int kPer = P::kTokens * kChunks / 32;        // ... of the item, per lane
                const unsigned char* k = p.k + token0 * P::kRow + 16 * lane;
                const unsigned char* v = p.v + token0 * P::kRow + 16 * lane;
                const int c = lane % kChunks;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int token = (i * 32 + lane) / kChunks;
                    cp_async16(stage + token * P::kRow + ((c ^ ((token & 1) << 2)) << 4), k + i * 512);
                }
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int token = (i * 32 + lane) / kChunks;
                    cp_async16(stage + (P::kTokens + token) * P::kRow + ((c ^ (((token >> 2) & 3) << 1)) << 4), v + i * 512);
                }
                if constexpr (FMT != kFmtBf16)
                    if (lane < P::kScaleBytes / 8)
                        cp_async16(stage + 2 * P::kTokens * P::kRow + 16 * lane,
                                   (lane < P::kScaleBytes / 16 ? p.k_scale : p.v_scale) + token0 + 4 * (lane % (P::kScaleBytes / 16)));
            }
            ++loaded;
            cursor_next<P::kShift>(load, p);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < P::kStages - 1; ++i) issue();

    WarpState<FMT> st;
    state_begin<FMT>(st, p, now.b, now.g, lane);
    for (int it = 0; it < count; ++it) {
        cp_async_wait<P::kStages - 2>();
        __syncwarp();          // every lane's copies of this item have landed; every lane is done with the slot filled next
        issue();
        const int rows = s_rows[warp][it % P::kStages];
        if (rows > 0) state_item<FMT>(st, ring + (it % P::kStages) * P::kStage, rows, lane);
        const int unit = now.b * p.Hkv + now.g;
        const bool last = now.item + 1 == now.items || it + 1 == count;
        cursor_next<P::kShift>(now, p);
        if (last && !whole) {
            const size_t row = (size_t)paged_slot(unit, part) * p.G;
            state_end<FMT>(st, p.G, p.part_lse + row, p.part_out + row * kD, lane);
            if (it + 1 < count) state_begin<FMT>(st, p, now.b, now.g, lane);
        } else if (last) {   // the warp's only segment: through its ring, in which nothing is in flight any more
            __syncwarp();
            state_end<FMT>(st, p.G, s_lse[warp], reinterpret_cast<float*>(smem + warp * P::kStages * P::kStage), lane);
            __syncthreads();
            const size_t row = (size_t)paged_slot(unit, part0) * p.G;
            for (int h = 0; h < p.G; ++h) {
                float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
                for (int w = 0; w < P::kWarps; ++w) top = fmaxf(top, s_lse[w][h]);
                const float use = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int w = 0; w < P::kWarps; ++w) {
                    const float f = fast_ex2(s_lse[w][h] - use);
                    sum += f;
                    if (f > 0.f) o += f * reinterpret_cast<const float*>(smem + w * P::kStages * P::kStage)[h * kD + threadIdx.x];
                }
                p.part_out[(row + h) * kD + threadIdx.x] = top > -INFINITY ? o / sum : 0.f;
                if (threadIdx.x == 0) p.part_lse[row + h] = top > -INFINITY ? top + log2f(sum) : -INFINITY;
            }
        }
    }
}
static_assert(Paged<kFmtInt8>::kWarps * 32 == kD && Paged<kFmtBf16>::kWarps * 32 == kD, "a thread per channel in the CTA's merge");
static_assert(Paged<kFmtInt8>::kStages * Paged<kFmtInt8>::kStage >= kMaxGroup * kD * 4, "a warp's ring holds its partial");

// ---- merge of the partials --------------------------------------------------------------------------------------------

constexpr int kMergeWarps = 8;

// WARPS warps per (sequence, query head), eight per CTA: weights 2^(lse_i - max), then the weighted mean of the partials; a
// lane has four channels.  Few partials for many heads: one warp each; many: all eight.  The weights of up to 32 WARPS
// partials are found at once, a lane each, while the first channels are already being read.
template <int WARPS>
__global__ void __launch_bounds__(kMergeWarps * 32) merge_partials_kernel(PagedParams p) {
    constexpr int kHeads = kMergeWarps / WARPS, kAhead = 4;
    __shared__ float s_max[kMergeWarps], s_weight[kMergeWarps][32], s_total[kMergeWarps];
    __shared__ float4 s_acc[kMergeWarps][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp % WARPS;
    const long long head = (long long)blockIdx.x * kHeads + warp / WARPS;   // b * Hq + h
    // No early launch of the next call's kernel from here: its CTAs would take their places while these still hold some SMs'
    // shared memory at this kernel's size, and an SM that got fewer of them would stay short for the whole pass (measured on
    // the ragged batch: 217 us a pass without, 303 us with).
    pdl_wait();
    if (WARPS == 1 && head >= (long long)p.batch * p.Hq) return;
    const int b = (int)quick_div(head, p.Hq), h = (int)(head - (long long)b * p.Hq), g = h / p.G, hl = h - g * p.G;
    const long long before = p.offsets[b], mine = p.offsets[b + 1] - before;
    // The unit's parts c0 .. c1.  CTAs whose four parts lie wholly inside the unit, k0 .. k1, left one partial, at their first
    // part's slot: partial i is part c0 + i in front of them, then one in four, then one by one again.
    constexpr int kCta = Paged<kFmtInt8>::kWarps;
    int c0 = 0, own = 0, single = 0x7fffffff, merged = 0;
    if (mine > 0) {
        const Shares shares = *p.shares;
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
    const int n = own + p.prefix_splits;
    const size_t own_row = ((size_t)paged_slot(b * p.Hkv + g, c0)) * p.G + hl;       // part c0 + i: + i * G
    const size_t rows = (size_t)p.batch * p.G;
    const size_t pre_row = (size_t)g * p.prefix_splits * rows + (size_t)b * p.G + hl;  // prefix partial i: + i * rows
    auto row_of = [&](int i) {
        return i < own ? own_row + (size_t)(i + (kCta - 1) * min(max(i - single, 0), merged)) * p.G : pre_row + (size_t)(i - own) * rows;
    };
    auto out_of = [&](int i) {
        return *reinterpret_cast<const float4*>((i < own ? p.part_out : p.prefix_out) + row_of(i) * kD + 4 * lane);
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
        if (high == -INFINITY) continue;             // (nothing so far; uniform over the warp)
        const float scale = fast_ex2(top - high), weight = fast_ex2(lse - high);
        top = high;
        s_weight[warp][lane] = weight;
        __syncwarp();
        sum = sum * scale + weight;                  // this lane's share
        acc.x *= scale; acc.y *= scale; acc.z *= scale; acc.w *= scale;
        auto add = [&](int x, const float4& y) {
            const float f = s_weight[warp][x];
            if (f > 0.f) {   // an empty partial's channels may hold anything
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
        if (w > 0) return;
#pragma unroll
        for (int x = 1; x < WARPS; ++x) top = fmaxf(top, s_max[x]);
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
        sum = 0.f;
        const float use = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
            const float4 y = s_acc[x][lane];
            const float f = fast_ex2(s_max[x] - use);
            sum += f * s_total[x];
            acc.x += f * y.x; acc.y += f * y.y; acc.z += f * y.z; acc.w += f * y.w;
        }
    }
    const float norm = sum > 0.f ? 1.f / sum : 0.f;
    acc.x *= norm; acc.y *= norm; acc.z *= norm; acc.w *= norm;
    const size_t at = (size_t)head * kD + 4 * lane;
    if (p.out_fp32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = acc;
    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at) = make_uint2(pack_bf16(acc.x, acc.y), pack_bf16(acc.z, acc.w));
    if (lane == 0 && p.lse) p.lse[head] = sum > 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

// ---- host side ----------------------------------------------------------------------------------------------------------

// Workspace of the calls in this file: header, partials of the own tokens, partials of the prefix.  A pure function of its
// arguments, so that ffd_workspace_bytes_prefix and the launch agree.
struct PagedPlan {
    int parts, prefix_splits;
    size_t off_offsets, off_shares, off_lse, off_out, off_plse, off_pout, total;
};

static PagedPlan make_paged_plan(const ffd_config* cfg, int batch, int max_blocks, int max_prefix_blocks, int sms) {
    PagedPlan pl;
    const int G = cfg->num_q_heads / cfg->num_kv_heads;
    const long long units = (long long)batch * cfg->num_kv_heads;
    // a warp for every resident slot, but none with fewer than 64 tokens if all sequences are as long as they can be
    const int warps = Paged<kFmtInt8>::kWarps;
    const long long ctas = min((units * max_blocks + warps - 1) / warps, (long long)kPagedCtasPerSm * sms);
    pl.parts = (int)ctas * warps;
    pl.prefix_splits = max_prefix_blocks > 0 ? prefix_splits(batch * G, cfg->num_kv_heads, max_prefix_blocks, sms) : 0;
    const size_t rows = (size_t)(units + pl.parts) * G;
    const size_t prows = (size_t)cfg->num_kv_heads * pl.prefix_splits * batch * G;
    pl.off_offsets = align_up(kInitBytes, 256);
    pl.off_shares = align_up(pl.off_offsets + ((size_t)batch + 1) * sizeof(long long), 256);
    pl.off_lse = pl.off_shares + 256;
    pl.off_out = align_up(pl.off_lse + rows * sizeof(float), 256);
    pl.off_plse = align_up(pl.off_out + rows * kD * sizeof(float), 256);
    pl.off_pout = align_up(pl.off_plse + prows * sizeof(float), 256);
    pl.total = align_up(pl.off_pout + prows * kD * sizeof(float), 256);
    return pl;
}

// the fields of the configuration that the byte cache and the shared prefix use; the others are not looked at
static ffd_status check_paged_config(const ffd_config* cfg) {
    if (!cfg) return FFD_ERR_NULL;
    if (cfg->head_dim != kD || cfg->block_tokens != kBlk) return FFD_ERR_UNSUPPORTED;
    if (cfg->num_q_heads <= 0 || cfg->num_kv_heads <= 0 || cfg->num_q_heads % cfg->num_kv_heads) return FFD_ERR_SHAPE;
    if (cfg->num_q_heads / cfg->num_kv_heads > kMaxGroup) return FFD_ERR_UNSUPPORTED;
    if (cfg->num_q_heads > 65535) return FFD_ERR_SHAPE;
    if (cfg->out_dtype != 0 && cfg->out_dtype != 1) return FFD_ERR_UNSUPPORTED;
    if (!(cfg->sm_scale >= 0.f) || isinf(cfg->sm_scale)) return FFD_ERR_SHAPE;
    return FFD_OK;
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

template <typename... Ps>
static bool any_misaligned(Ps... ptrs) { return (... || (ptrs && misaligned(ptrs))); }

// the merge reads lengths and tables of a call whose own tokens are in `format`
static ffd_status run_paged(int format, PagedParams& p, cudaStream_t s) {
    void (*kernel)(PagedParams) = format == kFmtInt8 ? paged_attention_kernel<kFmtInt8>
                                  : format == kFmtE4m3 ? paged_attention_kernel<kFmtE4m3> : paged_attention_kernel<kFmtBf16>;
    const bool half = format == kFmtBf16;
    const int smem = half ? Paged<kFmtBf16>::kSmem : Paged<kFmtInt8>::kSmem;
    const int warps = Paged<kFmtInt8>::kWarps;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return FFD_ERR_CUDA;
    launch_pdl(kernel, dim3(p.parts / warps), dim3(warps * 32), smem, s, p);
    // partials per head if the lengths are about equal: one warp per head reads a few faster than eight warps can divide them
    const long long heads = (long long)p.batch * p.Hq, expected = p.prefix_splits + p.parts / warps / ((long long)p.batch * p.Hkv) + 2;
    if (expected <= 24) launch_pdl(merge_partials_kernel<1>, dim3((unsigned)((heads + 7) / 8)), dim3(kMergeWarps * 32), 0, s, p);
    else launch_pdl(merge_partials_kernel<8>, dim3((unsigned)heads), dim3(kMergeWarps * 32), 0, s, p);
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
    p.parts = pl.parts;
    p.offsets = reinterpret_cast<long long*>(ws + pl.off_offsets);
    p.shares = reinterpret_cast<Shares*>(ws + pl.off_shares);
    p.prefix_lse = reinterpret_cast<const float*>(ws + pl.off_plse);
    p.prefix_out = reinterpret_cast<const float*>(ws + pl.off_pout);
    p.prefix_splits = pl.prefix_splits;
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
        pp.splits = pl.prefix_splits;
        pp.logit_scale = p.logit_scale;
        pp.out = reinterpret_cast<float*>(ws + pl.off_pout);
        pp.lse = reinterpret_cast<float*>(ws + pl.off_plse);
        pp.status = p.status;
        pp.two_piece = cfg->out_dtype == 1;
        st = launch_prefix(pp, pre.k, pre.v, s);
        if (st) return st;
    }
    return run_paged(own.format, p, s);
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
                  num_pages, 0};
    const int sms = device_sms(), pairs = (p.Hkv + 1) / 2;
    // few rows: a warp for every pair of heads; many: up to eight heads per warp, whose loads overlap
    const bool wide = (long long)num_rows * pairs > 32LL * sms;
    p.chunks = wide ? (pairs + 3) / 4 : pairs;
    const long long warps = (long long)num_rows * p.chunks;
    const unsigned grid = (unsigned)min((warps + kWriteWarps - 1) / kWriteWarps, 8LL * sms);
    void (*kernel)(WriteParams) = format == kFmtInt8 ? (wide ? write_byte_kernel<kFmtInt8, 4> : write_byte_kernel<kFmtInt8, 1>)
                                                     : (wide ? write_byte_kernel<kFmtE4m3, 4> : write_byte_kernel<kFmtE4m3, 1>);
    launch_pdl(kernel, dim3(grid), dim3(kWriteWarps * 32), 0, static_cast<cudaStream_t>(stream), p);
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
    const unsigned grid = (unsigned)min(items, 8LL * device_sms());
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
