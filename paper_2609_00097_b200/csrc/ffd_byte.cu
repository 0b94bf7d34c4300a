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
    const Share s = find_share<kReadThreads>(p.batch, p.Hkv, blockIdx.x, gridDim.x, count);
    if (s.begin >= s.end) return;
    int b = s.b;
    long long off = s.off;
    int n = paged_len(p.seq_lens, b, p.max_blocks, p.status), first = first_of(b);
    long long items = (long long)count(b) * p.Hkv;
    for (long long x = s.begin; x < s.end; ++x) {
        while (x >= off + items) {   // ends: x < s.end <= the total of all sequences
            off += items;
            ++b;
            n = paged_len(p.seq_lens, b, p.max_blocks, p.status);
            first = first_of(b);
            items = (long long)count(b) * p.Hkv;
        }
        const int blk = (first >> 6) + (int)((x - off) / p.Hkv), g = (int)((x - off) % p.Hkv);
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
// One warp works on 16 tokens at a time with mma.sync m16n8k16:
//   S = Q K^T : rows = query heads (8..15 zero), columns = tokens, two 8-token tiles
//   O = P V   : rows 0..7 = P rounded to 16 bits, rows 8..15 = what the rounding left, so that P keeps 22 (16) bits at no cost
// Token 4 j + 2 i + x of a group of 16 sits in tile i, column 2 j + x: the lane that holds S for columns 2 j, 2 j + 1 holds it
// for tokens 4 j .. 4 j + 3, whose scales are one 16-byte read, and the accumulator fragment of S is the A fragment of P.
// The order of the channels inside a contraction is permuted so that every shared-memory read is 16 bytes of one row.
//
// Byte formats.  Codes become f16 exactly, q is scaled by a power of two per head to below 2 (its 8 bits fit; elements
// 2^-14 below the head's largest lose bits only under 2^-25 of it), and the token's scales stay outside the products:
//   t = (q . code) * k_scale * logit_scale,   o += 2^(t + log2 v_scale - m') code_v,   l += 2^(t - m)
// with separate running references m' and m: the weights that meet the codes lie in [0, 2^8] whatever the scales are.
// 16-bit format: bf16 products, P in two bf16 pieces, m' = m.
//
// A CTA has four warps and takes an equal share of all (sequence, KV head, block) items; warp w has tokens 16 w .. 16 w + 15
// of each block.  Each warp keeps kStages - 1 groups in flight with cp.async into its own ring of shared memory, across the
// ends of sequences, so the copies never wait for the merge at the end of a segment.

template <int FMT>
struct Paged {
    static constexpr int kWarps = 4;
    static constexpr int kRow = FMT == kFmtBf16 ? 2 * kD : kD;                 // bytes of a token's key
    static constexpr int kScaleBytes = FMT == kFmtBf16 ? 0 : 16 * 4;
    static constexpr int kStage = 2 * 16 * kRow + 2 * kScaleBytes;
    static constexpr int kStages = FMT == kFmtBf16 ? 3 : 4;
    static constexpr int kCtasPerSm = FMT == kFmtBf16 ? 2 : 3;
    static constexpr int kMergeHeads = 4;                                      // heads merged at a time
    static constexpr int kMergeBytes = kWarps * kMergeHeads * kD * 4;
    static constexpr int kSmem = kWarps * kStages * kStage + kMergeBytes;
};

constexpr float kLazyMax = 8.f;   // a reference is raised when a logit exceeds it by this many powers of two

// place in the flattened list
struct Cursor {
    int b, g, blk, n, nblk;
};

__device__ __forceinline__ void cursor_next(Cursor& c, const PagedParams& p) {
    if (++c.blk < c.nblk) return;
    c.blk = 0;
    if (++c.g < p.Hkv) return;
    c.g = 0;
    do {
        if (++c.b >= p.batch) {   // behind the last item: never used
            c.n = c.nblk = 0;
            return;
        }
        c.n = paged_len(p.seq_lens, c.b, p.max_blocks, p.status);
        c.nblk = blocks_of(c.n);
    } while (c.nblk == 0);
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

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
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
    uint32_t qa[16];     // A fragments of Q, rows 0..7
    float q_scale;       // logit_scale and the power of two that was taken out of q
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
        uint32_t raw[16];
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
        const int e = min(max((int)(top >> 7), 1), 253);                    // biased exponent of the largest element
        const float down = __uint_as_float((uint32_t)(254 - e) << 23);      // 2^(127 - e)
        const float up = __uint_as_float((uint32_t)e << 23);                // 2^(e - 127)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 x = bf16x2_to_float2(raw[i]);
            st.qa[i] = pack_f16(x.x * down, x.y * down);
        }
        st.q_scale = p.logit_scale * up;
    }
    st.m = st.mp = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) st.acc[i][0] = st.acc[i][1] = st.acc[i][2] = st.acc[i][3] = 0.f;
}

// 16 tokens, of which the first `rows` (1..16) are the sequence's, in a stage of shared memory
template <int FMT>
__device__ __forceinline__ void state_group(WarpState<FMT>& st, uint32_t stage, int rows, int lane) {
    constexpr int kRow = Paged<FMT>::kRow;
    const int r = lane >> 2, j = lane & 3;
    float s[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float c0 = 0.f, c1 = 0.f;
        const uint32_t row = stage + (4 * (r >> 1) + 2 * i + (r & 1)) * kRow;
        const uint32_t swizzle = (r & 1) << 2;   // odd rows have their chunks XOR 4: eight rows' reads miss each other
#pragma unroll
        for (int h = 0; h < kRow / 64; ++h) {
            const uint4 x = lds128(row + (((4 * h + j) ^ swizzle) << 4));
            if constexpr (FMT == kFmtBf16) {
                mma_bf16_top(c0, c1, st.qa[4 * h], st.qa[4 * h + 1], x.x, x.y);
                mma_bf16_top(c0, c1, st.qa[4 * h + 2], st.qa[4 * h + 3], x.z, x.w);
            } else {
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    uint32_t b0, b1;
                    codes_to_f16<FMT>(w[y], b0, b1);
                    mma_f16_top(c0, c1, st.qa[8 * h + 2 * y], st.qa[8 * h + 2 * y + 1], b0, b1);
                }
            }
        }
        s[i][0] = c0;
        s[i][1] = c1;
    }
    // logits of tokens 4 j .. 4 j + 3, and with log2 of the values' scales
    float t[4], tv[4];
    float ks[4] = {1.f, 1.f, 1.f, 1.f}, lv[4] = {0.f, 0.f, 0.f, 0.f};
    if constexpr (FMT != kFmtBf16) {
        const uint4 a = lds128(stage + 32 * kRow + 16 * j), b = lds128(stage + 32 * kRow + 64 + 16 * j);
        const uint32_t au[4] = {a.x, a.y, a.z, a.w}, bu[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            ks[y] = __uint_as_float(au[y]);
            lv[y] = __log2f(__uint_as_float(bu[y]));   // a zero row: -inf, weight 0
        }
    }
    float top = -INFINITY, topv = -INFINITY;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const bool in = 4 * j + y < rows;
        t[y] = in ? s[y >> 1][y & 1] * (ks[y] * st.q_scale) : -INFINITY;
        tv[y] = in ? t[y] + lv[y] : -INFINITY;
        top = fmaxf(top, t[y]);
        topv = fmaxf(topv, tv[y]);
    }
    const bool raise = FMT == kFmtBf16 ? top > st.m + kLazyMax : top > st.m + kLazyMax || topv > st.mp + kLazyMax;
    if (__any_sync(kFull, raise)) {   // always for the first tokens: -inf + 8 is -inf
        const float m = fmaxf(st.m, quad_max(top));
        const float use = m == -INFINITY ? 0.f : m;
        st.l *= exp2f(st.m - use);
        float alpha;
        if constexpr (FMT == kFmtBf16) {
            alpha = exp2f(st.m - use);
            st.mp = m;
        } else {
            const float mp = fmaxf(st.mp, quad_max(topv));
            alpha = mp == -INFINITY ? 1.f : exp2f(st.mp - mp);
            st.mp = mp;
        }
        st.m = m;
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) st.acc[i][x] *= alpha;
    }
    const float use = st.m == -INFINITY ? 0.f : st.m, usep = st.mp == -INFINITY ? 0.f : st.mp;
    float hi[4], lo[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const float e = exp2f(t[y] - use);
        st.l += e;
        if constexpr (FMT == kFmtBf16) {
            hi[y] = bf16_round(e);
            lo[y] = e - hi[y];
        } else {
            const float w = exp2f(tv[y] - usep);
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
            const uint4 x = lds128(stage + 16 * kRow + (4 * j + y) * kRow + (((8 * hf + r) ^ (j << 1)) << 4));
            v[y][0] = x.x; v[y][1] = x.y; v[y][2] = x.z; v[y][3] = x.w;
        }
        if (rows < 16) {   // rows that are not the sequence's may hold NaN, which weight 0 would not silence
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (4 * j + y >= rows) v[y][0] = v[y][1] = v[y][2] = v[y][3] = 0u;
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

// channel of accumulator (i, x), x = 0, 1, in lane (r, j)
template <int FMT>
__device__ __forceinline__ int paged_channel(int i, int x, int j) {
    return FMT == kFmtBf16 ? 64 * (i >> 3) + 8 * (2 * j + x) + (i & 7) : 16 * (2 * j + x) + i;
}

__device__ __forceinline__ void store_out(const PagedParams& p, size_t at, float x) {
    if (p.out_fp32) static_cast<float*>(p.out)[at] = x;
    else static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(x);
}

template <int FMT>
__global__ void __launch_bounds__(Paged<FMT>::kWarps * 32, Paged<FMT>::kCtasPerSm) paged_attention_kernel(PagedParams p) {
    using P = Paged<FMT>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float s_lse[P::kWarps][kMaxGroup];
    __shared__ int s_rows[P::kWarps][P::kStages];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, j = lane & 3;
    pdl_launch_dependents();
    pdl_wait();
    const Share share = find_share<P::kWarps * 32>(p.batch, p.Hkv, blockIdx.x, p.parts,
                                                   [&](int b) { return blocks_of(paged_len(p.seq_lens, b, p.max_blocks, p.status)); });
    const long long count = share.end - share.begin;
    if (count <= 0) return;
    Cursor load;
    load.b = share.b;
    load.n = paged_len(p.seq_lens, load.b, p.max_blocks, p.status);
    load.nblk = blocks_of(load.n);
    load.g = (int)((share.begin - share.off) / load.nblk);
    load.blk = (int)((share.begin - share.off) % load.nblk);
    Cursor now = load;

    const uint32_t ring = smem_u32(smem) + warp * P::kStages * P::kStage;
    float* merge = reinterpret_cast<float*>(smem + P::kWarps * P::kStages * P::kStage);
    // pages of the loading cursor's blocks: lane x has block pages_from + x of sequence pages_b
    int pages = 0, pages_b = -1, pages_from = 0;
    long long loaded = 0;
    auto issue = [&]() {   // the copies of one group (or none), always one commit group
        if (loaded < count) {
            const int slot = (int)(loaded % P::kStages);
            if (load.b != pages_b || load.blk < pages_from || load.blk >= pages_from + 32) {
                pages_b = load.b;
                pages_from = load.blk;
                const int blk = load.blk + lane;
                const long long at = (long long)load.b * p.max_blocks + blk;
                pages = blk >= load.nblk ? -1 : p.block_table ? p.block_table[at] : at < p.num_pages ? (int)at : -1;
            }
            const int page = __shfl_sync(kFull, pages, load.blk - pages_from);
            const bool good = page >= 0 && page < p.num_pages;
            if (!good && tid == 0) atomicOr(p.status, kDevBadPage);
            const int rows = good ? min(16, load.n - load.blk * kBlk - 16 * warp) : 0;
            if (lane == 0) s_rows[warp][slot] = rows;
            if (rows > 0) {
                const size_t token0 = ((size_t)page * p.Hkv + load.g) * kBlk + 16 * warp;
                const uint32_t stage = ring + slot * P::kStage;
                constexpr int kChunks = P::kRow / 16;      // 16-byte chunks of a row
                constexpr int kPer = 16 * kChunks / 32;    // ... of the group, per lane
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int token = (i * 32 + lane) / kChunks, c = (i * 32 + lane) % kChunks;
                    cp_async16(stage + token * P::kRow + ((c ^ ((token & 1) << 2)) << 4), p.k + (token0 + token) * P::kRow + 16 * c);
                }
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int token = (i * 32 + lane) / kChunks, c = (i * 32 + lane) % kChunks;
                    cp_async16(stage + (16 + token) * P::kRow + ((c ^ (((token >> 2) & 3) << 1)) << 4),
                               p.v + (token0 + token) * P::kRow + 16 * c);
                }
                if (FMT != kFmtBf16 && lane < 8)
                    cp_async16(stage + 32 * P::kRow + 16 * lane, (lane < 4 ? p.k_scale : p.v_scale) + token0 + 4 * (lane & 3));
            }
            ++loaded;
            cursor_next(load, p);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < P::kStages - 1; ++i) issue();

    WarpState<FMT> st;
    state_begin<FMT>(st, p, now.b, now.g, lane);
    for (long long it = 0; it < count; ++it) {
        cp_async_wait<P::kStages - 2>();
        __syncwarp();          // every lane's copies of this group have landed; every lane is done with the slot filled next
        issue();
        const int slot = (int)(it % P::kStages);
        const int rows = s_rows[warp][slot];
        if (rows > 0) state_group<FMT>(st, ring + slot * P::kStage, rows, lane);
        const int b = now.b, g = now.g;
        const bool last = now.blk + 1 == now.nblk || it + 1 == count;
        cursor_next(now, p);
        if (!last) continue;

        // the segment ends: the four warps' results become one partial
        const float l = quad_sum(st.l);
        const bool some = l > 0.f;
        // acc / l in the reference of acc: 2^(m' - m) / l, and the remainder rows folded onto the rounded ones
        const float norm = some ? (FMT == kFmtBf16 ? 1.f : exp2f(fmaxf(st.mp - st.m, -200.f))) / l : 0.f;
        const float rest = FMT == kFmtBf16 ? 1.f : 1.f / 2048.f;
        if (j == 0) s_lse[warp][r] = some ? st.m + log2f(l) : -INFINITY;
        const int unit = b * p.Hkv + g;
        const size_t slot_row = (size_t)paged_slot(unit, blockIdx.x) * p.G;
        for (int h0 = 0; h0 < p.G; h0 += P::kMergeHeads) {
            if (r >= h0 && r < h0 + P::kMergeHeads) {
                float* to = merge + ((size_t)warp * P::kMergeHeads + (r - h0)) * kD;
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        to[paged_channel<FMT>(i, x, j)] = (st.acc[i][x] + st.acc[i][x + 2] * rest) * norm;
            }
            __syncthreads();
            const int heads = min(P::kMergeHeads, p.G - h0);
            for (int h = 0; h < heads; ++h) {
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < P::kWarps; ++w) top = fmaxf(top, s_lse[w][h0 + h]);
                float sum = 0.f, o = 0.f;
                if (top > -INFINITY) {
#pragma unroll
                    for (int w = 0; w < P::kWarps; ++w) {
                        const float f = exp2f(s_lse[w][h0 + h] - top);
                        if (f > 0.f) {
                            sum += f;
                            o += f * merge[((size_t)w * P::kMergeHeads + h) * kD + tid];
                        }
                    }
                    o /= sum;
                }
                p.part_out[(slot_row + h0 + h) * kD + tid] = o;
                if (tid == 0) p.part_lse[slot_row + h0 + h] = top > -INFINITY ? top + log2f(sum) : -INFINITY;
            }
            __syncthreads();   // the merge buffer (and s_lse, after the last round) may be written again
        }
        if (it + 1 < count) state_begin<FMT>(st, p, now.b, now.g, lane);
    }
}

// ---- merge of the partials --------------------------------------------------------------------------------------------

constexpr int kMergeThreads = 256;

// One CTA per (sequence, query head): weights 2^(lse_i - max), then the weighted mean of the partials; warp w takes partials
// w, w + 8, ..., a lane four channels.
__global__ void __launch_bounds__(kMergeThreads) merge_partials_kernel(PagedParams p) {
    constexpr int kWarpsM = kMergeThreads / 32;
    __shared__ long long s_sum[2][kWarpsM];
    __shared__ float s_max[kWarpsM], s_total[kWarpsM];
    __shared__ float4 s_acc[kWarpsM][32];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    pdl_wait();
    long long all = 0, before = 0;
    for (int x = tid; x < p.batch; x += kMergeThreads) {
        const int nb = blocks_of(min(max(p.seq_lens[x], 0), p.max_blocks * kBlk));
        all += nb;
        if (x < b) before += nb;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        all += __shfl_xor_sync(kFull, all, o);
        before += __shfl_xor_sync(kFull, before, o);
    }
    if (lane == 0) { s_sum[0][warp] = all; s_sum[1][warp] = before; }
    __syncthreads();
    all = before = 0;
#pragma unroll
    for (int w = 0; w < kWarpsM; ++w) { all += s_sum[0][w]; before += s_sum[1][w]; }
    const int g = h / p.G, hl = h % p.G;
    const int mine = blocks_of(min(max(p.seq_lens[b], 0), p.max_blocks * kBlk));
    const long long total = all * p.Hkv, off = before * p.Hkv + (long long)g * mine;
    int c0 = 0, own = 0;
    if (mine > 0) {
        c0 = part_of(off, total, p.parts);
        own = part_of(off + mine - 1, total, p.parts) - c0 + 1;
    }
    const int n = own + p.prefix_splits;
    const size_t own_row = ((size_t)paged_slot(b * p.Hkv + g, c0)) * p.G + hl;       // partial i < own: + i * G
    const size_t rows = (size_t)p.batch * p.G;
    const size_t pre_row = (size_t)g * p.prefix_splits * rows + (size_t)b * p.G + hl;  // prefix partial i: + i * rows
    auto lse_of = [&](int i) { return i < own ? p.part_lse[own_row + (size_t)i * p.G] : p.prefix_lse[pre_row + (size_t)(i - own) * rows]; };
    float top = -INFINITY;
    for (int i = tid; i < n; i += kMergeThreads) top = fmaxf(top, lse_of(i));
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
    if (lane == 0) s_max[warp] = top;
    __syncthreads();
    top = s_max[0];
#pragma unroll
    for (int w = 1; w < kWarpsM; ++w) top = fmaxf(top, s_max[w]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    if (top > -INFINITY) {
#pragma unroll 4
        for (int i = warp; i < n; i += kWarpsM) {
            const float f = exp2f(lse_of(i) - top);
            const float* from = i < own ? p.part_out + (own_row + (size_t)i * p.G) * kD : p.prefix_out + (pre_row + (size_t)(i - own) * rows) * kD;
            if (f > 0.f) {   // an empty partial's channels may hold anything
                const float4 x = *reinterpret_cast<const float4*>(from + 4 * lane);
                sum += f;
                acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
            }
        }
    }
    s_acc[warp][lane] = acc;
    if (lane == 0) s_total[warp] = sum;
    __syncthreads();
    if (tid < kD) {
        float total_w = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarpsM; ++w) {
            total_w += s_total[w];
            o += reinterpret_cast<const float*>(&s_acc[w][0])[tid];
        }
        const size_t head = (size_t)b * p.Hq + h;
        store_out(p, head * kD + tid, total_w > 0.f ? o / total_w : 0.f);
        if (tid == 0 && p.lse) p.lse[head] = total_w > 0.f ? (top + log2f(total_w)) * kLn2 : -INFINITY;
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------

// Workspace of the calls in this file: header, partials of the own tokens, partials of the prefix.  A pure function of its
// arguments, so that ffd_workspace_bytes_prefix and the launch agree.
struct PagedPlan {
    int parts, prefix_splits;
    size_t off_lse, off_out, off_plse, off_pout, total;
};

static PagedPlan make_paged_plan(const ffd_config* cfg, int format, int batch, int max_blocks, int max_prefix_blocks, int sms) {
    PagedPlan pl;
    const int G = cfg->num_q_heads / cfg->num_kv_heads;
    const long long units = (long long)batch * cfg->num_kv_heads, items = units * max_blocks;
    // one CTA per resident slot; the byte formats have more of them, so a workspace of theirs serves all
    const int per_sm = format == kFmtBf16 ? Paged<kFmtBf16>::kCtasPerSm : Paged<kFmtInt8>::kCtasPerSm;
    pl.parts = (int)min(items, (long long)per_sm * sms);
    pl.prefix_splits = max_prefix_blocks > 0 ? prefix_splits(batch * G, cfg->num_kv_heads, max_prefix_blocks, sms) : 0;
    const size_t rows = (size_t)(units + pl.parts) * G;
    const size_t prows = (size_t)cfg->num_kv_heads * pl.prefix_splits * batch * G;
    pl.off_lse = align_up(kInitBytes, 256);
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
    const size_t smem = format == kFmtBf16 ? Paged<kFmtBf16>::kSmem : Paged<kFmtInt8>::kSmem;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return FFD_ERR_CUDA;
    launch_pdl(kernel, dim3(p.parts), dim3(Paged<kFmtInt8>::kWarps * 32), smem, s, p);
    launch_pdl(merge_partials_kernel, dim3(p.Hq, p.batch), dim3(kMergeThreads), 0, s, p);
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
    const PagedPlan pl = make_paged_plan(cfg, own.format, own.batch, own.max_blocks, pre.max_blocks, sms);
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
    *bytes = make_paged_plan(cfg, kFmtInt8, batch, max_blocks_per_seq, max_prefix_blocks, device_sms()).total;
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
