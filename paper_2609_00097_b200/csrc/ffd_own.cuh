// Decode attention over the sequences' own pages (byte cache or 16 bits) by teams of four warps, which every kernel that
// needs it calls: the formats' conversions, one warp's work on an item, and a team's on its share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "ffd_paged.cuh"

namespace ffd {

// ---- conversions ------------------------------------------------------------------------------------------------

template <int FMT>
__device__ __forceinline__ constexpr float code_limit() { return FMT == kFmtInt8 ? 127.f : 448.f; }

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

// ---- attention over the sequences' own pages ----------------------------------------------------------------------
//
// A warp works alone on an equal share of all items (kTokens tokens of one sequence and KV head) with mma.sync, the cache being
// the A operand, so that one instruction covers 16 tokens (channels) and its eight columns are four heads in two pieces:
//   S^T = K Q^T : rows = tokens; column 2 h + piece = a piece of head h's query
//   O^T = V^T P^T : rows = channels; column 2 h + piece: P rounded to 16 bits, and what the rounding left, so that P keeps 22
//                   (16) bits at no cost
// NH such tiles of four heads share the cache's fragments.  In a tile, lane 4 r + j holds head j's logits of tokens r and r + 8 of
// 16, whole, since both pieces are its own; its weights, packed as (rounded, remainder), become the B fragment of P by an 8 x 8
// transpose (movmatrix).  The order of the channels inside a contraction, and of O's rows, is permuted so that every
// shared-memory read is 16 bytes of one row.
//
// Byte formats.  K meets the tensor cores as it is stored, with no conversion:
//   e4m3: q, scaled by a power of two per head to below 256, is the sum of two e4m3 numbers (4 bits each of its 8; elements
//         2^-10 below the head's largest lose bits, under 2^-17 of it)
//   int8: q, scaled by a power of two per head to below 2^22 and rounded to an integer, is 2^16 d0 + 2^8 d1 + d2 with digits of
//   -128 .. 127; d2 takes an instruction of its own
// V becomes f16 exactly and the tokens' scales stay outside the products:
//   t = (q . code) * k_scale * logit_scale,   o += 2^(t + log2 v_scale - m') code_v,   l += 2^(t - m)
// with separate running references m' and m: the weights that meet the codes lie in [0, 2^8] whatever the scales are.
// 16-bit format: bf16 products, P in two bf16 pieces, m' = m.
//
// Memory bounds it in short calls, power in a long series of them: the card then lowers its clock until 1000 W are enough, so
// every instruction costs time (heads as rows of A, with twice the products: 218 us for four sequences of 128 K in int8).
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
constexpr int kPagedMinShift = 5;   // log2 of the tokens that a part has at least: a pass of state_item

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
__device__ __forceinline__ float lds_f32(uint32_t addr) {
    float x;
    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(x) : "r"(addr));
    return x;
}
__device__ __forceinline__ float fast_lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}

// over the eight lanes of a head (the rows of a fragment)
__device__ __forceinline__ float rows_max(float x) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(kFull, x, o));
    return x;
}
__device__ __forceinline__ float rows_sum(float x) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) x += __shfl_xor_sync(kFull, x, o);
    return x;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
    return y;
}

// A warp's attention state for one unit.  Lane 4 r + j: as the owner of B fragments column r, that is piece r % 2 of the query
// of head 4 t + r / 2 of the group; as the owner of results head 4 t + j
template <int FMT, int NH>
struct WarpState {
    // B fragments of Q.  bf16: k-steps 2 h, 2 h + 1 at 4 h ..; bytes: register w covers channels 64 (w / 4) + 16 j + 4 (w % 4)
    // .. + 3, int8's d2 at 8 + w
    uint32_t qb[NH][FMT == kFmtE4m3 ? 8 : 16];
    float q_scale[NH];            // logit_scale and what was taken out of q
    float m[NH], mp[NH], l[NH];   // references (log2) of l and of acc; l is this lane's share
    float acc[NH][8][4];          // channel x (see state_end): rounded, remainder; channel x + 1: rounded, remainder
};

template <int FMT, int NH>
__device__ __forceinline__ void state_begin(WarpState<FMT, NH>& st, const PagedParams& p, int b, int g, int lane) {
    const int r = lane >> 2, j = lane & 3, piece = r & 1;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        const int head = 4 * n + (r >> 1);
        const bool in = head < p.G;
        const __nv_bfloat16* q = p.q + ((size_t)b * p.Hq + (size_t)g * p.G + head) * kD;
        if constexpr (FMT == kFmtBf16) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint4 x = make_uint4(0u, 0u, 0u, 0u);
                if (in && piece == 0) x = *reinterpret_cast<const uint4*>(q + 32 * h + 8 * j);
                st.qb[n][4 * h] = x.x; st.qb[n][4 * h + 1] = x.y; st.qb[n][4 * h + 2] = x.z; st.qb[n][4 * h + 3] = x.w;
            }
            st.q_scale[n] = p.logit_scale;
        } else {
            uint32_t raw[16];   // raw[2 w], raw[2 w + 1]: the four channels of register w
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    uint4 x = make_uint4(0u, 0u, 0u, 0u);
                    if (in) x = *reinterpret_cast<const uint4*>(q + 64 * h + 16 * j + 8 * y);
                    uint32_t* to = raw + 8 * h + 4 * y;
                    to[0] = x.x; to[1] = x.y; to[2] = x.z; to[3] = x.w;
                }
            uint32_t top2 = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) top2 = __vmaxu2(top2, raw[i] & 0x7fff7fffu);
            uint32_t top = max(top2 & 0xffffu, top2 >> 16);
            top = max(top, __shfl_xor_sync(kFull, top, 1));
            top = max(top, __shfl_xor_sync(kFull, top, 2));
            // 2^(e - 127) <= largest < 2^(e - 126): scaled by 2^(128 - e), a normal number for every e, it is in [2, 4)
            const int e = min(max((int)(top >> 7), 1), 254);
            const float down = __uint_as_float((uint32_t)(255 - e) << 23), up = __uint_as_float((uint32_t)e << 23);
            if constexpr (FMT == kFmtE4m3) {
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    const float2 a = bf16x2_to_float2(raw[2 * w]), c = bf16x2_to_float2(raw[2 * w + 1]);
                    const float v[4] = {a.x * down * 64.f, a.y * down * 64.f, c.x * down * 64.f, c.y * down * 64.f};
                    const uint32_t hi = floats_to_codes<kFmtE4m3>(v[0], v[1], v[2], v[3]);
                    uint32_t h0, h1;
                    codes_to_f16<kFmtE4m3>(hi, h0, h1);
                    const float2 f0 = f16x2_to_float2(h0), f1 = f16x2_to_float2(h1);
                    const uint32_t lo = floats_to_codes<kFmtE4m3>(v[0] - f0.x, v[1] - f0.y, v[2] - f1.x, v[3] - f1.y);
                    st.qb[n][w] = piece ? lo : hi;
                }
            } else {
                // adding 1.5 * 2^23 = the bits 0x4b400000 rounds to an integer X and leaves it in the low bits.  d2 is its low byte,
                // d1 the next one of X + 2^7, d0 the next one of X + 2^7 + 2^15
                const uint32_t add = (piece ? 0x80u : 0x8080u) - 0x4b400000u, byte = piece ? 0x0051u : 0x0062u;
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    const float2 a = bf16x2_to_float2(raw[2 * w]), c = bf16x2_to_float2(raw[2 * w + 1]);
                    const float x[4] = {a.x, a.y, c.x, c.y};
                    uint32_t v[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) v[y] = __float_as_uint(fmaf(x[y] * down, 1048576.f, 12582912.f));
                    st.qb[n][w] = __byte_perm(__byte_perm(v[0] + add, v[1] + add, byte), __byte_perm(v[2] + add, v[3] + add, byte), 0x5410);
                    st.qb[n][8 + w] = piece ? 0u : __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
                }
            }
            // of head j, from a lane that has its query.  The pieces cannot hold an infinity or a NaN, so that the scale does
            const float back = top >= 0x7f80u ? NAN : up * (FMT == kFmtE4m3 ? 0x1p-7f : 0x1p-5f);   // (d0's unit is 2^(16 - 21))
            st.q_scale[n] = p.logit_scale * __shfl_sync(kFull, back, 8 * j);
        }
        st.m[n] = st.mp[n] = -INFINITY;
        st.l[n] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) st.acc[n][i][0] = st.acc[n][i][1] = st.acc[n][i][2] = st.acc[n][i][3] = 0.f;
    }
}

// An item in a stage of shared memory: the first `rows` (1 .. kTokens) of its tokens are the sequence's
template <int FMT, int NH>
__device__ __forceinline__ void state_item(WarpState<FMT, NH>& st, uint32_t stage, int rows, int lane) {
    using P = Paged<FMT>;
    constexpr int kRow = P::kRow, kTok = P::kTokens, kSets = kTok / 16;   // sets of 16 tokens
    const int r = lane >> 2, j = lane & 3;
    float t[NH][kSets][2];   // q . k of tokens 16 u + r + 8 y, then the logits
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        const uint32_t row = stage + (16 * u + r) * kRow;
        const uint32_t swizzle = (r & 1) << 2;   // odd rows have their chunks XOR 4: eight rows' reads miss each other
        float c[NH][4];
        int ci[NH][4], di[NH][4];
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                c[n][x] = 0.f;
                ci[n][x] = di[n][x] = 0;
            }
#pragma unroll
        for (int h = 0; h < kRow / 64; ++h) {
            const uint32_t at = row + (((4 * h + j) ^ swizzle) << 4);
            const uint4 x = lds128(at), y = lds128(at + 8 * kRow);
#pragma unroll
            for (int n = 0; n < NH; ++n) {
                const uint32_t* qb = st.qb[n] + 4 * h;
                if constexpr (FMT == kFmtBf16) {
                    mma_bf16(c[n], x.x, y.x, x.y, y.y, qb[0], qb[1]);
                    mma_bf16(c[n], x.z, y.z, x.w, y.w, qb[2], qb[3]);
                } else if constexpr (FMT == kFmtE4m3) {
                    mma_e4m3(c[n], x.x, y.x, x.y, y.y, qb[0], qb[1]);
                    mma_e4m3(c[n], x.z, y.z, x.w, y.w, qb[2], qb[3]);
                } else {
                    mma_s8(ci[n], x.x, y.x, x.y, y.y, qb[0], qb[1]);
                    mma_s8(di[n], x.x, y.x, x.y, y.y, qb[8], qb[9]);
                    mma_s8(ci[n], x.z, y.z, x.w, y.w, qb[2], qb[3]);
                    mma_s8(di[n], x.z, y.z, x.w, y.w, qb[10], qb[11]);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y)
                t[n][u][y] = FMT == kFmtInt8 ? (float)ci[n][2 * y] + ((float)ci[n][2 * y + 1] + (float)di[n][2 * y] * 0x1p-8f) * 0x1p-8f
                             : FMT == kFmtE4m3 ? c[n][2 * y] + c[n][2 * y + 1] : c[n][2 * y];
    }
    float tv[NH][kSets][2];   // with log2 of the values' scales
    bool raise = false;
    float top[NH], topv[NH];
#pragma unroll
    for (int n = 0; n < NH; ++n) top[n] = topv[n] = -INFINITY;
#pragma unroll
    for (int u = 0; u < kSets; ++u)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int token = 16 * u + 8 * y + r;
            float ks = 1.f, lv = 0.f;
            if constexpr (FMT != kFmtBf16) {
                ks = lds_f32(stage + 2 * kTok * kRow + 4 * token);
                lv = fast_lg2(lds_f32(stage + 2 * kTok * kRow + P::kScaleBytes + 4 * token));   // a zero row: -inf, weight 0
            }
#pragma unroll
            for (int n = 0; n < NH; ++n) {
                t[n][u][y] *= ks * st.q_scale[n];
                tv[n][u][y] = t[n][u][y] + lv;
                if (rows < kTok && token >= rows) t[n][u][y] = tv[n][u][y] = -INFINITY;   // (the sequence's last item)
                top[n] = fmaxf(top[n], t[n][u][y]);
                if (FMT != kFmtBf16) topv[n] = fmaxf(topv[n], tv[n][u][y]);
            }
        }
#pragma unroll
    for (int n = 0; n < NH; ++n) raise |= top[n] > st.m[n] + kLazyMax || (FMT != kFmtBf16 && topv[n] > st.mp[n] + kLazyMax);
    if (__any_sync(kFull, raise)) {   // always for the first tokens: -inf + 8 is -inf
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const float m = fmaxf(st.m[n], rows_max(top[n]));
            const float use = m == -INFINITY ? 0.f : m;
            float alpha = fast_ex2(st.m[n] - use);
            st.l[n] *= alpha;
            st.m[n] = m;
            if constexpr (FMT != kFmtBf16) {
                const float mp = fmaxf(st.mp[n], rows_max(topv[n]));
                alpha = mp == -INFINITY ? 1.f : fast_ex2(st.mp[n] - mp);
                st.mp[n] = mp;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) st.acc[n][i][x] *= alpha;
        }
    }
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        uint32_t b[NH][2];   // B fragments of P
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const float use = st.m[n] == -INFINITY ? 0.f : st.m[n], usep = st.mp[n] == -INFINITY ? 0.f : st.mp[n];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const float e = fast_ex2(t[n][u][y] - use);
                st.l[n] += e;
                if constexpr (FMT == kFmtBf16) {
                    const float hi = bf16_round(e);
                    b[n][y] = transpose8(pack_bf16(hi, e - hi));
                } else {
                    const float w = fast_ex2(tv[n][u][y] - usep), hi = __half2float(__float2half_rn(w));
                    // the remainder 11 bits further down: that of a small weight stays normal in f16
                    b[n][y] = transpose8(pack_f16(hi, (w - hi) * 2048.f));
                }
            }
        }
#pragma unroll
        for (int hf = 0; hf < kRow / 128; ++hf) {
            uint32_t v[4][4];   // tokens 2 j, 2 j + 1, 2 j + 8, 2 j + 9 of the set
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int token = 16 * u + 2 * j + (y & 1) + 8 * (y >> 1);
                const uint4 x = lds128(stage + (kTok + token) * kRow + (((8 * hf + r) ^ (j << 1)) << 4));
                v[y][0] = x.x; v[y][1] = x.y; v[y][2] = x.z; v[y][3] = x.w;
                if (rows < kTok && token >= rows) v[y][0] = v[y][1] = v[y][2] = v[y][3] = 0u;   // may hold NaN, which weight 0
            }                                                                                    // would not silence
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if constexpr (FMT == kFmtBf16) {
                    const uint32_t a0 = __byte_perm(v[0][c], v[1][c], 0x5410), a1 = __byte_perm(v[0][c], v[1][c], 0x7632);
                    const uint32_t a2 = __byte_perm(v[2][c], v[3][c], 0x5410), a3 = __byte_perm(v[2][c], v[3][c], 0x7632);
#pragma unroll
                    for (int n = 0; n < NH; ++n) mma_bf16(st.acc[n][4 * hf + c], a0, a1, a2, a3, b[n][0], b[n][1]);
                } else {
                    uint32_t x0, x1, x2, x3, y0, y1, y2, y3;
                    codes_to_f16<FMT>(__byte_perm(v[0][c], v[1][c], 0x5140), x0, x1);
                    codes_to_f16<FMT>(__byte_perm(v[0][c], v[1][c], 0x7362), x2, x3);
                    codes_to_f16<FMT>(__byte_perm(v[2][c], v[3][c], 0x5140), y0, y1);
                    codes_to_f16<FMT>(__byte_perm(v[2][c], v[3][c], 0x7362), y2, y3);
#pragma unroll
                    for (int n = 0; n < NH; ++n) {
                        mma_f16(st.acc[n][2 * c], x0, x1, y0, y1, b[n][0], b[n][1]);
                        mma_f16(st.acc[n][2 * c + 1], x2, x3, y2, y3, b[n][0], b[n][1]);
                    }
                }
            }
        }
    }
}

// The segment's partial, [G] and [G][128]: acc / l in the reference of acc, 2^(m' - m) / l, with the remainders added to what was
// rounded.  Lane 4 r + j has head 4 n + j and channels 16 r .. 16 r + 15 (bf16: 8 r .. 8 r + 7 and 64 more), two per accumulator.
template <int FMT, int NH>
__device__ __forceinline__ void state_end(WarpState<FMT, NH>& st, int G, float* lse, float* out, int lane) {
    const int r = lane >> 2, j = lane & 3;
    const float rest = FMT == kFmtBf16 ? 1.f : 1.f / 2048.f;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        const float l = rows_sum(st.l[n]);
        const bool some = l != 0.f;   // (a NaN is handed on)
        const float norm = some ? (FMT == kFmtBf16 ? 1.f : fast_ex2(fmaxf(st.mp[n] - st.m[n], -200.f))) / l : 0.f;
        const int head = 4 * n + j;
        if (head >= G) continue;
        if (r == 0) lse[head] = some ? st.m[n] + log2f(l) : -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const int c = FMT == kFmtBf16 ? 64 * (i >> 2) + 8 * r + 2 * (i & 3) : 16 * r + 2 * i;
            const float(&a)[4] = st.acc[n][i];
            const float(&d)[4] = st.acc[n][i + 1];
            *reinterpret_cast<float4*>(out + head * kD + c) = make_float4((a[0] + a[1] * rest) * norm, (a[2] + a[3] * rest) * norm,
                                                                         (d[0] + d[1] * rest) * norm, (d[2] + d[3] * rest) * norm);
        }
    }
}

// What a team shares besides its rings
struct TeamShared {
    int rows[4][2];
    float lse[4][kMaxGroup];
};

// A team of four warps: its warps take parts 4 team .. 4 team + 3.  smem: Paged<FMT>::kSmem bytes of the team's own, 16-byte
// aligned; thread: 0 .. 127; sync: a barrier of the team's threads.  most_parts: of all teams; chunks: partial results of the
// prefix, for the merge.
template <int FMT, int NH, typename Sync>
__device__ __forceinline__ void attend_own(const PagedParams& p, int most_parts, int chunks, unsigned char* smem, TeamShared& sh,
                                           int team, int thread, Sync sync) {
    using P = Paged<FMT>;
    constexpr int kBlockShift = 6 - P::kShift;   // log2 of a block's items
    const int warp = __shfl_sync(kFull, thread >> 5, 0), lane = thread & 31;
    auto items_of = [&](int b) { return ceil_shift(paged_len(p.seq_lens, b, p.max_blocks, p.status), P::kShift); };
    const WarpScan<decltype(items_of)> scan(p.batch, items_of, lane);
    const Shares shares = Shares::of(scan.total * p.Hkv, most_parts, kPagedMinShift - P::kShift, chunks);
    const int part0 = team * P::kWarps, part = part0 + warp;
    if (team == 0 && warp == 0) {   // for the merge
        long long before = scan.before;
        for (int b = scan.lo; b < scan.hi; ++b) {
            p.offsets[b] = before;
            before += items_of(b);
        }
        if (lane == 0) {
            p.offsets[p.batch] = scan.total;
            *p.shares = shares;
        }
    }
    if (part >= shares.parts) return;
    const long long begin = shares.begin(part);
    const int count = (int)(shares.begin(part + 1) - begin);
    Cursor load;
    long long off;
    scan.find(begin, p.Hkv, load.b, off);
    load.n = paged_len(p.seq_lens, load.b, p.max_blocks, p.status);
    load.items = ceil_shift(load.n, P::kShift);
    load.g = (int)quick_div(begin - off, load.items);
    off += (long long)load.g * load.items;   // the unit's first item
    load.item = (int)(begin - off);
    Cursor now = load;
    // one partial for the CTA if all its items are of one unit
    const bool whole = part0 + P::kWarps <= shares.parts && shares.begin(part0) >= off &&
                       shares.begin(part0 + P::kWarps) <= off + load.items;
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
                pages = blk + lane >= blocks_of(load.n) ? -1 : p.block_table ? p.block_table[at] : at < p.num_pages ? (int)at : -1;
            }
            const int page = __shfl_sync(kFull, pages, blk - pages_from);
            const bool good = page >= 0 && page < p.num_pages;
            if (!good && lane == 0) atomicOr(p.status, kDevBadPage);
            const int rows = good ? min(P::kTokens, load.n - load.item * P::kTokens) : 0;
            if (lane == 0) sh.rows[warp][slot] = rows;
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
                    cp_async16(stage + (P::kTokens + token) * P::kRow + ((c ^ (((token >> 1) & 3) << 1)) << 4), v + i * 512);
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

    WarpState<FMT, NH> st;
    state_begin<FMT, NH>(st, p, now.b, now.g, lane);   // while the first item is on its way
    bool fresh = false;
    for (int it = 0; it < count; ++it) {
        cp_async_wait<P::kStages - 2>();
        __syncwarp();          // every lane's copies of this item have landed; every lane is done with the slot filled next
        issue();
        if (fresh) state_begin<FMT, NH>(st, p, now.b, now.g, lane);
        fresh = false;
        const int rows = sh.rows[warp][it % P::kStages];
        if (rows > 0) state_item<FMT, NH>(st, ring + (it % P::kStages) * P::kStage, rows, lane);
        const int unit = now.b * p.Hkv + now.g;
        const bool last = now.item + 1 == now.items || it + 1 == count;
        cursor_next<P::kShift>(now, p);
        if (last && !whole) {
            const size_t row = (size_t)paged_slot(unit, part) * p.G;
            state_end<FMT, NH>(st, p.G, p.part_lse + row, p.part_out + row * kD, lane);
            fresh = true;
        } else if (last) {   // the warp's only segment: through its ring, in which nothing is in flight any more
            __syncwarp();
            state_end<FMT, NH>(st, p.G, sh.lse[warp], reinterpret_cast<float*>(smem + warp * P::kStages * P::kStage), lane);
            sync();
            const size_t row = (size_t)paged_slot(unit, part0) * p.G;
            for (int h = warp; h < p.G; h += P::kWarps) {   // a warp for a head, a lane for four channels
                float top = -INFINITY, sum = 0.f;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < P::kWarps; ++w) top = fmaxf(top, sh.lse[w][h]);
                const float use = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int w = 0; w < P::kWarps; ++w) {
                    const float f = fast_ex2(sh.lse[w][h] - use);
                    const float4 x = reinterpret_cast<const float4*>(smem + w * P::kStages * P::kStage)[h * (kD / 4) + lane];
                    sum += f;
                    if (f != 0.f) { o.x += f * x.x; o.y += f * x.y; o.z += f * x.z; o.w += f * x.w; }
                }
                const float norm = sum != 0.f ? 1.f / sum : 0.f;
                reinterpret_cast<float4*>(p.part_out + (row + h) * kD)[lane] = make_float4(o.x * norm, o.y * norm, o.z * norm, o.w * norm);
                if (lane == 0) p.part_lse[row + h] = sum != 0.f ? use + log2f(sum) : -INFINITY;
            }
        }
    }
}
static_assert(Paged<kFmtInt8>::kStages * Paged<kFmtInt8>::kStage >= kMaxGroup * kD * 4, "a warp's ring holds its partial");

}  // namespace ffd
