// Norm and rotation of new tokens' queries and keys, and their way into the 16-bit pages, in one pass.
//
// A warp has a token and some of its heads, two at a time: 16 lanes of 8 channels each (16 bytes) for a head, so that loads and
// stores are whole 256-byte rows.  The cosines and sines of a lane's channels are loaded once for all its heads.  Elements of a
// pair are in the same lane if pairs are neighbours, and otherwise rotary_dim / 16 lanes apart: one exchange of the normalised
// values.  The mean of the squares is a sum over 16 lanes.
//
// Where there are many tokens, each row read once and written once, the bytes are the bound and the issue of instructions is not far
// behind it (eight ragged prompts, 33 K tokens of 48 heads, 810 MB: 158 to 165 us, 0.75 to 0.78 of the measured copy bandwidth, 154 on
// one state; 71 % of the issue slots).  Where there are few, latency: then a warp has two heads only (one token for 16 sequences: 4.4 us).  Weights and
// cosines multiplied once for a token, with the exchange in bf16, are a third fewer instructions, but the first head then waits for
// both: 165 to 185 us where this form took 153.  Several tokens per warp: 180.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "ffd_chunk.cuh"
#include "ffd_host.cuh"

namespace ffd {

constexpr uint32_t kDevBadPosition = FFD_DEV_BAD_POSITION;
constexpr int kRotWarps = 4;

struct RotateParams {
    ChunkRows r;
    const __nv_bfloat16 *q, *k, *v;
    long long q_stride, kv_stride;
    const int32_t* positions;
    const float* cos_sin;
    const __nv_bfloat16 *q_norm, *k_norm;
    __nv_bfloat16 *q_out, *k_cache, *v_cache;
    int Hq, Hkv, num_positions, half;      // half: rotary_dim / 2
    float eps;
    int slices, pairs;                     // warps per token, head pairs of each
};

__device__ __forceinline__ void unpack8(const uint4& x, float (&f)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// The last sequence before b that has new tokens; -1: none.  (Sequences without any may begin inside another one's rows.)
__device__ __noinline__ int sequence_with_rows(const ChunkRows& r, int b, int lane) {
    while (b > 0) {
        const int at = b - 1 - lane;
        const unsigned some = __ballot_sync(kFull, at >= 0 && chunk_seq(r, at).n > 0);
        if (some) return b - __ffs(some);
        b -= 32;
    }
    return -1;
}

// Rows that do not exist are nobody's when their sequences are looked for: so the first CTAs look at every sequence's numbers, for
// bad ones to be reported.  (In all CTAs, and not in a function of its own: 33 K rows of prompts took 2 us longer.)
constexpr unsigned kLookCtas = 64;
__device__ __noinline__ void look_over(const ChunkRows& r) {
    const int step = (int)min(gridDim.x, kLookCtas) * kRotWarps * 32;
    for (int b = (int)blockIdx.x * kRotWarps * 32 + threadIdx.x; b < r.batch; b += step) chunk_seq(r, b);
}

// Heads of a token are numbered queries, keys, values; a warp's slice is `pairs` pairs of neighbouring numbers.
template <bool INTERLEAVED>
__global__ void __launch_bounds__(kRotWarps * 32, 6) rotate_write_kernel(const __grid_constant__ RotateParams p) {
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, s = lane & 15, side = lane >> 4;
    const long long unit = (long long)blockIdx.x * kRotWarps + (threadIdx.x >> 5);
    const int row = (int)(unit / p.slices), slice = (int)(unit - (long long)row * p.slices);
    const bool looks = p.r.row_start && blockIdx.x < kLookCtas;
    if (row >= p.r.num_rows && !looks) return;
    const int heads = p.Hq + 2 * p.Hkv, first = 2 * slice * p.pairs, last = min(heads, first + 2 * p.pairs);
    auto source = [&](int head) {
        if (head < p.Hq) return p.q + row * p.q_stride + (size_t)head * kD + 8 * s;
        if (head < p.Hq + p.Hkv) return p.k + row * p.kv_stride + (size_t)(head - p.Hq) * kD + 8 * s;
        return p.v + row * p.kv_stride + (size_t)(head - p.Hq - p.Hkv) * kD + 8 * s;
    };
    constexpr int kAhead = 3;      // pairs whose rows are on their way at once
    uint4 next[kAhead];
    auto fetch = [&](int from) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int head = from + 2 * i + side;
            next[i] = make_uint4(0u, 0u, 0u, 0u);
            if (head < last) next[i] = ldg_stream(reinterpret_cast<const uint4*>(source(head)));
        }
    };
    pdl_wait();
    if (looks) {
        look_over(p.r);
        if (row >= p.r.num_rows) return;
    }
    fetch(first);                  // before it is known whose row it is
    int b = row, token;
    if (p.r.row_start) {
        b = sequence_of_row(p.r.row_start, p.r.batch, row, lane);
        if (b < 0) return;
        ChunkSeq c = chunk_seq(p.r, b);
        if (c.n == 0) {
            b = sequence_with_rows(p.r, b, lane);
            if (b < 0) return;
            c = chunk_seq(p.r, b);
        }
        if (row - c.row0 >= c.n) return;
        token = c.first + row - c.row0;
    } else {
        token = paged_len(p.r.seq_lens, b, p.r.max_blocks, p.r.status) - 1;
        if (token < 0) return;
    }
    const int page = chunk_page(p.r, b, token >> 6);
    if (page < 0 && lane == 0) atomicOr(p.r.status, kDevBadPage);
    const int rotary_lanes = p.half >> 2;       // lanes with channels that turn: rotary_dim / 8
    const bool turns = s < rotary_lanes;
    float cs[8], sn[8];
    if (p.half) {
        const int position = p.positions ? p.positions[row] : token;
        if (position < 0 || position >= p.num_positions) {
            if (lane == 0) atomicOr(p.r.status, kDevBadPosition);
            return;
        }
        if (turns) {
            const float* t = p.cos_sin + (size_t)position * 2 * p.half;
            if (INTERLEAVED) {      // pairs 4 s .. 4 s + 3
                const float4 c = *reinterpret_cast<const float4*>(t + 4 * s), d = *reinterpret_cast<const float4*>(t + p.half + 4 * s);
                const float cc[4] = {c.x, c.y, c.z, c.w}, dd[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    cs[i] = cc[i >> 1];
                    sn[i] = i & 1 ? dd[i >> 1] : -dd[i >> 1];
                }
            } else {                // channels 8 s .. + 7 of the first half, or the second half's with the same pairs
                const bool second = s >= rotary_lanes / 2;
                const float* c = t + 8 * (second ? s - rotary_lanes / 2 : s);
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 x = *reinterpret_cast<const float4*>(c + i), y = *reinterpret_cast<const float4*>(c + p.half + i);
                    cs[i] = x.x; cs[i + 1] = x.y; cs[i + 2] = x.z; cs[i + 3] = x.w;
                    sn[i] = y.x; sn[i + 1] = y.y; sn[i + 2] = y.z; sn[i + 3] = y.w;
                }
                if (!second) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) sn[i] = -sn[i];
                }
            }
        }
    }
    const int partner = INTERLEAVED ? lane : (s < rotary_lanes / 2 ? lane + rotary_lanes / 2 : lane - rotary_lanes / 2) & 31;
    const size_t place = ((size_t)max(page, 0) * p.Hkv * kBlk + (token & 63)) * kD + 8 * s;
#pragma unroll 1
    for (int x = first; x < last; x += 2 * kAhead) {
        uint4 raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = next[i];
        if (x + 2 * kAhead < last) fetch(x + 2 * kAhead);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (x + 2 * i >= last) break;
            const int head = x + 2 * i + side;
            const bool query = head < p.Hq, value = head >= p.Hq + p.Hkv;
            uint4 out = raw[i];
            if (x + 2 * i < p.Hq + p.Hkv) {      // (both heads are values: nothing to do)
                float f[8];
                unpack8(raw[i], f);
                const __nv_bfloat16* const weight = query ? p.q_norm : value ? nullptr : p.k_norm;
                if (p.q_norm || p.k_norm) {
                    float sum = 0.f;
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum += f[c] * f[c];
#pragma unroll
                    for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
                    if (weight) {
                        float w[8];
                        unpack8(*reinterpret_cast<const uint4*>(weight + 8 * s), w);   // (from the first level of the cache)
                        const float inv = rsqrtf(sum * (1.f / kD) + p.eps);
#pragma unroll
                        for (int c = 0; c < 8; ++c) f[c] = f[c] * inv * w[c];
                    }
                }
                if (p.half) {
                    float other[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) other[c] = INTERLEAVED ? f[c ^ 1] : __shfl_sync(kFull, f[c], partner);
                    if (turns) {
#pragma unroll
                        for (int c = 0; c < 8; ++c) f[c] = f[c] * cs[c] + other[c] * sn[c];
                    }
                }
                if (!value) out = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
            }
            if (head < last) {
                if (query) *reinterpret_cast<uint4*>(p.q_out + ((size_t)row * p.Hq + head) * kD + 8 * s) = out;
                else if (page >= 0)
                    *reinterpret_cast<uint4*>((value ? p.v_cache + (size_t)(head - p.Hq - p.Hkv) * kBlk * kD
                                                     : p.k_cache + (size_t)(head - p.Hq) * kBlk * kD) + place) = out;
            }
        }
    }
}

}  // namespace ffd

using namespace ffd;

extern "C" {

ffd_status ffd_rotate_write_kv(const ffd_config* cfg, const ffd_rotation* rotation, const void* q, int64_t q_stride,
                               const void* k_new, const void* v_new, int64_t kv_stride, int32_t num_rows, const int32_t* positions,
                               void* q_out, void* k_cache, void* v_cache, const int32_t* block_table, const int32_t* row_start,
                               const int32_t* first_token, const int32_t* seq_lens, int32_t batch, int32_t max_blocks_per_seq,
                               int32_t num_pages, void* workspace, size_t workspace_bytes, void* stream) {
    ffd_status st = check_chunk(cfg, batch, num_rows, max_blocks_per_seq, num_pages);
    if (st) return st;
    if (!rotation || !q || !k_new || !v_new || !q_out || !k_cache || !v_cache || !seq_lens || !workspace) return FFD_ERR_NULL;
    if ((row_start == nullptr) != (first_token == nullptr)) return FFD_ERR_NULL;
    if (!row_start && num_rows != batch) return FFD_ERR_SHAPE;
    const ffd_rotation& t = *rotation;
    if (t.rotary_dim < 0 || t.rotary_dim > kD || t.rotary_dim % 16 || (t.interleaved != 0 && t.interleaved != 1)) return FFD_ERR_UNSUPPORTED;
    if (t.rotary_dim && !t.cos_sin) return FFD_ERR_NULL;
    if (t.rotary_dim && t.num_positions <= 0) return FFD_ERR_SHAPE;
    if (!(t.eps >= 0.f) || isinf(t.eps)) return FFD_ERR_SHAPE;
    if (q_stride < (int64_t)cfg->num_q_heads * kD || q_stride % 8 || kv_stride < (int64_t)cfg->num_kv_heads * kD || kv_stride % 8)
        return FFD_ERR_SHAPE;
    if (workspace_bytes < kHeaderBytes) return FFD_ERR_WORKSPACE;
    if (any_misaligned(q, k_new, v_new, positions, q_out, k_cache, v_cache, block_table, row_start, first_token, seq_lens, workspace,
                       t.cos_sin, t.q_norm, t.k_norm))
        return FFD_ERR_ALIGN;
    RotateParams p;
    p.r = ChunkRows{row_start, first_token, seq_lens, block_table, static_cast<uint32_t*>(workspace), num_rows, batch, max_blocks_per_seq, num_pages};
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(k_new);
    p.v = static_cast<const __nv_bfloat16*>(v_new);
    p.q_stride = q_stride;
    p.kv_stride = kv_stride;
    p.positions = positions;
    p.cos_sin = t.cos_sin;
    p.q_norm = static_cast<const __nv_bfloat16*>(t.q_norm);
    p.k_norm = static_cast<const __nv_bfloat16*>(t.k_norm);
    p.q_out = static_cast<__nv_bfloat16*>(q_out);
    p.k_cache = static_cast<__nv_bfloat16*>(k_cache);
    p.v_cache = static_cast<__nv_bfloat16*>(v_cache);
    p.Hq = cfg->num_q_heads;
    p.Hkv = cfg->num_kv_heads;
    p.num_positions = t.num_positions;
    p.half = t.rotary_dim / 2;
    p.eps = t.eps;
    // pairs of heads of a warp: one while the warps do not fill the card once; all of a token's where there are rows enough, so
    // that its place and its cosines are looked up once
    const int pairs = (p.Hq + 2 * p.Hkv + 1) / 2, sms = device_sms();
    p.pairs = (long long)num_rows * pairs <= 64LL * sms ? 1 : num_rows <= 64LL * sms && pairs > 8 ? 8 : pairs;
    p.slices = (pairs + p.pairs - 1) / p.pairs;
    const long long warps = (long long)num_rows * p.slices;
    if ((warps + kRotWarps - 1) / kRotWarps > 0x7fffffffLL) return FFD_ERR_SHAPE;
    launch_pdl(t.interleaved ? rotate_write_kernel<true> : rotate_write_kernel<false>, dim3((unsigned)((warps + kRotWarps - 1) / kRotWarps)),
               dim3(kRotWarps * 32), 0, static_cast<cudaStream_t>(stream), p);
    return launch_status();
}

}  // extern "C"
