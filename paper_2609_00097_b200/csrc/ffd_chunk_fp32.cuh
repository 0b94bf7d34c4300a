// Attention of a chunk with binary32 results: the same products, rounded nowhere to less than binary32 rounds.
//
// Two things keep the other kernel from it.  Its weights have 8 bits; here they are three bf16 pieces, which are all 24.  And the tensor
// cores' sums cut off instead of rounding, which adds up with their number: 7.6e-6 of the result over 4 K keys.  So a step's
// product P V begins from nothing, the smallest pieces first (cut off is then only what is below the last four instructions' results),
// and the steps are added up in binary32 in the registers of the thread that owns the row.  Those sums, 128 for a row, are also the
// reason for the sizes: a tile has one row tile, a step is a page (64 keys), the two softmax warpgroups take alternate steps,
// each with sums of its own, and join them where a segment ends.  The warps that only wait and copy give them their registers.
//
// A warpgroup's 256 columns of tensor memory: the scores of a step in the first 64 of 128, its weights, three pieces of 16 columns for
// each 32 keys, where the scores of those keys or nothing are (weight_col), and the step's product in the other 128.
//
// What bounds it: the products, 256 cycles for the scores of a step and 768 for its three pieces, 2048 for 128 keys of a row tile.
#pragma once
#include <cuda.h>
#include <math.h>

#include "ffd_chunk.cuh"
#include "ffd_prefix_step.cuh"
#include "ffd_tensor.cuh"

namespace ffd {

constexpr int kPageBytes = kBlk * kD * 2, kPageHalf = kPageBytes / 2;     // a page's K or V of a head; 64 channels of it
constexpr int kC32Stages = 8;
constexpr int kC32Edges = kC32Stages;            // barriers for V with hidden values
constexpr int kC32Smem = 2 * kRowTileBytes + kC32Stages * kPageBytes + 1024;
constexpr int kC32MinShift = 8;                  // log2 of the smallest share of a CTA: about four pages
constexpr int kC32SumRegs = 216, kC32OtherRegs = 72;
static_assert(256 * kC32SumRegs + 128 * kC32OtherRegs == kCkThreads * 168, "the registers that the launch has");
constexpr uint32_t kIdescPage = 1u << 4 | 1u << 7 | 1u << 10 | (64u >> 3) << 17 | (128u >> 4) << 24;   // N = 64

// where the weights of the page's keys 32 half .. + 31 go: the scores that are still to be read are in columns 32 .. 63 or nowhere
__device__ __forceinline__ constexpr int weight_col(int half) { return half ? 0 : 64; }

__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

__global__ void __launch_bounds__(kCkThreads, 1) chunk_attention_fp32_kernel(const __grid_constant__ CUtensorMap k_map,
                                                                           const __grid_constant__ CUtensorMap v_map,
                                                                           const __grid_constant__ CUtensorMap q_map,
                                                                           const __grid_constant__ ChunkParams p) {
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kC32Stages], s_empty[kC32Stages], s_scores[2], s_probs[2], s_done[2], s_qfull[2], s_qempty[2],
        s_edge[kC32Edges], s_join, s_drain, s_segfull[kCkSegments], s_segempty[kCkSegments];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_failed;
    __shared__ ChunkSegment s_segment[kCkSegments];
    __shared__ int s_bad[kCkBadRing];                       // per step: is its page bad?
    __shared__ volatile int s_flawed[kCkFlawRing];          // whose notes s_flaw holds: that segment's number + 1 (0: nobody's)
    __shared__ int s_flaw[kCkFlawRing][kD];                 // per channel: the first token whose value there is no number
    __shared__ float2 s_ml[2][128];                         // (reference, sum) of both warpgroups' rows where they are joined
    const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_smem = base, ring = base + 2 * kRowTileBytes;
    const uint32_t full = smem_u32(s_full), empty = smem_u32(s_empty), scores = smem_u32(s_scores), probs = smem_u32(s_probs),
                   done = smem_u32(s_done), qfull = smem_u32(s_qfull), qempty = smem_u32(s_qempty), edge_bar = smem_u32(s_edge),
                   join = smem_u32(&s_join), seg_full = smem_u32(s_segfull), seg_empty = smem_u32(s_segempty);

    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];\nprefetch.tensormap [%2];\n" ::"l"(&k_map), "l"(&v_map), "l"(&q_map) : "memory");
        for (int i = 0; i < kC32Stages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(scores + 8 * i, 1);
            mbar_init(probs + 8 * i, 4);
            mbar_init(done + 8 * i, 1);
            mbar_init(qfull + 8 * i, 1);
            mbar_init(qempty + 8 * i, 1);
        }
        for (int i = 0; i < kC32Edges; ++i) mbar_init(edge_bar + 8 * i, 1);
        for (int i = 0; i < kCkSegments; ++i) {
            mbar_init(seg_full + 8 * i, 1);
            mbar_init(seg_empty + 8 * i, kCkTakers);
        }
        mbar_init(join, 8);
        mbar_init(smem_u32(&s_drain), 1);
        s_failed = 0;
        for (int i = 0; i < kCkFlawRing; ++i) s_flawed[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    if (warp == 11)
        for (int i = lane; i < kCkFlawRing * kD; i += 32) s_flaw[i / kD][i % kD] = 0x7fffffff;
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = __shfl_sync(kFull, s_tmem, 0);     // columns: scores and weights of warpgroup i at 256 i, its product at 256 i + 128
    pdl_launch_dependents();
    pdl_wait();

    auto wait = [&](uint32_t bar, uint32_t parity) {   // by whole warps
        bool ok = mbar_try(bar, parity);
        if (!__all_sync(kFull, ok)) {
            const long long t0 = clock64();
            while (!ok && !s_failed && clock64() - t0 < kSpinCycles) ok = mbar_try(bar, parity);
            if (!ok) s_failed = 1;
            ok = __all_sync(kFull, ok);
        }
        return ok;
    };
    // a copy of the share's segment i; one without steps where the wait runs out
    auto look = [&](int i) {
        ChunkSegment s;
        const bool ok = wait(seg_full + 8 * (i % kCkSegments), (i / kCkSegments) & 1);
        s = s_segment[i % kCkSegments];
        if (!ok) s.count = 0;
        return s;
    };
    auto take = [&](int i) {
        const ChunkSegment s = look(i);
        __syncwarp();
        if (lane == 0) mbar_arrive(seg_empty + 8 * (i % kCkSegments));
        return s;
    };
    const int T1 = p.T1;
    using Micro = ChunkMicro<kBlk>;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kC32OtherRegs));
        if (warp == 10) {
            // ---- this CTA's share, and the queries of its segments, which take turns in two places
            ChunkCut cut[2];
            {
                auto cost = [&](int b) { return ChunkTiles<1>(chunk_seq(p.r, b), T1).cost(); };
                WarpScan<decltype(cost)> scan(p.r.batch, cost, lane);
                const long long total = scan.total * p.Hkv;
                const int parts = (int)max(1LL, min((long long)gridDim.x, total >> kC32MinShift)), c = blockIdx.x;
                if (c == 0 && lane == 0) *p.parts = total > 0 ? parts : 0;
                cut[0] = cut[1] = ChunkCut{p.r.batch, 0, 0, 0};
                if (c < parts && total > 0) {
                    const long long each = quick_div(total, parts), more = total - each * parts;
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) cut[i] = chunk_cut<1>(p.r, scan, p.Hkv, T1, each * (c + i) + min((long long)(c + i), more));
                    if (lane == 0) {
                        p.cuts[c] = cut[0];
                        if (c + 1 == parts) p.cuts[parts] = cut[1];
                    }
                }
            }
            ChunkWalk<1> walk(p.r, T1, cut[0], cut[1]);
            int segment = 0;
            bool ok = true;
#pragma unroll 1
            for (;; ++segment) {
                if (segment >= kCkSegments) ok = wait(seg_empty + 8 * (segment % kCkSegments), (segment / kCkSegments - 1) & 1);
                if (!ok) break;
                const bool end = walk.done();
                const int token = walk.token0(T1), slot = segment & 1;
                if (lane == 0) {
                    ChunkSegment s;
                    s.b = walk.at.b;
                    s.g = walk.at.g;
                    s.step = walk.at.step;
                    s.count = end ? 0 : walk.count();
                    s.single = 1;
                    s.slot = 2 * blockIdx.x + (walk.at.step == 0);
                    s.whole = walk.at.step == 0 && walk.last == walk.steps;
                    s.pos = walk.s.first + token;
                    s.tokens = walk.s.n - token;
                    s.row = walk.s.row0 + token;
                    s.len = walk.s.len;
                    s_segment[segment % kCkSegments] = s;
                    mbar_arrive(seg_full + 8 * (segment % kCkSegments));
                }
                __syncwarp();
                if (end) break;
                if (segment >= 2) ok = wait(qempty + 8 * slot, (segment / 2 - 1) & 1);
                if (!ok) break;
                if (elect_one()) {
                    mbar_expect(qfull + 8 * slot, 2 * T1 * p.G * 128);
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        tma_load_3d(q_smem + slot * kRowTileBytes + half * kRowTileHalf, &q_map, 64 * half, walk.at.g * p.G, walk.s.row0 + token,
                                    qfull + 8 * slot);
                }
                __syncwarp();
                walk.next(p.r, p.Hkv, T1);
            }
            // (`segment` queries were asked for: the loop ends before it asks for one)
            for (int x = max(0, segment - 2); x < segment; ++x) mbar_wait(qfull + 8 * (x & 1), (x >> 1) & 1);
        } else if (warp == 8) {
            // ---- keys and values: the ring's entries in order of use
            struct Pages { int b, from, page; };
            Pages pages[2] = {{-1, 0, 0}, {-1, 0, 0}};       // of keys and of values; lane x: the page of block from + x
            int issued = 0, edges = 0;
            const int oob = p.r.num_pages * p.Hkv * kBlk;    // a row behind the pool: TMA fills zeros
            auto load = [&](const CUtensorMap* map, const Micro& m, Pages& pg, bool keys) {
                const int st = issued % kC32Stages, round = issued / kC32Stages, block = m.s.step + m.t;
                if (round > 0 && !wait(empty + 8 * st, (round - 1) & 1)) return false;
                if (pg.b != m.s.b || block < pg.from || block >= pg.from + 32) {
                    pg.b = m.s.b;
                    pg.from = block;
                    pg.page = -1;
                    if ((long long)(block + lane) * kBlk < m.s.len) {
                        pg.page = chunk_page(p.r, pg.b, block + lane);
                        if (pg.page < 0) atomicOr(p.r.status, kDevBadPage);
                    }
                }
                const int page = __shfl_sync(kFull, pg.page, block - pg.from);
                const bool hidden = !keys && m.edge();      // warp 11 has it first, and says `full`
                const uint32_t bar = hidden ? edge_bar + 8 * (edges % kC32Edges) : full + 8 * st;
                edges += hidden;
                if (elect_one()) {
                    const uint32_t dst = ring + st * kPageBytes;
                    const int y = page >= 0 ? (page * p.Hkv + m.s.g) * kBlk : oob;
                    if (keys) s_bad[m.step % kCkBadRing] = page < 0;   // read behind `full` and `scores`
                    mbar_expect(bar, kPageBytes);
                    tma_load(dst, map, 0, y, bar);
                    tma_load(dst + kPageHalf, map, 64, y, bar);
                }
                __syncwarp();
                ++issued;
                return true;
            };
            chunk_order<kBlk>(look, take, [&](const Micro& m) { return load(&k_map, m, pages[0], true); },
                              [&](const Micro& m) { return load(&v_map, m, pages[1], false); });
            // nothing may write into this CTA's shared memory once it has left, whatever became of the other roles
            for (int i = max(0, edges - kC32Edges); i < edges; ++i) mbar_wait(edge_bar + 8 * (i % kC32Edges), (i / kC32Edges) & 1);
            for (int i = max(0, issued - kC32Stages); i < issued; ++i) mbar_wait(full + 8 * (i % kC32Stages), (i / kC32Stages) & 1);
        } else if (warp == 9) {
            // ---- products
            int used = 0;                          // ring entries
            bool ok = true;
            auto ready = [&](int e) { return wait(full + 8 * (e % kC32Stages), (e / kC32Stages) & 1); };
            auto entry = [&](int e) { return ring + (e % kC32Stages) * kPageBytes; };
            chunk_order<kBlk>(
                look, take,
                [&](const Micro& m) {
                    const int e = used++, slot = m.segment & 1;
                    ok = ready(e) && (m.t > 0 || wait(qfull + 8 * slot, (m.segment >> 1) & 1));
                    if (!ok) return false;
                    tmem_after_sync();
                    const uint32_t d = tmem + 256 * (m.x & 1);
                    const uint64_t a = mma_desc(q_smem + slot * kRowTileBytes, 16, 1024), b = mma_desc(entry(e), 16, 1024);
                    const bool q_ends = m.t + 1 == m.s.count;
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            mma_ss(d, a + (((ks >> 2) * kRowTileHalf + (ks & 3) * 32) >> 4), b + (((ks >> 2) * kPageHalf + (ks & 3) * 32) >> 4),
                                   kIdescPage, ks > 0);
                        mma_commit(scores + 8 * (m.x & 1));
                        mma_commit(empty + 8 * (e % kC32Stages));
                        if (q_ends) mma_commit(qempty + 8 * slot);
                    }
                    __syncwarp();
                    return true;
                },
                [&](const Micro& m) {
                    const int e = used++, i = m.x & 1;
                    ok = ready(e) && wait(probs + 8 * i, (m.x >> 1) & 1);
                    if (!ok) return false;
                    tmem_after_sync();
                    const uint32_t w = tmem + 256 * i, d = w + 128;
                    const uint64_t v = mma_desc(entry(e), kPageHalf, 1024);
                    if (elect_one()) {
#pragma unroll
                        for (int piece = 2; piece >= 0; --piece)
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                mma_ts(d, w + weight_col(y >> 1) + 16 * piece + 8 * (y & 1), v + (y * 2048 >> 4), kIdescMnB, piece < 2 || y > 0);
                        mma_commit(done + 8 * i);
                        mma_commit(empty + 8 * (e % kC32Stages));
                    }
                    __syncwarp();
                    return true;
                });
            if (!ok) {   // products in flight still write tensor memory
                if (elect_one()) mma_commit(smem_u32(&s_drain));
                __syncwarp();
                mbar_wait(smem_u32(&s_drain), 0);
            }
        } else {
            // ---- values that some of a tile's rows do not see, as in the other kernel
            int edges = 0, step0 = 0;
            bool ok = true;
            ChunkSegment s = look(0);
#pragma unroll 1
            for (int segment = 0; ok && s.count > 0; ++segment) {
                const ChunkSegment next = look(segment + 1);
                const int buffer = segment % kCkFlawRing;
                bool fresh = true;
#pragma unroll 1
                for (int t = max(0, (s.pos >> 6) - s.step); t < s.count; ++t) {     // (steps before it are seen by all rows)
                    const int key0 = (s.step + t) * kBlk;
                    if (key0 + kBlk - 1 <= s.pos) continue;
                    if (!wait(edge_bar + 8 * (edges % kC32Edges), (edges / kC32Edges) & 1)) {
                        ok = false;
                        break;
                    }
                    ++edges;
                    if (fresh && s_flawed[buffer]) {   // of a segment eight or more before, whose results have been written
                        __syncwarp();
                        for (int c = lane; c < kD; c += 32) s_flaw[buffer][c] = 0x7fffffff;
                        if (lane == 0) s_flawed[buffer] = 0;
                        __syncwarp();
                    }
                    fresh = false;
                    // the ring's entry: step j's V is behind the keys of the steps before it, its own, and the next one's, if there is one
                    const int j = step0 + t, vc = 2 * j + 1 + (t + 1 < s.count || next.count > 0);
                    const uint32_t tile = ring + (vc % kC32Stages) * kPageBytes;
                    const int x0 = max(0, s.pos + 1 - key0), x1 = min(kBlk, s.pos + min(T1, s.tokens) - key0);
                    if (hide_values<kBlk>(tile, x0, x1, key0, s_flaw[buffer], lane) && lane == 0) s_flawed[buffer] = segment + 1;
                    __threadfence_block();
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full + 8 * (vc % kC32Stages));
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(seg_empty + 8 * (segment % kCkSegments));
                step0 += s.count;
                s = next;
            }
            __syncwarp();
        }
    } else {
        // ---- softmax, sums and results
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kC32SumRegs));
        const int i = warp >> 2, row = tid & 127;
        const int tok = row / p.G, h = row - tok * p.G;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t s_col = tmem + 256 * i + lanes, o_col = s_col + 128;
        const float scale = p.logit_scale;
        const unsigned long long scale2 = pair_of(scale, scale);
        uint32_t n = 0, joined = 0;               // micro-steps of this warpgroup, phases of `join`
        int x0 = 0;                               // micro-steps of the share before the present segment
        bool ok = true;
#pragma unroll 1
        for (int segment = 0; ok; ++segment) {
            const ChunkSegment s = take(segment);
            if (s.count == 0) break;
            const int t0 = i ^ (x0 & 1);
            const bool exists = tok < T1 && tok < s.tokens;
            const bool active = __any_sync(kFull, exists);
            const int sees = exists ? s.pos + tok + 1 : 0;
            float m = -INFINITY, l = 0.f;
            unsigned long long acc[kD / 2];       // the row's sums, two channels each
#pragma unroll
            for (int c = 0; c < kD / 2; ++c) acc[c] = 0ull;
#pragma unroll 1
            for (int t = t0; t < s.count; t += 2, ++n) {
                ok = wait(scores + 8 * i, n & 1);
                if (!ok) break;
                tmem_after_sync();
                if (!active) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(probs + 8 * i);
                    continue;
                }
                // no logits: tokens behind the row's own, or a bad page's rows of zeros
                const int keep = s_bad[(x0 + t) % kCkBadRing] ? 0 : min(max(0, sees - (s.step + t) * kBlk), kBlk);
                float top = -INFINITY;
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    float a[32];
                    tmem_ld32(s_col + 32 * half, a);
                    tmem_wait_ld();
                    float tops[2] = {-INFINITY, -INFINITY};
                    if (keep < kBlk) {
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (32 * half + x >= keep) a[x] = -INFINITY;
                    }
#pragma unroll
                    for (int x = 0; x < 32; x += 2) tops[x >> 1 & 1] = max3(tops[x >> 1 & 1], a[x], a[x + 1]);
                    top = max3(top, tops[0], tops[1]);
                }
                top *= scale;
                if (__any_sync(kFull, top > m + 8.f)) {   // the reference is raised where a row exceeds it by 2^8, as its first tokens do
                    const float raised = fmaxf(m, top), alpha = raised == -INFINITY ? 1.f : fast_ex2(m - raised);
                    const unsigned long long alpha2 = pair_of(alpha, alpha);
                    m = raised;
                    l *= alpha;
#pragma unroll
                    for (int c = 0; c < kD / 2; ++c) acc[c] = pair_fma(acc[c], alpha2, 0ull);
                }
                const float shift = m == -INFINITY ? 0.f : -m;
                const unsigned long long shift2 = pair_of(shift, shift);
                unsigned long long sums[2] = {0ull, 0ull};
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    float a[32];
                    tmem_ld32(s_col + 32 * half, a);
                    tmem_wait_ld();
                    if (keep < kBlk) {
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (32 * half + x >= keep) a[x] = -INFINITY;
                    }
                    const uint32_t to = s_col + weight_col(half);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {         // 16 keys: eight columns of each piece
                        uint32_t piece[3][8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            float u, v;
                            pair_split(pair_fma(pair_of(a[16 * c + 2 * x], a[16 * c + 2 * x + 1]), scale2, shift2), u, v);
                            u = fast_ex2(u);
                            v = fast_ex2(v);
                            sums[x & 1] = pair_add(sums[x & 1], pair_of(u, v));
#pragma unroll
                            for (int y = 0; y < 3; ++y) {     // (a difference from a rounding to 8 bits is exact: 24 bits in three pieces)
                                const uint32_t both = pack_bf16(u, v);
                                piece[y][x] = both;
                                u -= __uint_as_float(both << 16);
                                v -= __uint_as_float(both & 0xffff0000u);
                            }
                        }
#pragma unroll
                        for (int y = 0; y < 3; ++y) tmem_st8(to + 16 * y + 8 * c, piece[y]);
                    }
                }
                {
                    float u, v;
                    pair_split(pair_add(sums[0], sums[1]), u, v);
                    l += u + v;
                }
                tmem_wait_st();
                tmem_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(probs + 8 * i);
                ok = wait(done + 8 * i, n & 1);
                if (!ok) break;
                tmem_after_sync();
#pragma unroll
                for (int c = 0; c < kD; c += 32) {
                    float o[32];
                    tmem_ld32(o_col + c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 32; x += 2) acc[(c + x) / 2] = pair_add(acc[(c + x) / 2], pair_of(o[x], o[x + 1]));
                }
                tmem_before_sync();                       // (the next product overwrites them)
            }
            if (!ok) break;
            if (t0 < s.count) {
                const bool both = s.count > 1;            // the other warpgroup has sums of the same rows: each finishes 64 channels
                float fa = 1.f, fb = 0.f, top = m, sum = l;
                if (both) {
                    if (active) {
#pragma unroll
                        for (int c = 0; c < kD; c += 32) {
                            if ((c >> 6) == i) continue;
                            float o[32];
#pragma unroll
                            for (int x = 0; x < 32; x += 2) pair_split(acc[(c + x) / 2], o[x], o[x + 1]);
                            tmem_st32(o_col + c, reinterpret_cast<const uint32_t*>(o));
                        }
                        s_ml[i][row] = make_float2(m, l);
                        tmem_wait_st();
                    }
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(join);
                    ok = wait(join, joined++ & 1);
                    if (!ok) break;
                    tmem_after_sync();
                    if (active) {
                        const float2 o = s_ml[i ^ 1][row];
                        top = fmaxf(m, o.x);
                        const float use = top == -INFINITY ? 0.f : top;
                        fa = fast_ex2(m - use);
                        fb = fast_ex2(o.x - use);
                        sum = fa * l + fb * o.y;
                    }
                }
                if (active) {
                    const bool some = sum != 0.f, whole = s.whole;
                    const float norm = some ? 1.f / sum : 0.f;
                    fa *= norm;
                    fb *= norm;
                    const int part_row = s.slot * kCkRows + row;
                    const int at = whole ? (s.row + tok) * p.Hq + s.g * p.G + h : part_row;   // (heads of all rows: below 2^31)
                    if (exists && (!both || i == 0)) {
                        const float log2_sum = some ? top + log2f(sum) : -INFINITY;
                        if (!whole) p.part_lse[part_row] = log2_sum;
                        else if (p.lse) p.lse[at] = log2_sum * kLn2;
                    }
                    char* const to = static_cast<char*>(whole ? p.out : p.part_out) + (size_t)(unsigned)at * (kD * 4);
                    const bool sectors = (reinterpret_cast<uintptr_t>(to) & 31) == 0;
                    const bool flawed = s_flawed[segment % kCkFlawRing] == segment + 1;
#pragma unroll
                    for (int c = 0; c < kD; c += 32) {
                        if (both && (c >> 6) != i) continue;
                        float o[32];
#pragma unroll
                        for (int x = 0; x < 32; x += 2) {
                            float u, v;
                            pair_split(acc[(c + x) / 2], u, v);
                            o[x] = some ? u * fa : 0.f;
                            o[x + 1] = some ? v * fa : 0.f;
                        }
                        if (both) {
                            float o2[32];
                            tmem_ld32(tmem + 256 * (i ^ 1) + 128 + lanes + c, o2);
                            tmem_wait_ld();
#pragma unroll
                            for (int x = 0; x < 32; ++x) o[x] += some ? o2[x] * fb : 0.f;
                        }
                        if (flawed) {
#pragma unroll
                            for (int x = 0; x < 32; ++x) o[x] = s_flaw[segment % kCkFlawRing][c + x] < sees ? NAN : o[x];
                        }
                        if (!exists) continue;
#pragma unroll
                        for (int x = 0; x < 32; x += 8) store_sector(to + 4 * (c + x), reinterpret_cast<const uint32_t*>(o + x), sectors);
                    }
                }
                if (both) {   // the columns may be written again when both have read them
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(join);
                    ok = wait(join, joined++ & 1);
                    tmem_after_sync();
                }
            }
            x0 += s.count;
        }
    }
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    if (tid == 0 && s_failed) atomicOr(p.r.status, kDevTimeout);
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
}

}  // namespace ffd
