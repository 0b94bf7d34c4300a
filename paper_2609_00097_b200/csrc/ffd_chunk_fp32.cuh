// Attention of a chunk with binary32 results: the same products, rounded nowhere to less than binary32 rounds.
//
// Two things keep the other kernel from it.  Its weights have 8 bits; here they are three bf16 pieces, which are all 24.  And the tensor
// cores' sums cut off instead of rounding, which adds up with their number: 7.6e-6 of the result over 4 K keys.  So a step's
// product P V begins from nothing, the smallest pieces first (cut off is then only what is below the last four instructions' results),
// and the steps are added up in binary32 in the registers of the thread that owns the row.  Those sums, 128 for a row, are also the
// reason for the sizes: a tile has one row tile, a step is a page (64 keys), the two softmax warpgroups take alternate steps,
// each with sums of its own, and join them where a segment ends.  The warps that only wait and copy give them their registers.
// (Ragged prompts of up to 2 K: an error of 2.7e-7 of the result, 3.8e-7 in plain binary32 operations; with two pieces and sums of up
// to 1152 keys in tensor memory it was 2.1e-6.)
//
// A warpgroup's 256 columns of tensor memory: the scores of two steps, 64 each, so that those of the next one are there when it is done
// with one, and a step's product.  Weights go where the scores of their step were, high and middle pieces in 16 columns for each 32
// keys, and their third pieces, for which no columns are left, to shared memory, in two places.
//
// What bounds it: the products, 20 a step, whose issue takes the tensor cores' own time (46 cycles for one of the scores' with 64
// columns, 62 to 64 for one of the other twelve, 1112 in all, by a probe; 1280 in the kernel), with 450 cycles of asking for barriers and
// 200 of counting around them: 1930 cycles a step.  A warpgroup has the time of two steps for its one, and takes 3500 of these 3860.
// With the scores behind the product, in one place, and every barrier asked by itself, a step was 2100 cycles, and 2400 with one row.
// One token on 128 K: 131 us; five for each of eight users: 145; a prompt of 8 K: 1140, at 1.6 GHz under the power limit.
#pragma once
#include <cuda.h>
#include <math.h>

#include "ffd_chunk.cuh"
#include "ffd_prefix_step.cuh"
#include "ffd_tensor.cuh"

namespace ffd {

constexpr int kPageBytes = kBlk * kD * 2, kPageHalf = kPageBytes / 2;     // a page's K or V of a head; 64 channels of it
constexpr int kC32Stages = 5;                    // of the ring
constexpr int kC32Ahead = 4;                     // steps between scores and values: two for each warpgroup
constexpr int kC32Edges = kC32Stages;            // barriers for V with hidden values: no more are in the ring
constexpr int kLowBytes = 128 * kBlk * 2;        // third pieces of a step's weights: 128 rows of 64 keys
constexpr int kC32Smem = 2 * kRowTileBytes + 4 * kLowBytes + kC32Stages * kPageBytes + 1024;
constexpr int kC32MinShift = 8;                  // log2 of the smallest share of a CTA: about four pages
constexpr int kC32SumRegs = 216, kC32OtherRegs = 72;
static_assert(256 * kC32SumRegs + 128 * kC32OtherRegs == kCkThreads * 168, "the registers that the launch has");
constexpr uint32_t kIdescPage = 1u << 4 | 1u << 7 | 1u << 10 | (64u >> 3) << 17 | (128u >> 4) << 24;   // N = 64

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
    __shared__ __align__(8) uint64_t s_full[kC32Stages], s_empty[kC32Stages], s_scores[4], s_probs[2], s_done[2], s_qfull[2], s_qempty[2],
        s_edge[kC32Edges], s_join, s_drain, s_segfull[kCkSegments], s_segempty[kCkSegments];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_failed;
    __shared__ ChunkSegment s_segment[kCkSegments];
    __shared__ volatile int s_edge_entry[kC32Edges];        // the ring's entry with the values that a barrier of s_edge is for
    __shared__ int s_bad[kCkBadRing];                       // per step: is its page bad?
    __shared__ volatile int s_flawed[kCkFlawRing];          // whose notes s_flaw holds: that segment's number + 1 (0: nobody's)
    __shared__ int s_flaw[kCkFlawRing][kD];                 // per channel: the first token whose value there is no number
    __shared__ float2 s_ml[2][128];                         // (reference, sum) of both warpgroups' rows where they are joined
    const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_smem = base, low_smem = base + 2 * kRowTileBytes, ring = low_smem + 4 * kLowBytes;
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
            mbar_init(scores + 16 + 8 * i, 1);
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
    const uint32_t tmem = __shfl_sync(kFull, s_tmem, 0);     // columns: scores of warpgroup i at 256 i and 256 i + 64, its product at 256 i + 128
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
                    if (hidden) s_edge_entry[(edges - 1) % kC32Edges] = st;
                    mbar_expect(bar, kPageBytes);
                    tma_load(dst, map, 0, y, bar);
                    tma_load(dst + kPageHalf, map, 64, y, bar);
                }
                __syncwarp();
                ++issued;
                return true;
            };
            chunk_order<kBlk, kC32Ahead>(look, take, [&](const Micro& m) { return load(&k_map, m, pages[0], true); },
                              [&](const Micro& m) { return load(&v_map, m, pages[1], false); });
            // nothing may write into this CTA's shared memory once it has left, whatever became of the other roles
            for (int i = max(0, edges - kC32Edges); i < edges; ++i) mbar_wait(edge_bar + 8 * (i % kC32Edges), (i / kC32Edges) & 1);
            for (int i = max(0, issued - kC32Stages); i < issued; ++i) mbar_wait(full + 8 * (i % kC32Stages), (i / kC32Stages) & 1);
        } else if (warp == 9) {
            // ---- products: those of a step, and the scores of the one that is kC32Ahead behind it, go out together.  Few products wait in
            // the tensor core's queue (the third or fourth has to wait for its place), and a barrier answers after 130 cycles even if it
            // was passed long ago: so the barriers of both are asked together.
            int used = 0;                          // ring entries
            bool ok = true;
            Micro k, v;                            // of the next scores, of the next values
            k.begin(look);
            v.begin(take);
            auto full_of = [&](int e) { return full + 8 * (e % kC32Stages); };
            auto parity_of = [&](int e) { return (uint32_t)(e / kC32Stages) & 1u; };
            auto entry = [&](int e) { return ring + (e % kC32Stages) * kPageBytes; };
            auto issue_scores = [&](const Micro& m, int e) {   // by one thread
                const int slot = m.segment & 1, place = m.x & 3;     // of warpgroup x & 1 the scores (x >> 1) & 1
                const uint32_t d = tmem + 256 * (place & 1) + 64 * (place >> 1);
                const uint64_t a = mma_desc(q_smem + slot * kRowTileBytes, 16, 1024), b = mma_desc(entry(e), 16, 1024);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    mma_ss(d, a + (((ks >> 2) * kRowTileHalf + (ks & 3) * 32) >> 4), b + (((ks >> 2) * kPageHalf + (ks & 3) * 32) >> 4),
                           kIdescPage, ks > 0);
                mma_commit(scores + 8 * place);
                mma_commit(empty + 8 * (e % kC32Stages));
                if (m.t + 1 == m.s.count) mma_commit(qempty + 8 * slot);
            };
#pragma unroll 1
            for (int ahead = 0; ahead < kC32Ahead && ok && k.live(); ++ahead) {
                const int e = used++;
                ok = wait(full_of(e), parity_of(e)) && (k.t > 0 || wait(qfull + 8 * (k.segment & 1), (k.segment >> 1) & 1));
                if (!ok) break;
                tmem_after_sync();
                if (elect_one()) issue_scores(k, e);
                __syncwarp();
                k.advance(look);
            }
#pragma unroll 1
            while (ok && v.live()) {
                const int i = v.x & 1, place = v.x & 3, ev = used++;
                const bool more = k.live(), fresh = more && k.t == 0;
                const int ek = more ? used++ : ev;
                const uint32_t p_bar = probs + 8 * i, p_parity = (v.x >> 1) & 1, q_bar = qfull + 8 * (k.segment & 1), q_parity = (k.segment >> 1) & 1;
                const bool p_there = mbar_try(p_bar, p_parity), v_there = mbar_try(full_of(ev), parity_of(ev)),
                           k_there = mbar_try(full_of(ek), parity_of(ek)), q_there = !fresh || mbar_try(q_bar, q_parity);
                if (!__all_sync(kFull, p_there && v_there && k_there && q_there)) {
                    ok = wait(full_of(ev), parity_of(ev)) && wait(full_of(ek), parity_of(ek)) && (!fresh || wait(q_bar, q_parity)) && wait(p_bar, p_parity);
                    if (!ok) break;
                }
                tmem_after_sync();
                const uint32_t w = tmem + 256 * i + 64 * (place >> 1), d = tmem + 256 * i + 128;
                const uint64_t vd = mma_desc(entry(ev), kPageHalf, 1024), low = mma_desc(low_smem + place * kLowBytes, 16, 1024);
                if (elect_one()) {
#pragma unroll
                    for (int y = 0; y < 4; ++y) mma_ss(d, low + (y * 32 >> 4), vd + (y * 2048 >> 4), kIdescMnB, y > 0);
#pragma unroll
                    for (int piece = 1; piece >= 0; --piece)
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            mma_ts(d, w + 32 * (y >> 1) + 16 * piece + 8 * (y & 1), vd + (y * 2048 >> 4), kIdescMnB, true);
                    mma_commit(done + 8 * i);
                    mma_commit(empty + 8 * (ev % kC32Stages));
                    if (more) issue_scores(k, ek);
                }
                __syncwarp();
                v.advance(take);
                if (more) k.advance(look);
            }
            if (!ok) {   // products in flight still write tensor memory
                if (elect_one()) mma_commit(smem_u32(&s_drain));
                __syncwarp();
                mbar_wait(smem_u32(&s_drain), 0);
            }
        } else {
            // ---- values that some of a tile's rows do not see, as in the other kernel
            int edges = 0;
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
                    if (fresh && s_flawed[buffer]) {   // of a segment eight or more before, whose results have been written
                        __syncwarp();
                        for (int c = lane; c < kD; c += 32) s_flaw[buffer][c] = 0x7fffffff;
                        if (lane == 0) s_flawed[buffer] = 0;
                        __syncwarp();
                    }
                    fresh = false;
                    const int entry = s_edge_entry[edges % kC32Edges];
                    ++edges;
                    const uint32_t tile = ring + entry * kPageBytes;
                    const int x0 = max(0, s.pos + 1 - key0), x1 = min(kBlk, s.pos + min(T1, s.tokens) - key0);
                    if (hide_values<kBlk>(tile, x0, x1, key0, s_flaw[buffer], lane) && lane == 0) s_flawed[buffer] = segment + 1;
                    __threadfence_block();
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full + 8 * entry);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(seg_empty + 8 * (segment % kCkSegments));
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
        const uint32_t s_cols = tmem + 256 * i + lanes, o_col = s_cols + 128;
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
            // adds up the product of the step before, times `beta` where the reference was raised behind it
            auto add = [&](float beta) {
                ok = wait(done + 8 * i, (n - 1) & 1);
                if (!ok || !active) return;
                tmem_after_sync();
                const unsigned long long beta2 = pair_of(beta, beta);
#pragma unroll
                for (int c = 0; c < kD; c += 64) {
                    float o[64];
                    tmem_ld32(o_col + c, o);
                    tmem_ld32(o_col + c + 32, o + 32);
                    tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 64; x += 2) acc[(c + x) / 2] = pair_fma(pair_of(o[x], o[x + 1]), beta2, acc[(c + x) / 2]);
                }
                tmem_before_sync();                       // (the next product overwrites them)
            };
#pragma unroll 1
            for (int t = t0; t < s.count; t += 2) {
                const int place = 2 * (n & 1) + i;        // of the scores' barriers and the third pieces
                ok = wait(scores + 8 * place, n >> 1 & 1);
                if (!ok) break;
                float beta = 1.f;
                if (active) {
                    tmem_after_sync();
                    const uint32_t s_col = s_cols + 64 * (n & 1);
                    // no logits: tokens behind the row's own, or a bad page's rows of zeros
                    const int keep = !exists ? kBlk : s_bad[(x0 + t) % kCkBadRing] ? 0 : min(max(0, sees - (s.step + t) * kBlk), kBlk);
                    auto mask = [&](float* a, int count, int key) {
                        if (keep < kBlk) {
#pragma unroll
                            for (int x = 0; x < count; ++x)
                                if (key + x >= keep) a[x] = -INFINITY;
                        }
                    };
                    // (tensor memory answers after 200 cycles while it is multiplied with: loads are waited for in twos or later)
                    float a[32], top;
                    {
                        float b[32];
                        tmem_ld32(s_col, a);
                        tmem_ld32(s_col + 32, b);
                        tmem_wait_ld();
                        mask(a, 32, 0);
                        mask(b, 32, 32);
                        float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int x = 0; x < 32; x += 2) {
                            tops[x >> 1 & 1] = max3(tops[x >> 1 & 1], a[x], a[x + 1]);
                            tops[2 + (x >> 1 & 1)] = max3(tops[2 + (x >> 1 & 1)], b[x], b[x + 1]);
                        }
                        top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]);
                    }
                    top *= scale;
                    if (__any_sync(kFull, top > m + 8.f)) {   // the reference is raised where a row exceeds it by 2^8, as its first tokens do
                        const float raised = fmaxf(m, top);
                        beta = raised == -INFINITY ? 1.f : fast_ex2(m - raised);
                        const unsigned long long beta2 = pair_of(beta, beta);
                        m = raised;
                        l *= beta;
#pragma unroll
                        for (int c = 0; c < kD / 2; ++c) acc[c] = pair_fma(acc[c], beta2, 0ull);
                    }
                    const float shift = m == -INFINITY ? 0.f : -m;
                    const unsigned long long shift2 = pair_of(shift, shift);
                    unsigned long long sums[2] = {0ull, 0ull};
                    const uint32_t low_row = low_smem + place * kLowBytes + row * 128;
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        if (half) {
                            tmem_wait_ld();
                            mask(a, 32, 32);
                        }
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
                            if (half == 0) tmem_ld16(s_col + 32 + 16 * c, a + 16 * c);      // the other half's, ahead
                            tmem_st8(s_col + 32 * half + 8 * c, piece[0]);
                            tmem_st8(s_col + 32 * half + 16 + 8 * c, piece[1]);
#pragma unroll
                            for (int y = 0; y < 2; ++y)       // 16 bytes, in the order of the 128-byte swizzle
                                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};\n" ::"r"(low_row + (((4 * half + 2 * c + y) ^ (row & 7)) << 4)),
                                             "r"(piece[2][4 * y]), "r"(piece[2][4 * y + 1]), "r"(piece[2][4 * y + 2]), "r"(piece[2][4 * y + 3])
                                             : "memory");
                        }
                    }
                    float u, v;
                    pair_split(pair_add(sums[0], sums[1]), u, v);
                    l += u + v;
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                }
                // (all warps wait for the step before, also those without rows: nobody may be a step ahead of the others at `probs`)
                if (t > t0) add(beta);
                if (!ok) break;
                tmem_wait_st();
                tmem_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(probs + 8 * i);
                ++n;
            }
            if (ok && t0 < s.count) add(1.f);
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
