// Attention of a chunk of new tokens over a paged cache that holds them already: row (b, i) is token first + i of sequence b and
// sees the tokens up to itself.
//
// The rows of a sequence and KV head, G heads for every token, form row tiles of 128 rows, so that a key is read once for the
// whole group.  One CTA per SM: warps 0..3 and 4..7 are two softmax warpgroups (a thread owns one row: no shuffles), warp 8 moves K
// and V with TMA, warp 9 issues tcgen05.mma, warp 10 moves the queries, warp 11 looks after values that not all rows see.
// A CTA has a share of the list of all steps (ffd_chunk.cuh) and runs through it without a break: the products of the next
// tile's first step begin while the last tile's results are on their way out.
//
// A micro-step is a row tile times 128 keys:
//   S = Q K^T   A = Q and B = K in shared memory (K-major, 128-byte swizzle), S in 128 columns of tensor memory
//   P = 2^(c S - m), rounded to bf16, written over the columns of S in two halves, each multiplied as soon as it is there
//   O += P V    A = P in tensor memory, B = V in shared memory, O in 128 columns of tensor memory
// Micro-steps alternate between the warpgroups whatever they belong to.  A tile with two row tiles gives each warpgroup one of
// them, and a step's K and V serve both; of a tile with one, the warpgroups take alternate steps and their results are joined.
// Scores, sums and the results are in binary32.  Weights are rounded to one bf16 piece (8 bits), as the results are: both errors are of
// the same size.  Binary32 results have a kernel of their own (ffd_chunk_fp32.cuh), as that would lose most of their bits.
//
// What bounds it.  Many tiles: a step of 256 rows by 128 keys takes 3500 to 3700 cycles, of which the products are 2048.  They go out one
// micro-step after the other: about 800 of a micro-step's 1870 cycles are the issue of its last twelve instructions, the rest are
// answers of barriers and the loop around them, and none of its barriers is ever waited for.  Nor are the powers it: with a
// multiplication in their place a step took as long.  (With a warp for each warpgroup's products both warpgroups compute at the same
// time and wait at the same time: 4000 to 4300 cycles.)  Long series of calls are held back by power as well, 1.4 to 1.6 GHz: a
// prompt of 8 K takes 570 us (0.97 PFLOP/s), in a short series on one state 495 to 530; 512 new tokens on 16 K 218 to 225.  Few rows:
// the bytes of keys and values (five tokens each for eight users, 605 MB: 120 to 128 us, 0.72 to 0.77 of the measured copy bandwidth; on
// one state, part of which stays in L2, 110), and 25 to 30 us around them: finding the shares, the first keys' way, results, merge.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "ffd_chunk.cuh"
#include "ffd_chunk_fp32.cuh"
#include "ffd_host.cuh"
#include "ffd_prefix_step.cuh"
#include "ffd_tensor.cuh"

namespace ffd {

constexpr int kCkStages = 4;                     // of 32 KB: K or V of a step
constexpr int kCkSmem = (2 + kCkStages) * kRowTileBytes + 1024;
constexpr int kCkEdges = 4;                      // barriers for V with hidden values: at most three V are in the ring
constexpr int kCkMinShift = 10;                  // log2 of the smallest share of a CTA: about two steps

// 64 columns of this warp's 32 lanes, in one instruction
__device__ __forceinline__ void tmem_ld64(uint32_t addr, float* x) {
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
        "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
        "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(addr));
}

// A step of one softmax warpgroup: the weights of 128 tokens over their scores in tensor memory, in two halves, of which the first
// is announced (probs) while the second is computed.  A thread has a row; (m, l) is its reference (log2) and sum, and the new
// ones are returned.  keep0, keep1: tokens of each half that have logits (keep0 below 0: a pass that works on whatever tensor
// memory holds and changes nothing).  opens: the segment's first step; the first half's maximum is then the reference.
// halves: completes with the first half's product.  Weights are computed against the reference as it stands, while the maximum is
// found; only if a row exceeds it by 2^8 the reference is raised, O rescaled, and the half is computed again.  If the wait for
// the first half's product runs out, the whole warp gets NaN for m, which no logits make of it.
// It is not inlined, and both halves run through the same code: it is the only long stretch without a loop, the other
// warpgroup is somewhere else in it, and what does not stay in the instruction cache is fetched line by line.  (With a copy for
// each half, as softmax_step has it: one token for 16 sequences 53 us instead of 41, a prompt of 8 K 560 instead of 522.  In pieces
// of 32 tokens, half as much code again but more loops than work in flight: 48 and 620.)  The second half's scores are loaded when
// they are needed: tensor memory answers within 30 cycles.
__device__ __noinline__ float2 chunk_softmax(uint32_t s_col, uint32_t o_col, float m, float l, float scale, int keep0, int keep1, bool opens,
                                             uint32_t probs, uint32_t halves, uint32_t parity) {
    const bool live = keep0 >= 0;             // (else: a pass that fetches the code and changes nothing)
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
        const int keep = half ? keep1 : keep0;
        const uint32_t col = s_col + 64 * half;
        float s[64];
        uint32_t hi[32], none[1];
        float sum, top;
        bool first = opens && half == 0;
        for (;;) {
            tmem_ld64(col, s);
            tmem_wait_ld();
            if (keep < 64) {
#pragma unroll
                for (int x = 0; x < 64; ++x)
                    if (x >= keep) s[x] = -INFINITY;
            }
            if (first) {
                float tops[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int x = 0; x < 64; x += 2) tops[x >> 1 & 1] = max3(tops[x >> 1 & 1], s[x], s[x + 1]);
                m = fmaxf(tops[0], tops[1]) * scale;
            }
            weights_of<1>(s, scale, m == -INFINITY ? 0.f : -m, hi, none, sum, top);
            top *= scale;
            if (!__any_sync(kFull, top > m + 8.f) || !live || first) break;
            const float raised = fmaxf(m, top);
            const float alpha = raised == -INFINITY ? 1.f : fast_ex2(m - raised);
            m = raised;
            l *= alpha;
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
        l += sum;
        if (live) {
            tmem_st32(col, hi);               // over the half's own scores
            tmem_wait_st();
            tmem_before_sync();
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbar_arrive(probs + 8 * half);
        }
    }
    return make_float2(m, l);
}

__global__ void __launch_bounds__(kCkThreads, 1) chunk_attention_kernel(const __grid_constant__ CUtensorMap k_map,
                                                                      const __grid_constant__ CUtensorMap v_map,
                                                                      const __grid_constant__ CUtensorMap q_map,
                                                                      const __grid_constant__ ChunkParams p) {
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kCkStages], s_empty[kCkStages], s_scores[2], s_probs[4], s_done[2], s_halves[2], s_qfull[2],
        s_qempty[2], s_edge[kCkEdges], s_join, s_drain, s_segfull[kCkSegments], s_segempty[kCkSegments];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_failed;
    __shared__ ChunkSegment s_segment[kCkSegments];
    __shared__ int s_bad[kCkBadRing];                       // per step: bit 0 / 1 when the entry of its first / second page is bad
    __shared__ volatile int s_flawed[kCkFlawRing];          // whose notes s_flaw holds: that segment's number + 1 (0: nobody's)
    __shared__ int s_flaw[kCkFlawRing][kD];                 // per channel: the first token whose value there is no number
    __shared__ float2 s_ml[2][128];                         // (reference, sum) of both warpgroups' rows where they are joined
    const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_smem = base, ring = base + 2 * kRowTileBytes;
    const uint32_t full = smem_u32(s_full), empty = smem_u32(s_empty), scores = smem_u32(s_scores), probs = smem_u32(s_probs),
                   done = smem_u32(s_done), halves = smem_u32(s_halves), qfull = smem_u32(s_qfull), qempty = smem_u32(s_qempty),
                   edge_bar = smem_u32(s_edge), join = smem_u32(&s_join), seg_full = smem_u32(s_segfull), seg_empty = smem_u32(s_segempty);

    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];\nprefetch.tensormap [%2];\n" ::"l"(&k_map), "l"(&v_map), "l"(&q_map) : "memory");
        for (int i = 0; i < kCkStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(scores + 8 * i, 1);
            mbar_init(probs + 16 * i, 4);
            mbar_init(probs + 16 * i + 8, 4);
            mbar_init(done + 8 * i, 1);
            mbar_init(halves + 8 * i, 1);
            mbar_init(qfull + 8 * i, 1);
            mbar_init(qempty + 8 * i, 1);
        }
        for (int i = 0; i < kCkEdges; ++i) mbar_init(edge_bar + 8 * i, 1);
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
    const uint32_t tmem = __shfl_sync(kFull, s_tmem, 0);
    // columns: S of warpgroup i at 128 i (P over it), O at 256 + 128 i
    pdl_launch_dependents();
    if (warp < 8)   // (fetches the code)
        chunk_softmax(tmem + ((uint32_t)(warp & 3) << 21), 0u, 0.f, 0.f, p.logit_scale, -1, -1, true, 0u, 0u, 0u);
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
    using Micro = ChunkMicro<128>;

    if (warp == 10) {
        // ---- this CTA's share, and the queries of its segments: a row tile is a box of T1 tokens and G heads.  Rows of the box behind the
        // sequence's are other sequences' or zeros, and rows of the tile behind the box are left over: what becomes of them is not used.
        ChunkCut cut[2];
        {
            auto cost = [&](int b) { return ChunkTiles<2>(chunk_seq(p.r, b), T1).cost(); };
            WarpScan<decltype(cost)> scan(p.r.batch, cost, lane);
            const long long total = scan.total * p.Hkv;
            const int parts = (int)max(1LL, min((long long)gridDim.x, total >> kCkMinShift)), c = blockIdx.x;
            if (c == 0 && lane == 0) *p.parts = total > 0 ? parts : 0;
            cut[0] = cut[1] = ChunkCut{p.r.batch, 0, 0, 0};
            if (c < parts && total > 0) {
                const long long each = quick_div(total, parts), more = total - each * parts;
#pragma unroll 1
                for (int i = 0; i < 2; ++i) cut[i] = chunk_cut<2>(p.r, scan, p.Hkv, T1, each * (c + i) + min((long long)(c + i), more));
                if (lane == 0) {
                    p.cuts[c] = cut[0];
                    if (c + 1 == parts) p.cuts[parts] = cut[1];
                }
            }
        }
        ChunkWalk<2> walk(p.r, T1, cut[0], cut[1]);
        uint32_t uses0 = 0, uses1 = 0;
        bool ok = true;
#pragma unroll 1
        for (int i = 0;; ++i) {
            if (i >= kCkSegments) ok = wait(seg_empty + 8 * (i % kCkSegments), (i / kCkSegments - 1) & 1);
            if (!ok) break;
            const bool end = walk.done();
            const int token = walk.token0(T1);
            if (lane == 0) {
                ChunkSegment s;
                s.b = walk.at.b;
                s.g = walk.at.g;
                s.step = walk.at.step;
                s.count = end ? 0 : walk.count();
                s.single = walk.single;
                s.slot = 2 * blockIdx.x + (walk.at.step == 0);
                s.whole = walk.at.step == 0 && walk.last == walk.steps;
                s.pos = walk.s.first + token;
                s.tokens = walk.s.n - token;
                s.row = walk.s.row0 + token;
                s.len = walk.s.len;
                s_segment[i % kCkSegments] = s;
                mbar_arrive(seg_full + 8 * (i % kCkSegments));
            }
            __syncwarp();
            if (end) break;
            for (int r = 0; r < (walk.single ? 1 : 2) && ok; ++r) {
                uint32_t& uses = r ? uses1 : uses0;
                if (uses > 0) ok = wait(qempty + 8 * r, (uses - 1) & 1);
                if (!ok) break;
                if (elect_one()) {
                    mbar_expect(qfull + 8 * r, 2 * T1 * p.G * 128);
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        tma_load_3d(q_smem + r * kRowTileBytes + half * kRowTileHalf, &q_map, 64 * half, walk.at.g * p.G,
                                    walk.s.row0 + token + r * T1, qfull + 8 * r);
                }
                __syncwarp();
                ++uses;
            }
            if (!ok) break;
            walk.next(p.r, p.Hkv, T1);
        }
        if (uses0) mbar_wait(qfull, (uses0 - 1) & 1);
        if (uses1) mbar_wait(qfull + 8, (uses1 - 1) & 1);
    } else if (warp == 8) {
        // ---- keys and values: the ring's entries in order of use
        struct Pages { int b, from, page; };
        Pages pages[2] = {{-1, 0, 0}, {-1, 0, 0}};       // of keys and of values; lane x: the page of block from + x
        int issued = 0, edges = 0;
        const int oob = p.r.num_pages * p.Hkv * kBlk;    // a row behind the pool: TMA fills zeros
        auto load = [&](const CUtensorMap* map, const Micro& m, Pages& pg, bool keys) {
            if (m.r) return true;
            const int st = issued % kCkStages, round = issued / kCkStages;
            if (round > 0 && !wait(empty + 8 * st, (round - 1) & 1)) return false;
            const int first = m.key0() >> 6;
            if (pg.b != m.s.b || first < pg.from || first + 1 >= pg.from + 32) {
                pg.b = m.s.b;
                pg.from = first;
                pg.page = -2;                               // behind the last token: no rows
                if ((long long)(first + lane) * kBlk < m.s.len) {
                    pg.page = chunk_page(p.r, pg.b, first + lane);
                    if (pg.page < 0) atomicOr(p.r.status, kDevBadPage);
                }
            }
            const int page0 = __shfl_sync(kFull, pg.page, first - pg.from), page1 = __shfl_sync(kFull, pg.page, first - pg.from + 1);
            const bool hidden = !keys && m.edge();      // warp 11 has it first, and says `full`
            const uint32_t bar = hidden ? edge_bar + 8 * (edges % kCkEdges) : full + 8 * st;
            edges += hidden;
            if (elect_one()) {
                const uint32_t dst = ring + st * kRowTileBytes;
                const int y0 = page0 >= 0 ? (page0 * p.Hkv + m.s.g) * kBlk : oob, y1 = page1 >= 0 ? (page1 * p.Hkv + m.s.g) * kBlk : oob;
                if (keys) s_bad[m.step % kCkBadRing] = (page0 == -1 ? 1 : 0) | (page1 == -1 ? 2 : 0);   // read behind `full` and `scores`
                mbar_expect(bar, kRowTileBytes);
                tma_load(dst, map, 0, y0, bar);
                tma_load(dst + 64 * 128, map, 0, y1, bar);
                tma_load(dst + kRowTileHalf, map, 64, y0, bar);
                tma_load(dst + kRowTileHalf + 64 * 128, map, 64, y1, bar);
            }
            __syncwarp();
            ++issued;
            return true;
        };
        chunk_order<128, 2>(look, take, [&](const Micro& m) { return load(&k_map, m, pages[0], true); },
                    [&](const Micro& m) { return load(&v_map, m, pages[1], false); });
        // nothing may write into this CTA's shared memory once it has left, whatever became of the other roles
        for (int i = max(0, edges - kCkEdges); i < edges; ++i) mbar_wait(edge_bar + 8 * (i % kCkEdges), (i / kCkEdges) & 1);
        for (int i = max(0, issued - kCkStages); i < issued; ++i) mbar_wait(full + 8 * (i % kCkStages), (i / kCkStages) & 1);
    } else if (warp == 9) {
        // ---- products.  The warp shares its scheduler with two softmax warps, and what it does between a warpgroup's weights and its next
        // scores is in that warpgroup's way: so the loops over a segment's steps know all they need, and the general order is for
        // the two micro-steps of scores that run into the next segment.
        int used = 0, kc = 0;                  // ring entries
        uint32_t q_uses0 = 0, q_uses1 = 0, phases = 0, x = 0;   // phases: bit i for warpgroup i
        Micro k;                               // the micro-step of the next scores, where they are not this segment's
        bool ok = true;
        auto ready = [&](int e) { return wait(full + 8 * (e % kCkStages), (e / kCkStages) & 1); };
        auto entry = [&](int e) { return ring + (e % kCkStages) * kRowTileBytes; };
        auto issue_scores = [&](int i, int r, int e, bool q_ends, bool k_ends) {
            const uint64_t a = mma_desc(q_smem + r * kRowTileBytes, 16, 1024), b = mma_desc(entry(e), 16, 1024);
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    const uint32_t at = ((ks >> 2) * kRowTileHalf + (ks & 3) * 32) >> 4;   // in the descriptor's units
                    mma_ss(tmem + 128 * i, a + at, b + at, kIdesc, ks > 0);
                }
                mma_commit(scores + 8 * i);
                if (q_ends) mma_commit(qempty + 8 * r);
                if (k_ends) mma_commit(empty + 8 * (e % kCkStages));
            }
            __syncwarp();
        };
        auto next_scores = [&]() {
            if (!k.live()) return true;
            if (k.r == 0) {
                kc = used++;
                if (!ready(kc)) return false;
            }
            if (k.t == 0) {
                uint32_t& uses = k.r ? q_uses1 : q_uses0;
                if (!wait(qfull + 8 * k.r, uses++ & 1)) return false;
            }
            tmem_after_sync();
            issue_scores(k.x & 1, k.r, kc, k.t == k.s.count - 1, k.step_ends());
            k.advance(look);
            return true;
        };
        auto commit = [&](uint32_t bar) {
            if (elect_one()) mma_commit(bar);
            __syncwarp();
        };
        k.begin(look);
        ok = next_scores() && next_scores();
#pragma unroll 1
        for (int segment = 0; ok; ++segment) {
            const ChunkSegment s = take(segment);
            const int n = s.count, ahead = s.single ? 2 : 1;   // steps between P V and scores
            if (n == 0) break;
#pragma unroll 1
            for (int t = 0; t < n; ++t) {
                const int vc = used++;
                const bool more = t + ahead < n, opens = t < ahead;
                if (more) {
                    kc = used++;
                } else if (t + ahead == n && n > ahead) {   // k still stands where this segment's scores went on: at the next segment now
                    k.x = x + 2;
                    k.r = k.t = 0;
                    k.s = look(++k.segment);
                }
                const uint32_t v_bar = 8 * (vc % kCkStages), v_parity = (vc / kCkStages) & 1, k_bar = 8 * (kc % kCkStages), k_parity = (kc / kCkStages) & 1;
                const uint64_t vd = mma_desc(entry(vc), kRowTileHalf, 1024), kd = mma_desc(entry(kc), 16, 1024);
                const int rows = s.single ? 1 : 2;
                const bool q_ends = t + ahead + 1 == n;
#pragma unroll 1
                for (int r = 0; r < rows; ++r) {
                    // O += P V, each half of the step's tokens as soon as its weights are there, and the scores of the micro-step after the
                    // next.  A barrier answers after 130 cycles even if it was passed long ago: those of a micro-step are asked
                    // together (3710 cycles a step instead of 3840).
                    const int i = x & 1;
                    const uint32_t p_col = tmem + 128 * i, o_col = p_col + 256, bar = probs + 16 * i, parity = phases >> i & 1;
                    phases ^= 1u << i;
                    bool there = mbar_try(bar, parity);
                    if (r == 0) {
                        const bool v_there = mbar_try(full + v_bar, v_parity), k_there = !more || mbar_try(full + k_bar, k_parity);
                        there = there && v_there && k_there;
                    }
                    if (!__all_sync(kFull, there)) {
                        ok = (r || (ready(vc) && (!more || ready(kc)))) && wait(bar, parity);
                        if (!ok) break;
                    }
                    tmem_after_sync();
                    if (elect_one()) {
#pragma unroll
                        for (int y = 0; y < 4; ++y) mma_ts(o_col, p_col + 8 * y, vd + (y * 2048 >> 4), kIdescMnB, y ? true : !opens);
                        mma_commit(halves + 8 * i);
                    }
                    __syncwarp();
                    ok = wait(bar + 8, parity);
                    if (!ok) break;
                    tmem_after_sync();
                    if (elect_one()) {
#pragma unroll
                        for (int y = 0; y < 4; ++y) mma_ts(o_col, p_col + 64 + 8 * y, vd + ((4 + y) * 2048 >> 4), kIdescMnB, true);
                        if (more) {
                            const uint64_t qd = mma_desc(q_smem + r * kRowTileBytes, 16, 1024);
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks) {
                                const uint32_t at = ((ks >> 2) * kRowTileHalf + (ks & 3) * 32) >> 4;   // in the descriptor's units
                                mma_ss(p_col, qd + at, kd + at, kIdesc, ks > 0);
                            }
                            mma_commit(scores + 8 * i);
                            if (q_ends) mma_commit(qempty + 8 * r);
                            if (r + 1 == rows) mma_commit(empty + k_bar);
                        } else {
                            mma_commit(done + 8 * i);
                        }
                        if (r + 1 == rows) mma_commit(empty + v_bar);
                    }
                    __syncwarp();
                    if (!more) {
                        ok = next_scores();
                        if (!ok) break;
                    }
                    ++x;
                }
                if (!ok) break;
            }
        }
        if (!ok) {   // products in flight still write tensor memory
            commit(smem_u32(&s_drain));
            mbar_wait(smem_u32(&s_drain), 0);
        }
    } else if (warp == 11) {
        // ---- values that some of a tile's rows do not see: those of its tokens behind the first.  What is no number there is noted, and
        // the rows that see it get NaN from the results' code.  A buffer's notes carry their segment's number, as a segment without
        // such tokens never comes by here to take older ones away.
        int edges = 0, step0 = 0;
        bool ok = true;
        ChunkSegment s = look(0);
#pragma unroll 1
        for (int segment = 0; ok && s.count > 0; ++segment) {
            const ChunkSegment next = look(segment + 1);
            const int buffer = segment % kCkFlawRing;
            const int first = max(0, (s.pos >> 7) - s.step);     // steps before it are seen by all rows
            bool fresh = true;
#pragma unroll 1
            for (int t = first; t < s.count; ++t) {
                const int key0 = (s.step + t) * 128;
                if (key0 + 127 <= s.pos) continue;
                if (!wait(edge_bar + 8 * (edges % kCkEdges), (edges / kCkEdges) & 1)) {
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
                // The ring's entry: step j's V is behind the keys of the steps before it, its own, and where the scores are a step ahead
                // of the values (a tile with one row tile) those of the next step, if there is one.
                const int j = step0 + t, vc = 2 * j + 1 + (s.single && (t + 1 < s.count || next.count > 0));
                const int x0 = max(0, s.pos + 1 - key0), x1 = min(128, s.pos + min(2 * T1, s.tokens) - key0);
                if (hide_values<128>(ring + (vc % kCkStages) * kRowTileBytes, x0, x1, key0, s_flaw[buffer], lane) && lane == 0)
                    s_flawed[buffer] = segment + 1;
                __threadfence_block();
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(full + 8 * (vc % kCkStages));
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(seg_empty + 8 * (segment % kCkSegments));
            step0 += s.count;
            s = next;
        }
        __syncwarp();
    } else {
        // ---- softmax and results
        const int i = warp >> 2, quarter = warp & 3, row = tid & 127;
        const int tok = row / p.G, h = row - tok * p.G;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t s_col = tmem + 128 * i + lanes, o_col = tmem + 256 + 128 * i + lanes;
        uint32_t n = 0, closed = 0, joined = 0;   // micro-steps and segments of this warpgroup, phases of `join`
        int x0 = 0, step0 = 0;                    // of the share: micro-steps and steps before the present segment
        bool ok = true;
#pragma unroll 1
        for (int segment = 0; ok; ++segment) {
            const ChunkSegment s = take(segment);
            if (s.count == 0) break;
            const int mine = i ^ (x0 & 1);
            const int r = s.single ? 0 : mine, t0 = s.single ? mine : 0, stride = s.single ? 2 : 1;
            const int token = r * T1 + tok;                                       // of the tile
            const bool exists = tok < T1 && token < s.tokens;
            const bool active = __any_sync(kFull, exists);
            const int sees = exists ? s.pos + token + 1 : 0;
            float m = -INFINITY, l = 0.f;
#pragma unroll 1
            for (int t = t0; t < s.count; t += stride, ++n) {
                ok = wait(scores + 8 * i, n & 1);
                if (!ok) break;
                tmem_after_sync();
                if (active) {   // no logits: tokens behind the row's own, or a bad page's rows of zeros
                    const int left = max(0, sees - (s.step + t) * 128), bad = s_bad[(step0 + t) % kCkBadRing];
                    const int keep0 = bad & 1 ? 0 : min(left, 64), keep1 = bad & 2 ? 0 : min(max(left - 64, 0), 64);
                    const float2 ml = chunk_softmax(s_col, o_col, m, l, p.logit_scale, keep0, keep1, t == t0, probs + 16 * i, halves + 8 * i, n & 1);
                    m = ml.x;
                    l = ml.y;
                    if (__any_sync(kFull, m != m)) {   // its wait ran out
                        s_failed = 1;
                        ok = false;
                        break;
                    }
                } else {
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(probs + 16 * i);
                        mbar_arrive(probs + 16 * i + 8);
                    }
                }
            }
            if (!ok) break;
            if (t0 < s.count) {
                ok = wait(done + 8 * i, closed++ & 1);
                if (!ok) break;
                tmem_after_sync();
                const bool both = s.single && s.count > 1;   // the other warpgroup has results of the same rows
                float fa = 1.f, fb = 0.f, top = m, sum = l;
                if (both) {
                    s_ml[i][row] = make_float2(m, l);
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(join);
                    ok = wait(join, joined++ & 1);
                    if (!ok) break;
                    tmem_after_sync();
                    const float2 o = s_ml[i ^ 1][row];
                    top = fmaxf(m, o.x);
                    const float use = top == -INFINITY ? 0.f : top;
                    fa = fast_ex2(m - use);
                    fb = fast_ex2(o.x - use);
                    sum = fa * l + fb * o.y;
                }
                const bool some = sum != 0.f;
                const bool whole = s.whole;
                const float norm = some ? 1.f / sum : 0.f;
                fa *= norm;
                fb *= norm;
                const int part_row = s.slot * kCkRows + r * 128 + row;
                const int at = whole ? (s.row + token) * p.Hq + s.g * p.G + h : part_row;   // (heads of all rows: below 2^31)
                if (exists && (!both || i == 0)) {
                    const float log2_sum = some ? top + log2f(sum) : -INFINITY;
                    if (!whole) p.part_lse[part_row] = log2_sum;
                    else if (p.lse) p.lse[at] = log2_sum * kLn2;
                }
                if (active) {
                    const bool fp32 = !whole;                        // (partial results are)
                    char* const to = static_cast<char*>(whole ? p.out : p.part_out) + (size_t)(unsigned)at * (kD * (fp32 ? 4 : 2));
                    const bool sectors = (reinterpret_cast<uintptr_t>(to) & 31) == 0;
                    const bool flawed = s_flawed[segment % kCkFlawRing] == segment + 1;
                    const int c0 = both ? 64 * i : 0, c1 = both ? c0 + 64 : 128;
#pragma unroll 1
                    for (int c = c0; c < c1; c += 32) {
                        float o[32];
                        tmem_ld32(o_col + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = some ? o[x] * fa : 0.f;
                        if (both) {
                            float o2[32];
                            tmem_ld32(tmem + 256 + 128 * (i ^ 1) + lanes + c, o2);
                            tmem_wait_ld();
#pragma unroll
                            for (int x = 0; x < 32; ++x) o[x] += some ? o2[x] * fb : 0.f;
                        }
                        if (flawed) {
#pragma unroll
                            for (int x = 0; x < 32; ++x) o[x] = s_flaw[segment % kCkFlawRing][c + x] < sees ? NAN : o[x];
                        }
                        if (!exists) continue;
                        uint32_t w[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) w[x] = fp32 ? __float_as_uint(o[x]) : pack_bf16(o[2 * x], o[2 * x + 1]);
                        char* const here = to + c * (fp32 ? 4 : 2);
                        store_sector(here, w, sectors);
                        store_sector(here + 32, w + 8, sectors);
                        if (fp32) {
                            store_sector(here + 64, reinterpret_cast<const uint32_t*>(o + 16), sectors);
                            store_sector(here + 96, reinterpret_cast<const uint32_t*>(o + 24), sectors);
                        }
                    }
                }
                if (both) {   // the columns may be written again when both have read them
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(join);
                    ok = wait(join, joined++ & 1);
                }
            }
            x0 += s.single ? s.count : 2 * s.count;
            step0 += s.count;
        }
    }
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    if (tid == 0 && s_failed) atomicOr(p.r.status, kDevTimeout);
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
}

// Tiles that a cut falls into: eight CTAs for every cut, and the first cut inside a tile joins its partial results.  A warp has four
// rows, a lane four channels of each; the loads of two partial results for all of them are on their way at once (one row after the
// other, 147 tiles of two parts took 17 us).
constexpr int kCkMergeWarps = 8, kCkMergeCtas = 8;

template <int R>      // row tiles of a tile
__global__ void __launch_bounds__(kCkMergeWarps * 32) chunk_merge_kernel(const __grid_constant__ ChunkParams p) {
    constexpr int kCkMergeRows = 128 * R / (kCkMergeWarps * kCkMergeCtas);
    pdl_launch_dependents();
    pdl_wait();
    const int c = blockIdx.x + 1, parts = *p.parts, lane = threadIdx.x & 31;
    if (c >= parts) return;
    const ChunkCut cut = p.cuts[c], before = p.cuts[c - 1];
    if (cut.step == 0 || (before.same_tile(cut) && before.step > 0)) return;
    int end = c + 1;                                      // shares c - 1 .. end - 1 have the tile's steps, or none
    while (end < parts && p.cuts[end].same_tile(cut)) ++end;
    const ChunkSeq s = chunk_seq(p.r, cut.b);
    const int first = blockIdx.y * kCkMergeWarps + (threadIdx.x >> 5);
    int at[kCkMergeRows];                                 // (row, head) of the results; -1: no such row
    bool any = false;
#pragma unroll
    for (int x = 0; x < kCkMergeRows; ++x) {
        const int row = first + x * kCkMergeCtas * kCkMergeWarps, tok = (row & 127) / p.G, h = (row & 127) - tok * p.G;
        const int token = cut.j * R * p.T1 + (row >> 7) * p.T1 + tok;
        at[x] = tok < p.T1 && token < s.n ? (s.row0 + token) * p.Hq + cut.g * p.G + h : -1;
        any |= at[x] >= 0;
    }
    if (!any) return;
    float top[kCkMergeRows], sum[kCkMergeRows];
    float4 acc[kCkMergeRows];
#pragma unroll
    for (int x = 0; x < kCkMergeRows; ++x) {
        top[x] = -INFINITY;
        sum[x] = 0.f;
        acc[x] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll 1
    for (int k0 = c - 1; k0 < end; k0 += 2) {
        float lse[2][kCkMergeRows];
        float4 o[2][kCkMergeRows];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int k = k0 + y;
            const bool there = k < end && (k < c || !(p.cuts[k] == p.cuts[k + 1]));   // (not an empty share)
            const size_t base = (size_t)(2 * k + (k < c)) * kCkRows + first;
#pragma unroll
            for (int x = 0; x < kCkMergeRows; ++x) {
                lse[y][x] = -INFINITY;
                o[y][x] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (there && at[x] >= 0) {
                    const size_t row = base + x * kCkMergeCtas * kCkMergeWarps;
                    lse[y][x] = p.part_lse[row];
                    o[y][x] = *reinterpret_cast<const float4*>(p.part_out + row * kD + 4 * lane);
                }
            }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int x = 0; x < kCkMergeRows; ++x) {
                if (lse[y][x] == -INFINITY) continue;
                const float raised = fmaxf(top[x], lse[y][x]), keep = fast_ex2(top[x] - raised), f = fast_ex2(lse[y][x] - raised);
                top[x] = raised;
                sum[x] = sum[x] * keep + f;
                acc[x].x = acc[x].x * keep + f * o[y][x].x;
                acc[x].y = acc[x].y * keep + f * o[y][x].y;
                acc[x].z = acc[x].z * keep + f * o[y][x].z;
                acc[x].w = acc[x].w * keep + f * o[y][x].w;
            }
    }
#pragma unroll
    for (int x = 0; x < kCkMergeRows; ++x) {
        if (at[x] < 0) continue;
        const float norm = sum[x] != 0.f ? 1.f / sum[x] : 0.f;
        const size_t to = (size_t)at[x] * kD + 4 * lane;
        const float4 v = make_float4(acc[x].x * norm, acc[x].y * norm, acc[x].z * norm, acc[x].w * norm);
        if (p.out_fp32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = v;
        else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + to) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        if (lane == 0 && p.lse) p.lse[at[x]] = sum[x] != 0.f ? (top[x] + log2f(sum[x])) * kLn2 : -INFINITY;
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------------

struct ChunkPlan {
    size_t off_cuts, off_lse, off_out, total;
};
static ChunkPlan chunk_plan(int sms) {
    ChunkPlan pl;
    pl.off_cuts = align_up(kInitBytes, 256);          // (the number of shares in front of them)
    pl.off_lse = align_up(pl.off_cuts + 256 + ((size_t)sms + 1) * sizeof(ChunkCut), 256);
    pl.off_out = pl.off_lse + (size_t)2 * sms * kCkRows * sizeof(float);
    pl.total = pl.off_out + (size_t)2 * sms * kCkRows * kD * sizeof(float);
    return pl;
}

}  // namespace ffd

using namespace ffd;

extern "C" {

ffd_status ffd_workspace_bytes_chunk(const ffd_config* cfg, int32_t batch, int32_t num_rows, int32_t max_blocks_per_seq, size_t* bytes) {
    ffd_status st = check_chunk(cfg, batch, num_rows, max_blocks_per_seq, 1);
    if (st) return st;
    if (!bytes) return FFD_ERR_NULL;
    *bytes = chunk_plan(device_sms()).total;
    return FFD_OK;
}

ffd_status ffd_attend_chunk(const ffd_config* cfg, const void* q, const void* k_cache, const void* v_cache, const int32_t* block_table,
                            const int32_t* row_start, const int32_t* first_token, const int32_t* seq_lens, int32_t num_rows,
                            int32_t batch, int32_t max_blocks_per_seq, int32_t num_pages, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, void* stream) {
    ffd_status st = check_chunk(cfg, batch, num_rows, max_blocks_per_seq, num_pages);
    if (st) return st;
    if (!q || !k_cache || !v_cache || !seq_lens || !out || !workspace) return FFD_ERR_NULL;
    if ((row_start == nullptr) != (first_token == nullptr)) return FFD_ERR_NULL;
    if (!row_start && num_rows != batch) return FFD_ERR_SHAPE;
    if (any_misaligned(q, k_cache, v_cache, block_table, row_start, first_token, seq_lens, out, lse, workspace)) return FFD_ERR_ALIGN;
    const int sms = device_sms();
    const ChunkPlan pl = chunk_plan(sms);
    if (workspace_bytes < pl.total) return FFD_ERR_WORKSPACE;
    char* const ws = static_cast<char*>(workspace);
    ChunkParams p;
    memset(&p, 0, sizeof p);
    p.r = ChunkRows{row_start, first_token, seq_lens, block_table, reinterpret_cast<uint32_t*>(ws), num_rows, batch, max_blocks_per_seq, num_pages};
    p.Hq = cfg->num_q_heads;
    p.Hkv = cfg->num_kv_heads;
    p.G = p.Hq / p.Hkv;
    p.T1 = 128 / p.G;
    p.logit_scale = logit_scale_of(cfg);
    p.out = out;
    p.lse = lse;
    p.out_fp32 = cfg->out_dtype;
    p.parts = reinterpret_cast<int*>(ws + pl.off_cuts);
    p.cuts = reinterpret_cast<ChunkCut*>(ws + pl.off_cuts + 256);
    p.part_lse = reinterpret_cast<float*>(ws + pl.off_lse);
    p.part_out = reinterpret_cast<float*>(ws + pl.off_out);
    const EncodeTiled encode = encode_tiled();
    if (!encode) return FFD_ERR_CUDA;
    CUtensorMap k_map, v_map, q_map;
    const long long rows = (long long)num_pages * p.Hkv * kBlk;
    if (!page_map(encode, &k_map, k_cache, rows) || !page_map(encode, &v_map, v_cache, rows) ||
        !rows_map(encode, &q_map, q, p.Hq, p.G, num_rows))
        return FFD_ERR_CUDA;
    void (*const kernel)(CUtensorMap, CUtensorMap, CUtensorMap, ChunkParams) = p.out_fp32 ? chunk_attention_fp32_kernel : chunk_attention_kernel;
    const int smem = p.out_fp32 ? kC32Smem : kCkSmem;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return FFD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    launch_pdl(kernel, dim3(sms), dim3(kCkThreads), smem, s, k_map, v_map, q_map, p);
    st = launch_status();
    if (st || sms == 1) return st;
    launch_pdl(p.out_fp32 ? chunk_merge_kernel<1> : chunk_merge_kernel<2>, dim3(sms - 1, kCkMergeCtas), dim3(kCkMergeWarps * 32), 0, s, p);
    return launch_status();
}

}  // extern "C"
