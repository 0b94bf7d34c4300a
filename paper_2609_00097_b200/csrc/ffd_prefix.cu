// Decode attention over a prefix that all sequences of a batch share, as matrix products: the batch * G query rows of a KV
// head form tiles of 128 rows, so that every key and value of the prefix is read once for all sequences.
//
// One CTA per SM: warps 0..3 and 4..7 are two softmax warpgroups (a thread owns one row: no shuffles), warp 8
// moves K and V with TMA, warp 9 issues tcgen05.mma.  Per step of 128 tokens and row tile:
//   S = Q K^T   A = Q and B = K in shared memory (K-major, 128-byte swizzle), S in 128 columns of TMEM
//   P = 2^(c S - m), rounded to bf16, written over the columns of S in two halves, each multiplied as soon as it is there
//   O += P V    A = P in TMEM, B = V in shared memory (its channels are contiguous: MN-major), O in 128 columns of TMEM
// The running maximum is raised, and O rescaled in TMEM, only when a row's logits exceed it by 2^8: the sums stay in
// binary32 and the quotient does not change.  A second bf16 piece of P (the remainder of the rounding, a second chain of
// products) keeps 16 bits of it wherever the tensor pipe has time to spare (one row tile: memory is the bound) and when the
// result is wanted in fp32.
//
// What bounds it: one tile, the loads of K and V (16 sequences on 32 K, 32 query and 8 KV heads: 6.1 TB/s in the steps).  Two
// tiles, per step of 256 x 128 weights and 3350 cycles: neither the exponential unit (2048) nor the tensor pipe (16.8 MFLOP at 8192
// a cycle: 2048; 2130 counted) is busy for more than two thirds of it, and operands from shared memory keep up with the pipe.
// What is left is latency: a warpgroup's chain of scores, softmax, second half of P V and next scores is longer than the other
// warpgroup's work that should cover it.  With two pieces of P the tensor pipe has half as much work again.  In a long series
// of calls power counts too (64 sequences on 128 K: 1.5 GHz at 990 W).  About 12000 cycles of a CTA are neither: the query and the
// first keys on their way in, the results on their way out.
// Powers by polynomial on the FMA pipes, for a part of the weights, took longer.  So did scores in halves of 64 tokens, so that a
// warpgroup never waits for its next ones: the query is then read twice as often, and 48 KB of operands take 384 cycles of shared
// memory for 256 of products (128 sequences on 8 K: 80 us instead of 62).
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>

#include <atomic>

#include "ffd_host.cuh"
#include "ffd_kernels.cuh"
#include "ffd_own.cuh"
#include "ffd_prefix.cuh"
#include "ffd_prefix_step.cuh"

namespace ffd {

constexpr int kPfThreads = 384;                          // three warpgroups; of the third, two warps work
constexpr int kPfTileBytes = kPrefixTokens * kD * 2;      // 32 KB: 128 rows of Q, or a step's K or V
constexpr int kPfHalfBytes = kPfTileBytes / 2;            // 64 channels of it
__host__ __device__ constexpr int pf_stages(int tiles) { return tiles == 1 ? 6 : 5; }
__host__ __device__ constexpr int pf_smem(int tiles) { return (tiles + pf_stages(tiles)) * kPfTileBytes + 1024; }
constexpr int kPfTeams = kPfThreads / 128;                // of a CTA that works on own tokens
constexpr int kPfOutRow = kD * 4 + 16;                    // bytes of a row of results in shared memory: 16 more, against bank conflicts
static_assert(kPfTeams * Paged<kFmtInt8>::kSmem <= pf_smem(1) && kPfTeams * Paged<kFmtBf16>::kSmem <= pf_smem(1) &&
              pf_smem(1) == pf_smem(2), "the teams' rings take the tiles' place");
static_assert(2 * kPrefixRows * kPfOutRow <= pf_smem(2) - 1024, "and so do the results on their way out");

// steps of which the loads can be ahead of the softmax: at most the ring's entries and the two steps whose scores exist
constexpr int kPfBadRing = 16;

// ---- tcgen05 -----------------------------------------------------------------------------------------------------------

// shared-memory matrix descriptor, 128-byte swizzle: start, leading and stride offsets in 16-byte units, version 1
__device__ __forceinline__ uint64_t mma_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp32 accumulators, bf16 operands, M = 128, N = 128; B K-major or MN-major
constexpr uint32_t kIdesc = 1u << 4 | 1u << 7 | 1u << 10 | (128u >> 3) << 17 | (128u >> 4) << 24;
constexpr uint32_t kIdescMnB = kIdesc | 1u << 16;

// (every operand of these is the same in all lanes and derived from uniform values, so that it stays in uniform registers)
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// the barrier receives one arrival when all tcgen05 operations that this thread has issued so far are complete
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
}
// one lane of the (converged) warp, without a comparison that the compiler would take for divergence
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
    return p;
}
__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;\n" ::"r"(id), "r"(threads) : "memory"); }

// ---- the kernel -----------------------------------------------------------------------------------------------------------

// How a launch's CTAs divide: Hkv * groups * chunks on the prefix, own_ctas on the sequences' own tokens
struct Split {
    int chunks, own_ctas;
};

// Costs in clock cycles, measured: a CTA takes about kStart to begin and end, kStep per step of 128 prefix tokens, and, with
// its twelve warps on own tokens, kItem per item of each warp.  Lane x tries x + 1, x + 33, ... chunks and the warp takes the
// best: the number for which the longer of the two sides is shortest, the smaller one where it does not matter (fewer partial
// results).
template <int TILES, int PIECES, int FMT, int NH>
__device__ __forceinline__ Split split_of(const PrefixParams& p, const PagedParams& own, int steps, int lane) {
    constexpr int kStart = 12000, kStep = TILES == 1 ? 2400 : PIECES == 1 ? 3350 : 4500;
    constexpr int kItem = FMT == kFmtBf16 ? 2800 : NH == 1 ? 3500 : 7000;   // (of 16 tokens, or of 32 in one or two tiles of heads)
    long long count = 0;
    for (int b = lane; b < own.batch; b += 32)
        count += ceil_shift(paged_len(own.seq_lens, b, own.max_blocks, own.status), Paged<FMT>::kShift);
#pragma unroll
    for (int o = 16; o; o >>= 1) count += __shfl_xor_sync(kFull, count, o);
    const float total = (float)(count * own.Hkv);
    const int base = p.Hkv * p.groups;
    unsigned long long best = ~0ull;
    for (int c = lane + 1; c <= p.chunks; c += 32) {
        const int own_ctas = (int)gridDim.x - base * c;   // at least one
        const float prefix = kStart + (float)((steps + c - 1) / c) * kStep;
        const float items = ceilf(total / (float)(own_ctas * kPrefixCtaParts)), mine = items > 0.f ? kStart + items * kItem : 0.f;
        const unsigned long long key = (unsigned long long)__float_as_uint(fmaxf(prefix, mine)) << 32 | (unsigned)c;
        best = min(best, key);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) best = min(best, __shfl_xor_sync(kFull, best, o));
    Split s;
    s.chunks = (int)(unsigned)best;
    s.own_ctas = (int)gridDim.x - base * s.chunks;
    return s;
}

// One launch for the prefix and for the sequences' own tokens (FMT: their format).  The first CTAs take (KV head, group of row
// tiles, chunk of the prefix), the others are three teams of four warps each that share the own tokens; how many there are of
// each is found on the device from the lengths (split_of), every warp for itself, so that both end at about the same time.
//
// Prefix: TILES 1: row tile `group`; both warpgroups work on it, warpgroup i on steps i, i + 2, ... of the chunk, and their
// results are joined at the end.  TILES 2: row tiles 2 * group + i for warpgroup i, every step for both.  PIECES: bf16 pieces
// of P.
//
// Order of the tensor-core work (one thread issues it, so it runs in this order): S of a warpgroup's next step is issued
// right behind its P V, which frees the columns; while one warpgroup computes its softmax the other's products run.  Loads
// are issued in the order in which that sequence uses them, through one ring for K and V.
//
// Every wait is bounded: if one runs out, the role raises `failed`, all roles leave their loops, the copies in flight are
// waited for (again bounded), TMEM is freed and the status word says FFD_DEV_TIMEOUT.
template <int TILES, int PIECES, int FMT, int NH>
__global__ void __launch_bounds__(kPfThreads, 1) prefix_attention_kernel(const __grid_constant__ CUtensorMap k_map,
                                                                       const __grid_constant__ CUtensorMap v_map,
                                                                       const __grid_constant__ CUtensorMap q_map,
                                                                       const __grid_constant__ PrefixParams p,
                                                                       const __grid_constant__ PagedParams own) {
    constexpr int kStages = pf_stages(TILES);
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_scores[2], s_probs[4], s_done[2], s_halves[2], s_query, s_drain;
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_failed;
    __shared__ TeamShared s_team[kPfTeams];
    __shared__ int s_bad[kPfBadRing];   // per step: bit 0 / 1 when the table's entry for its first / second page is bad
    const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;   // (warp: known to be uniform)
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_smem = base, ring = base + TILES * kPfTileBytes;
    const uint32_t full = smem_u32(s_full), empty = smem_u32(s_empty), scores = smem_u32(s_scores), probs = smem_u32(s_probs),
                   done = smem_u32(s_done), halves = smem_u32(s_halves), query = smem_u32(&s_query);
    const int rows = p.batch * p.G;

    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];\n" ::"l"(&k_map), "l"(&v_map) : "memory");
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(scores + 8 * i, 1);
            mbar_init(probs + 16 * i, 4);
            mbar_init(probs + 16 * i + 8, 4);
            mbar_init(done + 8 * i, 1);
            mbar_init(halves + 8 * i, 1);
        }
        mbar_init(query, p.query_copy ? 1 : 8);
        mbar_init(smem_u32(&s_drain), 1);
        s_failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = __shfl_sync(kFull, s_tmem, 0);
    // TMEM columns: S of warpgroup i at 128 i (P over it), O at 256 + 128 i
    pdl_launch_dependents();
    if (warp < 8 && (int)blockIdx.x < p.Hkv * p.groups * p.chunks)
        softmax_step<PIECES>(tmem + ((uint32_t)(warp & 3) << 21), 0u, 0.f, 0.f, p.logit_scale, -1, -1, false, 0u, 0u, 0u);
    pdl_wait();

    const int len = paged_len(p.len, 0, p.max_blocks, p.status);
    const int steps = ceil_shift(len, 7);
    const Split split = split_of<TILES, PIECES, FMT, NH>(p, own, steps, lane);
    const int items = p.Hkv * p.groups * split.chunks;   // CTAs with a part of the prefix
    if ((int)blockIdx.x >= items) {
        // the pass that fetches code reads TMEM: nothing is freed under it
        tmem_before_sync();
        __syncthreads();
        tmem_after_sync();
        if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
        const int team = warp >> 2;
        attend_own<FMT, NH>(own, split.own_ctas * kPrefixCtaParts, split.chunks, smem_raw + team * Paged<FMT>::kSmem, s_team[team],
                            ((int)blockIdx.x - items) * kPfTeams + team, tid & 127, [team] { named_sync(2 + team, 128); });
        return;
    }
    const int base_items = p.Hkv * p.groups;
    const int chunk = blockIdx.x / base_items, group = blockIdx.x % base_items % p.groups, g = blockIdx.x % base_items / p.groups;
    const int step0 = (int)((long long)steps * chunk / split.chunks), step1 = (int)((long long)steps * (chunk + 1) / split.chunks);
    const int nt = step1 - step0;

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

    if (warp >= 8) {
        if (warp == 8) {
            // ---- loads: the ring's entries in order of use
            int issued = 0, pages = -1, pages_from = -1;
            const int oob = p.num_pages * p.Hkv * kBlk;    // a row behind the pool: TMA fills zeros
            auto load = [&](const CUtensorMap* map, int t, bool keys) {
                const int st = issued % kStages, round = issued / kStages;
                if (round > 0 && !wait(empty + 8 * st, (round - 1) & 1)) return false;
                const int first = 2 * (step0 + t);
                if (pages_from < 0 || first < pages_from || first + 1 >= pages_from + 32) {   // lane x: block first + x
                    pages_from = first;
                    const int blk = first + lane;
                    pages = blk < p.max_blocks && (long long)blk * kBlk < len ? p.table[blk] : -2;
                    if (pages != -2 && (pages < 0 || pages >= p.num_pages)) {
                        atomicOr(p.status, kDevBadPage);
                        pages = -1;
                    }
                }
                const int page0 = __shfl_sync(kFull, pages, first - pages_from), page1 = __shfl_sync(kFull, pages, first - pages_from + 1);
                if (elect_one()) {
                    const uint32_t dst = ring + st * kPfTileBytes, bar = full + 8 * st;
                    const int y0 = page0 >= 0 ? (page0 * p.Hkv + g) * kBlk : oob, y1 = page1 >= 0 ? (page1 * p.Hkv + g) * kBlk : oob;
                    if (keys) s_bad[t % kPfBadRing] = (page0 == -1 ? 1 : 0) | (page1 == -1 ? 2 : 0);   // read behind `full` and `scores`
                    mbar_expect(bar, kPfTileBytes);
                    tma_load(dst, map, 0, y0, bar);
                    tma_load(dst + 64 * 128, map, 0, y1, bar);
                    tma_load(dst + kPfHalfBytes, map, 64, y0, bar);
                    tma_load(dst + kPfHalfBytes + 64 * 128, map, 64, y1, bar);
                }
                __syncwarp();
                ++issued;
                return true;
            };
            if (p.query_copy && elect_one()) {   // the query's tiles: ahead of everything else
                mbar_expect(query, TILES * kPfTileBytes);
#pragma unroll
                for (int i = 0; i < TILES; ++i)
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        tma_load_3d(q_smem + i * kPfTileBytes + half * kPfHalfBytes, &q_map, 64 * half, g * p.G,
                                    (TILES * group + i) * (kPrefixRows / p.G), query);
            }
            __syncwarp();
            bool ok = true;
            if constexpr (TILES == 1) {
                if (nt > 0) ok = load(&k_map, 0, true);
                if (ok && nt > 1) ok = load(&k_map, 1, true);
                for (int t = 0; ok && t < nt; ++t) {
                    ok = load(&v_map, t, false);
                    if (ok && t + 2 < nt) ok = load(&k_map, t + 2, true);
                }
            } else {
                for (int t = 0; ok && t < nt; ++t) ok = load(&k_map, t, true) && load(&v_map, t, false);
            }
            // nothing may write into this CTA's shared memory once it has left, whatever became of the other roles
            mbar_wait(query, 0);
            for (int i = max(0, issued - kStages); i < issued; ++i) mbar_wait(full + 8 * (i % kStages), (i / kStages) & 1);
        } else if (warp == 9) {
            // ---- products
            int used = 0;          // ring entries consumed
            uint32_t steps_done[2] = {0u, 0u};
            auto entry_ready = [&](int e) { return wait(full + 8 * (e % kStages), (e / kStages) & 1); };
            auto entry_addr = [&](int e) { return ring + (e % kStages) * kPfTileBytes; };
            auto qk = [&](int i, int e) {
                const uint64_t a = mma_desc(q_smem + (TILES == 2 ? i : 0) * kPfTileBytes, 16, 1024), b = mma_desc(entry_addr(e), 16, 1024);
                if (elect_one()) {
    #pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        const uint32_t at = ((ks >> 2) * kPfHalfBytes + (ks & 3) * 32) >> 4;   // in the descriptor's units
                        mma_ss(tmem + 128 * i, a + at, b + at, kIdesc, ks > 0);
                    }
                    mma_commit(scores + 8 * i);
                }
                __syncwarp();
            };
            auto pv = [&](int i, int e, int half, bool first) {   // 64 of the step's tokens
                const uint64_t b = mma_desc(entry_addr(e), kPfHalfBytes, 1024);
                if (elect_one()) {
    #pragma unroll
                    for (int piece = 0; piece < PIECES; ++piece)
    #pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mma_ts(tmem + 256 + 128 * i, tmem + 128 * i + 64 * half + 32 * piece + 8 * x, b + ((4 * half + x) * 2048 >> 4),
                                   kIdescMnB, !(first && half == 0 && piece == 0 && x == 0));
                    if (half == 0) mma_commit(halves + 8 * i);
                }
                __syncwarp();
            };
            auto commit = [&](uint32_t bar) {
                if (elect_one()) mma_commit(bar);
                __syncwarp();
            };
            auto release = [&](int e) { commit(empty + 8 * (e % kStages)); };
            // rows of the last step behind the prefix's end: whatever the page holds there must not meet weight 0 as NaN
            auto clean = [&](int e, int t) {
                const int valid = len - (step0 + t) * kPrefixTokens;
                if (valid >= kPrefixTokens) return;
                for (int x = lane; x < (kPrefixTokens - valid) * 16; x += 32) {
                    const uint32_t to = entry_addr(e) + (x & 8 ? kPfHalfBytes : 0) + (valid + (x >> 4)) * 128 + (x & 7) * 16;
                    asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};\n" ::"r"(to), "r"(0u) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                __syncwarp();
            };
            // O += P V of warpgroup i's next step, each half of it as soon as its weights are there
            auto step_pv = [&](int i, int e, bool first) {
                const uint32_t parity = steps_done[i] & 1;
                ++steps_done[i];
    #pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (!wait(probs + 16 * i + 8 * half, parity)) return false;
                    tmem_after_sync();
                    pv(i, e, half, first);
                }
                return true;
            };
            bool ok = wait(query, 0);
            if constexpr (TILES == 1) {
                for (int t = 0; ok && t < 2 && t < nt; ++t) {
                    ok = entry_ready(used);
                    if (!ok) break;
                    tmem_after_sync();
                    qk(t, used);
                    release(used++);
                }
                for (int t = 0; ok && t < nt; ++t) {
                    const int i = t & 1;
                    ok = entry_ready(used);
                    if (!ok) break;
                    clean(used, t);
                    ok = step_pv(i, used, t < 2);
                    if (!ok) break;
                    release(used++);
                    if (t + 2 < nt) {
                        ok = entry_ready(used);
                        if (!ok) break;
                        qk(i, used);
                        release(used++);
                    } else {
                        commit(done + 8 * i);
                    }
                }
            } else {
                if (ok && nt > 0) {
                    ok = entry_ready(0);
                    if (ok) {
                        tmem_after_sync();
                        qk(0, 0);
                        qk(1, 0);
                        release(0);
                    }
                }
                for (int t = 0; ok && t < nt; ++t) {   // entry 2 t: K of step t, 2 t + 1: V
                    ok = entry_ready(2 * t + 1);
                    if (!ok) break;
                    clean(2 * t + 1, t);
                    for (int i = 0; i < 2 && ok; ++i) {
                        ok = step_pv(i, 2 * t + 1, t == 0);
                        if (!ok) break;
                        if (t + 1 < nt) {
                            ok = entry_ready(2 * t + 2);
                            if (ok) qk(i, 2 * t + 2);
                        } else {
                            commit(done + 8 * i);
                        }
                    }
                    if (!ok) break;
                    release(2 * t + 1);
                    if (t + 1 < nt) release(2 * t + 2);
                }
            }
            if (!ok) {   // products in flight still write TMEM
                commit(smem_u32(&s_drain));
                mbar_wait(smem_u32(&s_drain), 0);
            }
        }
    } else {
        // ---- softmax
        const int i = warp >> 2, quarter = warp & 3;
        const int tile = TILES == 2 ? 2 * group + i : group;
        const int row = tile * kPrefixRows + (tid & 127);
        const bool active = tile * kPrefixRows + quarter * 32 < rows;   // does the warp own any row?
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t s_col = tmem + 128 * i + lanes, o_col = tmem + 256 + 128 * i + lanes;
        const int mine = TILES == 2 ? nt : (nt - i + 1) / 2;
        if (!p.query_copy) {   // Q: row b * G + h of KV head g, 16-byte chunks XOR-ed with the row's low bits as the matrix
            // descriptor expects.  TILES 2: a warp has 32 rows and copies two at once (G = 3, 384 rows on 8 K: 44.6 us, against
            // 50.0 us with a thread for each row); TILES 1: a thread has half a row (45.8 against 43.9 us with four rows at once)
            constexpr int kLoads = TILES == 2 ? 16 : 8;
            const int first = TILES == 2 ? row - lane + (lane >> 4) : row;
            int b = first / p.G, h = first - b * p.G;
            uint4 x[kLoads];
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const int c = TILES == 2 ? lane & 15 : 8 * i + n;
                x[n] = make_uint4(0u, 0u, 0u, 0u);
                if (first + (TILES == 2 ? 2 * n : 0) < rows)
                    x[n] = *reinterpret_cast<const uint4*>(p.q + ((size_t)b * p.Hq + (size_t)g * p.G + h) * kD + 8 * c);
                if (TILES == 2 && (h += 2) >= p.G) {   // G is 3 at least: 1 and 2 divide the tile
                    h -= p.G;
                    ++b;
                }
            }
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const int c = TILES == 2 ? lane & 15 : 8 * i + n, r = TILES == 2 ? quarter * 32 + 2 * n + (lane >> 4) : tid & 127;
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};\n" ::"r"(q_smem + (TILES == 2 ? i * kPfTileBytes : 0) +
                                                                           (c >> 3) * kPfHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4)),
                             "r"(x[n].x), "r"(x[n].y), "r"(x[n].z), "r"(x[n].w)
                             : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(query);
        }
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int n = 0; n < mine && ok; ++n) {
            ok = wait(scores + 8 * i, n & 1);
            if (!ok) break;
            tmem_after_sync();
            const int t = TILES == 2 ? n : 2 * n + i;
            const int left = len - (step0 + t) * kPrefixTokens, bad = s_bad[t % kPfBadRing];
            if (active) {   // no logits: behind the prefix's end, or a bad page's rows of zeros
                const int keep0 = bad & 1 ? 0 : min(left, 64), keep1 = bad & 2 ? 0 : min(max(left - 64, 0), 64);
                const float2 ml = softmax_step<PIECES>(s_col, o_col, m, l, p.logit_scale, keep0, keep1, n > 0, probs + 16 * i, halves + 8 * i, n & 1);
                m = ml.x;
                l = ml.y;
                if (m != m) {   // its wait ran out
                    s_failed = 1;
                    ok = false;
                }
            } else {
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(probs + 16 * i);
                    mbar_arrive(probs + 16 * i + 8);
                }
            }
        }
        // The partial: O / l and log2 of the sum of weights.  A thread has a row, memory wants the rows' neighbouring bytes
        // together: the warp's 32 rows go through shared memory, where nothing else is left by now.  (16 bytes a row straight
        // from the threads took 5 us, and so did a bulk copy for each row.)
        if (mine > 0 && ok) ok = wait(done + 8 * i, 0);
        tmem_after_sync();
        if constexpr (TILES == 1) {   // (the warpgroups exchange m and l through the columns of S)
            tmem_st2(s_col, ok ? m : -INFINITY, ok ? l : 0.f);
            tmem_wait_st();
        }
        tmem_before_sync();
        named_sync(1, 256);
        tmem_after_sync();
        const size_t at = ((size_t)g * p.chunks + chunk) * rows + row;
        // TILES 1: both warpgroups' results for the row, each half of the channels by one of them
        constexpr int kCols = TILES == 1 ? 64 : 128;
        const int col0 = TILES == 1 ? 64 * i : 0;
        const bool pair = TILES == 1 && nt > 1;        // (else the second accumulator was never written)
        float fa, fb = 0.f;
        if constexpr (TILES == 1) {
            float a[2], b[2];   // (m, l)
            tmem_ld2(tmem + lanes, a);
            tmem_ld2(tmem + 128 + lanes, b);
            tmem_wait_ld();
            const float top = fmaxf(a[0], b[0]), use = top == -INFINITY ? 0.f : top;
            fa = fast_ex2(a[0] - use);
            fb = fast_ex2(b[0] - use);
            const float sum = fa * a[1] + fb * b[1], norm = sum != 0.f ? 1.f / sum : 0.f;
            fa *= norm;
            fb *= norm;
            if (i == 0 && row < rows) p.lse[at] = sum != 0.f ? use + log2f(sum) : -INFINITY;
        } else {
            const bool some = mine > 0 && ok && l != 0.f;
            fa = some ? 1.f / l : 0.f;
            if (row < rows) p.lse[at] = some ? m + log2f(l) : -INFINITY;
        }
        if (active && nt > 0 && ok) {
            const uint32_t out = base + ((TILES == 2 ? i * kPrefixRows : 0) + (tid & 127)) * kPfOutRow + 4 * col0;
#pragma unroll 1
            for (int c = 0; c < kCols; c += 16) {
                float o[16], o2[16];
                tmem_ld16((TILES == 1 ? tmem + 256 + lanes : o_col) + col0 + c, o);
                if (pair) tmem_ld16(tmem + 384 + lanes + col0 + c, o2);
                tmem_wait_ld();
#pragma unroll
                for (int x = 0; x < 16; ++x) o[x] = fa * o[x] + (pair ? fb * o2[x] : 0.f);
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};\n" ::"r"(out + 4 * c + 16 * x), "f"(o[4 * x]), "f"(o[4 * x + 1]),
                                 "f"(o[4 * x + 2]), "f"(o[4 * x + 3])
                                 : "memory");
            }
            __syncwarp();
            constexpr int kLanes = kCols / 4, kRowsAtOnce = 32 / kLanes;   // lanes that copy a row's piece
            const int row0 = row - lane, sub = lane / kLanes, piece = lane % kLanes;
            const uint32_t in = base + ((TILES == 2 ? i * kPrefixRows : 0) + quarter * 32) * kPfOutRow + 4 * col0 + 16 * piece;
            float* to = p.out + (at - lane) * kD + col0 + 4 * piece;
#pragma unroll 8
            for (int r = sub; r < 32; r += kRowsAtOnce) {
                const uint4 x = lds128(in + r * kPfOutRow);
                if (row0 + r < rows) *reinterpret_cast<uint4*>(to + (size_t)r * kD) = x;
            }
        }
    }
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    if (tid == 0 && s_failed) atomicOr(p.status, kDevTimeout);
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
}

// ---- host side -----------------------------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's function that fills a tensor map; looked up through the runtime, so that the library does not link libcuda.  Its
// address is kept, the same for all devices and calls; a look-up that fails (no driver yet) is tried again by the next call.
static EncodeTiled encode_tiled() {
    static std::atomic<EncodeTiled> found{nullptr};
    EncodeTiled f = found.load(std::memory_order_relaxed);
    if (f) return f;
    void* p = nullptr;
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &got) != cudaSuccess ||
        got != cudaDriverEntryPointSuccess) {
        (void)cudaGetLastError();
        return nullptr;
    }
    f = reinterpret_cast<EncodeTiled>(p);
    found.store(f, std::memory_order_relaxed);
    return f;
}

// a pool of pages as a matrix of 128-channel rows, copied in boxes of 64 rows (a page) by 64 channels
static bool page_map(EncodeTiled encode, CUtensorMap* map, const void* pool, long long rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)kD, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)kD * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)kBlk}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(pool), dims, strides, box, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the queries as [batch][Hq][128], copied in boxes of 64 channels of a row tile: 128 / G sequences, G heads each
static bool query_map(EncodeTiled encode, CUtensorMap* map, const PrefixParams& p) {
    const cuuint64_t dims[3] = {(cuuint64_t)kD, (cuuint64_t)p.Hq, (cuuint64_t)p.batch};
    const cuuint64_t strides[2] = {(cuuint64_t)kD * 2, (cuuint64_t)p.Hq * kD * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)(kPrefixRows / p.G)}, steps[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(p.q), dims, strides, box, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

using PrefixKernel = void (*)(CUtensorMap, CUtensorMap, CUtensorMap, PrefixParams, PagedParams);

template <int TILES, int PIECES, int NH>
static PrefixKernel prefix_kernel(int format) {
    return format == kFmtInt8 ? prefix_attention_kernel<TILES, PIECES, kFmtInt8, NH>
           : format == kFmtE4m3 ? prefix_attention_kernel<TILES, PIECES, kFmtE4m3, NH> : prefix_attention_kernel<TILES, PIECES, kFmtBf16, NH>;
}
template <int TILES, int PIECES>
static PrefixKernel prefix_kernel(int format, int G) {   // tiles of four heads for the own tokens
    return G > 4 ? prefix_kernel<TILES, PIECES, 2>(format) : prefix_kernel<TILES, PIECES, 1>(format);
}

ffd_status launch_prefix(const PrefixParams& p, const PrefixGeometry& geo, const void* k, const void* v, int format,
                         const PagedParams& own, cudaStream_t stream) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return FFD_ERR_CUDA;
    CUtensorMap k_map, v_map;
    const long long rows = (long long)p.num_pages * p.Hkv * kBlk;
    if (!page_map(encode, &k_map, k, rows) || !page_map(encode, &v_map, v, rows)) return FFD_ERR_CUDA;
    CUtensorMap q_map = k_map;   // (not used)
    if (p.query_copy && !query_map(encode, &q_map, p)) return FFD_ERR_CUDA;
    const PrefixKernel kernel = geo.tiles == 1 ? prefix_kernel<1, 2>(format, p.G)
                                : p.two_piece ? prefix_kernel<2, 2>(format, p.G) : prefix_kernel<2, 1>(format, p.G);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, pf_smem(geo.tiles)) != cudaSuccess) return FFD_ERR_CUDA;
    launch_pdl(kernel, dim3(geo.ctas), dim3(kPfThreads), pf_smem(geo.tiles), stream, k_map, v_map, q_map, p, own);
    return launch_status();
}

}  // namespace ffd
