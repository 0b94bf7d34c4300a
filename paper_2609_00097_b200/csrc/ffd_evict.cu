// The attention weight that cached tokens receive, and eviction by it.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "ffd_chunk.cuh"
#include "ffd_host.cuh"
#include "ffd_prefix_step.cuh"
#include "ffd_tensor.cuh"

namespace ffd {

// ---- weighing ---------------------------------------------------------------------------------------------------------------
//
// weight[t] = sum over rows r that see t of 2^(c S[t, r] - lse[r]), S = K Q^T, the product with the keys as the rows: a thread of a
// warpgroup owns a token, its sum over queries is a sum over columns of tensor memory, and nobody has to add to what
// another thread adds to.  An item is 256 tokens of a sequence and KV head, in two tiles, against the row tiles (128 / G tokens
// with G heads) that see them.  Two warpgroups share a tile of tokens, one has the first 64 rows of every row tile and the other
// the rest (with one warpgroup for both, the wait for tensor memory took as long as the powers: 45 us for 64 new tokens on 32 K).  Keys
// are read once; a sequence's queries stay in shared memory from item to item while there are at most two tiles of them, else they
// are read (from L2) for every item.
//
// What bounds it: the keys' bytes for few rows (one token for 16 sequences, 294 MB: 59 us, 0.76 of the measured copy bandwidth, 7 us of
// it before the first keys); for many, one exponential per key and row, 16 a cycle and SM (64 tokens on 32 K: 34 us of which 15 are
// those).  The items, in order, are cut into shares of about the same cost, one for each CTA, with the cost of an item counted in units of 16 cycles:
// kWeighItem for its keys (64 KB), G for every new token that sees it.
constexpr int kWgThreads = 576;                  // four warpgroups, a warp for the copies, one for the products
constexpr int kWgStages = 4;                     // tiles of keys in flight
constexpr int kWgSmem = (2 + kWgStages) * kRowTileBytes + 1024;
constexpr int kWeighItem = 170;

struct WeighParams {
    ChunkRows r;
    int Hq, Hkv, G, T1, add;
    float logit_scale;             // sm_scale * log2(e)
    const float* lse;              // [num_rows, Hq]
    float* weight;                 // [num_pages, Hkv, 64]
};

struct WeighItems {                // of one sequence and KV head
    long long first, n;
    int G, items;
    __device__ __forceinline__ WeighItems(const ChunkSeq& s, int g) : first(s.first), n(s.len - s.first), G(g), items(ceil_shift(s.len, 8)) {}
    // new tokens see item k: n of them where 256 k <= first, first + n - 256 k behind that
    __device__ __forceinline__ long long cost_before(int k) const {
        const long long k0 = first >> 8, more = k - 1 - k0;
        long long seen = k * n;
        if (more > 0) seen -= 128 * ((long long)(k - 1) * k - k0 * (k0 + 1)) - more * first;
        return (long long)k * kWeighItem + G * seen;
    }
};

struct WeighCut {
    int b, g, k;
    __device__ __forceinline__ bool operator==(const WeighCut& o) const { return b == o.b && g == o.g && k == o.k; }
};

template <typename Scan>
__device__ __forceinline__ WeighCut weigh_cut(const WeighParams& p, Scan& scan, long long x) {
    if (x >= scan.total * p.Hkv) return WeighCut{p.r.batch, 0, 0};
    WeighCut c;
    long long off;
    scan.find(x, p.Hkv, c.b, off);
    const WeighItems t(chunk_seq(p.r, c.b), p.G);
    long long y = x - off;
    const long long head = t.cost_before(t.items);
    c.g = (int)(head >> 31 ? y / head : quick_div(y, (int)head));
    y -= c.g * head;
    const int lo = warp_search(t.items, y, [&](int k) { return t.cost_before(k); });
    c.k = lo;
    if (2 * y > t.cost_before(lo) + t.cost_before(lo + 1) && ++c.k == t.items) {
        c.k = 0;
        if (++c.g == p.Hkv) {
            c.g = 0;
            do ++c.b;
            while (c.b < p.r.batch && chunk_seq(p.r, c.b).len == 0);
        }
    }
    return c;
}

struct WeighWalk {
    WeighCut at, end;
    ChunkSeq s;
    int items, tiles, from;      // of the head: items and row tiles; from: the first row tile that sees the item
    bool two;                    // the item has tokens in both tiles
    bool kept;                   // its row tiles are in shared memory already
    bool keep;                   // and are left there for the next item

    __device__ __forceinline__ WeighWalk(const WeighParams& p, const WeighCut& a, const WeighCut& b) : at(a), end(b) {
        kept = keep = false;
        if (at.b < p.r.batch) begin(p);
        settle(p);
    }
    __device__ __forceinline__ bool done() const { return at == end; }
    __device__ __forceinline__ void begin(const WeighParams& p) {
        s = chunk_seq(p.r, at.b);
        items = ceil_shift(s.len, 8);
        tiles = (s.n + p.T1 - 1) / p.T1;
    }
    __device__ __forceinline__ void settle(const WeighParams& p) {
        if (done()) return;
        const int behind = 256 * at.k - s.first;      // (a division only where there is something to divide)
        from = behind >= p.T1 ? min(tiles, behind / p.T1) : 0;
        two = s.len - 256 * at.k > 128;
        const bool same = at.k + 1 < items && !(at.b == end.b && at.g == end.g && at.k + 1 == end.k);   // the next item's head
        keep = same && tiles - from <= 2;
    }
    __device__ __forceinline__ void next(const WeighParams& p) {
        kept = keep;
        if (++at.k == items) {
            at.k = 0;
            if (++at.g == p.Hkv) {
                at.g = 0;
                do {
                    if (++at.b < p.r.batch) begin(p);
                } while (at.b < p.r.batch && s.len == 0);
            }
        }
        settle(p);
    }
    __device__ __forceinline__ int columns(const WeighParams& p, int j) const { return min(p.T1, s.n - j * p.T1) * p.G; }
};

__global__ void __launch_bounds__(kWgThreads, 1) weigh_kernel(const __grid_constant__ CUtensorMap k_map,
                                                             const __grid_constant__ CUtensorMap q_map,
                                                             const __grid_constant__ WeighParams p) {
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kWgStages], s_empty[kWgStages], s_qfull[2], s_qempty[2], s_dfull[4], s_dempty[4], s_drain;
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_failed;
    __shared__ __align__(16) float s_lse[16][2][64];    // per warp and slot of a row tile: minus the log2-sum-exp of its rows
    __shared__ float s_part[2][2][128];                 // sums of the second warpgroups, of even and odd items
    __shared__ __align__(8) uint64_t s_pfull[4], s_pempty[4];
    const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, q_smem = base, ring = base + 2 * kRowTileBytes;
    const uint32_t full = smem_u32(s_full), empty = smem_u32(s_empty), qfull = smem_u32(s_qfull), qempty = smem_u32(s_qempty),
                   dfull = smem_u32(s_dfull), dempty = smem_u32(s_dempty), pfull = smem_u32(s_pfull), pempty = smem_u32(s_pempty);
    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];\n" ::"l"(&k_map), "l"(&q_map) : "memory");
        for (int i = 0; i < kWgStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(qfull + 8 * i, 1);
            mbar_init(qempty + 8 * i, 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(dfull + 8 * i, 1);
            mbar_init(dempty + 8 * i, 8);
            mbar_init(pfull + 8 * i, 4);
            mbar_init(pempty + 8 * i, 4);
        }
        mbar_init(smem_u32(&s_drain), 1);
        s_failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = __shfl_sync(kFull, s_tmem, 0);     // buffer y of warpgroup i at column 256 i + 128 y
    pdl_launch_dependents();
    pdl_wait();

    WeighCut cut[2];
    {
        auto cost = [&](int b) {
            const WeighItems t(chunk_seq(p.r, b), p.G);
            return t.cost_before(t.items);
        };
        WarpScan<decltype(cost)> scan(p.r.batch, cost, lane);
        const long long total = scan.total * p.Hkv;
        const int parts = gridDim.x, c = blockIdx.x;
        const long long each = quick_div(total, parts), more = total - each * parts;
#pragma unroll 1
        for (int i = 0; i < 2; ++i) cut[i] = weigh_cut(p, scan, each * (c + i) + min((long long)(c + i), more));   // (one copy of the code)
    }
    WeighWalk walk(p, cut[0], cut[1]);

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

    if (warp == 16) {
        // ---- copies
        int issued = 0, pages_b = -1, pages_k = 0, page = -1;
        uint32_t uses0 = 0, uses1 = 0;
        const int oob = p.r.num_pages * p.Hkv * kBlk;    // a row behind the pool: TMA fills zeros
        bool ok = true;
        for (; ok && !walk.done(); walk.next(p)) {
            if (walk.from >= walk.tiles) continue;
            if (pages_b != walk.at.b || walk.at.k < pages_k || walk.at.k >= pages_k + 8) {   // lane x: block x of eight items
                pages_b = walk.at.b;
                pages_k = walk.at.k;
                page = -1;
                if ((long long)(4 * pages_k + lane) * kBlk < walk.s.len) {
                    page = chunk_page(p.r, pages_b, 4 * pages_k + lane);
                    if (page < 0) atomicOr(p.r.status, kDevBadPage);
                }
            }
            const int lane0 = 4 * (walk.at.k - pages_k);
            for (int i = 0; i < (walk.two ? 2 : 1) && ok; ++i) {
                const int st = issued % kWgStages, round = issued / kWgStages;
                if (round > 0) ok = wait(empty + 8 * st, (round - 1) & 1);
                const int page0 = __shfl_sync(kFull, page, lane0 + 2 * i), page1 = __shfl_sync(kFull, page, lane0 + 2 * i + 1);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t dst = ring + st * kRowTileBytes, bar = full + 8 * st;
                    const int y0 = page0 >= 0 ? (page0 * p.Hkv + walk.at.g) * kBlk : oob, y1 = page1 >= 0 ? (page1 * p.Hkv + walk.at.g) * kBlk : oob;
                    mbar_expect(bar, kRowTileBytes);
                    tma_load(dst, &k_map, 0, y0, bar);
                    tma_load(dst + 64 * 128, &k_map, 0, y1, bar);
                    tma_load(dst + kRowTileHalf, &k_map, 64, y0, bar);
                    tma_load(dst + kRowTileHalf + 64 * 128, &k_map, 64, y1, bar);
                }
                __syncwarp();
                ++issued;
            }
            for (int j = walk.from; j < walk.tiles && ok && !walk.kept; ++j) {
                const int slot = j & 1;
                uint32_t& uses = slot ? uses1 : uses0;
                if (uses > 0) ok = wait(qempty + 8 * slot, (uses - 1) & 1);
                if (!ok) break;
                if (elect_one()) {
                    mbar_expect(qfull + 8 * slot, 2 * p.T1 * p.G * 128);
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        tma_load_3d(q_smem + slot * kRowTileBytes + half * kRowTileHalf, &q_map, 64 * half, walk.at.g * p.G,
                                    walk.s.row0 + j * p.T1, qfull + 8 * slot);
                }
                __syncwarp();
                ++uses;
            }
        }
        // nothing may write into this CTA's shared memory once it has left, whatever became of the other roles
        for (int i = max(0, issued - kWgStages); i < issued; ++i) mbar_wait(full + 8 * (i % kWgStages), (i / kWgStages) & 1);
        if (uses0) mbar_wait(qfull, (uses0 - 1) & 1);
        if (uses1) mbar_wait(qfull + 8, (uses1 - 1) & 1);
    } else if (warp == 17) {
        // ---- products: D = K Q^T, 128 tokens by the row tile's rows
        int used = 0, held = 0;                 // held: bit of a slot with a row tile
        uint32_t uses0 = 0, uses1 = 0, steps0 = 0, steps1 = 0;
        auto commit = [&](uint32_t bar) {
            if (elect_one()) mma_commit(bar);
            __syncwarp();
        };
        bool ok = true;
        for (; ok && !walk.done(); walk.next(p)) {
            const int count = walk.tiles - walk.from;
            if (count > 0) {
                const int groups = walk.two ? 2 : 1;
                for (int i = 0; i < groups && ok; ++i) ok = wait(full + 8 * ((used + i) % kWgStages), ((used + i) / kWgStages) & 1);
                for (int j = walk.from; j < walk.tiles && ok; ++j) {
                    const int slot = j & 1;
                    if (!walk.kept) {
                        uint32_t& uses = slot ? uses1 : uses0;
                        ok = wait(qfull + 8 * slot, uses++ & 1);
                        if (!ok) break;
                        held |= 1 << slot;
                    }
                    const int cols = (walk.columns(p, j) + 15) & ~15;
                    const uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(cols >> 3) << 17 | (128u >> 4) << 24;
                    for (int i = 0; i < groups && ok; ++i) {
                        const uint32_t x = i ? steps1++ : steps0++, y = x & 1;
                        if (x >= 2) ok = wait(dempty + 16 * i + 8 * y, ((x >> 1) - 1) & 1);
                        if (!ok) break;
                        tmem_after_sync();
                        const uint64_t a = mma_desc(ring + (used + i) % kWgStages * kRowTileBytes, 16, 1024), b = mma_desc(q_smem + slot * kRowTileBytes, 16, 1024);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks) {
                                const uint32_t at = ((ks >> 2) * kRowTileHalf + (ks & 3) * 32) >> 4;
                                mma_ss(tmem + 256 * i + 128 * y, a + at, b + at, idesc, ks > 0);
                            }
                            mma_commit(dfull + 16 * i + 8 * y);
                        }
                        __syncwarp();
                    }
                    if (ok && count > 2) {
                        commit(qempty + 8 * slot);
                        held &= ~(1 << slot);
                    }
                }
                if (!ok) break;
                for (int i = 0; i < groups; ++i) commit(empty + 8 * ((used + i) % kWgStages));
                used += groups;
            }
            if (!walk.keep)
                for (int slot = 0; slot < 2; ++slot)
                    if (held >> slot & 1) {
                        commit(qempty + 8 * slot);
                        held &= ~(1 << slot);
                    }
        }
        if (!ok) {   // products in flight still write tensor memory
            commit(smem_u32(&s_drain));
            mbar_wait(smem_u32(&s_drain), 0);
        }
    } else {
        // ---- exponentials and sums
        const int i = warp >> 2 & 1, half = warp >> 3;   // the tile of tokens, and which 64 rows of a row tile
        const uint32_t col = tmem + 256 * i + 64 * half + ((uint32_t)(warp & 3) << 21);
        const unsigned long long scale2 = pair_of(p.logit_scale, p.logit_scale);
        uint32_t x = 0, joined = 0;
        bool ok = true;
        int ahead_k = -1, ahead_g = -1, ahead_b = -1, ahead_page = -1;   // the page of this thread's token in the next item
        int row_token[2], row_at[2];                     // of a row tile's rows 64 half + lane and + 32: the token, and its place in p.lse
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int at = 64 * half + 32 * c + lane;
            row_token[c] = at / p.G;
            row_at[c] = row_token[c] * p.Hq + at - row_token[c] * p.G;
        }
#pragma unroll 1
        for (; ok && !walk.done(); walk.next(p)) {
            const int count = walk.tiles - walk.from, token = 256 * walk.at.k + 128 * i + (tid & 127);
            const bool mine = token < walk.s.len;
            if (i && !walk.two) continue;                // (a head's last item)
            if (count <= 0 && p.add) continue;           // nobody saw it
            // (a page is looked up an item early: its latency, and behind it that of the old weight, would be in every item's way)
            int page = -1;
            if (half == 0) {
                const bool known = ahead_b == walk.at.b && ahead_g == walk.at.g && ahead_k == walk.at.k;
                page = !mine ? -1 : known ? ahead_page : chunk_page(p.r, walk.at.b, token >> 6);
                ahead_k = -1;
                if (token < walk.s.len - 256) {          // (a sum could be beyond 31 bits)
                    ahead_b = walk.at.b;
                    ahead_g = walk.at.g;
                    ahead_k = walk.at.k + 1;
                    ahead_page = chunk_page(p.r, walk.at.b, (token + 256) >> 6);
                }
            }
            float next_lse[2];
            auto fetch = [&](int j) {                    // lane c, c + 32: the log-sum-exp of this warpgroup's rows
                const int token0 = j * p.T1, some = j < walk.tiles ? min(p.T1, walk.s.n - token0) : 0;
                const float* const from = p.lse + (size_t)(walk.s.row0 + token0) * p.Hq + walk.at.g * p.G;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float v = row_token[c] < some ? from[row_at[c]] : -INFINITY;
                    next_lse[c] = v == -INFINITY ? -INFINITY : -v * kLog2e;   // (an empty row's weights are 0)
                }
            };
            if (!walk.kept) fetch(walk.from);             // on its way one row tile ahead
            float* to = nullptr;
            if (mine && half == 0) {
                if (page >= 0) to = p.weight + ((size_t)page * p.Hkv + walk.at.g) * kBlk + (token & 63);
                else atomicOr(p.r.status, kDevBadPage);
            }
            const float old = to && p.add && token < walk.s.first ? *to : 0.f;
            unsigned long long sums[4] = {0ull, 0ull, 0ull, 0ull};
            bool shared = false;                         // has the second warpgroup any rows?
#pragma unroll 1
            for (int j = walk.from; j < walk.tiles; ++j, ++x) {
                float* const lse_smem = s_lse[warp][j & 1];
                if (!walk.kept) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) lse_smem[32 * c + lane] = next_lse[c];
                    __syncwarp();
                    fetch(j + 1);
                }
                const uint32_t lse_addr = smem_u32(lse_smem);
                const int all_cols = walk.columns(p, j), cols = all_cols - 64 * half, y = x & 1;
                shared |= all_cols > 64;
                // columns before this one do not see the token
                const int hidden = max(0, token - walk.s.first - j * p.T1) * p.G - 64 * half;
                const bool all = !__any_sync(kFull, hidden > 0);
                ok = wait(dfull + 16 * i + 8 * y, (x >> 1) & 1);
                if (!ok) break;
                tmem_after_sync();
#pragma unroll 1
                for (int c0 = 0; c0 < 64 && c0 < cols; c0 += 32) {
                    float s[32];
                    tmem_ld32(col + 128 * y + c0, s);
                    tmem_wait_ld();
                    auto add_four = [&](int c, bool plain) {
                        const uint4 l = lds128(lse_addr + 4 * (c0 + c));
                        float w[4];
                        pair_split(pair_fma(pair_of(s[c], s[c + 1]), scale2, pair_of(__uint_as_float(l.x), __uint_as_float(l.y))), w[0], w[1]);
                        pair_split(pair_fma(pair_of(s[c + 2], s[c + 3]), scale2, pair_of(__uint_as_float(l.z), __uint_as_float(l.w))), w[2], w[3]);
                        if (!plain) {   // columns behind the row tile's were not computed: minus infinity there, whatever tensor memory holds
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[e] = c0 + c + e >= hidden && c0 + c + e < cols ? w[e] : -INFINITY;
                        }
                        sums[c >> 2 & 1] = pair_add(sums[c >> 2 & 1], pair_of(fast_ex2(w[0]), fast_ex2(w[1])));
                        sums[2 + (c >> 2 & 1)] = pair_add(sums[2 + (c >> 2 & 1)], pair_of(fast_ex2(w[2]), fast_ex2(w[3])));
                    };
                    if (all && c0 + 32 <= cols) {
#pragma unroll
                        for (int c = 0; c < 32; c += 4) add_four(c, true);
                    } else {
#pragma unroll
                        for (int c = 0; c < 32; c += 4)
                            if (c0 + c < cols) add_four(c, false);
                    }
                }
                tmem_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(dempty + 16 * i + 8 * y);
            }
            if (!ok) break;
            float a, b;
            pair_split(pair_add(pair_add(sums[0], sums[1]), pair_add(sums[2], sums[3])), a, b);
            a += b;
            if (shared) {                                // the first warpgroup adds the second's sums to its own, always in this order
                const uint32_t y = joined & 1, bar = 16 * i + 8 * y, phase = joined >> 1 & 1;
                float* const part = &s_part[y][i][tid & 127];
                if (half) {
                    if (joined >= 2) ok = wait(pempty + bar, phase ^ 1);
                    if (!ok) break;
                    *part = a;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pfull + bar);
                } else {
                    ok = wait(pfull + bar, phase);
                    if (!ok) break;
                    a += *part;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pempty + bar);
                }
                ++joined;
            }
            if (to) *to = old + a;
        }
    }
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    if (tid == 0 && s_failed) atomicOr(p.r.status, kDevTimeout);
    if (warp == 17) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
}

// ---- choosing ---------------------------------------------------------------------------------------------------------------
//
// One cluster for every sequence and KV head.  Its CTAs divide the tokens evenly, in order, and keep their weights in shared memory
// as integers of the same order, as many as fit (the others are read again).  The smallest weight that is kept is found 8 bits
// at a time: every CTA counts its tokens by those bits, and each adds up the counts of all through distributed shared
// memory.  (11 bits at a time are three rounds instead of four, but a cluster of eight took 2.4 us to add up 2048 counts.)  Then
// tokens are numbered in order: those above that weight all stay, of those equal to it the first ones.  Latency is the bound,
// six barriers of the cluster among it (32 K tokens of eight heads: 16 us; 16 ragged sequences, two CTAs each: 25).
constexpr int kChThreads = 512, kChWarps = kChThreads / 32, kChBins = 256;
constexpr int kChKeys = 40960;                    // weights in a CTA's shared memory: 160 KB
constexpr int kChMaxCluster = 8;

struct EvictParams {
    const __nv_bfloat16 *k, *v;
    const float* weight;
    const int32_t *block_table, *seq_lens, *out_table;
    __nv_bfloat16 *k_out, *v_out;
    float* weight_out;
    int32_t *out_lens, *kept;
    uint32_t* status;
    int batch, Hkv, max_blocks, num_pages, budget, n_sink, n_local, max_out_blocks, num_out_pages;
};

// integers in the order of the weights, 0 for a NaN; both zeros are equal
__device__ __forceinline__ uint32_t order_of(float w) {
    if (w != w) return 0u;
    const uint32_t x = __float_as_uint(w + 0.f);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

struct ChooseShared {
    int32_t pages[kChKeys / kBlk + 2];
    uint32_t bins[2][kChBins];                    // of even and odd rounds
    uint32_t warp_sums[2 * kChWarps];
    uint32_t above, equal;                        // of this CTA's tokens
    uint32_t digit, before;                       // result of a round: the digit, and how many tokens have a larger one
};

// the sums of `x` over the warps before this one; all threads
__device__ __forceinline__ uint32_t sum_before(uint32_t x, const uint32_t* warp_sums, int warp, int lane) {
    const uint32_t w = lane < warp && lane < kChWarps ? warp_sums[lane] : 0u;
    return x + __reduce_add_sync(kFull, w);
}

__global__ void __launch_bounds__(kChThreads, 2) choose_kernel(const __grid_constant__ EvictParams p, int cluster) {
    namespace cg = cooperative_groups;
    extern __shared__ __align__(16) uint32_t s_keys[];
    __shared__ ChooseShared s;
    cg::cluster_group team = cg::this_cluster();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = (int)team.block_rank();
    const int unit = blockIdx.x / cluster, b = unit / p.Hkv, g = unit - b * p.Hkv;
    pdl_launch_dependents();
    pdl_wait();
    const int len = paged_len(p.seq_lens, b, p.max_blocks, p.status);
    int32_t* const kept = p.kept + (size_t)unit * p.budget;
    const int out_len = min(len, p.budget);
    for (long long x = (long long)out_len + rank * kChThreads + tid; x < p.budget; x += cluster * kChThreads) kept[x] = -1;   // (up to 2^31 - 1)
    if (len <= p.budget) {                        // the same in all CTAs of the cluster
        for (long long x = rank * kChThreads + tid; x < len; x += cluster * kChThreads) kept[x] = (int)x;
        return;
    }
    // this CTA's tokens: a run of whole groups of 32
    const int groups = ceil_shift(len, 5), group0 = (int)((long long)groups * rank / cluster), group1 = (int)((long long)groups * (rank + 1) / cluster);
    const int low = group0 * 32, high = min(len, group1 * 32);
    const int tail = len - p.n_local;
    // tokens that stay whatever their weight have the largest key of all, which no weight has
    auto weigh = [&](int t) {
        if (t < p.n_sink || t >= tail) return 0xffffffffu;
        const long long index = (long long)b * p.max_blocks + (t >> 6), page = p.block_table ? (long long)p.block_table[index] : index;
        if (page < 0 || page >= p.num_pages) {
            atomicOr(p.status, kDevBadPage);
            return 0u;
        }
        return order_of(p.weight[((size_t)page * p.Hkv + g) * kBlk + (t & 63)]);
    };
    auto key_of = [&](int t) { return t - low < kChKeys ? s_keys[t - low] : weigh(t); };
    const int near = min(high, low + kChKeys);
    for (int x = (low >> 6) + tid; x <= (near - 1) >> 6; x += kChThreads) {      // the pages first, so that the weights' loads wait for no others
        const long long index = (long long)b * p.max_blocks + x, page = p.block_table ? (long long)p.block_table[index] : index;
        const bool good = page >= 0 && page < p.num_pages;
        s.pages[x - (low >> 6)] = good ? (int)page : -1;
        if (!good) atomicOr(p.status, kDevBadPage);
    }
    if (tid < kChBins) s.bins[0][tid] = 0;
    __syncthreads();
#pragma unroll 8
    for (unsigned t = low + tid; t < (unsigned)near; t += kChThreads) {   // (a step beyond the longest sequence is beyond 31 bits)
        const int page = s.pages[(t >> 6) - (low >> 6)];
        const uint32_t key = order_of(p.weight[((size_t)max(page, 0) * p.Hkv + g) * kBlk + (t & 63)]);   // (no branch: loads side by side)
        s_keys[t - low] = t < p.n_sink || t >= tail ? 0xffffffffu : page < 0 ? 0u : key;
    }
    uint32_t want = (uint32_t)p.budget, found = 0, mask = 0;   // want of the tokens whose key & mask == found
    __syncthreads();
#pragma unroll 1
    for (int round = 0; round < 4; ++round) {
        const int shift = 24 - 8 * round;
        uint32_t* const bins = s.bins[round & 1];
        // (tokens of equal weight are common, those that nobody looked at: a warp's additions of one to one place are a single one)
#pragma unroll 4
        for (unsigned t = low + tid; t < (unsigned)high; t += kChThreads) {
            const uint32_t key = key_of(t);
            if ((key & mask) == found) atomicAdd(&bins[key >> shift & 255u], 1u);
        }
        team.sync();
        if (tid < kChBins) s.bins[round & 1 ^ 1][tid] = 0;      // (read by all before the last barrier but one)
        // the cluster's counts, a thread for a digit; the largest first in the numbering
        uint32_t sum = 0;
        const int digit = kChBins - 1 - tid;
        if (tid < kChBins) {
#pragma unroll
            for (int c = 0; c < kChMaxCluster; ++c)
                if (c < cluster) sum += *(team.map_shared_rank(bins, c) + digit);
        }
        uint32_t scan = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(kFull, scan, o);
            if (lane >= o) scan += x;
        }
        if (lane == 31) s.warp_sums[warp] = scan;
        __syncthreads();
        const uint32_t before = sum_before(scan - sum, s.warp_sums, warp, lane);
        if (before < want && want <= before + sum) {   // one thread: the want-th largest has its digit
            s.digit = (uint32_t)digit;
            s.before = before;
        }
        __syncthreads();
        want -= s.before;
        found |= s.digit << shift;
        mask |= 255u << shift;
    }
    // `want` of the tokens equal to `found` stay, the first ones, and all above it.  A warp numbers a run of groups.
    const int mine = group1 - group0, w0 = group0 + mine * warp / kChWarps, w1 = group0 + mine * (warp + 1) / kChWarps;
    auto judge = [&](int t, bool& above, bool& equal) {
        const uint32_t key = t < high ? key_of(t) : 0u;
        above = t < high && key > found;
        equal = t < high && key == found;
    };
    uint32_t above_count = 0, equal_count = 0;
#pragma unroll 4
    for (int x = w0; x < w1; ++x) {
        bool above, equal;
        judge(32 * x + lane, above, equal);
        above_count += __popc(__ballot_sync(kFull, above));
        equal_count += __popc(__ballot_sync(kFull, equal));
    }
    if (lane == 0) {
        s.warp_sums[warp] = above_count;
        s.warp_sums[kChWarps + warp] = equal_count;
    }
    __syncthreads();
    if (warp == 0) {
        const uint32_t a = __reduce_add_sync(kFull, lane < kChWarps ? s.warp_sums[lane] : 0u),
                       e = __reduce_add_sync(kFull, lane < kChWarps ? s.warp_sums[kChWarps + lane] : 0u);
        if (lane == 0) {
            s.above = a;
            s.equal = e;
        }
    }
    team.sync();
    uint32_t above_before = 0, equal_before = 0;
    for (int c = 0; c < rank; ++c) {
        const ChooseShared* const o = team.map_shared_rank(&s, c);
        above_before += o->above;
        equal_before += o->equal;
    }
    team.sync();           // nobody leaves while others read its counts
    above_before = sum_before(above_before, s.warp_sums, warp, lane);
    equal_before = sum_before(equal_before, s.warp_sums + kChWarps, warp, lane);
#pragma unroll 4
    for (int x = w0; x < w1; ++x) {
        const int t = 32 * x + lane;
        bool above, equal;
        judge(t, above, equal);
        const unsigned a = __ballot_sync(kFull, above), e = __ballot_sync(kFull, equal), under = (1u << lane) - 1u;
        const uint32_t equal_rank = equal_before + __popc(e & under);
        // equal ones before this token that stay: at most `want`
        const uint32_t slot = above_before + __popc(a & under) + min(want, equal_rank);
        if ((above || (equal && equal_rank < want)) && slot < (uint32_t)p.budget) kept[slot] = t;
        above_before += __popc(a);
        equal_before += __popc(e);
    }
}

// ---- moving -----------------------------------------------------------------------------------------------------------------
//
// An item is a page of the result: 64 rows of K and V, 256 bytes each wherever they come from, 16 lanes for a row.  While an item's
// rows are on their way, the places of the next one's are looked up, and what is kept in the one after that: three loads that depend
// on one another would otherwise be in front of every item's data (250 MB: 41 us, 6.1 TB/s, instead of 52).
constexpr int kMvThreads = 256, kMvRows = kBlk / (kMvThreads / 16);      // rows of a thread

__global__ void __launch_bounds__(kMvThreads, 4) move_kernel(const __grid_constant__ EvictParams p, int blocks) {
    pdl_wait();
    const int tid = threadIdx.x, sub = tid >> 4, piece = tid & 15, step = gridDim.x, items = blocks * p.batch * p.Hkv;
    // (here and not where tokens are chosen, as both arrays may be the same: that kernel's CTAs all read a sequence's length)
    for (int b = blockIdx.x * kMvThreads + tid; b < p.batch; b += step * kMvThreads)
        p.out_lens[b] = min(paged_len(p.seq_lens, b, p.max_blocks, p.status), p.budget);
    struct Item { int row[kMvRows], to; };       // rows of the pool that is read, and the first one of the page that is written; -1: none
    auto kept_of = [&](int item, int (&t)[kMvRows]) {
        const int unit = item / blocks, blk = item - unit * blocks;
#pragma unroll
        for (int x = 0; x < kMvRows; ++x) {
            const int slot = blk * kBlk + sub + x * (kMvThreads / 16);
            t[x] = item < items && slot < p.budget ? p.kept[(size_t)unit * p.budget + slot] : -1;
        }
    };
    auto places_of = [&](int item, const int (&t)[kMvRows]) {
        Item m;
        m.to = -1;
        const int unit = item / blocks, blk = item - unit * blocks, b = unit / p.Hkv, g = unit - b * p.Hkv;
        if (item < items && blk < p.max_out_blocks) {
            const long long at = (long long)b * p.max_out_blocks + blk, page = p.out_table ? (long long)p.out_table[at] : at;
            if (page >= 0 && page < p.num_out_pages) m.to = (int)((page * p.Hkv + g) * kBlk);
        }
#pragma unroll
        for (int x = 0; x < kMvRows; ++x) {
            m.row[x] = -1;
            if (t[x] < 0) continue;
            const long long at = (long long)b * p.max_blocks + (t[x] >> 6), page = p.block_table ? (long long)p.block_table[at] : at;
            if (page >= 0 && page < p.num_pages) m.row[x] = (int)((page * p.Hkv + g) * kBlk + (t[x] & 63));
            if (piece == 0 && (m.row[x] < 0 || m.to < 0)) atomicOr(p.status, blk < p.max_out_blocks ? kDevBadPage : kDevBadSeqLen);
        }
        return m;
    };
    int t[kMvRows];
    kept_of(blockIdx.x, t);
    Item now = places_of(blockIdx.x, t);
    kept_of(blockIdx.x + step, t);
#pragma unroll 1
    for (int item = blockIdx.x; item < items; item += step) {
        uint4 k[kMvRows], v[kMvRows];
        float w[kMvRows];
#pragma unroll
        for (int x = 0; x < kMvRows; ++x) {
            if (now.row[x] < 0 || now.to < 0) continue;
            k[x] = ldg_plain(reinterpret_cast<const uint4*>(p.k + (size_t)now.row[x] * kD) + piece);
            v[x] = ldg_plain(reinterpret_cast<const uint4*>(p.v + (size_t)now.row[x] * kD) + piece);
            if (piece == 0 && p.weight_out) w[x] = p.weight[now.row[x]];
        }
        const Item next = places_of(item + step, t);
        kept_of(item + 2 * step, t);
#pragma unroll
        for (int x = 0; x < kMvRows; ++x) {
            if (now.row[x] < 0 || now.to < 0) continue;
            const size_t to = (size_t)now.to + sub + x * (kMvThreads / 16);
            reinterpret_cast<uint4*>(p.k_out + to * kD)[piece] = k[x];
            reinterpret_cast<uint4*>(p.v_out + to * kD)[piece] = v[x];
            if (piece == 0 && p.weight_out) p.weight_out[to] = w[x];
        }
        now = next;
    }
}

}  // namespace ffd

using namespace ffd;

extern "C" {

ffd_status ffd_weigh_kv(const ffd_config* cfg, const void* q, const float* lse, const void* k_cache, float* weight, int32_t add,
                        const int32_t* block_table, const int32_t* row_start, const int32_t* first_token, const int32_t* seq_lens,
                        int32_t num_rows, int32_t batch, int32_t max_blocks_per_seq, int32_t num_pages, void* workspace,
                        size_t workspace_bytes, void* stream) {
    ffd_status st = check_chunk(cfg, batch, num_rows, max_blocks_per_seq, num_pages);
    if (st) return st;
    if (!q || !lse || !k_cache || !weight || !seq_lens || !workspace) return FFD_ERR_NULL;
    if ((row_start == nullptr) != (first_token == nullptr)) return FFD_ERR_NULL;
    if (!row_start && num_rows != batch) return FFD_ERR_SHAPE;
    if (add != 0 && add != 1) return FFD_ERR_UNSUPPORTED;
    if (workspace_bytes < kHeaderBytes) return FFD_ERR_WORKSPACE;
    if (any_misaligned(q, lse, k_cache, weight, block_table, row_start, first_token, seq_lens, workspace)) return FFD_ERR_ALIGN;
    WeighParams p;
    p.r = ChunkRows{row_start, first_token, seq_lens, block_table, static_cast<uint32_t*>(workspace), num_rows, batch, max_blocks_per_seq, num_pages};
    p.Hq = cfg->num_q_heads;
    p.Hkv = cfg->num_kv_heads;
    p.G = p.Hq / p.Hkv;
    p.T1 = 128 / p.G;
    p.add = add;
    p.logit_scale = logit_scale_of(cfg);
    p.lse = lse;
    p.weight = weight;
    const EncodeTiled encode = encode_tiled();
    if (!encode) return FFD_ERR_CUDA;
    CUtensorMap k_map, q_map;
    if (!page_map(encode, &k_map, k_cache, (long long)num_pages * p.Hkv * kBlk) || !rows_map(encode, &q_map, q, p.Hq, p.G, num_rows))
        return FFD_ERR_CUDA;
    if (cudaFuncSetAttribute(weigh_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWgSmem) != cudaSuccess) return FFD_ERR_CUDA;
    launch_pdl(weigh_kernel, dim3(device_sms()), dim3(kWgThreads), kWgSmem, static_cast<cudaStream_t>(stream), k_map, q_map, p);
    return launch_status();
}

ffd_status ffd_evict_kv(const ffd_config* cfg, const void* k_cache, const void* v_cache, const float* weight, const int32_t* block_table,
                        const int32_t* seq_lens, int32_t batch, int32_t max_blocks_per_seq, int32_t num_pages, int32_t budget,
                        int32_t n_sink, int32_t n_local, void* k_out, void* v_out, float* weight_out, const int32_t* out_table,
                        int32_t max_out_blocks, int32_t num_out_pages, int32_t* out_lens, int32_t* kept, void* workspace,
                        size_t workspace_bytes, void* stream) {
    ffd_status st = check_chunk(cfg, batch, 1, max_blocks_per_seq, num_pages);
    if (st) return st;
    if (!k_cache || !v_cache || !weight || !seq_lens || !k_out || !v_out || !out_lens || !kept || !workspace) return FFD_ERR_NULL;
    if (check_chunk(cfg, batch, 1, max_out_blocks, num_out_pages)) return FFD_ERR_SHAPE;
    if (budget < 1 || n_sink < 0 || n_local < 0 || (int64_t)n_sink + n_local > budget) return FFD_ERR_SHAPE;
    const int units = batch * cfg->num_kv_heads;
    const long long blocks = ((long long)budget + kBlk - 1) / kBlk;
    if (blocks * units > 0x3fffffffLL) return FFD_ERR_SHAPE;   // (the pages of results that are counted in 32 bits)
    if (workspace_bytes < kHeaderBytes) return FFD_ERR_WORKSPACE;
    if (any_misaligned(k_cache, v_cache, weight, block_table, seq_lens, k_out, v_out, weight_out, out_table, out_lens, kept, workspace))
        return FFD_ERR_ALIGN;
    EvictParams p{static_cast<const __nv_bfloat16*>(k_cache), static_cast<const __nv_bfloat16*>(v_cache), weight, block_table, seq_lens, out_table,
                  static_cast<__nv_bfloat16*>(k_out), static_cast<__nv_bfloat16*>(v_out), weight_out, out_lens, kept,
                  static_cast<uint32_t*>(workspace), batch, cfg->num_kv_heads, max_blocks_per_seq, num_pages, budget, n_sink, n_local,
                  max_out_blocks, num_out_pages};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int sms = device_sms();
    // CTAs per head: one for every 4096 tokens that a sequence can have, while the launch stays within one round of the card
    const long long tokens = (long long)max_blocks_per_seq * kBlk;
    int cluster = 1;
    while (cluster < kChMaxCluster && tokens > 4096LL * cluster && (long long)units * cluster <= sms) cluster *= 2;   // (two CTAs fit an SM)
    const size_t keys = (size_t)min((long long)kChKeys, align_up((size_t)((tokens + cluster - 1) / cluster) + 32, 4) + 0LL) * sizeof(uint32_t);
    // (the most that any call takes: the attribute is the process's, and other threads may launch between this and the launch)
    if (cudaFuncSetAttribute(choose_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kChKeys * (int)sizeof(uint32_t)) != cudaSuccess)
        return FFD_ERR_CUDA;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(units * cluster));
    lc.blockDim = dim3(kChThreads);
    lc.dynamicSmemBytes = keys;
    lc.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = 2;
    (void)cudaLaunchKernelEx(&lc, choose_kernel, p, cluster);
    st = launch_status();
    if (st) return st;
    launch_pdl(move_kernel, dim3((unsigned)min(blocks * units, 4LL * sms)), dim3(kMvThreads), 0, s, p, (int)blocks);
    return launch_status();
}

}  // extern "C"
