// What the kernels of a chunk of new tokens have in common: where its rows are, and the walk over tiles of it.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "../../include/ffd.h"
#include "ffd_paged.cuh"

namespace ffd {

// The rows of a call: row row_start[b] + i is token first_token[b] + i of sequence b, up to token seq_lens[b] - 1; without
// row_start, row b is the last token of sequence b.
struct ChunkRows {
    const int32_t* row_start;
    const int32_t* first_token;
    const int32_t* seq_lens;
    const int32_t* block_table;    // [batch, max_blocks]; null: page b * max_blocks + blk
    uint32_t* status;
    int num_rows, batch, max_blocks, num_pages;
};

struct ChunkSeq {
    int first, n, len, row0;       // tokens first .. first + n - 1 = len - 1 are the rows row0 .. row0 + n - 1
};

// Every number that comes from the device is brought into its range, and reported if it was outside: what follows indexes with
// them.
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkRows& p, int b) {
    const bool listed = p.row_start != nullptr;
    const int len = p.seq_lens[b], first = listed ? p.first_token[b] : 0, row0 = listed ? p.row_start[b] : b;   // (side by side: none waits)
    const int cap = p.max_blocks * kBlk;
    ChunkSeq s;
    s.len = min(max(len, 0), cap);
    s.first = listed ? min(max(first, 0), s.len) : max(s.len - 1, 0);
    s.n = s.len - s.first;
    s.row0 = row0;
    const bool rows = s.n <= 0 || (row0 >= 0 && s.n <= p.num_rows - row0);   // do they exist?
    if (s.len != len || first < 0 || !rows) {
        atomicOr(p.status, kDevBadSeqLen);
        if (!rows) s.n = row0 < 0 ? 0 : max(0, p.num_rows - row0);
    }
    return s;
}

__device__ __forceinline__ int chunk_page(const ChunkRows& p, int b, int blk) {   // -1: none
    const long long index = (long long)b * p.max_blocks + blk, page = p.block_table ? (long long)p.block_table[index] : index;
    return page >= 0 && page < p.num_pages ? (int)page : -1;
}

// The largest j in [0, n) with before(j) <= x, where before(0) <= x and before does not decrease; 32 places at once.
template <typename Before>
__device__ __forceinline__ int warp_search(int n, long long x, Before&& before) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) >> 5, at = lo + (lane + 1) * step;
        lo += step * __popc(__ballot_sync(kFull, at < hi && before(at) <= x));
        hi = min(hi, lo + step);
    }
    return lo;
}

// ---- the walk of the attention kernel ------------------------------------------------------------------------------------
//
// The rows of a sequence and KV head are cut into tiles of R * T1 tokens with G heads each, T1 = 128 / G: R = 2 row tiles of at most
// 128 rows, or one for binary32 results.  A tile's keys are the tokens up to its last row's, in steps of R * 64.  The list of all
// steps, ordered by sequence, head, tile and step, is cut into shares of about the same cost, one for each CTA; a tile that a cut
// falls into is finished by the merge kernel.  So the work is spread evenly whatever the lengths: one long sequence with one
// new token (a few tiles, each shared by many CTAs) as well as many tiles for every CTA.
//
// Costs are counted in units of which a full tile's key costs kKey and that of a tile with one row tile of two kSingle, so that the
// cost of the tiles before one has a closed form; kTile tokens stand for a tile's beginning and end.  (R = 2 is a fit of the CTAs'
// cycles: 3600 a step, 2400 with one row tile, 8200 and 5000 a segment.  With 64 tokens a segment the slowest CTA of 512 new tokens on
// 16 K took 1.9 times the average, and the call 316 us instead of 246.  R = 1: 30 cycles a key, 11000 a segment; of 128, 256, 384 and 640
// tokens for it, 512 new tokens on 16 K took 448, 383, 409 and 400 us, ragged prompts 90, 81, 79 and 81.)
template <int R> struct ChunkCosts;
template <> struct ChunkCosts<2> { static constexpr int kKey = 5, kSingle = 3, kTile = 320, kShift = 7; };
template <> struct ChunkCosts<1> { static constexpr int kKey = 1, kSingle = 1, kTile = 256, kShift = 6; };

template <int R>
struct ChunkTiles {      // of one sequence and KV head
    using C = ChunkCosts<R>;
    long long first;
    int n, T1, tiles, last_cost;
    __device__ __forceinline__ ChunkTiles(const ChunkSeq& s, int t1) : first(s.first), n(s.n), T1(t1) {
        tiles = n > 0 ? (n - 1) / (R * t1) + 1 : 0;
        last_cost = n - (tiles - 1) * R * t1 <= t1 ? C::kSingle : C::kKey;
    }
    __device__ __forceinline__ int unit(int j) const { return j == tiles - 1 ? last_cost : C::kKey; }
    __device__ __forceinline__ bool single(int j) const { return R == 1 || unit(j) == C::kSingle; }
    __device__ __forceinline__ int keys(int j) const { return (int)first + min((j + 1) * R * T1, n); }   // that tile j sees
    __device__ __forceinline__ int steps(int j) const { return ceil_shift(keys(j), C::kShift); }
    __device__ __forceinline__ long long cost_before(int j) const {   // j < tiles: all of them full
        return (j * (first + C::kTile) + (long long)T1 * R * j * (j + 1) / 2) * C::kKey;
    }
    __device__ __forceinline__ long long cost() const {
        return tiles ? cost_before(tiles - 1) + (first + n + C::kTile) * last_cost : 0;
    }
};

struct ChunkCut {        // a place in the list: step `step` of tile j, or the list's end (b = batch)
    int b, g, j, step;
    __device__ __forceinline__ bool same_tile(const ChunkCut& o) const { return b == o.b && g == o.g && j == o.j; }
    __device__ __forceinline__ bool operator==(const ChunkCut& o) const { return same_tile(o) && step == o.step; }
};

// The place next to cost x, by the whole warp; every warp of the grid finds the same.
template <int R, typename Scan>
__device__ __forceinline__ ChunkCut chunk_cut(const ChunkRows& p, Scan& scan, int Hkv, int T1, long long x) {
    if (x >= scan.total * Hkv) return ChunkCut{p.batch, 0, 0, 0};
    ChunkCut c;
    long long off;
    scan.find(x, Hkv, c.b, off);
    const ChunkTiles<R> t(chunk_seq(p, c.b), T1);
    constexpr int kShift = ChunkCosts<R>::kShift;
    long long y = x - off;
    const long long head = t.cost();
    c.g = (int)(head >> 31 ? y / head : quick_div(y, (int)head));
    y -= c.g * head;
    const int lo = warp_search(t.tiles, y, [&](int j) { return t.cost_before(j); });
    c.j = lo;
    c.step = (int)min((long long)t.steps(lo), (quick_div(y - t.cost_before(lo), t.unit(lo)) + (1 << (kShift - 1))) >> kShift);
    if (c.step == t.steps(lo)) {   // the next tile's first
        c.step = 0;
        if (++c.j == t.tiles) {
            c.j = 0;
            if (++c.g == Hkv) {
                c.g = 0;
                do ++c.b;
                while (c.b < p.batch && chunk_seq(p, c.b).n == 0);
            }
        }
    }
    return c;
}

// The segments of a share: runs of steps of one tile
template <int R>
struct ChunkWalk {
    ChunkCut at, end;
    ChunkSeq s;
    int tiles, steps, last;      // of the tile: its number of steps; last: the segment ends before this step
    bool single;                 // the tile has rows in one row tile only

    __device__ __forceinline__ ChunkWalk(const ChunkRows& p, int T1, const ChunkCut& from, const ChunkCut& to) : at(from), end(to) {
        if (at.b < p.batch) s = chunk_seq(p, at.b);
        settle(p, T1);
    }
    __device__ __forceinline__ bool done() const { return last <= at.step; }
    __device__ __forceinline__ int count() const { return last - at.step; }
    __device__ __forceinline__ void settle(const ChunkRows& p, int T1) {
        last = 0;
        tiles = steps = 0;
        single = false;
        if (at.b >= p.batch || at == end) return;
        const ChunkTiles<R> t(s, T1);
        tiles = t.tiles;
        steps = t.steps(at.j);
        single = t.single(at.j);
        last = at.same_tile(end) ? end.step : steps;
    }
    __device__ __forceinline__ void next(const ChunkRows& p, int Hkv, int T1) {
        if (at.same_tile(end)) {
            at = end;
        } else {
            at.step = 0;
            if (++at.j == tiles) {
                at.j = 0;
                if (++at.g == Hkv) {
                    at.g = 0;
                    do ++at.b;
                    while (at.b < p.batch && (s = chunk_seq(p, at.b)).n == 0);
                }
            }
        }
        settle(p, T1);
    }
    __device__ __forceinline__ int token0(int T1) const { return at.j * R * T1; }   // of the chunk
};

// ---- what the attention kernels share ------------------------------------------------------------------------------------

constexpr int kCkThreads = 384;
constexpr int kCkRows = 256;                     // rows of a partial result's place
constexpr int kCkBadRing = 16;                   // steps that the loads can be ahead of the softmax, and more
constexpr int kCkFlawRing = 8;                   // segments whose notes are kept: as many as are handed out at once

struct ChunkParams {
    ChunkRows r;
    int Hq, Hkv, G, T1;
    float logit_scale;             // sm_scale * log2(e)
    void* out;                     // [num_rows, Hq, 128]
    float* lse;                    // nullable [num_rows, Hq]
    int out_fp32;
    int* parts;                    // number of shares: attention -> merge
    ChunkCut* cuts;                // [parts + 1]
    float* part_out;               // [2 * parts][256][128] normalised partial results; slot 2 c + 1 of share c is its tile that
    float* part_lse;               // begins there, 2 c the one that began before.  log2 of the sum of weights; -inf: empty
};

// A segment, a run of steps of one tile, as the scheduling warp hands it to the others
struct ChunkSegment {
    int b, g;
    int step, count;               // its steps are step .. step + count - 1; count 0: the share's end
    int single, whole;             // rows in one row tile only; the tile is all this share's
    int slot;                      // of its partial result
    int pos;                       // position of the tile's first token
    int tokens;                    // its tokens in the tile and behind it
    int row;                       // the first token's row
    int len;                       // tokens of the sequence
};
constexpr int kCkSegments = 8;     // handed out and not yet taken by everyone
constexpr int kCkTakers = 11;      // eight softmax warps, the copies, the products, the hidden values

// A micro-step of a share, in order: a row tile times the KEYS keys of a step
template <int KEYS>
struct ChunkMicro {
    ChunkSegment s;
    int x, t, r, step, segment;    // x: number; t: step of the segment; r: row tile; step, segment: of the share

    __device__ __forceinline__ bool live() const { return s.count > 0; }
    __device__ __forceinline__ int key0() const { return (s.step + t) * KEYS; }
    // does a row of the tile see only a part of the step's keys?
    __device__ __forceinline__ bool edge() const { return key0() + KEYS - 1 > s.pos; }
    __device__ __forceinline__ bool step_ends() const { return s.single || r == 1; }
    template <typename Take>
    __device__ __forceinline__ void begin(Take&& take) {
        x = t = r = step = segment = 0;
        s = take(0);
    }
    template <typename Take>
    __device__ __forceinline__ void advance(Take&& take) {
        ++x;
        if (!step_ends()) {
            r = 1;
            return;
        }
        r = 0;
        ++step;
        if (++t == s.count) {
            t = 0;
            s = take(++segment);
        }
    }
};

// The order of the products, which is also the order in which the ring's entries are first used: scores AHEAD micro-steps ahead.
// The segments are taken twice, and given back by `take_last`.
template <int KEYS, int AHEAD, typename Take, typename TakeLast, typename Scores, typename Values>
__device__ __forceinline__ void chunk_order(Take&& take, TakeLast&& take_last, Scores&& scores, Values&& values) {
    ChunkMicro<KEYS> k, v;
    k.begin(take);
    v.begin(take_last);
#pragma unroll 1
    for (int ahead = AHEAD;;) {   // (one copy of each function's code)
        if (ahead > 0) --ahead;
        else {
            if (!v.live() || !values(v)) break;
            v.advance(take_last);
        }
        if (k.live()) {
            if (!scores(k)) break;
            k.advance(take);
        } else if (ahead > 0) {
            ahead = 0;
        }
    }
}

// Values that some of a tile's rows do not see: a weight of 0 must not meet an infinity or a NaN.  `tile` has KEYS rows of 128 channels,
// key0 + 0 .., in two halves of 64.  Rows from x1 on, which none sees, become zeros, whatever they are.  Of the rows x0 .. x1 - 1
// elements that are no numbers become zeros, and the first such token of each channel is noted in `flaw`.  By a whole warp; any noted?
template <int KEYS>
__device__ __forceinline__ bool hide_values(uint32_t tile, int x0, int x1, int key0, int* flaw, int lane) {
    auto chunk_at = [&](int x) {   // 16 bytes: row x / 16, channels 8 (x % 16) ..
        const int row = x >> 4;
        return tile + (x & 8 ? KEYS * 128 : 0) + row * 128 + (((x & 7) ^ (row & 7)) << 4);
    };
    x0 *= 16;
    x1 *= 16;
    uint32_t top = 0;
#pragma unroll 8
    for (int x = x0 + lane; x < x1; x += 32) {
        const uint4 v = lds128(chunk_at(x));
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
    }
#pragma unroll 8
    for (int x = x1 + lane; x < KEYS * 16; x += 32)
        asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};\n" ::"r"(chunk_at(x)), "r"(0u) : "memory");
    if (!__any_sync(kFull, (top & 0xffffu) >= 0x7f80u || top >= 0x7f800000u)) return false;
#pragma unroll 1
    for (int x = x0 + lane; x < x1; x += 32) {
        const uint4 v = lds128(chunk_at(x));
        uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int y = 0; y < 8; ++y)
            if ((e[y >> 1] >> (16 * (y & 1)) & 0x7f80u) == 0x7f80u) {
                e[y >> 1] &= y & 1 ? 0x0000ffffu : 0xffff0000u;
                atomicMin(flaw + 8 * (x & 15) + y, key0 + (x >> 4));
            }
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};\n" ::"r"(chunk_at(x)), "r"(e[0]), "r"(e[1]), "r"(e[2]), "r"(e[3]) : "memory");
    }
    return true;
}

// A thread's own channels of a row: whole 32-byte sectors, so that nothing is gained by passing them to other lanes first.  (Through
// shared memory, 64 bytes of a row by neighbouring lanes, a tile's results took twice as long.)  The rows' beginnings are 16-byte
// aligned, as the caller's buffers are; a store of a whole sector needs 32.
__device__ __forceinline__ void store_sector(char* to, const uint32_t* w, bool whole) {
    if (whole) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                     "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4*>(to)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

}  // namespace ffd
