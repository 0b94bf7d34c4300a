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
// The rows of a sequence and KV head are cut into tiles of 2 * T1 tokens with G heads each, T1 = 128 / G: two row tiles of at most
// 128 rows.  A tile's keys are the tokens up to its last row's, in steps of 128.  The list of all steps, ordered by sequence,
// head, tile and step, is cut into shares of about the same cost, one for each CTA; a tile that a cut falls into is finished
// by the merge kernel.  So the work is spread evenly whatever the lengths: one long sequence with one new token (a few tiles,
// each shared by many CTAs) as well as many tiles for every CTA.
//
// Costs are counted in units of which a full tile's key costs kPairCost and a tile of one row tile's kSingleCost, so that the cost of
// the tiles before one has a closed form; kTileCost tokens stand for a tile's beginning and end.  (A fit of the CTAs' cycles: 3600
// a step, 2400 with one row tile, 8200 and 5000 a segment.  With 64 tokens a segment the slowest CTA of 512 new tokens on 16 K took 1.9
// times the average, and the call 316 us instead of 246.)
constexpr int kPairCost = 5, kSingleCost = 3, kTileCost = 320;

struct ChunkTiles {      // of one sequence and KV head
    long long first;
    int n, T1, tiles, last_cost;
    __device__ __forceinline__ ChunkTiles(const ChunkSeq& s, int t1) : first(s.first), n(s.n), T1(t1) {
        tiles = n > 0 ? (n - 1) / (2 * t1) + 1 : 0;
        last_cost = n - (tiles - 1) * 2 * t1 <= t1 ? kSingleCost : kPairCost;
    }
    __device__ __forceinline__ int unit(int j) const { return j == tiles - 1 ? last_cost : kPairCost; }
    __device__ __forceinline__ int keys(int j) const { return (int)first + min((j + 1) * 2 * T1, n); }   // that tile j sees
    __device__ __forceinline__ int steps(int j) const { return ceil_shift(keys(j), 7); }
    __device__ __forceinline__ long long cost_before(int j) const {   // j < tiles: all of them full
        return (j * (first + kTileCost) + (long long)T1 * j * (j + 1)) * kPairCost;
    }
    __device__ __forceinline__ long long cost() const {
        return tiles ? cost_before(tiles - 1) + (first + n + kTileCost) * last_cost : 0;
    }
};

struct ChunkCut {        // a place in the list: step `step` of tile j, or the list's end (b = batch)
    int b, g, j, step;
    __device__ __forceinline__ bool same_tile(const ChunkCut& o) const { return b == o.b && g == o.g && j == o.j; }
    __device__ __forceinline__ bool operator==(const ChunkCut& o) const { return same_tile(o) && step == o.step; }
};

// The place next to cost x, by the whole warp; every warp of the grid finds the same.
template <typename Scan>
__device__ __forceinline__ ChunkCut chunk_cut(const ChunkRows& p, Scan& scan, int Hkv, int T1, long long x) {
    if (x >= scan.total * Hkv) return ChunkCut{p.batch, 0, 0, 0};
    ChunkCut c;
    long long off;
    scan.find(x, Hkv, c.b, off);
    const ChunkTiles t(chunk_seq(p, c.b), T1);
    long long y = x - off;
    const long long head = t.cost();
    c.g = (int)(head >> 31 ? y / head : quick_div(y, (int)head));
    y -= c.g * head;
    const int lo = warp_search(t.tiles, y, [&](int j) { return t.cost_before(j); });
    c.j = lo;
    c.step = (int)min((long long)t.steps(lo), (quick_div(y - t.cost_before(lo), t.unit(lo)) + 64) >> 7);
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
        const ChunkTiles t(s, T1);
        tiles = t.tiles;
        steps = t.steps(at.j);
        single = t.unit(at.j) == kSingleCost;
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
    __device__ __forceinline__ int token0(int T1) const { return at.j * 2 * T1; }   // of the chunk
};

}  // namespace ffd
