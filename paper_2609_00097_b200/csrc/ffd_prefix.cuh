// Attention of all query rows of a batch over a prefix that its sequences share: geometry and launch.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ffd.h"

namespace ffd {

constexpr int kPrefixRows = 128;     // query rows of a tile: the M of one tensor-core instruction
constexpr int kPrefixTokens = 128;   // prefix tokens of a step: two pages

struct PrefixParams {
    const __nv_bfloat16* q;          // [batch, Hq, 128]
    const int32_t* table;            // [max_blocks] pages of the prefix
    const int32_t* len;              // [1] tokens of the prefix
    int batch, Hq, Hkv, G, max_blocks, num_pages;
    int splits;                      // partial results per (KV head, row)
    float logit_scale;               // sm_scale * log2(e)
    float* out;                      // [Hkv][splits][batch * G][128] normalised partial attention
    float* lse;                      // [Hkv][splits][batch * G] log2 of the sum of weights; -inf: empty
    uint32_t* status;
    int two_piece;                   // fp32 results: P keeps 16 bits in every geometry
};

// A CTA keeps one or two row tiles.  Up to 128 rows: one tile, whose two softmax warpgroups take alternate steps and leave
// two partials; more: two tiles per CTA, each step's K and V serving both, and ceil(rows / 256) groups of CTAs.  The prefix
// is then split so that the grid is about one CTA per SM.
struct PrefixGeometry {
    int tiles, groups, chunks, splits;   // chunks: parts of the prefix; splits: partials per row
};
static inline PrefixGeometry prefix_geometry(int rows, int kv_heads, int max_blocks, int sms) {
    PrefixGeometry g;
    g.tiles = rows <= kPrefixRows ? 1 : 2;
    g.groups = (rows + g.tiles * kPrefixRows - 1) / (g.tiles * kPrefixRows);
    const int steps = (max_blocks + 1) / 2, base = kv_heads * g.groups;
    g.chunks = sms / base;
    if (g.chunks > steps) g.chunks = steps;
    if (g.chunks < 1) g.chunks = 1;
    g.splits = g.tiles == 1 ? 2 * g.chunks : g.chunks;
    return g;
}
static inline int prefix_splits(int rows, int kv_heads, int max_blocks, int sms) {
    return prefix_geometry(rows, kv_heads, max_blocks, sms).splits;
}

// one kernel on `stream`; k and v are the 16-bit page pools
ffd_status launch_prefix(const PrefixParams& p, const void* k, const void* v, cudaStream_t stream);

}  // namespace ffd
