// Attention of all query rows of a batch over a prefix that its sequences share: geometry and launch.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ffd.h"

namespace ffd {

constexpr int kPrefixRows = 128;     // query rows of a tile: the M of one tensor-core instruction
constexpr int kPrefixTokens = 128;   // prefix tokens of a step: two pages

constexpr int kPrefixCtaParts = 8;   // softmax warps of a CTA: its shares of the sequences' own tokens

struct PrefixParams {
    const __nv_bfloat16* q;          // [batch, Hq, 128]
    const int32_t* table;            // [max_blocks] pages of the prefix
    const int32_t* len;              // [1] tokens of the prefix
    int batch, Hq, Hkv, G, max_blocks, num_pages;
    int groups, chunks;              // of the geometry
    int items;                       // CTAs with a part of the prefix: Hkv * groups * chunks
    float logit_scale;               // sm_scale * log2(e)
    float* out;                      // [Hkv][chunks][batch * G][128] normalised partial attention
    float* lse;                      // [Hkv][chunks][batch * G] log2 of the sum of weights; -inf: empty
    uint32_t* status;
    int two_piece;                   // fp32 results: P keeps 16 bits in every geometry
};

// A CTA keeps one or two row tiles.  Up to 128 rows: one tile, whose two softmax warpgroups take alternate steps; more: two
// tiles per CTA, each step's K and V serving both, and ceil(rows / 256) groups of CTAs.  The prefix is then split into chunks,
// each a partial result, so that the grid is about one CTA per SM; CTAs without a part of the prefix are added while there are
// SMs and own tokens for them.
struct PrefixGeometry {
    int tiles, groups, chunks, ctas;
};
static inline PrefixGeometry prefix_geometry(int rows, int kv_heads, int max_blocks, long long own_blocks, int sms) {
    PrefixGeometry g;
    g.tiles = rows <= kPrefixRows ? 1 : 2;
    g.groups = (rows + g.tiles * kPrefixRows - 1) / (g.tiles * kPrefixRows);
    const int steps = (max_blocks + 1) / 2, base = kv_heads * g.groups;
    g.chunks = sms / base;
    if (g.chunks > steps) g.chunks = steps;
    if (g.chunks < 1) g.chunks = 1;
    const long long wanted = (own_blocks + kPrefixCtaParts - 1) / kPrefixCtaParts;
    g.ctas = base * g.chunks;
    if (g.ctas < sms) g.ctas = (int)(wanted < g.ctas ? g.ctas : wanted > sms ? sms : wanted);
    return g;
}

// one kernel on `stream`: the prefix (k and v: the 16-bit page pools) and the sequences' own tokens, in `format`
struct PagedParams;
ffd_status launch_prefix(const PrefixParams& p, const PrefixGeometry& geo, const void* k, const void* v, int format,
                         const PagedParams& own, cudaStream_t stream);

}  // namespace ffd
