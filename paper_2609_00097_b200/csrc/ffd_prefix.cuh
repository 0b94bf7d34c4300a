// Attention of all query rows of a batch over a prefix that its sequences share: geometry and launch.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ffd.h"

namespace ffd {

constexpr int kPrefixRows = 128;     // query rows of a tile: the M of one tensor-core instruction
constexpr int kPrefixTokens = 128;   // prefix tokens of a step: two pages

constexpr int kPrefixCtaParts = 12;  // warps of a CTA that works on the sequences' own tokens

struct PrefixParams {
    const __nv_bfloat16* q;          // [batch, Hq, 128]
    const int32_t* table;            // [max_blocks] pages of the prefix
    const int32_t* len;              // [1] tokens of the prefix
    int batch, Hq, Hkv, G, max_blocks, num_pages;
    int groups, chunks;              // of the geometry
    float logit_scale;               // sm_scale * log2(e)
    float* out;                      // [Hkv][chunks][batch * G][128] normalised partial attention (the first ones of each head)
    float* lse;                      // [Hkv][chunks][batch * G] log2 of the sum of weights; -inf: empty
    uint32_t* status;
    int query_copy;                  // a tile holds whole sequences' heads: TMA copies it
    int two_piece;                   // fp32 results: P keeps 16 bits in every geometry
};

// A CTA on the prefix keeps one or two row tiles.  Up to 128 rows: one tile, whose two softmax warpgroups take alternate steps;
// more: two tiles per CTA, each step's K and V serving both, and ceil(rows / 256) groups of CTAs.  The prefix is split into at
// most `chunks` chunks, each a partial result, so that the grid is one CTA per SM with at least one left for the sequences'
// own tokens; the kernel settles for fewer when the lengths are such that the own tokens deserve more SMs.
struct PrefixGeometry {
    int tiles, groups, chunks, ctas, parts;   // parts: warps that the own tokens can have at most
};
static inline PrefixGeometry prefix_geometry(int rows, int kv_heads, int max_blocks, int sms) {
    PrefixGeometry g;
    g.tiles = rows <= kPrefixRows ? 1 : 2;
    g.groups = (rows + g.tiles * kPrefixRows - 1) / (g.tiles * kPrefixRows);
    const int steps = max_blocks / 2 + (max_blocks & 1), base = kv_heads * g.groups;
    g.ctas = base < sms ? sms : base + sms;
    g.chunks = (g.ctas - 1) / base;
    if (base >= sms) g.chunks = 1;
    if (g.chunks > steps) g.chunks = steps;
    g.parts = (g.ctas - base) * kPrefixCtaParts;
    return g;
}

// Rows of partial results that prefix_geometry can ask for (kv_heads * chunks * rows) with these or smaller rows and max_blocks.
// Up to 128 rows chunks * rows is at most min(steps, s) * rows, s = (sms - 1) / kv_heads; with ceil(rows / 256) groups it is at
// most s / groups * rows <= 256 s; and one chunk can always be had.
static inline size_t prefix_slots(int rows, int kv_heads, int max_blocks, int sms) {
    if (max_blocks <= 0) return 0;
    const size_t steps = ((size_t)max_blocks + 1) / 2, s = (size_t)(sms - 1) / kv_heads, n = (size_t)rows;
    const size_t split = s * (n < 2 * kPrefixRows ? n : 2 * kPrefixRows), all = steps * n < split ? steps * n : split;
    return kv_heads * (all > n ? all : n);
}

// one kernel on `stream`: the prefix (k and v: the 16-bit page pools) and the sequences' own tokens, in `format`
struct PagedParams;
ffd_status launch_prefix(const PrefixParams& p, const PrefixGeometry& geo, const void* k, const void* v, int format,
                         const PagedParams& own, cudaStream_t stream);

}  // namespace ffd
