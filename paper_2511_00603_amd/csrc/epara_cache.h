// What the cache's host half and its kernels have to agree on: the layout of a page, and how the sequences of a call are
// cut into work.  The formulas of the layout are the public header's.
#ifndef EPARA_CACHE_H
#define EPARA_CACHE_H

#include <stdint.h>

#include "epara.h"

#if defined(__HIPCC__) && defined(HIP_INCLUDE_HIP_HIP_RUNTIME_H)
#define EPARA_BOTH __host__ __device__ __forceinline__
#else
#define EPARA_BOTH inline
#endif

namespace epara_cache {

constexpr int PAGE = EPARA_CACHE_PAGE, BLOCK = EPARA_CACHE_BLOCK;

EPARA_BOTH int64_t head_bytes(int head_dim) { return 2 * PAGE * head_dim; }              // keys and values of a page and head

EPARA_BOTH int min_of(int a, int b) { return a < b ? a : b; }
EPARA_BOTH int max_of(int a, int b) { return a > b ? a : b; }

// ---- append: a wave per item.  First the blocks of 32 tokens that new tokens join, each with kv_heads items; then the
// queries: a lane takes 8 dims and their partners, so a wave takes `groups` pairs (row, head) at a time and QUERY_STEPS
// of those in an item: `rows` rows (a power of two) x heads.
constexpr int QUERY_STEPS = 4;
struct append_shape { int blocks, row_lanes, row_items, head_items; };
EPARA_BOTH append_shape shape_of_append(const epara_append_args& a, const epara_sequence& s)
{
    append_shape w = {0, 1, 0, 0};
    if (s.rows <= 0) return w;
    const int end = s.start + s.rows, from = max_of(s.start, 0);
    if (end > 0) w.blocks = (end - 1) / BLOCK - from / BLOCK + 1;
    if (a.Q) {
        const int groups = 64 / (a.head_dim / 16);
        while (w.row_lanes < groups && w.row_lanes < s.rows) w.row_lanes *= 2;
        const int heads = groups / w.row_lanes * QUERY_STEPS;
        w.row_items = (s.rows + w.row_lanes - 1) / w.row_lanes;
        w.head_items = (a.heads + heads - 1) / heads;
    }
    return w;
}
EPARA_BOTH int64_t append_items(const epara_append_args& a, const append_shape& w)
{
    return static_cast<int64_t>(w.blocks) * a.kv_heads + static_cast<int64_t>(w.row_items) * w.head_items;
}

// ---- attention: the rows of a sequence and key head are its tokens x the query heads that share the key head, token by
// token; a workgroup takes a tile of them against a part of the pages that the tile sees.
constexpr int FEW_TILE = 16, MANY_TILE = 128;
// Up to 32 rows to a key head are few.  Two tiles of 16 read a page twice, the second time from a die's cache, where a tile of 128 would leave three
// waves idle: 2 requests with 32 rows at 8000 tokens 16 us against 30, 16 of them 60 against 56; 64 rows 20 against 32 and 101 against 69.  (One limit for
// all loads: what is better at 32 to 64 rows depends on how many requests there are.)
constexpr int FEW_MAX_ROWS = 32;
constexpr int MAX_PARTS = 128;                             // of a tile's pages
constexpr int SLOT_FLOATS = 128 + 4;                       // per row of a part: the weighted sum of values, both references and the sum of weights
EPARA_BOTH bool has_few_rows(const epara_cache_attn_args& a, const epara_sequence& s) { return static_cast<int64_t>(s.rows) * (a.heads / a.kv_heads) <= FEW_MAX_ROWS; }

struct page_range { int lo, hi; };
// Pages that hold a key which the new rows first .. last of a sequence see; lo = hi = 0: none.  A row of a tree lies behind all rows that it follows, so it sees no key
// behind its own, but its position may be as low as the tree's first row's.
EPARA_BOTH page_range pages_of_rows(const epara_sequence& s, int window, bool tree, int first, int last)
{
    const int from = s.start + (tree ? 0 : first), to = s.start + last;
    if (to < 0) return {0, 0};
    const int lo = window > 0 && from >= window ? from - window + 1 : 0;
    return {lo / PAGE, to / PAGE + 1};
}

// ---- trees of drafted tokens: a sequence of up to EPARA_TREE_MAX_ROWS new rows is one where its service has bits of them
constexpr int TREE_ROWS = EPARA_TREE_MAX_ROWS, TREE_WORDS = TREE_ROWS / 64;
// The kinds of sequences of epara_tree_attention, by their rows to a key head: one tile of 32, several of them (up to mid_rows rows), tiles of 128.
constexpr int MID_TILE = 32, TREE_KINDS = 3;
EPARA_BOTH int tree_tile(int kind) { return kind < 2 ? MID_TILE : MANY_TILE; }
EPARA_BOTH int tree_kind(const epara_cache_attn_args& a, const epara_sequence& s, int mid_rows)
{
    const int64_t rows = static_cast<int64_t>(s.rows) * (a.heads / a.kv_heads);
    return rows <= MID_TILE ? 0 : rows <= mid_rows ? 1 : 2;
}
EPARA_BOTH bool is_tree(const epara_tree_args* trees, const epara_sequence& s) { return trees && s.rows <= TREE_ROWS && trees[s.service].visible; }

}  // namespace epara_cache

#endif
