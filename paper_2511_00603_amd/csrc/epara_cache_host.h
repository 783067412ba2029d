// Checks of the cache's calls (epara_cache_host.cpp), made before anything is enqueued (epara_cache.hip, epara_attend.hip).
#ifndef EPARA_CACHE_HOST_H
#define EPARA_CACHE_HOST_H

#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"
#include "epara_plan.h"

EPARA_HIDDEN int32_t epara_check_append_call(const epara_append_args* h_args, int32_t G, const epara_sequence_table* table, const int32_t* h_first);
EPARA_HIDDEN int32_t epara_check_attn_args(const epara_cache_attn_args* args, int32_t G, const epara_sequence_table* table, const epara_tree_args* trees);      // trees: or NULL
EPARA_HIDDEN int32_t epara_check_attn_call(const epara_cache_attn_launch& launch, bool cut[2]);      // cut: some context of few / many rows is in parts
EPARA_HIDDEN int32_t epara_check_copy_call(const epara_page_copy* caches, int32_t G, const epara_page_move* moves, int32_t n_moves, int32_t* n_chunks);

// Workspace of attention: a counter per workgroup of both kinds, padded to 256 bytes, then a slot per workgroup of each kind that is cut.
inline int64_t epara_attn_counter_bytes(const int32_t n_items[2]) { return ((static_cast<int64_t>(n_items[0]) + n_items[1]) * 4 + 255) & ~static_cast<int64_t>(255); }

// Pages to a workgroup.  work: pages x key heads that the tiles of each kind see; longest: pages that one tile sees at most.
// Few rows: one workgroup to a compute unit where the work is small (one request at 32768 tokens, 33 / 17 / 9 / 4 pages to a workgroup: 21.8 / 19.7 / 21.2 / 28.7 us; 4 at
// 8192: 21.6 / 18.1 / 18.6 / 25.5), at most 64 pages (16 requests at 16384: 64 pages 87 us, 33 93 us).  Many rows: two to a unit, at least 16 pages, since a part
// costs 64 KiB there and back.  There the times follow how the workgroups fill rounds of two to a unit more than a part's size (two pieces of 256 rows at 8000 tokens,
// at least 8 / 16 / 32 pages, 512 / 256 / 128 workgroups: 46.9 / 36.0 / 49.8 us; three pieces of 257 to 512 tokens at 3000 to 7000, 64 / 38 / 24 / 19 / 16 pages, all
// workgroups: 167 / 124 / 126 / 132 / 121 us, where this rule takes 38): a bound and an even load, not the best cut.
inline void epara_attn_part_pages(const int64_t work[2], const int64_t longest[2], int32_t n_compute_units, int32_t part_pages[2])
{
    for (int k = 0; k < 2; ++k) {
        const int64_t slots = (k + 1) * static_cast<int64_t>(n_compute_units), fewest = k ? 16 : 4;
        const int64_t even = work[k] / slots + 1, part = even < fewest ? fewest : even > 64 ? 64 : even;
        const int64_t least = (longest[k] + epara_cache::MAX_PARTS - 1) / epara_cache::MAX_PARTS;
        part_pages[k] = static_cast<int32_t>(part < least ? least : part);
    }
}

#endif
