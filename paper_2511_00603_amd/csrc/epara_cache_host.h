// Checks of the cache's calls (epara_cache_host.cpp), made before anything is enqueued (epara_cache.hip, epara_attend.hip).
#ifndef EPARA_CACHE_HOST_H
#define EPARA_CACHE_HOST_H

#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"
#include "epara_plan.h"

EPARA_HIDDEN int32_t epara_check_append_call(const epara_append_args* h_args, int32_t G, const epara_sequence_table* table, const int32_t* h_first);
EPARA_HIDDEN int32_t epara_check_attn_call(const epara_cache_attn_launch& launch, bool cut[2]);      // cut: some context of few / many rows is in parts
EPARA_HIDDEN int32_t epara_check_copy_call(const epara_page_copy* caches, int32_t G, const epara_page_move* moves, int32_t n_moves, int32_t* n_chunks);

// Workspace of attention: a counter per workgroup of both kinds, padded to 256 bytes, then a slot per workgroup of each kind that is cut.
inline int64_t epara_attn_counter_bytes(const int32_t n_items[2]) { return ((static_cast<int64_t>(n_items[0]) + n_items[1]) * 4 + 255) & ~static_cast<int64_t>(255); }

// Pages to a workgroup.  work: pages x key heads that the tiles of each kind see; longest: pages that one tile sees at most.
inline void epara_attn_part_pages(const int64_t work[2], const int64_t longest[2], int32_t n_compute_units, int32_t part_pages[2])
{
    for (int k = 0; k < 2; ++k) {
        const int64_t even = work[k] / ((k + 1) * static_cast<int64_t>(n_compute_units)) + 1, least = (longest[k] + epara_cache::MAX_PARTS - 1) / epara_cache::MAX_PARTS;
        const int64_t part = even < 4 ? 4 : even > 64 ? 64 : even;
        part_pages[k] = static_cast<int32_t>(part < least ? least : part);
    }
}

#endif
