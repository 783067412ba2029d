// What the host half of decoding by drafts and its kernels have to agree on: how verification is cut into work, and its workspace.
#ifndef EPARA_DRAFTS_H
#define EPARA_DRAFTS_H

#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"
#include "epara_plan.h"

namespace epara_drafts {

using epara_cache::TREE_ROWS;

// ---- verification.  A row of logits is taken in pieces of 16 bytes from the 16-byte boundary at or before its first element; a workgroup takes 256 * `pieces` of them.  A row
// of which nothing is known about alignment has up to one piece more than its length says.
EPARA_BOTH int element_bytes(int dtype) { return dtype == EPARA_F32 ? 4 : 2; }
EPARA_BOTH int pieces_of_row(int vocab, int dtype)
{
    const int per = 16 / element_bytes(dtype);
    return (vocab - 1 + per - 1) / per + 1;                // ceil((vocab + per - 1) / per)
}
EPARA_BOTH int chunks_of_row(int vocab, int dtype, int pieces) { return (pieces_of_row(vocab, dtype) + 256 * pieces - 1) / (256 * pieces); }

// The first kernel has a workgroup for each chunk of each row's logits, and of its draft logits behind those.
struct row_sum { float top; int32_t at; double sum; };     // of a chunk: the largest logit, where it is (greedy sequences only), sum of exp((x - top) / T)
EPARA_BOTH int64_t rows_items(const epara_verify_args& a, const epara_sequence& s, int chunks) { return static_cast<int64_t>(s.rows) * chunks * (a.draft_logits ? 2 : 1); }

// The second kernel, a workgroup to a sequence, leaves what the third has to know: the row behind which a token is drawn.
struct drawn_row {
    const void* p;                                         // its logits; NULL: nothing is left to draw
    const void* q;                                         // draft logits: the token comes from max(p - q, 0); else NULL
    double unit;                                           // weights are 2^((x - top) unit)
    double top_p, top_q, ratio;                            // ratio: sum of p's weights by sum of q's, as the first kernel has them
    int32_t vocab, n_without;
    float uniform;
    int32_t reserved;
    int32_t without[TREE_ROWS];                            // tokens that are left out
};
// The third has `chunks` workgroups for each sequence, as many as the largest vocabulary needs; with draw_pieces as `pieces` above.
struct chunk_sum { double p, q, rest, q_of_rest; };        // of a chunk: sums of p, of q, of max(p - ratio q, 0), and of q where that is not 0

// Workspace: a counter per sequence, drawn_row of each, then the first kernel's sums, then chunk_sum of each workgroup of the third.
EPARA_BOTH int64_t counter_bytes(int n_seqs) { return (static_cast<int64_t>(n_seqs) * 4 + 255) & ~static_cast<int64_t>(255); }

// ---- attention of trees.  Up to MID_ROWS rows to a key head are taken in tiles of 32 (32 trees of 32 with 128 rows to a head: 87 us, tiles of 128: 77), and up to MID_ROWS_ALONE where
// tiles of 128 would be too few to fill half the compute units (one tree of 64 with 256 rows to a head at 16000 tokens: 41 us, tiles of 128, whose parts take longer to join: 46; 183 rows
// of heads of 64 at 32768, capped: 32 and 44).  Fewer than 32 take one too, down to a single token: one request of 4 / 16 / 32 rows to a head at 4000 tokens 12.2 / 12.8 / 13.4 us, in the causal
// call's tiles of 16 9.0 / 10.6 / 12.4; 64 requests of 4 rows 85.8 and 82.8.
constexpr int MID_ROWS = 64, MID_ROWS_ALONE = 256;

// Pages to a workgroup: one workgroup (tiles of 128: two) to a compute unit where the work is small.  work: pages x key heads that the tiles of a kind see;
// longest: pages that one tile sees at most.  At least 8 / 16 pages: 8 drafts of one request at 4000 tokens 14.2 / 16.0 us; one workgroup to a unit / two: 16 rows of 2 requests at 8000
// 19.5 / 24.2; at most 32 / 64 / 128 pages: 9 to 16 rows of 105 requests 148 / 133 / 134, 64 rows of 8 requests, 40 heads 122 / 119 / 129.
inline int32_t tree_part_pages(int kind, int64_t work, int64_t longest, int32_t n_compute_units)
{
    const int64_t slots = (kind == 2 ? 2 : 1) * static_cast<int64_t>(n_compute_units), fewest = kind == 2 ? 16 : 8;
    const int64_t even = work / slots + 1, part = even < fewest ? fewest : even > 64 ? 64 : even;
    const int64_t least = (longest + epara_cache::MAX_PARTS - 1) / epara_cache::MAX_PARTS;
    return static_cast<int32_t>(part < least ? least : part);
}

// Workspace, where something is cut: a counter for each workgroup, then a slot for each workgroup of the kinds that are cut.
struct tree_workspace { int64_t slots[3], bytes; };
inline tree_workspace tree_workspace_of(const int32_t n_items[3], const bool cut[3])
{
    const int64_t items = static_cast<int64_t>(n_items[0]) + n_items[1] + n_items[2];
    tree_workspace w = {{0, 0, 0}, cut[0] || cut[1] || cut[2] ? (items * 4 + 255) & ~static_cast<int64_t>(255) : 0};
    for (int k = 0; k < 3; ++k) {
        w.slots[k] = w.bytes;
        if (cut[k]) w.bytes += static_cast<int64_t>(n_items[k]) * epara_cache::tree_tile(k) * epara_cache::SLOT_FLOATS * 4;
    }
    return w;
}

}  // namespace epara_drafts

EPARA_HIDDEN int32_t epara_check_trees_call(const epara_tree_args* h_args, int32_t G, const epara_sequence_table* table);
EPARA_HIDDEN int32_t epara_check_tree_attn_call(const epara_tree_attn_launch& launch, bool cut[3]);
EPARA_HIDDEN int32_t epara_check_verify_call(const epara_verify_launch& launch);
EPARA_HIDDEN int32_t epara_check_keep_call(const epara_keep_args* h_caches, int32_t n_caches, const epara_sequence_table* table, int32_t* n_items);

#endif
