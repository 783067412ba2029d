// Host half of decoding by drafts: argument checks and work counts.  Nothing here touches the GPU; no exception leaves an entry point.
#include "epara.h"
#include "epara_cache.h"
#include "epara_cache_checks.h"
#include "epara_cache_host.h"
#include "epara_drafts.h"

#include <algorithm>
#include <climits>
#include <functional>
#include <new>
#include <utility>
#include <vector>

using namespace epara_cache;
using namespace epara_drafts;

int32_t epara_check_trees_call(const epara_tree_args* args, int32_t G, const epara_sequence_table* t)
{
    if (G < 0) return EPARA_ERR_SHAPE;
    if (G > 0 && !args) return EPARA_ERR_NULL;
    for (int32_t g = 0; g < G; ++g) {
        const epara_tree_args& a = args[g];
        if (a.rows < 0) return EPARA_ERR_SHAPE;
        if (a.rows > 0 && (!a.parents || !a.visible)) return EPARA_ERR_NULL;
        if (misaligned(a.parents, 4) || misaligned(a.visible, 16) || misaligned(a.positions, 4)) return EPARA_ERR_ALIGN;
    }
    if (const int32_t rc = check_sequences(args, G, t)) return rc;
    for (int32_t i = 0; i < t->n_seqs; ++i)
        if (t->h_seqs[i].rows > 0 && t->h_seqs[i].rows <= TREE_ROWS && t->h_seqs[i].start < 0) return EPARA_ERR_SHAPE;
    return check_rows_once(args, t, [](const epara_tree_args&) { return true; });
}

namespace {

page_range pages_of_tile(const epara_cache_attn_args& a, const epara_sequence& s, bool tree, int size, int tile)
{
    const int group = a.heads / a.kv_heads, rows = s.rows * group;
    return pages_of_rows(s, a.window, tree, tile * size / group, (std::min(rows, tile * size + size) - 1) / group);
}
int tiles_of(const epara_cache_attn_args& a, const epara_sequence& s, int size) { return static_cast<int>(ceil_div(static_cast<int64_t>(s.rows) * (a.heads / a.kv_heads), size)); }

// Running sums of the workgroups of the three kinds of sequences, with parts of part_pages pages.
int32_t count_tree_attn(const epara_cache_attn_args* args, const epara_tree_args* trees, const epara_sequence_table* t, const int32_t part_pages[3], int32_t mid_rows,
                        int32_t* first, const int32_t* expected, int32_t n_items[3], bool cut[3])
{
    int64_t items[TREE_KINDS] = {};
    for (int k = 0; k < TREE_KINDS; ++k) cut[k] = false;
    for (int32_t i = 0; i <= t->n_seqs; ++i) {
        for (int k = 0; k < TREE_KINDS; ++k) {
            if (first) first[k * (t->n_seqs + 1) + i] = static_cast<int32_t>(items[k]);
            if (expected && expected[k * (t->n_seqs + 1) + i] != items[k]) return EPARA_ERR_SHAPE;
        }
        if (i == t->n_seqs) break;
        const epara_sequence& s = t->h_seqs[i];
        const epara_cache_attn_args& a = args[s.service];
        if (s.rows == 0) continue;
        const int k = tree_kind(a, s, mid_rows), size = tree_tile(k), tiles = tiles_of(a, s, size);
        int64_t parts = 1;
        for (int tile = 0; tile < tiles; ++tile) {
            const page_range r = pages_of_tile(a, s, is_tree(trees, s), size, tile);
            parts = std::max(parts, ceil_div(r.hi - r.lo, part_pages[k]));
        }
        if (parts > MAX_PARTS) return EPARA_ERR_SHAPE;
        cut[k] = cut[k] || parts > 1;
        items[k] += parts * tiles * a.kv_heads;
        if (items[k] > INT32_MAX / 256) return EPARA_ERR_CAPACITY;
    }
    for (int k = 0; k < TREE_KINDS; ++k) n_items[k] = static_cast<int32_t>(items[k]);
    return EPARA_OK;
}

}  // namespace

int32_t epara_check_tree_attn_call(const epara_tree_attn_launch& l, bool cut[3])
{
    if (l.G > 0 && !l.h_trees) return EPARA_ERR_NULL;
    if (const int32_t rc = epara_check_attn_args(l.h_args, l.G, &l.table, l.h_trees)) return rc;
    if (l.table.n_seqs == 0) return EPARA_OK;
    if (!l.h_first) return EPARA_ERR_NULL;
    for (int k = 0; k < TREE_KINDS; ++k)
        if (l.plan.part_pages[k] < 1) return EPARA_ERR_SHAPE;
    int32_t n[TREE_KINDS];
    if (const int32_t rc = count_tree_attn(l.h_args, l.h_trees, &l.table, l.plan.part_pages, l.plan.mid_rows, nullptr, l.h_first, n, cut)) return rc;
    if (!std::equal(n, n + TREE_KINDS, l.plan.n_items)) return EPARA_ERR_SHAPE;
    if (const int32_t rc = check_rows_once(l.h_args, &l.table, [](const epara_cache_attn_args&) { return true; })) return rc;
    const int64_t bytes = tree_workspace_of(n, cut).bytes;
    if (bytes > 0) {
        if (!l.d_workspace) return EPARA_ERR_NULL;
        if (misaligned(l.d_workspace, 256)) return EPARA_ERR_ALIGN;
        if (l.workspace_bytes < bytes) return EPARA_ERR_CAPACITY;
    }
    return EPARA_OK;
}

extern "C" int32_t epara_plan_tree_attention(const epara_cache_attn_args* h_args, const epara_tree_args* h_trees, int32_t G, const epara_sequence_table* table, int32_t n_compute_units,
                                             int32_t* first, epara_tree_attn_plan* plan)
{
    if (G > 0 && !h_trees) return EPARA_ERR_NULL;
    if (const int32_t rc = epara_check_attn_args(h_args, G, table, h_trees)) return rc;
    if (!first || !plan) return EPARA_ERR_NULL;
    if (n_compute_units < 1 || n_compute_units > 65536) return EPARA_ERR_SHAPE;
    *plan = {};
    int64_t many = 0;                                      // tiles of 128 that a rule by rows alone would give
    for (int32_t i = 0; i < table->n_seqs; ++i) {
        const epara_cache_attn_args& a = h_args[table->h_seqs[i].service];
        if (tree_kind(a, table->h_seqs[i], MID_ROWS) == 2) many += static_cast<int64_t>(tiles_of(a, table->h_seqs[i], MANY_TILE)) * a.kv_heads;
    }
    plan->mid_rows = many < n_compute_units / 2 ? MID_ROWS_ALONE : MID_ROWS;
    int64_t work[TREE_KINDS] = {}, longest[TREE_KINDS] = {};
    for (int32_t i = 0; i < table->n_seqs; ++i) {
        const epara_sequence& s = table->h_seqs[i];
        const epara_cache_attn_args& a = h_args[s.service];
        if (s.rows == 0) continue;
        const int k = tree_kind(a, s, plan->mid_rows), size = tree_tile(k), tiles = tiles_of(a, s, size);
        for (int tile = 0; tile < tiles; ++tile) {
            const page_range r = pages_of_tile(a, s, is_tree(h_trees, s), size, tile);
            work[k] += static_cast<int64_t>(r.hi - r.lo) * a.kv_heads;
            longest[k] = std::max<int64_t>(longest[k], r.hi - r.lo);
        }
    }
    for (int k = 0; k < TREE_KINDS; ++k) plan->part_pages[k] = tree_part_pages(k, work[k], longest[k], n_compute_units);
    bool cut[TREE_KINDS];
    if (const int32_t rc = count_tree_attn(h_args, h_trees, table, plan->part_pages, plan->mid_rows, first, nullptr, plan->n_items, cut)) return rc;
    plan->workspace_bytes = tree_workspace_of(plan->n_items, cut).bytes;
    return EPARA_OK;
}

namespace {

// Of a sequence's record only service, first_row and rows count.
int32_t check_verify(const epara_verify_args* args, int32_t G, const epara_sequence_table* t, int32_t dtype)
{
    if (G < 0) return EPARA_ERR_SHAPE;
    if (dtype != EPARA_BF16 && dtype != EPARA_F32) return EPARA_ERR_DTYPE;
    if ((G > 0 && !args) || !t) return EPARA_ERR_NULL;
    const uintptr_t size = static_cast<uintptr_t>(element_bytes(dtype));
    for (int32_t g = 0; g < G; ++g) {
        const epara_verify_args& a = args[g];
        if (a.rows < 0 || a.vocab < 1 || a.vocab > INT32_MAX / 8 || a.stride < a.vocab || (a.draft_logits && a.draft_stride < a.vocab)) return EPARA_ERR_SHAPE;
        if (a.rows > 0 && (!a.logits || !a.tokens || !a.uniforms || !a.path)) return EPARA_ERR_NULL;
        if (misaligned(a.logits, size) || misaligned(a.draft_logits, size) || misaligned(a.tokens, 4) || misaligned(a.parents, 4) || misaligned(a.uniforms, 4) ||
            misaligned(a.path, 4) || misaligned(a.probs, 4)) return EPARA_ERR_ALIGN;
    }
    if (t->n_seqs < 0) return EPARA_ERR_SHAPE;
    if (t->n_seqs > 0 && (!t->h_seqs || !t->d_seqs)) return EPARA_ERR_NULL;
    int32_t service = 0;
    for (int32_t i = 0; i < t->n_seqs; ++i) {
        const epara_sequence& s = t->h_seqs[i];
        if (s.service < service || s.service >= G) return EPARA_ERR_SHAPE;
        service = s.service;
        if (s.rows < 0 || s.rows > TREE_ROWS || s.first_row < 0 || static_cast<int64_t>(s.first_row) + s.rows > args[service].rows) return EPARA_ERR_SHAPE;
    }
    return EPARA_OK;
}

// The plan's numbers for its `pieces` and `draw_pieces`, and the running sums.
int32_t count_verify(const epara_verify_args* args, const epara_sequence_table* t, int32_t dtype, int32_t* first, const int32_t* expected, epara_verify_plan* plan)
{
    int64_t items = 0;
    plan->draw_chunks = 1;
    for (int32_t i = 0; i <= t->n_seqs; ++i) {
        if (first) first[i] = static_cast<int32_t>(items);
        if (expected && expected[i] != items) return EPARA_ERR_SHAPE;
        if (i == t->n_seqs) break;
        const epara_sequence& s = t->h_seqs[i];
        const int32_t vocab = args[s.service].vocab;
        items += rows_items(args[s.service], s, chunks_of_row(vocab, dtype, plan->pieces));
        plan->draw_chunks = std::max(plan->draw_chunks, chunks_of_row(vocab, dtype, plan->draw_pieces));
        if (items > INT32_MAX / 256 || static_cast<int64_t>(t->n_seqs) * plan->draw_chunks > INT32_MAX / 256) return EPARA_ERR_CAPACITY;
    }
    plan->n_items = static_cast<int32_t>(items);
    plan->workspace_bytes = counter_bytes(t->n_seqs) + static_cast<int64_t>(t->n_seqs) * sizeof(drawn_row) + items * sizeof(row_sum) +
                            static_cast<int64_t>(t->n_seqs) * plan->draw_chunks * sizeof(chunk_sum);
    return EPARA_OK;
}

}  // namespace

int32_t epara_check_verify_call(const epara_verify_launch& l)
{
    if (const int32_t rc = check_verify(l.h_args, l.G, &l.table, l.dtype)) return rc;
    if (l.table.n_seqs == 0) return EPARA_OK;
    if (!l.h_first || !l.d_kept || !l.d_next || !l.d_workspace) return EPARA_ERR_NULL;
    epara_verify_plan plan = l.plan;
    const int32_t p = plan.pieces, d = plan.draw_pieces;
    if ((p != 1 && p != 2 && p != 4 && p != 8) || (d != 1 && d != 2 && d != 4)) return EPARA_ERR_SHAPE;
    if (const int32_t rc = count_verify(l.h_args, &l.table, l.dtype, nullptr, l.h_first, &plan)) return rc;
    if (plan.n_items != l.plan.n_items || plan.draw_chunks != l.plan.draw_chunks) return EPARA_ERR_SHAPE;
    if (misaligned(l.d_temperatures, 4) || misaligned(l.d_kept, 4) || misaligned(l.d_next, 4) || misaligned(l.d_workspace, 256)) return EPARA_ERR_ALIGN;
    if (l.workspace_bytes < plan.workspace_bytes) return EPARA_ERR_CAPACITY;
    return check_rows_once(l.h_args, &l.table, [](const epara_verify_args&) { return true; });
}

int32_t epara_check_keep_call(const epara_keep_args* caches, int32_t n_caches, const epara_sequence_table* t, int32_t* n_items)
{
    *n_items = 0;
    if (n_caches < 0) return EPARA_ERR_SHAPE;
    if ((n_caches > 0 && !caches) || !t) return EPARA_ERR_NULL;
    if (t->n_seqs < 0 || t->n_table < 0) return EPARA_ERR_SHAPE;
    if (t->n_seqs > 0 && (!t->h_seqs || !t->d_seqs)) return EPARA_ERR_NULL;
    if (t->n_table > 0 && (!t->h_pages || !t->d_pages)) return EPARA_ERR_NULL;
    for (int32_t i = 0; i < t->n_seqs; ++i) {
        const epara_sequence& s = t->h_seqs[i];
        if (s.service < (i ? t->h_seqs[i - 1].service : 0) || s.rows < 0 || s.first_row < 0) return EPARA_ERR_SHAPE;
        if (s.first_page < 0 || s.n_pages < 0 || static_cast<int64_t>(s.first_page) + s.n_pages > t->n_table) return EPARA_ERR_SHAPE;
        if (s.start < -EPARA_CACHE_MAX_TOKENS || static_cast<int64_t>(s.start) + s.rows > std::min<int64_t>(EPARA_CACHE_MAX_TOKENS, static_cast<int64_t>(s.n_pages) * PAGE)) return EPARA_ERR_SHAPE;
        if (s.rows > 0 && s.rows <= TREE_ROWS && s.start < 0) return EPARA_ERR_SHAPE;
    }
    const auto by_service = [](const epara_sequence& s, int32_t service) { return s.service < service; };
    int64_t items = 0;
    try {
        std::vector<int32_t> written;
        std::vector<std::pair<const void*, int32_t>> codes;
        const epara_keep_args* before = nullptr;
        for (int32_t g = 0; g < n_caches; ++g) {
            const epara_keep_args& c = caches[g];
            if (c.service < 0 || c.rows < 0 || bad_heads(c.kv_heads, c.kv_heads, c.head_dim, c.n_pages)) return EPARA_ERR_SHAPE;
            const epara_sequence* lo = std::lower_bound(t->h_seqs, t->h_seqs + t->n_seqs, c.service, by_service);
            const epara_sequence* hi = std::lower_bound(lo, t->h_seqs + t->n_seqs, c.service + 1, by_service);
            if (c.first_seq != lo - t->h_seqs || c.first_item != items) return EPARA_ERR_SHAPE;
            items += static_cast<int64_t>(hi - lo) * c.kv_heads;
            if (items > INT32_MAX / 256) return EPARA_ERR_CAPACITY;
            if (lo == hi) continue;
            if (!c.codes || !c.scales || (c.rows > 0 && !c.path)) return EPARA_ERR_NULL;
            if (misaligned(c.codes, 16) || misaligned(c.scales, 4) || misaligned(c.path, 4)) return EPARA_ERR_ALIGN;
            codes.emplace_back(c.codes, g);
            // the layers of a service follow each other with as many rows and pages: looked at once
            if (before && before->service == c.service && before->rows == c.rows && before->n_pages == c.n_pages) continue;
            before = &c;
            written.clear();
            for (const epara_sequence* s = lo; s != hi; ++s) {
                if (static_cast<int64_t>(s->first_row) + s->rows > c.rows) return EPARA_ERR_SHAPE;
                if (s->rows == 0 || s->rows > TREE_ROWS) continue;
                const int from = s->start / PAGE, upto = (s->start + s->rows - 1) / PAGE + 1;
                if (!pages_inside(t, *s, from, upto, c.n_pages)) return EPARA_ERR_SHAPE;
                for (int p = from; p < upto; ++p) written.push_back(t->h_pages[s->first_page + p]);
            }
            std::sort(written.begin(), written.end());
            if (std::adjacent_find(written.begin(), written.end()) != written.end()) return EPARA_ERR_SHAPE;
        }
        std::sort(codes.begin(), codes.end(), [](const std::pair<const void*, int32_t>& a, const std::pair<const void*, int32_t>& b) { return std::less<const void*>()(a.first, b.first); });
        for (size_t i = 1; i < codes.size(); ++i)
            if (codes[i].first == codes[i - 1].first) return EPARA_ERR_SHAPE;
    } catch (const std::bad_alloc&) {
        return EPARA_ERR_CAPACITY;
    }
    *n_items = static_cast<int32_t>(items);
    return EPARA_OK;
}

extern "C" int32_t epara_plan_verify_drafts(const epara_verify_args* h_args, int32_t G, const epara_sequence_table* table, int32_t dtype, int32_t n_compute_units,
                                            int32_t* first, epara_verify_plan* plan)
{
    if (const int32_t rc = check_verify(h_args, G, table, dtype)) return rc;
    if (!first || !plan) return EPARA_ERR_NULL;
    if (n_compute_units < 1 || n_compute_units > 65536) return EPARA_ERR_SHAPE;
    int64_t pieces = 0, draws = 0;                         // of 16 bytes in all rows, and in one of each sequence
    for (int32_t i = 0; i < table->n_seqs; ++i) {
        const epara_verify_args& a = h_args[table->h_seqs[i].service];
        pieces += rows_items(a, table->h_seqs[i], 1) * pieces_of_row(a.vocab, dtype);
        draws += pieces_of_row(a.vocab, dtype);
    }
    // Chunks as large as leave 8 workgroups of the first kernel to a compute unit, 4 of the third.  1 / 2 / 4 / 8 pieces: 8 trees of 40 to 64 rows at 50021 tokens 40.6 / 31.9 / 28.9 / 28.0 us,
    // one chain of 6 at 32000 13.9 / 13.9 / 14.1 / 14.4; 1 / 2 / 4 draw_pieces: 64 chains at 131072 79.5 / 64.4 / 65.8 us, 32 trees at 100003 in fp32 45.1 / 38.3 / 37.2, the 8 trees
    // 28.0 / 28.4 / 30.8, the one chain 13.9 / 15.0 / 17.2
    *plan = {};
    plan->pieces = plan->draw_pieces = 1;
    while (plan->pieces < 8 && pieces >= static_cast<int64_t>(n_compute_units) * 8 * 256 * plan->pieces) plan->pieces *= 2;
    while (plan->draw_pieces < 4 && draws >= static_cast<int64_t>(n_compute_units) * 4 * 256 * plan->draw_pieces) plan->draw_pieces *= 2;
    return count_verify(h_args, table, dtype, first, nullptr, plan);
}
