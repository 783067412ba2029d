// Host half of the paged cache: argument checks and work counts of the calls on it, and the bookkeeping of its pages.
// Nothing here touches the GPU; no exception leaves an entry point.
#include "epara.h"
#include "epara_cache.h"
#include "epara_cache_host.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <functional>
#include <new>
#include <vector>

using namespace epara_cache;

namespace {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

bool bad_heads(int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t n_pages)
{
    return heads < 1 || kv_heads < 1 || heads % kv_heads != 0 || heads / kv_heads > EPARA_CACHE_MAX_GROUP || heads > 65536 || (head_dim != 64 && head_dim != 128) || n_pages < 0;
}

// The sequences of a call against the services' rows and the page table.
template <class Args>
int32_t check_sequences(const Args* args, int32_t G, const epara_sequence_table* t)
{
    if (!t) return EPARA_ERR_NULL;
    if (t->n_seqs < 0 || t->n_table < 0) return EPARA_ERR_SHAPE;
    if (t->n_seqs > 0 && (!t->h_seqs || !t->d_seqs)) return EPARA_ERR_NULL;
    if (t->n_table > 0 && (!t->h_pages || !t->d_pages)) return EPARA_ERR_NULL;
    int32_t service = 0;
    for (int32_t i = 0; i < t->n_seqs; ++i) {
        const epara_sequence& s = t->h_seqs[i];
        if (s.service < service || s.service >= G) return EPARA_ERR_SHAPE;
        service = s.service;
        if (s.rows < 0 || s.first_row < 0 || static_cast<int64_t>(s.first_row) + s.rows > args[service].rows) return EPARA_ERR_SHAPE;
        if (s.first_page < 0 || s.n_pages < 0 || static_cast<int64_t>(s.first_page) + s.n_pages > t->n_table) return EPARA_ERR_SHAPE;
        if (s.start < -EPARA_CACHE_MAX_TOKENS || static_cast<int64_t>(s.start) + s.rows > std::min<int64_t>(EPARA_CACHE_MAX_TOKENS, static_cast<int64_t>(s.n_pages) * PAGE)) return EPARA_ERR_SHAPE;
    }
    return EPARA_OK;
}

// The pages [lo, hi) of a sequence lie inside its service's cache.
bool pages_inside(const epara_sequence_table* t, const epara_sequence& s, int lo, int hi, int32_t n_pages)
{
    for (int p = lo; p < hi; ++p) {
        const int32_t id = t->h_pages[s.first_page + p];
        if (id < 0 || id >= n_pages) return false;
    }
    return true;
}

int32_t check_append(const epara_append_args* args, int32_t G, const epara_sequence_table* t)
{
    if (G < 0) return EPARA_ERR_SHAPE;
    if (G > 0 && !args) return EPARA_ERR_NULL;
    for (int32_t g = 0; g < G; ++g) {
        const epara_append_args& a = args[g];
        if (a.rows < 0 || bad_heads(a.heads, a.kv_heads, a.head_dim, a.n_pages)) return EPARA_ERR_SHAPE;
        const int64_t width = static_cast<int64_t>(a.heads + 2 * static_cast<int64_t>(a.kv_heads)) * a.head_dim;
        if (a.qkv_stride < width || (a.qkv_stride & 7) || (a.Q && (a.q_stride < static_cast<int64_t>(a.heads) * a.head_dim || (a.q_stride & 7)))) return EPARA_ERR_SHAPE;
        if (a.axis_pairs[0] < 0 || a.axis_pairs[1] < 0 || static_cast<int64_t>(a.axis_pairs[0]) + a.axis_pairs[1] > a.head_dim / 2) return EPARA_ERR_SHAPE;
        if (a.rotary && a.n_positions < 1) return EPARA_ERR_SHAPE;
        if (a.rows > 0 && (!a.QKV || !a.codes || !a.scales || (a.rotary && !a.Q))) return EPARA_ERR_NULL;
        if (a.rows > 0 && a.Q == a.QKV) return EPARA_ERR_SHAPE;
        if (misaligned(a.QKV, 16) || misaligned(a.Q, 16) || misaligned(a.codes, 16) || misaligned(a.scales, 4) || misaligned(a.rotary, 16) || misaligned(a.positions, 4)) return EPARA_ERR_ALIGN;
    }
    if (const int32_t rc = check_sequences(args, G, t)) return rc;
    for (int32_t i = 0; i < t->n_seqs; ++i) {
        const epara_sequence& s = t->h_seqs[i];
        const epara_append_args& a = args[s.service];
        const int end = s.start + s.rows;
        if (s.rows == 0 || end <= 0) continue;
        if (a.rotary && !a.positions && end > a.n_positions) return EPARA_ERR_SHAPE;
        if (!pages_inside(t, s, std::max(s.start, 0) / PAGE, (end - 1) / PAGE + 1, a.n_pages)) return EPARA_ERR_SHAPE;
    }
    return EPARA_OK;
}

// No row is written for two sequences of a service; writes(args): whether that service's rows are.  Sequences in the order of their rows, as a rule, need no list.
template <class Args, class Writes>
int32_t check_rows_once(const Args* args, const epara_sequence_table* t, Writes writes)
{
    bool ordered = true;
    int32_t service = -1, end = 0;
    for (int32_t i = 0; i < t->n_seqs && ordered; ++i) {
        const epara_sequence& s = t->h_seqs[i];
        if (s.rows == 0 || !writes(args[s.service])) continue;
        ordered = s.service != service || s.first_row >= end;
        service = s.service;
        end = s.first_row + s.rows;
    }
    if (ordered) return EPARA_OK;
    try {
        std::vector<epara_sequence> seqs;
        for (int32_t i = 0; i < t->n_seqs; ++i)
            if (t->h_seqs[i].rows > 0 && writes(args[t->h_seqs[i].service])) seqs.push_back(t->h_seqs[i]);
        std::sort(seqs.begin(), seqs.end(), [](const epara_sequence& a, const epara_sequence& b) { return a.service != b.service ? a.service < b.service : a.first_row < b.first_row; });
        const auto meet = [](const epara_sequence& a, const epara_sequence& b) { return a.service == b.service && b.first_row < a.first_row + a.rows; };
        return std::adjacent_find(seqs.begin(), seqs.end(), meet) == seqs.end() ? EPARA_OK : EPARA_ERR_SHAPE;
    } catch (const std::bad_alloc&) {
        return EPARA_ERR_CAPACITY;
    }
}

// No page of a cache is written for two sequences (or twice for one).
int32_t check_written_once(const epara_append_args* args, const epara_sequence_table* t)
{
    try {
        std::vector<std::pair<const void*, int32_t>> written;
        for (int32_t i = 0; i < t->n_seqs; ++i) {
            const epara_sequence& s = t->h_seqs[i];
            if (s.rows == 0 || s.start + s.rows <= 0) continue;
            for (int p = std::max(s.start, 0) / PAGE; p <= (s.start + s.rows - 1) / PAGE; ++p) written.emplace_back(args[s.service].codes, t->h_pages[s.first_page + p]);
        }
        std::sort(written.begin(), written.end());
        return std::adjacent_find(written.begin(), written.end()) == written.end() ? EPARA_OK : EPARA_ERR_SHAPE;
    } catch (const std::bad_alloc&) {
        return EPARA_ERR_CAPACITY;
    }
}

int32_t count_append(const epara_append_args* args, const epara_sequence_table* t, int32_t* first, const int32_t* expected)
{
    int64_t items = 0;
    for (int32_t i = 0; i <= t->n_seqs; ++i) {
        if (first) first[i] = static_cast<int32_t>(items);
        if (expected && expected[i] != items) return EPARA_ERR_SHAPE;
        if (i == t->n_seqs) break;
        items += append_items(args[t->h_seqs[i].service], shape_of_append(args[t->h_seqs[i].service], t->h_seqs[i]));
        if (items > INT32_MAX / 64) return EPARA_ERR_CAPACITY;
    }
    return EPARA_OK;
}

int32_t check_attn(const epara_cache_attn_args* args, int32_t G, const epara_sequence_table* t)
{
    if (G < 0) return EPARA_ERR_SHAPE;
    if (G > 0 && !args) return EPARA_ERR_NULL;
    for (int32_t g = 0; g < G; ++g) {
        const epara_cache_attn_args& a = args[g];
        if (a.rows < 0 || bad_heads(a.heads, a.kv_heads, a.head_dim, a.n_pages) || a.window < 0) return EPARA_ERR_SHAPE;
        if (a.q_stride < static_cast<int64_t>(a.heads) * a.head_dim || (a.q_stride & 7) || a.o_stride < static_cast<int64_t>(a.heads) * a.head_dim || (a.o_stride & 7)) return EPARA_ERR_SHAPE;
        if (!(a.scale > 0.f) || !std::isfinite(a.scale) || !(a.softcap >= 0.f) || !std::isfinite(a.softcap)) return EPARA_ERR_SHAPE;
        if (a.rows > 0 && (!a.Q || !a.O || !a.codes || !a.scales)) return EPARA_ERR_NULL;
        if (a.rows > 0 && a.Q == a.O) return EPARA_ERR_SHAPE;
        if (misaligned(a.Q, 16) || misaligned(a.O, 16) || misaligned(a.codes, 16) || misaligned(a.scales, 4)) return EPARA_ERR_ALIGN;
    }
    if (const int32_t rc = check_sequences(args, G, t)) return rc;
    for (int32_t i = 0; i < t->n_seqs; ++i) {
        const epara_sequence& s = t->h_seqs[i];
        const epara_cache_attn_args& a = args[s.service];
        if (s.rows == 0) continue;
        if (static_cast<int64_t>(s.rows) * (a.heads / a.kv_heads) > INT32_MAX / 2) return EPARA_ERR_CAPACITY;
        const page_range r = pages_of_tokens(s, a.window, std::min(std::max(-s.start, 0), s.rows - 1), s.rows - 1);
        if (!pages_inside(t, s, r.lo, r.hi, a.n_pages)) return EPARA_ERR_SHAPE;
    }
    return EPARA_OK;
}

struct seq_tiles { int few, tiles; };
seq_tiles tiles_of(const epara_cache_attn_args& a, const epara_sequence& s)
{
    const int few = has_few_rows(a, s) ? 1 : 0;
    return {few, static_cast<int>(ceil_div(static_cast<int64_t>(s.rows) * (a.heads / a.kv_heads), few ? FEW_TILE : MANY_TILE))};
}

page_range pages_of_tile(const epara_cache_attn_args& a, const epara_sequence& s, int few, int tile)
{
    const int group = a.heads / a.kv_heads, size = few ? FEW_TILE : MANY_TILE, rows = s.rows * group;
    return pages_of_tokens(s, a.window, tile * size / group, (std::min(rows, tile * size + size) - 1) / group);
}

// Running sums of workgroups of both kinds of sequences, with parts of part_pages pages.
int32_t count_attn(const epara_cache_attn_args* args, const epara_sequence_table* t, const int32_t part_pages[2], int32_t* first, const int32_t* expected,
                   int32_t n_items[2], bool cut[2])
{
    int64_t items[2] = {0, 0};
    cut[0] = cut[1] = false;
    for (int32_t i = 0; i <= t->n_seqs; ++i) {
        for (int k = 0; k < 2; ++k) {
            if (first) first[k * (t->n_seqs + 1) + i] = static_cast<int32_t>(items[k]);
            if (expected && expected[k * (t->n_seqs + 1) + i] != items[k]) return EPARA_ERR_SHAPE;
        }
        if (i == t->n_seqs) break;
        const epara_sequence& s = t->h_seqs[i];
        const epara_cache_attn_args& a = args[s.service];
        if (s.rows == 0) continue;
        const seq_tiles w = tiles_of(a, s);
        const int k = w.few ? 0 : 1;
        int64_t parts = 1;
        for (int tile = 0; tile < w.tiles; ++tile) {
            const page_range r = pages_of_tile(a, s, w.few, tile);
            parts = std::max(parts, ceil_div(r.hi - r.lo, part_pages[k]));
        }
        if (parts > MAX_PARTS) return EPARA_ERR_SHAPE;
        if (parts > 1) cut[k] = true;
        items[k] += parts * w.tiles * a.kv_heads;
        if (items[k] > INT32_MAX / 256) return EPARA_ERR_CAPACITY;
    }
    n_items[0] = static_cast<int32_t>(items[0]);
    n_items[1] = static_cast<int32_t>(items[1]);
    return EPARA_OK;
}

int64_t attn_workspace(const int32_t n_items[2], const bool cut[2])
{
    if (!cut[0] && !cut[1]) return 0;
    return epara_attn_counter_bytes(n_items) + (cut[0] ? static_cast<int64_t>(n_items[0]) * FEW_TILE * SLOT_FLOATS * 4 : 0) +
           (cut[1] ? static_cast<int64_t>(n_items[1]) * MANY_TILE * SLOT_FLOATS * 4 : 0);
}

}  // namespace

int32_t epara_check_append_call(const epara_append_args* h_args, int32_t G, const epara_sequence_table* table, const int32_t* h_first)
{
    if (const int32_t rc = check_append(h_args, G, table)) return rc;
    if (table->n_seqs > 0 && !h_first) return EPARA_ERR_NULL;
    if (table->n_seqs == 0) return EPARA_OK;
    if (const int32_t rc = count_append(h_args, table, nullptr, h_first)) return rc;
    if (const int32_t rc = check_rows_once(h_args, table, [](const epara_append_args& a) { return a.Q != nullptr; })) return rc;
    return check_written_once(h_args, table);
}

int32_t epara_check_attn_call(const epara_cache_attn_launch& l, bool cut[2])
{
    if (const int32_t rc = check_attn(l.h_args, l.G, &l.table)) return rc;
    cut[0] = cut[1] = false;
    if (l.table.n_seqs == 0) return EPARA_OK;
    if (!l.h_first) return EPARA_ERR_NULL;
    if (l.plan.part_pages[0] < 1 || l.plan.part_pages[1] < 1) return EPARA_ERR_SHAPE;
    int32_t n[2];
    if (const int32_t rc = count_attn(l.h_args, &l.table, l.plan.part_pages, nullptr, l.h_first, n, cut)) return rc;
    if (n[0] != l.plan.n_items[0] || n[1] != l.plan.n_items[1]) return EPARA_ERR_SHAPE;
    if (const int32_t rc = check_rows_once(l.h_args, &l.table, [](const epara_cache_attn_args&) { return true; })) return rc;
    const int64_t bytes = attn_workspace(n, cut);
    if (bytes > 0) {
        if (!l.d_workspace) return EPARA_ERR_NULL;
        if (misaligned(l.d_workspace, 256)) return EPARA_ERR_ALIGN;
        if (l.workspace_bytes < bytes) return EPARA_ERR_CAPACITY;
    }
    return EPARA_OK;
}

namespace {

// The moves of caches[order[0 .. n)], which are one cache: no page is twice a destination, or a destination and a source.  used: scratch.
int32_t check_moves(const epara_page_copy* caches, const int32_t* order, int32_t n, const epara_page_move* moves, std::vector<char>& used)
{
    const epara_page_copy& one = caches[order[0]];
    used.assign(static_cast<size_t>(one.n_pages), 0);            // per page: 1 a source, 2 a destination
    for (int32_t k = 0; k < n; ++k) {
        const epara_page_copy& c = caches[order[k]];
        if (c.n_pages != one.n_pages || c.kv_heads != one.kv_heads || c.head_dim != one.head_dim) return EPARA_ERR_SHAPE;
        for (int32_t i = c.first_move; i < c.first_move + c.n_moves; ++i) {
            const epara_page_move& m = moves[i];
            if (m.src < 0 || m.src >= c.n_pages || m.dst < 0 || m.dst >= c.n_pages || m.src == m.dst) return EPARA_ERR_SHAPE;
            if (used[static_cast<size_t>(m.src)] == 2 || used[static_cast<size_t>(m.dst)] != 0) return EPARA_ERR_SHAPE;
            used[static_cast<size_t>(m.src)] = 1;
            used[static_cast<size_t>(m.dst)] = 2;
        }
    }
    return EPARA_OK;
}

}  // namespace

int32_t epara_check_copy_call(const epara_page_copy* caches, int32_t G, const epara_page_move* moves, int32_t n_moves, int32_t* n_chunks)
{
    *n_chunks = 0;
    if (G < 0 || n_moves < 0) return EPARA_ERR_SHAPE;
    if (G == 0) return EPARA_OK;
    if (!caches || (n_moves > 0 && !moves)) return EPARA_ERR_NULL;
    int64_t chunks = 0;
    try {
        std::vector<char> used;
        std::vector<int32_t> order;                              // caches with moves
        for (int32_t g = 0; g < G; ++g) {
            const epara_page_copy& c = caches[g];
            if (bad_heads(c.kv_heads, c.kv_heads, c.head_dim, c.n_pages) || c.first_move < 0 || c.n_moves < 0 || static_cast<int64_t>(c.first_move) + c.n_moves > n_moves) return EPARA_ERR_SHAPE;
            if (c.first_chunk != chunks) return EPARA_ERR_SHAPE;
            chunks += static_cast<int64_t>(c.n_moves) * c.kv_heads;
            if (chunks > INT32_MAX / 256) return EPARA_ERR_CAPACITY;
            if (c.n_moves == 0) continue;
            if (!c.codes || !c.scales) return EPARA_ERR_NULL;
            if (misaligned(c.codes, 16) || misaligned(c.scales, 4)) return EPARA_ERR_ALIGN;
            order.push_back(g);
            // the layers of a service follow each other with the same moves and as many pages: looked at once
            if (g > 0 && caches[g - 1].first_move == c.first_move && caches[g - 1].n_moves == c.n_moves && caches[g - 1].n_pages == c.n_pages) continue;
            if (const int32_t rc = check_moves(caches, &g, 1, moves, used)) return rc;
        }
        // entries of the same cache are looked at together
        std::sort(order.begin(), order.end(), [caches](int32_t a, int32_t b) { return std::less<const void*>()(caches[a].codes, caches[b].codes); });
        for (size_t at = 0, end; at < order.size(); at = end) {
            for (end = at + 1; end < order.size() && caches[order[end]].codes == caches[order[at]].codes;) ++end;
            if (end == at + 1) continue;
            if (const int32_t rc = check_moves(caches, &order[at], static_cast<int32_t>(end - at), moves, used)) return rc;
        }
    } catch (const std::bad_alloc&) {
        return EPARA_ERR_CAPACITY;
    }
    *n_chunks = static_cast<int32_t>(chunks);
    return EPARA_OK;
}

extern "C" {

int32_t epara_plan_cache_append(const epara_append_args* h_args, int32_t G, const epara_sequence_table* table, int32_t* first)
{
    if (const int32_t rc = check_append(h_args, G, table)) return rc;
    if (!first) return EPARA_ERR_NULL;
    return count_append(h_args, table, first, nullptr);
}

int32_t epara_plan_cache_attention(const epara_cache_attn_args* h_args, int32_t G, const epara_sequence_table* table, int32_t n_compute_units,
                                   int32_t* first, epara_cache_attn_plan* plan)
{
    if (const int32_t rc = check_attn(h_args, G, table)) return rc;
    if (!first || !plan) return EPARA_ERR_NULL;
    if (n_compute_units < 1 || n_compute_units > 65536) return EPARA_ERR_SHAPE;
    int64_t work[2] = {0, 0}, longest[2] = {0, 0};
    for (int32_t i = 0; i < table->n_seqs; ++i) {
        const epara_sequence& s = table->h_seqs[i];
        const epara_cache_attn_args& a = h_args[s.service];
        if (s.rows == 0) continue;
        const seq_tiles w = tiles_of(a, s);
        const int k = w.few ? 0 : 1;
        for (int tile = 0; tile < w.tiles; ++tile) {
            const page_range r = pages_of_tile(a, s, w.few, tile);
            work[k] += static_cast<int64_t>(r.hi - r.lo) * a.kv_heads;
            longest[k] = std::max<int64_t>(longest[k], r.hi - r.lo);
        }
    }
    epara_attn_part_pages(work, longest, n_compute_units, plan->part_pages);
    bool cut[2];
    if (const int32_t rc = count_attn(h_args, table, plan->part_pages, first, nullptr, plan->n_items, cut)) return rc;
    plan->workspace_bytes = attn_workspace(plan->n_items, cut);
    return EPARA_OK;
}

int32_t epara_page_pool_init(epara_page_pool* pool, int32_t* refs, int32_t* free_pages, int32_t n_pages)
{
    if (n_pages < 0) return EPARA_ERR_SHAPE;
    if (!pool || (n_pages > 0 && (!refs || !free_pages))) return EPARA_ERR_NULL;
    *pool = {refs, free_pages, n_pages, n_pages};
    for (int32_t i = 0; i < n_pages; ++i) {
        refs[i] = 0;
        free_pages[i] = n_pages - 1 - i;
    }
    return EPARA_OK;
}

int32_t epara_pages_take(epara_page_pool* pool, int32_t n, int32_t* pages)
{
    if (!pool || (n > 0 && !pages)) return EPARA_ERR_NULL;
    if (n < 0) return EPARA_ERR_SHAPE;
    if (n > pool->n_free) return EPARA_ERR_CAPACITY;
    for (int32_t i = 0; i < n; ++i) {
        pages[i] = pool->free_pages[--pool->n_free];
        pool->refs[pages[i]] = 1;
    }
    return EPARA_OK;
}

int32_t epara_pages_fork(epara_page_pool* pool, const int32_t* pages, int32_t tokens, int32_t* child, epara_page_move* move, int32_t* n_moves)
{
    if (!pool || !n_moves) return EPARA_ERR_NULL;
    *n_moves = 0;
    if (tokens < 0) return EPARA_ERR_SHAPE;
    const int32_t n = static_cast<int32_t>(ceil_div(tokens, PAGE)), whole = tokens / PAGE;
    if (n > 0 && (!pages || !child)) return EPARA_ERR_NULL;
    if (n > whole && !move) return EPARA_ERR_NULL;
    for (int32_t i = 0; i < n; ++i) {
        if (pages[i] == -1 && i < whole) continue;
        if (pages[i] < 0 || pages[i] >= pool->n_pages || pool->refs[pages[i]] < 1 || pool->refs[pages[i]] == INT32_MAX) return EPARA_ERR_SHAPE;
    }
    if (n > whole && pool->n_free < 1) return EPARA_ERR_CAPACITY;
    for (int32_t i = 0; i < whole; ++i) {
        child[i] = pages[i];
        if (pages[i] != -1) ++pool->refs[pages[i]];
    }
    if (n > whole) {
        const int32_t src = pages[whole];
        const int32_t rc = epara_pages_take(pool, 1, child + whole);
        if (rc) return rc;
        *move = {src, child[whole]};
        *n_moves = 1;
    }
    return EPARA_OK;
}

int32_t epara_pages_free(epara_page_pool* pool, const int32_t* pages, int32_t n)
{
    if (!pool || (n > 0 && !pages)) return EPARA_ERR_NULL;
    if (n < 0) return EPARA_ERR_SHAPE;
    for (int32_t i = 0; i < n; ++i) {
        const int32_t p = pages[i];
        if (p == -1) continue;
        if (p >= 0 && p < pool->n_pages && pool->refs[p] > 0) {
            if (--pool->refs[p] == 0) pool->free_pages[pool->n_free++] = p;
            continue;
        }
        while (i-- > 0) {                                        // what was given back is taken again, in reverse
            const int32_t back = pages[i];
            if (back == -1) continue;
            if (pool->refs[back]++ == 0) --pool->n_free;
        }
        return EPARA_ERR_SHAPE;
    }
    return EPARA_OK;
}

int32_t epara_pages_compact(epara_page_pool* pool, int32_t* table, int32_t n_table, epara_page_move* moves, int32_t cap, int32_t* n_moves)
{
    if (!pool || !n_moves || (n_table > 0 && !table) || (cap > 0 && !moves)) return EPARA_ERR_NULL;
    *n_moves = 0;
    if (n_table < 0 || cap < 0) return EPARA_ERR_SHAPE;
    for (int32_t i = 0; i < n_table; ++i)
        if (table[i] != -1 && (table[i] < 0 || table[i] >= pool->n_pages || pool->refs[table[i]] < 1)) return EPARA_ERR_SHAPE;
    const int32_t used = pool->n_pages - pool->n_free;
    int32_t n = 0, below = 0;
    for (int32_t p = 0; p < pool->n_pages; ++p) (p < used ? below : n) += pool->refs[p] > 0;
    if (below + n != used) return EPARA_ERR_SHAPE;               // not what init, take, fork and free leave
    *n_moves = n;
    if (n > cap) return EPARA_ERR_CAPACITY;
    // the i-th free page below `used` takes the i-th page in use at or above it; the table then finds its page's move by its rank
    int32_t to = 0, at = 0;
    for (int32_t p = used; p < pool->n_pages; ++p) {
        if (pool->refs[p] <= 0) continue;
        while (pool->refs[to] > 0) ++to;
        moves[at++] = {p, to++};
    }
    for (int32_t i = 0; i < n_table; ++i) {
        if (table[i] < used) continue;
        const epara_page_move* m = std::lower_bound(moves, moves + n, table[i], [](const epara_page_move& x, int32_t page) { return x.src < page; });
        table[i] = m->dst;
    }
    for (int32_t i = 0; i < n; ++i) {
        pool->refs[moves[i].dst] = pool->refs[moves[i].src];
        pool->refs[moves[i].src] = 0;
    }
    for (int32_t i = 0; i < pool->n_free; ++i) pool->free_pages[i] = pool->n_pages - 1 - i;
    return EPARA_OK;
}

}  // extern "C"
