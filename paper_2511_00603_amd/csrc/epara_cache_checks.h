// Checks that the calls on sequences share, on the host copies of their arguments.
#ifndef EPARA_CACHE_CHECKS_H
#define EPARA_CACHE_CHECKS_H

#include <stdint.h>

#include <algorithm>
#include <new>
#include <vector>

#include "epara.h"
#include "epara_cache.h"

namespace {

using epara_cache::PAGE;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

inline bool bad_heads(int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t n_pages)
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
inline bool pages_inside(const epara_sequence_table* t, const epara_sequence& s, int lo, int hi, int32_t n_pages)
{
    for (int p = lo; p < hi; ++p) {
        const int32_t id = t->h_pages[s.first_page + p];
        if (id < 0 || id >= n_pages) return false;
    }
    return true;
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

}  // namespace

#endif
