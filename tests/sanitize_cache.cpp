// Seeded calls of the cache's host code, good and bad, for a build under the sanitizers.
#include <cstdio>
#include <cstdlib>
#include <algorithm>
#include <random>
#include <vector>

#include "epara.h"
#include "epara_cache_host.h"

static int failures = 0;
#define WANT(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); ++failures; } } while (0)

int main()
{
    std::mt19937 rng(603);
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    char* const d = reinterpret_cast<char*>(0x7000000);          // never dereferenced
    for (int round = 0; round < 300; ++round) {
        const int n_pages = pick(1, 200), n = pick(0, 20), group = pick(1, 8), kv = pick(1, 5), dim = pick(0, 1) ? 64 : 128;
        std::vector<epara_sequence> seqs;
        std::vector<int32_t> table;
        std::vector<int32_t> ids(n_pages);
        for (int i = 0; i < n_pages; ++i) ids[i] = i;
        std::shuffle(ids.begin(), ids.end(), rng);
        int rows = 0;
        for (int i = 0; i < n; ++i) {
            const int r = pick(0, 3) ? pick(0, 3) : pick(0, 200), start = pick(-5, 300), need = start + r > 0 ? (start + r + 63) / 64 : 0;
            if (static_cast<int>(table.size()) + need > n_pages) break;
            seqs.push_back({0, rows, r, start, static_cast<int32_t>(table.size()), need});
            for (int p = 0; p < need; ++p) table.push_back(ids[table.size()]);
            rows += r;
        }
        epara_sequence_table t = {seqs.data(), seqs.data(), table.data(), table.data(), static_cast<int32_t>(seqs.size()), static_cast<int32_t>(table.size())};
        epara_append_args a = {d, d + 0x1000, d + 0x2000, reinterpret_cast<uint8_t*>(d + 0x3000), reinterpret_cast<float*>(d + 0x4000), nullptr, rows, group * kv, kv, dim, n_pages,
                               (group + 2) * kv * dim, group * kv * dim, 1000, {dim / 4, dim / 8}};
        std::vector<int32_t> first(seqs.size() + 1), attn_first(2 * (seqs.size() + 1));
        WANT(epara_plan_cache_append(&a, 1, &t, first.data()) == EPARA_OK);
        WANT(epara_check_append_call(&a, 1, &t, first.data()) == EPARA_OK);
        epara_cache_attn_args q = {d, d + 0x1000, d, reinterpret_cast<uint8_t*>(d), rows, group * kv, kv, dim, n_pages, group * kv * dim, group * kv * dim, pick(0, 1) * pick(1, 300), 0.1f, 0.f, {0, 0}};
        epara_cache_attn_plan plan = {};
        WANT(epara_plan_cache_attention(&q, 1, &t, pick(1, 300), attn_first.data(), &plan) == EPARA_OK);
        epara_cache_attn_launch l = {&q, &q, attn_first.data(), attn_first.data(), reinterpret_cast<void*>(0x8000000), plan.workspace_bytes, t, plan, 1, 0};
        bool cut[2];
        WANT(epara_check_attn_call(l, cut) == EPARA_OK);
        if (!seqs.empty()) {                                     // anything in a record: an error or not, never a read outside
            for (int k = 0; k < 20; ++k) {
                std::vector<epara_sequence> wild = seqs;
                int32_t* field = reinterpret_cast<int32_t*>(&wild[pick(0, static_cast<int>(wild.size()) - 1)]) + pick(0, 5);
                *field = pick(0, 1) ? pick(-100, 500) : static_cast<int32_t>(rng());
                epara_sequence_table w = t;
                w.h_seqs = wild.data();
                (void)epara_plan_cache_append(&a, 1, &w, first.data());
                (void)epara_plan_cache_attention(&q, 1, &w, 256, attn_first.data(), &plan);
            }
        }
        // pages
        std::vector<int32_t> refs(n_pages), free_pages(n_pages), own, child(300);
        epara_page_pool pool;
        WANT(epara_page_pool_init(&pool, refs.data(), free_pages.data(), n_pages) == EPARA_OK);
        const int take = pick(0, n_pages);
        own.resize(take + 1);
        WANT(epara_pages_take(&pool, take, own.data()) == EPARA_OK);
        own.resize(take);
        epara_page_move mv;
        int32_t moves = 0;
        const int tokens = pick(0, take * 64);
        const int rc = epara_pages_fork(&pool, own.data(), tokens, child.data(), &mv, &moves);
        WANT(rc == EPARA_OK || (rc == EPARA_ERR_CAPACITY && pool.n_free == 0));
        WANT(epara_pages_free(&pool, own.data(), take) == EPARA_OK);
        if (rc == EPARA_OK) {
            const int held = (tokens + 63) / 64;
            std::vector<epara_page_move> list(n_pages);
            WANT(epara_pages_compact(&pool, child.data(), held, list.data(), n_pages, &moves) == EPARA_OK);
            for (int i = 0; i < held; ++i) WANT(child[i] < held);
            WANT(epara_pages_free(&pool, child.data(), held) == EPARA_OK);
        }
        WANT(pool.n_free == n_pages);
        // copies
        std::vector<epara_page_move> list;
        for (int i = 0; i + 1 < n_pages && i < 20; i += 2) list.push_back({ids[i], ids[i + 1]});
        epara_page_copy c = {d, reinterpret_cast<uint8_t*>(d), n_pages, kv, dim, 0, static_cast<int32_t>(list.size()), 0};
        int32_t chunks;
        WANT(epara_check_copy_call(&c, 1, list.data(), static_cast<int32_t>(list.size()), &chunks) == EPARA_OK && chunks == static_cast<int32_t>(list.size()) * kv);
        if (list.size() > 1) {
            list[0].dst = list[1].src;
            WANT(epara_check_copy_call(&c, 1, list.data(), static_cast<int32_t>(list.size()), &chunks) == EPARA_ERR_SHAPE);
        }
    }
    if (!failures) std::printf("sanitize_cache: ok\n");
    return failures != 0;
}
