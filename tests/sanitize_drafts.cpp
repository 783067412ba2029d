// Seeded calls of the host code of decoding by drafts, good and bad, for a build under the sanitizers.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "epara.h"
#include "epara_drafts.h"

static int failures = 0;
#define WANT(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); ++failures; } } while (0)

int main()
{
    std::mt19937 rng(604);
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    char* const d = reinterpret_cast<char*>(0x7000000);          // never dereferenced
    for (int round = 0; round < 300; ++round) {
        const int n = pick(0, 12), group = pick(1, 8), kv = pick(1, 5), dim = pick(0, 1) ? 64 : 128;
        std::vector<epara_sequence> seqs;
        std::vector<int32_t> table;
        int rows = 0;
        for (int i = 0; i < n; ++i) {
            const int r = pick(0, 3) ? pick(0, 40) : pick(0, 256), start = pick(0, 900), need = (start + r + 63) / 64;
            seqs.push_back({0, rows, r, start, static_cast<int32_t>(table.size()), need});
            for (int p = 0; p < need; ++p) table.push_back(static_cast<int32_t>(table.size()));
            rows += r;
        }
        const int n_pages = static_cast<int>(table.size()) + 1, n_seqs = static_cast<int>(seqs.size());
        epara_sequence_table t = {seqs.data(), seqs.data(), table.data(), table.data(), n_seqs, static_cast<int32_t>(table.size())};
        int32_t* const ints = reinterpret_cast<int32_t*>(d);
        epara_tree_args tree = {ints, reinterpret_cast<uint64_t*>(d), ints, rows, 0};
        WANT(epara_check_trees_call(&tree, 1, &t) == EPARA_OK);
        epara_cache_attn_args q = {d, d + 0x1000, d, reinterpret_cast<uint8_t*>(d), rows, group * kv, kv, dim, n_pages, group * kv * dim, group * kv * dim, pick(0, 1) * pick(256, 600), 0.1f, 0.f, {0, 0}};
        std::vector<int32_t> first(3 * (n_seqs + 1));
        epara_tree_attn_plan plan = {};
        WANT(epara_plan_tree_attention(&q, &tree, 1, &t, pick(1, 300), first.data(), &plan) == EPARA_OK);
        epara_tree_attn_launch l = {&q, &q, &tree, &tree, first.data(), first.data(), reinterpret_cast<void*>(0x8000000), plan.workspace_bytes, t, plan, 1, 0};
        bool cut[3];
        WANT(epara_check_tree_attn_call(l, cut) == EPARA_OK);
        const int vocab = pick(1, 200000);
        epara_verify_args v = {d, pick(0, 1) ? d : nullptr, ints, ints, reinterpret_cast<float*>(d), ints, reinterpret_cast<float*>(d), rows, vocab, vocab + pick(0, 9), vocab};
        std::vector<int32_t> vfirst(n_seqs + 1);
        epara_verify_plan vp = {};
        const int dtype = pick(0, 1) ? EPARA_BF16 : EPARA_F32;
        WANT(epara_plan_verify_drafts(&v, 1, &t, dtype, pick(1, 300), vfirst.data(), &vp) == EPARA_OK);
        epara_verify_launch vl = {&v, &v, vfirst.data(), vfirst.data(), nullptr, ints, ints, reinterpret_cast<void*>(0x8000000), vp.workspace_bytes, t, vp, 1, dtype};
        WANT(epara_check_verify_call(vl) == EPARA_OK);
        epara_keep_args keep = {d, reinterpret_cast<uint8_t*>(d), ints, 0, 0, rows, n_pages, kv, dim, 0, 0};
        int32_t items;
        WANT(epara_check_keep_call(&keep, 1, &t, &items) == EPARA_OK && items == n_seqs * kv);
        for (int k = 0; k < 20 && n_seqs; ++k) {                 // anything in a record: an error or not, never a read outside
            std::vector<epara_sequence> wild = seqs;
            int32_t* field = reinterpret_cast<int32_t*>(&wild[pick(0, n_seqs - 1)]) + pick(0, 5);
            *field = pick(0, 1) ? pick(-100, 500) : static_cast<int32_t>(rng());
            epara_sequence_table w = t;
            w.h_seqs = wild.data();
            (void)epara_check_trees_call(&tree, 1, &w);
            (void)epara_plan_tree_attention(&q, &tree, 1, &w, 256, first.data(), &plan);
            (void)epara_plan_verify_drafts(&v, 1, &w, dtype, 256, vfirst.data(), &vp);
            (void)epara_check_keep_call(&keep, 1, &w, &items);
        }
    }
    if (!failures) std::printf("sanitize_drafts: ok\n");
    return failures != 0;
}
