// libepara: trees of drafted tokens: who follows whom, and closing up the tokens that stay in a paged cache.
//
// Both are bound by latency: a tree is 12 KiB at most, and what stays of one are a few tokens of each head.  Trees of 205 sequences with 33 to 256 rows 4.7 us, of one 4.1, a launch and three
// trips to memory.  Keeping: one request in 32 layers of 8 heads 4.6 us, 40 requests in 16 layers 18.4 us: 5120 waves of some ten dependent trips each, four to a SIMD at 126 registers.
// (A value is a byte of each of a head's dims, so a token that moves costs a read and a write of its 16 tokens' chunks.)
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"
#include "epara_cache_device.h"
#include "epara_drafts.h"

using namespace epara_cache;

namespace {

constexpr int NT = 256;
constexpr int CONTEXT = -1, NOWHERE = -2;

// ---- a workgroup per sequence, a thread per row.  Paths double: after k rounds a row knows 2^k rows of its way up, and the row that its way goes on from.
__global__ __launch_bounds__(NT) void draft_trees_kernel(const epara_tree_args* __restrict__ args, const epara_sequence* __restrict__ seqs)
{
    __shared__ uint64_t bits[TREE_ROWS][TREE_WORDS];
    __shared__ int next[TREE_ROWS];
    const epara_sequence s = seqs[blockIdx.x];
    const epara_tree_args a = args[s.service];
    const int tid = threadIdx.x;
    EPARA_GLOBAL int32_t* positions = (EPARA_GLOBAL int32_t*)a.positions;
    auto put_position = [&](int row, int at) {
#pragma unroll
        for (int i = 0; i < 3; ++i) positions[(static_cast<size_t>(s.first_row) + row) * 3 + i] = at;
    };
    if (s.rows > TREE_ROWS) {
        if (positions)
            for (int row = tid; row < s.rows; row += NT) put_position(row, s.start + row);
        return;
    }
    int up = NOWHERE;
    if (tid < s.rows) {
        const int p = ((const EPARA_GLOBAL int32_t*)a.parents)[static_cast<size_t>(s.first_row) + tid];
        up = p == CONTEXT || (p >= 0 && p < tid) ? p : NOWHERE;
    }
    uint64_t mine[TREE_WORDS];
#pragma unroll
    for (int i = 0; i < TREE_WORDS; ++i) mine[i] = i == tid >> 6 ? 1ull << (tid & 63) : 0ull;
    while (true) {
        next[tid] = up;
#pragma unroll
        for (int i = 0; i < TREE_WORDS; ++i) bits[tid][i] = mine[i];
        if (!__syncthreads_or(up >= 0)) break;
        if (up >= 0) {
#pragma unroll
            for (int i = 0; i < TREE_WORDS; ++i) mine[i] |= bits[up][i];
            up = next[up];
        }
        __syncthreads();
    }
    if (tid >= s.rows) return;
    int n = 0;
#pragma unroll
    for (int i = 0; i < TREE_WORDS; ++i) {
        if (up == NOWHERE) mine[i] = 0;
        n += __builtin_popcountll(mine[i]);
    }
    EPARA_GLOBAL uint64_t* dst = (EPARA_GLOBAL uint64_t*)a.visible + (static_cast<size_t>(s.first_row) + tid) * TREE_WORDS;
#pragma unroll
    for (int i = 0; i < TREE_WORDS; ++i) dst[i] = mine[i];
    if (positions) put_position(tid, s.start + max_of(n - 1, 0));
}

// ---- keeping: a wave per cache, sequence and head

// Codes times 2^shift (shift <= 0), rounded again; as they are where there is no shift.  A NaN's code stays (the conversions would change its sign).
__device__ __forceinline__ int rescaled(int codes, int shift)
{
    if (shift == 0) return codes;
    const float f = __builtin_amdgcn_exp2f(static_cast<float>(shift));
    const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    const uint32_t nan = (((static_cast<uint32_t>(codes) & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xffu;
    return static_cast<int>((to_e4m3(a[0] * f, a[1] * f, b[0] * f, b[1] * f) & ~nan) | (static_cast<uint32_t>(codes) & nan));
}

// A sequence's part of a cache, for one head.
struct head_pages {
    char* codes;
    uint8_t* scales;
    const int32_t* pages;        // of the sequence
    int kv_heads, head;
    size_t bytes;                // of a page and head
    __device__ __forceinline__ EPARA_GLOBAL char* keys(int page) const { return (EPARA_GLOBAL char*)codes + (static_cast<size_t>(page) * kv_heads + head) * bytes; }
    __device__ __forceinline__ EPARA_GLOBAL uint8_t* scale(int page) const { return (EPARA_GLOBAL uint8_t*)scales + (static_cast<size_t>(page) * kv_heads + head) * 4; }
    __device__ __forceinline__ int page_of(int slot) const { return ((const EPARA_GLOBAL int32_t*)pages)[slot / PAGE]; }
};

// One block of 32 tokens: its tokens [lo, hi) come from the slots start + path[..] (all at or behind their own), those before lo are earlier ones.
// Lane t (and t + 32) knows token t.  All keys are read before any is written, and all values; nothing that a later block reads lies in this one.
template <int D>
__device__ __forceinline__ void keep_block(const head_pages& c, int block, int lo, int hi, int src, int lane)
{
    constexpr int CD = D / 16, PASSES = BLOCK * CD / 64, DIMS = D / 64;
    const int token = lane & 31, half = block & 1;
    const bool comes = token >= lo && token < hi;
    const int home = c.page_of(block * BLOCK), page = comes ? c.page_of(src) : home, from_half = comes ? src / BLOCK & 1 : half;
    const EPARA_GLOBAL uint8_t* sc = c.scale(page);
    const int was_k = sc[from_half] - 127, was_v = sc[2 + from_half] - 127;          // of where the token lies now
    int e_k = token < hi ? was_k : -1000, e_v = token < hi ? was_v : -1000;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        e_k = max_of(e_k, __shfl_xor(e_k, d));
        e_v = max_of(e_v, __shfl_xor(e_v, d));
    }
    // ---- keys: a lane takes pieces of 16 dims of a token
    v4i key[PASSES];
    int key_shift[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int piece = p * 64 + lane, t = piece / CD, chunk = piece % CD;
        const int from = __shfl(comes ? src : block * BLOCK + token, t), at = from & (PAGE - 1), in = __shfl(page, t);
        key_shift[p] = __shfl(was_k, t) - e_k;
        key[p] = v4i{0, 0, 0, 0};
        if (t < hi && (t >= lo || key_shift[p] != 0)) key[p] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(c.keys(in) + ((((at / 4) % 4) * CD + chunk) * 16 + 4 * (at / 16) + at % 4) * 16);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int piece = p * 64 + lane, t = piece / CD, chunk = piece % CD, at = half * BLOCK + t;
        if (t >= hi || (t < lo && key_shift[p] == 0)) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) key[p][j] = rescaled(key[p][j], key_shift[p]);
        *reinterpret_cast<EPARA_GLOBAL v4i*>(c.keys(home) + ((((at / 4) % 4) * CD + chunk) * 16 + 4 * (at / 16) + at % 4) * 16) = key[p];
    }
    // ---- values: a lane takes whole dims.  What the block holds, and the tokens that come, byte by byte: four at a time, whether all are wanted or not
    const int own_shift = lo > 0 ? __builtin_amdgcn_readfirstlane(was_v) - e_v : 0;          // token 0 is an earlier one then
    auto touched = [&](int q) { return hi > 16 * q && (lo < 16 * q + 16 || own_shift < 0); };
    v4i value[DIMS][2];
    EPARA_GLOBAL char* value_at[DIMS][2];
#pragma unroll
    for (int d = 0; d < DIMS; ++d)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int dim = lane + 64 * d;
            value_at[d][q] = c.keys(home) + PAGE * D + ((dim / 16 * 4 + 2 * half + q) * 16 + dim % 16) * 16;
            value[d][q] = v4i{0, 0, 0, 0};
            if (touched(q)) value[d][q] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(value_at[d][q]);
        }
    if (own_shift < 0) {                         // earlier tokens of a block that grows
#pragma unroll
        for (int d = 0; d < DIMS; ++d)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int mask = low_bytes(lo - 16 * q - 4 * j);
                    value[d][q][j] = (rescaled(value[d][q][j], own_shift) & mask) | (value[d][q][j] & ~mask);
                }
    }
    const int slot = comes ? src : block * BLOCK + token;
#pragma unroll
    for (int t0 = 0; t0 < BLOCK; t0 += 4) {
        if (t0 + 4 <= lo || t0 >= hi) continue;
        int byte[4][DIMS];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int at = __builtin_amdgcn_readlane(slot, t0 + t) & (PAGE - 1), in = __builtin_amdgcn_readlane(page, t0 + t);
#pragma unroll
            for (int d = 0; d < DIMS; ++d) {
                const int dim = lane + 64 * d;
                byte[t][d] = *reinterpret_cast<const EPARA_GLOBAL uint8_t*>(c.keys(in) + PAGE * D + ((dim / 16 * 4 + at / 16) * 16 + dim % 16) * 16 + at % 16);
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t0 + t < lo || t0 + t >= hi) continue;
            const int shift = __builtin_amdgcn_readlane(was_v, t0 + t) - e_v;
#pragma unroll
            for (int d = 0; d < DIMS; ++d) {
                const int others = value[d][t0 / 16][t0 % 16 / 4] & ~(0xff << 8 * t);
                value[d][t0 / 16][t0 % 16 / 4] = others | (rescaled(byte[t][d], shift) & 0xff) << 8 * t;
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int d = 0; d < DIMS; ++d)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (touched(q)) *reinterpret_cast<EPARA_GLOBAL v4i*>(value_at[d][q]) = value[d][q];
    if (lane == 0) {
        c.scale(home)[half] = static_cast<uint8_t>(e_k + 127);
        c.scale(home)[2 + half] = static_cast<uint8_t>(e_v + 127);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

__global__ __launch_bounds__(NT, 4) void cache_keep_kernel(const epara_keep_args* __restrict__ caches, int n_caches, const epara_sequence* __restrict__ seqs,
                                                       const int32_t* __restrict__ pages, const int32_t* __restrict__ kept, int n_items)
{
    const int lane = threadIdx.x & 63, item = blockIdx.x * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= n_items) return;
    int g = 0, n = n_caches;                               // the last cache whose first_item is <= item
    while (n > 1) {
        const int step = (n + 63) >> 6, at = lane * step;
        const int sum = at < n ? caches[g + at].first_item : 0x7fffffff;
        const int before = (__builtin_popcountll(__ballot(sum <= item)) - 1) * step;
        g += before;
        n = n - before < step ? n - before : step;
    }
    const epara_keep_args a = caches[__builtin_amdgcn_readfirstlane(g)];
    const int local = item - a.first_item, i = a.first_seq + local / a.kv_heads;
    const epara_sequence s = seqs[i];
    if (s.rows > TREE_ROWS) return;
    // ---- the path: four rows of it to a lane's word, 64 rows to a word
    int row[TREE_WORDS], last = -1, count = max_of(0, min_of(kept[i], s.rows)), still = 0;       // still: rows at the path's beginning that stay where they are
    bool rising = true, same = true;
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) {
        const int at = 64 * w + lane;
        row[w] = at < count ? ((const EPARA_GLOBAL int32_t*)a.path)[static_cast<size_t>(s.first_row) + at] : -1;
    }
    int good = 0;
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) {
        int before = __shfl_up(row[w], 1);
        if (lane == 0) before = last;
        last = __builtin_amdgcn_readlane(row[w], 63);
        const uint64_t up = __ballot(64 * w + lane < count && row[w] > before && row[w] >= 0 && row[w] < s.rows);
        const uint64_t stay = __ballot(row[w] == 64 * w + lane);
        const int n_up = ~up ? __builtin_ctzll(~up) : 64, n_stay = ~stay ? __builtin_ctzll(~stay) : 64;
        if (rising) good += n_up;
        if (same) still += n_stay;
        rising = rising && n_up == 64;
        same = same && n_stay == 64;
    }
    count = good;
    if (still >= count) return;
    const head_pages c = {static_cast<char*>(a.codes), a.scales, pages + s.first_page, a.kv_heads, local - local / a.kv_heads * a.kv_heads, static_cast<size_t>(head_bytes(a.head_dim))};
    for (int block = (s.start + still) / BLOCK; block <= (s.start + count - 1) / BLOCK; ++block) {
        const int first = block * BLOCK, lo = max_of(s.start - first, 0), hi = min_of(s.start + count - first, BLOCK);
        const int at = first + (lane & 31) - s.start;      // my token's place in the path
        int src = 0;
#pragma unroll
        for (int w = 0; w < TREE_WORDS; ++w) {
            const int r = __shfl(row[w], at & 63);
            if (at >> 6 == w) src = s.start + r;
        }
        if (a.head_dim == 128) keep_block<128>(c, block, lo, hi, src, lane);
        else                   keep_block<64>(c, block, lo, hi, src, lane);
    }
}

}  // namespace

extern "C" {

int32_t epara_draft_trees(const epara_tree_args* h_args, const epara_tree_args* d_args, int32_t G, const epara_sequence_table* table, void* stream)
{
    if (const int32_t rc = epara_check_trees_call(h_args, G, table)) return rc;
    if (table->n_seqs == 0) return EPARA_OK;
    if (!d_args) return EPARA_ERR_NULL;
    hipLaunchKernelGGL(draft_trees_kernel, dim3(static_cast<unsigned>(table->n_seqs)), dim3(NT), 0, static_cast<hipStream_t>(stream), d_args, table->d_seqs);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}

int32_t epara_cache_keep(const epara_keep_args* h_caches, const epara_keep_args* d_caches, int32_t n_caches, const epara_sequence_table* table,
                         const int32_t* d_kept, void* stream)
{
    int32_t n_items;
    if (const int32_t rc = epara_check_keep_call(h_caches, n_caches, table, &n_items)) return rc;
    if (n_items == 0) return EPARA_OK;
    if (!d_caches || !d_kept) return EPARA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(d_kept) & 3) return EPARA_ERR_ALIGN;
    hipLaunchKernelGGL(cache_keep_kernel, dim3(static_cast<unsigned>((n_items + NT / 64 - 1) / (NT / 64))), dim3(NT), 0, static_cast<hipStream_t>(stream),
                       d_caches, n_caches, table->d_seqs, table->d_pages, d_kept, n_items);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}

}  // extern "C"
