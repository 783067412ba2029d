// libepara: trees of drafted tokens: who follows whom, and closing up the tokens that stay in a paged cache.
//
// Both are bound by latency: a tree is 12 KiB at most, and what stays of one are a few tokens of each head.  Trees of 205 sequences with 33 to 256 rows 4.7 us, of one 4.1, a launch and three
// trips to memory.  Keeping: one request in 32 layers of 8 heads 4.6 us, 40 requests in 16 layers 15.4 us: 10240 waves, half of them for keys and half for values, of some nine dependent
// trips each, five to a SIMD at 90 registers.  One wave for both was longer and needed 126: 18.4 us.  A form of 106 registers, spilled for more waves: five 16.4, six 21.2,
// eight 29.0.
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

// ---- keeping: two waves per cache, sequence and head, for keys and for values

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
    int page, first;             // lane i has page first + i of the sequence's
    int kv_heads, head;
    size_t bytes;                // of a page and head
    __device__ __forceinline__ EPARA_GLOBAL char* keys(int page) const { return (EPARA_GLOBAL char*)codes + (static_cast<size_t>(page) * kv_heads + head) * bytes; }
    __device__ __forceinline__ EPARA_GLOBAL uint8_t* scale(int page) const { return (EPARA_GLOBAL uint8_t*)scales + (static_cast<size_t>(page) * kv_heads + head) * 4; }
    __device__ __forceinline__ int page_of(int slot) const { return __shfl(page, slot / PAGE - first); }        // (all lanes ask)
};

// A lane takes pieces of 16 dims of a token.
template <int D>
__device__ __forceinline__ void keep_keys(const head_pages& c, int half, int home, int lo, int hi, int from, int page, int was, int e, int lane)
{
    constexpr int CD = D / 16, PASSES = BLOCK * CD / 64;
    v4i key[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int piece = p * 64 + lane, t = piece / CD, chunk = piece % CD;
        const int at = __shfl(from, t) & (PAGE - 1), in = __shfl(page, t);
        const int shift = __shfl(was, t) - e;
        key[p] = v4i{0, 0, 0, 0};
        if (t < hi && (t >= lo || shift != 0)) key[p] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(c.keys(in) + ((((at / 4) % 4) * CD + chunk) * 16 + 4 * (at / 16) + at % 4) * 16);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int piece = p * 64 + lane, t = piece / CD, chunk = piece % CD, at = half * BLOCK + t, shift = __shfl(was, t) - e;
        if (t >= hi || (t < lo && shift == 0)) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) key[p][j] = rescaled(key[p][j], shift);
        *reinterpret_cast<EPARA_GLOBAL v4i*>(c.keys(home) + ((((at / 4) % 4) * CD + chunk) * 16 + 4 * (at / 16) + at % 4) * 16) = key[p];
    }
}
// A lane takes whole dims, 16 tokens of them at a time (they lie together; what comes into the second 16 lies at or behind them).  What is there, and the tokens that come, byte by byte: four at a
// time, whether all are wanted or not.
template <int D>
__device__ __forceinline__ void keep_values(const head_pages& c, int half, int home, int lo, int hi, int from, int page, int was, int e, unsigned lane)
{
    constexpr int DIMS = D / 64;
    const int own_shift = lo > 0 ? __builtin_amdgcn_readfirstlane(was) - e : 0;          // token 0 is an earlier one then
    const unsigned mine = lane / 16 * 1024 + lane % 16 * 16;   // of my first dim, in a page's values
#pragma unroll 1
    for (int q = 0; q < 2; ++q) {
        const int lo_q = lo - 16 * q, hi_q = hi - 16 * q;
        if (hi_q <= 0 || (lo_q >= 16 && own_shift == 0)) continue;
        EPARA_GLOBAL char* dst = c.keys(home) + PAGE * D + (2 * half + q) * 256;
        v4i value[DIMS];
#pragma unroll
        for (int d = 0; d < DIMS; ++d) {
            value[d] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(dst + mine + 4096u * d);
            if (own_shift < 0)                             // earlier tokens of a block that grows
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int mask = low_bytes(lo_q - 4 * j);
                    value[d][j] = (rescaled(value[d][j], own_shift) & mask) | (value[d][j] & ~mask);
                }
        }
#pragma unroll
        for (int t0 = 0; t0 < 16; t0 += 4) {
            if (t0 + 4 <= lo_q || t0 >= hi_q) continue;
            int byte[4][DIMS];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int at = __builtin_amdgcn_readlane(from, 16 * q + t0 + t) & (PAGE - 1), in = __builtin_amdgcn_readlane(page, 16 * q + t0 + t);
                const EPARA_GLOBAL uint8_t* src = reinterpret_cast<const EPARA_GLOBAL uint8_t*>(c.keys(in) + PAGE * D + at / 16 * 256 + at % 16);
#pragma unroll
                for (int d = 0; d < DIMS; ++d) byte[t][d] = src[mine + 4096u * d];
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (t0 + t < lo_q || t0 + t >= hi_q) continue;
                const int shift = __builtin_amdgcn_readlane(was, 16 * q + t0 + t) - e;
#pragma unroll
                for (int d = 0; d < DIMS; ++d) value[d][t0 / 4] = (value[d][t0 / 4] & ~(0xff << 8 * t)) | (rescaled(byte[t][d], shift) & 0xff) << 8 * t;
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int d = 0; d < DIMS; ++d) *reinterpret_cast<EPARA_GLOBAL v4i*>(dst + mine + 4096u * d) = value[d];
    }
}

// One block of 32 tokens: its tokens [lo, hi) come from the slots start + path[..] (all at or behind their own), those before lo are earlier ones.
// Lane t (and t + 32) knows token t.  All keys (of values: 16 tokens') are read before any is written; nothing that a later block reads lies in this one.
template <int D, bool KEYS>
__device__ __forceinline__ void keep_block(const head_pages& c, int block, int lo, int hi, int src, int lane)
{
    const int token = lane & 31, half = block & 1;
    const int from = token >= lo && token < hi ? src : block * BLOCK + token;       // the slot
    const int home = __builtin_amdgcn_readfirstlane(c.page_of(block * BLOCK)), page = c.page_of(from);
    constexpr int SCALE = KEYS ? 0 : 2;                    // of a page's scales
    const int was = c.scale(page)[SCALE + (from / BLOCK & 1)] - 127;        // of where the token lies now
    int e = token < hi ? was : -1000;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) e = max_of(e, __shfl_xor(e, d));
    if constexpr (KEYS) keep_keys<D>(c, half, home, lo, hi, from, page, was, e, lane);
    else                keep_values<D>(c, half, home, lo, hi, from, page, was, e, lane);
    if (lane == 0) c.scale(home)[SCALE + half] = static_cast<uint8_t>(e + 127);
}

// Path rows still .. count - 1.
template <int D, bool KEYS>
__device__ __forceinline__ void keep_blocks(const head_pages& c, const epara_sequence& s, int still, int count, const int (&row)[TREE_WORDS], int lane)
{
#pragma unroll 1
    for (int block = (s.start + still) / BLOCK; block <= (s.start + count - 1) / BLOCK; ++block) {
        const int first = block * BLOCK, lo = max_of(s.start - first, 0), hi = min_of(s.start + count - first, BLOCK);
        const int at = first + (lane & 31) - s.start;      // my token's place in the path
        int src = 0;
#pragma unroll
        for (int w = 0; w < TREE_WORDS; ++w) {
            const int r = __shfl(row[w], at & 63);
            if (at >> 6 == w) src = s.start + r;
        }
        keep_block<D, KEYS>(c, block, lo, hi, src, lane);
    }
}

__global__ __launch_bounds__(NT, 5) void cache_keep_kernel(const epara_keep_args* __restrict__ caches, int n_caches, const epara_sequence* __restrict__ seqs,
                                                       const int32_t* __restrict__ pages, const int32_t* __restrict__ kept, int n_items)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = blockIdx.x * (NT / 128) + (wave >> 1);
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
    const int local = item - a.first_item, nth = __builtin_amdgcn_readfirstlane(local / a.kv_heads), i = a.first_seq + nth;
    const epara_sequence s = seqs[i];
    if (s.rows == 0 || s.rows > TREE_ROWS) return;
    // ---- the pages from token `start` on: no more than a wave has lanes.  And the path, 64 rows to a word
    const int first_page = s.start / PAGE, page = ((const EPARA_GLOBAL int32_t*)pages)[static_cast<size_t>(s.first_page) + min_of(first_page + lane, s.n_pages - 1)];
    int row[TREE_WORDS], last = -1, count = max_of(0, min_of(kept[i], s.rows)), still = 0;       // still: rows at the path's beginning that stay where they are
    bool rising = true, same = true;
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) {
        const int at = 64 * w + lane;
        row[w] = at < s.rows ? ((const EPARA_GLOBAL int32_t*)a.path)[static_cast<size_t>(s.first_row) + at] : -1;      // (before `kept` has come)
    }
    int good = 0;
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) {
        if (64 * w + lane >= count) row[w] = -1;
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
    const head_pages c = {static_cast<char*>(a.codes), a.scales, page, first_page, a.kv_heads, local - nth * a.kv_heads, static_cast<size_t>(head_bytes(a.head_dim))};
    if (a.head_dim == 128) wave & 1 ? keep_blocks<128, false>(c, s, still, count, row, lane) : keep_blocks<128, true>(c, s, still, count, row, lane);
    else                   wave & 1 ? keep_blocks<64, false>(c, s, still, count, row, lane) : keep_blocks<64, true>(c, s, still, count, row, lane);
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
    hipLaunchKernelGGL(cache_keep_kernel, dim3(static_cast<unsigned>((n_items + NT / 128 - 1) / (NT / 128))), dim3(NT), 0, static_cast<hipStream_t>(stream),
                       d_caches, n_caches, table->d_seqs, table->d_pages, d_kept, n_items);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}

}  // extern "C"
