// libepara: which drafted tokens the target agrees to, and the token behind them.
//
// Three kernels.  The first reads all logits once and leaves for each chunk of a row its largest logit and sum exp((x - top) / T).  The second walks each sequence's tree with these
// sums.  The third finds the token behind the last row that stays.  The border between two tokens that a random number falls on may lie anywhere, so that row's weights are summed
// again in 64 bits, a chunk to a workgroup; the last of them finds the chunk and in it the token.
//
// Where the token comes from max(p - q, 0), with weights a and b of p and q relative to their largest, that is max(a - r b, 0) with r = sum a / sum b.  The third kernel would have to
// know r before it sums; it knows r0 from the first, off by some 10^-6.  F(r) = sum max(a - r b, 0) is piecewise linear, so it sums F(r0) and its slope -G = -sum of b where a > r0 b
// next to sum a and sum b, and the last workgroup has r and F(r) = F(r0) - (r - r0) G, wrong only by elements with a / b between r0 and r: (r - r0) times their share
// of q.  Where so little is left that this could matter, the last workgroup sums all chunks once more with r.  Where a and r b agree over a whole chunk, F and its
// correction cancel to their rounding, and a uniform of 0 could fall on a chunk without a token: r is taken 2^-44 larger than it is, which leaves nothing there.
//
// The first kernel is bound by HBM: chains of four drafts of 64 requests at 131072 tokens, with draft logits (0.15 GB), 31 us, 4.9 TB/s, of 65 for the whole call; the second takes 5 to 10 us, a
// chain of dependent trips to memory, and a workgroup to a sequence; the third 31 us there (two rows of 131072 weights in 64 bits to a sequence, at 4 waves to a SIMD) and 6 to 11 elsewhere.
// What was measured on the way: the walk by the last of the first kernel's workgroups instead of a kernel of its own 32 -> 70 us (each of 5760 short workgroups then waits for its store and
// its counter); the walk and the draw in one kernel, walked again by every workgroup, 36 us and more; a third kernel that sums first and a fourth that draws from max(p - q, 0): 26 + 48 us;
// loops over siblings that branch at each 14 us; scans through the LDS' shuffles and searches by atomics 5 us of the third kernel's 11 at one request.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"
#include "epara_cache_device.h"
#include "epara_drafts.h"

using namespace epara_cache;
using namespace epara_drafts;

namespace {

constexpr int NT = 256, WAVES = NT / 64;
constexpr float LOG2E = 1.4426950408889634f;
constexpr double LOG2E_64 = 1.4426950408889634;
constexpr float BELOW_ONE = 0x1.fffffep-1f;
constexpr double MORE = 1. + 0x1p-44;        // of r: over the rounding of r and of the sums behind it (2^-47 at most), so that nothing is left where a = r b

// Where the parts of a call's workspace are.
struct workspace {
    uint32_t* counters;          // [n_seqs]
    drawn_row* drawn;            // [n_seqs]
    row_sum* rows;               // [n_items]
    chunk_sum* chunks;           // [n_seqs][draw_chunks]
};

// 8 bytes for, or from, workgroups on other dies in the same kernel: past the dies' own caches.
__device__ __forceinline__ void put8(void* at, uint64_t x) { __hip_atomic_store(static_cast<unsigned long long*>(at), static_cast<unsigned long long>(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t get8(const void* at) { return __hip_atomic_load(static_cast<const unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double get_double(const double* at) { return __builtin_bit_cast(double, get8(at)); }

// Whether this thread's workgroup is the last of `n` to come; what the thread has written is there for whoever is.
__device__ __forceinline__ bool is_last(uint32_t* counter, int n)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != static_cast<uint32_t>(n - 1)) return false;
    __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

// 2^t for t <= 0, in 64 bits: a power of two, and the series of 2^f for |f| <= 1 / 2, whose first term that is left out, (ln 2 / 2)^11 / 11!, is under 2^-42.
__device__ __forceinline__ double exp2_64(double t)
{
    t = fmax(t, -1100.);
    const double n = __builtin_rint(t), f = t - n;
    double y = 7.054911620801121e-09;                      // (ln 2)^k / k!, k = 10 .. 0
    y = fma(y, f, 1.01780860092396959e-07);
    y = fma(y, f, 1.32154867901443053e-06);
    y = fma(y, f, 1.52527338040598393e-05);
    y = fma(y, f, 1.5403530393381606e-04);
    y = fma(y, f, 1.33335581464284411e-03);
    y = fma(y, f, 9.61812910762847687e-03);
    y = fma(y, f, 5.55041086648215762e-02);
    y = fma(y, f, 2.40226506959100694e-01);
    y = fma(y, f, 6.93147180559945286e-01);
    y = fma(y, f, 1.);
    return __builtin_ldexp(y, static_cast<int>(n));
}

// ---- a row of logits in pieces of 16 bytes

struct row_view {
    __amdgpu_buffer_rsrc_t rsrc; // from the 16-byte boundary at or before the row to the end of its last word: what lies behind reads as zero
    int skip, vocab;             // elements of the first piece that are not the row's
};
__device__ __forceinline__ const char* row_at(const void* logits, int row, int stride, int size) { return static_cast<const char*>(logits) + static_cast<size_t>(row) * stride * size; }
template <int SIZE>
__device__ __forceinline__ row_view view_of(const void* row, int vocab)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(row), base = at & ~static_cast<uintptr_t>(15);
    const int skip = static_cast<int>(at - base);
    return {__builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, (skip + vocab * SIZE + 3) & ~3, 0x00020000), skip / SIZE, vocab};
}

// The elements of pieces first, first + step, ..; what is not the row's is -infinity.
template <int SIZE, int U, int HINT = 0>
__device__ __forceinline__ void load_pieces(const row_view& v, int first, int step, float* x)
{
    constexpr int PER = 16 / SIZE;
    v4i raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(v.rsrc, (first + u * step) * 16, 0, HINT));
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t w = static_cast<uint32_t>(raw[u][j]);
            if constexpr (SIZE == 4) x[u * PER + j] = __uint_as_float(w);
            else {
                x[u * PER + 2 * j] = bf16_lo(w);
                x[u * PER + 2 * j + 1] = bf16_hi(w);
            }
        }
        const int at = (first + u * step) * PER - v.skip;  // of the piece's first element
        if (at < 0 || at > v.vocab - PER) {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (at + j < 0 || at + j >= v.vocab) x[u * PER + j] = -INFINITY;
        }
    }
}
template <int SIZE>
__device__ __forceinline__ float logit_at(const void* logits, int row, int stride, int at)
{
    const EPARA_GLOBAL char* p = (const EPARA_GLOBAL char*)logits + (static_cast<size_t>(row) * stride + at) * SIZE;
    if constexpr (SIZE == 4) return *reinterpret_cast<const EPARA_GLOBAL float*>(p);
    else return __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const EPARA_GLOBAL uint16_t*>(p)) << 16);
}

struct temperature { bool greedy; float t; };
__device__ __forceinline__ temperature temperature_of(const float* temperatures, int seq)
{
    const float t = temperatures ? temperatures[seq] : 0.f;
    if (!(t > 0.f)) return {true, 1.f};
    return {false, fminf(fmaxf(t, 0x1p-100f), 0x1p100f)};
}

// What is said to be the parent of row `row` of a sequence; the row that it follows, or -1.
__device__ __forceinline__ int parent_word(const epara_verify_args& a, const epara_sequence& s, int row)
{
    return a.parents ? ((const EPARA_GLOBAL int32_t*)a.parents)[static_cast<size_t>(s.first_row) + row] : row - 1;
}
__device__ __forceinline__ int parent_of(const epara_verify_args& a, const epara_sequence& s, int row)
{
    const int p = parent_word(a, s, row);
    return p >= 0 && p < row ? p : -1;
}

__device__ __forceinline__ double shuffle_xor(double x, int d)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, static_cast<uint64_t>(static_cast<uint32_t>(__shfl_xor(static_cast<int>(u), d))) |
                                          static_cast<uint64_t>(static_cast<uint32_t>(__shfl_xor(static_cast<int>(u >> 32), d))) << 32);
}
// A wave's lanes joined by neighbours' registers (rows of 16 lanes, then the ends of rows): a tenth of the time that trips through the LDS take.  Lane i gets the sum of lanes 0 .. i.
template <int CTRL, int ROWS>
__device__ __forceinline__ double from_lane(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, ROWS, 0xf, false));
    const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, ROWS, 0xf, false));
    return __builtin_bit_cast(double, lo | static_cast<uint64_t>(hi) << 32);
}
constexpr int ROW_SHIFT = 0x110, LAST_OF_ROW = 0x142, LAST_OF_HALF = 0x143;
__device__ __forceinline__ double wave_scan(double x)
{
    x += from_lane<ROW_SHIFT + 1, 0xf>(x);
    x += from_lane<ROW_SHIFT + 2, 0xf>(x);
    x += from_lane<ROW_SHIFT + 4, 0xf>(x);
    x += from_lane<ROW_SHIFT + 8, 0xf>(x);
    x += from_lane<LAST_OF_ROW, 0xa>(x);
    x += from_lane<LAST_OF_HALF, 0xc>(x);
    return x;
}
// Of the whole wave, in lane 63.
template <int CTRL, int ROWS>
__device__ __forceinline__ float larger_of(float x)
{
    return fmaxf(x, __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(static_cast<int>(__float_as_uint(x)), static_cast<int>(__float_as_uint(x)), CTRL, ROWS, 0xf, false))));
}
__device__ __forceinline__ float wave_max(float x)
{
    x = larger_of<ROW_SHIFT + 1, 0xf>(x);
    x = larger_of<ROW_SHIFT + 2, 0xf>(x);
    x = larger_of<ROW_SHIFT + 4, 0xf>(x);
    x = larger_of<ROW_SHIFT + 8, 0xf>(x);
    x = larger_of<LAST_OF_ROW, 0xa>(x);
    return larger_of<LAST_OF_HALF, 0xc>(x);
}
__device__ __forceinline__ float last_lane(float x) { return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(x)), 63))); }
__device__ __forceinline__ int wave_min(int x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x = min_of(x, __shfl_xor(x, d));
    return x;
}

// ---- the walk

struct walk_lds {
    float top[2][TREE_ROWS];     // of a row's logits and draft logits
    int place[TREE_ROWS];
    double sum[2][TREE_ROWS];    // NaN or 0: no distribution
    double takes[TREE_ROWS];     // what a row that is turned away takes from its siblings: its token's probability, unless an elder sibling has taken that
    int parent[TREE_ROWS], token[TREE_ROWS];
    int child[TREE_ROWS];        // the one that stays behind a row, if the row does
    int path[TREE_ROWS];
    int kept;
    int eldest, n_without;       // of the row that stays last: its first child, and its children's tokens
};

__device__ __forceinline__ bool has_distribution(double sum) { return sum > 0. && sum < static_cast<double>(INFINITY); }

// The second kernel, a workgroup to a sequence: which rows stay, and what is left to draw.
template <int SIZE>
__global__ __launch_bounds__(NT) void walk_kernel(const epara_verify_args* __restrict__ args, const epara_sequence* __restrict__ seqs, const int32_t* __restrict__ first,
                                                 const float* __restrict__ temperatures, const row_sum* __restrict__ all_sums, drawn_row* __restrict__ draws, int pieces,
                                                 int32_t* __restrict__ kept, int32_t* __restrict__ next)
{
    __shared__ walk_lds lds;
    const int tid = threadIdx.x, i = blockIdx.x;
    const epara_sequence s = seqs[i];
    const row_sum* __restrict__ sums = all_sums + first[i];
    const temperature temp = temperature_of(temperatures, i);
    drawn_row* draw = draws + i;
    if (s.rows == 0) {
        if (tid == 0) {
            kept[i] = 0;
            next[i] = -1;
            draw->p = nullptr;
        }
        return;
    }
    const epara_verify_args a = args[s.service];
    const int chunks = chunks_of_row(a.vocab, SIZE == 4 ? EPARA_F32 : EPARA_BF16, pieces);
    const bool drawn = a.draft_logits != nullptr;
    // ---- rows: a thread knows one
    int up = -1, parent = -1, token = -1;
    float uniform = 0.f;
    if (tid < s.rows) {
        up = parent_word(a, s, tid);
        parent = up >= 0 && up < tid ? up : -1;
        token = ((const EPARA_GLOBAL int32_t*)a.tokens)[static_cast<size_t>(s.first_row) + tid];
        uniform = ((const EPARA_GLOBAL float*)a.uniforms)[static_cast<size_t>(s.first_row) + tid];
    }
    const bool valid = token >= 0 && token < a.vocab;
    lds.parent[tid] = parent;
    lds.token[tid] = valid ? token : -1;
    lds.child[tid] = INT32_MAX;
    // ---- sums of the rows, 2^k lanes to a row
    int lanes = 1;
    while (lanes < 64 && lanes < chunks) lanes *= 2;
    const int lines = s.rows * (drawn && !temp.greedy ? 2 : 1);
    const float unit = LOG2E / temp.t;
    for (int line0 = 0; line0 < lines; line0 += NT / lanes) {
        const int line = line0 + tid / lanes;
        float top = -INFINITY;
        int place = INT32_MAX;
        double sum = 0.;
        auto join = [&](float t, int at, double y) {
            const float both = fmaxf(top, t);
            if (temp.greedy) {
                place = top == t ? min_of(place, at) : top > t ? place : at;
                sum += y;
            } else if (both > -INFINITY)
                sum = sum * __builtin_amdgcn_exp2f((top - both) * unit) + y * __builtin_amdgcn_exp2f((t - both) * unit);
            else
                sum += y;
            top = both;
        };
        if (line < lines) {
            const row_sum* src = sums + static_cast<size_t>(line) * chunks;
            for (int c = tid & (lanes - 1); c < chunks; c += lanes) {
                const row_sum r = src[c];
                join(r.top, r.at, r.sum);
            }
        }
        for (int d = lanes / 2; d >= 1; d >>= 1) {
            const float t = __shfl_xor(top, d);
            const int at = __shfl_xor(place, d);
            const double y = shuffle_xor(sum, d);
            join(t, at, y);
        }
        if (line < lines && (tid & (lanes - 1)) == 0) {
            const int draft = line >= s.rows, row = line - draft * s.rows;
            lds.top[draft][row] = top;
            lds.sum[draft][row] = sum;
            if (!draft) lds.place[row] = place;
        }
    }
    __syncthreads();
    // ---- probabilities of the rows' tokens
    double p = 0., q = 0.;
    if (parent >= 0 && valid) {
        const bool good = has_distribution(lds.sum[0][parent]);
        if (temp.greedy) p = good && lds.place[parent] == token ? 1. : 0.;
        else if (good) {
            const double per = LOG2E_64 / static_cast<double>(temp.t);
            const float x = logit_at<SIZE>(a.logits, s.first_row + parent, a.stride, token);
            p = exp2_64((static_cast<double>(x) - static_cast<double>(lds.top[0][parent])) * per) / lds.sum[0][parent];
            if (drawn) {
                const float y = logit_at<SIZE>(a.draft_logits, s.first_row + parent, a.draft_stride, token);
                q = exp2_64((static_cast<double>(y) - static_cast<double>(lds.top[1][parent])) * per) / lds.sum[1][parent];
                if (!has_distribution(lds.sum[1][parent])) q = __builtin_nan("");
            }
        }
    }
    if (a.probs && tid < s.rows) ((EPARA_GLOBAL float*)a.probs)[static_cast<size_t>(s.first_row) + tid] = static_cast<float>(p);
    // ---- elder siblings, and whether the row stays if its parent is the last that does
    // (all lanes look at the same row, and a branch would have each of these reads wait for the one before)
    const int upto = min_of(s.rows, __builtin_amdgcn_readfirstlane(tid) + 64);
    bool eldest = true, again = false;
#pragma unroll 8
    for (int j = 0; j < upto; ++j) {
        const bool sibling = (lds.parent[j] == parent) & (j < tid);
        eldest &= !sibling;
        again |= sibling & (lds.token[j] == token);
    }
    lds.takes[tid] = again ? 0. : p;
    __syncthreads();
    double mass = 1.;
    if (!drawn && !temp.greedy)
#pragma unroll 8
        for (int j = 0; j < upto; ++j) mass -= ((lds.parent[j] == parent) & (j < tid)) ? lds.takes[j] : 0.;
    if (parent >= 0 && valid && !again && has_distribution(lds.sum[0][parent])) {
        const double u = uniform > 0.f ? static_cast<double>(fminf(uniform, BELOW_ONE)) : 0.;
        const bool stays = temp.greedy ? p > 0. : u * (drawn ? q : mass) < p;
        if (stays && (eldest || !drawn)) atomicMin(&lds.child[parent], tid);
    }
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int row = up == -1 ? 0 : s.rows; row < s.rows; row = lds.child[row]) lds.path[n++] = row;      // (up: the first row's; without that row no other is there)
        lds.kept = n;
        lds.eldest = INT32_MAX;
        lds.n_without = 0;
    }
    __syncthreads();
    // ---- out
    const int n = lds.kept, last = n > 0 ? lds.path[n - 1] : 0;
    if (tid < s.rows) {
        ((EPARA_GLOBAL int32_t*)a.path)[static_cast<size_t>(s.first_row) + tid] = tid < n ? lds.path[tid] : -1;
        if (parent == last) {
            atomicMin(&lds.eldest, tid);
            if (!drawn && valid) draw->without[atomicAdd(&lds.n_without, 1)] = token;      // (in any order)
        }
    }
    __syncthreads();
    if (tid > 0) return;
    const bool good = n > 0 && has_distribution(lds.sum[0][last]);
    const bool rest = drawn && !temp.greedy && lds.eldest < s.rows && lds.token[lds.eldest] >= 0 && has_distribution(lds.sum[1][last]);
    kept[i] = n;
    if (!good || temp.greedy) next[i] = good ? lds.place[last] : -1;
    draw->p = good && !temp.greedy ? row_at(a.logits, s.first_row + last, a.stride, SIZE) : nullptr;
    draw->q = rest ? row_at(a.draft_logits, s.first_row + last, a.draft_stride, SIZE) : nullptr;
    draw->unit = LOG2E_64 / static_cast<double>(temp.t);
    draw->top_p = static_cast<double>(lds.top[0][last]);
    draw->top_q = rest ? static_cast<double>(lds.top[1][last]) : 0.;
    draw->ratio = rest ? lds.sum[0][last] / lds.sum[1][last] : 0.;
    draw->vocab = a.vocab;
    draw->n_without = lds.n_without;
    draw->uniform = uniform;                               // of the sequence's first row
}

// ---- the first kernel: a chunk of a row

// Thread 0 has the result.
template <int SIZE, int U>
__device__ __forceinline__ row_sum row_chunk(const epara_verify_args& a, const epara_sequence& s, const temperature& temp, int line, int chunk)
{
    constexpr int PER = 16 / SIZE, N = U * PER;
    __shared__ float tops[WAVES];
    __shared__ int places[WAVES];
    __shared__ double sums[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool draft = line >= s.rows;
    const int row = draft ? line - s.rows : line;
    if (draft) {                                           // only what a child was drawn from is looked at
        if (temp.greedy) return {};
        const bool child = tid > row && tid < s.rows && parent_of(a, s, tid) == row;
        if (!__syncthreads_or(child)) return {};
    }
    const row_view v = view_of<SIZE>(row_at(draft ? a.draft_logits : a.logits, s.first_row + row, draft ? a.draft_stride : a.stride, SIZE), a.vocab);
    float x[N];
    load_pieces<SIZE, U, 2>(v, chunk * (NT * U) + tid, NT, x);
    float top = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) top = fmaxf(top, x[j]);
    top = last_lane(wave_max(top));
    const float unit = LOG2E / temp.t;
    double sum = 0.;
    int place = INT32_MAX;
    if (temp.greedy) {
        bool bad = top == INFINITY;
#pragma unroll
        for (int u = U - 1; u >= 0; --u)
#pragma unroll
            for (int j = PER - 1; j >= 0; --j) {
                bad |= x[u * PER + j] != x[u * PER + j];
                if (x[u * PER + j] == top) place = (chunk * (NT * U) + tid + u * NT) * PER - v.skip + j;
            }
        place = top > -INFINITY ? wave_min(place) : INT32_MAX;
        sum = __ballot(bad) ? __builtin_nan("") : top > -INFINITY ? 1. : 0.;
    } else {
        const float from = top > -INFINITY ? top : 0.f;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < N; ++j) part[j & 1] += __builtin_amdgcn_exp2f((x[j] - from) * unit);
        sum = wave_scan(static_cast<double>(part[0] + part[1]));
    }
    if (lane == 63) {
        tops[wave] = top;
        places[wave] = place;
        sums[wave] = sum;
    }
    __syncthreads();
    if (tid > 0) return {};
    top = tops[0];
    place = places[0];
    sum = sums[0];
    for (int w = 1; w < WAVES; ++w) {
        const float both = fmaxf(top, tops[w]);
        if (temp.greedy) {
            place = top == tops[w] ? min_of(place, places[w]) : top == both ? place : places[w];
            sum += sums[w];                                // positive, or NaN
        } else if (both > -INFINITY)
            sum = sum * __builtin_amdgcn_exp2f((top - both) * unit) + sums[w] * __builtin_amdgcn_exp2f((tops[w] - both) * unit);
        else
            sum += sums[w];
        top = both;
    }
    return {top, place, sum};
}

template <int SIZE, int U>
__global__ __launch_bounds__(NT) void row_sums_kernel(const epara_verify_args* __restrict__ args, const epara_sequence* __restrict__ seqs, const int32_t* __restrict__ first,
                                                     int n_seqs, const float* __restrict__ temperatures, row_sum* __restrict__ out)
{
    const int item = blockIdx.x;
    const int i = find_sequence(first, n_seqs, item, threadIdx.x & 63);
    const epara_sequence s = seqs[i];
    const epara_verify_args a = args[s.service];
    const temperature temp = temperature_of(temperatures, i);
    const int chunks = chunks_of_row(a.vocab, SIZE == 4 ? EPARA_F32 : EPARA_BF16, U), line = (item - first[i]) / chunks, chunk = item - first[i] - line * chunks;
    const row_sum r = row_chunk<SIZE, U>(a, s, temp, line, chunk);
    if (threadIdx.x == 0) out[item] = r;
}

// ---- the token behind the last row that stays

struct block_lds {
    double sums[WAVES][4];
    int found[WAVES], some[WAVES];
    int place;
    double before;
    bool last;
};

// Sums over the workgroup: N at once; before: of the first, over the threads before this one.
template <int N>
__device__ __forceinline__ void block_sums(double* x, block_lds& lds, double& before)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double upto[N];
#pragma unroll
    for (int k = 0; k < N; ++k) upto[k] = wave_scan(x[k]);
    __syncthreads();                                       // (what was here before has been read)
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) lds.sums[wave][k] = upto[k];
    __syncthreads();
    before = upto[0] - x[0];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = 0.;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += lds.sums[w][0];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] += lds.sums[w][k];
    }
}

// The first thread whose share [before, before + share) of the sums reaches over goal; if rounding leaves none, the last one with a share.
__device__ __forceinline__ int block_find(double before, double share, double goal, block_lds& lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t some = __ballot(share > 0.), over = __ballot(share > 0. && before + share > goal);
    __syncthreads();
    if (lane == 0) {
        lds.found[wave] = over ? __builtin_ctzll(over) + 64 * wave : -1;
        lds.some[wave] = some ? 63 - __builtin_clzll(some) + 64 * wave : -1;
    }
    __syncthreads();
    int found = -1, last = -1;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (found < 0) found = lds.found[w];
        last = max_of(last, lds.some[w]);
    }
    return found >= 0 ? found : last;
}

template <int SIZE, int U>
__device__ __forceinline__ void load_like(const row_view& v, const row_view& like, int piece, float* x)
{
    if (v.skip == like.skip) return load_pieces<SIZE, U>(v, piece, 1, x);
    constexpr int PER = 16 / SIZE;                         // rows that begin at different places of a piece: element by element
#pragma unroll
    for (int j = 0; j < U * PER; ++j) {
        const int at = piece * PER - like.skip + j;
        const bool there = at >= 0 && at < v.vocab;
        const int byte = (v.skip + (there ? at : 0)) * SIZE;
        float y;
        if constexpr (SIZE == 4) y = __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b32(v.rsrc, byte, 0, 0)));
        else y = __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b16(v.rsrc, byte, 0, 0)) << 16);
        x[j] = there ? y : -INFINITY;
    }
}
// The third kernel: a chunk of the row behind which a sequence's token is drawn.  Thread t has the elements of pieces t U .. t U + U - 1 of the chunk, in order.
template <int SIZE, int U>
__global__ __launch_bounds__(NT) void draw_kernel(const drawn_row* __restrict__ draws, uint32_t* counters, chunk_sum* all_sums, int most_chunks, int32_t* __restrict__ next)
{
    constexpr int PER = 16 / SIZE, N = U * PER;
    __shared__ block_lds lds;
    const int tid = threadIdx.x, i = blockIdx.x / most_chunks;
    int chunk = blockIdx.x - i * most_chunks;
    const drawn_row& d = draws[i];
    const int vocab = d.vocab, n_without = d.n_without, chunks = chunks_of_row(vocab, SIZE == 4 ? EPARA_F32 : EPARA_BF16, U);
    if (!d.p || chunk >= chunks) return;
    const row_view p = view_of<SIZE>(d.p, vocab), q = view_of<SIZE>(d.q ? d.q : d.p, vocab);
    const bool rest = d.q != nullptr;
    const double unit = d.unit, top_p = d.top_p, top_q = d.top_q;
    const float u = d.uniform;
    chunk_sum* sums = all_sums + static_cast<size_t>(i) * most_chunks;
    double ratio = d.ratio * MORE, total = 0., goal = 0., base = 0.;
    bool exact = false;                                    // the chunks' sums are of the very weights that pass 2 looks at
    // 0: my chunk's sums; 1: all chunks' once more, one after the other (only where next to nothing is left); 2: the chunk with the token
    for (int pass = 0;;) {
        float x[N];
        double out[N], sums_of[4] = {0., 0., 0., 0.}, before;      // of what the token is drawn with, of p, of q, of q where something is left
        const int piece = chunk * (NT * U) + tid * U, at = piece * PER - p.skip;
        load_pieces<SIZE, U>(p, piece, 1, x);
        for (int k = 0; k < n_without; ++k) {
            const int place = d.without[k] - at;
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j == place) x[j] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            out[j] = exp2_64((static_cast<double>(x[j]) - top_p) * unit);
            sums_of[1] += out[j];
        }
        sums_of[0] = sums_of[1];
        if (rest) {
            load_like<SIZE, U>(q, p, piece, x);
            sums_of[0] = 0.;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const double b = exp2_64((static_cast<double>(x[j]) - top_q) * unit), left = out[j] - ratio * b;
                out[j] = fmax(left, 0.);
                sums_of[0] += out[j];
                sums_of[2] += b;
                sums_of[3] += left > 0. ? b : 0.;
            }
        }
        const double mine = sums_of[0];
        if (rest && pass == 0) block_sums<4>(sums_of, lds, before);
        else                   block_sums<1>(sums_of, lds, before);
        if (pass < 2) {
            if (tid == 0) {
                put8(&sums[chunk].rest, __builtin_bit_cast(uint64_t, sums_of[0]));
                if (pass == 0 && rest) {
                    put8(&sums[chunk].p, __builtin_bit_cast(uint64_t, sums_of[1]));
                    put8(&sums[chunk].q, __builtin_bit_cast(uint64_t, sums_of[2]));
                    put8(&sums[chunk].q_of_rest, __builtin_bit_cast(uint64_t, sums_of[3]));
                }
                if (pass == 0) lds.last = is_last(counters + i, chunks);
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            __syncthreads();
            if (!lds.last) return;
            if (pass == 1 && ++chunk < chunks) continue;
            exact = pass == 1;
            // ---- the chunk: a thread has some of them in a row
            const int share = (chunks + NT - 1) / NT, lo = min_of(tid * share, chunks), hi = min_of(lo + share, chunks);
            double move = 0., some[1] = {0.};              // of the ratio, from what the sums were made with
            if (pass == 0 && rest) {
                double both[2] = {0., 0.};
                for (int c = lo; c < hi; ++c) {
                    both[0] += get_double(&sums[c].p);
                    both[1] += get_double(&sums[c].q);
                }
                block_sums<2>(both, lds, before);
                total = both[0];
                move = total / both[1] * MORE - ratio;
                ratio += move;
            }
            auto chunk_share = [&](int c) { return move == 0. ? get_double(&sums[c].rest) : fmax(get_double(&sums[c].rest) - move * get_double(&sums[c].q_of_rest), 0.); };
            for (int c = lo; c < hi; ++c) some[0] += chunk_share(c);
            const double share_of_mine = some[0];
            block_sums<1>(some, lds, before);
            if (pass == 0 && rest && some[0] < total * 0x1p-10) {
                pass = 1;
                chunk = 0;
                continue;
            }
            if (!(some[0] > 0.)) break;
            goal = some[0] * (u > 0.f ? static_cast<double>(fminf(u, BELOW_ONE)) : 0.);
            if (tid == block_find(before, share_of_mine, goal, lds)) {
                int found = lo;
                double upto = before, at_found = before;
                for (int c = lo; share > 1 && c < hi; ++c) {
                    const double y = chunk_share(c);
                    if (y > 0.) {
                        found = c;
                        at_found = upto;
                        if (upto + y > goal) break;
                    }
                    upto += y;
                }
                lds.place = found;
                lds.before = at_found;
            }
            __syncthreads();
            chunk = __builtin_amdgcn_readfirstlane(lds.place);
            base = lds.before;
            pass = 2;
            continue;
        }
        // ---- and the token in it
        const int found = block_find(base + before, mine, goal, lds);
        if (found < 0) {                                   // (all threads: a corrected sum that is rounding after all)
            if (exact) break;
            pass = 1;
            chunk = 0;
            continue;
        }
        if (tid != found) return;
        int place = 0;
        double upto = base + before;
        bool done = false;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (!done && out[j] > 0.) place = j;
            upto += out[j];
            done |= out[j] > 0. && upto > goal;
        }
        next[i] = at + place;
        return;
    }
    // ---- nothing is left at all: the largest logit, the first of equal ones
    int place = INT32_MAX;
    for (int c = 0; c < chunks; ++c) {
        float x[N];
        load_pieces<SIZE, U>(p, c * (NT * U) + tid * U, 1, x);
#pragma unroll
        for (int j = N - 1; j >= 0; --j)
            if (static_cast<double>(x[j]) == top_p) place = min_of(place, (c * (NT * U) + tid * U) * PER - p.skip + j);
    }
    place = wave_min(place);
    __syncthreads();
    if ((tid & 63) == 0) lds.found[tid >> 6] = place;
    __syncthreads();
    if (tid == 0) next[i] = min_of(min_of(lds.found[0], lds.found[1]), min_of(lds.found[2], lds.found[3]));
}

template <int SIZE>
int32_t launch_verify(const epara_verify_launch& l, hipStream_t stream)
{
    const int n_seqs = l.table.n_seqs;
    workspace ws;
    char* at = static_cast<char*>(l.d_workspace);
    ws.counters = reinterpret_cast<uint32_t*>(at);
    at += counter_bytes(n_seqs);
    ws.drawn = reinterpret_cast<drawn_row*>(at);
    at += static_cast<size_t>(n_seqs) * sizeof(drawn_row);
    ws.rows = reinterpret_cast<row_sum*>(at);
    at += static_cast<size_t>(l.plan.n_items) * sizeof(row_sum);
    ws.chunks = reinterpret_cast<chunk_sum*>(at);
    if (l.plan.n_items > 0) {
        const auto kernel = l.plan.pieces == 1 ? row_sums_kernel<SIZE, 1> : l.plan.pieces == 2 ? row_sums_kernel<SIZE, 2> : l.plan.pieces == 4 ? row_sums_kernel<SIZE, 4> : row_sums_kernel<SIZE, 8>;
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(l.plan.n_items)), dim3(NT), 0, stream, l.d_args, l.table.d_seqs, l.d_first, n_seqs, l.d_temperatures, ws.rows);
    }
    hipLaunchKernelGGL(walk_kernel<SIZE>, dim3(static_cast<unsigned>(n_seqs)), dim3(NT), 0, stream, l.d_args, l.table.d_seqs, l.d_first, l.d_temperatures, ws.rows, ws.drawn,
                       l.plan.pieces, l.d_kept, l.d_next);
    if (l.d_temperatures) {                                // greedy sequences' tokens are known by now
        const auto kernel = l.plan.draw_pieces == 1 ? draw_kernel<SIZE, 1> : l.plan.draw_pieces == 2 ? draw_kernel<SIZE, 2> : draw_kernel<SIZE, 4>;
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(n_seqs) * static_cast<unsigned>(l.plan.draw_chunks)), dim3(NT), 0, stream, ws.drawn, ws.counters, ws.chunks,
                           l.plan.draw_chunks, l.d_next);
    }
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}

}  // namespace

extern "C" int32_t epara_verify_drafts(const epara_verify_launch* launch, void* stream)
{
    if (!launch) return EPARA_ERR_NULL;
    const epara_verify_launch& l = *launch;
    if (const int32_t rc = epara_check_verify_call(l)) return rc;
    if (l.table.n_seqs == 0) return EPARA_OK;
    if (!l.d_args || !l.d_first) return EPARA_ERR_NULL;
    return l.dtype == EPARA_F32 ? launch_verify<4>(l, static_cast<hipStream_t>(stream)) : launch_verify<2>(l, static_cast<hipStream_t>(stream));
}
