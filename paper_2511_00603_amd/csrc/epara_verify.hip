// libepara: which drafted tokens the target agrees to, and the token behind them.
//
// Three kernels at most.  The first reads all logits once and leaves for each chunk of a row its largest logit and sum exp((x - top) / T).  In the second every workgroup of
// a sequence walks its tree again from these sums (a few dependent trips to memory, which cost less than another launch), and sums one chunk of the row behind which the
// token is drawn, in 64 bits; who ends last finds the token.  Where the token comes from max(p - q, 0), whose weights need both sums first, a third kernel does that part.
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
constexpr float BELOW_ONE = 0x1.fffffep-1f;

// Where the parts of a call's workspace are.
struct workspace {
    uint32_t* counters;          // [n_seqs]
    drawn_row* drawn;            // [n_seqs]
    row_sum* rows;               // [n_items[0]]
    chunk_sum* chunks;           // [n_items[1]]
};

// ---- a row of logits in pieces of 16 bytes

struct row_view {
    __amdgpu_buffer_rsrc_t rsrc; // from the 16-byte boundary at or before the row to the end of its last word: what lies behind reads as zero
    int skip, vocab;             // elements of the first piece that are not the row's
};
template <int SIZE>
__device__ __forceinline__ row_view view_of(const void* logits, int row, int stride, int vocab)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(logits) + static_cast<size_t>(row) * stride * SIZE, base = at & ~static_cast<uintptr_t>(15);
    const int skip = static_cast<int>(at - base);
    return {__builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, (skip + vocab * SIZE + 3) & ~3, 0x00020000), skip / SIZE, vocab};
}

// The elements of pieces first, first + step, ..; what is not the row's is -infinity.
template <int SIZE, int U>
__device__ __forceinline__ void load_pieces(const row_view& v, int first, int step, float* x)
{
    constexpr int PER = 16 / SIZE;
    v4i raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(v.rsrc, (first + u * step) * 16, 0, 0));
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

// The row that row `row` of a sequence follows, or -1.
__device__ __forceinline__ int parent_of(const epara_verify_args& a, const epara_sequence& s, int row)
{
    const int p = a.parents ? ((const EPARA_GLOBAL int32_t*)a.parents)[static_cast<size_t>(s.first_row) + row] : row - 1;
    return p >= 0 && p < row ? p : -1;
}

__device__ __forceinline__ double shuffle_xor(double x, int d)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, static_cast<uint64_t>(static_cast<uint32_t>(__shfl_xor(static_cast<int>(u), d))) |
                                          static_cast<uint64_t>(static_cast<uint32_t>(__shfl_xor(static_cast<int>(u >> 32), d))) << 32);
}
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += shuffle_xor(x, d);
    return x;
}
__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ int wave_min(int x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x = min_of(x, __shfl_xor(x, d));
    return x;
}

// ---- the first kernel: a chunk of a row

template <int SIZE, int U>
__global__ __launch_bounds__(NT) void row_sums_kernel(const epara_verify_args* __restrict__ args, const epara_sequence* __restrict__ seqs, const int32_t* __restrict__ first,
                                                     int n_seqs, const float* __restrict__ temperatures, row_sum* __restrict__ out)
{
    constexpr int PER = 16 / SIZE, N = U * PER;
    __shared__ float tops[WAVES];
    __shared__ int places[WAVES];
    __shared__ double sums[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, item = blockIdx.x;
    const int i = find_sequence(first, n_seqs, item, lane);
    const epara_sequence s = seqs[i];
    const epara_verify_args a = args[s.service];
    const temperature temp = temperature_of(temperatures, i);
    const int chunks = chunks_of_row(a.vocab, SIZE == 4 ? EPARA_F32 : EPARA_BF16, U), line = (item - first[i]) / chunks, chunk = item - first[i] - line * chunks;
    const bool draft = line >= s.rows;
    const int row = draft ? line - s.rows : line;
    if (draft) {                                           // only what a child was drawn from is looked at
        if (temp.greedy) return;
        const bool child = tid > row && tid < s.rows && parent_of(a, s, tid) == row;
        if (!__syncthreads_or(child)) return;
    }
    const row_view v = view_of<SIZE>(draft ? a.draft_logits : a.logits, s.first_row + row, draft ? a.draft_stride : a.stride, a.vocab);
    float x[N];
    load_pieces<SIZE, U>(v, chunk * (NT * U) + tid, NT, x);
    float top = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) top = fmaxf(top, x[j]);
    top = wave_max(top);
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
        const float unit = LOG2E / temp.t, from = top > -INFINITY ? top : 0.f;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < N; ++j) part[j & 1] += __builtin_amdgcn_exp2f((x[j] - from) * unit);
        sum = wave_sum(static_cast<double>(part[0] + part[1]));
    }
    if (lane == 0) {
        tops[wave] = top;
        places[wave] = place;
        sums[wave] = sum;
    }
    __syncthreads();
    if (tid > 0) return;
    for (int w = 1; w < WAVES; ++w) {
        const float both = fmaxf(top, tops[w]);
        if (temp.greedy) {
            place = top == both && tops[w] == both ? min_of(place, places[w]) : top == both ? place : places[w];
            sum += sums[w];                                // positive, or NaN
        } else if (both > -INFINITY) {
            const float unit = LOG2E / temp.t;
            sum = sum * __builtin_amdgcn_exp2f((top - both) * unit) + sums[w] * __builtin_amdgcn_exp2f((tops[w] - both) * unit);
        } else
            sum += sums[w];
        top = both;
    }
    out[item] = {top, place, sum};
}

// ---- the walk

struct walk_lds {
    float top[2][TREE_ROWS];     // of a row's logits and draft logits
    int place[TREE_ROWS];
    double sum[2][TREE_ROWS];    // NaN or 0: no distribution
    double p[TREE_ROWS];         // of a row's token behind its parent
    int parent[TREE_ROWS], token[TREE_ROWS];
    int child[TREE_ROWS];        // the one that stays behind a row, if the row does
    bool again[TREE_ROWS];       // an elder sibling has its token, or it is none of the vocabulary
    int path[TREE_ROWS];
    int kept, eldest;            // eldest: child of the row that stays last
};

struct block_lds {
    double scan[WAVES];
    int found, place;
    double before;
    uint32_t last;
};

__device__ __forceinline__ bool has_distribution(double sum) { return sum > 0. && sum < static_cast<double>(INFINITY); }

// All threads of a workgroup: which rows of a sequence stay.  lds.path and kept; probs are written where given.
template <int SIZE>
__device__ void walk(const epara_verify_args& a, const epara_sequence& s, const temperature& temp, const row_sum* __restrict__ sums, int chunks, walk_lds& lds, bool writes)
{
    const int tid = threadIdx.x;
    const bool drawn = a.draft_logits != nullptr;
    // ---- rows: a thread knows one
    int parent = -1, token = -1;
    float uniform = 0.f;
    if (tid < s.rows) {
        parent = parent_of(a, s, tid);
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
    for (int line0 = 0; line0 < lines; line0 += NT / lanes) {
        const int line = line0 + tid / lanes;
        float top = -INFINITY;
        int place = INT32_MAX;
        double sum = 0.;
        const float unit = LOG2E / temp.t;
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
            const float x = logit_at<SIZE>(a.logits, s.first_row + parent, a.stride, token);
            p = exp((static_cast<double>(x) - static_cast<double>(lds.top[0][parent])) / static_cast<double>(temp.t)) / lds.sum[0][parent];
            if (drawn) {
                const float y = logit_at<SIZE>(a.draft_logits, s.first_row + parent, a.draft_stride, token);
                q = exp((static_cast<double>(y) - static_cast<double>(lds.top[1][parent])) / static_cast<double>(temp.t)) / lds.sum[1][parent];
                if (!has_distribution(lds.sum[1][parent])) q = __builtin_nan("");
            }
        }
    }
    lds.p[tid] = p;
    if (writes && a.probs && tid < s.rows) ((EPARA_GLOBAL float*)a.probs)[static_cast<size_t>(s.first_row) + tid] = static_cast<float>(p);
    __syncthreads();
    // ---- elder siblings, and whether the row stays if its parent is the last that does
    bool eldest = true, again = false;
    if (parent >= 0)
        for (int j = parent + 1; j < tid; ++j)
            if (lds.parent[j] == parent) {
                eldest = false;
                again |= lds.token[j] == lds.token[tid];
            }
    lds.again[tid] = again || !valid;
    __syncthreads();
    if (parent >= 0 && valid && !again && has_distribution(lds.sum[0][parent])) {
        const double u = uniform > 0.f ? static_cast<double>(fminf(uniform, BELOW_ONE)) : 0.;
        bool stays;
        if (temp.greedy) stays = p > 0.;
        else if (drawn)  stays = u * q < p;
        else {
            double mass = 1.;
            for (int j = parent + 1; j < tid; ++j)
                if (lds.parent[j] == parent && !lds.again[j]) mass -= lds.p[j];
            stays = u * mass < p;
        }
        if (stays && (eldest || !drawn)) atomicMin(&lds.child[parent], tid);
    }
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int row = 0; row < s.rows; row = lds.child[row]) lds.path[n++] = row;
        lds.kept = n;
    }
    __syncthreads();
}

// ---- the token behind the last row that stays

// Sum over the workgroup, and over the threads before this one; the same bits whoever computes it.
__device__ __forceinline__ double block_scan(double x, block_lds& lds, double& before)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double upto = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t u = __builtin_bit_cast(uint64_t, upto);
        const uint64_t y = static_cast<uint64_t>(static_cast<uint32_t>(__shfl_up(static_cast<int>(u), d))) | static_cast<uint64_t>(static_cast<uint32_t>(__shfl_up(static_cast<int>(u >> 32), d))) << 32;
        if (lane >= d) upto += __builtin_bit_cast(double, y);
    }
    __syncthreads();                                       // (a scan before this one has been read)
    if (lane == 63) lds.scan[wave] = upto;
    __syncthreads();
    double base = 0., total = 0.;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) base = total;
        total += lds.scan[w];
    }
    before = base + (upto - x);
    return total;
}

// The first thread whose share [before, before + share) of the sums reaches over goal; if rounding leaves none, the last one with a share.
__device__ __forceinline__ int block_find(double before, double share, double goal, block_lds& lds)
{
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) {
        lds.found = INT32_MAX;
        lds.place = -1;
    }
    __syncthreads();
    if (share > 0.) {
        if (before + share > goal) atomicMin(&lds.found, tid);
        atomicMax(&lds.place, tid);
    }
    __syncthreads();
    return lds.found < NT ? lds.found : lds.place;
}

// Weights of a chunk of a row: exp((x - top) / T) without some tokens, or max(p - q, 0).  Thread t has the elements of pieces t U .. t U + U - 1, in order.
struct row_weights {
    row_view p, q;
    bool rest;                   // max(p - q, 0)
    double top_p, top_q, inv_t, inv_p, inv_q;
    int without_children_of;     // or -1
    int rows;
};
template <int SIZE, int U>
__device__ __forceinline__ void load_like(const row_view& v, const row_view& like, int piece, float* x)
{
    if (v.skip == like.skip) return load_pieces<SIZE, U>(v, piece, 1, x);
    constexpr int PER = 16 / SIZE;                         // rows that begin at different places of a piece: element by element
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
template <int SIZE, int U>
__device__ __forceinline__ void chunk_weights(const row_weights& w, const walk_lds& lds, int chunk, double* out, double& sum_p, double& sum_q)
{
    constexpr int PER = 16 / SIZE, N = U * PER;
    const int piece = chunk * (NT * U) + threadIdx.x * U, at = piece * PER - w.p.skip;
    float x[N];
    load_pieces<SIZE, U>(w.p, piece, 1, x);
    if (w.without_children_of >= 0)
        for (int r = w.without_children_of + 1; r < w.rows; ++r) {
            if (lds.parent[r] != w.without_children_of || lds.token[r] < 0) continue;
            const int place = lds.token[r] - at;
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j == place) x[j] = -INFINITY;
        }
    sum_p = sum_q = 0.;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        out[j] = exp((static_cast<double>(x[j]) - w.top_p) * w.inv_t);
        sum_p += out[j];
    }
    if (!w.rest) return;
    load_like<SIZE, U>(w.q, w.p, piece, x);
    sum_p = 0.;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const double q = exp((static_cast<double>(x[j]) - w.top_q) * w.inv_t);
        sum_q += q;
        out[j] = fmax(out[j] * w.inv_p - q * w.inv_q, 0.);
        sum_p += out[j];
    }
}

// 8 bytes for, or from, workgroups on other dies in the same kernel: past the dies' own caches.
__device__ __forceinline__ void put_double(double* at, double x) { __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), __builtin_bit_cast(unsigned long long, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double get_double(const double* at) { return __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)); }

// A chunk's sum goes to the workspace; who is the last of a sequence's workgroups to come here finds the token.
template <int SIZE, int U>
__device__ void draw(const row_weights& w, const walk_lds& lds, block_lds& bl, uint32_t* counter, chunk_sum* sums, int chunk, int chunks, double sum, float uniform, int32_t* next)
{
    constexpr int PER = 16 / SIZE, N = U * PER;
    const int tid = threadIdx.x;
    if (tid == 0) {
        put_double(&sums[chunk].rest, sum);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        bl.last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<uint32_t>(chunks - 1);
    }
    __syncthreads();
    if (!bl.last) return;
    if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // ---- the chunk: a thread has some of them in a row
    const int share = (chunks + NT - 1) / NT, lo = min_of(tid * share, chunks), hi = min_of(lo + share, chunks);
    double mine = 0., before, out[N], other;
    for (int c = lo; c < hi; ++c) mine += get_double(&sums[c].rest);
    const double total = block_scan(mine, bl, before), goal = total * (uniform > 0.f ? static_cast<double>(fminf(uniform, BELOW_ONE)) : 0.);
    if (!(total > 0.)) {                                   // nothing is left: the largest logit, the first of equal ones
        int place = INT32_MAX;
        for (int c = 0; c < chunks; ++c) {
            float x[N];
            load_pieces<SIZE, U>(w.p, c * (NT * U) + tid * U, 1, x);
#pragma unroll
            for (int j = N - 1; j >= 0; --j)
                if (static_cast<double>(x[j]) == w.top_p) place = min_of(place, (c * (NT * U) + tid * U) * PER - w.p.skip + j);
        }
        __syncthreads();
        if (tid == 0) bl.found = INT32_MAX;
        __syncthreads();
        atomicMin(&bl.found, place);
        __syncthreads();
        if (tid == 0) *(EPARA_GLOBAL int32_t*)next = bl.found;
        return;
    }
    const int who = block_find(before, mine, goal, bl);
    if (tid == who) {
        int c = lo, some = lo;
        double upto = before, at_some = before;
        for (; c < hi; ++c) {
            const double x = get_double(&sums[c].rest);
            if (x > 0.) {
                some = c;
                at_some = upto;
                if (upto + x > goal) break;
            }
            upto += x;
        }
        bl.place = some;
        bl.before = at_some;
    }
    __syncthreads();
    const int at_chunk = __builtin_amdgcn_readfirstlane(bl.place);
    const double base = bl.before;
    // ---- and the token in it
    chunk_weights<SIZE, U>(w, lds, at_chunk, out, mine, other);
    block_scan(mine, bl, before);
    const int thread = block_find(base + before, mine, goal, bl);
    if (tid != thread) return;
    int place = 0;
    double upto = base + before;
    bool done = false;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (!done && out[j] > 0.) place = j;
        upto += out[j];
        done |= out[j] > 0. && upto > goal;
    }
    *(EPARA_GLOBAL int32_t*)next = (at_chunk * (NT * U) + tid * U) * PER - w.p.skip + place;
}

template <int SIZE, int U>
__global__ __launch_bounds__(NT) void walk_kernel(const epara_verify_args* __restrict__ args, const epara_sequence* __restrict__ seqs, const int32_t* __restrict__ first,
                                                 int n_seqs, const float* __restrict__ temperatures, workspace ws, int32_t* kept, int32_t* next)
{
    constexpr int N = U * 16 / SIZE;
    __shared__ walk_lds lds;
    __shared__ block_lds bl;
    const int tid = threadIdx.x, lane = tid & 63, item = blockIdx.x;
    const int i = find_sequence(first + n_seqs + 1, n_seqs, item, lane);
    const epara_sequence s = seqs[i];
    const epara_verify_args a = args[s.service];
    const temperature temp = temperature_of(temperatures, i);
    const int chunks = chunks_of_row(a.vocab, SIZE == 4 ? EPARA_F32 : EPARA_BF16, U), chunk = item - first[n_seqs + 1 + i];
    const bool writes = chunk == 0;
    if (s.rows == 0) {
        if (writes && tid == 0) {
            kept[i] = 0;
            next[i] = -1;
            ws.drawn[i].row = -1;
        }
        return;
    }
    walk<SIZE>(a, s, temp, ws.rows + first[i], chunks, lds, writes);
    const int n = __builtin_amdgcn_readfirstlane(lds.kept), last = __builtin_amdgcn_readfirstlane(lds.path[n - 1]);
    const bool good = has_distribution(lds.sum[0][last]);
    if (writes) {
        if (tid < s.rows) ((EPARA_GLOBAL int32_t*)a.path)[static_cast<size_t>(s.first_row) + tid] = tid < n ? lds.path[tid] : -1;
        if (tid == 0) {
            kept[i] = n;
            if (!good || temp.greedy) next[i] = good ? lds.place[last] : -1;
        }
    }
    const bool drawn = a.draft_logits != nullptr;
    if (tid == 0) lds.eldest = INT32_MAX;
    __syncthreads();
    if (tid < s.rows && lds.parent[tid] == last) atomicMin(&lds.eldest, tid);
    __syncthreads();
    const bool rest = good && !temp.greedy && drawn && lds.eldest < s.rows && lds.token[lds.eldest] >= 0 && has_distribution(lds.sum[1][last]);
    if (writes && tid == 0) ws.drawn[i] = {rest ? last : -1, lds.top[0][last], rest ? lds.top[1][last] : 0.f, 0};
    if (!good || temp.greedy) return;
    row_weights w;
    w.p = view_of<SIZE>(a.logits, s.first_row + last, a.stride, a.vocab);
    w.rest = false;
    w.top_p = static_cast<double>(lds.top[0][last]);
    w.inv_t = 1. / static_cast<double>(temp.t);
    w.without_children_of = drawn ? -1 : last;
    w.rows = s.rows;
    double out[N], sum, other, before;
    chunk_weights<SIZE, U>(w, lds, chunk, out, sum, other);
    sum = block_scan(sum, bl, before);
    chunk_sum* sums = ws.chunks + first[n_seqs + 1 + i];
    if (rest) {                                            // the weights need both rows' sums: the third kernel
        w.p = view_of<SIZE>(a.draft_logits, s.first_row + last, a.draft_stride, a.vocab);
        w.top_p = static_cast<double>(lds.top[1][last]);
        chunk_weights<SIZE, U>(w, lds, chunk, out, other, before);
        other = block_scan(other, bl, before);
        if (tid == 0) {
            sums[chunk].p = sum;
            sums[chunk].q = other;
        }
        return;
    }
    draw<SIZE, U>(w, lds, bl, ws.counters + i, sums, chunk, chunks, sum, ((const EPARA_GLOBAL float*)a.uniforms)[s.first_row], next + i);
}

template <int SIZE, int U>
__global__ __launch_bounds__(NT) void rest_kernel(const epara_verify_args* __restrict__ args, const epara_sequence* __restrict__ seqs, const int32_t* __restrict__ first,
                                                 int n_seqs, const float* __restrict__ temperatures, workspace ws, int32_t* next)
{
    constexpr int N = U * 16 / SIZE;
    __shared__ walk_lds lds;                               // (no children are left out: not read)
    __shared__ block_lds bl;
    const int tid = threadIdx.x, lane = tid & 63, item = blockIdx.x;
    const int i = find_sequence(first + n_seqs + 1, n_seqs, item, lane);
    drawn_row d = ws.drawn[i];
    d.row = __builtin_amdgcn_readfirstlane(d.row);
    if (d.row < 0) return;
    const epara_sequence s = seqs[i];
    const epara_verify_args a = args[s.service];
    const temperature temp = temperature_of(temperatures, i);
    const int chunks = chunks_of_row(a.vocab, SIZE == 4 ? EPARA_F32 : EPARA_BF16, U), chunk = item - first[n_seqs + 1 + i];
    chunk_sum* sums = ws.chunks + first[n_seqs + 1 + i];
    double p = 0., q = 0., before;
    for (int c = tid; c < chunks; c += NT) {
        p += sums[c].p;
        q += sums[c].q;
    }
    p = block_scan(p, bl, before);
    q = block_scan(q, bl, before);
    row_weights w;
    w.p = view_of<SIZE>(a.logits, s.first_row + d.row, a.stride, a.vocab);
    w.q = view_of<SIZE>(a.draft_logits, s.first_row + d.row, a.draft_stride, a.vocab);
    w.rest = true;
    w.top_p = static_cast<double>(d.top_p);
    w.top_q = static_cast<double>(d.top_q);
    w.inv_t = 1. / static_cast<double>(temp.t);
    w.inv_p = 1. / p;
    w.inv_q = 1. / q;
    w.without_children_of = -1;
    w.rows = 0;
    double out[N], sum, other;
    chunk_weights<SIZE, U>(w, lds, chunk, out, sum, other);
    sum = block_scan(sum, bl, before);
    draw<SIZE, U>(w, lds, bl, ws.counters + i, sums, chunk, chunks, sum, ((const EPARA_GLOBAL float*)a.uniforms)[s.first_row], next + i);
}

template <int SIZE, int U>
int32_t launch_verify(const epara_verify_launch& l, hipStream_t stream)
{
    workspace ws;
    char* at = static_cast<char*>(l.d_workspace);
    ws.counters = reinterpret_cast<uint32_t*>(at);
    at += counter_bytes(l.table.n_seqs);
    ws.drawn = reinterpret_cast<drawn_row*>(at);
    at += static_cast<size_t>(l.table.n_seqs) * sizeof(drawn_row);
    ws.rows = reinterpret_cast<row_sum*>(at);
    at += static_cast<size_t>(l.plan.n_items[0]) * sizeof(row_sum);
    ws.chunks = reinterpret_cast<chunk_sum*>(at);
    const int n_seqs = l.table.n_seqs;
    if (l.plan.n_items[0] > 0)
        hipLaunchKernelGGL((row_sums_kernel<SIZE, U>), dim3(static_cast<unsigned>(l.plan.n_items[0])), dim3(NT), 0, stream, l.d_args, l.table.d_seqs, l.d_first, n_seqs, l.d_temperatures, ws.rows);
    hipLaunchKernelGGL((walk_kernel<SIZE, U>), dim3(static_cast<unsigned>(l.plan.n_items[1])), dim3(NT), 0, stream, l.d_args, l.table.d_seqs, l.d_first, n_seqs, l.d_temperatures, ws, l.d_kept, l.d_next);
    bool rest = false;
    for (int32_t g = 0; g < l.G; ++g) rest |= l.h_args[g].draft_logits != nullptr;
    if (rest && l.d_temperatures)
        hipLaunchKernelGGL((rest_kernel<SIZE, U>), dim3(static_cast<unsigned>(l.plan.n_items[1])), dim3(NT), 0, stream, l.d_args, l.table.d_seqs, l.d_first, n_seqs, l.d_temperatures, ws, l.d_next);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}

template <int SIZE>
int32_t launch_pieces(const epara_verify_launch& l, hipStream_t stream)
{
    switch (l.plan.pieces) {
    case 1: return launch_verify<SIZE, 1>(l, stream);
    case 2: return launch_verify<SIZE, 2>(l, stream);
    case 4: return launch_verify<SIZE, 4>(l, stream);
    default: return launch_verify<SIZE, 8>(l, stream);
    }
}

}  // namespace

extern "C" int32_t epara_verify_drafts(const epara_verify_launch* launch, void* stream)
{
    if (!launch) return EPARA_ERR_NULL;
    const epara_verify_launch& l = *launch;
    if (const int32_t rc = epara_check_verify_call(l)) return rc;
    if (l.table.n_seqs == 0) return EPARA_OK;
    if (!l.d_args || !l.d_first) return EPARA_ERR_NULL;
    return l.dtype == EPARA_F32 ? launch_pieces<4>(l, static_cast<hipStream_t>(stream)) : launch_pieces<2>(l, static_cast<hipStream_t>(stream));
}
