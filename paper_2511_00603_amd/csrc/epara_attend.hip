// libepara: causal attention of new tokens over a paged cache in 8 bits (the decode and prefill services' attention).
//
//   o = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m),   z_j = scale q . k_j (capped: c tanh(z_j / c)),   m = max_j z_j
//
// Keys and values go from memory into the matrix cores as they lie in the cache, E4M3 codes with E8M0 scales: nothing is
// converted.  A query is the sum of two E4M3 numbers, q = hi + lo / 16 with the head's own power of two, which holds all 8
// significant bits of a bf16; so is a weight p = exp(z - m).  The scaled products of 8-bit operands run at twice the rate of bf16
// ones, so the two products cost what one in bf16 would.  (Weights rounded to bf16 would be 2.7 times coarser.)
//
// Both products are written transposed, so that what the first leaves in a lane is what the second wants there:
//   S^T = K Q^T   A = 16 keys x 128 (dims), B = the same dims of 16 rows
//   O^T = V^T P^T A = 16 dims x 64 tokens, B = the same tokens of 16 rows
// Lane (n = lane % 16, q = lane / 16) gets from the four tiles t of S^T of a page the scores of row n with the keys
// 16 q + 4 t + 0 .. 3: the 16 tokens of quarter q of the page, which is how the cache holds the values (a 16-byte chunk = 16
// tokens of a dim) and why it holds the keys in the order it does.  In the contraction of an instruction of 128 a lane's first 16
// bytes are elements 16 q .. of it, its second 16 bytes elements 64 + 16 q ..; elements 32 b .. 32 b + 31 take their scale from the lanes of quarter b.
// So O^T takes hi in the first half and lo in the second against the same values, one instruction for both.
//
// A workgroup takes a tile of 16 rows (tokens x the query heads of one key head) against a part of the pages; its
// four waves take pages in turn, each with its own running maximum and sum, and meet in the LDS at the end.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"
#include "epara_cache_device.h"
#include "epara_cache_host.h"

using namespace epara_cache;

namespace {

constexpr int NT = 256, WAVES = 4;
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ v8i join(v4i a, v4i b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ v4f mfma16(v8i a, v8i b, v4f c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

// What all kernels know about a workgroup's work.
struct work_item {
    epara_cache_attn_args a;
    epara_sequence s;
    int tile, part, head;        // rows tile * SIZE .., part of the tile's pages, key head
    int group, rows;             // query heads to a key head; rows = tokens x group
    int lo, hi, parts;           // the part's pages; parts of this tile
    int first_item;              // of the parts of this tile: where their counter is
    int stride;                  // from one part's item to the next
};

template <int SIZE>
__device__ __forceinline__ work_item find_work(const epara_cache_attn_args* __restrict__ args, const epara_sequence* __restrict__ seqs,
                                               const int32_t* __restrict__ first, int n_seqs, int part_pages, int item, int lane)
{
    work_item w;
    const int i = find_sequence(first, n_seqs, item, lane);
    w.s = seqs[i];
    w.a = args[w.s.service];
    w.group = w.a.heads / w.a.kv_heads;
    w.rows = w.s.rows * w.group;
    const int tiles = (w.rows + SIZE - 1) / SIZE, local = item - first[i];
    const int rest = local / w.a.kv_heads;
    w.head = local - rest * w.a.kv_heads;
    w.part = rest / tiles;
    const int back = rest - w.part * tiles;
    w.tile = tiles - 1 - back;                             // the tiles that see the most keys first
    const page_range r = pages_of_tokens(w.s, w.a.window, w.tile * SIZE / w.group, (min_of(w.rows, w.tile * SIZE + SIZE) - 1) / w.group);
    w.parts = (r.hi - r.lo + part_pages - 1) / part_pages;
    w.lo = r.lo + w.part * part_pages;
    w.hi = min_of(r.hi, w.lo + part_pages);
    w.stride = tiles * w.a.kv_heads;
    w.first_item = item - w.part * w.stride;
    return w;
}

// 16 bytes that another die has written or will read in this kernel: through to memory, past the dies' own caches.
__device__ __forceinline__ void put2(float* at, float a, float b)
{
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), (static_cast<unsigned long long>(__float_as_uint(b)) << 32) | __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ v2f get2(const float* at)
{
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return v2f{__uint_as_float(static_cast<uint32_t>(v)), __uint_as_float(static_cast<uint32_t>(v >> 32))};
}

// Sums with their maxima: (m, l, o) + (m2, l2, o2).  -inf: nothing seen yet.
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

template <int D>
struct few_lds {
    float o[WAVES][FEW_TILE][D + 4];
    float m[WAVES][FEW_TILE], l[WAVES][FEW_TILE];
    uint32_t last;
};

template <int D>
__device__ __forceinline__ void attend_few(const work_item& w, const int32_t* __restrict__ pages, uint32_t* counters, float* slots, char* lds_bytes, int item)
{
    few_lds<D>& lds = *reinterpret_cast<few_lds<D>*>(lds_bytes);
    constexpr int KS = D / 64;                             // 16-byte pieces of a key that a lane holds
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, q = lane >> 4;
    const epara_cache_attn_args& a = w.a;

    // ---- my row: a token and a query head
    const int row = min_of(w.tile * FEW_TILE + n, w.rows - 1), token = row / w.group, query_head = w.head * w.group + row - token * w.group;
    const int last_key = w.s.start + token, first_key = a.window > 0 ? last_key - a.window + 1 : 0;
    const int low_token = w.s.start + w.tile * FEW_TILE / w.group, high_token = w.s.start + (min_of(w.rows, w.tile * FEW_TILE + FEW_TILE) - 1) / w.group;
    const int end = w.s.start + w.s.rows;                  // tokens in the cache

    // ---- the query as two E4M3 numbers: dims 16 q .. and (heads of 128) 64 + 16 q ..
    v4i qhi[KS], qlo[KS];
    int q_exp;
    {
        const EPARA_GLOBAL char* src = (const EPARA_GLOBAL char*)a.Q + (static_cast<size_t>(w.s.first_row + token) * a.q_stride + static_cast<size_t>(query_head) * D) * 2;
        v4i raw[KS][2];
        float amax = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                raw[s][h] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + s * 128 + q * 32 + h * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(bf16_lo(raw[s][h][j])), fabsf(bf16_hi(raw[s][h][j]))));
            }
        amax = fmaxf(amax, __shfl_xor(amax, 16));
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        q_exp = block_exponent(amax);
        const float inv = exp2_int(-q_exp);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t u = raw[s][j >> 1][(j & 1) * 2], v = raw[s][j >> 1][(j & 1) * 2 + 1];
                int hi, lo;
                split_e4m3(bf16_lo(u) * inv, bf16_hi(u) * inv, bf16_lo(v) * inv, bf16_hi(v) * inv, hi, lo);
                qhi[s][j] = hi;
                qlo[s][j] = lo;
            }
    }
    // scales of the second operands: heads of 128 take hi and lo in two instructions, heads of 64 in the halves of one
    const int q_scale_hi = q_exp + 127, q_scale_lo = q_scale_hi - SPLIT_SHIFT, q_scale_both = q < 2 ? q_scale_hi : q_scale_lo;
    const int p_scale = q < 2 ? 127 : 127 - SPLIT_SHIFT;

    const size_t head_offset = static_cast<size_t>(w.head) * head_bytes(D);
    const size_t page_bytes = static_cast<size_t>(a.kv_heads) * head_bytes(D);
    v4i k[4][KS], v[D / 16];
    uint32_t scales = 0, scales_next = 0;
    auto base_of = [&](int page) { return (const EPARA_GLOBAL char*)a.codes + static_cast<size_t>(page) * page_bytes + head_offset + lane * 16; };
    auto load_keys = [&](const EPARA_GLOBAL char* base) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) k[t][s] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(base + (t * KS + s) * 1024);
    };
    auto load_values = [&](const EPARA_GLOBAL char* base) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) v[d] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(base + PAGE * D + d * 1024);
    };
    auto page_at = [&](int p) { return __builtin_amdgcn_readfirstlane(pages[w.s.first_page + p]); };
    auto scales_of = [&](int page) { return ((const EPARA_GLOBAL uint32_t*)a.scales)[static_cast<size_t>(page) * a.kv_heads + w.head]; };

    float m = -INFINITY, l = 0.f;
    v4f o[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] = v4f{0.f, 0.f, 0.f, 0.f};
    const float to_log2 = a.scale * LOG2E;
    const bool capped = a.softcap > 0.f;
    const float cap_in = capped ? 2.f * LOG2E * a.scale / a.softcap : 0.f, cap_out = a.softcap * LOG2E;

    int p = w.lo + wave;
    const EPARA_GLOBAL char* base = nullptr;
    if (p < w.hi) {
        const int page = page_at(p);
        base = base_of(page);
        scales = scales_of(page);
        load_keys(base);
        load_values(base);
    }
    for (; p < w.hi; p += WAVES) {
        const bool more = p + WAVES < w.hi;
        const EPARA_GLOBAL char* next = base;
        if (more) {
            const int page = page_at(p + WAVES);
            next = base_of(page);
            scales_next = scales_of(page);
        }
        // ---- scores
        v4f z[4];
        const int k_scale = (n < 8 ? scales : scales >> 8) & 0xff;          // row m of a tile: token 16 (m / 4) + .., so block m / 8
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const v4f zero = {0.f, 0.f, 0.f, 0.f};
            if constexpr (D == 128) {
                const v8i key = join(k[t][0], k[t][KS - 1]);
                z[t] = mfma16(key, join(qhi[0], qhi[KS - 1]), zero, k_scale, q_scale_hi);
                z[t] = mfma16(key, join(qlo[0], qlo[KS - 1]), z[t], k_scale, q_scale_lo);
            } else {
                z[t] = mfma16(join(k[t][0], k[t][0]), join(qhi[0], qlo[0]), zero, k_scale, q_scale_both);
            }
        }
        if (more) load_keys(next);
        const int at = p * PAGE + 16 * q;                  // my keys are at + 4 t + i
        if (capped) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)                // c tanh(z / c) = c (1 - 2 / (1 + e^(2 z / c)))
                    z[t][i] = cap_out - 2.f * cap_out * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z[t][i] * cap_in));
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[t][i] *= to_log2;
        }
        if (p * PAGE + PAGE - 1 > low_token || (a.window > 0 && p * PAGE <= high_token - a.window)) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = at + 4 * t + i;
                    if (key > last_key || key < first_key) z[t][i] = -INFINITY;
                }
        }
        // ---- running maximum and sum: mine are 16 keys of the page, the lanes n, n + 16, .. hold the others
        float top = m;
#pragma unroll
        for (int t = 0; t < 4; ++t) top = fmaxf(top, fmaxf(fmaxf(z[t][0], z[t][1]), fmaxf(z[t][2], z[t][3])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float ref = finite_or_zero(top), fade = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        l *= fade;
        // weights carry a factor of 2^8, which brings them into E4M3's upper range; it divides out at the end
        v4i hi, lo;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[t][i] = __builtin_amdgcn_exp2f(z[t][i] - ref + 8.f);
                l += z[t][i];
            }
            int h, r;
            split_e4m3(z[t][0], z[t][1], z[t][2], z[t][3], h, r);
            hi[t] = h;
            lo[t] = r;
        }
        // ---- values.  What lies behind the last token may be anything, a NaN too: cleared
        int v_scale = ((q & 1) ? scales >> 24 : scales >> 16) & 0xff;
        if (p * PAGE + PAGE > end) {
            if (p * PAGE + BLOCK * (q & 1) >= end) v_scale = 127;
            const int valid = end - at;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int mask = low_bytes(valid - 4 * j);
#pragma unroll
                for (int d = 0; d < D / 16; ++d) v[d][j] &= mask;
            }
        }
        const v8i weights = join(hi, lo);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            o[d] *= fade;
            o[d] = mfma16(join(v[d], v[d]), weights, o[d], v_scale, p_scale);
        }
        if (more) load_values(next);
        base = next;
        scales = scales_next;
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // ---- the four waves' sums: thread = (row, D / 16 columns)
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<v4f*>(&lds.o[wave][n][d * 16 + q * 4]) = o[d];
    if (q == 0) {
        lds.m[wave][n] = m;
        lds.l[wave][n] = l;
    }
    __syncthreads();
    constexpr int COLS = D / 16;
    const int r = tid >> 4, c = (tid & 15) * COLS;
    float mm = -INFINITY, ll = 0.f, oo[COLS];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mm = fmaxf(mm, lds.m[i][r]);
#pragma unroll
    for (int j = 0; j < COLS; ++j) oo[j] = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const float weight = __builtin_amdgcn_exp2f(lds.m[i][r] - finite_or_zero(mm));
        ll += weight * lds.l[i][r];
#pragma unroll
        for (int j = 0; j < COLS; ++j) oo[j] += weight * lds.o[i][r][c + j];
    }
    const int out_row = w.tile * FEW_TILE + r;
    if (w.parts > 1) {                                     // the part's sums go to its slot; who ends last adds up all of them, in order
        float* slot = slots + static_cast<size_t>(item) * FEW_TILE * SLOT_FLOATS + r * SLOT_FLOATS;
        if (out_row < w.rows) {
#pragma unroll
            for (int j = 0; j < COLS; j += 2) put2(slot + c + j, oo[j], oo[j + 1]);
            if (c == 0) put2(slot + 128, mm, ll);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) lds.last = __hip_atomic_fetch_add(counters + w.first_item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<uint32_t>(w.parts - 1);
        __syncthreads();
        if (!lds.last) return;
        if (tid == 0) __hip_atomic_store(counters + w.first_item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (out_row >= w.rows) return;
        mm = -INFINITY;
        ll = 0.f;
#pragma unroll
        for (int j = 0; j < COLS; ++j) oo[j] = 0.f;
        const float* from = slots + static_cast<size_t>(w.first_item) * FEW_TILE * SLOT_FLOATS + r * SLOT_FLOATS;
        for (int i = 0; i < w.parts; ++i, from += static_cast<size_t>(w.stride) * FEW_TILE * SLOT_FLOATS) {
            const v2f ml = get2(from + 128);
            const float both = fmaxf(mm, ml[0]), keep = __builtin_amdgcn_exp2f(mm - finite_or_zero(both)), add = __builtin_amdgcn_exp2f(ml[0] - finite_or_zero(both));
            mm = both;
            ll = ll * keep + ml[1] * add;
#pragma unroll
            for (int j = 0; j < COLS; j += 2) {
                const v2f x = get2(from + c + j);
                oo[j] = oo[j] * keep + x[0] * add;
                oo[j + 1] = oo[j + 1] * keep + x[1] * add;
            }
        }
    }
    if (out_row >= w.rows) return;
    const float inv = mm == -INFINITY ? 0.f : 1.f / ll;    // a row that sees no key: zeros
    const int out_token = out_row / w.group, out_head = w.head * w.group + out_row - out_token * w.group;
    EPARA_GLOBAL char* dst = (EPARA_GLOBAL char*)a.O + (static_cast<size_t>(w.s.first_row + out_token) * a.o_stride + static_cast<size_t>(out_head) * D + c) * 2;
    if constexpr (D == 128) {
        *reinterpret_cast<EPARA_GLOBAL v4i*>(dst) = v4i{static_cast<int>(pack_bf16(oo[0] * inv, oo[1] * inv)), static_cast<int>(pack_bf16(oo[2] * inv, oo[3] * inv)),
                                                        static_cast<int>(pack_bf16(oo[COLS - 4] * inv, oo[COLS - 3] * inv)), static_cast<int>(pack_bf16(oo[COLS - 2] * inv, oo[COLS - 1] * inv))};
    } else {
        typedef unsigned int v2u __attribute__((ext_vector_type(2)));
        *reinterpret_cast<EPARA_GLOBAL v2u*>(dst) = v2u{pack_bf16(oo[0] * inv, oo[1] * inv), pack_bf16(oo[2] * inv, oo[3] * inv)};
    }
}

__global__ __launch_bounds__(NT, 2) void attend_few_kernel(const epara_cache_attn_args* __restrict__ args, const epara_sequence* __restrict__ seqs,
                                                          const int32_t* __restrict__ pages, const int32_t* __restrict__ first, int n_seqs, int part_pages,
                                                          uint32_t* counters, float* slots)
{
    __shared__ __attribute__((aligned(16))) char lds[sizeof(few_lds<128>)];
    const int item = blockIdx.x;
    const work_item w = find_work<FEW_TILE>(args, seqs, first, n_seqs, part_pages, item, threadIdx.x & 63);
    if (w.part > 0 && w.part >= w.parts) return;           // this tile has fewer parts than the sequence's longest
    if (w.a.head_dim == 128) attend_few<128>(w, pages, counters, slots, lds, item);
    else                     attend_few<64>(w, pages, counters, slots, lds, item);
}

}  // namespace

extern "C" int32_t epara_cache_attention(const epara_cache_attn_launch* launch, void* stream)
{
    if (!launch) return EPARA_ERR_NULL;
    const epara_cache_attn_launch& l = *launch;
    bool cut[2];
    if (const int32_t rc = epara_check_attn_call(l, cut)) return rc;
    if (l.plan.n_items[0] + l.plan.n_items[1] == 0 || l.table.n_seqs == 0) return EPARA_OK;
    if (!l.d_args || !l.d_first) return EPARA_ERR_NULL;
    uint32_t* counters = static_cast<uint32_t*>(l.d_workspace);
    float* slots = reinterpret_cast<float*>(static_cast<char*>(l.d_workspace) + epara_attn_counter_bytes(l.plan.n_items));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (l.plan.n_items[0] > 0)
        hipLaunchKernelGGL(attend_few_kernel, dim3(static_cast<unsigned>(l.plan.n_items[0])), dim3(NT), 0, s, l.d_args, l.table.d_seqs, l.table.d_pages, l.d_first,
                           l.table.n_seqs, l.plan.part_pages[0], counters, slots);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}
