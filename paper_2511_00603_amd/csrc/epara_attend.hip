// libepara: causal attention of new tokens over a paged cache in 8 bits (the decode and prefill services' attention).
//
//   o = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m),   z_j = scale q . k_j (capped: c tanh(z_j / c)),   m = max_j z_j
//
// Keys and values go from memory into the matrix cores as they lie in the cache, E4M3 codes with E8M0 scales: nothing is
// converted.  A query is the sum of two E4M3 numbers, q = hi + lo / 16 with its own power of two, which holds all 8
// significant bits of a bf16; so is a weight p = exp(z - m).  Products of 8-bit operands run at twice the rate of bf16
// ones, so the two products cost what one in bf16 would.  (Weights rounded to bf16 would be 2.7 times coarser.)
//
// The matrix cores' scales also carry the running maximum.  The weights of a page are taken relative to the page's own largest score,
// rounded up to an integer r in units of log 2: p = 2^(z - r), and enter the product with the scale 2^(r - M), where M is the
// row's reference.  M only has to be near enough for fp32 (MAX_ABOVE), so sums are almost never rescaled, and the weights of a page
// keep their 8 bits however far they lie under the row's maximum (thousands of keys that share what one strong key leaves).
//
// Both products are written transposed, so that what the first leaves in a lane is what the second wants there:
//   S^T = K Q^T   A = keys x dims, B = dims x rows;   O^T = V^T P^T   A = dims x tokens, B = tokens x rows
// For this the cache holds keys and values in the order it does.  In an instruction with a contraction of length C over 64 / N
// groups of lanes (N rows of B), a lane's first 16 bytes are elements 16 g .. 16 g + 15 of it and its second 16 bytes elements
// C / 2 + 16 g ..; elements 32 b .. 32 b + 31 take their scale from the lanes of group b.
//
//   few rows (a workgroup has a tile of 16): 16x16x128.  Lane (n = lane % 16, q = lane / 16) gets from the four tiles t of S^T of a page the
//     scores of row n with the keys 16 q + 4 t + 0 .. 3: the 16 tokens of a 16-byte chunk of a dim's values.  O^T takes hi in the first half
//     and lo in the second against the same values.  Pages go from memory to registers, the four waves take them in turn and meet in the LDS at the end.
//   many rows (a tile of 128, 32 to a wave): 32x32x64.  Lane (n = lane % 32, h = lane / 32) gets from the two tiles u of S^T of a page the scores of row n
//     with the keys 32 u + 16 h + 0 .. 15, again a chunk.  Pages go to the LDS by direct loads, where all four waves read them.
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

template <bool V> struct flag { static constexpr bool value = V; };
constexpr float NOTHING = -1e30f;                          // reference of a row that has seen no key
constexpr float MAX_ABOVE = 16.f;                          // a page's reference may exceed the row's by that much (sums then grow to 2^(16 + 8) of a value)
constexpr float LIFT = 8.f;                                // weights are taken as 2^(8 + z - r) <= 2^8: E4M3's upper range; it divides out at the end

struct row_state { float ref, sum; };                      // M, and the sum of the weights relative to it (of this lane's keys)

// The page's reference for a row whose largest score here is `top` (units of log 2; -inf: it sees none of them), and whether the row's own
// has to be raised.
__device__ __forceinline__ float page_reference(float top) { return top == -INFINITY ? NOTHING : __builtin_ceilf(top); }
__device__ __forceinline__ float raise_reference(row_state& s, float ref)
{
    const float to = fmaxf(s.ref, ref), f = __builtin_amdgcn_exp2f(s.ref - to);
    s.ref = to;
    s.sum *= f;
    return f;
}
// Scale byte of the page's weights, hi part.
__device__ __forceinline__ int weight_scale(const row_state& s, float ref) { return 127 + static_cast<int>(fmaxf(ref - s.ref, -120.f)); }

__device__ __forceinline__ float capped_score(float z, float in, float out)      // c tanh(z / c) = c (1 - 2 / (1 + e^(2 z / c))), in units of log 2
{
    return out - 2.f * out * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * in));
}

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
    const int p_shift = q < 2 ? 0 : SPLIT_SHIFT;

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

    row_state state = {NOTHING, 0.f};
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
        float unit = to_log2;                              // of a score, to log 2
        if (capped) {
            unit = 1.f;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[t][i] = capped_score(z[t][i], cap_in, cap_out);
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
        // ---- the row's largest score here: mine are 16 keys of the page, the lanes n, n + 16, .. hold the others
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t) top = fmaxf(top, fmaxf(fmaxf(z[t][0], z[t][1]), fmaxf(z[t][2], z[t][3])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float ref = page_reference(top * unit);
        if (__ballot(ref > state.ref + MAX_ABOVE)) {
            const float f = raise_reference(state, ref);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d] *= f;
        }
        const float lift = LIFT - ref;
        float sum = 0.f;
        v4i hi, lo;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[t][i] = __builtin_amdgcn_exp2f(fmaf(z[t][i], unit, lift));
                sum += z[t][i];
            }
            int h, r;
            split_e4m3(z[t][0], z[t][1], z[t][2], z[t][3], h, r);
            hi[t] = h;
            lo[t] = r;
        }
        state.sum = fmaf(sum, __builtin_amdgcn_exp2f(ref - state.ref), state.sum);
        const int p_scale = weight_scale(state, ref) - p_shift;
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
        for (int d = 0; d < D / 16; ++d) o[d] = mfma16(join(v[d], v[d]), weights, o[d], v_scale, p_scale);
        if (more) load_values(next);
        base = next;
        scales = scales_next;
    }
    state.sum += __shfl_xor(state.sum, 16);
    state.sum += __shfl_xor(state.sum, 32);

    // ---- the four waves' sums: thread = (row, D / 16 columns)
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<v4f*>(&lds.o[wave][n][d * 16 + q * 4]) = o[d];
    if (q == 0) {
        lds.m[wave][n] = state.ref;
        lds.l[wave][n] = state.sum;
    }
    __syncthreads();
    constexpr int COLS = D / 16;
    const int r = tid >> 4, c = (tid & 15) * COLS;
    float mm = NOTHING, ll = 0.f, oo[COLS];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mm = fmaxf(mm, lds.m[i][r]);
#pragma unroll
    for (int j = 0; j < COLS; ++j) oo[j] = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const float weight = __builtin_amdgcn_exp2f(lds.m[i][r] - mm);
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
        mm = NOTHING;
        ll = 0.f;
#pragma unroll
        for (int j = 0; j < COLS; ++j) oo[j] = 0.f;
        const float* from = slots + static_cast<size_t>(w.first_item) * FEW_TILE * SLOT_FLOATS + r * SLOT_FLOATS;
        for (int i = 0; i < w.parts; ++i, from += static_cast<size_t>(w.stride) * FEW_TILE * SLOT_FLOATS) {
            const v2f ml = get2(from + 128);
            const float both = fmaxf(mm, ml[0]), keep = __builtin_amdgcn_exp2f(mm - both), add = __builtin_amdgcn_exp2f(ml[0] - both);
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
    const float inv = mm == NOTHING ? 0.f : 1.f / ll;    // a row that sees no key: zeros
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

// ---- many rows -------------------------------------------------------------------------------------------------

constexpr int RING = 3;                                    // pages in the LDS: one is read, two are on their way
typedef __attribute__((address_space(3))) char* ldsptr;
typedef const __attribute__((address_space(4))) uint32_t* constant_words;
typedef unsigned int v2u __attribute__((ext_vector_type(2)));

__device__ __forceinline__ v16f mfma32(v8i a, v8i b, v16f c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}
__device__ __forceinline__ v4i lds16(ldsptr at) { return *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(at); }

template <int D>
__device__ __forceinline__ void attend_many(const work_item& w, const int32_t* __restrict__ pages, uint32_t* counters, char* slots, ldsptr ring, int item)
{
    constexpr int KS = D / 64, DT = D / 32;                // steps of 64 dims, tiles of 32 dims
    constexpr int PAGE_BYTES = 2 * PAGE * D, LOADS = PAGE_BYTES / 1024 / WAVES;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const epara_cache_attn_args& a = w.a;

    const int first_row = w.tile * MANY_TILE + wave * 32;  // of my wave
    const bool live = first_row < w.rows;
    const int row = min_of(first_row + n, w.rows - 1), token = row / w.group, query_head = w.head * w.group + row - token * w.group;
    const int last_key = w.s.start + token, first_key = a.window > 0 ? last_key - a.window + 1 : 0;
    const int low_token = w.s.start + min_of(first_row, w.rows - 1) / w.group, high_token = w.s.start + (min_of(w.rows, first_row + 32) - 1) / w.group;
    const int end = w.s.start + w.s.rows;

    // ---- the query: its dims 64 p + 32 h + 16 s ..; hi and lo
    v8i qhi[KS], qlo[KS];
    int q_scale;
    {
        const EPARA_GLOBAL char* src = (const EPARA_GLOBAL char*)a.Q + (static_cast<size_t>(w.s.first_row + token) * a.q_stride + static_cast<size_t>(query_head) * D) * 2;
        v4i raw[KS][4];
        float amax = 0.f;
#pragma unroll
        for (int p = 0; p < KS; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                raw[p][i] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + p * 128 + h * 64 + i * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(bf16_lo(raw[p][i][j])), fabsf(bf16_hi(raw[p][i][j]))));
            }
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        const int e = block_exponent(amax);
        q_scale = e + 127;
        const float inv = exp2_int(-e);
#pragma unroll
        for (int p = 0; p < KS; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t u = raw[p][i][2 * j], v = raw[p][i][2 * j + 1];
                    int hi, lo;
                    split_e4m3(bf16_lo(u) * inv, bf16_hi(u) * inv, bf16_lo(v) * inv, bf16_hi(v) * inv, hi, lo);
                    qhi[p][2 * i + j] = hi;
                    qlo[p][2 * i + j] = lo;
                }
    }

    // ---- pages to the LDS: a wave brings a quarter of each
    const constant_words table = (constant_words)(pages + w.s.first_page);
    const constant_words scales = (constant_words)a.scales;
    const size_t page_bytes = static_cast<size_t>(a.kv_heads) * PAGE_BYTES;
    auto fetch = [&](int p, int slot) -> uint32_t {        // returns the page's scales
        const uint32_t page = table[p];
        const char* base = static_cast<const char*>(a.codes) + page * page_bytes + static_cast<size_t>(w.head) * PAGE_BYTES;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, PAGE_BYTES, 0x00020000);
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(ring + slot * PAGE_BYTES + (wave * LOADS + i) * 1024), 16,
                                                     lane * 16, (wave * LOADS + i) * 1024, 0, 0);
        return scales[static_cast<size_t>(page) * a.kv_heads + w.head];
    };

    row_state state = {NOTHING, 0.f};
    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    const float to_log2 = a.scale * LOG2E;
    const bool capped = a.softcap > 0.f;
    const float cap_in = capped ? 2.f * LOG2E * a.scale / a.softcap : 0.f, cap_out = a.softcap * LOG2E;
    // where my chunks lie in a page: keys, tile u and step p: rows of the tile are the keys 32 u + 16 (row / 4 % 2) + 4 (row / 8) + row % 4
    const int key_at = ((n >> 3) * (D / 16) + 2 * h) * 256 + (n & 7) * 16, value_at = PAGE * D + ((n >> 4) * 4 + h) * 256 + (n & 15) * 16;

    uint32_t sc[2] = {0, 0};                               // scales of the page that is read and of the next one
    if (w.lo < w.hi) sc[0] = fetch(w.lo, 0);
    if (w.lo + 1 < w.hi) sc[1] = fetch(w.lo + 1, 1);
    int slot = 0;
    for (int p = w.lo; p < w.hi; ++p) {
        // page p is here once all but the loads of page p + 1 have arrived, everybody's once all waves are past this point; page p - 1 has been read then
        // (the LDS reads of page p - 1 have returned before anybody's loads may overwrite it: lgkmcnt)
        if (p + 1 < w.hi) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LOADS) : "memory");
        else              asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
        const uint32_t now = sc[0];
        sc[0] = sc[1];
        if (p + 2 < w.hi) sc[1] = fetch(p + 2, slot + 2 >= RING ? slot + 2 - RING : slot + 2);
        ldsptr here = ring + slot * PAGE_BYTES;
        slot = slot + 1 == RING ? 0 : slot + 1;
        if (!live || p * PAGE > high_token || (a.window > 0 && p * PAGE + PAGE <= low_token - a.window + 1)) continue;

        // ---- scores
        v16f z[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k_scale = now >> (8 * u) & 0xff;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[u][i] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const v8i key = join(lds16(here + key_at + u * 128 + s * 1024), lds16(here + key_at + u * 128 + s * 1024 + 256));
                z[u] = mfma32(key, qhi[s], z[u], k_scale, q_scale);
                z[u] = mfma32(key, qlo[s], z[u], k_scale, q_scale - SPLIT_SHIFT);
            }
        }
        float unit = to_log2;
        if (capped) {
            unit = 1.f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[u][i] = capped_score(z[u][i], cap_in, cap_out);
        }
        if (p * PAGE + PAGE - 1 > low_token || (a.window > 0 && p * PAGE <= high_token - a.window)) {
            const int last = last_key - p * PAGE - 16 * h, from = first_key - p * PAGE - 16 * h;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * u + i > last || 32 * u + i < from) z[u][i] = -INFINITY;
        }
        // ---- weights
        float top = fmaxf(z[0][0], z[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, fmaxf(z[0][i], z[1][i]));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float ref = page_reference(top * unit);
        if (__ballot(ref > state.ref + MAX_ABOVE)) {
            const float f = raise_reference(state, ref);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        const float lift = LIFT - ref;
        float sum[2] = {0.f, 0.f};
        v8i hi, lo;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = __builtin_amdgcn_exp2f(fmaf(z[u][4 * j + i], unit, lift));
                    sum[u] += x[i];
                }
                int a4, b4;
                split_e4m3(x[0], x[1], x[2], x[3], a4, b4);
                hi[4 * u + j] = a4;
                lo[4 * u + j] = b4;
            }
        state.sum = fmaf(sum[0] + sum[1], __builtin_amdgcn_exp2f(ref - state.ref), state.sum);
        const int p_scale = weight_scale(state, ref);
        // ---- values.  What lies behind the last token may be anything, a NaN too: cleared
        int v_scale = now >> (16 + 8 * h) & 0xff;
        const bool ragged = p * PAGE + PAGE > end;
        if (ragged && p * PAGE + BLOCK * h >= end) v_scale = 127;
        auto add_values = [&](auto clear_tag) {
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                v4i v0 = lds16(here + value_at + d * 2048), v1 = lds16(here + value_at + d * 2048 + 512);
                if constexpr (decltype(clear_tag)::value) {
                    const int valid = end - p * PAGE - 16 * h;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v0[j] &= low_bytes(valid - 4 * j);
                        v1[j] &= low_bytes(valid - BLOCK - 4 * j);
                    }
                }
                const v8i value = join(v0, v1);
                o[d] = mfma32(value, hi, o[d], v_scale, p_scale);
                o[d] = mfma32(value, lo, o[d], v_scale, p_scale - SPLIT_SHIFT);
            }
        };
        if (ragged) add_values(flag<true>{}); else add_values(flag<false>{});
    }
    state.sum += __shfl_xor(state.sum, 32);

    if (w.parts > 1) {
        // a slot: per wave 1 KiB for each quad of registers, then the references and sums
        char* slot_at = slots + static_cast<size_t>(item) * MANY_TILE * SLOT_FLOATS * 4;
        __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(slot_at, 0, MANY_TILE * SLOT_FLOATS * 4, 0x00020000);
        constexpr int WAVE_BYTES = 32 * SLOT_FLOATS * 4;
        const int at = wave * WAVE_BYTES + lane * 16;
        if (live) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, v4f{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]}), rsrc, at, (d * 4 + j) * 1024, 16);   // 16: device scope
            if (h == 0) put2(reinterpret_cast<float*>(slot_at + wave * WAVE_BYTES + 16384) + 2 * n, state.ref, state.sum);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        __attribute__((address_space(3))) uint32_t* box = (__attribute__((address_space(3))) uint32_t*)ring;
        if (tid == 0) *box = __hip_atomic_fetch_add(counters + w.first_item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (*box != static_cast<uint32_t>(w.parts - 1)) return;
        if (tid == 0) __hip_atomic_store(counters + w.first_item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (!live) return;
        state = {NOTHING, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        for (int i = 0; i < w.parts; ++i) {
            char* from = slots + (static_cast<size_t>(w.first_item) + static_cast<size_t>(i) * w.stride) * MANY_TILE * SLOT_FLOATS * 4;
            rsrc = __builtin_amdgcn_make_buffer_rsrc(from, 0, MANY_TILE * SLOT_FLOATS * 4, 0x00020000);
            const v2f ml = get2(reinterpret_cast<const float*>(from + wave * WAVE_BYTES + 16384) + 2 * n);
            v4i in[DT][4];
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) in[d][j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, (d * 4 + j) * 1024, 16);
            const float both = fmaxf(state.ref, ml[0]), keep = __builtin_amdgcn_exp2f(state.ref - both), add = __builtin_amdgcn_exp2f(ml[0] - both);
            state.ref = both;
            state.sum = state.sum * keep + ml[1] * add;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const v4f x = __builtin_bit_cast(v4f, in[d][j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[d][4 * j + e] = o[d][4 * j + e] * keep + x[e] * add;
                }
        }
    }
    if (!live) return;
    // ---- rows out.  Lane (n, h) holds dims 32 d + 8 j + 4 h + 0 .. 3; two quads change places between the halves of the wave, so that a lane stores 8 in a row
    const float inv = state.ref == NOTHING ? 0.f : 1.f / state.sum;
    const bool mine = first_row + n < w.rows;
    EPARA_GLOBAL char* dst = (EPARA_GLOBAL char*)a.O + (static_cast<size_t>(w.s.first_row + token) * a.o_stride + static_cast<size_t>(query_head) * D) * 2;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            v4i out;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t x = pack_bf16(o[d][4 * j + 2 * e] * inv, o[d][4 * j + 2 * e + 1] * inv), y = pack_bf16(o[d][4 * j + 4 + 2 * e] * inv, o[d][4 * j + 5 + 2 * e] * inv);
                const v2u both = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(x, y, false, false));
                out[e] = static_cast<int>(both[0]);
                out[2 + e] = static_cast<int>(both[1]);
            }
            if (mine) *reinterpret_cast<EPARA_GLOBAL v4i*>(dst + d * 64 + j * 16 + h * 16) = out;
        }
}

__global__ __launch_bounds__(NT, 2) void attend_many_kernel(const epara_cache_attn_args* __restrict__ args, const epara_sequence* __restrict__ seqs,
                                                           const int32_t* __restrict__ pages, const int32_t* __restrict__ first, int n_seqs, int part_pages,
                                                           uint32_t* counters, char* slots)
{
    __shared__ __attribute__((aligned(1024))) char ring[RING * 2 * PAGE * 128];
    const int item = blockIdx.x;
    const work_item w = find_work<MANY_TILE>(args, seqs, first, n_seqs, part_pages, item, threadIdx.x & 63);
    if (w.part > 0 && w.part >= w.parts) return;
    if (w.a.head_dim == 128) attend_many<128>(w, pages, counters, slots, (ldsptr)ring, item);
    else                     attend_many<64>(w, pages, counters, slots, (ldsptr)ring, item);
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
    char* slots = static_cast<char*>(l.d_workspace) + epara_attn_counter_bytes(l.plan.n_items);
    char* many_slots = slots + (cut[0] ? static_cast<size_t>(l.plan.n_items[0]) * FEW_TILE * SLOT_FLOATS * 4 : 0);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (l.plan.n_items[1] > 0)
        hipLaunchKernelGGL(attend_many_kernel, dim3(static_cast<unsigned>(l.plan.n_items[1])), dim3(NT), 0, s, l.d_args, l.table.d_seqs, l.table.d_pages,
                           l.d_first + l.table.n_seqs + 1, l.table.n_seqs, l.plan.part_pages[1], counters + l.plan.n_items[0], many_slots);
    if (l.plan.n_items[0] > 0)
        hipLaunchKernelGGL(attend_few_kernel, dim3(static_cast<unsigned>(l.plan.n_items[0])), dim3(NT), 0, s, l.d_args, l.table.d_seqs, l.table.d_pages, l.d_first,
                           l.table.n_seqs, l.plan.part_pages[0], counters, reinterpret_cast<float*>(slots));
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}
