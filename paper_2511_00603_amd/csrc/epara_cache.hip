// libepara: new tokens into a paged cache in 8 bits (rotary positions on the way), and copies of its pages.
//
// Both are bound by memory.  Append: a wave takes the new tokens of one block (32 tokens that share a scale) and key head: its
// keys and values are read once, stay in registers as fp32 until the block's largest value is known, and leave as whole
// 16-byte chunks of the page; or a few rows x heads of the queries, with the angles of a row read once for its heads.  Copy: a workgroup per page and head.
// Measured: prompts of 6 requests (0.47 GB in and out) 116 us, 4.1 TB/s at two waves per SIMD; a token of 105 requests 8 us,
// a chain of dependent trips to memory; 3001 pages of 128 KiB copied in 153 us, 5.1 TB/s, as fast as a plain copy of this size.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"
#include "epara_cache_device.h"
#include "epara_cache_host.h"

using namespace epara_cache;

namespace {

constexpr int NT = 256;

__device__ __forceinline__ float finite_abs(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }       // NaN and infinities do not count
__device__ __forceinline__ float nan_to_zero(float x) { return x == x ? x : 0.f; }

// Four codes times 2^shift, rounded again.
__device__ __forceinline__ int rescaled(int codes, float factor)
{
    const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    return static_cast<int>(to_e4m3(a[0] * factor, a[1] * factor, b[0] * factor, b[1] * factor));
}

// cos and sin of N pairs from `pair` on for one row: its position on the pairs' axes.
struct row_angles {
    const EPARA_GLOBAL float* table;     // [n_positions, half, 2]
    int at[3];
    int a0, a1;                          // pairs of axis 0, of axes 0 and 1
    int half;
};
__device__ __forceinline__ row_angles angles_of(const epara_append_args& a, int row, int position)
{
    row_angles r;
    r.table = (const EPARA_GLOBAL float*)a.rotary;
    r.half = a.head_dim / 2;
    r.a0 = a.axis_pairs[0];
    r.a1 = r.a0 + a.axis_pairs[1];
    const EPARA_GLOBAL int32_t* p = (const EPARA_GLOBAL int32_t*)a.positions;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const int at = p ? p[static_cast<size_t>(row) * 3 + i] : position;
        r.at[i] = max_of(0, min_of(at, a.n_positions - 1));
    }
    return r;
}
template <int N>
__device__ __forceinline__ void load_angles(const row_angles& r, int pair, float* cs, float* sn)
{
    if (r.at[0] == r.at[1] && r.at[1] == r.at[2]) {
        const EPARA_GLOBAL float* src = r.table + (static_cast<size_t>(r.at[0]) * r.half + pair) * 2;
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            const v4f v = *reinterpret_cast<const EPARA_GLOBAL v4f*>(src + 2 * j);
            cs[j] = v[0];
            sn[j] = v[1];
            cs[j + 1] = v[2];
            sn[j + 1] = v[3];
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = pair + j, at = i < r.a0 ? r.at[0] : i < r.a1 ? r.at[1] : r.at[2];
            const v2f v = *reinterpret_cast<const EPARA_GLOBAL v2f*>(r.table + (static_cast<size_t>(at) * r.half + i) * 2);
            cs[j] = v[0];
            sn[j] = v[1];
        }
    }
}

__device__ __forceinline__ void unpack8(const v4i& v, float* x)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = bf16_lo(static_cast<uint32_t>(v[j]));
        x[2 * j + 1] = bf16_hi(static_cast<uint32_t>(v[j]));
    }
}

// ---- the new tokens of one block, one key head
template <int D>
__device__ __forceinline__ void append_block(const epara_append_args& a, const epara_sequence& s, const int32_t* __restrict__ pages, int block, int head, int lane)
{
    constexpr int CD = D / 16;                             // chunks of a key
    constexpr int CP = CD / 2;                             // pairs of chunks (c, c + CP) that turn together: lanes of a token
    constexpr int PASSES = BLOCK * CP / 64;                // 2 or 1
    constexpr int VT = D == 128 ? 32 : 16;                 // tokens of a lane's two dims
    const int from = max_of(s.start, 0), end = s.start + s.rows;
    const int first_token = block * BLOCK;                 // position of the block's token 0
    const int had = max_of(from - first_token, 0), upto = min_of(end - first_token, BLOCK);      // its tokens [0, had) are old, [had, upto) new
    const int page = __builtin_amdgcn_readfirstlane(pages[s.first_page + first_token / PAGE]), half = block & 1;
    EPARA_GLOBAL char* keys = (EPARA_GLOBAL char*)a.codes + static_cast<size_t>(page) * a.kv_heads * head_bytes(D) + static_cast<size_t>(head) * head_bytes(D);
    EPARA_GLOBAL char* values = keys + PAGE * D;
    EPARA_GLOBAL uint8_t* scales = (EPARA_GLOBAL uint8_t*)a.scales + (static_cast<size_t>(page) * a.kv_heads + head) * 4;
    const EPARA_GLOBAL char* qkv = (const EPARA_GLOBAL char*)a.QKV;
    auto row_of = [&](int token) { return s.first_row + first_token + token - s.start; };
    auto source = [&](int token, int which) {
        return qkv + (static_cast<size_t>(row_of(token)) * a.qkv_stride + static_cast<size_t>(a.heads + which * a.kv_heads + head) * D) * 2;
    };
    const int old_k = scales[half] - 127, old_v = scales[2 + half] - 127;

    // ---- values: two dims of a lane, token by token; what the chunks hold already, if there are old tokens
    const int dim = D == 128 ? 2 * lane : 2 * (lane & 31), v_first = D == 128 ? 0 : (lane >> 5) * 16;
    uint32_t v[VT];
#pragma unroll
    for (int i = 0; i < VT; ++i) {
        const int token = v_first + i;
        v[i] = 0;
        if (token >= had && token < upto) v[i] = *reinterpret_cast<const EPARA_GLOBAL uint32_t*>(source(token, 1) + dim * 2);
    }
    // ---- keys: 16 dims of a token and their partners
    const int cp = lane & (CP - 1);
    float x[PASSES][32];
    int token_of[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int i = lane / CP;                           // which of a pass's tokens: 16 or 32 of them; neighbours lie in neighbouring chunks
        const int t = (D == 128 ? 2 * p : 0) + (i >> 3), token = 16 * ((i >> 2) & 1) + 4 * t + (i & 3);
        token_of[p] = token;
#pragma unroll
        for (int j = 0; j < 32; ++j) x[p][j] = 0.f;
        if (token >= had && token < upto) {
            const EPARA_GLOBAL char* src = source(token, 0) + cp * 32;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const v4i raw = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + h * D + c * 16);
                    unpack8(raw, &x[p][h * 16 + c * 8]);
                }
            if (a.rotary) {
                float cs[16], sn[16];
                load_angles<16>(angles_of(a, row_of(token), first_token + token), cp * 16, cs, sn);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float u = x[p][j], w = x[p][16 + j];
                    x[p][j] = u * cs[j] - w * sn[j];
                    x[p][16 + j] = w * cs[j] + u * sn[j];
                }
            }
        }
    }
    // ---- largest values, and tokens with a NaN
    float top_k = 0.f, top_v = 0.f;
    bool nan_k[PASSES], nan_v = false;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        nan_k[p] = false;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            top_k = fmaxf(top_k, finite_abs(x[p][j]));
            nan_k[p] |= x[p][j] != x[p][j];
        }
    }
#pragma unroll
    for (int i = 0; i < VT; ++i) {
        top_v = fmaxf(top_v, fmaxf(finite_abs(bf16_lo(v[i])), finite_abs(bf16_hi(v[i]))));
        nan_v |= bf16_lo(v[i]) != bf16_lo(v[i]) || bf16_hi(v[i]) != bf16_hi(v[i]);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        top_k = fmaxf(top_k, __shfl_xor(top_k, d));
        top_v = fmaxf(top_v, __shfl_xor(top_v, d));
    }
    uint32_t broken = 0;                                   // tokens whose key is held as NaN
    bool any_nan = nan_v;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) any_nan |= nan_k[p];
    if (__ballot(any_nan)) {
#pragma unroll
        for (int i = 0; i < VT; ++i) {
            const unsigned long long who = __ballot(bf16_lo(v[i]) != bf16_lo(v[i]) || bf16_hi(v[i]) != bf16_hi(v[i]));
            if constexpr (D == 128) broken |= who ? 1u << i : 0u;
            else broken |= (static_cast<uint32_t>(who) ? 1u << i : 0u) | (static_cast<uint32_t>(who >> 32) ? 1u << (16 + i) : 0u);
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            uint32_t mine = nan_k[p] ? 1u << token_of[p] : 0u;
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) mine |= __shfl_xor(mine, d);
            broken |= mine;
        }
    }
    int e_k = block_exponent(top_k), e_v = block_exponent(top_v);
    const bool grow_k = had > 0 && e_k > old_k, grow_v = had > 0 && e_v > old_v;
    if (had > 0) {
        e_k = max_of(e_k, old_k);
        e_v = max_of(e_v, old_v);
    }
    e_k = min_of(e_k, 120);                                // a byte that no call has written may say more
    e_v = min_of(e_v, 120);
    const float inv_k = exp2_int(-e_k), inv_v = exp2_int(-e_v);

    // ---- keys out: chunk (t, c, m)
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int token = token_of[p], t = (token >> 2) & 3, m = 4 * (2 * half + (token >> 4)) + (token & 3);
        EPARA_GLOBAL char* at = keys + ((t * CD + cp) * 16 + m) * 16;
        if (token >= had && token < upto) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v4i out;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float* y = &x[p][h * 16 + 4 * j];
                    out[j] = static_cast<int>(to_e4m3(clamp448(nan_to_zero(y[0]) * inv_k), clamp448(nan_to_zero(y[1]) * inv_k), clamp448(nan_to_zero(y[2]) * inv_k), clamp448(nan_to_zero(y[3]) * inv_k)));
                }
                if (h == 0 && cp == 0 && (broken >> token & 1)) out[0] = (out[0] & ~0xff) | 0x7f;
                *reinterpret_cast<EPARA_GLOBAL v4i*>(at + h * CP * 256) = out;
            }
        } else if (grow_k && token < had) {
            const float factor = __builtin_amdgcn_exp2f(static_cast<float>(old_k - e_k));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v4i out = *reinterpret_cast<EPARA_GLOBAL v4i*>(at + h * CP * 256);
#pragma unroll
                for (int j = 0; j < 4; ++j) out[j] = rescaled(out[j], factor);
                *reinterpret_cast<EPARA_GLOBAL v4i*>(at + h * CP * 256) = out;
            }
        }
    }
    // ---- values out: chunk (dim, 16 tokens)
    const float factor_v = __builtin_amdgcn_exp2f(static_cast<float>(old_v - e_v));
#pragma unroll
    for (int c = 0; c < VT / 16; ++c) {
        const int chunk_first = v_first + 16 * c;          // its first token in the block
        if (upto <= chunk_first || (!grow_v && had >= chunk_first + 16)) continue;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            EPARA_GLOBAL char* at = values + (((dim + d) / 16 * 4 + 2 * half + chunk_first / 16) * 16 + (dim + d) % 16) * 16;
            v4i out;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t u = v[16 * c + 4 * j + i];
                    y[i] = clamp448(nan_to_zero(d ? bf16_hi(u) : bf16_lo(u)) * inv_v);
                }
                out[j] = static_cast<int>(to_e4m3(y[0], y[1], y[2], y[3]));
            }
            if (had > chunk_first || upto < chunk_first + 16) {        // old tokens keep their places, and so does what lies behind
                const v4i old = *reinterpret_cast<EPARA_GLOBAL v4i*>(at);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int before = low_bytes(had - chunk_first - 4 * j), upper = ~low_bytes(upto - chunk_first - 4 * j);
                    out[j] = (out[j] & ~(before | upper)) | ((grow_v ? rescaled(old[j], factor_v) : old[j]) & before) | (old[j] & upper);
                }
            }
            *reinterpret_cast<EPARA_GLOBAL v4i*>(at) = out;
        }
    }
    if (lane == 0) {
        scales[half] = static_cast<uint8_t>(e_k + 127);
        scales[2 + half] = static_cast<uint8_t>(e_v + 127);
    }
}

// ---- queries: row_lanes rows x a few heads; a lane takes 8 dims and their partners
template <int D>
__device__ __forceinline__ void rotate_queries(const epara_append_args& a, const epara_sequence& s, const append_shape& w, int item, int lane)
{
    constexpr int LANES = D / 16, GROUPS = 64 / LANES;
    const int row_item = item / w.head_items, head_item = item - row_item * w.head_items;
    const int group = lane / LANES, dims = (lane & (LANES - 1)) * 8;
    const int row = row_item * w.row_lanes + (group & (w.row_lanes - 1));
    const int heads_at_once = GROUPS / w.row_lanes, first_head = head_item * heads_at_once * QUERY_STEPS + group / w.row_lanes;
    if (row >= s.rows) return;
    const size_t global_row = static_cast<size_t>(s.first_row) + row;
    const EPARA_GLOBAL char* src = (const EPARA_GLOBAL char*)a.QKV + global_row * a.qkv_stride * 2 + dims * 2;
    EPARA_GLOBAL char* dst = (EPARA_GLOBAL char*)a.Q + global_row * a.q_stride * 2 + dims * 2;
    v4i in[QUERY_STEPS][2];
#pragma unroll
    for (int i = 0; i < QUERY_STEPS; ++i) {
        const int head = first_head + i * heads_at_once;
        if (head < a.heads) {
            in[i][0] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + static_cast<size_t>(head) * D * 2);
            in[i][1] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + static_cast<size_t>(head) * D * 2 + D);
        }
    }
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        cs[j] = 1.f;
        sn[j] = 0.f;
    }
    if (a.rotary) load_angles<8>(angles_of(a, static_cast<int>(global_row), s.start + row), dims, cs, sn);
#pragma unroll
    for (int i = 0; i < QUERY_STEPS; ++i) {
        const int head = first_head + i * heads_at_once;
        if (head >= a.heads) break;
        float u[8], v[8];
        unpack8(in[i][0], u);
        unpack8(in[i][1], v);
        v4i lo = in[i][0], hi = in[i][1];
        if (a.rotary) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int e = 2 * j, o = 2 * j + 1;
                lo[j] = static_cast<int>(pack_bf16(u[e] * cs[e] - v[e] * sn[e], u[o] * cs[o] - v[o] * sn[o]));
                hi[j] = static_cast<int>(pack_bf16(v[e] * cs[e] + u[e] * sn[e], v[o] * cs[o] + u[o] * sn[o]));
            }
        }
        *reinterpret_cast<EPARA_GLOBAL v4i*>(dst + static_cast<size_t>(head) * D * 2) = lo;
        *reinterpret_cast<EPARA_GLOBAL v4i*>(dst + static_cast<size_t>(head) * D * 2 + D) = hi;
    }
}

__global__ __launch_bounds__(NT) void cache_append_kernel(const epara_append_args* __restrict__ args, const epara_sequence* __restrict__ seqs,
                                                         const int32_t* __restrict__ pages, const int32_t* __restrict__ first, int n_seqs, int n_items)
{
    const int lane = threadIdx.x & 63;
    int item = blockIdx.x * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= n_items) return;
    const int i = find_sequence(first, n_seqs, item, lane);
    const epara_sequence s = seqs[i];
    const epara_append_args a = args[s.service];
    const append_shape w = shape_of_append(a, s);
    item -= first[i];
    if (item < w.blocks * a.kv_heads) {
        const int block = item / a.kv_heads, head = item - block * a.kv_heads;
        const int at = max_of(s.start, 0) / BLOCK + block;
        if (a.head_dim == 128) append_block<128>(a, s, pages, at, head, lane);
        else                   append_block<64>(a, s, pages, at, head, lane);
    } else {
        item -= w.blocks * a.kv_heads;
        if (a.head_dim == 128) rotate_queries<128>(a, s, w, item, lane);
        else                   rotate_queries<64>(a, s, w, item, lane);
    }
}

// ---- copies of pages: a workgroup per (move, head)
__global__ __launch_bounds__(NT) void copy_pages_kernel(const epara_page_copy* __restrict__ caches, int G, const epara_page_move* __restrict__ moves)
{
    const int chunk = blockIdx.x, tid = threadIdx.x;
    int g = 0, n = G;                                      // the last cache whose first_chunk is <= chunk
    while (n > 1) {
        const int step = (n + 63) >> 6, at = (tid & 63) * step;
        const int sum = at < n ? caches[g + at].first_chunk : 0x7fffffff;
        const int before = (__builtin_popcountll(__ballot(sum <= chunk)) - 1) * step;
        g += before;
        n = n - before < step ? n - before : step;
    }
    const epara_page_copy c = caches[__builtin_amdgcn_readfirstlane(g)];
    const int local = chunk - c.first_chunk, move = local / c.kv_heads, head = local - move * c.kv_heads;
    const epara_page_move mv = moves[c.first_move + move];
    const size_t bytes = head_bytes(c.head_dim), from = (static_cast<size_t>(mv.src) * c.kv_heads + head), to = (static_cast<size_t>(mv.dst) * c.kv_heads + head);
    const EPARA_GLOBAL char* src = (const EPARA_GLOBAL char*)c.codes + from * bytes + tid * 16;
    EPARA_GLOBAL char* dst = (EPARA_GLOBAL char*)c.codes + to * bytes + tid * 16;
    const int steps = c.head_dim / 32;                     // 4 or 2 pieces of 4 KiB
    v4i v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < steps) v[i] = __builtin_nontemporal_load(reinterpret_cast<const EPARA_GLOBAL v4i*>(src + i * NT * 16));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < steps) __builtin_nontemporal_store(v[i], reinterpret_cast<EPARA_GLOBAL v4i*>(dst + i * NT * 16));
    if (tid == 0) ((EPARA_GLOBAL uint32_t*)c.scales)[to] = ((const EPARA_GLOBAL uint32_t*)c.scales)[from];
}

}  // namespace

extern "C" {

int32_t epara_cache_append(const epara_append_args* h_args, const epara_append_args* d_args, int32_t G, const epara_sequence_table* table,
                           const int32_t* h_first, const int32_t* d_first, void* stream)
{
    if (const int32_t rc = epara_check_append_call(h_args, G, table, h_first)) return rc;
    const int32_t n_items = table->n_seqs > 0 ? h_first[table->n_seqs] : 0;
    if (n_items == 0) return EPARA_OK;
    if (!d_args || !d_first) return EPARA_ERR_NULL;
    hipLaunchKernelGGL(cache_append_kernel, dim3(static_cast<unsigned>((n_items + NT / 64 - 1) / (NT / 64))), dim3(NT), 0, static_cast<hipStream_t>(stream),
                       d_args, table->d_seqs, table->d_pages, d_first, table->n_seqs, n_items);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}

int32_t epara_copy_pages(const epara_page_copy* h_caches, const epara_page_copy* d_caches, int32_t G,
                         const epara_page_move* h_moves, const epara_page_move* d_moves, int32_t n_moves, void* stream)
{
    int32_t n_chunks;
    if (const int32_t rc = epara_check_copy_call(h_caches, G, h_moves, n_moves, &n_chunks)) return rc;
    if (n_chunks == 0) return EPARA_OK;
    if (!d_caches || !d_moves) return EPARA_ERR_NULL;
    hipLaunchKernelGGL(copy_pages_kernel, dim3(static_cast<unsigned>(n_chunks)), dim3(NT), 0, static_cast<hipStream_t>(stream), d_caches, G, d_moves);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}

}  // extern "C"
