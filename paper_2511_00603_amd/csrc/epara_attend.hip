// libepara: causal attention of new tokens over a paged cache in 8 bits (the decode and prefill services' attention).
//
//   o = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m),   z_j = scale q . k_j (capped: c tanh(z_j / c)),   m = max_j z_j
//
// Both products run on the matrix cores in f16 with fp32 sums.  E4M3 codes widen to f16 exactly, two to an instruction; a query (bf16,
// 8 significant bits) becomes f16 exactly once its own power of two is taken out, and a weight p = exp(z - m) keeps 11 bits, where bf16
// would keep 8.  (The 8-bit matrix instructions would take the codes as they are, and a query or weight as the sum of two E4M3 numbers at the
// same rate; but they hold a sum only to some 2^-12 of its largest term, which is 10^-2 of a weight where a score has terms of 40.)
// The blocks' scales are powers of two: those of the keys go into the factor between scores and the exponential, those of the values
// into the exponent of the weights.
//
// What a key gives to a row is its weight times its block's scale 2^e, so a row's references are two: M for z and V for the scales, with M + V for z + e.
// Weights are 2^(z + e - M - V + LIFT) in f16, and all that a row sees counts by what it gives: a block that is hidden from the row or has no
// weight takes no bits from the others, however large its values are.  (With the largest e of the pages read in place of V it would.)  The
// references are lazy: f16 bears ABOVE over them, so sums are rescaled only where z or z + e exceeds its reference by more than that
// (many rows: where the weights' sum says that one may).  Weights keep their 11 bits down to 2^-23 of M + V, so thousands of keys that share
// what one strong key leaves are held.  The weights' own sum, without scales, is fp32's, relative to M.
//
// Both products are written transposed, so that what the first leaves in a lane is what the second wants there:
//   S^T = K Q^T   A = keys x dims, B = dims x rows;   O^T = V^T P^T   A = dims x tokens, B = tokens x rows
// For this the cache holds keys and values in the order it does: a 16-byte chunk is what a lane needs for two instructions.
//
//   few rows (a workgroup has a tile of 16): 16x16x32.  Lane (n = lane % 16, q = lane / 16) gets from the four tiles t of S^T of a page the
//     scores of row n with the keys 16 q + 4 t + 0 .. 3: the 16 tokens of a chunk of a dim's values.  Pages go from memory to registers; the four
//     waves take them in turn and meet in the LDS at the end.
//   many rows (a tile of 128, 32 to a wave): 32x32x16.  Lane (n = lane % 32, h = lane / 32) gets from the two tiles u of S^T of a page the scores of row n
//     with the keys 32 u + 16 h + 0 .. 15, again a chunk.  Pages go through the registers, where they are widened once for all four waves, to the LDS.
//
// Few rows are bound by HBM: a token of 105 requests (0.42 GB of cache) 77 us, 5.5 TB/s; of 16 requests at 16384 tokens 87 us, 6.2 TB/s; of one at 32768
// 19.4 us, of which 7 are start, joining and launch.  The pages of a wave are 16 KiB in whole lines; two waves per SIMD have 128 KiB in flight in a compute unit.
// They are read with the non-temporal hint, since a model's layers together pass any cache (without it 86 and 98 us; one request the same).
// Many rows are bound by no single unit: two prompts of 4096 tokens 274 us, 1000 TFLOP/s, with the matrix cores busy 46 % of the time, the
// LDS 35 %; two workgroups of a compute unit wait on barriers and the LDS in turn.  Widening once for all four waves instead of in each took 314 us to 291.
// (The results of the matrix instructions are never read by an inline instruction: the compiler puts the waits they need only in front of its own.)
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

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));

// Eight E4M3 codes -> eight f16, exactly.
__device__ __forceinline__ v8h widen(int a, int b)
{
    const v2h p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
    const v2h r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
    return v8h{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
// Eight fp32 -> eight f16, round to nearest even.
__device__ __forceinline__ v8h narrow(const float* x)
{
    const v2h p = __builtin_convertvector((v2f{x[0], x[1]}), v2h), q = __builtin_convertvector((v2f{x[2], x[3]}), v2h);
    const v2h r = __builtin_convertvector((v2f{x[4], x[5]}), v2h), s = __builtin_convertvector((v2f{x[6], x[7]}), v2h);
    return v8h{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
// Eight bf16 times a power of two -> f16.
__device__ __forceinline__ v8h query8(const v4i& raw, float inv)
{
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = bf16_lo(static_cast<uint32_t>(raw[j])) * inv;
        x[2 * j + 1] = bf16_hi(static_cast<uint32_t>(raw[j])) * inv;
    }
    return narrow(x);
}
__device__ __forceinline__ float largest8(const v4i& raw)
{
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(bf16_lo(static_cast<uint32_t>(raw[j]))), fabsf(bf16_hi(static_cast<uint32_t>(raw[j])))));
    return top;
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
    w.a.window = min_of(w.a.window, EPARA_CACHE_MAX_TOKENS);        // no more tokens are there, and positions less a window stay in 32 bits
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

// 8 bytes that a workgroup on another die has written in this kernel: past the dies' own caches.  (Each lane of its own slot: a buffer's descriptor would have to be
// the same for all lanes.)
__device__ __forceinline__ v2f get2(const float* at)
{
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return v2f{__uint_as_float(static_cast<uint32_t>(v)), __uint_as_float(static_cast<uint32_t>(v >> 32))};
}

constexpr float NOTHING = -3e38f;                          // reference of a row that has seen no key
constexpr float LARGE = 4096.f;                            // references from which on a score is rounded before M is taken from it
constexpr float ABOVE = 6.f, LIFT = 9.f;                   // a weight is at most 2^(ABOVE + LIFT) = 2^15
constexpr float MOST = 32768.f;                            // sum of weights in which none can be more than that
constexpr float FAR = 4000.f;                              // farther than any two scales
constexpr int NO_SCALE = -1000;                            // the values' reference before any page
constexpr int LEAST_SHIFT = -60;                           // of a block's scale under V: such weights are zeros in f16, their sum still is fp32's

struct row_state { float ref; int scale; float sum; };     // M, V, and the sum of the weights relative to M (of this lane's keys)

// Makes the references those of what has been and of a page, and gives the factor for sums of weights times values.  top: the row's largest score
// of the page in units of log 2 (-inf: the row sees none of it); mine: of this lane's keys, whose block's scale is 2^exponent; LANES:
// distances of the lanes that hold the others.
template <int... LANES>
__device__ __forceinline__ float raise_references(row_state& s, float top, float mine, int exponent)
{
    const float to = top > s.ref ? __builtin_ceilf(top) : s.ref, gone = s.ref - to;
    int scale = static_cast<int>(__builtin_ceilf(fmaxf(mine - to, -FAR))) + exponent;
    ((scale = max_of(scale, __shfl_xor(scale, LANES))), ...);
    scale = max_of(scale, s.scale + static_cast<int>(fmaxf(gone, -FAR)));
    const float f = __builtin_amdgcn_exp2f(gone + static_cast<float>(s.scale - scale));
    s.ref = to;
    s.scale = scale;
    s.sum *= __builtin_amdgcn_exp2f(gone);
    return f;
}

// Exponent of a weight, z unit - M + (LIFT + shift).  In one operation, which keeps the product's bits beyond fp32, as long as M is small: they are under 2^-12 then.
// For large scores they would tell equal ones apart, up to 2^x where M is of 2^(x + 24), and what is added to M would be lost in it: the product is
// rounded as the one that M comes from, and M taken off first.
template <bool V> struct flag { static constexpr bool value = V; };
__device__ __forceinline__ bool is_large(float ref) { return __ballot(fabsf(ref) > LARGE && ref != NOTHING) != 0; }
__device__ __forceinline__ float large_exponent(float z, float unit, float ref, float more)
{
#pragma clang fp contract(off)
    const float score = z * unit;
    return score - ref + more;
}

// The scales of a page and head: keys' and values' exponents of both blocks.  A block behind the last token has whatever the memory holds.
struct page_scales { float key[2]; int value[2]; };
__device__ __forceinline__ page_scales scales_of(uint32_t word, bool second_block)
{
    page_scales s;
    s.key[0] = exp2_int(static_cast<int>(word & 0xff) - 127);
    s.key[1] = exp2_int(static_cast<int>(word >> 8 & 0xff) - 127);
    s.value[0] = static_cast<int>(word >> 16 & 0xff) - 127;
    s.value[1] = second_block ? static_cast<int>(word >> 24) - 127 : s.value[0];
    return s;
}

// A service's cap, c: in units of log 2 a score is c tanh(z / c) = c (1 - 2 / (1 + e^(2 z / c))), whose error is c's share of fp32's, some 2e-7 c: 1e-4 at
// WIDE.  Above, scores far under c are taken from the series of tanh, which keeps their own bits.  A cap beyond LARGEST changes no score that
// fp32 could tell from another; one under LEAST makes all weights of a sign 1, as LEAST does.
struct score_cap {
    static constexpr float WIDE = 512.f, LARGEST = 0x1p64f, LEAST = 0x1p-64f;
    bool on, wide;
    float in, out;                                         // of a score in units of the query's head: to 2 z / (c log 2), and c / log 2
};
__device__ __forceinline__ score_cap cap_of(const epara_cache_attn_args& a, float q_unit)
{
    const float c = fmaxf(a.softcap, score_cap::LEAST);
    const bool on = a.softcap > 0.f && a.softcap < score_cap::LARGEST;
    return {on, on && c > score_cap::WIDE, (on ? 2.f * LOG2E * a.scale / c : a.scale * LOG2E) * q_unit, c * LOG2E};
}
__device__ __forceinline__ float capped_score(float z, float in, float out) { return out - 2.f * out * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * in)); }
// tanh u = u - u^3 / 3 + 2 u^5 / 15 - 17 u^7 / 315 + 62 u^9 / 2835 - ..: what is left out is under 1e-8 of it at 1 / 4.
__device__ __forceinline__ float widely_capped_score(float z, float in, float out)
{
    const float u = z * in * (0.5f / LOG2E), s = u * u;
    const float series = u + u * s * fmaf(s, fmaf(s, fmaf(s, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f);
    return fabsf(u) < 0.25f ? out * series : capped_score(z, in, out);
}

// The page numbers and scales of 64 pages of a part, one to a lane: a page costs two register reads instead of two dependent trips to memory.
// (Scalar loads would have every wait for the LDS wait for them too.)
struct page_list {
    const EPARA_GLOBAL int32_t* table;
    const EPARA_GLOBAL uint32_t* scales;
    int kv_heads, head, hi;
    int base, id;
    uint32_t word;
    __device__ __forceinline__ void fill(int from, int lane)
    {
        base = from;
        id = table[min_of(from + lane, hi - 1)];
        word = scales[static_cast<size_t>(static_cast<uint32_t>(id)) * kv_heads + head];
    }
    __device__ __forceinline__ void reach(int p, int lane) { if (p - base >= 64) fill(p, lane); }
    __device__ __forceinline__ uint32_t page(int p) const { return __builtin_amdgcn_readlane(id, p - base); }
    __device__ __forceinline__ uint32_t scale_word(int p) const { return __builtin_amdgcn_readlane(word, p - base); }
};
__device__ __forceinline__ page_list pages_of(const work_item& w, const int32_t* pages, int lane)
{
    page_list l = {(const EPARA_GLOBAL int32_t*)pages + w.s.first_page, (const EPARA_GLOBAL uint32_t*)w.a.scales, w.a.kv_heads, w.head, w.hi, w.lo, 0, 0};
    if (w.lo < w.hi) l.fill(w.lo, lane);
    return l;
}

template <int D>
struct few_lds {
    union {
        float o[WAVES][FEW_TILE][D + 4];                   // a part: the waves' sums
        v4f joined[WAVES][FEW_TILE * D / 4];               // joining the parts: the waves' sums again
    };
    float m[WAVES][FEW_TILE], l[WAVES][FEW_TILE], v[WAVES][FEW_TILE];
    float weight[MAX_PARTS][FEW_TILE];                     // of a part's sums in the result
    int scale[FEW_TILE];                                   // of the rows' results
    uint32_t last;
};

// 16 bytes that a workgroup on another die has written or will read in this kernel: past the dies' own caches (16: device scope).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t slot_of(char* slots, size_t item, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(slots + item * bytes, 0, bytes, 0x00020000);
}
__device__ __forceinline__ void put4(__amdgpu_buffer_rsrc_t slot, int at, v4f x) { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, x), slot, at, 0, 16); }
__device__ __forceinline__ v4f get4(__amdgpu_buffer_rsrc_t slot, int at) { return __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(slot, at, 0, 16)); }

__device__ __forceinline__ v4f scaled4(v4f x, int e) { return v4f{__builtin_ldexpf(x[0], e), __builtin_ldexpf(x[1], e), __builtin_ldexpf(x[2], e), __builtin_ldexpf(x[3], e)}; }

// Four consecutive columns of an output row of a tile of `size` rows.
__device__ __forceinline__ void store_out4(const work_item& w, int row, int col, v4f x)
{
    const int token = row / w.group, head = w.head * w.group + row - token * w.group;
    EPARA_GLOBAL char* dst = (EPARA_GLOBAL char*)w.a.O + (static_cast<size_t>(w.s.first_row + token) * w.a.o_stride + static_cast<size_t>(head) * w.a.head_dim + col) * 2;
    *reinterpret_cast<EPARA_GLOBAL v2u*>(dst) = v2u{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
}

// Sums that several waves or parts have of a row are of references (M, V) of their own.  They are added relative to the largest M and the largest
// V + M - that M, and get their scale once they have been divided by the sum of weights: before, they may leave fp32's range.

// A slot of few rows: 16 rows of D sums, then 16 x (M, sum of weights, V).
constexpr int FEW_SLOT = FEW_TILE * SLOT_FLOATS * 4;

// A wave's share of the parts: the first STEPS * 64 pieces of 16 bytes of each.  No branch lies between the loads, so those of several parts are in flight.
template <int D, int STEPS>
__device__ __forceinline__ void add_parts(const work_item& w, char* slots, few_lds<D>& lds, int wave, int lane)
{
    v4f acc[STEPS];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) acc[k] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = wave; i < w.parts; i += WAVES) {
        const __amdgpu_buffer_rsrc_t slot = slot_of(slots, w.first_item + static_cast<size_t>(i) * w.stride, FEW_SLOT);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int e = lane + 64 * k;                   // a piece past the rows reads what the slot holds, and is not stored
            acc[k] += get4(slot, e * 16) * lds.weight[i][e / (D / 4)];
        }
    }
#pragma unroll
    for (int k = 0; k < STEPS; ++k) lds.joined[wave][lane + 64 * k] = acc[k];
}

// All parts of a tile are in their slots: their weighted sum, in the order of the parts inside a wave and of the waves, so the same bits every time.
template <int D>
__device__ __forceinline__ void join_few(const work_item& w, char* slots, few_lds<D>& lds, int wave, int lane)
{
    const int tid = wave * 64 + lane, rows = min_of(FEW_TILE, w.rows - w.tile * FEW_TILE);
    {   // thread = (row, one of 16): weights of the parts.  A row that sees no key: zeros
        const int r = tid >> 4, j = tid & 15;
        float ref[MAX_PARTS / 16], sum[MAX_PARTS / 16], scale[MAX_PARTS / 16], top = NOTHING;
        v2f in[MAX_PARTS / 16][2];
#pragma unroll
        for (int i = 0; i < MAX_PARTS / 16; ++i) {         // (a part or row that is not there: what another one's place holds)
            if (16 * i >= w.parts) break;
            const float* s = reinterpret_cast<const float*>(slots + (w.first_item + static_cast<size_t>(min_of(j + 16 * i, w.parts - 1)) * w.stride) * FEW_SLOT) + FEW_TILE * D + 4 * r;
            in[i][0] = get2(s);
            in[i][1] = get2(s + 2);
        }
#pragma unroll
        for (int i = 0; i < MAX_PARTS / 16; ++i) {
            const bool there = j + 16 * i < w.parts && r < rows;
            ref[i] = there ? in[i][0][0] : NOTHING;
            sum[i] = there ? in[i][0][1] : 0.f;
            scale[i] = there ? in[i][1][0] : NO_SCALE;
        }
#pragma unroll
        for (int i = 0; i < MAX_PARTS / 16; ++i) top = fmaxf(top, ref[i]);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        float total = 0.f, widest = NO_SCALE;
#pragma unroll
        for (int i = 0; i < MAX_PARTS / 16; ++i) {
            total += sum[i] * __builtin_amdgcn_exp2f(ref[i] - top);
            scale[i] += ref[i] - top;
            widest = fmaxf(widest, scale[i]);
        }
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) {
            total += __shfl_xor(total, d);
            widest = fmaxf(widest, __shfl_xor(widest, d));
        }
        const float inv = top == NOTHING ? 0.f : 1.f / total;
#pragma unroll
        for (int i = 0; i < MAX_PARTS / 16; ++i)
            if (j + 16 * i < w.parts) lds.weight[j + 16 * i][r] = __builtin_amdgcn_exp2f(scale[i] - widest) * inv;
        if (j == 0) lds.scale[r] = static_cast<int>(widest);
    }
    __syncthreads();
    constexpr int STEPS = FEW_TILE * D / 256;              // 16-byte pieces of a slot per lane
    const int pieces = rows * D / 4;
    if (pieces <= 64)                  add_parts<D, 1>(w, slots, lds, wave, lane);
    else if (pieces <= 128)            add_parts<D, 2>(w, slots, lds, wave, lane);
    else if (STEPS == 4 || pieces <= 256) add_parts<D, 4>(w, slots, lds, wave, lane);
    else                               add_parts<D, STEPS>(w, slots, lds, wave, lane);
    __syncthreads();
    for (int e = tid; e < pieces; e += NT) {
        v4f x = lds.joined[0][e];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) x += lds.joined[i][e];
        x = scaled4(x, lds.scale[e / (D / 4)]);
        store_out4(w, w.tile * FEW_TILE + e / (D / 4), e % (D / 4) * 4, x);
    }
}

template <int D>
__device__ __forceinline__ void attend_few(const work_item& w, const int32_t* __restrict__ pages, uint32_t* counters, char* slots, char* lds_bytes, int item)
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

    // ---- the query: dims 16 q .. and (heads of 128) 64 + 16 q .., 8 to an instruction
    v8h query[KS][2];
    float q_unit;
    {
        const EPARA_GLOBAL char* src = (const EPARA_GLOBAL char*)a.Q + (static_cast<size_t>(w.s.first_row + token) * a.q_stride + static_cast<size_t>(query_head) * D) * 2;
        v4i raw[KS][2];
        float amax = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                raw[s][h] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + s * 128 + q * 32 + h * 16);
                amax = fmaxf(amax, largest8(raw[s][h]));
            }
        amax = fmaxf(amax, __shfl_xor(amax, 16));
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        const int e = block_exponent(amax);
        q_unit = exp2_int(e);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) query[s][h] = query8(raw[s][h], exp2_int(-e));
    }

    const size_t head_offset = static_cast<size_t>(w.head) * head_bytes(D);
    const size_t page_bytes = static_cast<size_t>(a.kv_heads) * head_bytes(D);
    v4i k[4][KS], v[D / 16];
    uint32_t scales = 0, scales_next = 0;
    auto base_of = [&](uint32_t page) { return (const EPARA_GLOBAL char*)a.codes + static_cast<size_t>(page) * page_bytes + head_offset + lane * 16; };
    auto load_keys = [&](const EPARA_GLOBAL char* base) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) k[t][s] = __builtin_nontemporal_load(reinterpret_cast<const EPARA_GLOBAL v4i*>(base + (t * KS + s) * 1024));
    };
    auto load_values = [&](const EPARA_GLOBAL char* base) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) v[d] = __builtin_nontemporal_load(reinterpret_cast<const EPARA_GLOBAL v4i*>(base + PAGE * D + d * 1024));
    };
    page_list list = pages_of(w, pages, lane);

    row_state state = {NOTHING, NO_SCALE, 0.f};
    bool large = false;                                    // some row's scores are
    v4f o[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] = v4f{0.f, 0.f, 0.f, 0.f};
    const score_cap cap = cap_of(a, q_unit);

    int p = w.lo + wave;
    const EPARA_GLOBAL char* base = nullptr;
    if (p < w.hi) {
        list.reach(p, lane);
        base = base_of(list.page(p));
        scales = list.scale_word(p);
        load_keys(base);
        load_values(base);
    }
    for (; p < w.hi; p += WAVES) {
        const bool more = p + WAVES < w.hi;
        const EPARA_GLOBAL char* next = base;
        if (more) {
            list.reach(p + WAVES, lane);
            next = base_of(list.page(p + WAVES));
            scales_next = list.scale_word(p + WAVES);
        }
        // ---- scores
        const page_scales ps = scales_of(scales, p * PAGE + BLOCK < end);
        v4f z[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            z[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    z[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(k[t][s][2 * h], k[t][s][2 * h + 1]), query[s][h], z[t], 0, 0, 0);
        }
        if (more) load_keys(next);
        const int at = p * PAGE + 16 * q;                  // my keys are at + 4 t + i
        float unit = cap.in * (q < 2 ? ps.key[0] : ps.key[1]);             // of a score, to log 2: my keys are of block q / 2
        if (cap.on) {
            if (cap.wide) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[t][i] = widely_capped_score(z[t][i], unit, cap.out);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[t][i] = capped_score(z[t][i], unit, cap.out);
            }
            unit = 1.f;
        }
        if (p * PAGE + PAGE - 1 > low_token || (a.window > 0 && p * PAGE <= high_token - a.window)) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = at + 4 * t + i;
                    z[t][i] = key > last_key || key < first_key ? -INFINITY : z[t][i] * unit;
                }
            unit = 1.f;
        }
        // ---- the row's largest score here: mine are 16 keys of one block, the lanes n, n + 16, .. hold the others
        float mine = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t) mine = fmaxf(mine, fmaxf(fmaxf(z[t][0], z[t][1]), fmaxf(z[t][2], z[t][3])));
        mine *= unit;
        const int exponent = q < 2 ? ps.value[0] : ps.value[1];
        const float over = mine - state.ref;
        if (__ballot(over > ABOVE || over + static_cast<float>(exponent - state.scale) > ABOVE)) {
            float top = fmaxf(mine, __shfl_xor(mine, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float f = raise_references<16, 32>(state, top, mine, exponent);
            large = is_large(state.ref);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d] *= f;
        }
        const int shift = max_of(exponent - state.scale, LEAST_SHIFT);      // my block's scale against V
        const float on_top = LIFT + static_cast<float>(shift), lift = on_top - state.ref;
        if (large) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[t][i] = large_exponent(z[t][i], unit, state.ref, on_top);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[t][i] = fmaf(z[t][i], unit, lift);
        }
        float sum = 0.f, weight[16];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                weight[4 * t + i] = __builtin_amdgcn_exp2f(z[t][i]);
                sum += weight[4 * t + i];
            }
        state.sum += __builtin_ldexpf(sum, -shift);
        const v8h w0 = narrow(weight), w1 = narrow(weight + 8);
        // ---- values.  What lies behind the last token may be anything, a NaN too: cleared
        if (p * PAGE + PAGE > end) {
            const int valid = end - at;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int mask = low_bytes(valid - 4 * j);
#pragma unroll
                for (int d = 0; d < D / 16; ++d) v[d][j] &= mask;
            }
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(v[d][0], v[d][1]), w0, o[d], 0, 0, 0);
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(v[d][2], v[d][3]), w1, o[d], 0, 0, 0);
        }
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
        lds.v[wave][n] = static_cast<float>(state.scale);
    }
    __syncthreads();
    constexpr int COLS = D / 16;
    const int r = tid >> 4, c = (tid & 15) * COLS;
    float mm = NOTHING, ll = 0.f, vv = NO_SCALE, oo[COLS];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mm = fmaxf(mm, lds.m[i][r]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) vv = fmaxf(vv, lds.v[i][r] + (lds.m[i][r] - mm));
#pragma unroll
    for (int j = 0; j < COLS; ++j) oo[j] = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const float over = lds.m[i][r] - mm, weight = __builtin_amdgcn_exp2f(lds.v[i][r] + over - vv);
        ll += __builtin_amdgcn_exp2f(over) * lds.l[i][r];
#pragma unroll
        for (int j = 0; j < COLS; ++j) oo[j] += weight * lds.o[i][r][c + j];
    }
    const int out_row = w.tile * FEW_TILE + r;
    if (w.parts > 1) {                                     // the part's sums go to its slot; who ends last adds up all of them
        const __amdgpu_buffer_rsrc_t slot = slot_of(slots, item, FEW_SLOT);
        if (out_row < w.rows) {
#pragma unroll
            for (int j = 0; j < COLS; j += 4) put4(slot, (r * D + c + j) * 4, v4f{oo[j], oo[j + 1], oo[j + 2], oo[j + 3]});
            if (c == 0) put4(slot, (FEW_TILE * D + 4 * r) * 4, v4f{mm, ll, vv, 0.f});
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) lds.last = __hip_atomic_fetch_add(counters + w.first_item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<uint32_t>(w.parts - 1);
        __syncthreads();
        if (!lds.last) return;
        if (tid == 0) __hip_atomic_store(counters + w.first_item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        join_few<D>(w, slots, lds, wave, lane);
        return;
    }
    if (out_row >= w.rows) return;
    const float inv = mm == NOTHING ? 0.f : 1.f / ll;      // a row that sees no key: zeros
#pragma unroll
    for (int j = 0; j < COLS; j += 4) store_out4(w, out_row, c + j, scaled4(v4f{oo[j], oo[j + 1], oo[j + 2], oo[j + 3]} * inv, static_cast<int>(vv)));
}

__global__ __launch_bounds__(NT, 2) void attend_few_kernel(const epara_cache_attn_args* __restrict__ args, const epara_sequence* __restrict__ seqs,
                                                          const int32_t* __restrict__ pages, const int32_t* __restrict__ first, int n_seqs, int part_pages,
                                                          uint32_t* counters, char* slots)
{
    __shared__ __attribute__((aligned(16))) char lds[sizeof(few_lds<128>)];
    const int item = blockIdx.x;
    const work_item w = find_work<FEW_TILE>(args, seqs, first, n_seqs, part_pages, item, threadIdx.x & 63);
    if (w.part > 0 && w.part >= w.parts) return;           // this tile has fewer parts than the sequence's longest
    if (w.a.head_dim == 128) attend_few<128>(w, pages, counters, slots, lds, item);
    else                     attend_few<64>(w, pages, counters, slots, lds, item);
}

// ---- many rows -------------------------------------------------------------------------------------------------

typedef __attribute__((address_space(3))) char* ldsptr;
__device__ __forceinline__ v8h lds8h(ldsptr at) { return *reinterpret_cast<const __attribute__((address_space(3))) v8h*>(at); }
__device__ __forceinline__ void lds_put(ldsptr at, v8h x) { *reinterpret_cast<__attribute__((address_space(3))) v8h*>(at) = x; }

template <int D>
__device__ __forceinline__ void attend_many(const work_item& w, const int32_t* __restrict__ pages, uint32_t* counters, char* slots, ldsptr ring, int item)
{
    constexpr int DT = D / 32;                             // tiles of 32 dims
    constexpr int PAGE_BYTES = 2 * PAGE * D, LOADS = PAGE_BYTES / 1024 / WAVES, VALUES = PAGE * D * 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const epara_cache_attn_args& a = w.a;

    const int first_row = w.tile * MANY_TILE + wave * 32;  // of my wave
    const bool live = first_row < w.rows;
    const int row = min_of(first_row + n, w.rows - 1), token = row / w.group, query_head = w.head * w.group + row - token * w.group;
    const int last_key = w.s.start + token, first_key = a.window > 0 ? last_key - a.window + 1 : 0;
    const int low_token = w.s.start + min_of(first_row, w.rows - 1) / w.group, high_token = w.s.start + (min_of(w.rows, first_row + 32) - 1) / w.group;
    const int end = w.s.start + w.s.rows;

    // ---- the query: dims 32 p + 16 h .., 8 to an instruction
    constexpr int QS = D / 32;
    v8h query[QS][2];
    float q_unit;
    {
        const EPARA_GLOBAL char* src = (const EPARA_GLOBAL char*)a.Q + (static_cast<size_t>(w.s.first_row + token) * a.q_stride + static_cast<size_t>(query_head) * D) * 2;
        v4i raw[QS][2];
        float amax = 0.f;
#pragma unroll
        for (int p = 0; p < QS; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                raw[p][i] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + p * 64 + h * 32 + i * 16);
                amax = fmaxf(amax, largest8(raw[p][i]));
            }
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        const int e = block_exponent(amax);
        q_unit = exp2_int(e);
#pragma unroll
        for (int p = 0; p < QS; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) query[p][i] = query8(raw[p][i], exp2_int(-e));
    }

    // ---- pages to the LDS, widened on the way: a wave brings a quarter of each, waves 0 and 1 the keys.  A page in the LDS is in f16, in pieces of
    // 1 KiB of which lane l reads 16 bytes at 16 l: keys (tile u, dims 32 s + 16 h + 8 j ..), then values (dims 32 d .., tile u, tokens 16 h + 8 j ..)
    page_list list = pages_of(w, pages, lane);
    const size_t page_bytes = static_cast<size_t>(a.kv_heads) * PAGE_BYTES;
    const bool brings_values = wave >= 2;
    const int piece = (wave & 1) * LOADS;                  // of its half of the page
    const int put_at = brings_values ? VALUES + (lane >> 5) * 2048 + ((lane >> 4) & 1) * 512 + (lane & 15) * 16
                                     : ((lane >> 3) & 1) * (D * 64) + (lane >> 5) * 2048 + ((lane >> 4) & 1) * 512 + (lane & 7) * 16;
    v4i raw[LOADS];
    auto fetch = [&](int p) -> uint32_t {                  // returns the page's scales
        list.reach(p, lane);
        const EPARA_GLOBAL char* base = (const EPARA_GLOBAL char*)a.codes + list.page(p) * page_bytes + static_cast<size_t>(w.head) * PAGE_BYTES + wave * LOADS * 1024 + lane * 16;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) raw[i] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(base + i * 1024);
        return list.scale_word(p);
    };
    auto clear_behind = [&](int p) {                       // values behind the last token may be anything, a NaN too
        if (!brings_values || p * PAGE + PAGE <= end) return;
        const int valid = end - p * PAGE - 16 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                raw[i][j] &= low_bytes(valid - 4 * j);
            }
    };
    auto put = [&](ldsptr to) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = piece + i, key_off = D == 128 ? (at & 1) * 4096 + (at >> 1) * 128 : at * 128, value_off = (at >> 1) * 4096 + (at & 1) * 256;
            ldsptr dst = to + put_at + (brings_values ? value_off : key_off);
            lds_put(dst, widen(raw[i][0], raw[i][1]));
            lds_put(dst + 1024, widen(raw[i][2], raw[i][3]));
        }
    };

    row_state state = {NOTHING, NO_SCALE, 0.f};
    float most = MOST;                                     // of a sum; -1 where some row's scores are large, so that every sum is looked at
    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    const score_cap cap = cap_of(a, q_unit);
    // my rows see the pages [my_lo, my_hi) of the tile's; the others I only bring
    const int my_hi = live ? max_of(min_of(w.hi, (high_token + PAGE) / PAGE), w.lo) : w.lo;
    const int my_lo = min_of(my_hi, max_of(w.lo, a.window > 0 && low_token >= a.window ? (low_token - a.window + 1) / PAGE : 0));
    uint32_t now = 0, next = 0;                            // scales of the page that is read and of the one in my registers
    int p = w.lo;
    ldsptr here = ring + lane * 16, there = ring + 2 * PAGE_BYTES;           // the page that is read (for this lane), and the next one's place
    // page p lies in the LDS, page p + 1 in the registers of the waves that bring it (behind the last page: the last one once more, so that nothing branches)
    auto page_or_last = [&](int i) { return min_of(i, w.hi - 1); };
    if (w.lo < w.hi) {
        now = fetch(w.lo);
        clear_behind(w.lo);
        put(ring);
        next = fetch(page_or_last(w.lo + 1));
    }
    auto turn = [&]() {                                    // page p is in the LDS once all waves are here, and page p - 1 has been read
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        clear_behind(page_or_last(p + 1));
    };
    auto swap = [&]() {
        ldsptr t = here - lane * 16;
        here = there + lane * 16;
        there = t;
        now = next;
        ++p;
    };
    auto only_bring = [&](int upto) {
        while (p < upto) {
            turn();
            put(there);
            const uint32_t later = fetch(page_or_last(p + 2));
            swap();
            next = later;
        }
    };
    only_bring(my_lo);
    while (p < my_hi) {
        turn();
        const page_scales ps = scales_of(now, p * PAGE + BLOCK < end);
        // ---- scores, and the next page's widening
        v16f z[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) z[u][i] = 0.f;
#pragma unroll
        for (int s = 0; s < QS; ++s)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int u = 0; u < 2; ++u) z[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds8h(here + ((u * QS + s) * 2 + j) * 1024), query[s][j], z[u], 0, 0, 0);
        put(there);
        const uint32_t later = fetch(page_or_last(p + 2));
        float unit[2] = {cap.in * ps.key[0], cap.in * ps.key[1]};          // of a score, to log 2
        if (cap.on) {
            if (cap.wide) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[u][i] = widely_capped_score(z[u][i], unit[u], cap.out);
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[u][i] = capped_score(z[u][i], unit[u], cap.out);
            }
            unit[0] = unit[1] = 1.f;
        }
        if (p * PAGE + PAGE - 1 > low_token || (a.window > 0 && p * PAGE <= high_token - a.window)) {
            const int last = last_key - p * PAGE - 16 * h, from = first_key - p * PAGE - 16 * h;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int i = 0; i < 16; ++i) z[u][i] = 32 * u + i > last || 32 * u + i < from ? -INFINITY : z[u][i] * unit[u];
                unit[u] = 1.f;
            }
        }
        auto scale_sums = [&](float f) {
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= f;
        };
        // ---- weights of a tile, and their sum with and without (`plain`) the values' scale (in fp32 before they are rounded: a block of small values may leave f16
        // nothing of its weights, but the sum needs them).  The references are raised only where the sum says that a weight may have left f16's range: no
        // maximum is formed otherwise.  The first page's weights are infinite against NOTHING.
        auto weigh = [&](int u, v8h* weights, float& plain, auto careful) -> float {
            const int shift = max_of(ps.value[u] - state.scale, LEAST_SHIFT);
            const float on_top = LIFT + static_cast<float>(shift), lift = on_top - state.ref;
            float x[16], sum[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = __builtin_amdgcn_exp2f(careful.value ? large_exponent(z[u][i], unit[u], state.ref, on_top) : fmaf(z[u][i], unit[u], lift));
                sum[i & 1] += x[i];
            }
            weights[0] = narrow(x);
            weights[1] = narrow(x + 8);
            plain = __builtin_ldexpf(sum[0] + sum[1], -shift);
            return sum[0] + sum[1];
        };
        auto raise = [&](int u) {
            float top = z[u][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, z[u][i]);
            top *= unit[u];
            top = fmaxf(top, __shfl_xor(top, 32));         // the other half of the row
            scale_sums(raise_references<>(state, top, top, ps.value[u]));
            most = is_large(state.ref) ? -1.f : MOST;
        };
        auto add_values = [&](int u, const v8h* weights) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds8h(here + VALUES + ((d * 2 + u) * 2 + j) * 1024), weights[j], o[d], 0, 0, 0);
        };
        v8h first[2], second[2];
        auto settle = [&](int u, v8h* weights) {           // one branch, seldom taken: to raise the references, and for large scores
            float plain;
            if (__ballot(weigh(u, weights, plain, flag<false>()) > most)) {
                raise(u);                                  // (references that need not rise stay)
                weigh(u, weights, plain, flag<true>());
            }
            state.sum += plain;
        };
        settle(0, first);
        add_values(0, first);
        settle(1, second);
        add_values(1, second);
        swap();
        next = later;
    }
    only_bring(w.hi);
    state.sum += __shfl_xor(state.sum, 32);

    float scale = static_cast<float>(state.scale);
    if (w.parts > 1) {
        // a slot: per wave 1 KiB for each quad of registers, then 32 x (M, sum of weights, V)
        char* slot_at = slots + static_cast<size_t>(item) * MANY_TILE * SLOT_FLOATS * 4;
        __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(slot_at, 0, MANY_TILE * SLOT_FLOATS * 4, 0x00020000);
        constexpr int WAVE_BYTES = 32 * SLOT_FLOATS * 4;
        const int at = wave * WAVE_BYTES + lane * 16, refs_at = wave * WAVE_BYTES + 16384 + n * 16;
        if (live) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, v4f{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]}), rsrc, at, (d * 4 + j) * 1024, 16);   // 16: device scope
            if (h == 0) put4(rsrc, refs_at, v4f{state.ref, state.sum, scale, 0.f});
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        __attribute__((address_space(3))) uint32_t* box = (__attribute__((address_space(3))) uint32_t*)ring;
        if (tid == 0) *box = __hip_atomic_fetch_add(counters + w.first_item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (*box != static_cast<uint32_t>(w.parts - 1)) return;
        if (tid == 0) __hip_atomic_store(counters + w.first_item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (!live) return;
        state = {NOTHING, NO_SCALE, 0.f};
        scale = NO_SCALE;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        for (int i = 0; i < w.parts; ++i) {
            char* from = slots + (static_cast<size_t>(w.first_item) + static_cast<size_t>(i) * w.stride) * MANY_TILE * SLOT_FLOATS * 4;
            rsrc = __builtin_amdgcn_make_buffer_rsrc(from, 0, MANY_TILE * SLOT_FLOATS * 4, 0x00020000);
            const v4f s = get4(rsrc, refs_at);
            v4i in[DT][4];
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) in[d][j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, (d * 4 + j) * 1024, 16);
            const float both = fmaxf(state.ref, s[0]), gone = state.ref - both, over = s[0] - both, wider = fmaxf(scale + gone, s[2] + over);
            const float keep = __builtin_amdgcn_exp2f(scale + gone - wider), add = __builtin_amdgcn_exp2f(s[2] + over - wider);
            state.ref = both;
            state.sum = state.sum * __builtin_amdgcn_exp2f(gone) + s[1] * __builtin_amdgcn_exp2f(over);
            scale = wider;
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
    const int unit = static_cast<int>(scale);
    const bool mine = first_row + n < w.rows;
    EPARA_GLOBAL char* dst = (EPARA_GLOBAL char*)a.O + (static_cast<size_t>(w.s.first_row + token) * a.o_stride + static_cast<size_t>(query_head) * D) * 2;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            v4i out;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int a = 4 * j + 2 * e, b = a + 4;
                const uint32_t x = pack_bf16(__builtin_ldexpf(o[d][a] * inv, unit), __builtin_ldexpf(o[d][a + 1] * inv, unit));
                const uint32_t y = pack_bf16(__builtin_ldexpf(o[d][b] * inv, unit), __builtin_ldexpf(o[d][b + 1] * inv, unit));
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
    __shared__ __attribute__((aligned(1024))) char ring[2 * 4 * PAGE * 128];        // two pages in f16: one is read, one on its way
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
                           l.table.n_seqs, l.plan.part_pages[0], counters, slots);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}
