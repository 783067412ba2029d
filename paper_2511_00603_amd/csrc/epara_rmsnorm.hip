// libepara: residual + root-mean-square normalisation of decoder blocks, with bf16 or E4M3 output.
//
//   s = x + r,  y = s / sqrt(mean(s^2) + eps) * gamma;   8 bits: code = sat(RNE(y / scale))
//
// A wave or a workgroup per row: the row is read once and stays in registers; its sum of squares and (8 bits with a scale per row) the
// maximum of |s gamma| are reduced together, since max |y| = max |s gamma| / sqrt(..).  A row whose squares leave fp32's range (values from 2^57 on, or
// all under 2^-48 with an eps no larger than their squares) is taken once more, from the registers, with its power of two taken out.
// Bound by HBM: 8192 rows of 5120 in bf16 64 us (5.2 TB/s), in 8 bits with a scale per row 57 us (5.1 TB/s); with a wave per row, whose 80 chunks
// left room for one wave per SIMD, 96 and 91.  105 rows of 4096 (a launch and its trips to memory) 3.5 us alone, 6.1 with a wave per row.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "epara.h"
#include "epara_cast.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
#define EPARA_GLOBAL __attribute__((address_space(1)))

constexpr int NT = 256;
constexpr int NORM_GRID = 2048;

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2bf));
}

// Group of row `row`: the last one whose first_row is <= row.
__device__ __forceinline__ int find_group(const epara_rmsnorm_args* __restrict__ args, int G, int row, int first)
{
    if (G <= 64) return __builtin_popcountll(__ballot(first <= row)) - 1;
    int lo = 0, hi = G - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (args[mid].first_row <= row) lo = mid; else hi = mid - 1;
    }
    return lo;
}

constexpr float LEAST_MEAN = 0x1p-96f;                     // of s^2, plus eps: above, what underflows in the squares does not count
constexpr float LEAST_SCALE = 0x1p-126f;                   // of a row's codes: the smallest whose inverse is finite

// THREADS threads share a row (64: a wave, narrow rows; 256: a workgroup), CH = 16-byte chunks (8 values) of it per thread that the widest row of
// the launch needs.  The loads of the next row are in flight while one is reduced and stored, and gamma stays in registers for as long as the
// rows are of one service.
template <int THREADS, int CH, bool BITS8>
__global__ __launch_bounds__(NT) void add_rmsnorm_kernel(const epara_rmsnorm_args* __restrict__ args, int G, int n_rows)
{
    constexpr int ROWS = NT / THREADS, WAVES = THREADS / 64;
    __shared__ float part[2][2][WAVES];                    // [turn][sum, maximum][wave]
    __shared__ float again[3][WAVES];                      // of a row that is taken once more: [largest value, sum, maximum][wave]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int at = THREADS == 64 ? lane : static_cast<int>(threadIdx.x);           // my place in the row
    const int first = G <= 64 && lane < G ? args[lane].first_row : 0x7fffffff;
    const int stride = gridDim.x * ROWS;
    v4i xv[CH], rv[CH];
    epara_rmsnorm_args a;
    auto load = [&](int global_row, epara_rmsnorm_args& q, int& group) {
        group = __builtin_amdgcn_readfirstlane(find_group(args, G, global_row, first));
        q = args[group];
        const size_t base = static_cast<size_t>(global_row - q.first_row) * q.d * 2;
        const EPARA_GLOBAL char* x = (const EPARA_GLOBAL char*)q.X + base;
        const EPARA_GLOBAL char* r = q.R ? (const EPARA_GLOBAL char*)q.R + base : nullptr;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int chunk = c * THREADS + at;
            xv[c] = v4i{0, 0, 0, 0};
            rv[c] = v4i{0, 0, 0, 0};
            if (chunk < q.d >> 3) {
                xv[c] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(x + chunk * 16);
                if (r) rv[c] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(r + chunk * 16);
            }
        }
    };
    int row = blockIdx.x * ROWS + (THREADS == 64 ? wave : 0);
    if (row >= n_rows) return;                             // (a whole wave, or a whole workgroup)
    int group, gamma_of = -1, turn = 0;
    load(row, a, group);
    v4f gm[CH][2];
    for (;;) {
        const int n_chunks = a.d >> 3;
        if (group != gamma_of) {
            gamma_of = group;
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (c * THREADS + at < n_chunks) {
                    const EPARA_GLOBAL float* gamma = (const EPARA_GLOBAL float*)a.gamma + (c * THREADS + at) * 8;
                    gm[c][0] = *reinterpret_cast<const EPARA_GLOBAL v4f*>(gamma);
                    gm[c][1] = *reinterpret_cast<const EPARA_GLOBAL v4f*>(gamma + 4);
                }
        }
        float s[CH][8], sum = 0.f, top = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t xu = static_cast<uint32_t>(xv[c][j]), ru = static_cast<uint32_t>(rv[c][j]);
                s[c][2 * j] = bf16_lo(xu) + bf16_lo(ru);   // chunks past the row hold zeros and add nothing
                s[c][2 * j + 1] = bf16_hi(xu) + bf16_hi(ru);
                sum += s[c][2 * j] * s[c][2 * j] + s[c][2 * j + 1] * s[c][2 * j + 1];
            }
        const epara_rmsnorm_args now = a;
        const size_t base = static_cast<size_t>(row - now.first_row) * now.d;
        const int row_of_group = row - now.first_row;
        const bool more = row < n_rows - stride;           // (row + stride may pass 2^31)
        if (more) load(row + stride, a, group);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int chunk = c * THREADS + at;
            if (chunk >= n_chunks) continue;
            if (now.S) {
                v4i out;
#pragma unroll
                for (int j = 0; j < 4; ++j) out[j] = static_cast<int>(pack_bf16(s[c][2 * j], s[c][2 * j + 1]));
                *reinterpret_cast<EPARA_GLOBAL v4i*>((EPARA_GLOBAL char*)now.S + base * 2 + chunk * 16) = out;
            }
            if constexpr (BITS8)
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(s[c][j] * gm[c][j >> 2][j & 3]));
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
            sum += __shfl_xor(sum, d);
            if constexpr (BITS8) top = fmaxf(top, __shfl_xor(top, d));
        }
        if constexpr (WAVES > 1) {                         // the turns alternate, so the next row's sums do not overtake a slow wave's reads
            if (lane == 0) {
                part[turn][0][wave] = sum;
                part[turn][1][wave] = top;
            }
            __syncthreads();
            sum = part[turn][0][0];
            top = part[turn][1][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) {
                sum += part[turn][0][i];
                if constexpr (BITS8) top = fmaxf(top, part[turn][1][i]);
            }
            turn ^= 1;
        }
        float mean = sum / static_cast<float>(now.d) + now.eps;
        if (!(mean < INFINITY) || mean < LEAST_MEAN) {     // (the same for all threads of the row)
            auto all = [&](float x, int which, bool add) {
#pragma unroll
                for (int d = 32; d >= 1; d >>= 1) x = add ? x + __shfl_xor(x, d) : fmaxf(x, __shfl_xor(x, d));
                if constexpr (WAVES > 1) {
                    if (lane == 0) again[which][wave] = x;
                    __syncthreads();
                    x = again[which][0];
#pragma unroll
                    for (int i = 1; i < WAVES; ++i) x = add ? x + again[which][i] : fmaxf(x, again[which][i]);
                }
                return x;
            };
            float largest = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) largest = fmaxf(largest, fabsf(s[c][j]));
            largest = fmaxf(all(largest, 0, false), sqrtf(now.eps));
            const int e = static_cast<int>(__float_as_uint(largest) >> 23) - 127;       // 0: -127
            sum = top = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s[c][j] = __builtin_ldexpf(s[c][j], -e);
                    sum += s[c][j] * s[c][j];
                    if (BITS8 && c * THREADS + at < n_chunks) top = fmaxf(top, fabsf(s[c][j] * gm[c][j >> 2][j & 3]));
                }
            mean = all(sum, 1, true) / static_cast<float>(now.d) + __builtin_ldexpf(now.eps, -2 * e);
            if constexpr (BITS8) top = all(top, 2, false);
        }
        const float factor = mean == 0.f ? 0.f : 1.f / sqrtf(mean);         // a row of zeros stays one
        if constexpr (BITS8) {
            float inv = now.out_inv_scale;
            if (now.row_scales) {
                float scale = top * factor == 0.f ? 1.f : top * factor / 448.f;          // a NaN in the row is a NaN here
                if (scale < LEAST_SCALE) scale = LEAST_SCALE;
                inv = 1.f / scale;
                if (at == 0) ((EPARA_GLOBAL float*)now.row_scales)[row_of_group] = scale;
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int chunk = c * THREADS + at;
                if (chunk >= n_chunks) continue;
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = s[c][j] * gm[c][j >> 2][j & 3] * factor * inv;
                const v2u codes = {epara_cast::f32x4_to_e4m3(y[0], y[1], y[2], y[3]), epara_cast::f32x4_to_e4m3(y[4], y[5], y[6], y[7])};
                *reinterpret_cast<EPARA_GLOBAL v2u*>((EPARA_GLOBAL char*)now.Y + base + chunk * 8) = codes;
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int chunk = c * THREADS + at;
                if (chunk >= n_chunks) continue;
                v4i out;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = 2 * j, o = e + 1;
                    out[j] = static_cast<int>(pack_bf16(s[c][e] * gm[c][e >> 2][e & 3] * factor, s[c][o] * gm[c][o >> 2][o & 3] * factor));
                }
                *reinterpret_cast<EPARA_GLOBAL v4i*>((EPARA_GLOBAL char*)now.Y + base * 2 + chunk * 16) = out;
            }
        }
        if (!more) return;
        row += stride;
    }
}

template <bool BITS8>
void enqueue(int widest, int rows, hipStream_t s, const epara_rmsnorm_args* d_args, int G)
{
    const int per_lane = (widest + 511) >> 9, per_thread = (widest + 2047) >> 11;
    const bool narrow = per_lane <= 2;
    const int items = narrow ? static_cast<int>((static_cast<int64_t>(rows) + NT / 64 - 1) / (NT / 64)) : rows;
    const dim3 grid(items < NORM_GRID ? items : NORM_GRID), wg(NT);
    if (per_lane <= 1)        hipLaunchKernelGGL((add_rmsnorm_kernel<64, 1, BITS8>), grid, wg, 0, s, d_args, G, rows);
    else if (narrow)          hipLaunchKernelGGL((add_rmsnorm_kernel<64, 2, BITS8>), grid, wg, 0, s, d_args, G, rows);
    else if (per_thread <= 1) hipLaunchKernelGGL((add_rmsnorm_kernel<256, 1, BITS8>), grid, wg, 0, s, d_args, G, rows);
    else if (per_thread <= 2) hipLaunchKernelGGL((add_rmsnorm_kernel<256, 2, BITS8>), grid, wg, 0, s, d_args, G, rows);
    else if (per_thread <= 3) hipLaunchKernelGGL((add_rmsnorm_kernel<256, 3, BITS8>), grid, wg, 0, s, d_args, G, rows);
    else                      hipLaunchKernelGGL((add_rmsnorm_kernel<256, 4, BITS8>), grid, wg, 0, s, d_args, G, rows);
}

inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace

extern "C" int32_t epara_add_rmsnorm(const epara_rmsnorm_args* h_args, const epara_rmsnorm_args* d_args, int32_t G, int32_t out_dtype, void* stream)
{
    if (G < 0) return EPARA_ERR_SHAPE;
    if (out_dtype != EPARA_BF16 && out_dtype != EPARA_FP8_E4M3) return EPARA_ERR_DTYPE;
    if (G == 0) return EPARA_OK;
    if (!h_args || !d_args) return EPARA_ERR_NULL;
    const bool bits8 = out_dtype == EPARA_FP8_E4M3;
    int64_t rows = 0;
    int32_t widest = 8;
    for (int32_t g = 0; g < G; ++g) {
        const epara_rmsnorm_args& a = h_args[g];
        if (a.M < 0 || a.d < 8 || a.d > EPARA_NORM_MAX_D || (a.d & 7) || !(a.eps >= 0.f) || !(a.eps < INFINITY)) return EPARA_ERR_SHAPE;
        if (a.first_row != rows) return EPARA_ERR_SHAPE;
        if (a.M > 0 && (!a.X || !a.gamma || !a.Y)) return EPARA_ERR_NULL;
        if (!bits8 && a.row_scales) return EPARA_ERR_SHAPE;
        if (bits8 && a.M > 0 && !a.row_scales && (!(a.out_inv_scale > 0.f) || !(a.out_inv_scale < INFINITY))) return EPARA_ERR_SHAPE;
        if (a.M > 0 && (a.Y == a.S || (bits8 && (a.Y == a.X || a.Y == a.R)))) return EPARA_ERR_SHAPE;
        if (misaligned(a.X, 16) || misaligned(a.R, 16) || misaligned(a.S, 16) || misaligned(a.Y, 16) || misaligned(a.gamma, 16) || misaligned(a.row_scales, 4)) return EPARA_ERR_ALIGN;
        rows += a.M;
        if (a.M > 0 && a.d > widest) widest = a.d;
        if (rows > INT32_MAX) return EPARA_ERR_SHAPE;
    }
    if (rows == 0) return EPARA_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (bits8) enqueue<true>(widest, static_cast<int>(rows), s, d_args, G);
    else       enqueue<false>(widest, static_cast<int>(rows), s, d_args, G);
    return hipGetLastError() == hipSuccess ? EPARA_OK : EPARA_ERR_HIP;
}
