// Attention for some 10 to 64 rows to a key head (trees of drafted tokens, mostly), or more where there are few sequences.  The products are those of many rows, 32x32x16, but pages go as
// for few rows from memory to registers, and nothing but the waves' sums passes the LDS: a workgroup has 32 rows, and its four waves take pages in turn.
//
// One tile to a head (ONCE) is bound by HBM as few rows are: trees of 5 of 64 requests (0.28 GB) 57 us, 4.8 TB/s, read with the non-temporal hint (without it 63).  Two tiles read a page
// twice, the second time from a die's cache: 9 to 16 rows of 105 requests (0.47 GB) 133 us, 3.5 TB/s (with the hint 153; tiles of 128 rows 164); there the waves' own time
// counts, some 3000 cycles of matrix and vector work to a page, and the start and end of a workgroup, 7 us.  Two tiles in one workgroup of eight waves 149 us (one workgroup fills a compute
// unit, and nothing runs while it starts); tiles of 64 rows to a wave 228 (one wave per SIMD, and registers spill).
// Included by epara_attend.hip, which has the parts that all its kernels share.

constexpr int MID_LANES = NT / MID_TILE;                   // threads to a row
// A slot: 32 x D sums, then 32 x (M, sum of weights, V).
constexpr int MID_SLOT = MID_TILE * SLOT_FLOATS * 4;

template <int D>
struct mid_lds {
    union {
        float o[WAVES][MID_TILE][D + 4];                       // a part: the waves' sums
        struct { float weight[MAX_PARTS][MID_TILE], sums[MAX_PARTS][MID_TILE], scales[MAX_PARTS][MID_TILE]; };        // joining the parts
    };
    float m[WAVES][MID_TILE], l[WAVES][MID_TILE], v[WAVES][MID_TILE];
    int scale[MID_TILE];                                       // of the rows' results
    uint32_t last;
    v8h query[D / 32][2][64];                   // as a lane wants it: the waves' are the same, and have no place in the registers
};

// All parts of a tile and head are in their slots: their weighted sum in the order of the parts, so the same bits every time.
template <int D>
__device__ __forceinline__ void join_mid(const work_item& w, char* slots, mid_lds<D>& lds)
{
    const int tid = threadIdx.x, rows = min_of(MID_TILE, w.rows - w.tile * MID_TILE);
    auto slot_at = [&](int part) { return slot_of(slots, w.first_item + static_cast<size_t>(part) * w.stride, MID_SLOT); };
    float (*weight)[MID_TILE] = lds.weight;
    {
        const int r = tid / MID_LANES, j = tid % MID_LANES;
        float top = NOTHING, widest = NO_SCALE, total = 0.f;
        for (int i = j; i < w.parts; i += MID_LANES) {
            const v4f x = get4(slot_at(i), (MID_TILE * D + 4 * r) * 4);
            weight[i][r] = x[0];                           // M; sum of weights and V follow below
            lds.sums[i][r] = x[1];
            lds.scales[i][r] = x[2];
            top = fmaxf(top, r < rows ? x[0] : NOTHING);
        }
#pragma unroll
        for (int d = MID_LANES / 2; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        for (int i = j; i < w.parts; i += MID_LANES) {
            const float over = weight[i][r] - top;
            total += lds.sums[i][r] * __builtin_amdgcn_exp2f(over);
            widest = fmaxf(widest, lds.scales[i][r] + over);
        }
#pragma unroll
        for (int d = MID_LANES / 2; d >= 1; d >>= 1) {
            total += __shfl_xor(total, d);
            widest = fmaxf(widest, __shfl_xor(widest, d));
        }
        const float inv = top == NOTHING ? 0.f : 1.f / total;              // a row that sees no key: zeros
        for (int i = j; i < w.parts; i += MID_LANES) weight[i][r] = __builtin_amdgcn_exp2f(lds.scales[i][r] + (weight[i][r] - top) - widest) * inv;
        if (j == 0) lds.scale[r] = static_cast<int>(widest);
    }
    __syncthreads();
    constexpr int PIECES = MID_TILE * D / 4 / NT;          // of 16 bytes, to a thread
    v4f x[PIECES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) x[k] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < w.parts; ++i) {
        const __amdgpu_buffer_rsrc_t slot = slot_at(i);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const int e = tid + NT * k;                    // a piece past the rows reads what the slot holds, and is not stored
            x[k] += get4(slot, e * 16) * weight[i][e / (D / 4)];
        }
    }
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int e = tid + NT * k, r = e / (D / 4);
        if (r < rows) store_out4(w, w.tile * MID_TILE + r, e % (D / 4) * 4, scaled4(x[k], lds.scale[r]));
    }
}

template <int D, bool ONCE>
__device__ __forceinline__ void attend_mid(const work_item& w, const int32_t* __restrict__ pages, uint32_t* counters, char* slots, char* lds_bytes, int item)
{
    mid_lds<D>& lds = *reinterpret_cast<mid_lds<D>*>(lds_bytes);
    constexpr int QS = D / 32, DT = D / 32;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const epara_cache_attn_args& a = w.a;
    const int end = w.s.start + w.s.rows;
    const bool tree = w.visible != nullptr;

    // ---- my row
    const int first_row = w.tile * MID_TILE, row = min_of(first_row + n, w.rows - 1), token = row / w.group, query_head = w.head * w.group + row - token * w.group;
    int last_key = w.s.start + token, low_token = w.s.start + first_row / w.group;       // pages up to low_token are seen by all rows of the tile
    const int high_token = w.s.start + (min_of(w.rows, first_row + MID_TILE) - 1) / w.group;
    if (tree) {
        const tree_row bits = tree_row_of(w, token);
        last_key = w.s.start + bits.follows;               // its position
        low_token = __ballot(!bits.there) ? -1 : w.s.start - 1;
    }
    const int first_key = a.window > 0 ? last_key - a.window + 1 : 0;
    float q_unit;
    {
        const EPARA_GLOBAL char* src = (const EPARA_GLOBAL char*)a.Q + (static_cast<size_t>(w.s.first_row + token) * a.q_stride + static_cast<size_t>(query_head) * D) * 2;
        v4i raw[QS][2];
        float amax = 0.f;
#pragma unroll
        for (int s = 0; s < QS; ++s)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                raw[s][j] = *reinterpret_cast<const EPARA_GLOBAL v4i*>(src + s * 64 + h * 32 + j * 16);
                amax = fmaxf(amax, largest8(raw[s][j]));
            }
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        const int e = block_exponent(amax);
        q_unit = exp2_int(e);
        if (wave == 0)
#pragma unroll
            for (int s = 0; s < QS; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j) lds.query[s][j][lane] = query8(raw[s][j], exp2_int(-e));
    }
    __syncthreads();

    // ---- pages: a lane's chunk of keys is row n of tile u of S^T = K Q^T with dims 32 s + 16 h .. + 15; of values, row n of tile d of O^T = V^T P^T with tokens 32 u + 16 h .. + 15
    const size_t head_offset = static_cast<size_t>(w.head) * head_bytes(D), page_bytes = static_cast<size_t>(a.kv_heads) * head_bytes(D);
    const int key_at = (n >> 3) * D * 16 + h * 256 + (n & 7) * 16, value_at = PAGE * D + (n >> 4) * 1024 + h * 256 + (n & 15) * 16;
    v4i k[2][QS], v[DT][2];
    auto base_of = [&](uint32_t page) { return (const EPARA_GLOBAL char*)a.codes + static_cast<size_t>(page) * page_bytes + head_offset; };
    auto load_keys = [&](const EPARA_GLOBAL char* base) {
        const EPARA_GLOBAL v4i* src = reinterpret_cast<const EPARA_GLOBAL v4i*>(base + key_at);
#pragma unroll
        for (int s = 0; s < QS; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) k[u][s] = ONCE ? __builtin_nontemporal_load(src + s * 32 + u * 8) : src[s * 32 + u * 8];
    };
    auto load_values = [&](const EPARA_GLOBAL char* base) {
        const EPARA_GLOBAL v4i* src = reinterpret_cast<const EPARA_GLOBAL v4i*>(base + value_at);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) v[d][u] = ONCE ? __builtin_nontemporal_load(src + d * 128 + u * 32) : src[d * 128 + u * 32];
    };
    page_list list = pages_of(w, pages, lane);

    row_state state = {NOTHING, NO_SCALE, 0.f};
    float most = MOST;                                     // of a sum of weights; -1 where some row's scores are large, so that every sum is looked at
    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    const score_cap cap = cap_of(a, q_unit);
    int p = w.lo + wave;
    const EPARA_GLOBAL char* base = nullptr;
    uint32_t scales = 0, scales_next = 0;
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
        const page_scales ps = scales_of(scales, p * PAGE + BLOCK < end);
        // ---- scores
        v16f z[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) z[u][i] = 0.f;
#pragma unroll
        for (int s = 0; s < QS; ++s)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const v8h q = lds.query[s][j][lane];
#pragma unroll
                for (int u = 0; u < 2; ++u) z[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen(k[u][s][2 * j], k[u][s][2 * j + 1]), q, z[u], 0, 0, 0);
            }
        if (more) load_keys(next);
        float unit[2] = {cap.in * ps.key[0], cap.in * ps.key[1]};          // of a score, to log 2
        if (cap.on) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (cap.wide) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[u][i] = widely_capped_score(z[u][i], unit[u], cap.out);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[u][i] = capped_score(z[u][i], unit[u], cap.out);
                }
                unit[u] = 1.f;
            }
        }
        if (p * PAGE + PAGE - 1 > low_token || (a.window > 0 && p * PAGE <= high_token - a.window)) {
            const int last = last_key - p * PAGE - 16 * h, from = first_key - p * PAGE - 16 * h;
            const uint64_t seen = tree ? seen_of_page(tree_row_of(w, token), p * PAGE - w.s.start) >> (16 * h) : last < 0 ? 0ull : last >= 63 ? ~0ull : (2ull << last) - 1;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t mine = static_cast<uint32_t>(seen >> (32 * u));
#pragma unroll
                for (int i = 0; i < 16; ++i) z[u][i] = !(mine >> i & 1) || 32 * u + i < from ? -INFINITY : z[u][i] * unit[u];
                unit[u] = 1.f;
            }
        }
        // ---- weights of a block, and their sum with and without (`plain`) the values' scale.  The references are raised only where the sum says that a weight may have left f16's range
        v8h weights[2][2];
        auto weigh = [&](int u, float& plain, auto careful) -> float {
            const int shift = max_of(ps.value[u] - state.scale, LEAST_SHIFT);
            const float on_top = LIFT + static_cast<float>(shift), lift = on_top - state.ref;
            float x[16], sum[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = __builtin_amdgcn_exp2f(careful.value ? large_exponent(z[u][i], unit[u], state.ref, on_top) : fmaf(z[u][i], unit[u], lift));
                sum[i & 1] += x[i];
            }
            weights[u][0] = narrow(x);
            weights[u][1] = narrow(x + 8);
            plain = __builtin_ldexpf(sum[0] + sum[1], -shift);
            return sum[0] + sum[1];
        };
        float plain[2], over[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) over[u] = weigh(u, plain[u], flag<false>());
        if (__ballot(over[0] > most || over[1] > most)) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {                  // (references that need not rise stay)
                float top = z[u][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) top = fmaxf(top, z[u][i]);
                top *= unit[u];
                top = fmaxf(top, __shfl_xor(top, 32));
                const float f = raise_references<>(state, top, top, ps.value[u]);
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= f;
            }
            most = is_large(state.ref) ? -1.f : MOST;
#pragma unroll
            for (int u = 0; u < 2; ++u) weigh(u, plain[u], flag<true>());
        }
        state.sum += plain[0] + plain[1];
        __builtin_amdgcn_sched_barrier(0);                 // (what the scheduler would take across costs registers: 132 us became 143)
        // ---- values.  What lies behind the last token may be anything, a NaN too: cleared
        if (p * PAGE + PAGE > end) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int mask = low_bytes(end - p * PAGE - 32 * u - 16 * h - 4 * j);
#pragma unroll
                    for (int d = 0; d < DT; ++d) v[d][u][j] &= mask;
                }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int d = 0; d < DT; ++d)               // (neighbours go to different sums)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen(v[d][u][2 * j], v[d][u][2 * j + 1]), weights[u][j], o[d], 0, 0, 0);
        if (more) load_values(next);
        base = next;
        scales = scales_next;
    }

    // ---- the four waves' sums
    state.sum += __shfl_xor(state.sum, 32);
    {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<v4f*>(&lds.o[wave][n][d * 32 + j * 8 + h * 4]) = v4f{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
        if (h == 0) {
            lds.m[wave][n] = state.ref;
            lds.l[wave][n] = state.sum;
            lds.v[wave][n] = static_cast<float>(state.scale);
        }
    }
    __syncthreads();
    const int r = tid / MID_LANES, c0 = tid % MID_LANES * 4;               // a row's threads take its columns by fours in turn
    const int out_row = w.tile * MID_TILE + r;
    const bool there = out_row < w.rows;
    float mm = NOTHING, ll = 0.f, vv = NO_SCALE, part[WAVES];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mm = fmaxf(mm, lds.m[i][r]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) vv = fmaxf(vv, lds.v[i][r] + (lds.m[i][r] - mm));
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const float over = lds.m[i][r] - mm;
        part[i] = __builtin_amdgcn_exp2f(lds.v[i][r] + over - vv);
        ll += __builtin_amdgcn_exp2f(over) * lds.l[i][r];
    }
    const __amdgpu_buffer_rsrc_t slot = slot_of(slots, item, MID_SLOT);
    const float inv = mm == NOTHING ? 0.f : 1.f / ll;      // a row that sees no key: zeros
#pragma unroll
    for (int c = 0; c < D; c += MID_LANES * 4) {
        v4f x = *reinterpret_cast<const v4f*>(&lds.o[0][r][c0 + c]) * part[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) x += *reinterpret_cast<const v4f*>(&lds.o[i][r][c0 + c]) * part[i];
        if (!there) continue;
        if (w.parts > 1) put4(slot, (r * D + c0 + c) * 4, x);
        else             store_out4(w, out_row, c0 + c, scaled4(x * inv, static_cast<int>(vv)));
    }
    if (w.parts <= 1) return;
    // ---- the part's sums are in its slot; who ends last adds up all of them
    if (there && c0 == 0) put4(slot, (MID_TILE * D + 4 * r) * 4, v4f{mm, ll, vv, 0.f});
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) lds.last = __hip_atomic_fetch_add(counters + w.first_item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<uint32_t>(w.parts - 1);
    __syncthreads();
    if (!lds.last) return;
    if (tid == 0) __hip_atomic_store(counters + w.first_item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    join_mid<D>(w, slots, lds);
}

template <bool ONCE>
__global__ __launch_bounds__(NT, 2) void attend_mid_kernel(const epara_cache_attn_args* __restrict__ args, const epara_tree_args* __restrict__ trees,
                                                          const epara_sequence* __restrict__ seqs, const int32_t* __restrict__ pages, const int32_t* __restrict__ first,
                                                          int n_seqs, int part_pages, uint32_t* counters, char* slots)
{
    __shared__ __attribute__((aligned(16))) char lds[sizeof(mid_lds<128>)];
    const int item = blockIdx.x;
    const work_item w = find_work<MID_TILE, true>(args, trees, seqs, first, n_seqs, part_pages, item, threadIdx.x & 63);
    if (w.part > 0 && w.part >= w.parts) return;           // this tile has fewer parts than the sequence's longest
    if (w.a.head_dim == 128) attend_mid<128, ONCE>(w, pages, counters, slots, lds, item);
    else                     attend_mid<64, ONCE>(w, pages, counters, slots, lds, item);
}
