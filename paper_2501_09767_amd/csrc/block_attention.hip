// Attention over the key blocks that a list names for every query block (lemo_block_attention and its form for single tokens).
//
//   O[i,h,:] = sum_j softmax_j(scale <Q[i,h], K[j,g]>) V[j,g,:]     over keys j of the listed blocks, j <= position of i if causal
//   lse2[h,i] = log2 sum_j 2^(c2 <Q[i,h], K[j,g]>),  c2 = scale log2 e
//
// The rows that share a list, R = bq * G of them, are a matrix: 32 rows a wave, resident as MFMA B operands, against the listed keys in
// stages of 128 (four subtiles) that all waves of the workgroup read from LDS.  Both products are taken transposed, as in the attention
// over kept tokens: S^T = K Q^T leaves a lane with 16 logits of one row, and P^T is then the B operand of O^T += V^T P^T as it
// lies in the registers.  KS waves share rows and take the subtiles of a stage in turn, for lists of few rows; their sums meet in LDS at
// the end.  Where lists are few as well (single tokens), n_parts workgroups take shares of a list and a second kernel joins them.
// P is rounded to bf16 for the second product; sums and normaliser are binary32, from the unrounded values.
#include "block_attention.hpp"

namespace lemo {

// Stages are kept to 64 KB for two of them, K and V, where that suits the sharing waves: two workgroups fit a CU then, and the one's list,
// rows and last stores pass while the other computes.
template <int D, int KS> constexpr int BA_STAGE = D == 128 && KS <= 2 ? 2 : 4;  // subtiles of a stage

template <int D, int WAVES, int BA_STAGE> struct BaGeo {
    using Tile = HeadTile<D>;
    static constexpr int SUB = 32 * Tile::ROWB, STAGE = 2 * BA_STAGE * SUB;  // bytes of a subtile; K and V subtiles of a stage
    static constexpr int PITCH = D + 4;                                      // floats of a row where waves' results meet
    static constexpr int JOIN = WAVES * 32 * (PITCH * 4 + 8);
    static constexpr int LIST = 2 * STAGE > JOIN ? 2 * STAGE : JOIN;         // the list's subtiles stand behind both
    static constexpr int lds(int subtiles) { return LIST + 16 + subtiles * 4; }  // (the number of them first, and whether sums are not finite)
};

// PACK: the rows belong to several lists, whose union is worked on; a row sees the subtiles that its own list names.
template <int D, int WAVES, int KS, bool PACK>
__global__ __launch_bounds__(WAVES * 64, 2) void block_attention_kernel(BlockAttnParams p) {
    constexpr int STAGE = BA_STAGE<D, KS>;
    using Geo = BaGeo<D, WAVES, STAGE>;
    using Tile = HeadTile<D>;
    constexpr int ROWS = WAVES / KS * 32;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    int* const keys = reinterpret_cast<int*>(smem + Geo::LIST) + 4;
    int &listed = keys[-4], &not_finite = keys[-3];

    int g, rank;
    decode_block(p.order, p.H_kv, p.n_qb * p.n_rt * p.n_parts, g, rank, p.first + blockIdx.x);
    const int share = rank % p.n_parts, rt = rank / p.n_parts % p.n_rt, qb = rank / p.n_parts / p.n_rt;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool causal = (p.flags & LEMO_CAUSAL) != 0;
    const int S = p.lengths ? min(max(p.lengths[qb], 0), p.S_k) : p.S_k;            // keys there are
    const long long pos0 = p.lengths ? S - 1 : p.q_start + (long long)qb * p.bq;  // position of the block's first query
    const int queries = min(p.bq, p.S_q - qb * p.bq);                               // (single tokens: 1)
    const int rows = queries * p.G, row_end = min(rows, (rt + 1) * ROWS);
    // last key that a row may see
    auto limit_of = [&](int row) { return causal ? (int)min(pos0 + row / p.G, (long long)S - 1) : S - 1; };

    int room = 0;  // (PACK) of the union's subtiles
    if constexpr (PACK) {
        if (tid == 0) not_finite = 0;
        const long long first = (long long)qb * p.pack;
        const int lists = (int)min((long long)p.pack, p.n_lists - first);
        room = min(p.pack * p.T, p.nb) * (p.b / 32);
        union_subtiles<WAVES>(p.blocks + (first * p.H_kv + g) * p.T, (long long)p.H_kv * p.T, lists, p.T, p.b, p.nb, limit_of(rows - 1), reinterpret_cast<unsigned*>(smem), keys,
                              room, &listed, wave, lane);
    } else {
        if (wave == 0) {
            const int n = rt * ROWS < rows ? list_subtiles(p.blocks + ((long long)qb * p.H_kv + g) * p.T, p.T, p.b, p.nb, limit_of(row_end - 1), keys, lane) : 0;
            if (lane == 0) listed = n;
        }
        __syncthreads();
    }
    const int s_begin = (int)((long long)listed * share / p.n_parts), n_sub = (int)((long long)listed * (share + 1) / p.n_parts) - s_begin;
    const int n_stage = (n_sub + STAGE - 1) / STAGE;

    // resident operand: this wave's 32 rows
    const int row0 = rt * ROWS + wave / KS * 32, row = row0 + l32;
    const bool live = row < rows;
    const int lim = live ? limit_of(row) : -1;
    const int member = PACK ? l32 / (p.R / p.pack) : 0;  // the row's list (there is one tile of rows)
    const int clean = row0 < rows ? limit_of(row0) : -1;              // a subtile that ends at or before it needs no mask
    const int reach = row0 < rows ? limit_of(min(row0 + 31, rows - 1)) : -1;  // one that begins behind it is nothing to the wave
    u32x4 qf[Tile::CHUNKS];
#pragma unroll
    for (int c = 0; c < Tile::CHUNKS; ++c) qf[c] = u32x4{0u, 0u, 0u, 0u};
    if (live) {
        const uint16_t* q = p.Q + ((long long)qb * p.bq + row / p.G) * p.q_ts + (long long)(g * p.G + row % p.G) * p.q_hs;
#pragma unroll
        for (int c = 0; c < Tile::CHUNKS; ++c) qf[c] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(q) + c * 32 + half * 16);
    }

    // staging by LDS-direct loads: an instruction of a wave fills 1 KB, whole rows; a subtile's rows are addressed from its first key, so
    // that no offset passes 32 bits, and what lies past the keys there are arrives as zeros
    const char* const kbase = reinterpret_cast<const char*>(p.K + (long long)g * p.k_hs + (p.lengths ? qb * p.k_ss : 0));
    const char* const vbase = reinterpret_cast<const char*>(p.V + (long long)g * p.v_hs + (p.lengths ? qb * p.v_ss : 0));
    constexpr int RPI = 1024 / Tile::ROWB, PER_SUB = 32 / RPI;            // rows of an instruction, instructions of a subtile
    constexpr int LOADS = 2 * STAGE * PER_SUB / WAVES;                 // of a wave and stage
    static_assert(2 * STAGE * PER_SUB % WAVES == 0, "");
    const int in_row = lane / Tile::PIECES, pos = lane % Tile::PIECES;
    auto load_stage = [&](int t, int buf) {
        int first_key[STAGE];  // all of them before the first load: a load orders memory accesses
#pragma unroll
        for (int s = 0; s < STAGE; ++s) first_key[s] = t * STAGE + s < n_sub ? __builtin_amdgcn_readfirstlane(keys[s_begin + t * STAGE + s]) : S;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            constexpr int AT_ONCE = WAVES / PER_SUB > 1 ? WAVES / PER_SUB : 1;  // subtiles that the waves load together
            const int unit = i * WAVES + wave, part = unit % PER_SUB, which = AT_ONCE > 1 ? i * AT_ONCE + wave / PER_SUB : i * WAVES / PER_SUB;
            const bool v = i * WAVES >= STAGE * PER_SUB;  // K subtiles, then V
            int key = first_key[i * WAVES / PER_SUB % STAGE];
#pragma unroll
            for (int k = 1; k < AT_ONCE; ++k) key = wave / PER_SUB == k ? first_key[(i * WAVES / PER_SUB + k) % STAGE] : key;
            const int pitch = (int)(v ? p.v_ts : p.k_ts) * 2;
            const u32x4 rsrc = subtile_rsrc<D>(v ? vbase : kbase, min(key, S), S, pitch);
            const int r = part * RPI + in_row;
            lds_direct_b128(rsrc, lds_offset_of(smem) + buf * Geo::STAGE + which * Geo::SUB + part * 1024, r * pitch + ((pos ^ Tile::swz(r)) << 4));
        }
    };

    f32x16 o[Tile::COLS];
    float ref, l = 0.f;  // reference of the exponentials (same in both half-waves); this half-wave's share of the normaliser
    // PACK: what is not finite in V of a block that only some rows list comes to the others as 0 times it, which is not 0.  Then the
    // workgroup goes through its list once more and adds to the sums of the rows that see a subtile alone: code of its own, since a branch
    // beside the products would cost the first turn 7 % (a list for each of 8192 queries, 32 / 8 heads, 1170 us / 1240).
#pragma unroll
    for (int turn = 0; turn < (PACK ? 2 : 1); ++turn) {
#pragma unroll
    for (int dv = 0; dv < Tile::COLS; ++dv) o[dv] = f32x16{0};
    ref = -INFINITY;
    l = 0.f;
    if (n_stage > 0) {
        load_stage(0, 0);
        settle_stage();
    }
    for (int t = 0; t < n_stage; ++t) {
        __syncthreads();  // stage t is there; every wave is done with stage t - 1
        if (t + 1 < n_stage) load_stage(t + 1, (t + 1) & 1);
        const char* const sk = smem + (t & 1) * Geo::STAGE;
#pragma unroll 1
        for (int j = wave % KS; j < STAGE; j += KS) {
            if (t * STAGE + j >= n_sub) break;
            const int key = __builtin_amdgcn_readfirstlane(keys[s_begin + t * STAGE + j]);
            if (key > reach) continue;
            const char* const ks = sk + j * Geo::SUB;
            const char* const vs = ks + STAGE * Geo::SUB;
            f32x16 acc = {0};
#pragma unroll
            for (int c = 0; c < Tile::CHUNKS; ++c) mma_chunk<bf16_t>(acc, Tile::row_fragment(ks, c, lane), qf[c]);  // acc[key][row]
            int mine = lim;
            bool whole = key + 31 <= clean;
            if constexpr (PACK) {
                const unsigned bits = keys[room + s_begin + t * STAGE + j];
                whole = whole && __popc(bits) == p.pack;
                mine = bits >> member & 1 ? lim : -1;
            }
            if (!whole) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = key + acc_row(r, lane) <= mine ? acc[r] : -INFINITY;
            }
            float top = acc[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) top = fmaxf(top, acc[r]);
            top = half_waves_max(top * p.c2);
            // the reference only moves when a tile exceeds it by more than 2^8: binary32 and bf16 hold what is below as well as 1
            const float moved = top > ref + 8.f ? top : ref;
            const float at = moved == -INFINITY ? 0.f : moved;  // nothing allowed so far: keep the arguments finite
            const float corr = __builtin_amdgcn_exp2f(ref - at);
            float pr[16], s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                pr[r] = __builtin_amdgcn_exp2f(fmaf(acc[r], p.c2, -at));
                if (r & 1) s1 += pr[r]; else s0 += pr[r];
            }
            l = fmaf(l, corr, s0 + s1);
            if (__any(moved > ref)) {
#pragma unroll
                for (int dv = 0; dv < Tile::COLS; ++dv)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dv][r] *= corr;
            }
            ref = moved;
            u32x4 pb[2];
#pragma unroll
            for (int c = 0; c < 2; ++c)
                pb[c] = u32x4{pack_bf16x2_hw(pr[8 * c + 0], pr[8 * c + 1]), pack_bf16x2_hw(pr[8 * c + 2], pr[8 * c + 3]),
                              pack_bf16x2_hw(pr[8 * c + 4], pr[8 * c + 5]), pack_bf16x2_hw(pr[8 * c + 6], pr[8 * c + 7])};
            if (turn == 0) {
#pragma unroll
                for (int dv = 0; dv < Tile::COLS; ++dv)
#pragma unroll
                    for (int c = 0; c < 2; ++c) mma_chunk<bf16_t>(o[dv], Tile::column_fragment(vs, dv, c, lane), pb[c]);  // o[value column][row]
            } else {
#pragma unroll
                for (int dv = 0; dv < Tile::COLS; ++dv) {
                    f32x16 sum = o[dv];
#pragma unroll
                    for (int c = 0; c < 2; ++c) mma_chunk<bf16_t>(sum, Tile::column_fragment(vs, dv, c, lane), pb[c]);
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dv][r] = key <= mine ? sum[r] : o[dv][r];
                }
            }
        }
        settle_stage();
    }
    if (!PACK || turn == 1) break;
    float zero = 0.f;
#pragma unroll
    for (int dv = 0; dv < Tile::COLS; ++dv)
#pragma unroll
        for (int r = 0; r < 16; ++r) zero = fmaf(o[dv][r], 0.f, zero);
    if (zero != 0.f) not_finite = 1;
    __syncthreads();
    if (!__builtin_amdgcn_readfirstlane(not_finite)) break;
    }

    // the waves that share rows bring their sums to the largest reference of them, in LDS (the stages are done with), and each finishes
    // its part of the rows, whole 16-byte pieces
    l += __shfl_xor(l, 32);
    __syncthreads();
    constexpr int LPR = D / 8;
    const int first = wave - wave % KS;
    float* const sums = reinterpret_cast<float*>(smem);
    float2* const stats = reinterpret_cast<float2*>(smem + WAVES * 32 * Geo::PITCH * 4);
    if (half == 0) stats[wave * 32 + l32] = make_float2(ref, l);
    __syncthreads();
    {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < KS; ++w) top = fmaxf(top, stats[(first + w) * 32 + l32].x);
        const float f = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top);
#pragma unroll
        for (int dv = 0; dv < Tile::COLS; ++dv)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(sums + (wave * 32 + l32) * Geo::PITCH + dv * 32 + q * 8 + half * 4) =
                    f32x4{o[dv][q * 4] * f, o[dv][q * 4 + 1] * f, o[dv][q * 4 + 2] * f, o[dv][q * 4 + 3] * f};
    }
    __syncthreads();
    const int c0 = lane % LPR * 8;
#pragma unroll
    for (int r = 0; r < 32 / KS; r += 64 / LPR) {
        const int in = wave % KS * (32 / KS) + r + lane / LPR, out = row0 + in;
        if (64 / LPR > 32 / KS && r + lane / LPR >= 32 / KS) continue;
        if (out >= rows) continue;
        float top = -INFINITY, total = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < KS; ++w) top = fmaxf(top, stats[(first + w) * 32 + in].x);
#pragma unroll
        for (int w = 0; w < KS; ++w) {
            const int at = (first + w) * 32 + in;
            const float2 st = stats[at];
            total += st.x == -INFINITY ? 0.f : st.y * __builtin_amdgcn_exp2f(st.x - top);
            const f32x4 lo = *reinterpret_cast<const f32x4*>(sums + at * Geo::PITCH + c0), hi = *reinterpret_cast<const f32x4*>(sums + at * Geo::PITCH + c0 + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[e + 4] += hi[e]; }
        }
        if (p.n_parts > 1) {
            float* part = p.parts + ((((long long)qb * p.H_kv + g) * p.n_parts + share) * p.R + out) * PART_ROW<D>;
            *reinterpret_cast<f32x4*>(part + c0) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(part + c0 + 4) = f32x4{v[4], v[5], v[6], v[7]};
            if (c0 == 0) *reinterpret_cast<float2*>(part + D) = make_float2(top, total);
            continue;
        }
        const long long i = (long long)qb * p.bq + out / p.G;
        const int h = g * p.G + out % p.G;
        const float inv = total == 0.f ? 0.f : 1.f / total;  // a row that sees no key: zeros
        u32x4 piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) piece[e] = pack_bf16x2_hw(v[2 * e] * inv, v[2 * e + 1] * inv);
        *reinterpret_cast<u32x4*>(p.O + i * p.o_ts + (long long)h * p.o_hs + c0) = piece;
        if (p.lse2 && c0 == 0) p.lse2[(long long)h * p.S_q + i] = total == 0.f ? -INFINITY : top + log2f(total);
    }
}

// Joins the shares of a list: a row's D / 8 lanes take the parts in their order.
template <int D> __global__ __launch_bounds__(256) void block_attention_join_kernel(BlockAttnParams p) {
    constexpr int LPR = D / 8;
    const long long n = (long long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    if (n >= (long long)p.n_qb * p.H_kv * p.R) return;
    const int row = (int)(n % p.R), g = (int)(n / p.R % p.H_kv), c0 = threadIdx.x % LPR * 8;
    const long long qb = n / p.R / p.H_kv;
    const long long i = qb * p.bq + row / p.G;
    if (i >= p.S_q) return;
    const int h = g * p.G + row % p.G;
    const float* const part = p.parts + ((qb * p.H_kv + g) * p.n_parts * p.R + row) * PART_ROW<D>;
    const long long pitch = (long long)p.R * PART_ROW<D>;
    float top = -INFINITY, total = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < p.n_parts; ++w) top = fmaxf(top, part[w * pitch + D]);
    for (int w = 0; w < p.n_parts; ++w) {
        const float2 st = *reinterpret_cast<const float2*>(part + w * pitch + D);
        const float f = st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - top);
        total += st.y * f;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(part + w * pitch + c0), hi = *reinterpret_cast<const f32x4*>(part + w * pitch + c0 + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = fmaf(lo[e], f, v[e]); v[e + 4] = fmaf(hi[e], f, v[e + 4]); }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    u32x4 piece;
#pragma unroll
    for (int e = 0; e < 4; ++e) piece[e] = pack_bf16x2_hw(v[2 * e] * inv, v[2 * e + 1] * inv);
    *reinterpret_cast<u32x4*>(p.O + i * p.o_ts + (long long)h * p.o_hs + c0) = piece;
    if (p.lse2 && c0 == 0) p.lse2[(long long)h * p.S_q + i] = total == 0.f ? -INFINITY : top + log2f(total);
}

// Rows of a workgroup by the rows that share a list: no more waves than have rows, the others share.  `walk`: there may be workgroups that
// walk over the lists (not for single tokens, whose sequences have keys and lengths of their own).
int block_attention_tile_rows(int R, bool walk) { return R > 128 && walk ? 256 : R > 64 ? 128 : R > 32 ? 64 : 32; }

// Lists of few rows together, as many as fill 32 rows; the union of what they name has to fit the workgroup's memory.  us one by one /
// together, a list for every query: 1000 queries, 16 / 4 heads of 64, 8 blocks of 32 52.5 / 17.2 (gradients 87 / 53); 3001, 16 of 64, 12
// blocks 697 / 85 (794 / 165); 8192, 32 / 8 of 128, 16 blocks of 64 2672 / 1167 (4484 / 2024).
static int block_attention_pack(int R, int T, int b, long long nb, long long lists) {
    int pack = R >= 32 ? 1 : 32 / R;
    if (nb > 16384) return 1;
    while (pack > 1 && (pack > lists || (pack * (long long)T < nb ? pack * (long long)T : nb) * (b / 32) > MAX_PACKED_SUBTILES)) --pack;
    return pack;
}

// Makes the lists that are worked on together one query block; returns the subtiles that its list may have.
int block_attention_packed(BlockAttnParams& p) {
    const int nb = p.nb;
    p.n_lists = p.n_qb;
    p.pack = p.lengths ? 1 : block_attention_pack(p.R, p.T, p.b, nb, p.n_qb);
    if (p.pack == 1) return p.T * (p.b / 32);
    p.bq *= p.pack;
    p.R *= p.pack;
    p.n_qb = (p.n_qb + p.pack - 1) / p.pack;
    return (p.pack * p.T < nb ? p.pack * p.T : nb) * (p.b / 32);
}

// Shares of a list: a workgroup for every CU, at least a stage each.
int block_attention_parts(long long tiles, long long subtiles) {
    const long long most = (subtiles + 3) / 4;
    long long parts = tiles >= 256 ? 1 : (256 + tiles - 1) / tiles;
    if (parts > most) parts = most;
    return parts < 1 ? 1 : (int)parts;
}

template <int D> constexpr int FEW = D == 128 ? 2 : 4;  // waves that share lists of few rows, where there are many of these

template <int D, int WAVES, int KS> constexpr int ba_lds(int subtiles) { return BaGeo<D, WAVES, BA_STAGE<D, KS>>::lds(subtiles); }

template <int D> static int prepare_block_attention() {
    static const int err = raise_lds_limits({{reinterpret_cast<const void*>(&block_attention_kernel<D, 4, 1, false>), ba_lds<D, 4, 1>(MAX_LISTED_SUBTILES)},
                                             {reinterpret_cast<const void*>(&block_attention_kernel<D, 4, 2, false>), ba_lds<D, 4, 2>(MAX_LISTED_SUBTILES)},
                                             {reinterpret_cast<const void*>(&block_attention_kernel<D, FEW<D>, FEW<D>, false>), ba_lds<D, FEW<D>, FEW<D>>(MAX_LISTED_SUBTILES)},
                                             {reinterpret_cast<const void*>(&block_attention_kernel<D, FEW<D>, FEW<D>, true>), ba_lds<D, FEW<D>, FEW<D>>(2 * MAX_PACKED_SUBTILES)},
                                             {reinterpret_cast<const void*>(&block_attention_kernel<D, 4, 4, false>), ba_lds<D, 4, 4>(MAX_LISTED_SUBTILES)},
                                             {reinterpret_cast<const void*>(&block_attention_kernel<D, 4, 4, true>), ba_lds<D, 4, 4>(2 * MAX_PACKED_SUBTILES)}});
    return err;
}

template <int D, int WAVES, int KS, bool PACK> static int run_block_attention(BlockAttnParams p, int subtiles, hipStream_t st) {
    return launch_in_turns((long long)p.n_qb * p.n_rt * p.n_parts * p.H_kv, WAVES * 64, [&](long long first, unsigned count) {
        p.first = (int)first;
        hipLaunchKernelGGL((block_attention_kernel<D, WAVES, KS, PACK>), dim3(count), dim3(WAVES * 64), (ba_lds<D, WAVES, KS>(PACK ? 2 * subtiles : subtiles)), st, p);
    });
}

template <int D> static int launch_block_attention_d(BlockAttnParams p, hipStream_t st) {
    const int unready = D == 128 ? first_error(prepare_block_attention<D>, prepare_block_attention_pipe) : prepare_block_attention<D>();
    if (unready) return unready;
    const int subtiles = block_attention_packed(p);
    const int tile = block_attention_tile_rows(p.R, D == 128 && !p.lengths);
    p.n_rt = (p.R + tile - 1) / tile;
    p.n_parts = p.parts ? block_attention_parts((long long)p.n_qb * p.n_rt * p.H_kv, subtiles) : 1;
    p.order = head_order(p.H_kv, false, 8);
    // lists of few rows: four waves share them; many of them, heads of 128: two waves with stages of 64 keys, so that two workgroups fit a CU
    // (us, 4 / 2 waves: one token of 1, 8, 64, 256 sequences, 32 / 8 heads, 16 blocks of 64: 14.8 / 16.1, 15.8 / 18.9, 53.5 / 50.8, 217 / 207;
    // 8192 tokens, 32 heads, a list for 16: 1134 / 1070, 16 heads, 12 blocks of 32: 315 / 278)
    const bool many = D == 128 && (long long)p.n_qb * p.n_parts * p.H_kv >= 512;
    const int rc = tile == 256 ? launch_block_attention_pipe(p, st) : tile == 128 ? run_block_attention<D, 4, 1, false>(p, subtiles, st)
                 : tile == 64 ? run_block_attention<D, 4, 2, false>(p, subtiles, st)
                 : p.pack == 1 ? (many ? run_block_attention<D, FEW<D>, FEW<D>, false>(p, subtiles, st) : run_block_attention<D, 4, 4, false>(p, subtiles, st))
                 : many ? run_block_attention<D, FEW<D>, FEW<D>, true>(p, subtiles, st) : run_block_attention<D, 4, 4, true>(p, subtiles, st);
    if (rc || p.n_parts == 1) return rc;
    const long long rows = (long long)p.n_qb * p.H_kv * p.R, per = 256 / (D / 8);
    hipLaunchKernelGGL((block_attention_join_kernel<D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, p);
    return (int)hipGetLastError();
}

int launch_block_attention(BlockAttnParams p, int d, hipStream_t st) { return d == 64 ? launch_block_attention_d<64>(p, st) : launch_block_attention_d<128>(p, st); }

}  // namespace lemo
