// The products of the loss over a vocabulary (bf16), on the main loops of the selective-load GEMM, with what is done to a tile while it is still in
// registers:
//
//   statistics      x = X[idx] W^T: of every row of a tile its largest logit, the sum of exponentials against that, the sum of logits (smoothed
//                   labels) and the label's logit.  8 to 12 bytes a row leave the tile in the place of 512.
//   probabilities   the same product again, turned into the gradient of the logits with the row's log-sum-exp: G, bf16, one piece of the
//                   vocabulary at a time.  bf16 because the two products that follow take it so: off by 2^-9 of each element, at random.
//                   The largest error is that of the label's element, whose rest dX gets back (vocab_planes_kernel); and one
//                   gradient for all losses is left out of G and multiplied into the results instead, since its rounding would be the same
//                   relative error in every label's element (4096 rows, 131072 words, mean: dX and dW 3.0e-3 from 64 bits, so 1.8e-3; their own store alone 1.7e-3).
//                   Up to 32 rows stand in G in two parts for dW, which few rows' labels would otherwise leave as far off again as its store.
//   planes          dX = G W over the piece's columns, in binary32: a piece adds to what the pieces before left, and where the
//                   output has few tiles the contraction is split, with a plane for each part; a kernel of its own rounds their sum once.
//   the weight's    dW = G^T X[idx], the piece's rows, times what was left out of G, rounded once.
//
// What bounds it: the matrix cores, as in gather_gemm_large.hip; the epilogues read no memory but a few bytes a row.  8192 rows, 4096 columns, 131072 words:
// statistics 6.1 to 6.3 ms by the card, 1.40 to 1.44 PFLOP/s, matrix cores busy for 75 % of the cycles; the gradients of 4096 rows 9.6 to 10.0 ms, 1.32 to 1.37 (probabilities 69 %, planes 73 %,
// the weight's 64 %).  Narrow rows are few slabs a tile, whose epilogue nothing overlaps: 256 columns take 1.75 times the products' time, the gradients 2.4.
#include "gather_gemm_tiles.hpp"
#include "vocab_softmax.hpp"

namespace lemo {

// A tile kind: UA = 0 the 256 x 256 tile, otherwise 64 UA x 128.  A lane holds ROWS rows (one of each 16-row tile of its wave) by 4 x 4 columns.
template <int LAYOUT, int UA> struct VocabTile {
    static constexpr bool LARGE = UA == 0;
    static constexpr int BM = LARGE ? LG_BM : 64 * UA, BN = LARGE ? LG_BN : 128;
    static constexpr int ROWS = LARGE ? 2 * LG_TA : UA, ACROSS = LARGE ? LG_WN : 2;  // ACROSS: waves along the columns
    static constexpr int PITCH = BN * 2 + 16;                                         // of a row of bf16 in LDS
    static constexpr int LDS_LOOP = LARGE ? LG_LDS : MdGeo<LAYOUT, LARGE ? 1 : UA>::LDS;
    static constexpr int LDS = LDS_LOOP > BM * PITCH ? LDS_LOOP : BM * PITCH;
    static constexpr int GROUP = LARGE ? 4 : UA <= 2 ? 16 / UA : 4;  // tile rows walked together
    using Acc = std::conditional_t<LARGE, f32x4[2][LG_TA][2][LG_TB], f32x4[LARGE ? 1 : UA][MD_TB]>;
    static_assert(LDS <= 160 * 1024 && ACROSS * BM * 12 <= LDS, "a workgroup's LDS");

    __device__ static __forceinline__ void product(const GgParams& p, long long m0, int n0, char* smem, Acc& acc) {
        if constexpr (LARGE) lg_product<LAYOUT>(p, m0, n0, smem, acc);
        else md_product<LAYOUT, UA>(p, m0, n0, smem, acc);
    }
    __device__ static __forceinline__ f32x4& at(Acc& acc, int i, int j) {
        if constexpr (LARGE) return acc[i / LG_TA][i % LG_TA][j / LG_TB][j % LG_TB];
        else return acc[i][j];
    }
    __device__ static __forceinline__ int across(int wave) { return LARGE ? wave % LG_WN : wave & 1; }
    __device__ static __forceinline__ int row(int wave, int lane, int i) {
        if constexpr (LARGE) return i / LG_TA * 128 + (wave / LG_WN * LG_TA + i % LG_TA) * 16 + (lane & 15);
        else return md_a_tile<LAYOUT, LARGE ? 1 : UA>(wave >> 1, i) * 16 + (lane & 15);
    }
    __device__ static __forceinline__ int col(int wave, int lane, int j) {  // the first of four
        if constexpr (LARGE) return j / LG_TB * 128 + (wave % LG_WN * LG_TB + j % LG_TB) * 16 + (lane >> 4) * 4;
        else return ((wave & 1) * MD_TB + j) * 16 + (lane >> 4) * 4;
    }
};

// Over the lanes of a row: lane, lane ^ 16, lane ^ 32, lane ^ 48.  The swaps leave a lane's value and its partner's in two registers.
__device__ __forceinline__ float2 swapped32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float2 swapped16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float row_lanes_max(float v) {
    const float2 a = swapped32(v);
    const float2 b = swapped16(fmaxf(a.x, a.y));
    return fmaxf(b.x, b.y);
}
__device__ __forceinline__ float row_lanes_sum(float v) {
    const float2 a = swapped32(v);
    const float2 b = swapped16(a.x + a.y);
    return b.x + b.y;
}

constexpr int vocab_layout(int what) { return what == VOCAB_PLANES ? GG_NN : what == VOCAB_WEIGHT ? GG_TN : GG_NT; }

// rows of bf16 in LDS -> rows of a matrix, whose columns below `cols` (a multiple of 8) are written.  In two parts (of up to BM / 2 rows): the second half's go behind the first's.
template <typename Tile> __device__ __forceinline__ void store_rows(const char* smem, int wave, int lane, void* to, long long ld, long long m0, long long M, int n0, int cols, bool two = false) {
    constexpr int LPR = Tile::BN / 8, RPP = 64 / LPR, OWN = Tile::BM / RG_WAVES;  // lanes of a row, rows at a time, rows of a wave
    const int c = lane % LPR * 8;
    if (n0 + c >= cols) return;
#pragma unroll 4
    for (int k = 0; k < OWN / RPP; ++k) {
        const int row = wave * OWN + k * RPP + lane / LPR;
        long long m = m0 + (two ? row % (Tile::BM / 2) : row);
        if (m >= M) continue;
        if (two && row >= Tile::BM / 2) m += M;
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(to) + m * ld + n0 + c) = *reinterpret_cast<const u32x4*>(smem + row * Tile::PITCH + c * 2);
    }
}

// softcap, in place
template <typename Tile> __device__ __forceinline__ void cap_tile(const VocabRule& rule, typename Tile::Acc& acc) {
    if (rule.softcap <= 0.f) return;
    const float inv_cap = 1.f / rule.softcap;
#pragma unroll
    for (int i = 0; i < Tile::ROWS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) Tile::at(acc, i, j)[r] = vocab_cap(Tile::at(acc, i, j)[r], rule.softcap, inv_cap);
}

// The statistics of tile (m0, column tile tn).  labels(row, i) of the rows of a lane; red [3][ACROSS][BM] in LDS: maxima, sums of exponentials, sums.
template <typename Tile, class Labels>
__device__ __forceinline__ void tile_stats(const VocabTileParams& p, typename Tile::Acc& acc, Labels&& labels, float* red, int tid, long long m0, int tn) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n0 = tn * Tile::BN;
    const bool whole = n0 + Tile::BN <= p.N;
    cap_tile<Tile>(p.rule, acc);
#pragma unroll
    for (int i = 0; i < Tile::ROWS; ++i) {
        const int row = Tile::row(wave, lane, i);
        const long long m = min(m0 + row, p.M - 1);
        float top = -INFINITY, sum, all = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x4& v = Tile::at(acc, i, j);
            if (!whole) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n0 + Tile::col(wave, lane, j) + r >= p.N) v[r] = -INFINITY;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, v[r]);
        }
        // the label's logit: few tiles hold one (a label outside the vocabulary is no column below N)
        const unsigned label = (unsigned)labels(row, i) - (unsigned)(p.v0 + n0);
        if (__any(label < (unsigned)min(Tile::BN, p.N - n0))) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned at = label - (unsigned)Tile::col(wave, lane, j);
                const f32x4 v = Tile::at(acc, i, j);
                if (at < 4u && label < (unsigned)(p.N - n0)) p.picked[m] = at < 2 ? at ? v[1] : v[0] : at == 2 ? v[2] : v[3];
            }
        }
        top = row_lanes_max(top);
        const float base = top == -INFINITY ? 0.f : top * LOG2E;
        f32x4 some = {0.f, 0.f, 0.f, 0.f};  // (four chains of additions)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) some[r] += __builtin_amdgcn_exp2f(fmaf(Tile::at(acc, i, j)[r], LOG2E, -base));
        sum = row_lanes_sum((some[0] + some[1]) + (some[2] + some[3]));
        if (p.sums) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) all += whole || n0 + Tile::col(wave, lane, j) + r < p.N ? Tile::at(acc, i, j)[r] : 0.f;
            all = row_lanes_sum(all);
        }
        if (lane < 16) {
            float* const to = red + Tile::across(wave) * Tile::BM + row;
            to[0] = top;
            to[Tile::ACROSS * Tile::BM] = sum;
            to[2 * Tile::ACROSS * Tile::BM] = all;
        }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // (in a run: the next tile's first slabs)
    __syncthreads();
    const int row = tid;
    if (row < Tile::BM && m0 + row < p.M) {
        float top = red[row], sum = red[Tile::ACROSS * Tile::BM + row], all = red[2 * Tile::ACROSS * Tile::BM + row];
#pragma unroll
        for (int w = 1; w < Tile::ACROSS; ++w) {
            const float* const from = red + w * Tile::BM + row;
            vocab_join(top, sum, from[0], from[Tile::ACROSS * Tile::BM]);
            all += from[2 * Tile::ACROSS * Tile::BM];
        }
        const long long to = (long long)tn * p.M + m0 + row;
        p.parts[to] = make_float2(top, sum);
        if (p.sums) p.sums[to] = all;
    }
}

template <int WHAT, int UA>
__global__ __launch_bounds__(RG_THREADS, 1) void vocab_tile_kernel(VocabTileParams p) {
    constexpr int LAYOUT = vocab_layout(WHAT);
    using Tile = VocabTile<LAYOUT, UA>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tm, tn, split = 0;
    GgParams q = p;
    if constexpr (WHAT == VOCAB_PLANES) {
        if (!gg_part_tile(blockIdx.x, p.splits, p.tiles_m, p.tiles_n, Tile::GROUP, split, tm, tn)) return;
        const int k0 = split * p.k_split;  // (host: below the contraction's length for every split)
        q.A = static_cast<const bf16_t*>(p.A) + k0;
        q.B = static_cast<const bf16_t*>(p.B) + (long long)k0 * p.ldb;
        q.K = min(p.k_split, p.K - k0);
        q.a_bytes = p.a_bytes - (unsigned)k0 * 2u;
    } else {
        if (!gg_tile(blockIdx.x, p.tiles_m, p.tiles_n, Tile::GROUP, tm, tn)) return;
    }
    const long long m0 = (long long)tm * Tile::BM;
    const int n0 = tn * Tile::BN;
    typename Tile::Acc acc;
    Tile::product(q, m0, n0, smem, acc);

    if constexpr (WHAT == VOCAB_PLANES) {
        float* const plane = p.planes + (long long)split * p.M * p.N;
#pragma unroll
        for (int i = 0; i < Tile::ROWS; ++i) {
            const long long m = m0 + Tile::row(wave, lane, i);
            if (m >= p.M) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = n0 + Tile::col(wave, lane, j);
                if (n >= p.N) continue;  // (N is a multiple of 8)
                f32x4* const to = reinterpret_cast<f32x4*>(plane + m * p.N + n);
                f32x4 v = Tile::at(acc, i, j);
                if (p.add) v += *to;
                *to = v;
            }
        }
        return;
    }
    if constexpr (WHAT == VOCAB_WEIGHT) {
        float scale = p.scale ? *p.scale * p.scale_by : 1.f;
        if (!isfinite(scale)) {  // (the same in all threads)  Where no row counts, nothing is added, whatever their gradient holds
            int* const some = reinterpret_cast<int*>(smem);
            if (tid == 0) *some = 0;
            __syncthreads();
            for (long long m = tid; m < p.n_labels; m += RG_THREADS)
                if (p.labels[m] >= 0 && p.labels[m] < p.rule.V) *some = 1;
            __syncthreads();
            if (*some == 0) scale = 0.f;
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < Tile::ROWS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 v = Tile::at(acc, i, j) * scale;
                *reinterpret_cast<uint2*>(smem + Tile::row(wave, lane, i) * Tile::PITCH + Tile::col(wave, lane, j) * 2) =
                    make_uint2(pack_bf16x2_hw(v[0], v[1]), pack_bf16x2_hw(v[2], v[3]));
            }
        __syncthreads();
        store_rows<Tile>(smem, wave, lane, p.Y, p.ldy, m0, p.M, n0, p.N);
        return;
    }
    if constexpr (WHAT == VOCAB_STATS) {
        int labels[Tile::ROWS];
#pragma unroll
        for (int i = 0; i < Tile::ROWS; ++i) labels[i] = p.labels[min(m0 + Tile::row(wave, lane, i), p.M - 1)];
        tile_stats<Tile>(p, acc, [&](int, int i) { return labels[i]; }, reinterpret_cast<float*>(smem), tid, m0, tn);
        return;
    }
    const bool whole = n0 + Tile::BN <= p.N, capped = p.rule.softcap > 0.f;
    const float inv_cap = capped ? 1.f / p.rule.softcap : 0.f;
    cap_tile<Tile>(p.rule, acc);
    if constexpr (WHAT == VOCAB_PROBS) {
        const bool two = UA == 1 && p.side.parts == 2;  // (host: up to half the rows of the smallest tile, whose other half holds what rounding has left)
        constexpr int LEFT = Tile::BM / 2 * Tile::PITCH;
        if (p.side.rows) {
            if (tn == 0 && tid < Tile::BM && m0 + tid < p.M) vocab_list_row(p.rule, p.side, p.labels, p.idx, m0 + tid, p.M);
            if (p.side.zero_row && tm == p.tiles_m - 1 && tid < Tile::BN / 8 && n0 + tid * 8 < p.N)
                *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.G) + p.side.parts * p.M * p.ldg + n0 + tid * 8) = u32x4{0u, 0u, 0u, 0u};
        }
        VocabRow rows[Tile::ROWS];
#pragma unroll
        for (int i = 0; i < Tile::ROWS; ++i) {
            const long long m = min(m0 + Tile::row(wave, lane, i), p.M - 1);
            rows[i] = vocab_row_of(p.rule, p.side, p.lse, p.labels, m);
        }
#pragma unroll
        for (int i = 0; i < Tile::ROWS; ++i) {
            const int row = Tile::row(wave, lane, i);
            if (two && row >= Tile::BM / 2) continue;
            const long long m = min(m0 + row, p.M - 1);
            const VocabRow of = rows[i];
            const uint32_t mask = of.counts ? ~0u : 0u;
            char* const to = smem + row * Tile::PITCH;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = Tile::col(wave, lane, j);
                float g[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) g[r] = vocab_share(of, Tile::at(acc, i, j)[r]);
                if (capped) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) g[r] = vocab_slope(p.rule, g[r], Tile::at(acc, i, j)[r], inv_cap);
                }
                if (!whole) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) g[r] = n0 + c + r < p.N ? g[r] : 0.f;
                }
                const uint2 v = make_uint2(pack_bf16x2_hw(g[0], g[1]), pack_bf16x2_hw(g[2], g[3]));
                *reinterpret_cast<uint2*>(to + c * 2) = make_uint2(v.x & mask, v.y & mask);
                if (two)
                    *reinterpret_cast<uint2*>(to + LEFT + c * 2) = make_uint2(pack_bf16x2_hw(g[0] - bf16lo_to_f32(v.x), g[1] - bf16hi_to_f32(v.x)) & mask,
                                                                              pack_bf16x2_hw(g[2] - bf16lo_to_f32(v.y), g[3] - bf16hi_to_f32(v.y)) & mask);
            }
            // the label's element, over what the lane has just written there: few tiles hold one
            const unsigned label = (unsigned)of.label - (unsigned)(p.v0 + n0);
            if (__any(label < (unsigned)min(Tile::BN, p.N - n0))) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned at = label - (unsigned)Tile::col(wave, lane, j);
                    if (at >= 4u || label >= (unsigned)(p.N - n0)) continue;
                    const f32x4 v = Tile::at(acc, i, j);
                    const float g = vocab_grad(p.rule, of, at < 2 ? at ? v[1] : v[0] : at == 2 ? v[2] : v[3], true, inv_cap);
                    const uint32_t stored = pack_bf16x2_hw(g, 0.f);
                    const float left = g - bf16lo_to_f32(stored);
                    *reinterpret_cast<uint16_t*>(to + label * 2) = (uint16_t)stored;
                    if (two) *reinterpret_cast<uint16_t*>(to + LEFT + label * 2) = (uint16_t)pack_bf16x2_hw(left, 0.f);
                    p.rest[m] = left;
                }
            }
        }
        __syncthreads();
        store_rows<Tile>(smem, wave, lane, p.G, p.ldg, m0, p.M, n0, (p.N + 7) & ~7, two);
    }
}

// Statistics of 256 x 256 tiles by 256 workgroups, each for runs of tiles of the same rows: a tile's first slabs are on their way during the statistics of the one
// before.  A die has a part of the tiles in grouped order, four rows of tiles by a range of columns at a time (or two, or one), whose columns go round its
// workgroups: at any time four of them read the same columns and eight the same rows.  4096 rows, 131072 words: 256 columns 376 -> 303 us, 512 555 -> 471, 1024 918 -> 856;
// wide rows have little to hide and their workgroups fall out of step (2048 columns as long either way, 4096 3 % longer), and one tile a workgroup
// has no next (300 rows of 512, 32000 words 25.4, so 25.8).
constexpr int VR_WIDEST = 1536;
constexpr int VR_GRID = 256, VR_PER_XCD = VR_GRID / NUM_XCD, VR_RED = LG_TOK, VR_LABELS = VR_RED + 3 * LG_WN * LG_BM * 4, VR_LDS = VR_LABELS + LG_BM * 4;
static_assert(VR_LDS <= 160 * 1024, "a workgroup's LDS");
using VrTile = VocabTile<GG_NT, 0>;
struct StatsRun {
    static constexpr bool MORE = true;
    const VocabTileParams& p;
    char* smem;
    long long m0;
    int tn, step, end;  // column tiles
    u32x4 b[2];         // descriptors of this tile's columns and of the next one's
    __device__ __forceinline__ StatsRun(const VocabTileParams& p, char* smem, long long m0, int tn, int step, int end) : p(p), smem(smem), m0(m0), tn(tn), step(step), end(end) {
        b[0] = columns(tn);
        b[1] = columns(tn + step);
    }
    __device__ __forceinline__ u32x4 columns(int t) const {
        const int n0 = min(t, p.tiles_n - 1) * LG_BN;
        u32x4 r = raw_rsrc(static_cast<const bf16_t*>(p.B) + (long long)n0 * p.ldb, (unsigned)(min(LG_BN, p.N - n0) - 1) * (unsigned)p.ldb * 2 + (unsigned)p.K * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_readfirstlane(r[e]);
        return r;
    }
    template <class Loads> __device__ __forceinline__ int slabs(const Loads& ld) const { return (ld.nk + 1) / 2 * 2; }
    template <class Loads> __device__ __forceinline__ typename Loads::Slab slab(const Loads& ld, int kt) const { return of(ld, kt, b[0], true); }
    template <class Loads> __device__ __forceinline__ typename Loads::Slab next(const Loads& ld, int kt) const { return of(ld, kt, b[1], tn + step < end); }
    template <class Loads> __device__ __forceinline__ typename Loads::Slab of(const Loads& ld, int kt, u32x4 columns, bool some) const {
        typename Loads::Slab s;
        s.soff = min(kt, ld.nk - 1) * RG_KB;  // (a slab behind the contraction: offsets at the descriptors' sizes or past them, zeros)
        s.in_k = some && ld.kpos < ld.K * 2 - kt * RG_KB;
        s.a = raw_rsrc(ld.a_base, ld.a_size);
        s.b = columns;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s.a[e] = __builtin_amdgcn_readfirstlane(s.a[e]);
            s.b[e] = __builtin_amdgcn_readfirstlane(s.b[e]);
        }
        return s;
    }
    __device__ __forceinline__ bool done(VrTile::Acc& acc) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));  // (what comes of it is not kept in registers through the products)
        const int* const labels = reinterpret_cast<const int*>(smem + VR_LABELS);
        tile_stats<VrTile>(p, acc, [&](int row, int) { return labels[row]; }, reinterpret_cast<float*>(smem + VR_RED), tid, m0, tn);
        tn += step;
        b[0] = b[1];
        b[1] = columns(tn + step);
        return tn < end;
    }
};
__global__ __launch_bounds__(RG_THREADS, 1) void vocab_stats_run_kernel(VocabTileParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int xcd = blockIdx.x % NUM_XCD, w = blockIdx.x / NUM_XCD;
    const long long total = (long long)p.tiles_m * p.tiles_n, from = total * xcd / NUM_XCD, to = total * (xcd + 1) / NUM_XCD;
    long long before = 0;  // tiles of the groups before
    for (int g = 0, rows; g < p.tiles_m; g += rows) {
        rows = p.tiles_m - g >= 4 ? 4 : p.tiles_m - g >= 2 ? 2 : 1;
        const int first = (int)min(max(from - before, 0ll) / rows, (long long)p.tiles_n), last = (int)min(max(to - before, 0ll) / rows, (long long)p.tiles_n);
        before += (long long)rows * p.tiles_n;
        const int step = VR_PER_XCD / rows, start = first + w / rows;
        if (start >= last) continue;
        const long long m0 = (long long)(g + w % rows) * LG_BM;
        if (threadIdx.x < LG_BM) reinterpret_cast<int*>(smem + VR_LABELS)[threadIdx.x] = p.labels[min(m0 + (int)threadIdx.x, p.M - 1)];  // (seen by all after the products' barriers)
        VrTile::Acc acc;
        lg_product<GG_NT>(p, m0, start * LG_BN, smem, acc, StatsRun(p, smem, m0, start, step, last));
    }
}
static int launch_stats_run(VocabTileParams p, hipStream_t st) {
    p.tiles_m = (int)((p.M + LG_BM - 1) / LG_BM);
    p.tiles_n = (p.N + LG_BN - 1) / LG_BN;
    hipLaunchKernelGGL(vocab_stats_run_kernel, dim3(VR_GRID), dim3(RG_THREADS), VR_LDS, st, p);
    return (int)hipGetLastError();
}

template <int WHAT, int UA> constexpr LdsLimit vocab_limit() { return {reinterpret_cast<const void*>(&vocab_tile_kernel<WHAT, UA>), VocabTile<vocab_layout(WHAT), UA>::LDS}; }
template <int WHAT> static int prepare_what() {
    static const int err = [] {
        if constexpr (WHAT == VOCAB_STATS)
            return raise_lds_limits({{reinterpret_cast<const void*>(&vocab_stats_run_kernel), VR_LDS}, vocab_limit<WHAT, 0>(), vocab_limit<WHAT, 1>(), vocab_limit<WHAT, 2>(), vocab_limit<WHAT, 4>()});
        else if constexpr (WHAT == VOCAB_WEIGHT) return raise_lds_limits({vocab_limit<WHAT, 0>(), vocab_limit<WHAT, 2>(), vocab_limit<WHAT, 4>()});
        else return raise_lds_limits({vocab_limit<WHAT, 0>(), vocab_limit<WHAT, 1>(), vocab_limit<WHAT, 2>(), vocab_limit<WHAT, 4>()});
    }();
    return err;
}
int prepare_vocab_tiles() {
    return first_error(prepare_what<VOCAB_STATS>, prepare_what<VOCAB_PROBS>, prepare_what<VOCAB_PLANES>, prepare_what<VOCAB_WEIGHT>);
}

int vocab_tile_cols(GgTile tile) { return tile == GG_T256 ? 256 : 128; }

template <int WHAT, int UA> static int launch_one(VocabTileParams p, hipStream_t st) {
    using Tile = VocabTile<vocab_layout(WHAT), UA>;
    p.tiles_m = (int)((p.M + Tile::BM - 1) / Tile::BM);
    p.tiles_n = (p.N + Tile::BN - 1) / Tile::BN;
    const long long blocks = ((long long)p.tiles_m * p.tiles_n * (WHAT == VOCAB_PLANES ? p.splits : 1) + NUM_XCD - 1) / NUM_XCD * NUM_XCD;
    if (blocks * RG_THREADS >= 1ll << 32) return (int)hipErrorInvalidValue;  // (the callers' pieces are far below)
    hipLaunchKernelGGL((vocab_tile_kernel<WHAT, UA>), dim3((unsigned)blocks), dim3(RG_THREADS), Tile::LDS, st, p);
    return (int)hipGetLastError();
}
template <int WHAT> static int launch_what(const VocabTileParams& p, GgTile tile, hipStream_t st) {
    switch (tile) {
        case GG_T256:
            if constexpr (WHAT == VOCAB_STATS) {
                if (p.K <= VR_WIDEST && (p.M + LG_BM - 1) / LG_BM * ((p.N + LG_BN - 1) / LG_BN) > VR_GRID) return launch_stats_run(p, st);
            }
            return launch_one<WHAT, 0>(p, st);
        case GG_T256x128: return launch_one<WHAT, 4>(p, st);
        case GG_T128: return launch_one<WHAT, 2>(p, st);
        default:
            if constexpr (WHAT == VOCAB_WEIGHT) return (int)hipErrorInvalidValue;  // (contraction-major rows come in whole regions)
            else return launch_one<WHAT, 1>(p, st);
    }
}
int launch_vocab_tiles(VocabTileParams p, int what, GgTile tile, hipStream_t st) {
    switch (what) {
        case VOCAB_STATS: return launch_what<VOCAB_STATS>(p, tile, st);
        case VOCAB_PROBS: return launch_what<VOCAB_PROBS>(p, tile, st);
        case VOCAB_PLANES: return launch_what<VOCAB_PLANES>(p, tile, st);
        default: return launch_what<VOCAB_WEIGHT>(p, tile, st);
    }
}

}  // namespace lemo
