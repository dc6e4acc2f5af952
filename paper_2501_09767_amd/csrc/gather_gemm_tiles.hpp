// The main loops of the selective-load GEMM kernels with workgroups of eight waves (bf16): a tile's product, in registers.  What is done with it is
// the kernels': gather_gemm_large.hip and gather_gemm_mid.hip, which describe the two schemes and what bounds them, store it or add it to the rows
// of a matrix; vocab_loss_tiles.hip takes a softmax's statistics or probabilities of it.
#pragma once
#include "gather_gemm_regions.hpp"

namespace lemo {

constexpr int LG_BM = 256, LG_BN = 256;
constexpr int LG_STAGE = 2 * RG_BYTES;   // regions: rows (columns of the output) 0-127, 128-255
constexpr int LG_OPER = 2 * LG_STAGE;    // two stages of A, then two of B: 64 KB, the reach of an LDS read's immediate offset
constexpr int LG_TOK = 2 * LG_OPER;      // (GG_TN) token rings
constexpr int LG_EP = LG_BN * 2 + 16;    // epilogue: LDS pitch of a row of bf16, ...
constexpr int LG_EPF = LG_BN * 4 + 16;   // ... of binary32 (128 rows at a time)
constexpr int LG_WN = 4;                 // waves along the columns
constexpr int LG_TA = 4, LG_TB = 2;      // 16-row tiles of a wave per half of A, of B
constexpr int LG_LDS_EPI = LG_BM * LG_EP > 128 * LG_EPF ? LG_BM * LG_EP : 128 * LG_EPF;
constexpr int LG_LDS = LG_TOK + RG_TOK > LG_LDS_EPI ? LG_TOK + RG_TOK : LG_LDS_EPI;
static_assert(LG_LDS <= 160 * 1024, "a workgroup's LDS");

// The product of a 256 x 256 tile at row m0, column n0: acc[a][i][b][j][r] is row a*128 + (wm*TA + i)*16 + lane % 16, column
// b*128 + (wn*TB + j)*16 + 4*(lane / 16) + r of the tile, wm = wave / LG_WN, wn = wave % LG_WN.  At the end nothing is on its way to LDS, and everyone is done with it.
//
// With a run that has MORE tiles (its first at m0, n0): what is asked for ahead in a tile's last slabs is the next tile's, run.next(), on its way while run.done(acc)
// does with the tile what is to be done; it leaves the stages alone, returns with all loads landed for everyone, and says whether there is another tile.
struct LgOne {
    static constexpr bool MORE = false;
    template <class Loads> __device__ __forceinline__ int slabs(const Loads& ld) const { return ld.nk; }
    template <class Loads> __device__ __forceinline__ typename Loads::Slab slab(const Loads& ld, int kt) const { return ld.slab(kt); }
    template <class Loads> __device__ typename Loads::Slab next(const Loads& ld, int kt) const;  // (there is none)
};
template <int LAYOUT, class Run = LgOne>
__device__ __forceinline__ void lg_product(const GgParams& p, long long m0, int n0, char* smem, f32x4 (&acc)[2][LG_TA][2][LG_TB], Run&& run = {}) {
    constexpr bool MORE = std::remove_reference_t<Run>::MORE;
    static_assert(!MORE || LAYOUT == GG_NT, "runs of tiles along the contraction");
    constexpr bool A_KMAJOR = LAYOUT == GG_TN, B_KMAJOR = LAYOUT != GG_NT;
    constexpr int TA = LG_TA, TB = LG_TB, NL = RG_NLD;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / LG_WN, wn = wave % LG_WN;
    using Loads = RgLoads<LAYOUT, 4, 4>;
    using Slab = typename Loads::Slab;
    Loads ld(p, m0, n0, tid, smem + LG_TOK + wave * 1024);
    const int nk = run.slabs(ld);  // (MORE: an even number)
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_offset_of(smem) + wave * 1024);
    auto load_a = [&](const Slab& s, int kt, int r, int i) { ld.load_a(s, 2 * r + i, lds0 + (kt & 1) * LG_STAGE); };
    auto load_b = [&](const Slab& s, int kt, int r, int i) { ld.load_b(s, 2 * r + i, lds0 + LG_OPER + (kt & 1) * LG_STAGE); };

    auto clear = [&] {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int j = 0; j < TB; ++j) acc[a][i][b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    clear();
    // fragments: the current half of A, both halves of B
    u32x4 fa[2][TA], fb[2][2][TB];
    unsigned at[2][2];  // (MORE) places of a chunk's first fragments of A, of B, which the compiler would otherwise add up for each read
    if constexpr (MORE) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int row = lane & 15, piece = (4 * c + (lane >> 4)) ^ ((row >> 1) & 7);  // as rg_fragment finds them
            at[0][c] = (wm * TA * 16 + row) * RG_KB + piece * 16;
            at[1][c] = LG_OPER + (wn * TB * 16 + row) * RG_KB + piece * 16;
            asm volatile("" : "+v"(at[0][c]), "+v"(at[1][c]));
        }
    }
    auto read_a = [&](int st, int r, int c, int i) {
        if constexpr (MORE) fa[c][i] = *reinterpret_cast<const u32x4*>(smem + at[0][c] + (st * LG_STAGE + r * RG_BYTES + i * 16 * RG_KB));
        else fa[c][i] = rg_fragment(smem + st * LG_STAGE + r * RG_BYTES, A_KMAJOR, wm * TA + i, c, lane);
    };
    auto read_b = [&](int st, int r, int c, int j) {
        if constexpr (MORE) fb[r][c][j] = *reinterpret_cast<const u32x4*>(smem + at[1][c] + (st * LG_STAGE + r * RG_BYTES + j * 16 * RG_KB));
        else fb[r][c][j] = rg_fragment(smem + LG_OPER + st * LG_STAGE + r * RG_BYTES, B_KMAJOR, wn * TB + j, c, lane);
    };

    constexpr int NM = 2 * TA * TB;  // MFMAs of a quarter
    // One quarter of a slab: the MFMAs of (half AH of A) x (half BH of B), `mem(q, c, i, j)` behind MFMA q, which is of chunk c
    // and tile (i, j).  The source order is the issue order.
    auto quarter = [&](auto ah, auto bh, bool by_columns, auto mem) {
        constexpr int AH = decltype(ah)::value, BH = decltype(bh)::value;
#pragma unroll
        for (int q = 0; q < NM; ++q) {  // the tiles back and forth, row by row or column by column: neighbours share a fragment
            const int c = q / (TA * TB), w = q % (TA * TB), u = by_columns ? w / TA : w / TB, v = by_columns ? w % TA : w % TB;
            const int back = by_columns ? TA - 1 - v : TB - 1 - v, t = u & 1 ? back : v, i = by_columns ? t : u, j = by_columns ? u : t;
            __builtin_amdgcn_sched_barrier(0);
            rg_mma(acc[AH][i][BH][j], fa[c][i], fb[BH][c][j]);
            mem(q, c, i, j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    auto load_region = [&](const Slab& s, int kt, bool a, int r) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            if (a) load_a(s, kt, r, i); else load_b(s, kt, r, i);
        }
    };

    // What would have been asked for in the halves before: {B 0} {A 0, B 1} of slab 0, {A 1 of 0, B 1 of 1}, {A 0, B 0 of 1}
    if constexpr (LAYOUT == GG_TN) {
        for (int kt = 0; kt < 4; ++kt) ld.issue_tokens(kt, lane);
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        asm volatile("" ::: "memory");
    }
    {
        const Slab s0 = run.slab(ld, 0), s1 = run.slab(ld, 1);
        ld.read_tokens(0);
        load_region(s0, 0, false, 0);
        load_region(s0, 0, true, 0);
        load_region(s0, 0, false, 1);
        load_region(s0, 0, true, 1);
        ld.read_tokens(1);
        load_region(s1, 1, false, 1);
        load_region(s1, 1, true, 0);
        load_region(s1, 1, false, 0);
        ld.read_tokens(2);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(5 * NL));
    rg_barrier();
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int j = 0; j < TB; ++j) read_b(0, 0, c, j);
#pragma unroll
        for (int i = 0; i < TA; ++i) read_a(0, 0, c, i);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(3 * NL));
    __builtin_amdgcn_s_waitcnt(LGKMCNT0);

    // Waves of one SIMD do not take turns: one of them goes first (X W^T 752 -> 742 us at 8192^3, the gradients no change)
    auto go_first = [&] {
        if constexpr (LAYOUT == GG_NT)
            if (wave < RG_WAVES / 2) __builtin_amdgcn_s_setprio(1);
    };
    go_first();
    // Slab kt, kt & 1 == PAR.  Halves of a slab begin with a barrier, before which every wave has seen to it that the regions
    // read in this half have landed (its own part: all loads but the last IN_FLIGHT, which complete in order) and that it
    // has read what this half's loads overwrite: all but the fragments read in the quarter before.
    constexpr int IN_FLIGHT = 3 * NL;
    auto ahead = [&](int kt, auto next_tag) {  // slab kt, or of the next tile
        if constexpr (decltype(next_tag)::value < 0) return run.slab(ld, kt);
        else return run.next(ld, decltype(next_tag)::value);
    };
    auto slab = [&](int kt, auto par_tag, auto next1, auto next2) {
        constexpr int PAR = decltype(par_tag)::value, F = PAR, L = PAR ^ 1;
        using IF = std::integral_constant<int, F>;
        using IL = std::integral_constant<int, L>;
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(IN_FLIGHT));
        __builtin_amdgcn_s_waitcnt(lgkmcnt_imm(A_KMAJOR ? 15 : 2 * TA));
        rg_barrier();
        const Slab s1 = ahead(kt + 1, next1), s2 = ahead(kt + 2, next2);
        quarter(I0{}, IF{}, false, [&](int q, int c, int i, int j) {
            if (q < 2 * TB) read_b(PAR, L, q / TB, q % TB);
            if (q < 2 * NL) {
                if (q < NL) load_a(s1, PAR ^ 1, 1, q); else load_b(s2, PAR, F, q - NL);
            }
        });
        quarter(I0{}, IL{}, false, [&](int q, int c, int i, int j) {
            if (q % TB == TB - 1) read_a(PAR, 1, c, i);
        });
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(IN_FLIGHT));
        rg_barrier();
        ld.issue_tokens(kt + 4, lane);
        quarter(I1{}, IL{}, true, [&](int q, int c, int i, int j) {
            if (q % TA == TA - 1) read_b(PAR ^ 1, L, c, j);
            if (q < 2 * NL) {
                if (q < NL) load_a(s2, PAR, 0, q); else load_b(s2, PAR, L, q - NL);
            }
        });
        ld.read_tokens(kt + 3);
        quarter(I1{}, IF{}, false, [&](int q, int c, int i, int j) {
            if (q % TB == TB - 1) read_a(PAR ^ 1, 0, c, i);
        });
    };
    using Own = std::integral_constant<int, -1>;
    if constexpr (MORE) {
        for (;;) {
            for (int kt = 0; kt + 2 < nk; kt += 2) {
                slab(kt, I0{}, Own{}, Own{});
                slab(kt + 1, I1{}, Own{}, Own{});
            }
            slab(nk - 2, I0{}, Own{}, I0{});
            slab(nk - 1, I1{}, I0{}, I1{});
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_s_waitcnt(LGKMCNT0);  // (the next slab's fragments, read again below: the registers are wanted meanwhile)
            if (!run.done(acc)) break;
            clear();
#pragma unroll
            for (int c = 0; c < 2; ++c) {  // (as above; in one function for both places the single tile's kernel spilled registers)
#pragma unroll
                for (int j = 0; j < TB; ++j) read_b(0, 0, c, j);
#pragma unroll
                for (int i = 0; i < TA; ++i) read_a(0, 0, c, i);
            }
            __builtin_amdgcn_s_waitcnt(LGKMCNT0);
            go_first();
        }
    } else {
        int kt = 0;
        for (; kt + 1 < nk; kt += 2) {
            slab(kt, I0{}, Own{}, Own{});
            slab(kt + 1, I1{}, Own{}, Own{});
        }
        if (kt < nk) slab(kt, I0{}, Own{}, Own{});
        if constexpr (LAYOUT == GG_NT) __builtin_amdgcn_s_setprio(0);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // requests past the end write (zeros) to the stages, too
    __builtin_amdgcn_s_waitcnt(LGKMCNT0);
    __syncthreads();
}

constexpr int MD_TB = 4;  // 16-column tiles of a wave
template <int LAYOUT, int UA> struct MdGeo {               // UA: the tile's rows / 64
    static constexpr int BM = 64 * UA, BN = 128;
    static constexpr int A_BYTES = BM * RG_KB, STAGE = A_BYTES + RG_BYTES;  // A's rows, then B's region
    static constexpr int TOKENS = LAYOUT == GG_TN ? RG_TOK : 0;
    static constexpr int NS = UA == 4 ? 3 : 4;             // stages
    static constexpr int TOK = NS * STAGE;                 // (GG_TN) token rings
    static constexpr int EP = BN * 4 + 16;                 // epilogue: LDS pitch of a row of floats
    static constexpr int LDS_LOOP = TOK + TOKENS, LDS_EPI = BM * EP;
    static constexpr int LDS = LDS_LOOP > LDS_EPI ? LDS_LOOP : LDS_EPI;
    static_assert(LDS <= 160 * 1024, "a workgroup's LDS");
};

// 16-row tile i of a wave, among the tile's: contraction-major rows come in regions of 128, of which a wave takes 32
template <int LAYOUT, int UA> __device__ __forceinline__ int md_a_tile(int wm, int i) { return LAYOUT == GG_TN ? i / 2 * 8 + wm * 2 + i % 2 : wm * UA + i; }

// The product of a 64 UA x 128 tile: acc[i][j][r] is row md_a_tile(wm, i)*16 + lane % 16, column (wn*MD_TB + j)*16 + 4*(lane / 16) + r of the tile,
// wm = wave / 2, wn = wave % 2.  At the end nothing is on its way to LDS, and everyone is done with it.
template <int LAYOUT, int UA>
__device__ __forceinline__ void md_product(const GgParams& p, long long m0, int n0, char* smem, f32x4 (&acc)[UA][MD_TB]) {
    using G = MdGeo<LAYOUT, UA>;
    constexpr bool A_KMAJOR = LAYOUT == GG_TN, B_KMAJOR = LAYOUT != GG_NT;
    constexpr int TA = UA, TB = MD_TB, NS = G::NS;  // 16-row tiles of a wave of A, of B
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    auto a_tile = [&](int i) { return md_a_tile<LAYOUT, UA>(wm, i); };
    using Loads = RgLoads<LAYOUT, UA, 2>;
    Loads ld(p, m0, n0, tid, smem + G::TOK + wave * 1024);
    const int nk = ld.nk;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_offset_of(smem) + wave * 1024);
    constexpr int LOADS = UA + 2, BATCH = LOADS + (LAYOUT == GG_TN ? 1 : 0);
    constexpr int AHEAD = NS - 1;  // (GG_TN) the indices of a slab are asked for this many slabs ahead of its rows
    auto load = [&](const typename Loads::Slab& s, unsigned stage, int k) {  // load k of a slab
        if (k < UA) ld.load_a(s, k, stage);
        else ld.load_b(s, k - UA, stage + G::A_BYTES);
    };

#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 fa[2][2][TA], fb[2][2][TB];  // fragments of two slabs
    constexpr int NF = 2 * (TA + TB);
    auto read = [&](auto set_tag, const char* stage, int f) {  // fragment f of a slab: B's, then A's
        constexpr int SET = decltype(set_tag)::value;
        if (f < 2 * TB) { fb[SET][f / TB][f % TB] = rg_fragment(stage + G::A_BYTES, B_KMAJOR, wn * TB + f % TB, f / TB, lane); return; }
        f -= 2 * TB;
        const int c = f / TA, t = a_tile(f % TA);
        fa[SET][c][f % TA] = A_KMAJOR ? rg_fragment(stage + t / 8 * RG_BYTES, true, t % 8, c, lane) : rg_fragment(stage, false, t, c, lane);
    };

    if constexpr (LAYOUT == GG_TN) {
        for (int kt = 0; kt < 4; ++kt) ld.issue_tokens(kt, lane);
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        asm volatile("" ::: "memory");
    }
    // (the batches as the loop issues them: a slab's rows, then the indices of the slab AHEAD, into the entry of a slab that is done)
#pragma unroll
    for (int kt = 0; kt < NS; ++kt) {
        const typename Loads::Slab s = ld.slab(kt);
        ld.read_tokens(kt);
#pragma unroll
        for (int k = 0; k < LOADS; ++k) load(s, lds0 + kt * G::STAGE, k);
        if constexpr (LAYOUT == GG_TN) {
            __builtin_amdgcn_s_waitcnt(LGKMCNT0);
            asm volatile("" ::: "memory");
            ld.issue_tokens(kt + AHEAD, lane);
        }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 1) * BATCH));
    rg_barrier();
#pragma unroll
    for (int f = 0; f < NF; ++f) read(std::integral_constant<int, 0>{}, smem, f);

    constexpr int NM = 2 * TA * TB;
    int st = 0;  // stage of slab kt
    // Slab kt (kt & 1 == PAR), its fragments in set PAR.  Behind the barrier slab kt + 1 has landed (all batches but the last
    // NS - 2) and stage st is free; the source order is the issue order, neighbouring MFMAs share a fragment.
    auto step = [&](int kt, auto par_tag) {
        constexpr int PAR = decltype(par_tag)::value;
        __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 2) * BATCH));
        __builtin_amdgcn_s_waitcnt(LGKMCNT0);
        rg_barrier();
        const typename Loads::Slab s = ld.slab(kt + NS);
        const int nxt = st + 1 == NS ? 0 : st + 1;
        const char* next = smem + nxt * G::STAGE;
        const unsigned free_stage = lds0 + st * G::STAGE;
        if constexpr (LAYOUT == GG_TN) ld.read_tokens(kt + NS);
#pragma unroll
        for (int q = 0; q < NM; ++q) {
            const int c = q / (TA * TB), w = q % (TA * TB), i = w / TB, j = i & 1 ? TB - 1 - w % TB : w % TB;
            __builtin_amdgcn_sched_barrier(0);
            rg_mma(acc[i][j], fa[PAR][c][i], fb[PAR][c][j]);
#pragma unroll
            for (int f = q * NF / (NM * 3 / 4); f < (q + 1) * NF / (NM * 3 / 4); ++f)
                if (f < NF) read(std::integral_constant<int, PAR ^ 1>{}, next, f);
#pragma unroll
            for (int k = q * LOADS / (NM / 2); k < (q + 1) * LOADS / (NM / 2); ++k)
                if (k < LOADS) load(s, free_stage, k);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (LAYOUT == GG_TN) ld.issue_tokens(kt + NS + AHEAD, lane);
        st = nxt;
    };
    int kt = 0;
    for (; kt + 1 < nk; kt += 2) {
        step(kt, std::integral_constant<int, 0>{});
        step(kt + 1, std::integral_constant<int, 1>{});
    }
    if (kt < nk) step(kt, std::integral_constant<int, 0>{});
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // requests past the end write (zeros) to the stages, too
    __builtin_amdgcn_s_waitcnt(LGKMCNT0);
    __syncthreads();
}

}  // namespace lemo
