// Attention over listed key blocks, heads of 128, lists of more than 32 rows: 64 rows a wave, one wave per SIMD, matrix and vector work
// interleaved by hand as in the attention over kept tokens (attention.hip says why and how): with 32 rows a wave the fragments of K and V
// alone take the CU's whole LDS bandwidth at full matrix rate.  Stages of 128 listed keys that need no mask run as a branch-free
// stream of groups of 16 MFMAs -- logits of the next tile, product of the last one, exponentials of this one -- against a reference
// that the first stage froze; a normaliser that shows that a later logit exceeded it by too much sends the workgroup through its list
// again with the ordinary softmax, before anything is stored.  Lists ascend, so the stages that need a mask come last.
// A stage's four subtiles of keys lie anywhere: each is addressed by a descriptor of its own, from its first key on.
// Figures stand at launch_block_attention.
#include <type_traits>

#include "block_attention.hpp"

namespace lemo {

constexpr int BP_SUB = 32 * 256, BP_STAGE = 8 * BP_SUB;          // bytes of a subtile of K or V, of a stage
constexpr int BP_PITCH = 132, BP_JOIN = 256 * (BP_PITCH * 4 + 8);  // floats of a row where waves' results meet; LDS for all of them
static_assert(BP_JOIN >= 2 * BP_STAGE, "");
constexpr int bp_lds(int subtiles) { return BP_JOIN + subtiles * 4; }
constexpr float BP_FROZEN_LIMIT = 0x1p100f;  // a flushed factor (below 2^-126) drops less than 2^-26 of a smaller normaliser

__device__ __forceinline__ void bp_fence() { __builtin_amdgcn_sched_barrier(0); }
// keeps an addition where it is written; otherwise the compiler postpones the sums and parks every exponential in a register
__device__ __forceinline__ void bp_pin(float& x) { asm volatile("" : "+v"(x)); }

// KS waves share 64 rows and take 4 / KS subtiles of a stage each.
template <int KS>
__global__ __launch_bounds__(256, 1) void block_attention_pipe_kernel(BlockAttnParams p) {
    using Tile = HeadTile<128>;
    constexpr int NCH = 8, ROWS = 256 / KS, SHARE = 4 / KS;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int listed;
    int* const all_keys = reinterpret_cast<int*>(smem + BP_JOIN);

    int g, rank;
    decode_block(p.order, p.H_kv, p.n_qb * p.n_rt * p.n_parts, g, rank);
    const int share = rank % p.n_parts, rt = rank / p.n_parts % p.n_rt, qb = rank / p.n_parts / p.n_rt;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool causal = (p.flags & LEMO_CAUSAL) != 0;
    const int S = p.S_k;
    const long long pos0 = p.q_start + (long long)qb * p.bq;
    const int rows = min(p.bq, p.S_q - qb * p.bq) * p.G, row_end = min(rows, (rt + 1) * ROWS);
    auto limit_of = [&](int row) { return causal ? (int)min(pos0 + row / p.G, (long long)S - 1) : S - 1; };

    if (wave == 0) {
        const int n = rt * ROWS < rows ? list_subtiles(p.blocks + ((long long)qb * p.H_kv + g) * p.T, p.T, p.b, (p.S_k + p.b - 1) / p.b, limit_of(row_end - 1), all_keys, lane) : 0;
        if (lane == 0) listed = n;
    }
    // resident operand: this wave's 64 rows, as MFMA B fragments
    const int row0 = rt * ROWS + wave / KS * 64;
    int lim[2], clean[2], reach[2];  // last key of the lane's row, of the subtile's first row, of its last
    u32x4 qf[2][NCH];
#pragma unroll
    for (int qs = 0; qs < 2; ++qs) {
        const int first = row0 + qs * 32, row = first + l32;
        lim[qs] = row < rows ? limit_of(row) : -1;
        clean[qs] = first < rows ? limit_of(first) : -1;
        reach[qs] = first < rows ? limit_of(min(first + 31, rows - 1)) : -1;
#pragma unroll
        for (int c = 0; c < NCH; ++c) qf[qs][c] = u32x4{0u, 0u, 0u, 0u};
        if (row < rows) {
            const uint16_t* q = p.Q + ((long long)qb * p.bq + row / p.G) * p.q_ts + (long long)(g * p.G + row % p.G) * p.q_hs;
#pragma unroll
            for (int c = 0; c < NCH; ++c) qf[qs][c] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(q) + c * 32 + half * 16);
        }
    }
    const bool active = row0 < rows;
    __syncthreads();
    const int s_begin = (int)((long long)listed * share / p.n_parts), n_sub = (int)((long long)listed * (share + 1) / p.n_parts) - s_begin;
    const int* const keys = all_keys + s_begin;
    // subtiles that no row of the workgroup needs a mask for, the first ones of the list.  All but the first stage's are hot: that takes as
    // few as leave whole stages, and the last stages hold what needs a mask
    const int wg_clean = rt * ROWS < rows ? limit_of(rt * ROWS) : -1;
    int n_clean = 0;
    for (int s0 = 0; s0 < n_sub; s0 += 64) n_clean += (int)__popcll(__ballot(s0 + lane < n_sub && keys[s0 + lane] + 31 <= wg_clean));
    const int head = n_clean > 0 ? min((n_clean - 1) % 4 + 1, n_sub) : min(4, n_sub);  // subtiles of the first stage
    const int nstage = (n_sub - head + 3) / 4 + (n_sub > 0);
    auto stage_begin = [&](int t) { return t == 0 ? 0 : head + 4 * (t - 1); };
    auto stage_end = [&](int t) { return min(head + 4 * t, n_sub); };

    // ---- staging: LDS-direct loads.  Load n (0..15) of a wave: subtile n / 2 (K, then V), rows ((n & 1) * 4 + wave) * 4 + lane / 16
    const char* const kbase = reinterpret_cast<const char*>(p.K + (long long)g * p.k_hs);
    const char* const vbase = reinterpret_cast<const char*>(p.V + (long long)g * p.v_hs);
    const int k_pitch = (int)p.k_ts * 2, v_pitch = (int)p.v_ts * 2;
    const int s_row = wave * 4 + (lane >> 4), s_piece = (((lane & 15) ^ Tile::swz(s_row)) << 4);  // (rows 16 apart share the exchange of pieces)
    int voff[2][2];
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
        voff[0][odd] = (s_row + 16 * odd) * k_pitch + s_piece;
        voff[1][odd] = (s_row + 16 * odd) * v_pitch + s_piece;
    }
    const unsigned lds_w = lds_offset_of(smem) + (unsigned)wave * 1024u;
    int want[4];  // first keys of the stage to be requested; S where there is none
    auto take_keys = [&](int t) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int at = stage_begin(t) + s;
            want[s] = at < stage_end(t) ? __builtin_amdgcn_readfirstlane(keys[min(at, n_sub - 1)]) : S;
        }
    };
    auto stage_load_one = [&](int n, int buf) {
        const bool v = n >= 8;
        const int sub = n / 2, key = want[sub & 3];
        const long long pitch = v ? v_pitch : k_pitch;
        const u32x4 rsrc = raw_rsrc((v ? vbase : kbase) + key * pitch, key < S ? (long long)(S - 1 - key) * pitch + 256 : 0);
        lds_direct_b128(rsrc, lds_w + (unsigned)buf * BP_STAGE + (unsigned)sub * BP_SUB + (unsigned)(n & 1) * 4096u, voff[v][n & 1]);
    };
    auto k_frag = [&](const char* st, int ks, int c) { return Tile::row_fragment(st + ks * BP_SUB, c, lane); };
    auto v_frag = [&](const char* st, int ks, int n) { return Tile::column_fragment(st + (4 + ks) * BP_SUB, n >> 1, n & 1, lane); };
    const int sub0 = wave % KS * SHARE;

    bool frozen = true;  // workgroup-uniform: which pass this is
    f32x16 o[2][4];      // o[qs][dv][r] = element (value column dv*32 + acc_row(r), row l32 of subtile qs)
    float ltot[2], o_ref[2];
    for (;;) {
#pragma unroll
    for (int qs = 0; qs < 2; ++qs)
#pragma unroll
        for (int dv = 0; dv < 4; ++dv) o[qs][dv] = f32x16{0};
    float mrun[2] = {-INFINITY, -INFINITY}, la[2] = {0.f, 0.f}, lb[2] = {0.f, 0.f};

    auto slow_tile = [&](int qs, int key, const u32x4 (&kfr)[NCH], const u32x4 (&vfr)[8]) {  // the ordinary online softmax
        if (key > reach[qs]) return;
        f32x16 acc = {0};
#pragma unroll
        for (int c = 0; c < NCH; ++c) mma_chunk<bf16_t>(acc, kfr[c], qf[qs][c]);
        if (key + 31 > clean[qs]) {
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = key + acc_row(r, lane) <= lim[qs] ? acc[r] : -INFINITY;
        }
        float top = acc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, acc[r]);
        top = half_waves_max(top * p.c2);
        const float mn = top > mrun[qs] + 8.f ? top : mrun[qs];
        const float ms = mn == -INFINITY ? 0.f : mn;
        const float corr = __builtin_amdgcn_exp2f(mrun[qs] - ms);
        float pr[16], s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            pr[r] = __builtin_amdgcn_exp2f(fmaf(acc[r], p.c2, -ms));
            if (r & 1) s1 += pr[r]; else s0 += pr[r];
        }
        la[qs] = fmaf(la[qs], corr, s0);
        lb[qs] = fmaf(lb[qs], corr, s1);
        if (__any(mn > mrun[qs])) {
#pragma unroll
            for (int dv = 0; dv < 4; ++dv)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[qs][dv][r] *= corr;
        }
        mrun[qs] = mn;
        u32x4 pbs[2];
#pragma unroll
        for (int c = 0; c < 2; ++c)
            pbs[c] = u32x4{pack_bf16x2_hw(pr[8 * c + 0], pr[8 * c + 1]), pack_bf16x2_hw(pr[8 * c + 2], pr[8 * c + 3]),
                           pack_bf16x2_hw(pr[8 * c + 4], pr[8 * c + 5]), pack_bf16x2_hw(pr[8 * c + 6], pr[8 * c + 7])};
#pragma unroll
        for (int n = 0; n < 8; ++n) mma_chunk<bf16_t>(o[qs][n >> 1], vfr[n], pbs[n & 1]);
    };

    f32x16 S0, S1;  // state of the hot stream, see attention.hip
    u32x4 pb[2][2];
    u32x4 kf[NCH], vf[8];
    float nm[2];

    if (nstage > 0) {
        take_keys(0);
#pragma unroll
        for (int n = 0; n < 16; ++n) stage_load_one(n, 0);
        take_keys(1);
        settle_stage();
    }
    auto slow_stage = [&](int t) {
        __syncthreads();
        const char* const st = smem + (t & 1) * BP_STAGE;
        if (t + 1 < nstage) {
#pragma unroll
            for (int n = 0; n < 16; ++n) stage_load_one(n, (t + 1) & 1);
        }
        if (active) {
#pragma unroll 1
            for (int ks = sub0; ks < sub0 + SHARE; ++ks) {
                if (stage_begin(t) + ks >= stage_end(t)) break;
                const int key = __builtin_amdgcn_readfirstlane(keys[stage_begin(t) + ks]);
                if (key > reach[0] && key > reach[1]) break;
                u32x4 kfr[NCH], vfr[8];
#pragma unroll
                for (int c = 0; c < NCH; ++c) kfr[c] = k_frag(st, ks, c);
#pragma unroll
                for (int n = 0; n < 8; ++n) vfr[n] = v_frag(st, ks, n);
                slow_tile(0, key, kfr, vfr);
                slow_tile(1, key, kfr, vfr);
            }
        }
        settle_stage();
        take_keys(t + 2);
    };
    struct Hold { float prev, even; };
    Hold h0{0.f, 0.f}, h1{0.f, 0.f};
    auto consume = [&](Hold& hd, int j, int qs) {
        if (j & 1) {
            lb[qs] += hd.prev;
            bp_pin(lb[qs]);
            pb[qs][j >> 3][(j & 7) >> 1] = pack_bf16x2_hw(hd.even, hd.prev);
        } else {
            la[qs] += hd.prev;
            bp_pin(la[qs]);
            hd.even = hd.prev;
        }
    };
    auto feed = [&](Hold& hd, int j, float logit, int qs) {
        const float e = __builtin_amdgcn_exp2f(fmaf(logit, p.c2, nm[qs]));
        if (j > 0) consume(hd, j - 1, qs);
        hd.prev = e;
    };
    // One group of 16 slots: EVEN(n) logits of (subtile n, rows 1), product of (n - 1, rows 1), exponentials of (n, rows 0);
    // ODD(n) logits of (n + 1, rows 0), product of (n, rows 0), exponentials of (n, rows 1)
    auto group = [&](auto odd_tag, const char* st, int ks, bool refill_k, auto&& ride) {
        constexpr bool ODD = decltype(odd_tag)::value;
        constexpr int QL = ODD ? 0 : 1, QP = ODD ? 0 : 1, QE = ODD ? 1 : 0;
        f32x16& SL = ODD ? S0 : S1;
        f32x16& SE = ODD ? S1 : S0;
        Hold& hd = ODD ? h1 : h0;
        Hold& hp = ODD ? h0 : h1;
        SL = f32x16{0};
        bp_fence();
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            mma_chunk<bf16_t>(SL, kf[c], qf[QL][c]);
            if (!ODD && refill_k) kf[c] = k_frag(st, ks + 1, c);
            ride(2 * c);
            if (c == 0) consume(hp, 15, QP);
            feed(hd, 2 * c, SE[2 * c], QE);
            bp_fence();
            mma_chunk<bf16_t>(o[QP][c & 3], vf[(c & 3) * 2 + (c >> 2)], pb[QP][c >> 2]);
            if (!ODD) vf[(c & 3) * 2 + (c >> 2)] = v_frag(st, ks, (c & 3) * 2 + (c >> 2));
            ride(2 * c + 1);
            feed(hd, 2 * c + 1, SE[2 * c + 1], QE);
            bp_fence();
        }
    };
    using EvenT = std::integral_constant<bool, false>;
    using OddT = std::integral_constant<bool, true>;
    auto hot_stage = [&](int t) {
        __syncthreads();
        const char* const st = smem + (t & 1) * BP_STAGE;
        const int nbuf = (t + 1) & 1;
#pragma unroll
        for (int c = 0; c < NCH; ++c) kf[c] = k_frag(st, sub0, c);
        auto ride = [&](int n) { stage_load_one(n, nbuf); };  // (no next stage: descriptors of size zero)
        auto no_ride = [&](int) {};
        group(OddT{}, st, sub0, false, ride);
#pragma unroll
        for (int ks = 0; ks < SHARE; ++ks) {
            group(EvenT{}, st, sub0 + ks, ks < SHARE - 1, no_ride);
            if (ks < SHARE - 1) group(OddT{}, st, sub0 + ks, false, no_ride);
        }
        settle_stage();
        take_keys(t + 2);
    };
    const int t_hot = frozen && active ? max(1, (n_clean - head) / 4 + 1) : 1;
    if (nstage > 0) slow_stage(0);
    if (t_hot > 1) {
#pragma unroll
        for (int r = 0; r < 16; ++r) S1[r] = -INFINITY;
        pb[0][0] = pb[0][1] = pb[1][0] = pb[1][1] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int n = 0; n < 8; ++n) vf[n] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int qs = 0; qs < 2; ++qs) {
            mrun[qs] = mrun[qs] == -INFINITY ? 0.f : mrun[qs];
            nm[qs] = -mrun[qs];
        }
        for (int t = 1; t < t_hot; ++t) hot_stage(t);
        consume(h0, 15, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) mma_chunk<bf16_t>(o[0][i & 3], vf[(i & 3) * 2 + (i >> 2)], pb[0][i >> 2]);
#pragma unroll
        for (int j = 0; j < 16; ++j) feed(h1, j, S1[j], 1);
        consume(h1, 15, 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) mma_chunk<bf16_t>(o[1][i & 3], vf[(i & 3) * 2 + (i >> 2)], pb[1][i >> 2]);
#pragma unroll
        for (int qs = 0; qs < 2; ++qs) la[qs] = la[qs] + lb[qs] < BP_FROZEN_LIMIT ? la[qs] : INFINITY;
    }
    for (int t = t_hot; t < nstage; ++t) slow_stage(t);

    bool bad = false;
#pragma unroll
    for (int qs = 0; qs < 2; ++qs) {
        const float l = la[qs] + lb[qs];
        ltot[qs] = l + __shfl_xor(l, 32);
        o_ref[qs] = mrun[qs];
        bad |= lim[qs] >= 0 && !(ltot[qs] < BP_FROZEN_LIMIT);
    }
    if (!frozen || !__syncthreads_or(bad)) break;
    frozen = false;
    }

    // the waves that share rows bring their sums to the largest reference of them, in LDS, and each finishes its part of the rows
    __syncthreads();
    const int first = wave - wave % KS;
    float* const sums = reinterpret_cast<float*>(smem);
    float2* const stats = reinterpret_cast<float2*>(smem + 256 * BP_PITCH * 4);
#pragma unroll
    for (int qs = 0; qs < 2; ++qs)
        if (half == 0) stats[wave * 64 + qs * 32 + l32] = make_float2(o_ref[qs], ltot[qs]);
    __syncthreads();
#pragma unroll
    for (int qs = 0; qs < 2; ++qs) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < KS; ++w) top = fmaxf(top, stats[(first + w) * 64 + qs * 32 + l32].x);
        const float f = o_ref[qs] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(o_ref[qs] - top);
#pragma unroll
        for (int dv = 0; dv < 4; ++dv)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(sums + (wave * 64 + qs * 32 + l32) * BP_PITCH + dv * 32 + q * 8 + half * 4) =
                    f32x4{o[qs][dv][q * 4] * f, o[qs][dv][q * 4 + 1] * f, o[qs][dv][q * 4 + 2] * f, o[qs][dv][q * 4 + 3] * f};
    }
    __syncthreads();
    const int c0 = lane % 16 * 8;
#pragma unroll 2
    for (int r = 0; r < 64 / KS; r += 4) {
        const int in = wave % KS * (64 / KS) + r + lane / 16, out = row0 + in;
        if (out >= rows) continue;
        float top = -INFINITY, total = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < KS; ++w) top = fmaxf(top, stats[(first + w) * 64 + in].x);
#pragma unroll
        for (int w = 0; w < KS; ++w) {
            const int at = (first + w) * 64 + in;
            const float2 st = stats[at];
            total += st.x == -INFINITY ? 0.f : st.y * __builtin_amdgcn_exp2f(st.x - top);
            const f32x4 lo = *reinterpret_cast<const f32x4*>(sums + at * BP_PITCH + c0), hi = *reinterpret_cast<const f32x4*>(sums + at * BP_PITCH + c0 + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[e + 4] += hi[e]; }
        }
        if (p.n_parts > 1) {
            float* part = p.parts + ((((long long)qb * p.H_kv + g) * p.n_parts + share) * p.R + out) * PART_ROW<128>;
            *reinterpret_cast<f32x4*>(part + c0) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(part + c0 + 4) = f32x4{v[4], v[5], v[6], v[7]};
            if (c0 == 0) *reinterpret_cast<float2*>(part + 128) = make_float2(top, total);
            continue;
        }
        const long long i = (long long)qb * p.bq + out / p.G;
        const int h = g * p.G + out % p.G;
        const float inv = total == 0.f ? 0.f : 1.f / total;
        u32x4 piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) piece[e] = pack_bf16x2_hw(v[2 * e] * inv, v[2 * e + 1] * inv);
        *reinterpret_cast<u32x4*>(p.O + i * p.o_ts + (long long)h * p.o_hs + c0) = piece;
        if (p.lse2 && c0 == 0) p.lse2[(long long)h * p.S_q + i] = total == 0.f ? -INFINITY : top + log2f(total);
    }
}

int prepare_block_attention_pipe() {
    static const int err = raise_lds_limits({{reinterpret_cast<const void*>(&block_attention_pipe_kernel<1>), bp_lds(MAX_LISTED_SUBTILES)},
                                             {reinterpret_cast<const void*>(&block_attention_pipe_kernel<2>), bp_lds(MAX_LISTED_SUBTILES)},
                                             {reinterpret_cast<const void*>(&block_attention_pipe_kernel<4>), bp_lds(MAX_LISTED_SUBTILES)}});
    return err;
}

template <int KS> static int run_pipe(const BlockAttnParams& p, hipStream_t st) {
    hipLaunchKernelGGL((block_attention_pipe_kernel<KS>), dim3((unsigned)((long long)p.n_qb * p.n_rt * p.n_parts * p.H_kv)), dim3(256), (bp_lds(p.T * (p.b / 32))), st, p);
    return (int)hipGetLastError();
}

int launch_block_attention_pipe(const BlockAttnParams& p, hipStream_t st) { return p.R > 128 ? run_pipe<1>(p, st) : p.R > 64 ? run_pipe<2>(p, st) : run_pipe<4>(p, st); }

}  // namespace lemo
