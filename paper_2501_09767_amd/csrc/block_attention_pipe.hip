// Attention over listed key blocks, heads of 128, lists of more than 128 rows: 64 rows a wave, one wave per SIMD, matrix and vector work
// interleaved by hand as in the attention over kept tokens (attention.hip says why and how): with 32 rows a wave the fragments of K and V
// alone take the CU's whole LDS bandwidth at full matrix rate.  Stages of 128 listed keys that need no mask run as a branch-free
// stream of groups of 16 MFMAs -- logits of the next tile, product of the last one, exponentials of this one -- against a reference
// that the first stage froze; a normaliser that shows that a later logit exceeded it by too much sends the workgroup through its list
// again with the ordinary softmax, before anything is stored.  Lists ascend, so the stages that need a mask come last.
// A stage's four subtiles of keys lie anywhere: each is addressed by a descriptor of its own, from its first key on.
// A workgroup has a CU to itself, so nothing else would fill the time that a list, its rows and its first keys take to arrive, half of
// what 16 blocks of 64 keys take to work on.  It therefore walks over the lists, and the next one's subtiles are found and its first stage
// requested while the last stage of the one before is worked on; its rows are requested before that one's results are stored.
// Figures stand at launch_block_attention_pipe.
#include <type_traits>

#include "block_attention.hpp"

namespace lemo {

constexpr int BP_SUB = 32 * 256, BP_STAGE = 8 * BP_SUB;  // bytes of a subtile of K or V, of a stage
constexpr int BP_ROWS = 256;
constexpr int bp_lds(int subtiles) { return 2 * BP_STAGE + 2 * (16 + subtiles * 4); }  // two lists, the number of subtiles before each
constexpr float BP_FROZEN_LIMIT = 0x1p100f;  // a flushed factor (below 2^-126) drops less than 2^-26 of a smaller normaliser

__device__ __forceinline__ void bp_fence() { __builtin_amdgcn_sched_barrier(0); }
// keeps an addition where it is written; otherwise the compiler postpones the sums and parks every exponential in a register
__device__ __forceinline__ void bp_pin(float& x) { asm volatile("" : "+v"(x)); }

__global__ __launch_bounds__(256, 1) void block_attention_pipe_kernel(BlockAttnParams p, int tiles, int room) {
    using Tile = HeadTile<128>;
    constexpr int NCH = 8, SUBS = 4;  // chunks of a head row, subtiles of a stage
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool causal = (p.flags & LEMO_CAUSAL) != 0;
    const int S = p.S_k, nb = p.nb;
    auto list_at = [&](int buf) { return reinterpret_cast<int*>(smem + 2 * BP_STAGE) + buf * (4 + room) + 4; };  // [-4]: how many

    // ---- a tile of rows and its list
    struct Place { int g, share, rt, qb, rows; long long pos0; };
    auto place_of = [&](int tile) {
        Place w;
        int rank;
        decode_block(p.order, p.H_kv, p.n_qb * p.n_rt * p.n_parts, w.g, rank, tile);
        w.share = rank % p.n_parts;
        w.rt = rank / p.n_parts % p.n_rt;
        w.qb = rank / p.n_parts / p.n_rt;
        w.rows = min(p.bq, p.S_q - w.qb * p.bq) * p.G;
        w.pos0 = p.q_start + (long long)w.qb * p.bq;
        return w;
    };
    auto limit_in = [&](const Place& w, int row) { return causal ? (int)min(w.pos0 + row / p.G, (long long)S - 1) : S - 1; };  // last key a row may see
    auto list_of = [&](const Place& w) { return p.blocks + ((long long)w.qb * p.H_kv + w.g) * p.T; };
    auto find_subtiles = [&](const Place& w, int buf, int first_entries) {  // one wave
        int n = 0;
        if (w.rt * BP_ROWS < w.rows)
            n = list_subtiles(list_of(w), p.T, p.b, nb, limit_in(w, min(w.rows, (w.rt + 1) * BP_ROWS) - 1), list_at(buf), lane, first_entries);
        if (lane == 0) list_at(buf)[-4] = n;
    };
    // The first subtiles of a list need no mask for any row of the workgroup.  All but the first stage's are hot: that takes as few as leave whole
    // stages, and the last stages hold what needs a mask
    struct Stages { int n_sub, n_clean, head, count; const int* keys; };
    auto stages_of = [&](const Place& w, int buf) {
        Stages s;
        const int listed = __builtin_amdgcn_readfirstlane(list_at(buf)[-4]);
        const int begin = (int)((long long)listed * w.share / p.n_parts);
        s.n_sub = (int)((long long)listed * (w.share + 1) / p.n_parts) - begin;
        s.keys = list_at(buf) + begin;
        const int clean = w.rt * BP_ROWS < w.rows ? limit_in(w, w.rt * BP_ROWS) : -1;
        s.n_clean = 0;
        for (int s0 = 0; s0 < s.n_sub; s0 += 64) s.n_clean += (int)__popcll(__ballot(s0 + lane < s.n_sub && s.keys[s0 + lane] + 31 <= clean));
        s.head = s.n_clean > 0 ? min((s.n_clean - 1) % 4 + 1, s.n_sub) : min(4, s.n_sub);
        s.count = (s.n_sub - s.head + 3) / 4 + (s.n_sub > 0);
        return s;
    };
    auto stage_begin = [](const Stages& s, int t) { return t == 0 ? 0 : s.head + 4 * (t - 1); };
    auto stage_end = [](const Stages& s, int t) { return min(s.head + 4 * t, s.n_sub); };

    // ---- staging: LDS-direct loads.  Load n (0..15) of a wave: subtile n / 2 (K, then V), rows ((n & 1) * 4 + wave) * 4 + lane / 16
    const int k_pitch = (int)p.k_ts * 2, v_pitch = (int)p.v_ts * 2;
    const int s_row = wave * 4 + (lane >> 4), s_piece = (((lane & 15) ^ Tile::swz(s_row)) << 4);  // (rows 16 apart share the exchange of pieces)
    int voff[2][2];
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
        voff[0][odd] = (s_row + 16 * odd) * k_pitch + s_piece;
        voff[1][odd] = (s_row + 16 * odd) * v_pitch + s_piece;
    }
    const unsigned lds_w = lds_offset_of(smem) + (unsigned)wave * 1024u;
    int want[4], want_g;  // the stage to be requested: its first keys, S where there is none, and its group
    auto take_keys = [&](const Place& w, const Stages& s, int t) {
        want_g = w.g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = stage_begin(s, t) + i;
            want[i] = at < stage_end(s, t) ? __builtin_amdgcn_readfirstlane(s.keys[min(at, s.n_sub - 1)]) : S;
        }
    };
    auto take_none = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) want[i] = S;
    };
    auto stage_load_one = [&](int n, int buf) {
        const bool v = n >= 8;
        const int sub = n / 2, key = want[sub & 3];
        const char* const base = v ? reinterpret_cast<const char*>(p.V + (long long)want_g * p.v_hs) : reinterpret_cast<const char*>(p.K + (long long)want_g * p.k_hs);
        lds_direct_b128(subtile_rsrc<128>(base, key, S, v ? v_pitch : k_pitch), lds_w + (unsigned)buf * BP_STAGE + (unsigned)sub * BP_SUB + (unsigned)(n & 1) * 4096u, voff[v][n & 1]);
    };
    auto stage_load = [&](int buf) {
#pragma unroll
        for (int n = 0; n < 16; ++n) stage_load_one(n, buf);
    };
    auto k_frag = [&](const char* st, int ks, int c) { return Tile::row_fragment(st + ks * BP_SUB, c, lane); };
    auto v_frag = [&](const char* st, int ks, int n) { return Tile::column_fragment(st + (4 + ks) * BP_SUB, n >> 1, n & 1, lane); };

    // ---- this wave's 64 rows, as MFMA B fragments
    u32x4 qf[2][NCH];
    auto load_rows = [&](const Place& w) {
#pragma unroll
        for (int qs = 0; qs < 2; ++qs) {
            const int row = w.rt * BP_ROWS + wave * 64 + qs * 32 + l32;
#pragma unroll
            for (int c = 0; c < NCH; ++c) qf[qs][c] = u32x4{0u, 0u, 0u, 0u};
            if (row < w.rows) {
                const uint16_t* q = p.Q + ((long long)w.qb * p.bq + row / p.G) * p.q_ts + (long long)(w.g * p.G + row % p.G) * p.q_hs;
#pragma unroll
                for (int c = 0; c < NCH; ++c) qf[qs][c] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(q) + c * 32 + half * 16);
            }
        }
    };

    Place now = place_of(blockIdx.x);
    if (wave == 0) find_subtiles(now, 0, list_head(list_of(now), p.T, lane));
    __syncthreads();
    Stages s_now = stages_of(now, 0);
    take_keys(now, s_now, 0);
    stage_load(0);
    load_rows(now);
    int tile = blockIdx.x, par = 0, list_buf = 0;  // par: buffer of the tile's first stage
    Place then = now;
    int first_entries = -1;  // (wave 0) of the list of the tile after this one
    if (tile + (int)gridDim.x < tiles) {
        then = place_of(tile + gridDim.x);
        if (wave == 0) first_entries = list_head(list_of(then), p.T, lane);
    }
    for (;;) {
    const bool more = tile + (int)gridDim.x < tiles;  // a tile follows: its list is found now, its first stage requested in the last stage of this one
    if (more && wave == 0) find_subtiles(then, list_buf ^ 1, first_entries);
    const Place after = tile + 2 * (int)gridDim.x < tiles ? place_of(tile + 2 * gridDim.x) : then;
    if (wave == 0) first_entries = list_head(list_of(after), p.T, lane);
    settle_stage();
    __syncthreads();
    Stages s_then = s_now;
    if (more) s_then = stages_of(then, list_buf ^ 1);
    const int nstage = s_now.count;
    auto take_next = [&](int t) {  // keys of stage t of this tile, or of the first stage of the next
        if (t < nstage) take_keys(now, s_now, t);
        else if (t == nstage && more) take_keys(then, s_then, 0);
        else take_none();
    };
    const int row0 = now.rt * BP_ROWS + wave * 64;
    const bool active = row0 < now.rows;
    int lim[2], clean[2], reach[2];  // last key of the lane's row, of the subtile's first row, of its last
#pragma unroll
    for (int qs = 0; qs < 2; ++qs) {
        const int first = row0 + qs * 32, row = first + l32;
        lim[qs] = row < now.rows ? limit_in(now, row) : -1;
        clean[qs] = first < now.rows ? limit_in(now, first) : -1;
        reach[qs] = first < now.rows ? limit_in(now, min(first + 31, now.rows - 1)) : -1;
    }

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

    take_next(1);
    auto slow_stage = [&](int t) {
        __syncthreads();
        const char* const st = smem + ((par + t) & 1) * BP_STAGE;
        stage_load((par + t + 1) & 1);  // (descriptors of size zero where no stage follows)
        if (active) {
#pragma unroll 1
            for (int ks = 0; ks < SUBS; ++ks) {
                if (stage_begin(s_now, t) + ks >= stage_end(s_now, t)) break;
                const int key = __builtin_amdgcn_readfirstlane(s_now.keys[stage_begin(s_now, t) + ks]);
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
        take_next(t + 2);
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
        const char* const st = smem + ((par + t) & 1) * BP_STAGE;
        const int nbuf = (par + t + 1) & 1;
#pragma unroll
        for (int c = 0; c < NCH; ++c) kf[c] = k_frag(st, 0, c);
        auto ride = [&](int n) { stage_load_one(n, nbuf); };  // (no next stage: descriptors of size zero)
        auto no_ride = [&](int) {};
        group(OddT{}, st, 0, false, ride);
#pragma unroll
        for (int ks = 0; ks < SUBS; ++ks) {
            group(EvenT{}, st, ks, ks < SUBS - 1, no_ride);
            if (ks < SUBS - 1) group(OddT{}, st, ks, false, no_ride);
        }
        settle_stage();
        take_next(t + 2);
    };
    const int t_hot = frozen && active ? max(1, (s_now.n_clean - s_now.head) / 4 + 1) : 1;
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
    if (t_hot > 1) {  // probabilities up to the limit, times large values, may have passed binary32 where the ordinary softmax does not
        float zero = 0.f;
#pragma unroll
        for (int qs = 0; qs < 2; ++qs)
#pragma unroll
            for (int dv = 0; dv < 4; ++dv)
#pragma unroll
                for (int r = 0; r < 16; ++r) zero = fmaf(o[qs][dv][r], 0.f, zero);
        bad |= zero != 0.f;
    }
    if (!__syncthreads_or(frozen && bad)) break;  // (the barrier also ends the last stage: its buffer is free)
    // once more with the ordinary softmax: the first stage comes again, into the buffer that the next tile's has just filled
    frozen = false;
    par = (par + nstage) & 1;
    take_keys(now, s_now, 0);
    stage_load(par);
    settle_stage();
    }
    if (nstage == 0 && more) {  // no stage has requested the next tile's first
        take_keys(then, s_then, 0);
        stage_load(par);
    }
    const int free_buf = (par + nstage + 1) & 1;  // holds no stage that is still needed, nor one under way
    if (more) load_rows(then);

    if (p.n_parts > 1) {
#pragma unroll
        for (int qs = 0; qs < 2; ++qs) {
            const int row = row0 + qs * 32 + l32;
            if (row >= now.rows) continue;
            float* const part = p.parts + ((((long long)now.qb * p.H_kv + now.g) * p.n_parts + now.share) * p.R + row) * PART_ROW<128>;
#pragma unroll
            for (int dv = 0; dv < 4; ++dv)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4*>(part + dv * 32 + q * 8 + half * 4) = f32x4{o[qs][dv][q * 4], o[qs][dv][q * 4 + 1], o[qs][dv][q * 4 + 2], o[qs][dv][q * 4 + 3]};
            if (half == 0) *reinterpret_cast<float2*>(part + 128) = make_float2(o_ref[qs], ltot[qs]);
        }
    } else {
        // normalised rows go through LDS, 64 to a wave and nobody else's, so that whole rows are stored
        char* const mine = smem + free_buf * BP_STAGE + wave * 16384;
#pragma unroll
        for (int qs = 0; qs < 2; ++qs) {
            const float inv = ltot[qs] == 0.f ? 0.f : 1.f / ltot[qs];
            const int in = qs * 32 + l32, row = row0 + in;
#pragma unroll
            for (int dv = 0; dv < 4; ++dv)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint2 v;
                    v.x = pack_bf16x2_hw(o[qs][dv][q * 4 + 0] * inv, o[qs][dv][q * 4 + 1] * inv);
                    v.y = pack_bf16x2_hw(o[qs][dv][q * 4 + 2] * inv, o[qs][dv][q * 4 + 3] * inv);
                    *reinterpret_cast<uint2*>(mine + in * 256 + (((dv * 4 + q) ^ (in & 15)) << 4) + half * 8) = v;
                }
            if (p.lse2 && half == 0 && row < now.rows)
                p.lse2[(long long)(now.g * p.G + row % p.G) * p.S_q + (long long)now.qb * p.bq + row / p.G] = ltot[qs] == 0.f ? -INFINITY : o_ref[qs] + log2f(ltot[qs]);
        }
        const int piece = lane & 15;
#pragma unroll 4
        for (int r = 0; r < 64; r += 4) {
            const int in = r + (lane >> 4), row = row0 + in;
            const u32x4 v = *reinterpret_cast<const u32x4*>(mine + in * 256 + ((piece ^ (in & 15)) << 4));
            if (row < now.rows)
                *reinterpret_cast<u32x4*>(p.O + ((long long)now.qb * p.bq + row / p.G) * p.o_ts + (long long)(now.g * p.G + row % p.G) * p.o_hs + piece * 8) = v;
        }
    }
    if (!more) break;
    par = (par + nstage) & 1;
    tile += gridDim.x;
    list_buf ^= 1;
    now = then;
    s_now = s_then;
    then = after;
    }
}

int prepare_block_attention_pipe() {
    static const int err = raise_lds_limits({{reinterpret_cast<const void*>(&block_attention_pipe_kernel), bp_lds(MAX_LISTED_SUBTILES)}});
    return err;
}

// One workgroup for every CU.  us with tiles of 128 rows of block_attention_kernel / with this: 32768 tokens, 32 / 8 heads, 16 blocks of 64
// for 64 queries (256 rows a list) 716 / 600, 880 TFLOP/s of the listed pairs; with a workgroup for each tile, which does not walk,
// 707.  Lists of fewer rows leave waves without rows: 8192 tokens, 32 heads, 128 rows 170 / 260, 64 rows 205 / 493.
int launch_block_attention_pipe(const BlockAttnParams& p, hipStream_t st) {
    const long long tiles = (long long)p.n_qb * p.n_rt * p.n_parts * p.H_kv;
    const int subtiles = p.T * (p.b / 32), room = (subtiles + 3) / 4 * 4;
    hipLaunchKernelGGL(block_attention_pipe_kernel, dim3((unsigned)(tiles < 256 ? tiles : 256)), dim3(256), bp_lds(room), st, p, (int)tiles, room);
    return (int)hipGetLastError();
}

}  // namespace lemo
