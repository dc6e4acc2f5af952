// Gradients of the attention over listed key blocks (lemo_block_attention_grad).
//
//   P = 2^(c2 <q,k> - lse2[q])      delta = <dO, O> of a row      dS = P (<dO, v> - delta)
//   dQ = scale dS K      dK = scale dS^T Q      dV = P^T dO        sums over what the lists pair, keys of a group shared by its heads
//
// Two passes without atomics, so that the same bits come on every run.  The first goes by query blocks, as the forward pass does, and
// leaves dQ and delta.  The second goes by key blocks: a key block's queries are those whose lists name it, which are turned
// round first -- a bit for every (query block, key block), counted, laid out as lists of ascending query blocks, and cut into items
// of at most `share` query blocks, since a popular block may be on every list.  The parts of a block that was cut are added in
// order.  Each pass forms its logits and probabilities again: 7 products for the 5 of the definition, which costs less than writing and
// reading dS (2 bytes a pair) would.
// delta comes from O as the forward call left it, rounded to bf16 (the gradient of the results that there are: O and lse2), and dS goes to
// the products as bf16: a value of either is off by at most 2^-8 of it.  P, dS and delta are formed in binary32, and so are all sums.
// 8192 tokens, 32 heads of 128, 16 blocks of 64 for 64 queries: 680 us (dQ 40 %, the lists 3 %, dK and dV 57 %), 460 TFLOP/s of the
// definition's 5 products, 640 of the 7; matrix cores are busy for 28 % of the first pass' cycles and 27 % of the second's, instructions
// go to them or the vector unit in 36 and 37 %, LDS is read in 17 and 27 %.  None of them bounds the passes: between two barriers a wave has one subtile of 32 rows
// or keys, whose logits, exponentials and products wait for each other, and two waves a SIMD cover it in part.  Eight waves on the same 64
// keys and one workgroup a CU: 725 us; fragments 3 or 4 steps ahead or precedence for waves in their products: within 1 %.
#include "block_attention.hpp"

namespace lemo {

// Stages are kept to 64 KB for two of them, where that suits the sharing waves: two workgroups fit a CU then, and the one's rows, lists and
// stores pass while the other computes.
template <int D, int SHARES> constexpr int BG_STAGE = D == 128 && SHARES <= 2 ? 2 : 4;  // subtiles of 32 of a stage

// ---- by query blocks: dQ, delta -----------------------------------------------------------------------

template <int D, int WAVES, int SUBS> struct DqGeo {
    using Tile = HeadTile<D>;
    static constexpr int SUB = 32 * Tile::ROWB, STAGE = 2 * SUBS * SUB;
    static constexpr int PITCH = D + 4, JOIN = WAVES * 32 * PITCH * 4;
    static constexpr int LIST = 2 * STAGE > JOIN ? 2 * STAGE : JOIN;
    static constexpr int lds(int subtiles) { return LIST + 16 + subtiles * 4; }  // (the number of them first, and whether sums are not finite)
};

template <int D, int WAVES, int KS, bool PACK>
__global__ __launch_bounds__(WAVES * 64, 2) void block_dq_kernel(BlockGradParams gp) {
    const BlockAttnParams& p = gp.a;
    constexpr int SUBS = BG_STAGE<D, KS>;
    using Geo = DqGeo<D, WAVES, SUBS>;
    using Tile = HeadTile<D>;
    constexpr int ROWS = WAVES / KS * 32;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    int* const keys = reinterpret_cast<int*>(smem + Geo::LIST) + 4;
    int &listed = keys[-4], &not_finite = keys[-3];

    int g, rank;
    decode_block(p.order, p.H_kv, p.n_qb * p.n_rt, g, rank, p.first + blockIdx.x);
    const int rt = rank % p.n_rt, qb = rank / p.n_rt;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool causal = (p.flags & LEMO_CAUSAL) != 0;
    const int S = p.S_k;
    for (long long n = (long long)blockIdx.x * (WAVES * 64) + tid; n < p.H_kv * gp.nb; n += (long long)gridDim.x * (WAVES * 64)) gp.counts[n] = 0;  // for the lists turned round
    const long long pos0 = p.q_start + (long long)qb * p.bq;
    const int rows = min(p.bq, p.S_q - qb * p.bq) * p.G, row_end = min(rows, (rt + 1) * ROWS);
    auto limit_of = [&](int row) { return causal ? (int)min(pos0 + row / p.G, (long long)S - 1) : S - 1; };

    int room = 0;  // (PACK) of the union's subtiles
    if constexpr (PACK) {
        if (tid == 0) not_finite = 0;
        const long long first = (long long)qb * p.pack;
        const int lists = (int)min((long long)p.pack, p.n_lists - first);
        room = min(p.pack * p.T, gp.nb) * (p.b / 32);
        union_subtiles<WAVES>(p.blocks + (first * p.H_kv + g) * p.T, (long long)p.H_kv * p.T, lists, p.T, p.b, gp.nb, limit_of(rows - 1), reinterpret_cast<unsigned*>(smem), keys,
                              room, &listed, wave, lane);
    } else {
        if (wave == 0) {
            const int n = rt * ROWS < rows ? list_subtiles(p.blocks + ((long long)qb * p.H_kv + g) * p.T, p.T, p.b, gp.nb, limit_of(row_end - 1), keys, lane) : 0;
            if (lane == 0) listed = n;
        }
        __syncthreads();
    }
    const int n_sub = listed, n_stage = (n_sub + SUBS - 1) / SUBS;

    const int row0 = rt * ROWS + wave / KS * 32, row = row0 + l32;
    const bool live = row < rows;
    const int lim = live ? limit_of(row) : -1;
    const int member = PACK ? l32 / (p.R / p.pack) : 0;  // the row's list
    const int clean = row0 < rows ? limit_of(row0) : -1, reach = row0 < rows ? limit_of(min(row0 + 31, rows - 1)) : -1;
    const long long i_row = (long long)qb * p.bq + row / p.G;
    const int h_row = g * p.G + row % p.G;
    u32x4 qf[Tile::CHUNKS], dof[Tile::CHUNKS];
    float delta = 0.f, lse = INFINITY;  // a row that is not there, or saw no key: probabilities 0
#pragma unroll
    for (int c = 0; c < Tile::CHUNKS; ++c) qf[c] = dof[c] = u32x4{0u, 0u, 0u, 0u};
    if (live) {
        const char* const q = reinterpret_cast<const char*>(p.Q + i_row * p.q_ts + h_row * p.q_hs);
        const char* const o = reinterpret_cast<const char*>(p.O + i_row * p.o_ts + h_row * p.o_hs);
        const char* const d = reinterpret_cast<const char*>(gp.dO + i_row * gp.do_ts + h_row * gp.do_hs);
#pragma unroll
        for (int c = 0; c < Tile::CHUNKS; ++c) {
            qf[c] = *reinterpret_cast<const u32x4*>(q + c * 32 + half * 16);
            dof[c] = *reinterpret_cast<const u32x4*>(d + c * 32 + half * 16);
            const u32x4 of = *reinterpret_cast<const u32x4*>(o + c * 32 + half * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                delta = fmaf(bf16lo_to_f32(of[e]), bf16lo_to_f32(dof[c][e]), fmaf(bf16hi_to_f32(of[e]), bf16hi_to_f32(dof[c][e]), delta));
        }
        const float stored = p.lse2[(long long)h_row * p.S_q + i_row];
        lse = stored == -INFINITY ? INFINITY : stored;
    }
    delta += __shfl_xor(delta, 32);
    if (live && half == 0 && wave % KS == 0) gp.delta[(long long)h_row * p.S_q + i_row] = delta;

    const char* const kbase = reinterpret_cast<const char*>(p.K + (long long)g * p.k_hs);
    const char* const vbase = reinterpret_cast<const char*>(p.V + (long long)g * p.v_hs);
    constexpr int RPI = 1024 / Tile::ROWB, PER_SUB = 32 / RPI, LOADS = 2 * SUBS * PER_SUB / WAVES;
    const int in_row = lane / Tile::PIECES, pos = lane % Tile::PIECES;
    auto load_stage = [&](int t, int buf) {
        int first_key[SUBS];  // all of them before the first load: a load orders memory accesses
#pragma unroll
        for (int s = 0; s < SUBS; ++s) first_key[s] = t * SUBS + s < n_sub ? __builtin_amdgcn_readfirstlane(keys[t * SUBS + s]) : S;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            constexpr int AT_ONCE = WAVES / PER_SUB > 1 ? WAVES / PER_SUB : 1;  // subtiles that the waves load together
            const int unit = i * WAVES + wave, part = unit % PER_SUB, which = AT_ONCE > 1 ? i * AT_ONCE + wave / PER_SUB : i * WAVES / PER_SUB;
            const bool v = i * WAVES >= SUBS * PER_SUB;
            int key = first_key[i * WAVES / PER_SUB % SUBS];
#pragma unroll
            for (int k = 1; k < AT_ONCE; ++k) key = wave / PER_SUB == k ? first_key[(i * WAVES / PER_SUB + k) % SUBS] : key;
            const int pitch = (int)(v ? p.v_ts : p.k_ts) * 2;
            const u32x4 rsrc = subtile_rsrc<D>(v ? vbase : kbase, min(key, S), S, pitch);
            const int r = part * RPI + in_row;
            lds_direct_b128(rsrc, lds_offset_of(smem) + buf * Geo::STAGE + which * Geo::SUB + part * 1024, r * pitch + ((pos ^ Tile::swz(r)) << 4));
        }
    };
    f32x16 dq[Tile::COLS];
    // PACK: what is not finite in K or V of blocks that other rows list, as in the forward pass
#pragma unroll
    for (int turn = 0; turn < (PACK ? 2 : 1); ++turn) {
#pragma unroll
    for (int c = 0; c < Tile::COLS; ++c) dq[c] = f32x16{0};
    if (n_stage > 0) {
        load_stage(0, 0);
        settle_stage();
    }
    for (int t = 0; t < n_stage; ++t) {
        __syncthreads();
        if (t + 1 < n_stage) load_stage(t + 1, (t + 1) & 1);
        const char* const sk = smem + (t & 1) * Geo::STAGE;
#pragma unroll 1
        for (int j = wave % KS; j < SUBS; j += KS) {
            if (t * SUBS + j >= n_sub) break;
            const int key = __builtin_amdgcn_readfirstlane(keys[t * SUBS + j]);
            if (key > reach) continue;
            const char* const ks = sk + j * Geo::SUB;
            const char* const vs = ks + SUBS * Geo::SUB;
            f32x16 acc = {0}, dp = {0};
#pragma unroll
            for (int c = 0; c < Tile::CHUNKS; ++c) {
                mma_chunk<bf16_t>(acc, Tile::row_fragment(ks, c, lane), qf[c]);  // [key][row]
                mma_chunk<bf16_t>(dp, Tile::row_fragment(vs, c, lane), dof[c]);
            }
            float ds[16];
            int mine = lim;
            bool masked = key + 31 > clean;
            if constexpr (PACK) {
                const unsigned bits = keys[room + t * SUBS + j];
                masked = masked || __popc(bits) != p.pack;
                mine = bits >> member & 1 ? lim : -1;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float x = fmaf(acc[r], p.c2, -lse);
                if (masked) x = key + acc_row(r, lane) <= mine ? x : -INFINITY;
                ds[r] = __builtin_amdgcn_exp2f(x) * (dp[r] - delta);
            }
            u32x4 pb[2];
#pragma unroll
            for (int c = 0; c < 2; ++c)
                pb[c] = u32x4{pack_bf16x2_hw(ds[8 * c + 0], ds[8 * c + 1]), pack_bf16x2_hw(ds[8 * c + 2], ds[8 * c + 3]),
                              pack_bf16x2_hw(ds[8 * c + 4], ds[8 * c + 5]), pack_bf16x2_hw(ds[8 * c + 6], ds[8 * c + 7])};
            if (turn == 0) {
#pragma unroll
                for (int col = 0; col < Tile::COLS; ++col)
#pragma unroll
                    for (int c = 0; c < 2; ++c) mma_chunk<bf16_t>(dq[col], Tile::column_fragment(ks, col, c, lane), pb[c]);  // [head column][row]
            } else {
#pragma unroll
                for (int col = 0; col < Tile::COLS; ++col) {
                    f32x16 sum = dq[col];
#pragma unroll
                    for (int c = 0; c < 2; ++c) mma_chunk<bf16_t>(sum, Tile::column_fragment(ks, col, c, lane), pb[c]);
#pragma unroll
                    for (int r = 0; r < 16; ++r) dq[col][r] = key <= mine ? sum[r] : dq[col][r];
                }
            }
        }
        settle_stage();
    }
    if (!PACK || turn == 1) break;
    float zero = 0.f;
#pragma unroll
    for (int col = 0; col < Tile::COLS; ++col)
#pragma unroll
        for (int r = 0; r < 16; ++r) zero = fmaf(dq[col][r], 0.f, zero);
    if (zero != 0.f) not_finite = 1;
    __syncthreads();
    if (!__builtin_amdgcn_readfirstlane(not_finite)) break;
    }
    // the waves that share rows add in LDS, in wave order
    __syncthreads();
    constexpr int LPR = D / 8;
    const int first = wave - wave % KS;
    float* const sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int col = 0; col < Tile::COLS; ++col)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4*>(sums + (wave * 32 + l32) * Geo::PITCH + col * 32 + q * 8 + half * 4) =
                f32x4{dq[col][q * 4], dq[col][q * 4 + 1], dq[col][q * 4 + 2], dq[col][q * 4 + 3]};
    __syncthreads();
    const int c0 = lane % LPR * 8;
#pragma unroll
    for (int r = 0; r < 32 / KS; r += 64 / LPR) {
        const int in = wave % KS * (32 / KS) + r + lane / LPR, out = row0 + in;
        if (out >= rows) continue;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < KS; ++w) {
            const float* at = sums + ((first + w) * 32 + in) * Geo::PITCH + c0;
            const f32x4 lo = *reinterpret_cast<const f32x4*>(at), hi = *reinterpret_cast<const f32x4*>(at + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[e + 4] += hi[e]; }
        }
        u32x4 piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) piece[e] = pack_bf16x2_hw(v[2 * e] * gp.scale, v[2 * e + 1] * gp.scale);
        *reinterpret_cast<u32x4*>(gp.dQ + (((long long)qb * p.bq + out / p.G) * p.H + g * p.G + out % p.G) * D + c0) = piece;
    }
}

// ---- the lists turned round ---------------------------------------------------------------------------

// A workgroup: 32 query blocks of one group; its four waves walk eight lists each and leave the blocks' bits in LDS.  The counts are zeros
// when it starts: the pass by query blocks cleared them.
__global__ __launch_bounds__(256) void block_bits_kernel(BlockGradParams gp) {
    const BlockAttnParams& p = gp.a;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    unsigned* const bits = reinterpret_cast<unsigned*>(smem);
    const int w = blockIdx.x, g = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int n = threadIdx.x; n < gp.nb; n += 256) bits[n] = 0;
    __syncthreads();
    for (int i = wave; i < 32; i += 4) {
        const int qb = w * 32 + i;
        if (qb >= p.n_qb) break;
        const long long last = p.q_start + min((long long)(qb + 1) * p.bq, (long long)p.S_q) - 1;
        walk_list(p.blocks + ((long long)qb * p.H_kv + g) * p.T, p.T, gp.nb, lane, [&](int n, bool counts) {
            if (counts && (!(p.flags & LEMO_CAUSAL) || (long long)n * p.b <= last)) atomicOr(bits + n, 1u << i);
        });
    }
    __syncthreads();
    for (int n = threadIdx.x; n < gp.nb; n += 256) {
        gp.bits[((long long)g * gp.nb + n) * gp.words + w] = bits[n];
        if (bits[n]) atomicAdd(gp.counts + g * gp.nb + n, __popc(bits[n]));  // (whole numbers: the order is nothing to the sum)
    }
}

// One workgroup: where every key block's list, items and partial results start.
__global__ __launch_bounds__(1024) void block_layout_kernel(BlockGradParams gp) {
    __shared__ int sums[3][16];
    const int total = gp.a.H_kv * gp.nb, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base[3] = {0, 0, 0};
    for (int n0 = 0; n0 < total; n0 += 1024) {
        const int n = n0 + (int)threadIdx.x;
        const int count = n < total ? gp.counts[n] : 0;
        const int items = n < total ? max(1, (count + gp.share - 1) / gp.share) : 0;
        const int mine[3] = {count, items, items > 1 ? items : 0};
        int sum[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            sum[k] = mine[k];
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) {
                const int other = __shfl_up(sum[k], s);
                if (lane >= s) sum[k] += other;
            }
            if (lane == 63) sums[k][wave] = sum[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            int all = 0;
            for (int v = 0; v < 16; ++v) {
                if (v < wave) sum[k] += sums[k][v];
                all += sums[k][v];
            }
            sum[k] += base[k] - mine[k];
            base[k] += all;
        }
        __syncthreads();
        if (n < total) {
            gp.first[n] = sum[0];
            gp.slots[n] = items > 1 ? sum[2] : -1;
            for (int i = 0; i < items; ++i)
                gp.items[sum[1] + i] = make_int4(n, sum[0] + i * gp.share, min(gp.share, count - i * gp.share), items > 1 ? sum[2] + i : -1);
        }
    }
    if (threadIdx.x == 0) gp.totals[0] = base[1];
}

// A wave: the list of a key block, a word of bits a lane.
__global__ __launch_bounds__(256) void block_lists_kernel(BlockGradParams gp) {
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6), g = blockIdx.y, lane = threadIdx.x & 63;
    if (n >= gp.nb) return;
    int* out = gp.lists + gp.first[g * gp.nb + n];
    for (int w0 = 0; w0 < gp.words; w0 += 64) {
        const int w = w0 + lane;
        unsigned set = w < gp.words ? gp.bits[((long long)g * gp.nb + n) * gp.words + w] : 0;
        const int mine = __popc(set);
        int sum = mine;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int other = __shfl_up(sum, s);
            if (lane >= s) sum += other;
        }
        for (int* at = out + sum - mine; set; set &= set - 1) *at++ = w * 32 + __ffs(set) - 1;
        out += __shfl(sum, 63);
    }
}

// ---- by key blocks: dK, dV ----------------------------------------------------------------------------

// KW waves hold 32 keys each, and SHARES as many share them and take the row subtiles of a stage in turn.  K stays in registers, and of V
// what fits beside it: with heads of 128 the columns from 16 V_HELD on come from LDS, 16 bytes of 32 keys side by side.
template <int D, int KW, int SHARES> struct DkvGeo {
    using Tile = HeadTile<D>;
    static constexpr int SUBS = SHARES, SUB = 32 * Tile::ROWB, STAGE = 2 * SUBS * SUB, ROWS = SUBS * 32;
    static constexpr int V = 2 * STAGE, V_HELD = D == 128 ? 2 : D / 16, V_SUB = (D / 16 - V_HELD) * 1024;  // where the keys' V stands; bytes of it for 32 keys
    static constexpr int PITCH = D + 4, JOIN = KW * SHARES * 32 * PITCH * 4;
    static constexpr int TABLE = V + KW * V_SUB > JOIN ? V + KW * V_SUB : JOIN;  // three tables of rows stand behind
    static constexpr int LDS = TABLE + 3 * ROWS * 5 * 4;
};

template <int D, int KW, int SHARES>
__global__ __launch_bounds__(KW * SHARES * 64, 2) void block_dkv_kernel(BlockGradParams gp) {
    const BlockAttnParams& p = gp.a;
    using Geo = DkvGeo<D, KW, SHARES>;
    using Tile = HeadTile<D>;
    constexpr int ROWS = Geo::ROWS, SUBS = Geo::SUBS, WAVES = KW * SHARES;
    // each die takes a contiguous range of the items: those at work on it together share a head's Q and dO in its L2
    const int total = __builtin_amdgcn_readfirstlane(gp.totals[0]), per_die = (total + NUM_XCD - 1) / NUM_XCD;
    const unsigned block = p.first + blockIdx.x;
    const int in_die = block / NUM_XCD, at_item = block % NUM_XCD * per_die + in_die;
    if (in_die >= per_die || at_item >= total) return;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    // tables: [ring of 3][ROWS] of each field
    unsigned* const t_q = reinterpret_cast<unsigned*>(smem + Geo::TABLE);
    unsigned* const t_d = t_q + 3 * ROWS;
    float* const t_lse = reinterpret_cast<float*>(t_d + 3 * ROWS);
    float* const t_delta = t_lse + 3 * ROWS;
    int* const t_pos = reinterpret_cast<int*>(t_delta + 3 * ROWS);

    int4 item = gp.items[at_item];  // (loaded by vector instructions, but uniform)
    item.x = __builtin_amdgcn_readfirstlane(item.x);
    item.z = __builtin_amdgcn_readfirstlane(item.z);
    const int g = item.x / gp.nb, n = item.x % gp.nb;
    const int* const list = gp.lists + item.y;
    const int n_rows = item.z * p.R, n_stage = (n_rows + ROWS - 1) / ROWS;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool causal = (p.flags & LEMO_CAUSAL) != 0;
    const int key0 = n * p.b + (blockIdx.y * KW + wave % KW) * 32;
    const int share = wave / KW;

    constexpr int V_HELD = Geo::V_HELD;
    u32x4 kf[Tile::CHUNKS], vf[V_HELD];
#pragma unroll
    for (int c = 0; c < Tile::CHUNKS; ++c) kf[c] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int c = 0; c < V_HELD; ++c) vf[c] = u32x4{0u, 0u, 0u, 0u};
    if (key0 + l32 < p.S_k) {  // (what no query sees are zeros, whatever it holds)
        const char* const k = reinterpret_cast<const char*>(p.K + (key0 + l32) * p.k_ts + g * p.k_hs);
        const char* const v = reinterpret_cast<const char*>(p.V + (key0 + l32) * p.v_ts + g * p.v_hs);
#pragma unroll
        for (int c = 0; c < Tile::CHUNKS; ++c) kf[c] = *reinterpret_cast<const u32x4*>(k + c * 32 + half * 16);
#pragma unroll
        for (int c = 0; c < V_HELD; ++c) vf[c] = *reinterpret_cast<const u32x4*>(v + c * 32 + half * 16);
    }
    const unsigned sv = lds_offset_of(smem) + Geo::V + wave % KW * Geo::V_SUB;

    // Rows of a stage: row v of the item is row v % R of query block list[v / R].  A thread looks after one row, in three steps a stage
    // apart, so that nothing waits for what it needs: its query block is loaded; its place goes into the table and its statistics are
    // loaded; they go into the table.  v / R and v % R are carried on from stage to stage, not divided anew.
    unsigned run_entry = (unsigned)tid / (unsigned)p.R, run_row = (unsigned)tid % (unsigned)p.R;
    const unsigned step_entry = (unsigned)ROWS / (unsigned)p.R, step_row = (unsigned)ROWS % (unsigned)p.R;
    int entry = -1;  // query block of the row that is placed next, and which of its rows that is
    unsigned row = 0;
    float r_lse = -INFINITY, r_delta = 0.f;
    auto fetch_entry = [&] {
        row = run_row;
        entry = -1;
        if (tid < ROWS && run_entry < (unsigned)item.z) entry = list[run_entry];
        run_entry += step_entry;
        run_row += step_row;
        if (run_row >= (unsigned)p.R) {
            run_row -= p.R;
            ++run_entry;
        }
    };
    auto place_row = [&](int t) {
        if (tid >= ROWS) return;
        const int at = t % 3 * ROWS + tid, in = (int)(row / (unsigned)p.G), h = g * p.G + (int)row - in * p.G, i = entry * p.bq + in;
        const bool there = entry >= 0 && i < p.S_q;  // otherwise: offsets past every operand, probabilities 0
        t_q[at] = there ? (unsigned)((i * p.q_ts + h * p.q_hs) * 2) : 0xffffff00u;
        t_d[at] = there ? (unsigned)((i * gp.do_ts + h * gp.do_hs) * 2) : 0xffffff00u;
        t_pos[at] = !there ? -1 : causal ? (int)min(p.q_start + i, (long long)0x7fffffff) : 0x7fffffff;
        r_lse = -INFINITY;
        r_delta = 0.f;
        if (there) {
            r_lse = p.lse2[(long long)h * p.S_q + i];
            r_delta = gp.delta[(long long)h * p.S_q + i];
        }
    };
    auto keep_row = [&](int t) {
        if (tid >= ROWS) return;
        const int at = t % 3 * ROWS + tid;
        t_lse[at] = r_lse == -INFINITY ? INFINITY : r_lse;
        t_delta[at] = r_delta;
    };
    const u32x4 q_rsrc = raw_rsrc(p.Q, ((p.S_q - 1) * p.q_ts + (p.H - 1) * p.q_hs + D) * 2);
    const u32x4 d_rsrc = raw_rsrc(gp.dO, ((p.S_q - 1) * gp.do_ts + (p.H - 1) * gp.do_hs + D) * 2);
    constexpr int RPI = 1024 / Tile::ROWB, UNITS = ROWS / RPI, LOADS = 2 * UNITS / WAVES;
    static_assert(UNITS % WAVES == 0, "");
    if constexpr (Geo::V_SUB > 0) {  // keys that are not there arrive as zeros
        for (int sub = wave; sub < KW; sub += WAVES) {
            const int begin = n * p.b + (blockIdx.y * KW + sub) * 32, pitch = (int)p.v_ts * 2;
            const u32x4 rsrc = subtile_rsrc<D>(reinterpret_cast<const char*>(p.V + (long long)g * p.v_hs), min(begin, p.S_k), p.S_k, pitch);
#pragma unroll
            for (int i = 0; i < Geo::V_SUB / 1024; ++i)
                lds_direct_b128(rsrc, lds_offset_of(smem) + Geo::V + sub * Geo::V_SUB + i * 1024, l32 * pitch + (V_HELD + i) * 32 + half * 16);
        }
    }
    auto load_stage = [&](int t, int buf) {
        int lane_here = lane;
        asm volatile("" : "+v"(lane_here));
        const int in_row = lane_here / Tile::PIECES, place = lane_here % Tile::PIECES;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int unit = i * WAVES + wave, part = unit % UNITS, r = part * RPI + in_row;
            const bool d = i * WAVES >= UNITS;  // the first half: Q, then dO
            const unsigned row = (d ? t_d : t_q)[t % 3 * ROWS + r];
            lds_direct_b128(d ? d_rsrc : q_rsrc, lds_offset_of(smem) + buf * Geo::STAGE + (d ? SUBS * Geo::SUB : 0) + part * 1024,
                            (int)(row + ((unsigned)(place ^ Tile::swz(r & 31)) << 4)));
        }
    };

    f32x16 dk[Tile::COLS], dv[Tile::COLS];
#pragma unroll
    for (int c = 0; c < Tile::COLS; ++c) dk[c] = dv[c] = f32x16{0};
    if (n_stage > 0) {
        fetch_entry();
        place_row(0);
        fetch_entry();
        __syncthreads();
        load_stage(0, 0);
        keep_row(0);
        place_row(1);
        fetch_entry();
        keep_row(1);
    }
    settle_stage();
    for (int t = 0; t < n_stage; ++t) {
        __syncthreads();  // stage t and the table of stage t + 1 are there
        place_row(t + 2);
        fetch_entry();
        if (t + 1 < n_stage) load_stage(t + 1, (t + 1) & 1);
        const char* const sq = smem + (t & 1) * Geo::STAGE;
        const int table = t % 3 * ROWS;
#pragma unroll 1
        for (int j = share; j < SUBS; j += SHARES) {
            if (t * ROWS + j * 32 >= n_rows) break;
            const int at = table + j * 32;
            const int top = __builtin_amdgcn_readfirstlane(t_pos[at + 31]);  // rows ascend: the last one has the highest position, if it is there
            if (top >= 0 && top < key0) continue;
            const unsigned qs = lds_offset_of(sq) + j * Geo::SUB, ds_ = qs + SUBS * Geo::SUB;
            int lane_here = lane;  // what follows from it is formed here, not kept through the loop: registers are short
            asm volatile("" : "+v"(lane_here));
            const TilePlace<D> place_in(lane_here);
            const int half = lane_here >> 5, key = key0 + (lane_here & 31);
            f32x16 acc = {0}, dp = {0};
            // Fragments come AHEAD steps before their products, and no earlier: all of them at once would not fit the registers, and what
            // then went to scratch would come back only after the stage's loads, which a wait for memory cannot tell from it.
            constexpr int AHEAD = 2;
            auto v_fragment = [&](int c) { return c < V_HELD ? vf[min(c, V_HELD - 1)] : *lds_pointer<const u32x4>(sv + lane_here * 16 + (c - V_HELD) * 1024); };
            {
                u32x4 fq[AHEAD], fd[AHEAD], fv[AHEAD];
#pragma unroll
                for (int c = 0; c < AHEAD; ++c) {
                    fq[c] = place_in.row_fragment(qs, c);
                    fd[c] = place_in.row_fragment(ds_, c);
                    fv[c] = v_fragment(c);
                }
#pragma unroll
                for (int c = 0; c < Tile::CHUNKS; ++c) {
                    __builtin_amdgcn_sched_barrier(0);
                    mma_chunk<bf16_t>(acc, fq[c % AHEAD], kf[c]);  // [row][key]
                    mma_chunk<bf16_t>(dp, fd[c % AHEAD], fv[c % AHEAD]);
                    if (c + AHEAD < Tile::CHUNKS) {
                        fq[c % AHEAD] = place_in.row_fragment(qs, c + AHEAD);
                        fd[c % AHEAD] = place_in.row_fragment(ds_, c + AHEAD);
                        fv[c % AHEAD] = v_fragment(c + AHEAD);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            float pr[16], ds[16];
            const bool masked = __builtin_amdgcn_readfirstlane(t_pos[at]) < key0 + 31;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 lse = *reinterpret_cast<const f32x4*>(t_lse + at + 8 * q + 4 * half);
                const f32x4 delta = *reinterpret_cast<const f32x4*>(t_delta + at + 8 * q + 4 * half);
                const int4 rp = *reinterpret_cast<const int4*>(t_pos + at + 8 * q + 4 * half);
                const int rpos[4] = {rp.x, rp.y, rp.z, rp.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * q + e;
                    float x = fmaf(acc[r], p.c2, -lse[e]);
                    if (masked) x = key <= rpos[e] ? x : -INFINITY;
                    pr[r] = __builtin_amdgcn_exp2f(x);
                    ds[r] = pr[r] * (dp[r] - delta[e]);
                }
            }
            u32x4 pp[2], pd[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                pp[c] = u32x4{pack_bf16x2_hw(pr[8 * c + 0], pr[8 * c + 1]), pack_bf16x2_hw(pr[8 * c + 2], pr[8 * c + 3]),
                              pack_bf16x2_hw(pr[8 * c + 4], pr[8 * c + 5]), pack_bf16x2_hw(pr[8 * c + 6], pr[8 * c + 7])};
                pd[c] = u32x4{pack_bf16x2_hw(ds[8 * c + 0], ds[8 * c + 1]), pack_bf16x2_hw(ds[8 * c + 2], ds[8 * c + 3]),
                              pack_bf16x2_hw(ds[8 * c + 4], ds[8 * c + 5]), pack_bf16x2_hw(ds[8 * c + 6], ds[8 * c + 7])};
            }
            {
                constexpr int STEPS = 2 * Tile::COLS;  // step i: column tile i / 2, chunk i % 2
                u32x4 fd[AHEAD], fq[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    fd[i] = place_in.column_fragment(ds_, i / 2, i % 2);
                    fq[i] = place_in.column_fragment(qs, i / 2, i % 2);
                }
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    mma_chunk<bf16_t>(dv[i / 2], fd[i % AHEAD], pp[i % 2]);  // [head column][key]
                    mma_chunk<bf16_t>(dk[i / 2], fq[i % AHEAD], pd[i % 2]);
                    if (i + AHEAD < STEPS) {
                        fd[i % AHEAD] = place_in.column_fragment(ds_, (i + AHEAD) / 2, (i + AHEAD) % 2);
                        fq[i % AHEAD] = place_in.column_fragment(qs, (i + AHEAD) / 2, (i + AHEAD) % 2);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        keep_row(t + 2);
        settle_stage();
    }
    // dK, then dV: the waves that share keys add in LDS, in wave order
    constexpr int LPR = D / 8;
    float* const sums = reinterpret_cast<float*>(smem);
    const int c0 = lane % LPR * 8;
    const int slot = item.w;
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int col = 0; col < Tile::COLS; ++col)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = which ? dv[col][q * 4 + e] : dk[col][q * 4 + e] * gp.scale;
                *reinterpret_cast<f32x4*>(sums + (wave * 32 + l32) * Geo::PITCH + col * 32 + q * 8 + half * 4) = v;
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 32 / SHARES; r += 64 / LPR) {
            const int in = share * (32 / SHARES) + r + lane / LPR;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < SHARES; ++w) {
                const float* at = sums + ((w * KW + wave % KW) * 32 + in) * Geo::PITCH + c0;
                const f32x4 lo = *reinterpret_cast<const f32x4*>(at), hi = *reinterpret_cast<const f32x4*>(at + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[e + 4] += hi[e]; }
            }
            const int j = key0 + in;
            if (slot >= 0) {
                float* part = gp.partial + (((long long)slot * 2 + which) * p.b + (j - n * p.b)) * D + c0;
                *reinterpret_cast<f32x4*>(part) = f32x4{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4*>(part + 4) = f32x4{v[4], v[5], v[6], v[7]};
            } else if (j < gp.S_all) {
                u32x4 piece;
#pragma unroll
                for (int e = 0; e < 4; ++e) piece[e] = pack_bf16x2_hw(v[2 * e], v[2 * e + 1]);
                *reinterpret_cast<u32x4*>((which ? gp.dV : gp.dK) + ((long long)j * p.H_kv + g) * D + c0) = piece;
            }
        }
    }
}

// The key blocks that were cut: their parts added in order.
template <int D> __global__ __launch_bounds__(256) void block_dkv_join_kernel(BlockGradParams gp) {
    const BlockAttnParams& p = gp.a;
    const int at = p.first + blockIdx.x, g = at / gp.nb, n = at % gp.nb, slot = gp.slots[at];
    if (slot < 0) return;
    const int parts = (gp.counts[at] + gp.share - 1) / gp.share;
    constexpr int LPR = D / 8;
    for (int u = blockIdx.y * 256 + threadIdx.x; u < 2 * p.b * LPR; u += gridDim.y * 256) {
        const int which = u / (p.b * LPR), j = u / LPR % p.b, c0 = u % LPR * 8, key = n * p.b + j;
        if (key >= gp.S_all) continue;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < parts; ++w) {
            const float* part = gp.partial + (((long long)(slot + w) * 2 + which) * p.b + j) * D + c0;
            const f32x4 lo = *reinterpret_cast<const f32x4*>(part), hi = *reinterpret_cast<const f32x4*>(part + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[e + 4] += hi[e]; }
        }
        u32x4 piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) piece[e] = pack_bf16x2_hw(v[2 * e], v[2 * e + 1]);
        *reinterpret_cast<u32x4*>((which ? gp.dV : gp.dK) + ((long long)key * p.H_kv + g) * D + c0) = piece;
    }
}

// ---- host ---------------------------------------------------------------------------------------------

BlockGradLayout block_grad_layout(long long S_q, long long S_k, int H, int H_kv, int d, int T, int b, int bq) {
    BlockGradLayout l{};
    const long long n_qb = (S_q + bq - 1) / bq, nb = (S_k + b - 1) / b, words = (n_qb + 31) / 32, R = (long long)bq * (H / H_kv);
    const long long entries = n_qb * H_kv * (T < nb ? T : nb);
    // Items: some thousand for the whole launch and one a key block, of 256 rows at least.  The whole call, us, for about 512 / 1024 / 1536 / 2048:
    // 8192 tokens, 32 heads, 16 blocks of 64 666 / 667 / 733 / 750, with 8 key heads 789 / 683 / 660 / 659; 32768, 32 / 8 heads 2400 / 2786 / 2407 /
    // 2534; 2999, 32 / 8 heads, lists of 12 for 16 queries 262 / 243 / 233 / 247
    long long share = (entries + 1023) / 1024;
    const long long least = (256 + R - 1) / R;
    if (share < least) share = least;
    l.share = (int)(share < n_qb ? share : n_qb);
    l.max_items = (int)(entries / l.share + H_kv * nb);  // (each key block one at least)
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    l.delta = take((size_t)H * S_q * 4);
    l.bits = take((size_t)H_kv * words * nb * 4);
    l.counts = take((size_t)H_kv * nb * 4);
    l.first = take((size_t)H_kv * nb * 4);
    l.lists = take((size_t)entries * 4);
    l.slots = take((size_t)H_kv * nb * 4);
    l.items = take((size_t)l.max_items * 16);
    l.totals = take(4);
    // parts of key blocks with more than one: at most twice as many as their query blocks fill
    const long long parts = 2 * (entries / l.share) < l.max_items ? 2 * (entries / l.share) : l.max_items;
    l.partial = take((size_t)parts * 2 * b * d * 4);
    l.bytes = at;
    return l;
}

template <int D, int KS> constexpr int dq_lds(int subtiles) { return DqGeo<D, 4, BG_STAGE<D, KS>>::lds(subtiles); }

template <int D, int KS, bool PACK> static int run_dq(BlockGradParams gp, int subtiles, hipStream_t st) {
    return launch_in_turns((long long)gp.a.n_qb * gp.a.n_rt * gp.a.H_kv, 256, [&](long long first, unsigned count) {
        gp.a.first = (int)first;
        hipLaunchKernelGGL((block_dq_kernel<D, 4, KS, PACK>), dim3(count), dim3(256), (dq_lds<D, KS>(PACK ? 2 * subtiles : subtiles)), st, gp);
    });
}

// Waves that share keys in the pass by key blocks.  Heads of 128: so many that two workgroups fit a CU, and the one's begin and end pass
// while the other computes; heads of 64, whose tiles are half as large: more.  us of the whole call, 8192 tokens: 32 heads of 128, 8
// blocks of 128 keys 735 with 1 / 746 with 2; 16 of 64 678 with 2 / 725 with 4; 32 of 32 997 with 2 / 1083 with 4; 32 / 8 heads of 64,
// lists for 16 queries, 8 of 128 489 with 1 / 480 with 2; 16 of 64 513 with 2 / 526 with 4; 32 of 32 643 with 2 / 578 with 4.
template <int D, int KW> constexpr int DKV_SHARES = KW == 4 ? (D == 128 ? 1 : 2) : KW == 2 || D == 128 ? 2 : 4;

template <int D, int KW> static int run_dkv(BlockGradParams gp, hipStream_t st) {
    constexpr int SHARES = DKV_SHARES<D, KW>;
    return launch_in_turns(((long long)gp.max_items + NUM_XCD - 1) / NUM_XCD * NUM_XCD, KW * SHARES * 64, [&](long long first, unsigned count) {
        gp.a.first = (int)first;
        hipLaunchKernelGGL((block_dkv_kernel<D, KW, SHARES>), dim3(count, (unsigned)(gp.a.b / (32 * KW))), dim3(KW * SHARES * 64), (DkvGeo<D, KW, SHARES>::LDS), st, gp);
    });
}

template <int D> static int launch_grad(BlockGradParams gp, hipStream_t st) {
    static const int unready = raise_lds_limits({{reinterpret_cast<const void*>(&block_dq_kernel<D, 4, 1, false>), dq_lds<D, 1>(MAX_LISTED_SUBTILES)},
                                                 {reinterpret_cast<const void*>(&block_dq_kernel<D, 4, 2, false>), dq_lds<D, 2>(MAX_LISTED_SUBTILES)},
                                                 {reinterpret_cast<const void*>(&block_dq_kernel<D, 4, 4, false>), dq_lds<D, 4>(MAX_LISTED_SUBTILES)},
                                                 {reinterpret_cast<const void*>(&block_dq_kernel<D, 4, 4, true>), dq_lds<D, 4>(2 * MAX_PACKED_SUBTILES)},
                                                 {reinterpret_cast<const void*>(&block_dkv_kernel<D, 1, DKV_SHARES<D, 1>>), DkvGeo<D, 1, DKV_SHARES<D, 1>>::LDS},
                                                 {reinterpret_cast<const void*>(&block_dkv_kernel<D, 2, DKV_SHARES<D, 2>>), DkvGeo<D, 2, DKV_SHARES<D, 2>>::LDS},
                                                 {reinterpret_cast<const void*>(&block_dkv_kernel<D, 4, DKV_SHARES<D, 4>>), DkvGeo<D, 4, DKV_SHARES<D, 4>>::LDS}});
    if (unready) return unready;
    BlockAttnParams& p = gp.a;
    BlockGradParams by_rows = gp;  // (the pass by query blocks may take several lists together)
    {
        BlockAttnParams& q = by_rows.a;
        q.lengths = nullptr;
        const int subtiles = block_attention_packed(q), tile = block_attention_tile_rows(q.R, false);
        q.n_rt = (q.R + tile - 1) / tile;
        q.n_parts = 1;
        q.order = head_order(q.H_kv, false, 8);
        const int rc = tile == 128 ? run_dq<D, 1, false>(by_rows, subtiles, st) : tile == 64 ? run_dq<D, 2, false>(by_rows, subtiles, st)
                     : q.pack == 1 ? run_dq<D, 4, false>(by_rows, subtiles, st) : run_dq<D, 4, true>(by_rows, subtiles, st);
        if (rc) return rc;
    }
    hipLaunchKernelGGL(block_bits_kernel, dim3((unsigned)gp.words, (unsigned)p.H_kv), dim3(256), gp.nb * 4, st, gp);
    hipLaunchKernelGGL(block_layout_kernel, dim3(1), dim3(1024), 0, st, gp);
    hipLaunchKernelGGL(block_lists_kernel, dim3((unsigned)((gp.nb + 3) / 4), (unsigned)p.H_kv), dim3(256), 0, st, gp);
    int rc = (int)hipGetLastError();
    if (rc) return rc;
    // as many keys a workgroup as a key block has, so that rows are gathered for all of them at once (us of the whole call with eight, eight and
    // four waves on 128, 64 and 32 keys, 8192 tokens: 32 heads of 128, 8 blocks of 128 746 / 827 / 1229)
    const int subs = p.b / 32;
    rc = subs % 4 == 0 ? run_dkv<D, 4>(gp, st) : subs % 2 == 0 ? run_dkv<D, 2>(gp, st) : run_dkv<D, 1>(gp, st);
    if (rc) return rc;
    return launch_in_turns((long long)p.H_kv * gp.nb, 256, [&](long long first, unsigned count) {
        p.first = (int)first;
        hipLaunchKernelGGL((block_dkv_join_kernel<D>), dim3(count, 2), dim3(256), 0, st, gp);
    });
}

int launch_block_attention_grad(BlockGradParams gp, int d, hipStream_t st) { return d == 64 ? launch_grad<64>(gp, st) : launch_grad<128>(gp, st); }

}  // namespace lemo
