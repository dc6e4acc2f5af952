// The cheap score and the choice: means of the key blocks, and for every query block and group of heads the T blocks whose mean key
// agrees best with the group's queries.
//
//   means[n,g,:] = mean of K[j,g,:] over block n            s[m,g,n] = < sum of the block's queries over the heads of g, means[n,g,:] >
//
// The means read K once and are memory bound.  Scores are formed and compared in 64 bits: which of two nearly equal scores is the larger
// then does not depend on the order of a sum, and a list is the definition's but for ties closer than 2^-50 of the terms.  2 d flops in
// 64 bits for every query block and key block are far less than what the attention does with the lists.
#include <type_traits>

#include "block_attention.hpp"

namespace lemo {

template <typename T> struct KeyPiece;
template <> struct KeyPiece<bf16_t> {
    static constexpr int E = 8;
    __device__ static void get(const u32x4& v, float (&x)[E]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo_to_f32(v[i]); x[2 * i + 1] = bf16hi_to_f32(v[i]); }
    }
};
template <> struct KeyPiece<float> {
    static constexpr int E = 4;
    __device__ static void get(const u32x4& v, float (&x)[E]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
    }
};

// A workgroup: one block of keys, 64 pieces of the rows [H_kv * d]; its four waves take every fourth key.
template <typename T>
__device__ __forceinline__ void block_mean(const char* K, long long first, int keys, int H_kv, int d, long long k_ts, long long k_hs, float* out) {
    constexpr int E = KeyPiece<T>::E;
    __shared__ double share[4][64][E + 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, piece = blockIdx.y * 64 + lane, per_head = d / E;
    const int g = piece / per_head, c = piece % per_head * E;
    double sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0;
    if (g < H_kv) {
        const char* at = K + (first * k_ts + g * k_hs + c) * (long long)(16 / E);
#pragma unroll 4
        for (int j = wave; j < keys; j += 4) {
            float x[E];
            KeyPiece<T>::get(*reinterpret_cast<const u32x4*>(at + j * k_ts * (long long)(16 / E)), x);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += (double)x[e];
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) share[wave][lane][e] = sum[e];
    __syncthreads();
    if (wave != 0 || g >= H_kv) return;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = (float)(((share[0][lane][e + i] + share[1][lane][e + i]) + (share[2][lane][e + i] + share[3][lane][e + i])) / (double)keys);
        *reinterpret_cast<f32x4*>(out + g * d + c + e) = v;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void block_means_kernel(const void* K, long long S, int H_kv, int d, long long k_ts, long long k_hs, int b, float* means,
                                                          long long first_block) {
    const long long n = first_block + blockIdx.x, first = n * b;
    block_mean<T>(static_cast<const char*>(K), first, (int)min((long long)b, S - first), H_kv, d, k_ts, k_hs, means + n * H_kv * d);
}

// Single tokens: the block that the newest token of a sequence has filled, if it has.
template <typename T>
__global__ __launch_bounds__(256) void block_means_step_kernel(const void* K, const int* lengths, long long S_max, int H_kv, int d, long long k_ss,
                                                               long long k_ts, long long k_hs, int b, float* means, int nb, int first) {
    const int s = first + blockIdx.x, S = (int)min((long long)lengths[s], S_max);
    if (S <= 0 || S % b != 0) return;  // the whole workgroup
    const long long n = S / b - 1;
    block_mean<T>(static_cast<const char*>(K) + s * k_ss * (long long)(16 / KeyPiece<T>::E), n * b, b, H_kv, d, k_ts, k_hs,
                  means + ((long long)s * nb + n) * H_kv * d);
}

// Scores as whole numbers in the same order.  Not a candidate: 0; the block of a query itself: the highest; what is not a number lies
// somewhere between, so that a list stays in range whatever the scores are.
__device__ __forceinline__ unsigned long long score_key(double s) {
    const unsigned long long u = __double_as_longlong(s + 0.0);  // (-0 becomes +0: they tie)
    const unsigned long long k = u >> 63 ? ~u : u | 1ull << 63;
    return k == 0 ? 1 : k == ~0ull ? ~0ull - 1 : k;
}

// the sum over the 16 lanes of a row, in every lane: four rotations within the row
template <int BY> __device__ __forceinline__ double rotated(double v) {
    const unsigned long long u = __double_as_longlong(v);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)u, 0x120 + BY, 0xf, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), 0x120 + BY, 0xf, 0xf, false);
    return __longlong_as_double((unsigned long long)(unsigned)hi << 32 | (unsigned)lo);
}
__device__ __forceinline__ double row_total(double v) {
    v += rotated<8>(v);
    v += rotated<4>(v);
    v += rotated<2>(v);
    return v + rotated<1>(v);
}

// A workgroup makes the lists of RB query blocks of one group.
//   1  the queries of a list are added up: teams of lanes that hold a row of 16-byte pieces, several to a list where RB is small
//   2  scores.  16 lists: 16 lists by 16 key blocks a chain of 64-bit MFMAs (v_mfma_f64_16x16x4: lane l holds row l % 16, one value
//      of the contraction, the (l / 16)-th; the result's register i is row 4 i + l / 16), at the rate of the vector unit but with
//      no sums across lanes.  Fewer lists would leave its rows empty: 16 lanes a key block, vector arithmetic.
//   3  a wave a list: the highest threshold that T scores reach, bit by bit, in the upper halves of the scores first, whose 20
//      mantissa bits nearly always tell them apart; then the blocks at or above it, in order
typedef __attribute__((ext_vector_type(4))) double f64x4;
constexpr int SEL_LEAST = 512, SEL_LDS = 32 << 10;

template <typename T, int D, int RB, int THREADS> struct SelGeo {
    static constexpr int E = KeyPiece<T>::E, LANES = D / E, TEAMS = THREADS / LANES, TPL = TEAMS > RB ? TEAMS / RB : 1;  // teams a list
    static constexpr int PITCH = D + 2;                                                                          // of a list's sums
    static constexpr int SUMS = RB * PITCH * 8, SCRATCH = RB * TPL * D * 8;
    static constexpr int lds(int nb) { return SUMS + (RB * nb * 8 > SCRATCH ? RB * nb * 8 : SCRATCH); }
};

template <typename T, int D, int RB, int THREADS>
__global__ __launch_bounds__(THREADS) void select_blocks_kernel(BlockSelectParams p) {
    using Geo = SelGeo<T, D, RB, THREADS>;
    constexpr int WAVES = THREADS / 64;
    constexpr int E = Geo::E, TPL = Geo::TPL;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int counts[RB], owns[RB];
    double* const sums = reinterpret_cast<double*>(smem);                                  // [RB][PITCH]
    double* const scratch = reinterpret_cast<double*>(smem + Geo::SUMS);                    // [RB * TPL][D]; then
    unsigned long long* const keys = reinterpret_cast<unsigned long long*>(smem + Geo::SUMS);  // [RB][nb]
    const unsigned block = p.first + blockIdx.x;
    const int g = block % p.H_kv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long qb0 = (long long)(block / p.H_kv) * RB;
    const bool causal = (p.flags & LEMO_CAUSAL) != 0;
    const int S = p.lengths ? min(max(p.lengths[qb0], 0), p.S_k) : p.S_k;  // (single tokens: RB = 1)
    auto queries_of = [&](long long qb) { return (int)max(0ll, min((long long)p.bq, p.S_q - qb * p.bq)); };
    if (tid < RB) {
        const long long qb = qb0 + tid, pos0 = p.lengths ? S - 1 : p.q_start + qb * p.bq;
        const int queries = queries_of(qb), nb = (S + p.b - 1) / p.b;
        const long long last = min(pos0 + queries - 1, (long long)S - 1);
        // candidates: blocks that begin before the last query ends; causal: those from `owns` on hold a query
        counts[tid] = S <= 0 || queries == 0 ? 0 : causal ? (int)min((long long)nb, last / p.b + 1) : nb;
        owns[tid] = causal ? (int)min(pos0 / p.b, (long long)nb) : nb;
    }
    for (int u = tid / Geo::LANES; u < RB * TPL; u += Geo::TEAMS) {
        const long long qb = qb0 + u / TPL;
        const int rows = queries_of(qb) * p.G, c = tid % Geo::LANES * E;
        const char* const base = reinterpret_cast<const char*>(p.Q) + (qb * p.bq * p.q_ts + (long long)g * p.G * p.q_hs + c) * (16 / E);
        double sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0;
#pragma unroll 8
        for (int r = u % TPL; r < rows; r += TPL) {
            const int i = r / p.G;
            float x[E];
            KeyPiece<T>::get(*reinterpret_cast<const u32x4*>(base + (i * p.q_ts + (long long)(r - i * p.G) * p.q_hs) * (16 / E)), x);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += (double)x[e];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) scratch[u * D + c + e] = sum[e];
    }
    __syncthreads();
    for (int u = tid; u < RB * D; u += THREADS) {
        const int list = u / D, c = u % D;
        double all = scratch[list * TPL * D + c];
        for (int t = 1; t < TPL; ++t) all += scratch[(list * TPL + t) * D + c];
        sums[list * Geo::PITCH + c] = all;
    }
    __syncthreads();
    int most = 0;
#pragma unroll
    for (int r = 0; r < RB; ++r) most = max(most, counts[r]);
    const float* const means = p.means + (p.lengths ? qb0 * p.means_ss : 0) + (long long)g * D;
    if constexpr (RB < 16) {
        constexpr int PER = D / 16;  // 16 lanes a block, PER columns each
        const int l16 = lane & 15;
        double q[RB][PER];
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int i = 0; i < PER; ++i) q[r][i] = sums[r * Geo::PITCH + (i / 4 * 16 + l16) * 4 + i % 4];
        constexpr int AHEAD = RB == 1 ? 4 : 2;  // blocks whose means are under way together
        for (int n0 = wave * 4; n0 < most; n0 += AHEAD * WAVES * 4) {
            f32x4 m[AHEAD][PER / 4];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int i = 0; i < PER / 4; ++i)
                    m[k][i] = *reinterpret_cast<const f32x4*>(means + (long long)min(n0 + k * WAVES * 4 + (lane >> 4), most - 1) * p.H_kv * D + l16 * 4 + i * 64);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int n = n0 + k * WAVES * 4 + (lane >> 4);
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    double s = 0.0;
#pragma unroll
                    for (int i = 0; i < PER; ++i) s = fma(q[r][i], (double)m[k][i / 4][i % 4], s);
                    s = row_total(s);
                    if (l16 == 0 && n < counts[r]) keys[r * p.nb + n] = n >= owns[r] ? ~0ull : score_key(s);
                }
            }
        }
    } else {
        const int l16 = lane & 15, q4 = lane >> 4;
        double a[D / 4];  // MFMA 4 j + s contracts columns 16 j + 4 (l / 16) + s
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s) a[4 * j + s] = l16 < RB ? sums[l16 * Geo::PITCH + 16 * j + 4 * q4 + s] : 0.0;
        for (int n0 = wave * 16; n0 < most; n0 += WAVES * 16) {
            const int n = min(n0 + l16, most - 1);
            f32x4 m[D / 16];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) m[j] = *reinterpret_cast<const f32x4*>(means + (long long)n * p.H_kv * D + 4 * q4 + 16 * j);
            f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int s = 0; s < 4; ++s) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(a[4 * j + s], (double)m[j][s], acc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int list = 4 * i + q4;
                if (list < RB && n0 + l16 < counts[list]) keys[list * p.nb + n0 + l16] = n0 + l16 >= owns[list] ? ~0ull : score_key(acc[i]);
            }
        }
    }
    __syncthreads();
    // The whole 64 bits of a list's scores, one wave: where the upper halves do not tell (or are too many for the registers)
    auto choose = [&](int list) {
        const int count = counts[list], wanted = min(p.T, count);
        const unsigned long long* const mine = keys + list * p.nb;
        int* const out = p.blocks + ((qb0 + list) * p.H_kv + g) * p.T;
        unsigned long long cut = 1;
        bool exact = count <= p.T;
        if (!exact) {
            constexpr int HELD = 8;  // upper halves of the first 512 scores stay in registers
            unsigned high[HELD], top = 0;
#pragma unroll
            for (int i = 0; i < HELD; ++i) high[i] = i * 64 + lane < count ? (unsigned)(mine[i * 64 + lane] >> 32) : 0;
            for (int bit = 31; bit >= 0 && !exact; --bit) {
                const unsigned mark = top | 1u << bit;
                int reach = 0;
#pragma unroll
                for (int i = 0; i < HELD; ++i) reach += (int)__popcll(__ballot(high[i] >= mark));
                for (int n0 = HELD * 64; n0 < count; n0 += 64) reach += (int)__popcll(__ballot(n0 + lane < count && (unsigned)(mine[n0 + lane] >> 32) >= mark));
                if (reach >= wanted) top = mark;
                exact = reach == wanted;
            }
            cut = (unsigned long long)top << 32;
            for (int bit = 31; bit >= 0 && !exact; --bit) {
                const unsigned long long mark = cut | 1ull << bit;
                int reach = 0;
                for (int n0 = 0; n0 < count; n0 += 64) reach += (int)__popcll(__ballot(n0 + lane < count && mine[n0 + lane] >= mark));
                if (reach >= wanted) cut = mark;
                exact = reach == wanted;
            }
        }
        int ties = 0, at = 0;  // of the keys that equal the threshold, the first ones
        if (!exact) {
            ties = wanted;
            for (int n0 = 0; n0 < count; n0 += 64) ties -= (int)__popcll(__ballot(n0 + lane < count && mine[n0 + lane] > cut));
        }
        const unsigned long long before = (1ull << lane) - 1;
        for (int n0 = 0; n0 < count; n0 += 64) {
            const unsigned long long k = n0 + lane < count ? mine[n0 + lane] : 0;
            const unsigned long long equal = __ballot(!exact && k == cut);
            const bool taken = exact ? k >= cut : k > cut || (k == cut && (int)__popcll(equal & before) < ties);
            ties = max(0, ties - (int)__popcll(equal));
            const unsigned long long all = __ballot(taken);
            if (taken) out[at + (int)__popcll(all & before)] = n0 + lane;
            at += (int)__popcll(all);
        }
        for (int e = at + lane; e < p.T; e += 64) out[e] = -1;
    };
    if constexpr (RB < 16) {
        for (int list = wave; list < RB; list += WAVES)
            if (queries_of(qb0 + list) > 0) choose(list);
    } else {
        // four lists a wave at a time, each in 16 lanes, by the upper halves of the scores
        const int list = wave * 4 + (lane >> 4), l16 = lane & 15, shift = lane & 48;
        const bool there = queries_of(qb0 + list) > 0;
        const int count = there ? counts[list] : 0, wanted = min(p.T, count);
        const unsigned long long* const mine = keys + list * p.nb;
        bool exact = count <= p.T;
        unsigned top = 0;
        auto by_halves = [&](auto held) {
            constexpr int HELD = decltype(held)::value;
            unsigned high[HELD];
#pragma unroll
            for (int i = 0; i < HELD; ++i) high[i] = i * 16 + l16 < count ? (unsigned)(mine[i * 16 + l16] >> 32) : 0;
            for (int bit = 31; bit >= 0 && !__all(exact); --bit) {
                const unsigned mark = top | 1u << bit;
                int reach = 0;
#pragma unroll
                for (int i = 0; i < HELD; ++i) reach += high[i] >= mark;
                reach += __builtin_amdgcn_update_dpp(0, reach, 0x128, 0xf, 0xf, false);  // (the sum of the 16 lanes, by rotations)
                reach += __builtin_amdgcn_update_dpp(0, reach, 0x124, 0xf, 0xf, false);
                reach += __builtin_amdgcn_update_dpp(0, reach, 0x122, 0xf, 0xf, false);
                reach += __builtin_amdgcn_update_dpp(0, reach, 0x121, 0xf, 0xf, false);
                if (!exact) {
                    if (reach >= wanted) top = mark;
                    exact = reach == wanted;
                }
            }
            int at = 0;
            int* const out = p.blocks + ((qb0 + list) * p.H_kv + g) * p.T;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const bool taken = exact && i * 16 + l16 < count && high[i] >= top;
                const unsigned all = (unsigned)(__ballot(taken) >> shift) & 0xffffu;
                if (taken) out[at + __popc(all & ((1u << l16) - 1))] = i * 16 + l16;
                at += __popc(all);
            }
            if (there && exact)
                for (int e = at + l16; e < p.T; e += 16) out[e] = -1;
        };
        if (most <= 128) by_halves(std::integral_constant<int, 8>{});
        else by_halves(std::integral_constant<int, SEL_LDS / (16 * 8) / 16>{});
        for (unsigned long long rest = __ballot(!exact && l16 == 0); rest; rest &= rest - 1) choose(wave * 4 + (__ffsll(rest) - 1) / 16);
    }
}

int launch_block_means(const void* K, long long S, int H_kv, int d, lemo_dtype_t dt, long long k_ts, long long k_hs, int b, float* means, hipStream_t st) {
    const int pieces = H_kv * (d / (dt == LEMO_BF16 ? 8 : 4));
    return launch_in_turns((S + b - 1) / b, 256, [&](long long first, unsigned count) {
        const dim3 grid(count, (unsigned)((pieces + 63) / 64));
        if (dt == LEMO_BF16) hipLaunchKernelGGL((block_means_kernel<bf16_t>), grid, dim3(256), 0, st, K, S, H_kv, d, k_ts, k_hs, b, means, first);
        else hipLaunchKernelGGL((block_means_kernel<float>), grid, dim3(256), 0, st, K, S, H_kv, d, k_ts, k_hs, b, means, first);
    });
}

int launch_block_means_step(const void* K, const int* lengths, int B, long long S_max, int H_kv, int d, lemo_dtype_t dt, long long k_ss, long long k_ts,
                            long long k_hs, int b, float* means, int nb, hipStream_t st) {
    const int pieces = H_kv * (d / (dt == LEMO_BF16 ? 8 : 4));
    return launch_in_turns(B, 256, [&](long long first, unsigned count) {
        const dim3 grid(count, (unsigned)((pieces + 63) / 64));
        if (dt == LEMO_BF16)
            hipLaunchKernelGGL((block_means_step_kernel<bf16_t>), grid, dim3(256), 0, st, K, lengths, S_max, H_kv, d, k_ss, k_ts, k_hs, b, means, nb, (int)first);
        else hipLaunchKernelGGL((block_means_step_kernel<float>), grid, dim3(256), 0, st, K, lengths, S_max, H_kv, d, k_ss, k_ts, k_hs, b, means, nb, (int)first);
    });
}

template <typename T, int D, int RB, int THREADS> static int run_select_lists(BlockSelectParams p, hipStream_t st) {
    return launch_in_turns(((long long)p.n_qb + RB - 1) / RB * p.H_kv, THREADS, [&](long long first, unsigned count) {
        p.first = (int)first;
        hipLaunchKernelGGL((select_blocks_kernel<T, D, RB, THREADS>), dim3(count), dim3(THREADS), (SelGeo<T, D, RB, THREADS>::lds(p.nb)), st, p);
    });
}

template <typename T, int D> static int run_select_blocks(const BlockSelectParams& p, hipStream_t st) {
    static const int err = raise_lds_limits({{reinterpret_cast<const void*>(&select_blocks_kernel<T, D, 1, 256>), SelGeo<T, D, 1, 256>::lds(MAX_LISTED_BLOCKS)},
                                             {reinterpret_cast<const void*>(&select_blocks_kernel<T, D, 1, 1024>), SelGeo<T, D, 1, 1024>::lds(MAX_LISTED_BLOCKS)}});
    if (err) return err;
    const long long lists = (long long)p.n_qb * p.H_kv;
    // few lists: 16 waves each (us, 1024 / 256 threads, one token of 1, 8, 64, 256 sequences, 32 / 8 heads, 512 to 64 blocks: 11.9 / 13.5,
    // 10.2 / 10.2, 27 / 22, 42 / 10)
    if (lists <= 64) return run_select_lists<T, D, 1, 1024>(p, st);
    // lists of few rows: the more of them a workgroup makes, the less often it reads the means; their scores take LDS, and there have
    // to be workgroups (single tokens have means of their own each).  us for 16 / 4 / 1 lists a workgroup: 3001 queries, 16 heads of 64, a list
    // each from 94 blocks 30 / 78 / 137; 8192, 16 of 128, a list for 8 from 128 blocks 22 / 47 / 79; 800, 8 of 64, from 25 - / 12 / 19
    if (p.bq * p.G < 64 && !p.lengths) {
        if (lists >= 16 * SEL_LEAST && p.nb * 16 * 8 <= SEL_LDS) return run_select_lists<T, D, 16, 256>(p, st);
        if (lists >= 4 * SEL_LEAST && p.nb * 4 * 8 <= SEL_LDS) return run_select_lists<T, D, 4, 256>(p, st);
    }
    return run_select_lists<T, D, 1, 256>(p, st);
}

int launch_select_blocks(const BlockSelectParams& p, lemo_dtype_t dt, hipStream_t st) {
    if (dt == LEMO_BF16) return p.d == 64 ? run_select_blocks<bf16_t, 64>(p, st) : run_select_blocks<bf16_t, 128>(p, st);
    return p.d == 64 ? run_select_blocks<float, 64>(p, st) : run_select_blocks<float, 128>(p, st);
}

}  // namespace lemo
