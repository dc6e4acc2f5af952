// The cheap score and the choice: means of the key blocks, and for every query block and group of heads the T blocks whose mean key
// agrees best with the group's queries.
//
//   means[n,g,:] = mean of K[j,g,:] over block n            s[m,g,n] = < sum of the block's queries over the heads of g, means[n,g,:] >
//
// The means read K once and are memory bound.  Scores are formed and compared in 64 bits: which of two nearly equal scores is the larger
// then does not depend on the order of a sum, and a list is the definition's but for ties closer than 2^-50 of the terms.  2 d flops in
// 64 bits for every query block and key block are far less than what the attention does with the lists.
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
__global__ __launch_bounds__(256) void block_means_kernel(const void* K, long long S, int H_kv, int d, long long k_ts, long long k_hs, int b, float* means) {
    const long long first = (long long)blockIdx.x * b;
    block_mean<T>(static_cast<const char*>(K), first, (int)min((long long)b, S - first), H_kv, d, k_ts, k_hs, means + (long long)blockIdx.x * H_kv * d);
}

// Single tokens: the block that the newest token of a sequence has filled, if it has.
template <typename T>
__global__ __launch_bounds__(256) void block_means_step_kernel(const void* K, const int* lengths, long long S_max, int H_kv, int d, long long k_ss,
                                                               long long k_ts, long long k_hs, int b, float* means, int nb) {
    const int s = blockIdx.x, S = (int)min((long long)lengths[s], S_max);
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



template <typename T, int D>
__global__ __launch_bounds__(256) void select_blocks_kernel(BlockSelectParams p) {
    constexpr int E = KeyPiece<T>::E, LANES = D / E;     // lanes of a row when the queries are added up
    constexpr int TEAMS = 256 / LANES, PER = D / 16;     // (scores: 16 lanes a block, PER values each)
    extern __shared__ __attribute__((aligned(16))) char smem[];
    double* const total = reinterpret_cast<double*>(smem);                      // [TEAMS][D], then [D]
    unsigned long long* const keys = reinterpret_cast<unsigned long long*>(smem + TEAMS * D * 8);
    const int g = blockIdx.x % p.H_kv, tid = threadIdx.x, lane = tid & 63;
    const long long qb = blockIdx.x / p.H_kv;
    const bool causal = (p.flags & LEMO_CAUSAL) != 0;
    const int S = p.lengths ? min(max(p.lengths[qb], 0), p.S_k) : p.S_k;
    const long long pos0 = p.lengths ? S - 1 : p.q_start + qb * p.bq;
    const int queries = (int)min((long long)p.bq, p.S_q - qb * p.bq), rows = queries * p.G;
    const long long last = min(pos0 + queries - 1, (long long)S - 1);
    const int nb = (S + p.b - 1) / p.b;
    const int count = S <= 0 ? 0 : causal ? (int)min((long long)nb, last / p.b + 1) : nb;  // candidates: blocks that begin before the last query ends
    const int own0 = causal ? (int)min(pos0 / p.b, (long long)nb) : nb;                     // causal: blocks from here on hold a query
    int* const out = p.blocks + (qb * p.H_kv + g) * p.T;
    if (count <= 0) {  // (uniform) no keys
        for (int e = tid; e < p.T; e += 256) out[e] = -1;
        return;
    }
    {
        const int team = tid / LANES, c = tid % LANES * E;
        double sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0;
        for (int r = team; r < rows; r += TEAMS) {
            const char* at = reinterpret_cast<const char*>(p.Q) + ((qb * p.bq + r / p.G) * p.q_ts + (long long)(g * p.G + r % p.G) * p.q_hs + c) * (16 / E);
            float x[E];
            KeyPiece<T>::get(*reinterpret_cast<const u32x4*>(at), x);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += (double)x[e];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) total[team * D + c + e] = sum[e];
        __syncthreads();
        double all = 0.0;
        if (tid < D)
            for (int t = 0; t < TEAMS; ++t) all += total[t * D + tid];
        __syncthreads();
        if (tid < D) total[tid] = all;
        __syncthreads();
    }
    {
        const int l16 = tid & 15;
        const float* const means = p.means + (p.lengths ? qb * p.means_ss : 0) + (long long)g * D;
        double q[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) q[i] = total[(i / 4 * 16 + l16) * 4 + i % 4];
        for (int n0 = 0; n0 < count; n0 += 16) {
            const int n = n0 + (tid >> 4);
            double s = 0.0;
            if (n < count && n < own0) {
                const float* at = means + (long long)n * p.H_kv * D;
#pragma unroll
                for (int i = 0; i < PER; i += 4) {
                    const f32x4 m = *reinterpret_cast<const f32x4*>(at + (i / 4 * 16 + l16) * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = fma(q[i + e], (double)m[e], s);
                }
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) s += __shfl_xor(s, x);
            if (l16 == 0 && n < count) keys[n] = n >= own0 ? ~0ull : score_key(s);
        }
    }
    __syncthreads();
    if (tid >= 64) return;
    // the highest threshold that T keys reach, bit by bit; done when exactly T reach it
    unsigned long long cut = 0;
    const int wanted = min(p.T, count);
    bool exact = count <= p.T;
    if (exact) cut = 1;
    for (int bit = 63; bit >= 0 && !exact; --bit) {
        const unsigned long long mark = cut | 1ull << bit;
        int reach = 0;
        for (int n = lane; n < count + lane; n += 64) reach += __popcll(__ballot(n < count && keys[n] >= mark));
        if (reach >= wanted) cut = mark;
        exact = reach == wanted;
    }
    int above = 0;
    if (!exact)
        for (int n = lane; n < count + lane; n += 64) above += __popcll(__ballot(n < count && keys[n] > cut));
    int ties = wanted - above, at = 0;  // of the keys that equal the threshold, the first ones
    for (int n = lane; n < count + lane; n += 64) {
        const unsigned long long k = n < count ? keys[n] : 0;
        const unsigned long long before = (1ull << lane) - 1;
        const unsigned long long equal = __ballot(!exact && k == cut);
        const bool taken = exact ? k >= cut : k > cut || (k == cut && (int)__popcll(equal & before) < ties);
        ties = max(0, ties - (int)__popcll(equal));
        const unsigned long long all = __ballot(taken);
        if (taken) out[at + __popcll(all & before)] = n;
        at += __popcll(all);
    }
    for (int e = at + lane; e < p.T; e += 64) out[e] = -1;
}

int launch_block_means(const void* K, long long S, int H_kv, int d, lemo_dtype_t dt, long long k_ts, long long k_hs, int b, float* means, hipStream_t st) {
    const int pieces = H_kv * (d / (dt == LEMO_BF16 ? 8 : 4));
    const dim3 grid((unsigned)((S + b - 1) / b), (unsigned)((pieces + 63) / 64));
    if (dt == LEMO_BF16) hipLaunchKernelGGL((block_means_kernel<bf16_t>), grid, dim3(256), 0, st, K, S, H_kv, d, k_ts, k_hs, b, means);
    else hipLaunchKernelGGL((block_means_kernel<float>), grid, dim3(256), 0, st, K, S, H_kv, d, k_ts, k_hs, b, means);
    return (int)hipGetLastError();
}

int launch_block_means_step(const void* K, const int* lengths, int B, long long S_max, int H_kv, int d, lemo_dtype_t dt, long long k_ss, long long k_ts,
                            long long k_hs, int b, float* means, int nb, hipStream_t st) {
    const int pieces = H_kv * (d / (dt == LEMO_BF16 ? 8 : 4));
    const dim3 grid((unsigned)B, (unsigned)((pieces + 63) / 64));
    if (dt == LEMO_BF16)
        hipLaunchKernelGGL((block_means_step_kernel<bf16_t>), grid, dim3(256), 0, st, K, lengths, S_max, H_kv, d, k_ss, k_ts, k_hs, b, means, nb);
    else hipLaunchKernelGGL((block_means_step_kernel<float>), grid, dim3(256), 0, st, K, lengths, S_max, H_kv, d, k_ss, k_ts, k_hs, b, means, nb);
    return (int)hipGetLastError();
}

template <typename T, int D> static int run_select_blocks(const BlockSelectParams& p, hipStream_t st) {
    constexpr int SUMS = 256 / (D / KeyPiece<T>::E) * D * 8;
    static const int err = raise_lds_limits({{reinterpret_cast<const void*>(&select_blocks_kernel<T, D>), SUMS + MAX_LISTED_BLOCKS * 8}});
    if (err) return err;
    hipLaunchKernelGGL((select_blocks_kernel<T, D>), dim3((unsigned)((long long)p.n_qb * p.H_kv)), dim3(256), SUMS + p.nb * 8, st, p);
    return (int)hipGetLastError();
}

int launch_select_blocks(const BlockSelectParams& p, lemo_dtype_t dt, hipStream_t st) {
    if (dt == LEMO_BF16) return p.d == 64 ? run_select_blocks<bf16_t, 64>(p, st) : run_select_blocks<bf16_t, 128>(p, st);
    return p.d == 64 ? run_select_blocks<float, 64>(p, st) : run_select_blocks<float, 128>(p, st);
}

}  // namespace lemo
