// What stands between two blocks of a layer, on the kept rows in place: the norm of a block's result, its gate, the scaled
// add into the residual rows, and the norm that the next block reads; and the gradients of that.
//
//   u = post(Y[m])      r = a R[idx[m]] + beta g_m u      R[idx[m]] = r      N[m] = next(R[idx[m]])
//
//   post, next: none, x rstd w + b (root mean square), (x - mean) rstd w + b (centred); rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//
// Gradients, with xhat = (R - mean) rstd and t = dN w:
//   dr = dR + rstd (t - xhat mean(t xhat) - [centred] mean(t))      dR = a dr      dg = beta u dr      du = beta g dr
//   dY = the same formula with (du, yhat, w_post)      dw_next = sum_m dN xhat, db_next = sum_m dN, dw_post, db_post likewise
//
// Memory bound: a row is read once into registers, and all that is known about it follows from there.  Forward: a wave, or a
// workgroup for long rows and few of them, owns a row; the mean and the squares about it are two sums over registers, so that
// nothing cancels.  Gradients: a workgroup owns a row at a time and walks the rows in steps of the grid, because the sums over
// the rows stay with the thread that owns a column, in registers up to 8192 columns; what the workgroups hold at the end goes through the
// workspace and is added in their order by a second kernel (no atomics: the same bits on every run).
#include <algorithm>

#include "lemo_common.hpp"
#include "norm_residual.hpp"

namespace lemo {

template <typename T> struct Piece;  // 16 bytes of a row as binary32 values
template <> struct Piece<bf16_t> {
    static constexpr int E = 8;
    __device__ static void get(const u32x4& v, float (&x)[E]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo_to_f32(v[i]); x[2 * i + 1] = bf16hi_to_f32(v[i]); }
    }
    __device__ static u32x4 put(const float (&x)[E]) {
        return u32x4{pack_bf16x2_hw(x[0], x[1]), pack_bf16x2_hw(x[2], x[3]), pack_bf16x2_hw(x[4], x[5]), pack_bf16x2_hw(x[6], x[7])};
    }
};
template <> struct Piece<float> {
    static constexpr int E = 4;
    __device__ static void get(const u32x4& v, float (&x)[E]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
    }
    __device__ static u32x4 put(const float (&x)[E]) {
        return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};

template <typename T> __device__ __forceinline__ u32x4 load_piece(const void* base, long long element) {
    return *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(base) + element * (long long)(16 / Piece<T>::E));
}
template <typename T> __device__ __forceinline__ void store_piece(void* base, long long element, const u32x4& v) {
    *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(base) + element * (long long)(16 / Piece<T>::E)) = v;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s);
    return v;
}

// Sums over the threads of a row.  One wave needs no LDS; more leave a partial sum each and add all of them in wave order.  A call
// uses the half of `lds` that the call before it did not, so one barrier a call is enough.
template <int THREADS, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float* lds, int& turn) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
    if constexpr (THREADS > 64) {
        constexpr int WAVES = THREADS / 64;
        float* const at = lds + turn * 2 * WAVES;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) at[n * WAVES + (threadIdx.x >> 6)] = v[n];
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = at[n * WAVES];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v[n] += at[n * WAVES + w];
        }
    }
}

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)); }

// TPR threads own a row of at most TPR * NP pieces: thread t holds pieces t, t + TPR, ...
template <typename T, int TPR, int NP>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_residual_kernel(NormParams p) {
    constexpr int E = Piece<T>::E, TEAMS = TPR < 256 ? 256 / TPR : 1;
    __shared__ float lds[4 * (TPR / 64)];
    int turn = 0;
    const long long m = (p.first + blockIdx.x) * TEAMS + threadIdx.x / TPR;
    if (m >= p.M) return;  // (a team is a wave, or the whole workgroup)
    const int t = threadIdx.x % TPR;
    const long long row = p.idx ? (long long)p.idx[m] : m;
    const bool there = row >= 0 && row < p.S;
    const float inv_C = 1.f / (float)p.C;
    float x[NP][E];
    float4 stats = make_float4(0.f, 0.f, 0.f, 0.f);

    // mean and 1 / deviation of x, by the mode of a norm
    auto measure = [&](int mode, float& mean, float& rstd) {
        mean = 0.f;
        float s[1] = {0.f};
        if (mode == LEMO_NORM_LAYER) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) s[0] += x[i][e];  // (pieces past the row are zeros)
            row_sum<TPR>(s, lds, turn);
            mean = s[0] * inv_C;
        }
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if ((t + i * TPR) * E >= p.C) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float c = x[i][e] - mean;
                s[0] = fmaf(c, c, s[0]);
            }
        }
        row_sum<TPR>(s, lds, turn);
        rstd = 1.f / sqrtf(fmaf(s[0], inv_C, p.eps));
    };
    // x = (x - mean) rstd w + b
    auto apply = [&](float mean, float rstd, const void* w, const void* b) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * TPR) * E;
            if (c >= p.C) continue;
            float ww[E], bb[E];
            if (w) Piece<T>::get(load_piece<T>(w, c), ww);
            if (b) Piece<T>::get(load_piece<T>(b, c), bb);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[i][e] = (x[i][e] - mean) * rstd;
                if (w) x[i][e] *= ww[e];
                if (b) x[i][e] += bb[e];
            }
        }
    };

    if (there) {
        // every load of the row is under way before the first sum
        u32x4 y[NP], g[NP], r[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * TPR) * E;
            y[i] = g[i] = r[i] = u32x4{0u, 0u, 0u, 0u};
            if (c >= p.C) continue;
            if (p.Y) y[i] = load_piece<T>(p.Y, m * p.ldy + c);
            r[i] = load_piece<T>(p.R, row * p.ldr + c);
            if (p.gate) g[i] = load_piece<T>(p.gate, m * p.ldg + c);
        }
        if (p.Y) {
#pragma unroll
            for (int i = 0; i < NP; ++i) Piece<T>::get(y[i], x[i]);
            if (p.post != LEMO_NORM_NONE) {
                measure(p.post, stats.x, stats.y);
                apply(stats.x, stats.y, p.w_post, p.b_post);
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = (t + i * TPR) * E;
                float old[E];
                Piece<T>::get(r[i], old);
                if (p.gate) {
                    float gg[E];
                    Piece<T>::get(g[i], gg);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[i][e] *= p.flags & LEMO_GATE_SIGMOID ? sigmoid(gg[e]) : gg[e];
                }
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][e] = fmaf(p.beta, x[i][e], p.a * old[e]);
                r[i] = Piece<T>::put(x[i]);
                if (c < p.C) store_piece<T>(p.R, row * p.ldr + c, r[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {  // the next norm is that of the stored row: the gradient will see no other
            Piece<T>::get(r[i], x[i]);
            if ((t + i * TPR) * E >= p.C)
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][e] = 0.f;
        }
        if (p.next != LEMO_NORM_NONE) {
            measure(p.next, stats.z, stats.w);
            apply(stats.z, stats.w, p.w_next, p.b_next);
        }
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] = 0.f;
    }
    if (p.next != LEMO_NORM_NONE) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * TPR) * E;
            if (c < p.C) store_piece<T>(p.N, m * p.ldn + c, Piece<T>::put(x[i]));
        }
    }
    if (p.stats && t == 0) *reinterpret_cast<float4*>(p.stats + m * 4) = stats;
}

// Column sums of the gradients, as planes of [C]: which of them a call needs (its bit), and in which plane of a workgroup's part
// they stand follows from the order.
enum { SUM_W_NEXT = 1, SUM_B_NEXT = 2, SUM_W_POST = 4, SUM_B_POST = 8, SUM_GATE = 16 };

// POST: there is a norm of the block's result; SHARED: all rows share the gate.  What a call does not have takes no registers.
template <typename T, int THREADS, int NP, bool POST, bool SHARED>
__global__ __launch_bounds__(THREADS) void norm_residual_grad_kernel(NormGradParams p) {
    constexpr int E = Piece<T>::E;
    __shared__ float lds[4 * (THREADS / 64)];
    int turn = 0;
    const int t = threadIdx.x;
    const float inv_C = 1.f / (float)p.C;
    const bool next = p.next != LEMO_NORM_NONE;
    constexpr bool post = POST;
    float w_next_sum[NP][E], b_next_sum[NP][E], w_post_sum[NP][E], b_post_sum[NP][E], gate_sum[NP][E];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) w_next_sum[i][e] = b_next_sum[i][e] = w_post_sum[i][e] = b_post_sum[i][e] = gate_sum[i][e] = 0.f;

    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const long long row = p.idx ? (long long)p.idx[m] : m;
        const bool there = row >= 0 && row < p.S;  // uniform: the workgroup owns the row
        if (!there) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = (t + i * THREADS) * E;
                if (c >= p.C) continue;
                if (p.dY) store_piece<T>(p.dY, m * p.lddy + c, u32x4{0u, 0u, 0u, 0u});
                if (p.dgate) store_piece<T>(p.dgate, m * p.lddg + c, u32x4{0u, 0u, 0u, 0u});
            }
            continue;
        }
        u32x4 vn[NP], vr[NP], vx[NP], vy[NP], vg[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * THREADS) * E;
            vn[i] = vr[i] = vx[i] = vy[i] = vg[i] = u32x4{0u, 0u, 0u, 0u};
            if (c >= p.C) continue;
            vr[i] = load_piece<T>(p.dR, row * p.lddr + c);
            if (next) {
                vn[i] = load_piece<T>(p.dN, m * p.lddn + c);
                vx[i] = load_piece<T>(p.R, row * p.ldr + c);
            }
            if (p.Y) vy[i] = load_piece<T>(p.Y, m * p.ldy + c);
            if (p.gate) vg[i] = load_piece<T>(p.gate, m * p.ldg + c);
        }
        const float4 stats = next || post ? *reinterpret_cast<const float4*>(p.stats + m * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
        float dr[NP][E];
#pragma unroll
        for (int i = 0; i < NP; ++i) Piece<T>::get(vr[i], dr[i]);
        if (next) {
            float s[2] = {0.f, 0.f}, tt[NP][E], xh[NP][E];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = (t + i * THREADS) * E;
                float dn[E], ww[E];
                Piece<T>::get(vn[i], dn);
                Piece<T>::get(vx[i], xh[i]);
                if (p.w_next && c < p.C) Piece<T>::get(load_piece<T>(p.w_next, c), ww);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    xh[i][e] = c < p.C ? (xh[i][e] - stats.z) * stats.w : 0.f;
                    tt[i][e] = p.w_next && c < p.C ? dn[e] * ww[e] : dn[e];
                    s[0] = fmaf(tt[i][e], xh[i][e], s[0]);
                    s[1] += tt[i][e];
                    w_next_sum[i][e] = fmaf(dn[e], xh[i][e], w_next_sum[i][e]);
                    b_next_sum[i][e] += dn[e];
                }
            }
            row_sum<THREADS>(s, lds, turn);
            const float c1 = s[0] * inv_C, c0 = p.next == LEMO_NORM_LAYER ? s[1] * inv_C : 0.f;
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e)  // (past the row the means would leave something that the sums below must not see)
                    if ((t + i * THREADS) * E < p.C) dr[i][e] = fmaf(stats.w, tt[i][e] - xh[i][e] * c1 - c0, dr[i][e]);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * THREADS) * E;
            float out[E];
#pragma unroll
            for (int e = 0; e < E; ++e) out[e] = p.a * dr[i][e];
            if (c < p.C) store_piece<T>(p.dR, row * p.lddr + c, Piece<T>::put(out));
        }
        if (!p.Y) continue;
        float s[2] = {0.f, 0.f}, du[NP][E], yh[NP][E];  // du: du, then du w
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * THREADS) * E;
            float ww[E], bb[E], gg[E], u[E], slope[E];
            Piece<T>::get(vy[i], yh[i]);
            if (post && c < p.C) {
                if (p.w_post) Piece<T>::get(load_piece<T>(p.w_post, c), ww);
                if (p.b_post) Piece<T>::get(load_piece<T>(p.b_post, c), bb);
            }
            if (p.gate) Piece<T>::get(vg[i], gg);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (post) yh[i][e] = c < p.C ? (yh[i][e] - stats.x) * stats.y : 0.f;
                const float wv = post && p.w_post && c < p.C ? ww[e] : 1.f;
                u[e] = yh[i][e] * wv;
                if (post && p.b_post && c < p.C) u[e] += bb[e];
                slope[e] = 1.f;
                if (p.gate && (p.flags & LEMO_GATE_SIGMOID)) {
                    gg[e] = sigmoid(gg[e]);
                    slope[e] = gg[e] * (1.f - gg[e]);
                }
                const float bdr = p.beta * dr[i][e], dg = bdr * u[e] * slope[e];
                du[i][e] = p.gate ? bdr * gg[e] : bdr;
                if constexpr (SHARED) gate_sum[i][e] += dg;
                u[e] = dg;
                if constexpr (POST) {
                    w_post_sum[i][e] = fmaf(du[i][e], yh[i][e], w_post_sum[i][e]);
                    b_post_sum[i][e] += du[i][e];
                }
                du[i][e] *= wv;
                s[0] = fmaf(du[i][e], yh[i][e], s[0]);
                s[1] += du[i][e];
            }
            if (p.dgate && c < p.C) store_piece<T>(p.dgate, m * p.lddg + c, Piece<T>::put(u));
        }
        if (post) {
            row_sum<THREADS>(s, lds, turn);
            const float c1 = s[0] * inv_C, c0 = p.post == LEMO_NORM_LAYER ? s[1] * inv_C : 0.f;
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) du[i][e] = stats.y * (du[i][e] - yh[i][e] * c1 - c0);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * THREADS) * E;
            if (p.dY && c < p.C) store_piece<T>(p.dY, m * p.lddy + c, Piece<T>::put(du[i]));
        }
    }

    float* part = p.parts + (long long)blockIdx.x * p.planes * p.C;
    auto leave = [&](int bit, const float (&v)[NP][E]) {
        if (!(p.sums & bit)) return;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (t + i * THREADS) * E;
            if (c >= p.C) continue;
#pragma unroll
            for (int e = 0; e < E; e += 4) *reinterpret_cast<f32x4*>(part + c + e) = f32x4{v[i][e], v[i][e + 1], v[i][e + 2], v[i][e + 3]};
        }
        part += p.C;
    };
    leave(SUM_W_NEXT, w_next_sum);
    leave(SUM_B_NEXT, b_next_sum);
    leave(SUM_W_POST, w_post_sum);
    leave(SUM_B_POST, b_post_sum);
    leave(SUM_GATE, gate_sum);
}

// Adds the workgroups' parts: 64 columns a workgroup, its 16 waves take every sixteenth part, in order; no parts give zeros.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float* __restrict__ parts, int count, int planes, int C, NormSums out) {
    __shared__ float share[16][64];
    const int lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane, wave = threadIdx.x >> 6, plane = blockIdx.y;
    float s = 0.f;
    if (c < C)
#pragma unroll 8
        for (int n = wave; n < count; n += 16) s += parts[((long long)n * planes + plane) * C + c];
    share[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= C) return;
    s = share[0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) s += share[w][lane];
    out.to[plane][c] = s;
}

template <typename T, int TPR, int NP> static int run_norm(NormParams p, hipStream_t st) {
    constexpr int TEAMS = TPR < 256 ? 256 / TPR : 1, THREADS = TPR < 256 ? 256 : TPR;
    return launch_in_turns((p.M + TEAMS - 1) / TEAMS, THREADS, [&](long long first, unsigned count) {
        p.first = first;
        hipLaunchKernelGGL((norm_residual_kernel<T, TPR, NP>), dim3(count), dim3(THREADS), 0, st, p);
    });
}

// Short rows: a wave each, which needs no LDS and no barrier; from 256 pieces on (bf16: 2048 columns) a workgroup, whose threads have more
// loads under way and less to add up.  bf16 with gate and both norms, us, wave / workgroup: 8192 rows of 1024 18.2 / 21.9, of 2048
// 32.0 / 28.4, of 4096 73.3 / 53.7 (5.0 TB/s, as fast as a copy); 8 rows of 1024 5.8 / 5.8, of 2048 6.8 / 5.8, of 4096 10.6 / 5.6.
int launch_norm_residual(const NormParams& p, lemo_dtype_t dt, hipStream_t st) {
    const int pieces = p.C / (dt == LEMO_BF16 ? 8 : 4);
    auto go = [&](auto tag) {
        using T = decltype(tag);
        if (pieces <= 64) return run_norm<T, 64, 1>(p, st);
        if (pieces <= 128) return run_norm<T, 64, 2>(p, st);
        if (pieces <= 256) return run_norm<T, 256, 1>(p, st);
        if (pieces <= 512) return run_norm<T, 256, 2>(p, st);
        if (pieces <= 1024) return run_norm<T, 256, 4>(p, st);
        if constexpr (Piece<T>::E == 4) {  // (bf16 has no more pieces)
            if (pieces > 2048) return run_norm<T, 1024, 4>(p, st);
        }
        return run_norm<T, 512, 4>(p, st);
    };
    return dt == LEMO_BF16 ? go(bf16_t{}) : go(float{});
}

// Threads that own a row, 16 columns each, and workgroups: two waves a SIMD, but two rows a workgroup at least, whose sums are one more
// row to write and to read.  bf16 with gate and both norms, us for 256 / 512 / 1024 / 2048 workgroups: 8192 rows of 1024 (a wave each) 117 /
// 70 / 54 / 47; of 2048 134 / 82 / 64 / -; of 4096 (256 threads) 175 / 130 / 136 / -.  One workgroup for 4, 2 or 1 rows: 512 rows of 4096
// 25 / 20 / 23.  8192 rows of 4096 without a norm of the block's result (537 MB): 125 us, 4.3 TB/s; what is missing to a copy's rate is
// the barrier between a row's loads and its stores, with two waves a SIMD to cover it: registers hold the columns' sums.  Beyond 8192
// columns they do not: 1024 threads have 128 registers each, and 68 to 280 of what a thread holds goes through scratch in the loop over the
// rows.  bf16 with gate and both norms, as many bytes each: 8192 rows of 4096 134 us, 4096 of 8192 153, 2048 of 16384 442.
static int norm_grad_threads(int C) { return C <= 1024 ? 64 : C <= 2048 ? 128 : C <= 4096 ? 256 : C <= 8192 ? 512 : 1024; }
int norm_grad_parts(int64_t M, int C) {
    const int most = std::max(512, 512 * 256 / norm_grad_threads(C));
    return (int)(M >= 2 * most ? most : M >= 256 ? M / 2 : M < 128 ? M : 128);
}

template <typename T, int THREADS, int NP> static int run_norm_grad(const NormGradParams& p, int parts, hipStream_t st) {
    const bool post = p.post != LEMO_NORM_NONE, shared = (p.sums & SUM_GATE) != 0;
    if (post && shared) hipLaunchKernelGGL((norm_residual_grad_kernel<T, THREADS, NP, true, true>), dim3((unsigned)parts), dim3(THREADS), 0, st, p);
    else if (post) hipLaunchKernelGGL((norm_residual_grad_kernel<T, THREADS, NP, true, false>), dim3((unsigned)parts), dim3(THREADS), 0, st, p);
    else if (shared) hipLaunchKernelGGL((norm_residual_grad_kernel<T, THREADS, NP, false, true>), dim3((unsigned)parts), dim3(THREADS), 0, st, p);
    else hipLaunchKernelGGL((norm_residual_grad_kernel<T, THREADS, NP, false, false>), dim3((unsigned)parts), dim3(THREADS), 0, st, p);
    return (int)hipGetLastError();
}

int launch_norm_residual_grad(NormGradParams p, float* dw_next, float* db_next, float* dw_post, float* db_post, float* dgate_sum, void* workspace,
                              lemo_dtype_t dt, hipStream_t st) {
    const int threads = norm_grad_threads(p.C), parts = norm_grad_parts(p.M, p.C);
    NormSums out{};
    p.sums = p.planes = 0;
    p.parts = static_cast<float*>(workspace);
    float* const to[5] = {dw_next, db_next, dw_post, db_post, dgate_sum};  // in the order of the bits
    for (int i = 0; i < 5; ++i)
        if (to[i]) {
            p.sums |= 1 << i;
            out.to[p.planes++] = to[i];
        }
    auto go = [&](auto tag) {
        using T = decltype(tag);
        constexpr int NP = 16 / Piece<T>::E;  // 16 columns a thread, whose sums it holds
        if (threads == 64) return run_norm_grad<T, 64, NP>(p, parts, st);
        if (threads == 128) return run_norm_grad<T, 128, NP>(p, parts, st);
        if (threads == 256) return run_norm_grad<T, 256, NP>(p, parts, st);
        if (threads == 512) return run_norm_grad<T, 512, NP>(p, parts, st);
        return run_norm_grad<T, 1024, NP>(p, parts, st);
    };
    if (p.M > 0) {
        const int rc = dt == LEMO_BF16 ? go(bf16_t{}) : go(float{});
        if (rc) return rc;
    }
    if (p.planes == 0) return 0;
    hipLaunchKernelGGL(norm_sums_kernel, dim3((unsigned)((p.C + 63) / 64), (unsigned)p.planes), dim3(1024), 0, st, p.parts, parts, p.planes, p.C, out);
    return (int)hipGetLastError();
}

}  // namespace lemo
