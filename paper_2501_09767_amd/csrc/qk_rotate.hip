// Norms of queries and keys, head by head, and their rotation by the tokens' positions, in one pass; the same for single tokens, which
// go to a cache; and the gradients.
//
//   u = w (x - [centred] mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps), over the d channels of a head
//   y_a = a cos - b sin, y_b = b cos + a sin   of every pair (a, b) of u's first `rot` channels, angle = position * inv_freq[pair]
//
// Gradients: t = the rotation by -position of dy;  dw = sum t xhat;  dx = rstd (w t - xhat mean(w t xhat) - [centred] mean(w t)).
//
// Memory bound: a lane holds two 16-byte pieces of a head, those whose channels are each other's partners in the rotation, so that
// a head is d / 2 channels' worth of lanes and nothing but the sums of the norm crosses lanes (by DPP).  cos and sin are formed once for a
// token and stand in LDS, in the order in which the lanes want them.  Angles are taken in revolutions in binary64: the product of a position with a
// frequency, and that with 1 / (2 pi), each in two parts, so that what is left after whole revolutions is off by 2^-53 whatever their number.  What binary32 leaves of that, as
// much as sincospif's own error, turns the result on to first order.  cos and sin are off by 1.4 * 2^-24 at any position up to 2^32 (one product with a rounded frequency in
// revolutions, then binary32: 1.9 near, 10.8 far; 32768 tokens, 32 + 8 heads, bf16: up to 2 % less time).
//
// Measured: 32768 tokens, 32 + 8 heads of 128, bf16, 671 MB: 139 us = 4.8 TB/s; the gradient of 8192, 403 MB: 83 us; a single token's step: 5.6 us, its launch.
#include <algorithm>
#include <type_traits>

#include "qk_rotate.hpp"
#include "row_pieces.hpp"

namespace lemo {

constexpr int RT_THREADS = 256, RT_MOST = 16;  // RT_MOST: tokens of a workgroup

// Sum over the LANES neighbouring lanes of a head, the same bits in all of them.
template <int LANES> __device__ __forceinline__ float head_sum(float v) {
    auto from = [&](auto ctrl) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    v += from(std::integral_constant<int, 0xB1>{});                             // lanes 1 0 3 2
    v += from(std::integral_constant<int, 0x4E>{});                             // lanes 2 3 0 1
    if constexpr (LANES >= 8) v += from(std::integral_constant<int, 0x141>{});  // mirrored within 8
    if constexpr (LANES >= 16) v += from(std::integral_constant<int, 0x140>{}); // within 16
    return v;
}

// cos and sin of the angles of one position, entry r of lane-wise order: r = e * rp + j is the e-th pair of lane j (of rp = rot / (2 E)
// lanes that rotate).  Halves: lane j holds pieces j and rp + j, pair e = channels (j E + e, rot / 2 + j E + e).  Adjacent pairs: the same
// pieces, whose pairs lie within a piece each.
template <int E> __device__ __forceinline__ float2 turn_of(const float* inv_freq, long long position, int r, int rp, bool pairs, float amplitude) {
    const int e = r / rp, j = r - e * rp;
    const int f = !pairs ? j * E + e : e < E / 2 ? j * (E / 2) + e : (rp + j) * (E / 2) + e - E / 2;
    const double x = (double)position, y = (double)inv_freq[f], angle = x * y, angle_left = fma(x, y, -angle);
    constexpr double PER = 0.15915494309189535, PER_LEFT = -9.839338337591243e-18;  // 1 / (2 pi)
    double part = fma(angle, PER, -rint(angle * PER)) + fma(angle, PER_LEFT, angle_left * PER);
    part -= rint(part);  // (more than half a revolution where their number passes 2^52)
    const double half = 2.0 * part;  // half turns
    const float h = (float)half, left = (float)((half - (double)h) * 3.141592653589793);
    float s, c;
    sincospif(h, &s, &c);
    const float by = s;
    s = fmaf(c, left, s);
    c = fmaf(-by, left, c);
    return make_float2(c * amplitude, s * amplitude);
}

// (x0, x1) of a lane turned by the angles at `tab`, forwards (SIGN 1) or back (-1)
template <int E, int SIGN> __device__ __forceinline__ void turn(float (&x0)[E], float (&x1)[E], const float2* tab, int rp, bool pairs) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float2 cs = tab[e * rp];
        const float sn = SIGN * cs.y;
        auto spin = [&](float& a, float& b) {
            const float p = a * cs.x - b * sn, q = b * cs.x + a * sn;
            a = p;
            b = q;
        };
        if (!pairs) spin(x0[e], x1[e]);
        else if (e < E / 2) spin(x0[2 * e], x0[2 * e + 1]);
        else spin(x1[2 * e - E], x1[2 * e - E + 1]);
    }
}

// channels of a lane's two pieces
template <int E> __device__ __forceinline__ void lane_pieces(int j, int rp, int& c0, int& c1) {
    c0 = (j < rp ? j : 2 * j) * E;
    c1 = (j < rp ? rp + j : 2 * j + 1) * E;
}

// x -> (x - mean) rstd
template <int E, int LANES> __device__ __forceinline__ float head_norm(float (&x0)[E], float (&x1)[E], int norm, float eps) {
    constexpr float INV = 1.f / (2 * E * LANES);
    if (norm == LEMO_NORM_NONE) return 1.f;
    if (norm == LEMO_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += x0[e] + x1[e];
        const float mean = head_sum<LANES>(s) * INV;
#pragma unroll
        for (int e = 0; e < E; ++e) { x0[e] -= mean; x1[e] -= mean; }
    }
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) q = fmaf(x0[e], x0[e], fmaf(x1[e], x1[e], q));
    const float rstd = 1.f / sqrtf(fmaf(head_sum<LANES>(q), INV, eps));
#pragma unroll
    for (int e = 0; e < E; ++e) { x0[e] *= rstd; x1[e] *= rstd; }
    return rstd;
}

template <typename T, int D>
__global__ __launch_bounds__(RT_THREADS) void qk_rotate_kernel(RotateParams p) {
    constexpr int E = RowPiece<T>::E, LANES = D / (2 * E);
    __shared__ float2 table[RT_MOST * D / 2];
    const int rp = p.rot / (2 * E), angles = rp * E;
    const long long block = p.first + blockIdx.x;
    const long long m0 = block / p.slots * p.tokens;
    const int slot = (int)(block % p.slots);
    const int heads = p.side[0].heads + p.side[1].heads + p.side[2].heads;
    const int h0 = (int)((long long)heads * slot / p.slots), h1 = (int)((long long)heads * (slot + 1) / p.slots);
    const int tokens = (int)min((long long)p.tokens, p.M - m0);
    auto length_of = [&](long long m) { return min(max((long long)p.lengths[m], 0ll), p.S_max); };
    auto position_of = [&](long long m) { return p.lengths ? length_of(m) - 1 : p.pos_start + (p.positions ? (long long)p.positions[m] : m); };
    for (int r = threadIdx.x; r < tokens * angles; r += RT_THREADS) {
        const int t = r / angles;
        table[r] = turn_of<E>(p.inv_freq, position_of(m0 + t), r - t * angles, rp, p.pairs, p.amplitude);
    }
    __syncthreads();
    const int j = threadIdx.x % LANES;
    int c0, c1;
    lane_pieces<E>(j, rp, c0, c1);
    const int items = tokens * (h1 - h0);
    for (int i = threadIdx.x / LANES; i < items; i += RT_THREADS / LANES) {  // (a head's lanes go together)
        const int t = i / (h1 - h0);
        int h = h0 + i - t * (h1 - h0);
        int which = 0;
        if (h >= p.side[0].heads) { h -= p.side[0].heads; which = 1; }
        if (which && h >= p.side[1].heads) { h -= p.side[1].heads; which = 2; }
        const RotateSide s = which == 0 ? p.side[0] : which == 1 ? p.side[1] : p.side[2];
        const long long m = m0 + t;
        const long long from = m * s.x_ts + h * s.x_hs;
        long long to = m * s.y_ts + h * s.y_hs;
        bool there = true;
        if (p.lengths) {
            const long long n = length_of(m);
            there = n > 0;
            if (which) {
                if (!there) continue;
                to = m * s.y_ss + (n - 1) * s.y_ts + h * s.y_hs;
            }
        }
        u32x4 a = row_load<T>(s.X, from + c0), b = row_load<T>(s.X, from + c1);
        if (!there) a = b = u32x4{0u, 0u, 0u, 0u};  // a sequence without a token
        if (which < 2 && there) {
            float x0[E], x1[E];
            RowPiece<T>::get(a, x0);
            RowPiece<T>::get(b, x1);
            head_norm<E, LANES>(x0, x1, p.norm, p.eps);
            if (s.w) {
                float w0[E], w1[E];
                RowPiece<T>::get(row_load<T>(s.w, (long long)h * s.w_hs + c0), w0);
                RowPiece<T>::get(row_load<T>(s.w, (long long)h * s.w_hs + c1), w1);
#pragma unroll
                for (int e = 0; e < E; ++e) { x0[e] *= w0[e]; x1[e] *= w1[e]; }
            }
            if (j < rp) turn<E, 1>(x0, x1, table + t * angles + j, rp, p.pairs);
            a = RowPiece<T>::put(x0);
            b = RowPiece<T>::put(x1);
        }
        row_store<T>(s.Y, to + c0, a);
        row_store<T>(s.Y, to + c1, b);
    }
}

// A workgroup's RT_THREADS / LANES places are `own` heads by `teams` tokens.  It walks the tokens in steps of the grid: the sums over the tokens
// stay with the lane that owns a channel.  One token at a time, and four waves a SIMD instead (8192 tokens, 32 / 32 heads of 128: four tokens
// ahead on two waves 95 us, one on three 100, on four 83; 32768 tokens, 32 / 8 heads 218 / 233 / 198: 5.1 TB/s).
constexpr int RT_TEAMS = 8;
template <typename T, int D>
__global__ __launch_bounds__(RT_THREADS, 4) void qk_rotate_grad_kernel(RotateGradParams p, int chunks, int own, int teams) {
    constexpr int E = RowPiece<T>::E, LANES = D / (2 * E), PLACES = RT_THREADS / LANES;
    constexpr float INV = 1.f / D;
    constexpr int MOST = PLACES < RT_TEAMS ? PLACES : RT_TEAMS;
    __shared__ float2 table[MOST * D / 2];
    __shared__ float sums[PLACES][D];
    const int rp = p.rot / (2 * E), angles = rp * E;
    const int chunk = blockIdx.x % chunks, walker = blockIdx.x / chunks, walkers = gridDim.x / chunks;
    const int heads = p.side[0].heads + p.side[1].heads;
    const int place = threadIdx.x / LANES, j = threadIdx.x % LANES;
    const int team = place / own, head = chunk * own + place - team * own;
    const bool live = head < heads && team < teams;
    const bool keys = head >= p.side[0].heads;
    const int h = keys ? head - p.side[0].heads : head;
    const RotateSide s = keys ? p.side[1] : p.side[0];
    const char* const dY = static_cast<const char*>(keys ? p.dY[1] : p.dY[0]);
    const long long dy_ts = keys ? p.dy_ts[1] : p.dy_ts[0], dy_hs = keys ? p.dy_hs[1] : p.dy_hs[0];
    int c0, c1;
    lane_pieces<E>(j, rp, c0, c1);
    float w0[E], w1[E], dw0[E], dw1[E];
#pragma unroll
    for (int e = 0; e < E; ++e) { w0[e] = w1[e] = 1.f; dw0[e] = dw1[e] = 0.f; }
    if (live && s.w && p.norm != LEMO_NORM_NONE) {
        RowPiece<T>::get(row_load<T>(s.w, (long long)h * s.w_hs + c0), w0);
        RowPiece<T>::get(row_load<T>(s.w, (long long)h * s.w_hs + c1), w1);
    }
    for (long long m0 = (long long)walker * teams; m0 < p.M; m0 += (long long)walkers * teams) {
        const int tokens = (int)min((long long)teams, p.M - m0);
        const bool there = live && team < tokens;
        const long long m = m0 + team;
        u32x4 x[2], g[2];
        if (there) {
            g[0] = row_load<T>(dY, m * dy_ts + h * dy_hs + c0);
            g[1] = row_load<T>(dY, m * dy_ts + h * dy_hs + c1);
            if (p.norm != LEMO_NORM_NONE) {
                x[0] = row_load<T>(s.X, m * s.x_ts + h * s.x_hs + c0);
                x[1] = row_load<T>(s.X, m * s.x_ts + h * s.x_hs + c1);
            }
        }
        __syncthreads();  // the table of the tokens before has been read
        for (int r = threadIdx.x; r < tokens * angles; r += RT_THREADS) {
            const int t = r / angles;
            table[r] = turn_of<E>(p.inv_freq, p.pos_start + (p.positions ? (long long)p.positions[m0 + t] : m0 + t), r - t * angles, rp, p.pairs, p.amplitude);
        }
        __syncthreads();
        if (!there) continue;
        float t0[E], t1[E];
        RowPiece<T>::get(g[0], t0);
        RowPiece<T>::get(g[1], t1);
        if (j < rp) turn<E, -1>(t0, t1, table + team * angles + j, rp, p.pairs);
        if (p.norm != LEMO_NORM_NONE) {
            float x0[E], x1[E];
            RowPiece<T>::get(x[0], x0);
            RowPiece<T>::get(x[1], x1);
            const float rstd = head_norm<E, LANES>(x0, x1, p.norm, p.eps);
            float both = 0.f, alone = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                dw0[e] = fmaf(t0[e], x0[e], dw0[e]);
                dw1[e] = fmaf(t1[e], x1[e], dw1[e]);
                t0[e] *= w0[e];
                t1[e] *= w1[e];
                both = fmaf(t0[e], x0[e], fmaf(t1[e], x1[e], both));
                alone += t0[e] + t1[e];
            }
            both = head_sum<LANES>(both) * INV;
            alone = p.norm == LEMO_NORM_LAYER ? head_sum<LANES>(alone) * INV : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                t0[e] = (t0[e] - fmaf(x0[e], both, alone)) * rstd;
                t1[e] = (t1[e] - fmaf(x1[e], both, alone)) * rstd;
            }
        }
        row_store<T>(s.Y, m * s.y_ts + h * s.y_hs + c0, RowPiece<T>::put(t0));
        row_store<T>(s.Y, m * s.y_ts + h * s.y_hs + c1, RowPiece<T>::put(t1));
    }
    if (!p.sums) return;
    // a channel's sums of the workgroup's places, in their order: of a head's teams, or of all queries and of all keys
#pragma unroll
    for (int e = 0; e < E; ++e) {
        sums[place][c0 + e] = live ? dw0[e] : 0.f;
        sums[place][c1 + e] = live ? dw1[e] : 0.f;
    }
    __syncthreads();
    const int here = min(heads - chunk * own, own);  // heads of this workgroup
    if (p.per_head) {
        for (int c = threadIdx.x; c < here * D; c += RT_THREADS) {
            float v = 0.f;
            for (int t = 0; t < teams; ++t) v += sums[t * own + c / D][c % D];
            p.parts[((long long)walker * heads + chunk * own) * D + c] = v;
        }
        return;
    }
    for (int c = threadIdx.x; c < 2 * D; c += RT_THREADS) {
        const int queries = min(max(p.side[0].heads - chunk * own, 0), here);
        const int first = c < D ? 0 : queries, last = c < D ? queries : here;
        float v = 0.f;
        for (int t = 0; t < teams; ++t)
            for (int i = first; i < last; ++i) v += sums[t * own + i][c % D];
        p.parts[(long long)blockIdx.x * 2 * D + c] = v;
    }
}

// out[c] = sum of parts[r][c] over r, in a fixed order: 32 threads a column, each every 32nd row.  Columns [0, split) go to `a`, the others to `b`.
__global__ __launch_bounds__(RT_THREADS) void rotate_sums_kernel(const float* parts, int rows, int cols, int split, float* a, float* b) {
    __shared__ float lds[32][8];
    const int c = blockIdx.x * 8 + threadIdx.x % 8, r0 = threadIdx.x / 8;
    float v = 0.f;
#pragma unroll 8
    for (int r = r0; r < rows; r += 32) v += parts[(long long)r * cols + c];  // (cols: a multiple of 8)
    lds[r0][threadIdx.x % 8] = v;
    __syncthreads();
    if (r0) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) v += lds[i][threadIdx.x];
    float* const to = c < split ? a : b;
    if (to) to[c < split ? c : c - split] = v;
}

template <typename T, int D> static int launch_rotate(RotateParams p, hipStream_t st) {
    constexpr int HEADS = RT_THREADS / (D / (2 * RowPiece<T>::E));
    const int heads = p.side[0].heads + p.side[1].heads + p.side[2].heads;
    // A workgroup has the tokens that give its threads two passes at least, or one; few tokens are spread over as many workgroups as have a pass
    // each.  8192 tokens, 32 / 32 heads of 128: 4 tokens 57 us, 2 55, 1 54 (5.0 TB/s);  4 / 4 heads of 64: 4 tokens 7.9, 2 9.3, 1 13.6.
    const long long lanes = (long long)heads * (D / (2 * RowPiece<T>::E));
    const bool many = p.M * lanes >= 1 << 18;
    p.tokens = many ? (int)std::min<long long>(RT_MOST, std::max<long long>(1, 2 * RT_THREADS / lanes)) : 1;
    p.slots = many ? 1 : (heads + HEADS - 1) / HEADS;
    const long long blocks = (p.M + p.tokens - 1) / p.tokens * p.slots;
    return launch_in_turns(blocks, RT_THREADS, [&](long long first, unsigned count) {
        p.first = first;
        hipLaunchKernelGGL((qk_rotate_kernel<T, D>), dim3(count), dim3(RT_THREADS), 0, st, p);
    });
}

int launch_qk_rotate(RotateParams p, lemo_dtype_t dt, hipStream_t st) {
    if (dt == LEMO_BF16) return p.d == 64 ? launch_rotate<bf16_t, 64>(p, st) : launch_rotate<bf16_t, 128>(p, st);
    return p.d == 64 ? launch_rotate<float, 64>(p, st) : launch_rotate<float, 128>(p, st);
}

// How the gradient's workgroups share the work: `chunks` of `own` heads each, `teams` of tokens in one, `walkers` over the tokens.  The fewest chunks that leave
// a tenth of the places empty at most, or fewest empty ones (32768 tokens, 32 / 8 heads of 128: 2 chunks of 32 and 8 heads 266 us, 4 of 10 by 3 tokens 218).
struct RotateGrid { int chunks, own, teams, walkers; };
static RotateGrid rotate_grid(int64_t M, int heads, int d, lemo_dtype_t dt) {
    const int places = RT_THREADS / (d / (dt == LEMO_BF16 ? 16 : 8));
    RotateGrid g{};
    double most = 0.;
    for (int c = 1; c <= heads && most < 0.9; ++c) {
        const int own = (heads + c - 1) / c, chunks = (heads + own - 1) / own;
        if (own > places) continue;
        const int teams = std::min(RT_TEAMS, places / own);
        const double used = (double)heads * teams / ((double)chunks * places);
        if (used > most) {
            most = used;
            g = {chunks, own, teams, 0};
        }
    }
    const int64_t steps = (M + g.teams - 1) / g.teams;
    g.walkers = (int)std::max<int64_t>(1, std::min<int64_t>(steps, std::max(64, 1024 / g.chunks)));
    return g;
}

size_t qk_rotate_grad_parts(int64_t M, int heads, int d, lemo_dtype_t dt, bool per_head) {
    const RotateGrid g = rotate_grid(M, heads, d, dt);
    return per_head ? (size_t)g.walkers * heads * d : (size_t)g.walkers * g.chunks * 2 * d;
}

template <typename T, int D> static int launch_rotate_grad(const RotateGradParams& p, RotateGrid g, hipStream_t st) {
    hipLaunchKernelGGL((qk_rotate_grad_kernel<T, D>), dim3((unsigned)(g.chunks * g.walkers)), dim3(RT_THREADS), 0, st, p, g.chunks, g.own, g.teams);
    return (int)hipGetLastError();
}

int launch_qk_rotate_grad(RotateGradParams p, float* dw_q, float* dw_k, lemo_dtype_t dt, hipStream_t st) {
    const int heads = p.side[0].heads + p.side[1].heads;
    const RotateGrid g = rotate_grid(p.M, heads, p.d, dt);
    p.sums = dw_q || dw_k;
    int rc;
    if (dt == LEMO_BF16) rc = p.d == 64 ? launch_rotate_grad<bf16_t, 64>(p, g, st) : launch_rotate_grad<bf16_t, 128>(p, g, st);
    else rc = p.d == 64 ? launch_rotate_grad<float, 64>(p, g, st) : launch_rotate_grad<float, 128>(p, g, st);
    if (rc || !p.sums) return rc;
    const int rows = p.per_head ? g.walkers : g.walkers * g.chunks;
    const int cols = p.per_head ? heads * p.d : 2 * p.d, split = p.per_head ? p.side[0].heads * p.d : p.d;
    hipLaunchKernelGGL(rotate_sums_kernel, dim3((unsigned)(cols / 8)), dim3(RT_THREADS), 0, st, p.parts, rows, cols, split, dw_q, dw_k);
    return (int)hipGetLastError();
}

}  // namespace lemo
