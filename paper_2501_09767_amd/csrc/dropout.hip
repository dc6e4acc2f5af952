// Dropout of a block's result and its add into the residual rows, and the gradient of that; the mask is formed where it is used and
// never stored.
//
//   R[idx[m], c] += keep(idx[m], c) ? scale Y[m, c] : 0          dY[m, c] = keep(idx[m], c) ? scale dR[idx[m], c] : 0
//
// keep comes from Philox 4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011), whose
// block for key = seed and counter = (c / 8, token, stream) is 128 bits for eight columns: a thread's share, so that nothing of the generator crosses
// threads.  16 bits an element are steps of 2^-16 in the probability, finer than a rate is chosen, and the scale is that of the probability
// as it is.  A block for every four elements takes as long from memory (9856 rows of 4096, bf16: 49.7 us, and 49.9 with one for eight) with twice the
// vector work.
//
// Memory bound: two reads and a write of 81 MB there, 49 us = 4.9 TB/s, a large copy's rate 5.2; 2999 rows of 768 in binary32, gradient: 5.0 us.
#include "dropout.hpp"
#include "row_pieces.hpp"

namespace lemo {

constexpr int DO_THREADS = 256;

struct Philox { unsigned x[4]; };
__device__ __forceinline__ Philox philox(unsigned c0, unsigned c1, unsigned long long stream, unsigned long long seed) {
    unsigned x0 = c0, x1 = c1, x2 = (unsigned)stream, x3 = (unsigned)(stream >> 32), k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long p = (unsigned long long)x0 * 0xD2511F53u, q = (unsigned long long)x2 * 0xCD9E8D57u;
        x0 = (unsigned)(q >> 32) ^ x1 ^ k0;
        x1 = (unsigned)q;
        x2 = (unsigned)(p >> 32) ^ x3 ^ k1;
        x3 = (unsigned)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{x0, x1, x2, x3}};
}

template <typename T, bool GRAD>
__global__ __launch_bounds__(DO_THREADS) void dropout_kernel(DropoutParams p) {
    constexpr int E = RowPiece<T>::E, NP = 8 / E;  // 16-byte pieces of eight columns
    const int per_row = DO_THREADS / p.rows;
    const long long m = (p.first + blockIdx.x) * p.rows + threadIdx.x / per_row;
    if (m >= p.M) return;
    const long long row = p.idx ? (long long)p.idx[m] : m;
    const bool there = row >= 0 && row < p.S;
    if (!GRAD && !there) return;
    const unsigned long long seed = p.rng[0], stream = p.rng[1] + p.site;
    const long long from = (GRAD ? row : m) * p.ldx, to = (GRAD ? m : row) * p.ldy;
    const unsigned C = (unsigned)p.C;
    for (unsigned c = threadIdx.x % per_row * 8; c < C; c += per_row * 8) {  // (rows of up to 2^31 - 8 columns: a step past them is below 2^32)
        u32x4 in[NP], old[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            in[i] = old[i] = u32x4{0u, 0u, 0u, 0u};
            if (c + i * E >= C) continue;
            if (there) in[i] = row_load<T>(p.X, from + c + i * E);
            if (!GRAD) old[i] = row_load<T>(p.Y, to + c + i * E);
        }
        const Philox bits = philox(c / 8, (unsigned)row, stream, seed);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (c + i * E >= C) continue;
            float x[E], y[E];
            RowPiece<T>::get(in[i], x);
            RowPiece<T>::get(old[i], y);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int n = i * E + e;
                const bool keep = (bits.x[n / 2] >> (n % 2 * 16) & 0xffffu) < p.keep16;
                y[e] = keep ? GRAD ? x[e] * p.scale : fmaf(x[e], p.scale, y[e]) : y[e];  // (chosen, not multiplied: what is dropped may be anything)
            }
            row_store<T>(p.Y, to + c + i * E, RowPiece<T>::put(y));
        }
    }
}

template <typename T> static int launch_rows(DropoutParams p, bool grad, hipStream_t st) {
    // as many rows a workgroup as leave no thread without a column; a thread has two or more places of eight where rows are longer
    p.rows = 1;
    while (p.rows < DO_THREADS / 16 && (long long)p.C * p.rows * 2 <= DO_THREADS * 8) p.rows *= 2;
    return launch_in_turns((p.M + p.rows - 1) / p.rows, DO_THREADS, [&](long long first, unsigned count) {
        p.first = first;
        if (grad) hipLaunchKernelGGL((dropout_kernel<T, true>), dim3(count), dim3(DO_THREADS), 0, st, p);
        else hipLaunchKernelGGL((dropout_kernel<T, false>), dim3(count), dim3(DO_THREADS), 0, st, p);
    });
}

int launch_dropout(DropoutParams p, bool grad, lemo_dtype_t dt, hipStream_t st) {
    return dt == LEMO_BF16 ? launch_rows<bf16_t>(p, grad, st) : launch_rows<float>(p, grad, st);
}

}  // namespace lemo
