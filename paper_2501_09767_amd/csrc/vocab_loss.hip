// Cross entropy over a vocabulary from hidden rows and the head's weight, and its gradients; the logits are never stored as a whole.
//
//   x = X[idx] W^T,  u = softcap tanh(x / softcap) or x,  lse = log sum exp u
//   loss = lse - (1 - s) u[label] - s mean(u) + z lse^2            0 for rows without a label in [0, V)
//   G = dloss (exp(u - lse) (1 + 2 z lse) - (1 - s) [label] - s / V) (1 - (u / softcap)^2)      dX = G W      dW = G^T X[idx]
//
// Forward: one pass over the tiles of the product (vocab_loss_tiles.hip), which leave (maximum, sum of exponentials) a row and tile; the tiles' parts are
// joined in their order by a kernel here, and the rows' losses added by another, in 64 bits.  Gradients: the vocabulary in pieces; of a piece its
// logits once more, turned into G, then its rows of dW (finished: every token is in them) and its part of dX, which is added up in
// binary32 over the pieces and rounded once.  No atomics: the same bits on every run.
//
// What bounds it: the matrix cores, 2 M C V products forward and 6 in the gradients (8192 rows of 4096, 131072 words, bf16: loss 6.1 to 6.3 ms by
// the card, 1.40 to 1.44 PFLOP/s; 777 rows of 768, 50001 words, binary32: gradients 1.21 to 1.28 ms, 140 to 148 TFLOP/s of a library product's 154); with few rows the weight's bytes (16 rows of 4096,
// 32000 words, bf16: loss 61 us = 4.3 TB/s).  Keeping G of the whole vocabulary would save a piece's tail and the additions to dX, and is what
// the operator is there to avoid.
//
// binary32: the products are the selective-load GEMM's, a piece at a time in both directions, with the softmax in kernels of its own between them.  For dX
// that GEMM wants both operands along the contraction, or neither: the smaller of G and the weight's piece is transposed, and the contraction cut into
// parts like bf16's.
#include <algorithm>

#include "vocab_softmax.hpp"
#include "row_pieces.hpp"

namespace lemo {

constexpr int VL_THREADS = 256;
constexpr long long VL_ROWS = 16384;  // rows of a forward launch: bounds what the tiles leave
constexpr int VL_CHUNK = 8192;        // (binary32) columns of a workgroup: few long rows fill the machine, too

// ---- rows --------------------------------------------------------------------------------------------

// sum, number, mean and 1 / number of the rows that count
__device__ __forceinline__ void write_total(double sum, long long n, float* total) {
    total[0] = (float)sum;
    total[1] = (float)n;
    total[2] = n ? (float)(sum / (double)n) : 0.f;
    total[3] = n ? (float)(1. / (double)n) : 0.f;
}

// Joins the parts of a row: `per` rows a workgroup (a power of two up to 64), VL_THREADS / per threads a row, each a part in so many; then the threads of a
// wave, then the waves.  One workgroup for all rows: the losses' sum, too (total; a launch less).
__global__ __launch_bounds__(VL_THREADS) void vocab_join_kernel(VocabRule rule, const float2* parts, const float* sums, const float* picked, const int* labels,
                                                                long long M, int n, int per, float* loss, float* lse, float* total) {
    constexpr int WAVES = VL_THREADS / 64;
    __shared__ float lds[3][WAVES][64];
    __shared__ float losses[64];
    const int threads = VL_THREADS / per, mine = threadIdx.x / per;
    const long long m = (long long)blockIdx.x * per + threadIdx.x % per;
    float top = -INFINITY, sum = 0.f, all = 0.f;
    if (m < M) {
#pragma unroll 8
        for (int t = mine; t < n; t += threads) {
            const float2 v = parts[(long long)t * M + m];
            vocab_join(top, sum, v.x, v.y);
            if (sums) all += sums[(long long)t * M + m];
        }
    }
    for (int s = per; s < 64; s <<= 1) {
        const float top2 = __shfl_xor(top, s), sum2 = __shfl_xor(sum, s);
        vocab_join(top, sum, top2, sum2);
        all += __shfl_xor(all, s);
    }
    const int lane = threadIdx.x & 63;
    if (lane < per) {
        lds[0][threadIdx.x >> 6][lane] = top;
        lds[1][threadIdx.x >> 6][lane] = sum;
        lds[2][threadIdx.x >> 6][lane] = all;
    }
    __syncthreads();
    if (threadIdx.x < per) {
        for (int w = 1; w < WAVES; ++w) {
            vocab_join(top, sum, lds[0][w][lane], lds[1][w][lane]);
            all += lds[2][w][lane];
        }
        float v = 0.f;
        if (m < M) {
            const float whole = top + logf(sum);
            lse[m] = whole;
            const int label = labels[m];
            if (label >= 0 && label < rule.V) {
                v = fmaf(rule.z * whole, whole, whole) - rule.hit * picked[m];
                if (sums) v -= rule.all * all;
            }
            loss[m] = v;
        }
        losses[threadIdx.x] = v;
    }
    if (!total) return;
    __syncthreads();
    if (threadIdx.x) return;
    double of = 0.;
    long long counted = 0;
    for (long long i = 0; i < M; ++i) {
        of += (double)losses[i];
        counted += labels[i] >= 0 && labels[i] < rule.V;
    }
    write_total(of, counted, total);
}

// the same of many rows
__global__ __launch_bounds__(1024) void vocab_total_kernel(const float* loss, const int* labels, long long M, int V, float* total) {
    __shared__ double sums[16];
    __shared__ int counts[16];
    double sum = 0.;
    long long n = 0;
    for (long long m = threadIdx.x; m < M; m += 1024) {
        sum += (double)loss[m];
        n += labels[m] >= 0 && labels[m] < V;
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        sum += __shfl_xor(sum, s);
        n += __shfl_xor(n, s);
    }
    if ((threadIdx.x & 63) == 0) {
        sums[threadIdx.x >> 6] = sum;
        counts[threadIdx.x >> 6] = (int)n;
    }
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 16; ++w) {
        sum += sums[w];
        n += counts[w];
    }
    write_total(sum, n, total);
}

// dX = the sum of the planes, rounded once; in bf16 with the label's row of W times what G's rounding has left of its element, and times the gradient
// that was left out of G.  A thread has 16 bytes of a row.
template <typename T>
__global__ __launch_bounds__(VL_THREADS) void vocab_planes_kernel(const float* planes, long long plane, int n, const float* rest, const float* scale, float scale_by,
                                                                  const int* labels, int V, const void* W, long long ldw, long long M, int C, void* dX, long long lddx, long long first) {
    constexpr int E = RowPiece<T>::E;
    const long long per_row = C / E, i = (first + blockIdx.x) * VL_THREADS + threadIdx.x;
    const long long m = i / per_row;
    if (m >= M) return;
    const int c = (int)(i - m * per_row) * E, label = labels[m];
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = 0.f;
    if (label >= 0 && label < V) {
#pragma unroll 4
        for (int s = 0; s < n; ++s) {
            const f32x4* const at = reinterpret_cast<const f32x4*>(planes + s * plane + m * C + c);
#pragma unroll
            for (int h = 0; h < E / 4; ++h) {
                const f32x4 x = at[h];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[h * 4 + e] += x[e];
            }
        }
        if constexpr (E == 8) {
            const float left = rest[m], by = scale ? *scale * scale_by : 1.f;
            float w[E];
            RowPiece<T>::get(row_load<T>(W, label * ldw + c), w);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = fmaf(left, w[e], v[e]) * by;
        }
    }
    row_store<T>(dX, m * lddx + c, RowPiece<T>::put(v));
}

// ---- binary32: a piece's logits in memory -----------------------------------------------------------

// A workgroup a chunk of a row (16-byte aligned): its part of the statistics, as a tile leaves it
__global__ __launch_bounds__(VL_THREADS) void vocab_stats_f32_kernel(VocabRule rule, const float* x, long long ldx, int N, int chunks, int v0, const int* labels,
                                                                     long long M, float2* parts, float* sums, float* picked, long long first) {
    __shared__ float lds[3][VL_THREADS / 64];
    const long long block = first + blockIdx.x, m = block / chunks;
    const int chunk = (int)(block - m * chunks), end = min(N, (chunk + 1) * VL_CHUNK);
    const float* const row = x + m * ldx;
    const bool capped = rule.softcap > 0.f;
    const float inv_cap = capped ? 1.f / rule.softcap : 0.f;
    const unsigned label = (unsigned)labels[m] - (unsigned)v0;
    float top = -INFINITY, sum = 0.f, all = 0.f;
    for (int n = chunk * VL_CHUNK + threadIdx.x * 4; n < end; n += VL_THREADS * 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(row + n);  // (the pitch is a multiple of 64: what lies behind the row is there, and not used)
        float u[4], t = top;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            u[e] = n + e >= N ? -INFINITY : capped ? vocab_cap(v[e], rule.softcap, inv_cap) : v[e];
            if (n + e < N && (unsigned)(n + e) == label) picked[m] = u[e];
            t = fmaxf(t, u[e]);
        }
        sum *= vocab_scale(top, t);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum += vocab_scale(u[e], t);
            all += n + e < N ? u[e] : 0.f;
        }
        top = t;
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        vocab_join(top, sum, __shfl_xor(top, s), __shfl_xor(sum, s));
        all += __shfl_xor(all, s);
    }
    if ((threadIdx.x & 63) == 0) {
        lds[0][threadIdx.x >> 6] = top;
        lds[1][threadIdx.x >> 6] = sum;
        lds[2][threadIdx.x >> 6] = all;
    }
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < VL_THREADS / 64; ++w) {
        vocab_join(top, sum, lds[0][w], lds[1][w]);
        all += lds[2][w];
    }
    parts[chunk * M + m] = make_float2(top, sum);
    if (sums) sums[chunk * M + m] = all;
}

// logits -> G in place, and zeros in the columns from N up to a multiple of 64
__global__ __launch_bounds__(VL_THREADS) void vocab_probs_f32_kernel(VocabRule rule, VocabSide side, float* x, long long ldx, int N, int chunks, int v0,
                                                                     const int* labels, const float* lse, const int* idx, long long M, long long first) {
    const long long block = first + blockIdx.x, m = block / chunks;
    const int chunk = (int)(block - m * chunks), end = min((N + 63) / 64 * 64, (chunk + 1) * VL_CHUNK);
    if (side.rows && chunk == 0) {
        if (threadIdx.x == 0) vocab_list_row(rule, side, labels, idx, m, M);
        if (side.zero_row && m == M - 1)
            for (int n = threadIdx.x * 4; n < N; n += VL_THREADS * 4) *reinterpret_cast<f32x4*>(x + M * ldx + n) = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float* const row = x + m * ldx;
    const bool capped = rule.softcap > 0.f;
    const float inv_cap = capped ? 1.f / rule.softcap : 0.f;
    const VocabRow of = vocab_row_of(rule, side, lse, labels, m);
    for (int n = chunk * VL_CHUNK + threadIdx.x * 4; n < end; n += VL_THREADS * 4) {
        f32x4* const at = reinterpret_cast<f32x4*>(row + n);
        f32x4 v = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = capped ? vocab_cap(v[e], rule.softcap, inv_cap) : v[e];
            v[e] = n + e < N && of.counts ? vocab_grad(rule, of, u, v0 + n + e == of.label, inv_cap) : 0.f;
        }
        *at = v;
    }
}

// ---- launches ------------------------------------------------------------------------------------------

static size_t vl_round(size_t v) { return (v + 255) / 256 * 256; }
static long long vl_pitch(int piece) { return (piece + 63) / 64 * 64; }

static int vl_chunks(int N) { return (N + VL_CHUNK - 1) / VL_CHUNK; }

// Columns at a time.  A piece costs what its launches leave idle and, of dX, 8 bytes for each of M C elements; G of a piece costs memory: 256 MiB, which also is what the
// last-level cache holds, but no fewer than 8192 columns, for whose products that traffic is little (bf16, gradients of 65536 rows, 1024 columns, 32768 words: 8192 at a time 12.2 ms
// with 1.34 GB, 4096 14.1 with 0.81, 1024 29.0 with 0.40, 16384 12.3 with 2.41;  32768 rows, 131072 words: 24.5 / 28.2 / 58.2 / 22.7 ms).
static int vl_choice(long long M, int V, int esz) {
    const long long most = std::max<long long>(8192, (256ll << 20) / (std::max<long long>(M, 1) * esz) / 1024 * 1024);
    const long long n = (V + most - 1) / most;
    return (int)((V + n - 1) / n + 255) / 256 * 256;
}

// Parts of G's elements (bf16).  Rounded once, the label's element of a row is as far off as the store of the results it makes, and the weight's gradient of few rows has no
// mean of many such roundings (1 to 32 rows of 1024, 8000 words, gradients of their own: dW 2.1e-3 to 2.4e-3 from 64 bits on the mean of draws, up to 3.9e-3; in two parts
// 1.6e-3 to 1.7e-3, as its store alone).  Both parts within the slab that the contraction is padded to: 16 rows of 4096, 131072 words 688 -> 707 us, one row 679 -> 676;  16 rows
// of 1024, 8000 words 28.0 -> 28.5.  More rows in two parts would be products of twice the length.
static int vl_parts(long long M, int V, lemo_dtype_t dt) { return dt == LEMO_BF16 && 2 * M + (V % 8 != 0) <= 64 ? 2 : 1; }

int vocab_piece(long long M, int C, int V, long long ldw, int wanted, lemo_dtype_t dt) {
    const long long esz = dt == LEMO_BF16 ? 2 : 4, span = (1ll << 31) - 1;
    long long piece = wanted > 0 ? (std::min(wanted, V) + 63) / 64 * 64ll : vl_choice(M, V, (int)esz);
    piece = std::min(piece, vl_pitch(V));
    piece = std::min(piece, span / (ldw * esz) / 64 * 64);       // the piece's rows of W, and
    piece = std::min(piece, span / ((vl_parts(M, V, dt) * M + 1) * esz) / 64 * 64);  // G lie within 32-bit offsets,
    piece = std::min(piece, ((8ll << 20) / esz - 64) / 64 * 64); // G's pitch within a load's
    if (piece < 64) return 0;
    if (wanted == 0) piece = std::min(piece, vl_pitch((int)((V + (V + piece - 1) / piece - 1) / ((V + piece - 1) / piece))));  // no small rest
    return (int)piece;
}

// forward: what the tiles, or binary32's pieces, leave
struct LossSpace { float2* parts; float* sums; float* picked; float* logits; long long rows; int piece; size_t bytes; };
static LossSpace loss_space(long long M, int C, int V, lemo_dtype_t dt, void* base) {
    LossSpace s{};
    s.rows = std::min(M, VL_ROWS);
    s.piece = dt == LEMO_F32 ? std::min<int>(vl_choice(s.rows, V, 4), (int)vl_pitch(V)) : 0;
    const size_t n = dt == LEMO_F32 ? (size_t)((V + s.piece - 1) / s.piece) * vl_chunks(s.piece) : (size_t)(V + 127) / 128;
    char* at = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        char* const here = at + s.bytes;
        s.bytes += vl_round(bytes);
        return here;
    };
    s.parts = reinterpret_cast<float2*>(take(n * s.rows * sizeof(float2)));
    s.sums = reinterpret_cast<float*>(take(n * s.rows * sizeof(float)));
    s.picked = reinterpret_cast<float*>(take(s.rows * sizeof(float)));
    if (dt == LEMO_F32) s.logits = reinterpret_cast<float*>(take((size_t)s.rows * s.piece * sizeof(float)));
    return s;
}
size_t vocab_loss_workspace(long long M, int C, int V, lemo_dtype_t dt) { return M > 0 ? loss_space(M, C, V, dt, nullptr).bytes : 0; }

int prepare_vocab_loss(lemo_dtype_t dt) { return dt == LEMO_BF16 ? prepare_vocab_tiles() : prepare_gather_gemm_small(dt, false, GG_NT); }
int prepare_vocab_grad(lemo_dtype_t dt) {
    if (dt == LEMO_BF16) return prepare_vocab_tiles();
    const int rc = first_error([&] { return prepare_vocab_loss(dt); }, [&] { return prepare_gather_gemm_dw(dt); });
    return rc ? rc : prepare_gather_gemm_parts();
}

static unsigned vl_span(long long rows, long long ld, long long cols, int esz) { return (unsigned)(((rows - 1) * ld + cols) * esz); }

// binary32.  Up to 32 rows are one row of 32 x 32 tiles, on which the weight passes at memory's rate; 128 x 128 tiles would multiply by 96 rows of nothing
// (16 rows, 4096 columns, 131072 words: 663 us).
static int launch_logits_f32(const void* X, long long S, long long ldx, const int* idx, long long M, const void* W, long long ldw, float* Y, long long ldy, int C, int N,
                             hipStream_t st) {
    if (M > 32) return launch_gather_gemm(X, S, ldx, idx, M, W, ldw, nullptr, Y, ldy, C, N, LEMO_F32, st);
    GgParams t{};
    t.A = X; t.B = W; t.Y = Y; t.idx = idx; t.lda = ldx; t.ldb = ldw; t.ldy = ldy; t.M = M; t.K = C; t.N = N;
    t.a_bytes = vl_span(S, ldx, C, 4);
    return launch_gather_gemm_small(t, LEMO_F32, false, GG_NT, GG_T64, st);
}

int launch_vocab_loss(const VocabLossParams& p, lemo_dtype_t dt, hipStream_t st) {
    int rc = prepare_vocab_loss(dt);
    if (rc) return rc;
    const int V = p.rule.V;
    const LossSpace s = loss_space(p.M, p.C, V, dt, p.workspace);
    float* const sums = p.rule.all != 0.f ? s.sums : nullptr;
    for (long long m0 = 0; m0 < p.M; m0 += VL_ROWS) {
        const long long M = std::min(VL_ROWS, p.M - m0);
        const int* const idx = p.idx ? p.idx + m0 : nullptr;
        const int esz = dt == LEMO_BF16 ? 2 : 4;
        const char* const X = static_cast<const char*>(p.X) + (p.idx ? 0 : m0 * p.ldx * esz);  // (without a list the rows of X themselves move on)
        const long long S = p.idx ? p.S : p.S - m0;
        int n;
        if (dt == LEMO_BF16) {
            VocabTileParams t{};
            t.A = X; t.B = p.W; t.idx = idx; t.lda = p.ldx; t.ldb = p.ldw; t.M = M; t.K = p.C; t.N = V;
            t.a_bytes = vl_span(S, p.ldx, p.C, 2);
            t.rule = p.rule; t.labels = p.labels + m0; t.parts = s.parts; t.sums = sums; t.picked = s.picked;
            int one = 1;
            const GgTile tile = gg_choose_tile(M, V, p.C, GG_NT, 1, 0., &one);
            n = (V + vocab_tile_cols(tile) - 1) / vocab_tile_cols(tile);
            rc = launch_vocab_tiles(t, VOCAB_STATS, tile, st);
        } else {
            n = 0;
            for (int v0 = 0; v0 < V && rc == 0; v0 += s.piece) {
                const int N = std::min(s.piece, V - v0), chunks = vl_chunks(N);
                rc = launch_logits_f32(X, S, p.ldx, idx, M, static_cast<const float*>(p.W) + v0 * p.ldw, p.ldw, s.logits, s.piece, p.C, N, st);
                if (rc) break;
                rc = launch_in_turns(M * chunks, VL_THREADS, [&](long long first, unsigned count) {
                    hipLaunchKernelGGL(vocab_stats_f32_kernel, dim3(count), dim3(VL_THREADS), 0, st, p.rule, s.logits, (long long)s.piece, N, chunks, v0, p.labels + m0,
                                       M, s.parts + n * M, sums ? sums + n * M : nullptr, s.picked, first);
                });
                n += chunks;
            }
        }
        if (rc) return rc;
        // few rows: more threads a row, whose parts are as many as the vocabulary's tiles; up to 16: one workgroup
        const int per = M >= 4096 ? 32 : p.M <= 16 ? 16 : 4;
        hipLaunchKernelGGL(vocab_join_kernel, dim3((unsigned)((M + per - 1) / per)), dim3(VL_THREADS), 0, st, p.rule, s.parts, sums, s.picked, p.labels + m0, M, n, per,
                           p.loss + m0, p.lse + m0, p.M <= 16 ? p.total : nullptr);
        rc = (int)hipGetLastError();
        if (rc) return rc;
    }
    if (!p.total || (p.M > 0 && p.M <= 16)) return 0;
    hipLaunchKernelGGL(vocab_total_kernel, dim3(1), dim3(1024), 0, st, p.loss, p.labels, p.M, V, p.total);
    return (int)hipGetLastError();
}

// binary32: into how many parts dX's contraction is cut.  128 x 128 tiles, two a CU: a round of 512 of them takes 0.104 us for each element of the contraction (161
// TFLOP/s), one of up to 256 0.06; a plane 8 bytes an element at 4 TB/s.  (M = 777, 768 columns, V = 50001: 32 x 32 tiles without parts 700 us)
static int f32_splits(long long M, int C, int K, int* k_part) {
    const long long tiles = (M + 127) / 128 * ((C + 127) / 128);
    int best = 1;
    double least = INFINITY;
    for (int s = 1; s <= 64 && s * 64 <= std::max(K, 64); ++s) {
        const int k = (K + s * 64 - 1) / (s * 64) * 64;
        if ((long long)k * (s - 1) >= K) continue;
        const long long n = tiles * s, left = n % 512;
        const double us = (double)k * ((double)(n / 512) * 0.104 + (left == 0 ? 0. : left <= 256 ? 0.06 : 0.104)) + s * (double)M * C * 8e-6 / 4.;
        if (us < least) { least = us; best = s; *k_part = k; }
    }
    return best;
}

// gradient: rows, G, dX's planes, and in binary32 what is transposed: G, with rows of `rows` to a multiple of 64, or the weight's piece
struct GradSpace { float* rest; int* rows; char* G; float *planes, *turned; long long ldg, plane_rows; bool turn_G; GgTile tile; int parts, splits, k_split; size_t bytes; };
static GradSpace grad_space(long long M, int C, int V, int piece, lemo_dtype_t dt, void* base) {
    GradSpace s{};
    s.plane_rows = M;
    const int esz = dt == LEMO_BF16 ? 2 : 4;
    s.ldg = vl_pitch(piece);
    s.parts = vl_parts(M, V, dt);
    char* at = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        char* const here = at + s.bytes;
        s.bytes += vl_round(bytes);
        return here;
    };
    s.rest = reinterpret_cast<float*>(take((size_t)M * sizeof(float)));
    s.rows = reinterpret_cast<int*>(take((size_t)(s.parts * M + 1) * sizeof(int)));
    s.G = take((size_t)(s.parts * M + 1) * s.ldg * esz);
    if (dt == LEMO_BF16) {
        // a plane is written and read once for every piece: 8 bytes an element, at 4 TB/s
        s.tile = gg_choose_tile(M, C, std::min(piece, V), GG_NN, 32, (double)M * C * 8e-6 / 4., &s.splits);
        const int k = std::min(piece, V);
        s.k_split = (k + s.splits * 64 - 1) / (s.splits * 64) * 64;
    } else {
        s.splits = f32_splits(M, C, std::min(piece, V), &s.k_split);
        s.turn_G = M < C;
        if (s.turn_G) s.plane_rows = (M + 63) / 64 * 64;
        s.turned = reinterpret_cast<float*>(take((size_t)(s.turn_G ? s.plane_rows : C) * s.ldg * sizeof(float)));
    }
    s.planes = reinterpret_cast<float*>(take((size_t)s.splits * s.plane_rows * C * sizeof(float)));
    return s;
}
size_t vocab_grad_workspace(long long M, int C, int V, int piece, lemo_dtype_t dt) { return M > 0 ? grad_space(M, C, V, piece, dt, nullptr).bytes : 0; }

// bf16: one piece.  W: its first row.
static int grad_piece_bf16(const VocabGradParams& p, const GradSpace& s, const VocabSide& side, int v0, int N, const void* W, hipStream_t st) {
    int one = 1;
    VocabTileParams t{};
    t.A = p.X; t.B = W; t.idx = p.idx; t.lda = p.ldx; t.ldb = p.ldw; t.M = p.M; t.K = p.C; t.N = N;
    t.a_bytes = vl_span(p.S, p.ldx, p.C, 2);
    t.rule = p.rule; t.labels = p.labels; t.v0 = v0; t.lse = p.lse; t.side = side; t.rest = s.rest; t.G = s.G; t.ldg = s.ldg;
    const GgTile tile = side.parts == 2 ? GG_T64x128 : gg_choose_tile(p.M, N, p.C, GG_NT, 1, 0., &one);  // (the same for so few rows, and the kernel that has parts)
    int rc = launch_vocab_tiles(t, VOCAB_PROBS, tile, st);
    if (rc) return rc;
    if (p.dW) {
        VocabTileParams g{};
        g.A = s.G; g.B = p.X; g.idx = s.rows; g.lda = s.ldg; g.ldb = p.ldx; g.M = N; g.N = p.C;
        g.K = side.parts * (int)p.M + (N % 8 != 0);
        g.Y = static_cast<char*>(p.dW) + v0 * p.lddw * 2; g.ldy = p.lddw;
        g.b_bytes = vl_span(p.S, p.ldx, p.C, 2);
        if (side.uniform != 0.f) {
            g.scale = p.dloss; g.scale_by = 1.f / side.uniform;
            g.labels = p.labels; g.n_labels = p.M; g.rule = p.rule;
        }
        rc = launch_vocab_tiles(g, VOCAB_WEIGHT, gg_choose_tile(N, p.C, g.K, GG_TN, 1, 0., &one), st);
        if (rc) return rc;
    }
    if (!p.dX) return 0;
    VocabTileParams x{};
    x.A = s.G; x.B = W; x.lda = s.ldg; x.ldb = p.ldw; x.M = p.M; x.K = N; x.N = p.C;
    x.a_bytes = vl_span(p.M, s.ldg, (N + 7) / 8 * 8, 2);
    x.planes = s.planes; x.k_split = s.k_split; x.add = v0 > 0;
    x.splits = (N + s.k_split - 1) / s.k_split;  // (the last piece may be shorter: its parts that are empty leave their planes as they are)
    return launch_vocab_tiles(x, VOCAB_PLANES, s.tile, st);
}

static int grad_piece_f32(const VocabGradParams& p, const GradSpace& s, const VocabSide& side, int v0, int N, const float* W, hipStream_t st) {
    const int N4 = (N + 3) / 4 * 4;
    float* const G = reinterpret_cast<float*>(s.G);
    int rc = launch_logits_f32(p.X, p.S, p.ldx, p.idx, p.M, W, p.ldw, G, s.ldg, p.C, N, st);
    if (rc) return rc;
    const int chunks = vl_chunks(N);  // (a multiple of 64 columns each: what fills up the last 64 belongs to the last)
    rc = launch_in_turns(p.M * chunks, VL_THREADS, [&](long long first, unsigned count) {
        hipLaunchKernelGGL(vocab_probs_f32_kernel, dim3(count), dim3(VL_THREADS), 0, st, p.rule, side, G, s.ldg, N, chunks, v0, p.labels, p.lse, p.idx, p.M, first);
    });
    if (rc) return rc;
    if (p.dW) {
        rc = launch_gather_gemm_dw_direct(G, s.ldg, p.X, p.S, p.ldx, s.rows, p.M + (N % 4 != 0), static_cast<float*>(p.dW) + v0 * p.lddw, p.lddw, p.C, N, LEMO_F32, st);
        if (rc) return rc;
    }
    if (!p.dX) return 0;
    GgParams x{};
    x.Y = s.planes; x.ldy = p.C; x.M = x.out_rows = s.plane_rows; x.N = p.C;
    x.y_bytes = vl_span(s.plane_rows, p.C, p.C, 4);
    if (s.turn_G) {  // G^T [N, plane_rows], zeros behind M, and W as it lies
        rc = launch_transpose(G, s.ldg, nullptr, p.M, s.plane_rows, N4, s.turned, st);
        x.A = s.turned; x.B = W; x.lda = s.plane_rows; x.ldb = p.ldw; x.K = N;
        x.b_bytes = vl_span(N, p.ldw, p.C, 4);
    } else {
        const long long pad = vl_pitch(N);
        rc = launch_transpose(W, p.ldw, nullptr, N, pad, p.C, s.turned, st);
        x.A = G; x.B = s.turned; x.lda = s.ldg; x.ldb = pad; x.K = N4;
        x.a_bytes = vl_span(p.M, s.ldg, N4, 4);
    }
    if (rc) return rc;
    return launch_gather_gemm_parts(x, v0 > 0, s.turn_G ? GG_TN : GG_NT, (x.K + s.k_split - 1) / s.k_split, s.k_split, st);
}

int launch_vocab_grad(const VocabGradParams& p, lemo_dtype_t dt, hipStream_t st) {
    int rc = prepare_vocab_grad(dt);
    if (rc) return rc;
    const int V = p.rule.V, C = p.C, esz = dt == LEMO_BF16 ? 2 : 4;
    if (p.M == 0) return p.dW ? launch_zero_matrix(p.dW, p.lddw, C, V, dt, st) : 0;
    if (!p.dX && !p.dW) return 0;
    const GradSpace s = grad_space(p.M, C, V, p.piece, dt, p.workspace);
    const bool shared = p.dloss_stride == 0 && dt == LEMO_BF16;
    VocabSide side{p.dloss, p.dloss_stride, !shared ? 0.f : p.rule.hit > 0.f ? 1.f / p.rule.hit : 1.f, s.rows, (int)p.S, V % (16 / esz) != 0, p.dW ? s.parts : 1};
    for (int v0 = 0; v0 < V && rc == 0; v0 += p.piece) {
        const int N = std::min(p.piece, V - v0);
        const char* const W = static_cast<const char*>(p.W) + v0 * p.ldw * esz;
        rc = dt == LEMO_BF16 ? grad_piece_bf16(p, s, side, v0, N, W, st) : grad_piece_f32(p, s, side, v0, N, reinterpret_cast<const float*>(W), st);
        side.rows = nullptr;
    }
    if (rc || !p.dX) return rc;
    auto planes = [&](auto kernel, int e) {
        return launch_in_turns((p.M * (C / e) + VL_THREADS - 1) / VL_THREADS, VL_THREADS, [&](long long first, unsigned count) {
            hipLaunchKernelGGL(kernel, dim3(count), dim3(VL_THREADS), 0, st, s.planes, s.plane_rows * C, s.splits, s.rest, shared ? p.dloss : nullptr,
                               shared ? 1.f / side.uniform : 1.f, p.labels, V, p.W, p.ldw, p.M, C, p.dX, p.lddx, first);
        });
    };
    return dt == LEMO_BF16 ? planes(vocab_planes_kernel<bf16_t>, 8) : planes(vocab_planes_kernel<float>, 4);
}

}  // namespace lemo
