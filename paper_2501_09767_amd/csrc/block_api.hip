// Host side of the attention over chosen key blocks (lemo.h): argument validation and kernel launches only.
#include <algorithm>
#include <cmath>
#include <numeric>

#include "api_checks.hpp"
#include "block_attention.hpp"

using namespace lemo;

namespace {

constexpr int64_t MOST_TOKENS = ((int64_t)1 << 31) - 4096;  // positions, and those of the next few subtiles of keys, are ints (a block may end past them)

bool pitch_fits(int64_t ts) { return ts < (1 << 22); }

// sizes of heads and blocks that all calls share
int check_sizes(int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, int32_t b) {
    if (!valid_dtype(dt)) return LEMO_ERR_DTYPE;
    if (H <= 0 || H_kv <= 0 || H % H_kv || b <= 0) return LEMO_ERR_SHAPE;
    return (d != 64 && d != 128) || b % 32 || b > 65536 || H_kv > 65535 ? LEMO_ERR_UNSUPPORTED : LEMO_OK;
}

// element strides of a [tokens, heads, d] tensor
int check_strides(const void* p, int64_t ts, int64_t hs, lemo_dtype_t dt) {
    if (!p) return LEMO_ERR_NULL;
    if (ts < 0 || hs < 0) return LEMO_ERR_SHAPE;
    if (!pitch_fits(ts)) return LEMO_ERR_UNSUPPORTED;
    const int e16 = elems_per_16B(dt);
    return aligned16(p) && ts % e16 == 0 && hs % e16 == 0 ? LEMO_OK : LEMO_ERR_ALIGN;
}

// a list's length and the query blocks
int check_lists(int64_t S_q, int64_t S_k, int64_t q_start, int32_t H, int32_t H_kv, int32_t T, int32_t b, int32_t bq) {
    if (S_q <= 0 || S_q >= MOST_TOKENS || S_k <= 0 || S_k >= MOST_TOKENS || q_start < 0 || q_start >= MOST_TOKENS || T <= 0 || bq <= 0) return LEMO_ERR_SHAPE;
    if ((int64_t)T * (b / 32) > MAX_LISTED_SUBTILES) return LEMO_ERR_UNSUPPORTED;
    const int64_t q = bq < S_q ? bq : S_q;
    return q * (H / H_kv) >= (1 << 24) || (S_q + q - 1) / q * H_kv >= (int64_t)1 << 28 ? LEMO_ERR_UNSUPPORTED : LEMO_OK;
}

// sizes of the gradient: places in the lists turned round, and in the rows that a key block gathers, are ints
int check_turned_lists(int64_t S_q, int64_t S_k, int32_t H, int32_t H_kv, int32_t T, int32_t b, int32_t bq) {
    const int64_t q = bq < S_q ? bq : S_q, n_qb = (S_q + q - 1) / q, nb = (S_k - 1) / b + 1, limit = (int64_t)1 << 31;
    if (nb > MAX_LISTED_BLOCKS) return LEMO_ERR_UNSUPPORTED;
    return n_qb * H_kv * (T < nb ? T : nb) >= limit || n_qb * q * (H / H_kv) >= limit - 4096 ? LEMO_ERR_UNSUPPORTED : LEMO_OK;
}

// whether T blocks hold the positions of any query block, b keys each.  How a query block of q lies to the blocks repeats after b / gcd(q, b)
// of them at most; blocks at the far ends of queries and keys only have fewer positions.
bool room_for_own_blocks(int64_t S_q, int64_t S_k, int64_t q_start, int64_t b, int64_t q, int64_t T) {
    if (T >= (q + b - 2) / b + 1) return true;
    const int64_t n_qb = (S_q + q - 1) / q, period = b / std::gcd(q, b);
    for (int64_t m = 0; m < n_qb && m < period; ++m) {
        const int64_t first = q_start + m * q, last = std::min(q_start + std::min((m + 1) * q, S_q), S_k) - 1;
        if (last / b - first / b + 1 > T) return false;
    }
    return true;
}

int64_t span_bytes(int64_t S, int64_t ts, int64_t H, int64_t hs, int64_t d) { return ((S - 1) * ts + (H - 1) * hs + d) * 2; }

float base2(float scale, int32_t d) { return (float)((scale > 0.f ? (double)scale : 1.0 / std::sqrt((double)d)) * 1.4426950408889634); }

// room for the shares of the lists; S_k bounds what lists of few rows name together (single tokens do not come together)
size_t part_bytes(int64_t n_qb, int64_t bq, int64_t S_k, int32_t H, int32_t H_kv, int32_t d, int32_t T, int32_t b, bool step) {
    BlockAttnParams p{};
    static const int one = 0;
    p.lengths = step ? &one : nullptr;  // (not read)
    p.n_qb = (int)n_qb; p.bq = (int)bq; p.nb = (int)((S_k - 1) / b + 1); p.H_kv = H_kv; p.T = T; p.b = b;
    p.R = (int)(bq * (H / H_kv));
    const int subtiles = block_attention_packed(p), tile = block_attention_tile_rows(p.R, d == 128 && !step);
    const int parts = block_attention_parts((int64_t)p.n_qb * ((p.R + tile - 1) / tile) * H_kv, subtiles);
    return parts > 1 ? round_up((size_t)p.n_qb * H_kv * parts * p.R * (d + 4) * sizeof(float), 256) : 0;
}

// what forward and gradient take alike; fills the parameter block
int check_attention(const void* Q, const void* K, const void* V, int64_t S_q, int64_t S_k, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt,
                    int64_t q_ts, int64_t q_hs, int64_t k_ts, int64_t k_hs, int64_t v_ts, int64_t v_hs, const int32_t* blocks, int32_t T, int32_t b,
                    int32_t bq, int64_t q_start, float scale, uint32_t flags, BlockAttnParams& p) {
    int rc = check_sizes(H, H_kv, d, dt, b);
    if (rc == LEMO_OK) rc = check_lists(S_q, S_k, q_start, H, H_kv, T, b, bq);
    if (rc != LEMO_OK) return rc;
    if ((flags & ~(uint32_t)LEMO_CAUSAL) || !std::isfinite(scale)) return LEMO_ERR_SHAPE;
    if (dt != LEMO_BF16) return LEMO_ERR_UNSUPPORTED;
    if (!blocks) return LEMO_ERR_NULL;
    rc = check_strides(Q, q_ts, q_hs, dt);
    if (rc == LEMO_OK) rc = check_strides(K, k_ts, k_hs, dt);
    if (rc == LEMO_OK) rc = check_strides(V, v_ts, v_hs, dt);
    if (rc != LEMO_OK) return rc;
    if (reinterpret_cast<uintptr_t>(blocks) & 3u) return LEMO_ERR_ALIGN;
    p = BlockAttnParams{};
    p.Q = static_cast<const uint16_t*>(Q); p.K = static_cast<const uint16_t*>(K); p.V = static_cast<const uint16_t*>(V);
    p.blocks = blocks;
    p.S_q = (int)S_q; p.S_k = (int)S_k; p.H = H; p.H_kv = H_kv; p.G = H / H_kv; p.T = T; p.b = b;
    p.nb = (int)((S_k - 1) / b + 1);
    p.bq = (int)(bq < S_q ? bq : S_q);
    p.n_qb = (int)((S_q + p.bq - 1) / p.bq);
    p.R = p.bq * p.G;
    p.q_start = q_start;
    p.q_ts = q_ts; p.q_hs = q_hs; p.k_ts = k_ts; p.k_hs = k_hs; p.v_ts = v_ts; p.v_hs = v_hs;
    p.c2 = base2(scale, d);
    p.flags = flags;
    return LEMO_OK;
}

// Keys up to the last query's under the mask: what stands behind them (a cache's room, for instance) is never loaded
int keys_seen(const BlockAttnParams& p) { return p.flags & LEMO_CAUSAL ? (int)std::min<int64_t>(p.S_k, p.q_start + p.S_q) : p.S_k; }

}  // namespace

extern "C" {

int lemo_block_means(const void* K, int64_t S, int32_t H_kv, int32_t d, lemo_dtype_t dt, int64_t k_tok_stride, int64_t k_head_stride, int32_t b, float* means,
                     void* stream) {
    int rc = check_sizes(H_kv, H_kv, d, dt, b);
    if (rc != LEMO_OK) return rc;
    if (S <= 0 || S >= MOST_TOKENS) return LEMO_ERR_SHAPE;
    if (!means) return LEMO_ERR_NULL;
    rc = check_strides(K, k_tok_stride, k_head_stride, dt);
    if (rc != LEMO_OK) return rc;
    if (!aligned16(means)) return LEMO_ERR_ALIGN;
    return hip_rc(launch_block_means(K, S, H_kv, d, dt, k_tok_stride, k_head_stride, b, means, static_cast<hipStream_t>(stream)));
}

int lemo_select_blocks(const void* Q, int64_t S_q, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, int64_t q_tok_stride, int64_t q_head_stride,
                       const float* means, int64_t S_k, int64_t q_start, int32_t b, int32_t bq, int32_t T, uint32_t flags, int32_t* blocks, void* stream) {
    int rc = check_sizes(H, H_kv, d, dt, b);
    if (rc == LEMO_OK) rc = check_lists(S_q, S_k, q_start, H, H_kv, T, b, bq);
    if (rc != LEMO_OK) return rc;
    if (flags & ~(uint32_t)LEMO_CAUSAL) return LEMO_ERR_SHAPE;
    if (!means || !blocks) return LEMO_ERR_NULL;
    rc = check_strides(Q, q_tok_stride, q_head_stride, dt);
    if (rc != LEMO_OK) return rc;
    if (!aligned16(means) || (reinterpret_cast<uintptr_t>(blocks) & 3u)) return LEMO_ERR_ALIGN;
    if ((S_k + b - 1) / b > MAX_LISTED_BLOCKS) return LEMO_ERR_UNSUPPORTED;
    const int32_t q = bq < S_q ? bq : (int32_t)S_q;
    if (flags & LEMO_CAUSAL) {  // the blocks that hold the queries themselves are always listed: there has to be room for them
        if (!room_for_own_blocks(S_q, S_k, q_start, b, q, T)) return LEMO_ERR_SHAPE;
    }
    BlockSelectParams p{};
    p.Q = Q; p.means = means; p.blocks = blocks;
    p.S_q = (int)S_q; p.S_k = (int)S_k; p.H = H; p.H_kv = H_kv; p.G = H / H_kv; p.d = d; p.T = T; p.b = b; p.bq = q;
    p.n_qb = (int)((S_q + q - 1) / q); p.nb = (int)((S_k + b - 1) / b);
    p.q_start = q_start; p.q_ts = q_tok_stride; p.q_hs = q_head_stride;
    p.flags = flags;
    return hip_rc(launch_select_blocks(p, dt, static_cast<hipStream_t>(stream)));
}

int lemo_block_attention_workspace_bytes(int64_t S_q, int64_t S_k, int32_t H, int32_t H_kv, int32_t d, int32_t T, int32_t b, int32_t bq, size_t* bytes) {
    if (!bytes) return LEMO_ERR_NULL;
    int rc = check_sizes(H, H_kv, d, LEMO_BF16, b);
    if (rc == LEMO_OK) rc = check_lists(S_q, S_k, 0, H, H_kv, T, b, bq);
    if (rc != LEMO_OK) return rc;
    const int64_t q = bq < S_q ? bq : S_q;
    *bytes = part_bytes((S_q + q - 1) / q, q, S_k, H, H_kv, d, T, b, false);
    return LEMO_OK;
}

int lemo_block_attention(const void* Q, const void* K, const void* V, int64_t S_q, int64_t S_k, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt,
                         int64_t q_tok_stride, int64_t q_head_stride, int64_t k_tok_stride, int64_t k_head_stride, int64_t v_tok_stride,
                         int64_t v_head_stride, const int32_t* blocks, int32_t T, int32_t b, int32_t bq, int64_t q_start, float scale, uint32_t flags,
                         void* O, int64_t o_tok_stride, int64_t o_head_stride, float* lse2, void* workspace, size_t workspace_bytes, void* stream) {
    BlockAttnParams p;
    int rc = check_attention(Q, K, V, S_q, S_k, H, H_kv, d, dt, q_tok_stride, q_head_stride, k_tok_stride, k_head_stride, v_tok_stride, v_head_stride,
                             blocks, T, b, bq, q_start, scale, flags, p);
    if (rc != LEMO_OK) return rc;
    rc = check_strides(O, o_tok_stride, o_head_stride, dt);
    if (rc != LEMO_OK) return rc;
    if (reinterpret_cast<uintptr_t>(lse2) & 3u) return LEMO_ERR_ALIGN;
    const size_t need = part_bytes(p.n_qb, p.bq, S_k, H, H_kv, d, T, b, false);
    if (need && !workspace) return LEMO_ERR_NULL;
    if (need && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return LEMO_ERR_ALIGN;
    if (workspace_bytes < need) return LEMO_ERR_WORKSPACE;
    p.S_k = keys_seen(p);
    p.O = static_cast<uint16_t*>(O); p.o_ts = o_tok_stride; p.o_hs = o_head_stride; p.lse2 = lse2;
    p.parts = need ? static_cast<float*>(workspace) : nullptr;
    return hip_rc(launch_block_attention(p, d, static_cast<hipStream_t>(stream)));
}

int lemo_block_attention_grad_workspace_bytes(int64_t S_q, int64_t S_k, int32_t H, int32_t H_kv, int32_t d, int32_t T, int32_t b, int32_t bq, size_t* bytes) {
    if (!bytes) return LEMO_ERR_NULL;
    int rc = check_sizes(H, H_kv, d, LEMO_BF16, b);
    if (rc == LEMO_OK) rc = check_lists(S_q, S_k, 0, H, H_kv, T, b, bq);
    if (rc == LEMO_OK) rc = check_turned_lists(S_q, S_k, H, H_kv, T, b, bq);
    if (rc != LEMO_OK) return rc;
    *bytes = block_grad_layout(S_q, S_k, H, H_kv, d, T, b, (int)(bq < S_q ? bq : S_q)).bytes;
    return LEMO_OK;
}

int lemo_block_attention_grad(const void* dO, const void* Q, const void* K, const void* V, const void* O, const float* lse2, int64_t S_q, int64_t S_k,
                              int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, int64_t do_tok_stride, int64_t do_head_stride, int64_t q_tok_stride,
                              int64_t q_head_stride, int64_t k_tok_stride, int64_t k_head_stride, int64_t v_tok_stride, int64_t v_head_stride,
                              int64_t o_tok_stride, int64_t o_head_stride, const int32_t* blocks, int32_t T, int32_t b, int32_t bq, int64_t q_start,
                              float scale, uint32_t flags, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, void* stream) {
    BlockGradParams gp{};
    int rc = check_attention(Q, K, V, S_q, S_k, H, H_kv, d, dt, q_tok_stride, q_head_stride, k_tok_stride, k_head_stride, v_tok_stride, v_head_stride,
                             blocks, T, b, bq, q_start, scale, flags, gp.a);
    if (rc != LEMO_OK) return rc;
    if (!lse2 || !dQ || !dK || !dV || !workspace) return LEMO_ERR_NULL;
    rc = check_strides(dO, do_tok_stride, do_head_stride, dt);
    if (rc == LEMO_OK) rc = check_strides(O, o_tok_stride, o_head_stride, dt);
    if (rc != LEMO_OK) return rc;
    if (!aligned16(dQ) || !aligned16(dK) || !aligned16(dV) || (reinterpret_cast<uintptr_t>(lse2) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return LEMO_ERR_ALIGN;
    rc = check_turned_lists(S_q, S_k, H, H_kv, T, b, bq);
    if (rc != LEMO_OK) return rc;
    // the rows that a key block gathers are addressed with 32-bit offsets
    const int64_t most = ((int64_t)1 << 32) - 4096;
    if (span_bytes(S_q, q_tok_stride, H, q_head_stride, d) > most || span_bytes(S_q, do_tok_stride, H, do_head_stride, d) > most) return LEMO_ERR_UNSUPPORTED;
    BlockAttnParams& p = gp.a;
    const BlockGradLayout l = block_grad_layout(S_q, S_k, H, H_kv, d, T, b, p.bq);
    if (workspace_bytes < l.bytes) return LEMO_ERR_WORKSPACE;
    p.O = static_cast<uint16_t*>(const_cast<void*>(O)); p.o_ts = o_tok_stride; p.o_hs = o_head_stride; p.lse2 = const_cast<float*>(lse2);
    gp.dO = static_cast<const uint16_t*>(dO); gp.do_ts = do_tok_stride; gp.do_hs = do_head_stride;
    gp.dQ = static_cast<uint16_t*>(dQ); gp.dK = static_cast<uint16_t*>(dK); gp.dV = static_cast<uint16_t*>(dV);
    gp.scale = scale > 0.f ? scale : (float)(1.0 / std::sqrt((double)d));
    char* const ws = static_cast<char*>(workspace);
    gp.delta = reinterpret_cast<float*>(ws + l.delta);
    gp.bits = reinterpret_cast<unsigned*>(ws + l.bits);
    gp.counts = reinterpret_cast<int*>(ws + l.counts);
    gp.first = reinterpret_cast<int*>(ws + l.first);
    gp.lists = reinterpret_cast<int*>(ws + l.lists);
    gp.slots = reinterpret_cast<int*>(ws + l.slots);
    gp.items = reinterpret_cast<int4*>(ws + l.items);
    gp.totals = reinterpret_cast<int*>(ws + l.totals);
    gp.partial = reinterpret_cast<float*>(ws + l.partial);
    gp.nb = p.nb;
    gp.S_all = p.S_k;
    p.S_k = keys_seen(p);
    gp.words = (p.n_qb + 31) / 32;
    gp.share = l.share;
    gp.max_items = l.max_items;
    return hip_rc(launch_block_attention_grad(gp, d, static_cast<hipStream_t>(stream)));
}

int lemo_block_means_step(const void* K, int32_t B, int64_t S_max, int32_t H_kv, int32_t d, lemo_dtype_t dt, int64_t k_seq_stride, int64_t k_tok_stride,
                          int64_t k_head_stride, const int32_t* lengths, int32_t b, float* means, void* stream) {
    int rc = check_sizes(H_kv, H_kv, d, dt, b);
    if (rc != LEMO_OK) return rc;
    if (S_max <= 0 || S_max >= MOST_TOKENS || B < 0 || k_seq_stride < 0) return LEMO_ERR_SHAPE;
    if (B == 0) return LEMO_OK;
    if (!means || !lengths) return LEMO_ERR_NULL;
    rc = check_strides(K, k_tok_stride, k_head_stride, dt);
    if (rc != LEMO_OK) return rc;
    if (!aligned16(means) || k_seq_stride % elems_per_16B(dt) || (reinterpret_cast<uintptr_t>(lengths) & 3u)) return LEMO_ERR_ALIGN;
    return hip_rc(launch_block_means_step(K, lengths, B, S_max, H_kv, d, dt, k_seq_stride, k_tok_stride, k_head_stride, b, means, (int)((S_max + b - 1) / b),
                                          static_cast<hipStream_t>(stream)));
}

int lemo_select_blocks_step(const void* Q, int32_t B, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, int64_t q_tok_stride, int64_t q_head_stride,
                            const float* means, int64_t S_max, const int32_t* lengths, int32_t b, int32_t T, int32_t* blocks, void* stream) {
    int rc = check_sizes(H, H_kv, d, dt, b);
    if (rc != LEMO_OK) return rc;
    if (B < 0) return LEMO_ERR_SHAPE;
    rc = check_lists(B > 0 ? B : 1, S_max, 0, H, H_kv, T, b, 1);
    if (rc != LEMO_OK) return rc;
    if (B == 0) return LEMO_OK;
    if (!means || !blocks || !lengths) return LEMO_ERR_NULL;
    rc = check_strides(Q, q_tok_stride, q_head_stride, dt);
    if (rc != LEMO_OK) return rc;
    if (!aligned16(means) || (reinterpret_cast<uintptr_t>(blocks) & 3u) || (reinterpret_cast<uintptr_t>(lengths) & 3u)) return LEMO_ERR_ALIGN;
    if ((S_max + b - 1) / b > MAX_LISTED_BLOCKS) return LEMO_ERR_UNSUPPORTED;
    BlockSelectParams p{};
    p.Q = Q; p.means = means; p.blocks = blocks; p.lengths = lengths;
    p.S_q = B; p.S_k = (int)S_max; p.H = H; p.H_kv = H_kv; p.G = H / H_kv; p.d = d; p.T = T; p.b = b; p.bq = 1;
    p.n_qb = B; p.nb = (int)((S_max + b - 1) / b);
    p.q_ts = q_tok_stride; p.q_hs = q_head_stride; p.means_ss = (long long)p.nb * H_kv * d;
    p.flags = LEMO_CAUSAL;
    return hip_rc(launch_select_blocks(p, dt, static_cast<hipStream_t>(stream)));
}

int lemo_block_attention_step_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t d, int32_t T, int32_t b, size_t* bytes) {
    if (!bytes) return LEMO_ERR_NULL;
    if (B < 0) return LEMO_ERR_SHAPE;
    int rc = check_sizes(H, H_kv, d, LEMO_BF16, b);
    if (rc == LEMO_OK) rc = check_lists(B > 0 ? B : 1, 1, 0, H, H_kv, T, b, 1);
    if (rc != LEMO_OK) return rc;
    *bytes = part_bytes(B > 0 ? B : 1, 1, 1, H, H_kv, d, T, b, true);
    return LEMO_OK;
}

int lemo_block_attention_step(const void* Q, const void* K, const void* V, int32_t B, int64_t S_max, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt,
                              int64_t q_tok_stride, int64_t q_head_stride, int64_t k_seq_stride, int64_t k_tok_stride, int64_t k_head_stride,
                              int64_t v_seq_stride, int64_t v_tok_stride, int64_t v_head_stride, const int32_t* lengths, const int32_t* blocks, int32_t T,
                              int32_t b, float scale, void* O, int64_t o_tok_stride, int64_t o_head_stride, void* workspace, size_t workspace_bytes,
                              void* stream) {
    if (B < 0 || k_seq_stride < 0 || v_seq_stride < 0) return LEMO_ERR_SHAPE;
    BlockAttnParams p;
    if (B == 0) {
        int rc = check_sizes(H, H_kv, d, dt, b);
        return rc == LEMO_OK ? check_lists(1, S_max, 0, H, H_kv, T, b, 1) : rc;
    }
    int rc = check_attention(Q, K, V, B, S_max, H, H_kv, d, dt, q_tok_stride, q_head_stride, k_tok_stride, k_head_stride, v_tok_stride, v_head_stride,
                             blocks, T, b, 1, 0, scale, LEMO_CAUSAL, p);
    if (rc != LEMO_OK) return rc;
    if (!lengths) return LEMO_ERR_NULL;
    rc = check_strides(O, o_tok_stride, o_head_stride, dt);
    if (rc != LEMO_OK) return rc;
    if (k_seq_stride % 8 || v_seq_stride % 8 || (reinterpret_cast<uintptr_t>(lengths) & 3u)) return LEMO_ERR_ALIGN;
    const size_t need = part_bytes(B, 1, S_max, H, H_kv, d, T, b, true);
    if (need && !workspace) return LEMO_ERR_NULL;
    if (need && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return LEMO_ERR_ALIGN;
    if (workspace_bytes < need) return LEMO_ERR_WORKSPACE;
    p.lengths = lengths; p.k_ss = k_seq_stride; p.v_ss = v_seq_stride;
    p.O = static_cast<uint16_t*>(O); p.o_ts = o_tok_stride; p.o_hs = o_head_stride;
    p.parts = need ? static_cast<float*>(workspace) : nullptr;
    return hip_rc(launch_block_attention(p, d, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
