// Host side of the norms and rotation of queries and keys and of dropout (lemo.h): argument validation and kernel launches only.
#include <algorithm>
#include <cmath>
#include <utility>

#include "api_checks.hpp"
#include "dropout.hpp"
#include "qk_rotate.hpp"

using namespace lemo;

namespace {

// a [M, heads, d] operand: there, its rows and heads at 16-byte multiples
int check_heads(const void* p, int64_t ts, int64_t hs, int32_t heads, int e16) {
    if (heads == 0) return LEMO_OK;
    if (!p) return LEMO_ERR_NULL;
    if (ts < 0 || hs < 0) return LEMO_ERR_SHAPE;
    return aligned16(p) && ts % e16 == 0 && hs % e16 == 0 ? LEMO_OK : LEMO_ERR_ALIGN;
}

// the same for a result, whose rows do not lie on each other: of its dimensions, from the shortest stride on, each steps over what those before it span
int check_result(const void* p, int64_t ts, int64_t hs, int64_t M, int32_t heads, int32_t d, int e16, int64_t seqs = 1, int64_t ss = 0) {
    const int rc = check_heads(p, ts, hs, heads, e16);
    if (rc != LEMO_OK || heads == 0) return rc;
    std::pair<int64_t, int64_t> dims[3] = {{ts, M}, {hs, heads}, {ss, seqs}};
    std::sort(dims, dims + 3);
    __int128 span = d;
    for (const auto& [stride, n] : dims) {
        if (n > 1 && stride < span) return LEMO_ERR_SHAPE;
        if (n > 1) span += (__int128)(n - 1) * stride;
    }
    return LEMO_OK;
}

// what the three calls on heads share
int check_rotation(int64_t M, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, const float* inv_freq, int32_t rot, float amplitude, int32_t norm,
                   const void* w_q, const void* w_k, float eps, uint32_t flags) {
    if (!valid_dtype(dt)) return LEMO_ERR_DTYPE;
    if (norm != LEMO_NORM_NONE && norm != LEMO_NORM_RMS && norm != LEMO_NORM_LAYER) return LEMO_ERR_SHAPE;
    if (flags & ~(uint32_t)(LEMO_ROTATE_PAIRS | LEMO_WEIGHTS_PER_HEAD)) return LEMO_ERR_SHAPE;
    if (M < 0 || M >= (int64_t)1 << 31 || H < 0 || H_kv < 0 || (H == 0 && H_kv == 0) || rot < 0 || rot > d) return LEMO_ERR_SHAPE;
    if (!(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(amplitude)) return LEMO_ERR_SHAPE;
    if ((d != 64 && d != 128) || (int64_t)H + H_kv > 65535 || rot % (2 * elems_per_16B(dt))) return LEMO_ERR_UNSUPPORTED;
    if (M > 0 && rot > 0 && !inv_freq) return LEMO_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(inv_freq) & 3u) return LEMO_ERR_ALIGN;
    if (norm != LEMO_NORM_NONE && (!aligned16(w_q) || !aligned16(w_k))) return LEMO_ERR_ALIGN;
    return LEMO_OK;
}

bool small_position(int64_t p) { return p > -((int64_t)1 << 31) && p < (int64_t)1 << 31; }

RotateSide side(const void* X, int64_t x_ts, int64_t x_hs, void* Y, int64_t y_ts, int64_t y_hs, int32_t heads, const void* w, int32_t norm, int32_t d, uint32_t flags) {
    RotateSide s{};
    s.X = X; s.Y = Y; s.x_ts = x_ts; s.x_hs = x_hs; s.y_ts = y_ts; s.y_hs = y_hs; s.heads = heads;
    s.w = norm == LEMO_NORM_NONE ? nullptr : w;
    s.w_hs = flags & LEMO_WEIGHTS_PER_HEAD ? d : 0;
    return s;
}

int check_matrix(const void* p, int64_t ld, int32_t C, int e16) {
    if (!p) return LEMO_ERR_NULL;
    if (ld < C) return LEMO_ERR_SHAPE;
    return aligned16(p) && ld % e16 == 0 ? LEMO_OK : LEMO_ERR_ALIGN;
}

int dropout(const void* X, int64_t ldx, void* Y, int64_t ldy, int64_t S, const int32_t* kept_idx, int64_t M, double p, const uint64_t* rng, uint64_t site,
            int32_t C, lemo_dtype_t dt, bool grad, void* stream) {
    if (!valid_dtype(dt)) return LEMO_ERR_DTYPE;
    if (!(p >= 0.) || !(p < 1.) || S <= 0 || S >= (int64_t)1 << 31 || M < 0 || M > S || C <= 0) return LEMO_ERR_SHAPE;
    const int e16 = elems_per_16B(dt);
    if (M == 0) return LEMO_OK;
    int rc = check_matrix(X, ldx, C, e16);
    if (rc == LEMO_OK) rc = check_matrix(Y, ldy, C, e16);
    if (rc != LEMO_OK) return rc;
    if (!rng) return LEMO_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(kept_idx) & 3u) || (reinterpret_cast<uintptr_t>(rng) & 7u)) return LEMO_ERR_ALIGN;
    if (C % e16) return LEMO_ERR_UNSUPPORTED;
    DropoutParams q{};
    q.X = X; q.Y = Y; q.idx = kept_idx; q.rng = reinterpret_cast<const unsigned long long*>(rng); q.site = site;
    q.ldx = ldx; q.ldy = ldy; q.S = S; q.M = M; q.C = C;
    const double keep = std::floor((1. - p) * 65536. + 0.5);
    q.keep16 = keep < 1. ? 1u : (unsigned)keep;
    q.scale = (float)(65536. / q.keep16);
    return hip_rc(launch_dropout(q, grad, dt, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int lemo_qk_rotate(const void* Q, int64_t q_tok_stride, int64_t q_head_stride, const void* K, int64_t k_tok_stride, int64_t k_head_stride, int64_t M,
                   int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, const int32_t* positions, int64_t pos_start, const float* inv_freq, int32_t rot,
                   float amplitude, int32_t norm, const void* w_q, const void* w_k, float eps, uint32_t flags, void* Q_out, int64_t qo_tok_stride,
                   int64_t qo_head_stride, void* K_out, int64_t ko_tok_stride, int64_t ko_head_stride, void* stream) {
    int rc = check_rotation(M, H, H_kv, d, dt, inv_freq, rot, amplitude, norm, w_q, w_k, eps, flags);
    if (rc != LEMO_OK) return rc;
    if (!small_position(pos_start)) return LEMO_ERR_SHAPE;
    if (M == 0) return LEMO_OK;
    const int e16 = elems_per_16B(dt);
    rc = check_heads(Q, q_tok_stride, q_head_stride, H, e16);
    if (rc == LEMO_OK) rc = check_result(Q_out, qo_tok_stride, qo_head_stride, M, H, d, e16);
    if (rc == LEMO_OK) rc = check_heads(K, k_tok_stride, k_head_stride, H_kv, e16);
    if (rc == LEMO_OK) rc = check_result(K_out, ko_tok_stride, ko_head_stride, M, H_kv, d, e16);
    if (rc != LEMO_OK) return rc;
    if (reinterpret_cast<uintptr_t>(positions) & 3u) return LEMO_ERR_ALIGN;
    RotateParams p{};
    p.side[0] = side(Q, q_tok_stride, q_head_stride, Q_out, qo_tok_stride, qo_head_stride, H, w_q, norm, d, flags);
    p.side[1] = side(K, k_tok_stride, k_head_stride, K_out, ko_tok_stride, ko_head_stride, H_kv, w_k, norm, d, flags);
    p.positions = positions; p.inv_freq = inv_freq; p.M = M; p.pos_start = pos_start;
    p.d = d; p.rot = rot; p.norm = norm; p.pairs = (flags & LEMO_ROTATE_PAIRS) != 0; p.eps = eps; p.amplitude = amplitude;
    return hip_rc(launch_qk_rotate(p, dt, static_cast<hipStream_t>(stream)));
}

int lemo_qk_rotate_grad_workspace_bytes(int64_t M, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, uint32_t flags, size_t* bytes) {
    if (!bytes) return LEMO_ERR_NULL;
    const int rc = check_rotation(M, H, H_kv, d, dt, nullptr, 0, 1.f, LEMO_NORM_NONE, nullptr, nullptr, 0.f, flags);
    if (rc != LEMO_OK) return rc;
    *bytes = round_up(qk_rotate_grad_parts(M, H + H_kv, d, dt, (flags & LEMO_WEIGHTS_PER_HEAD) != 0) * sizeof(float), 256);
    return LEMO_OK;
}

int lemo_qk_rotate_grad(const void* dQ_out, int64_t dqo_tok_stride, int64_t dqo_head_stride, const void* dK_out, int64_t dko_tok_stride, int64_t dko_head_stride,
                        const void* Q, int64_t q_tok_stride, int64_t q_head_stride, const void* K, int64_t k_tok_stride, int64_t k_head_stride, int64_t M,
                        int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt, const int32_t* positions, int64_t pos_start, const float* inv_freq, int32_t rot,
                        float amplitude, int32_t norm, const void* w_q, const void* w_k, float eps, uint32_t flags, void* dQ, int64_t dq_tok_stride,
                        int64_t dq_head_stride, void* dK, int64_t dk_tok_stride, int64_t dk_head_stride, float* dw_q, float* dw_k, void* workspace,
                        size_t workspace_bytes, void* stream) {
    int rc = check_rotation(M, H, H_kv, d, dt, inv_freq, rot, amplitude, norm, w_q, w_k, eps, flags);
    if (rc != LEMO_OK) return rc;
    if (!small_position(pos_start)) return LEMO_ERR_SHAPE;
    if (norm == LEMO_NORM_NONE && (dw_q || dw_k)) return LEMO_ERR_SHAPE;
    if ((H == 0 && dw_q) || (H_kv == 0 && dw_k)) return LEMO_ERR_SHAPE;
    const bool sums = dw_q || dw_k;
    const int e16 = elems_per_16B(dt);
    if (M > 0) {
        rc = check_heads(dQ_out, dqo_tok_stride, dqo_head_stride, H, e16);
        if (rc == LEMO_OK) rc = check_result(dQ, dq_tok_stride, dq_head_stride, M, H, d, e16);
        if (rc == LEMO_OK) rc = check_heads(dK_out, dko_tok_stride, dko_head_stride, H_kv, e16);
        if (rc == LEMO_OK) rc = check_result(dK, dk_tok_stride, dk_head_stride, M, H_kv, d, e16);
        if (rc == LEMO_OK && norm != LEMO_NORM_NONE) rc = check_heads(Q, q_tok_stride, q_head_stride, H, e16);
        if (rc == LEMO_OK && norm != LEMO_NORM_NONE) rc = check_heads(K, k_tok_stride, k_head_stride, H_kv, e16);
        if (rc != LEMO_OK) return rc;
    } else if (!sums) {
        return LEMO_OK;
    }
    if (sums && !workspace) return LEMO_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(dw_q) & 3u) || (reinterpret_cast<uintptr_t>(dw_k) & 3u)) return LEMO_ERR_ALIGN;
    if (sums && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return LEMO_ERR_ALIGN;
    size_t need = 0;
    lemo_qk_rotate_grad_workspace_bytes(M, H, H_kv, d, dt, flags, &need);
    if (sums && workspace_bytes < need) return LEMO_ERR_WORKSPACE;
    RotateGradParams p{};
    p.side[0] = side(Q, q_tok_stride, q_head_stride, dQ, dq_tok_stride, dq_head_stride, H, w_q, norm, d, flags);
    p.side[1] = side(K, k_tok_stride, k_head_stride, dK, dk_tok_stride, dk_head_stride, H_kv, w_k, norm, d, flags);
    p.dY[0] = dQ_out; p.dY[1] = dK_out;
    p.dy_ts[0] = dqo_tok_stride; p.dy_ts[1] = dko_tok_stride; p.dy_hs[0] = dqo_head_stride; p.dy_hs[1] = dko_head_stride;
    p.positions = positions; p.inv_freq = inv_freq; p.parts = static_cast<float*>(workspace); p.M = M; p.pos_start = pos_start;
    p.d = d; p.rot = rot; p.norm = norm; p.pairs = (flags & LEMO_ROTATE_PAIRS) != 0; p.per_head = (flags & LEMO_WEIGHTS_PER_HEAD) != 0;
    p.eps = eps; p.amplitude = amplitude;
    return hip_rc(launch_qk_rotate_grad(p, dw_q, dw_k, dt, static_cast<hipStream_t>(stream)));
}

int lemo_qk_rotate_step(const void* Q, int64_t q_tok_stride, int64_t q_head_stride, const void* K, int64_t k_tok_stride, int64_t k_head_stride, const void* V,
                        int64_t v_tok_stride, int64_t v_head_stride, int32_t B, int64_t S_max, int32_t H, int32_t H_kv, int32_t d, lemo_dtype_t dt,
                        const int32_t* lengths, const float* inv_freq, int32_t rot, float amplitude, int32_t norm, const void* w_q, const void* w_k, float eps,
                        uint32_t flags, void* Q_out, int64_t qo_tok_stride, int64_t qo_head_stride, void* K_cache, int64_t kc_seq_stride,
                        int64_t kc_tok_stride, int64_t kc_head_stride, void* V_cache, int64_t vc_seq_stride, int64_t vc_tok_stride, int64_t vc_head_stride,
                        void* stream) {
    int rc = check_rotation(B, H, H_kv, d, dt, inv_freq, rot, amplitude, norm, w_q, w_k, eps, flags);
    if (rc != LEMO_OK) return rc;
    if (S_max <= 0 || S_max >= (int64_t)1 << 31 || (V == nullptr) != (V_cache == nullptr)) return LEMO_ERR_SHAPE;
    if (B == 0) return LEMO_OK;
    if (!lengths) return LEMO_ERR_NULL;
    const int e16 = elems_per_16B(dt);
    const int32_t H_v = V ? H_kv : 0;
    rc = check_heads(Q, q_tok_stride, q_head_stride, H, e16);
    if (rc == LEMO_OK) rc = check_result(Q_out, qo_tok_stride, qo_head_stride, B, H, d, e16);
    if (rc == LEMO_OK) rc = check_heads(K, k_tok_stride, k_head_stride, H_kv, e16);
    if (rc == LEMO_OK) rc = check_result(K_cache, kc_tok_stride, kc_head_stride, S_max, H_kv, d, e16, B, kc_seq_stride);
    if (rc == LEMO_OK) rc = check_heads(V, v_tok_stride, v_head_stride, H_v, e16);
    if (rc == LEMO_OK) rc = check_result(V_cache, vc_tok_stride, vc_head_stride, S_max, H_v, d, e16, B, vc_seq_stride);
    if (rc != LEMO_OK) return rc;
    if ((H_kv > 0 && kc_seq_stride < 0) || (H_v > 0 && vc_seq_stride < 0)) return LEMO_ERR_SHAPE;
    if ((H_kv > 0 && kc_seq_stride % e16) || (H_v > 0 && vc_seq_stride % e16) || (reinterpret_cast<uintptr_t>(lengths) & 3u)) return LEMO_ERR_ALIGN;
    RotateParams p{};
    p.side[0] = side(Q, q_tok_stride, q_head_stride, Q_out, qo_tok_stride, qo_head_stride, H, w_q, norm, d, flags);
    p.side[1] = side(K, k_tok_stride, k_head_stride, K_cache, kc_tok_stride, kc_head_stride, H_kv, w_k, norm, d, flags);
    p.side[2] = side(V, v_tok_stride, v_head_stride, V_cache, vc_tok_stride, vc_head_stride, H_v, nullptr, norm, d, flags);
    p.side[1].y_ss = kc_seq_stride;
    p.side[2].y_ss = vc_seq_stride;
    p.lengths = lengths; p.inv_freq = inv_freq; p.M = B; p.S_max = S_max;
    p.d = d; p.rot = rot; p.norm = norm; p.pairs = (flags & LEMO_ROTATE_PAIRS) != 0; p.eps = eps; p.amplitude = amplitude;
    return hip_rc(launch_qk_rotate(p, dt, static_cast<hipStream_t>(stream)));
}

int lemo_dropout_add(const void* Y, int64_t ldy, void* R, int64_t ldr, int64_t S, const int32_t* kept_idx, int64_t M, double p, const uint64_t* rng,
                     uint64_t site, int32_t C, lemo_dtype_t dt, void* stream) {
    return dropout(Y, ldy, R, ldr, S, kept_idx, M, p, rng, site, C, dt, false, stream);
}

int lemo_dropout_add_grad(const void* dR, int64_t lddr, int64_t S, const int32_t* kept_idx, int64_t M, double p, const uint64_t* rng, uint64_t site,
                          void* dY, int64_t lddy, int32_t C, lemo_dtype_t dt, void* stream) {
    return dropout(dR, lddr, dY, lddy, S, kept_idx, M, p, rng, site, C, dt, true, stream);
}

}  // extern "C"
