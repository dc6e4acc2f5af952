// Host side of the norms around a block (lemo.h): argument validation and kernel launches only.
#include <cmath>

#include "api_checks.hpp"
#include "norm_residual.hpp"

using namespace lemo;

namespace {

bool valid_norm(int32_t mode) { return mode == LEMO_NORM_NONE || mode == LEMO_NORM_RMS || mode == LEMO_NORM_LAYER; }

// a [rows, C] operand that is there: its row pitch, then its alignment
int check_rows(const void* p, int64_t ld, int32_t C, int e16) {
    if (!p) return LEMO_OK;
    if (ld < C) return LEMO_ERR_SHAPE;
    return aligned16(p) && ld % e16 == 0 ? LEMO_OK : LEMO_ERR_ALIGN;
}

}  // namespace

extern "C" {

int lemo_norm_residual(const void* Y, int64_t ldy, const void* gate, int64_t ld_gate, void* R, int64_t ldr, int64_t S, const int32_t* kept_idx,
                       int64_t M, const void* w_post, const void* b_post, int32_t post, const void* w_next, const void* b_next, int32_t next,
                       float eps, float residual_scale, float block_scale, void* N, int64_t ldn, float* stats, int32_t C, lemo_dtype_t dt,
                       uint32_t flags, void* stream) {
    if (!valid_dtype(dt)) return LEMO_ERR_DTYPE;
    if (!valid_norm(post) || !valid_norm(next) || (flags & ~(uint32_t)LEMO_GATE_SIGMOID)) return LEMO_ERR_SHAPE;
    if (!(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(residual_scale) || !std::isfinite(block_scale)) return LEMO_ERR_SHAPE;
    if (M == 0) return LEMO_OK;
    if (!R || (next != LEMO_NORM_NONE && !N)) return LEMO_ERR_NULL;
    if (!Y && (gate || post != LEMO_NORM_NONE || next == LEMO_NORM_NONE)) return LEMO_ERR_SHAPE;
    if ((flags & LEMO_GATE_SIGMOID) && !gate) return LEMO_ERR_SHAPE;
    if (S <= 0 || S >= (int64_t)1 << 31 || M < 0 || M > S || C <= 0) return LEMO_ERR_SHAPE;
    const int e16 = elems_per_16B(dt);
    int rc = check_rows(R, ldr, C, e16);
    if (rc == LEMO_OK) rc = check_rows(Y, ldy, C, e16);
    if (rc == LEMO_OK) rc = check_rows(gate, ld_gate == 0 ? C : ld_gate, C, ld_gate == 0 ? 1 : e16);
    if (rc == LEMO_OK && next != LEMO_NORM_NONE) rc = check_rows(N, ldn, C, e16);
    if (rc != LEMO_OK) return rc;
    if (!aligned16(w_post) || !aligned16(b_post) || !aligned16(w_next) || !aligned16(b_next) || !aligned16(stats)) return LEMO_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(kept_idx) & 3u) return LEMO_ERR_ALIGN;
    if (C % e16 || C > NORM_MAX_C) return LEMO_ERR_UNSUPPORTED;
    NormParams p{};
    p.Y = Y; p.gate = gate; p.R = R; p.idx = kept_idx; p.N = N; p.stats = stats;
    p.w_post = w_post; p.b_post = b_post; p.w_next = w_next; p.b_next = b_next;
    p.ldy = ldy; p.ldg = ld_gate; p.ldr = ldr; p.ldn = ldn; p.S = S; p.M = M;
    p.C = C; p.post = post; p.next = next; p.flags = flags;
    p.eps = eps; p.a = residual_scale; p.beta = block_scale;
    return hip_rc(launch_norm_residual(p, dt, static_cast<hipStream_t>(stream)));
}

int lemo_norm_residual_grad_workspace_bytes(int64_t M, int32_t C, size_t* bytes) {
    if (!bytes) return LEMO_ERR_NULL;
    if (M < 0 || M >= (int64_t)1 << 31 || C <= 0) return LEMO_ERR_SHAPE;
    *bytes = round_up((size_t)norm_grad_parts(M, C) * 5 * (size_t)C * sizeof(float), 256);
    return LEMO_OK;
}

int lemo_norm_residual_grad(const void* dN, int64_t lddn, void* dR, int64_t lddr, int64_t S, const void* R, int64_t ldr, const void* Y, int64_t ldy,
                            const void* gate, int64_t ld_gate, const int32_t* kept_idx, int64_t M, const void* w_post, const void* b_post,
                            int32_t post, const void* w_next, int32_t next, float residual_scale, float block_scale, const float* stats, void* dY,
                            int64_t lddy, void* dgate, int64_t ld_dgate, float* dw_post, float* db_post, float* dw_next, float* db_next,
                            float* dgate_sum, int32_t C, lemo_dtype_t dt, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream) {
    if (!valid_dtype(dt)) return LEMO_ERR_DTYPE;
    if (!valid_norm(post) || !valid_norm(next) || (flags & ~(uint32_t)LEMO_GATE_SIGMOID)) return LEMO_ERR_SHAPE;
    if (!std::isfinite(residual_scale) || !std::isfinite(block_scale)) return LEMO_ERR_SHAPE;
    if (S <= 0 || S >= (int64_t)1 << 31 || M < 0 || M > S || C <= 0) return LEMO_ERR_SHAPE;
    const bool sums = dw_post || db_post || dw_next || db_next || dgate_sum;
    if (M > 0) {
        if (!dR || (next != LEMO_NORM_NONE && (!dN || !R)) || ((next != LEMO_NORM_NONE || post != LEMO_NORM_NONE) && !stats)) return LEMO_ERR_NULL;
        if (sums && !workspace) return LEMO_ERR_NULL;
        // what has no gradient: a block, a norm or a gate that is not there; a shared gate's is a sum over the rows
        if (!Y && (gate || post != LEMO_NORM_NONE || dY)) return LEMO_ERR_SHAPE;
        if ((next == LEMO_NORM_NONE && (dw_next || db_next)) || (post == LEMO_NORM_NONE && (dw_post || db_post))) return LEMO_ERR_SHAPE;
        if ((!gate && (dgate || dgate_sum || (flags & LEMO_GATE_SIGMOID))) || (gate && ld_gate == 0 && dgate)) return LEMO_ERR_SHAPE;
    }
    const int e16 = elems_per_16B(dt);
    if (M > 0) {
        int rc = check_rows(dR, lddr, C, e16);
        if (rc == LEMO_OK && next != LEMO_NORM_NONE) rc = check_rows(dN, lddn, C, e16);
        if (rc == LEMO_OK && next != LEMO_NORM_NONE) rc = check_rows(R, ldr, C, e16);
        if (rc == LEMO_OK) rc = check_rows(Y, ldy, C, e16);
        if (rc == LEMO_OK) rc = check_rows(gate, ld_gate == 0 ? C : ld_gate, C, ld_gate == 0 ? 1 : e16);
        if (rc == LEMO_OK) rc = check_rows(dY, lddy, C, e16);
        if (rc == LEMO_OK) rc = check_rows(dgate, ld_dgate, C, e16);
        if (rc != LEMO_OK) return rc;
    }
    if (!aligned16(w_post) || !aligned16(b_post) || !aligned16(w_next) || !aligned16(stats)) return LEMO_ERR_ALIGN;
    for (const float* sum : {dw_post, db_post, dw_next, db_next, dgate_sum})
        if (reinterpret_cast<uintptr_t>(sum) & 3u) return LEMO_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(kept_idx) & 3u) || (sums && (reinterpret_cast<uintptr_t>(workspace) & 255u))) return LEMO_ERR_ALIGN;
    if (C % e16 || C > NORM_MAX_C) return LEMO_ERR_UNSUPPORTED;
    size_t need = 0;
    lemo_norm_residual_grad_workspace_bytes(M, C, &need);
    if (sums && workspace_bytes < need) return LEMO_ERR_WORKSPACE;
    NormGradParams p{};
    p.dN = dN; p.dR = dR; p.R = R; p.Y = Y; p.gate = gate; p.idx = kept_idx; p.stats = stats; p.dY = dY; p.dgate = dgate;
    p.w_post = w_post; p.b_post = b_post; p.w_next = w_next;
    p.lddn = lddn; p.lddr = lddr; p.ldr = ldr; p.ldy = ldy; p.ldg = ld_gate; p.lddy = lddy; p.lddg = ld_dgate; p.S = S; p.M = M;
    p.C = C; p.post = post; p.next = next; p.flags = flags;
    p.a = residual_scale; p.beta = block_scale;
    return hip_rc(launch_norm_residual_grad(p, dw_next, db_next, dw_post, db_post, dgate_sum, workspace, dt, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
