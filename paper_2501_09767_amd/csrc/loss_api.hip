// Host side of the loss over a vocabulary (lemo.h): argument validation and kernel launches only.
#include <cmath>

#include "api_checks.hpp"
#include "vocab_loss.hpp"

using namespace lemo;

namespace {

constexpr int64_t MOST_ROWS = (int64_t)1 << 22;
constexpr int32_t MOST_WORDS = 1 << 21, MOST_WIDTH = 1 << 16;  // (launches below 2^32 threads)

int check_sizes(int64_t M, int32_t C, int32_t V, lemo_dtype_t dt) {
    if (!valid_dtype(dt)) return LEMO_ERR_DTYPE;
    if (M < 0 || C <= 0 || V <= 0) return LEMO_ERR_SHAPE;
    return M > MOST_ROWS || V > MOST_WORDS || C > MOST_WIDTH || C % elems_per_16B(dt) ? LEMO_ERR_UNSUPPORTED : LEMO_OK;
}

bool valid_rule(float softcap, float smoothing, float z_weight) {
    return std::isfinite(softcap) && softcap >= 0.f && (softcap == 0.f || std::isfinite(1.f / softcap)) && smoothing >= 0.f && smoothing <= 1.f && std::isfinite(z_weight);
}
VocabRule rule_of(float softcap, float smoothing, float z_weight, int32_t V) { return {softcap, 1.f - smoothing, smoothing / (float)V, z_weight, V}; }

// X, W and the lists, of both calls
int check_operands(const void* X, int64_t S, int64_t ldx, const int32_t* kept_idx, int64_t M, const void* W, int64_t ldw, int32_t C, lemo_dtype_t dt,
                   const int32_t* labels) {
    const int64_t esz = dt == LEMO_BF16 ? 2 : 4, e16 = elems_per_16B(dt);
    if (!X || !W || !labels) return LEMO_ERR_NULL;
    if (S <= 0 || S >= (int64_t)1 << 31 || ldx < C || ldw < C || (!kept_idx && M > S)) return LEMO_ERR_SHAPE;
    if (!aligned16(X) || !aligned16(W) || ldx % e16 || ldw % e16) return LEMO_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(kept_idx) & 3u) || (reinterpret_cast<uintptr_t>(labels) & 3u)) return LEMO_ERR_ALIGN;
    // pitches and the span of X within the loads' 32-bit offsets, with room for a row past its end and a tile's last columns
    if (ldx * esz >= (int64_t)1 << 23 || ldw * esz >= (int64_t)1 << 23 || (S + 1) * ldx * esz + 4096 > (int64_t)1 << 32) return LEMO_ERR_UNSUPPORTED;
    return LEMO_OK;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

extern "C" {

int lemo_vocab_loss_workspace_bytes(int64_t M, int32_t C, int32_t V, lemo_dtype_t dt, size_t* bytes) {
    if (!bytes) return LEMO_ERR_NULL;
    const int rc = check_sizes(M, C, V, dt);
    if (rc == LEMO_OK) *bytes = vocab_loss_workspace(M, C, V, dt);
    return rc;
}

int lemo_vocab_loss(const void* X, int64_t S, int64_t ldx, const int32_t* kept_idx, int64_t M, const void* W, int64_t ldw, int32_t C, int32_t V,
                    lemo_dtype_t dt, const int32_t* labels, float softcap, float smoothing, float z_weight, float* loss, float* lse, float* total,
                    void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(M, C, V, dt);
    if (rc != LEMO_OK) return rc;
    if (!valid_rule(softcap, smoothing, z_weight)) return LEMO_ERR_SHAPE;
    if (!aligned4(loss) || !aligned4(lse) || !aligned4(total)) return LEMO_ERR_ALIGN;
    if (M > 0) {
        rc = check_operands(X, S, ldx, kept_idx, M, W, ldw, C, dt, labels);
        if (rc != LEMO_OK) return rc;
        if (!loss || !lse || !workspace) return LEMO_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 255u) return LEMO_ERR_ALIGN;
        if (workspace_bytes < vocab_loss_workspace(M, C, V, dt)) return LEMO_ERR_WORKSPACE;
    }
    VocabLossParams p{};
    p.X = X; p.W = W; p.idx = kept_idx; p.labels = labels; p.S = S; p.ldx = ldx; p.ldw = ldw; p.M = M; p.C = C;
    p.rule = rule_of(softcap, smoothing, z_weight, V);
    p.loss = loss; p.lse = lse; p.total = total; p.workspace = workspace;
    return hip_rc(launch_vocab_loss(p, dt, static_cast<hipStream_t>(stream)));
}

int lemo_vocab_loss_grad_workspace_bytes(int64_t M, int32_t C, int32_t V, int64_t ldw, lemo_dtype_t dt, int32_t piece, size_t* bytes) {
    if (!bytes) return LEMO_ERR_NULL;
    int rc = check_sizes(M, C, V, dt);
    if (rc != LEMO_OK) return rc;
    if (ldw < C || piece < 0) return LEMO_ERR_SHAPE;
    const int cols = vocab_piece(M, C, V, ldw, piece, dt);
    if (cols == 0) return LEMO_ERR_UNSUPPORTED;
    *bytes = vocab_grad_workspace(M, C, V, cols, dt);
    return LEMO_OK;
}

int lemo_vocab_loss_grad(const float* dloss, int64_t dloss_stride, const void* X, int64_t S, int64_t ldx, const int32_t* kept_idx, int64_t M, const void* W,
                         int64_t ldw, int32_t C, int32_t V, lemo_dtype_t dt, const int32_t* labels, const float* lse, float softcap, float smoothing,
                         float z_weight, void* dX, int64_t lddx, void* dW, int64_t lddw, int32_t piece, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(M, C, V, dt);
    if (rc != LEMO_OK) return rc;
    if (!valid_rule(softcap, smoothing, z_weight) || (dloss_stride != 0 && dloss_stride != 1) || piece < 0) return LEMO_ERR_SHAPE;
    const int64_t esz = dt == LEMO_BF16 ? 2 : 4, e16 = elems_per_16B(dt);
    if ((dX && lddx < C) || (dW && lddw < C)) return LEMO_ERR_SHAPE;
    if (!aligned16(dX) || !aligned16(dW) || (dX && lddx % e16) || (dW && lddw % e16)) return LEMO_ERR_ALIGN;
    if (dW && lddw * esz >= (int64_t)1 << 23) return LEMO_ERR_UNSUPPORTED;
    if (dX && dt == LEMO_F32 && (M + 63) * C * esz >= (int64_t)1 << 32) return LEMO_ERR_UNSUPPORTED;  // (a plane's 32-bit offsets)
    int cols = 0;
    if (M > 0) {
        rc = check_operands(X, S, ldx, kept_idx, M, W, ldw, C, dt, labels);
        if (rc != LEMO_OK) return rc;
        cols = vocab_piece(M, C, V, ldw, piece, dt);
        if (cols == 0) return LEMO_ERR_UNSUPPORTED;
        if (!dloss || !lse || !workspace) return LEMO_ERR_NULL;
        if (!aligned4(dloss) || !aligned4(lse) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return LEMO_ERR_ALIGN;
        if (workspace_bytes < vocab_grad_workspace(M, C, V, cols, dt)) return LEMO_ERR_WORKSPACE;
    }
    VocabGradParams p{};
    p.X = X; p.W = W; p.idx = kept_idx; p.labels = labels; p.S = S; p.ldx = ldx; p.ldw = ldw; p.M = M; p.C = C;
    p.rule = rule_of(softcap, smoothing, z_weight, V);
    p.lse = lse; p.dloss = dloss; p.dloss_stride = dloss_stride; p.dX = dX; p.dW = dW; p.lddx = lddx; p.lddw = lddw; p.piece = cols; p.workspace = workspace;
    return hip_rc(launch_vocab_grad(p, dt, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
