// Parameter blocks and launchers of the norms around a block (norm_residual.hip).
#pragma once
#include "lemo_common.hpp"

namespace lemo {

struct NormParams {
    const void* Y;     // [M, C] or null
    const void* gate;  // [M, C], one row for all (ldg 0), or null
    void* R;           // [S, C], rows idx in place
    const int* idx;    // [M] or null
    const void *w_post, *b_post, *w_next, *b_next;  // [C] each or null
    void* N;           // [M, C]
    float* stats;      // [M, 4]: mean and 1 / deviation of post, of next; or null
    long long ldy, ldg, ldr, ldn, S, M;
    long long first;   // workgroup of the launch's first one
    int C, post, next;
    unsigned flags;
    float eps, a, beta;
};

struct NormGradParams {
    const void* dN;
    void* dR;
    const void *R, *Y, *gate;
    const int* idx;
    const void *w_post, *b_post, *w_next;
    const float* stats;
    void *dY, *dgate;  // dgate: of a gate with rows of its own
    float* parts;      // [workgroups][planes][C]
    long long lddn, lddr, ldr, ldy, ldg, lddy, lddg, S, M;
    int C, post, next, sums, planes;
    unsigned flags;
    float a, beta;
};

struct NormSums { float* to[5]; };

constexpr int NORM_MAX_C = 16384;  // what the threads of a workgroup hold of a row in registers

int launch_norm_residual(const NormParams& p, lemo_dtype_t dt, hipStream_t st);
int norm_grad_parts(int64_t M, int C);  // workgroups of the gradient, each with a part of the column sums
int launch_norm_residual_grad(NormGradParams p, float* dw_next, float* db_next, float* dw_post, float* db_post, float* dgate_sum, void* workspace,
                              lemo_dtype_t dt, hipStream_t st);

}  // namespace lemo
