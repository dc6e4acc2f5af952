// Parameter blocks and launchers of the norms and the rotation of queries and keys (qk_rotate.hip).
#pragma once
#include "lemo_common.hpp"

namespace lemo {

// One of the operands: heads of d channels.  Single tokens (lengths given): keys and values go to row lengths[s] - 1 of sequence s of a cache.
struct RotateSide {
    const void* X;
    void* Y;
    const void* w;                         // [d], or [heads, d] (w_hs = d), or null
    long long x_ts, x_hs, y_ts, y_hs, y_ss;  // element strides: token, head, sequence of a cache
    int heads, w_hs;
};
struct RotateParams {
    RotateSide side[3];     // queries, keys, values (copied; single tokens only)
    const int* positions;   // [M] or null
    const int* lengths;     // [M] or null
    const float* inv_freq;  // [rot / 2]
    long long M, pos_start, S_max;
    long long first;        // workgroup of the launch's first one
    int d, rot, norm, pairs, tokens, slots;  // tokens of a workgroup, heads of one; slots: workgroups that share a token's heads
    float eps, amplitude;
};
struct RotateGradParams {
    RotateSide side[2];     // X: the inputs, Y: their gradients
    const void* dY[2];      // gradients of the results
    long long dy_ts[2], dy_hs[2];
    const int* positions;
    const float* inv_freq;
    float* parts;           // [workgroups][2 or heads][d]
    long long M, pos_start;
    int d, rot, norm, pairs, per_head, sums;
    float eps, amplitude;
};

int launch_qk_rotate(RotateParams p, lemo_dtype_t dt, hipStream_t st);
size_t qk_rotate_grad_parts(int64_t M, int heads, int d, lemo_dtype_t dt, bool per_head);  // floats
int launch_qk_rotate_grad(RotateGradParams p, float* dw_q, float* dw_k, lemo_dtype_t dt, hipStream_t st);

}  // namespace lemo
