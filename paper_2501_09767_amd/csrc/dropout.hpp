// Parameter block and launcher of dropout into the residual rows (dropout.hip).
#pragma once
#include "lemo_common.hpp"

namespace lemo {

struct DropoutParams {
    const void* X;                  // forward: the block's result [M, C]; gradient: that of the residual rows [S, C]
    void* Y;                        // forward: the residual rows [S, C], in place; gradient: that of the block's result [M, C]
    const int* idx;                 // [M] or null
    const unsigned long long* rng;  // seed, stream
    unsigned long long site;        // added to the stream
    long long ldx, ldy, S, M;
    long long first;                // workgroup of the launch's first one
    int C, rows;                    // rows of a workgroup
    unsigned keep16;                // of 65536 values of an element's bits, those that keep it
    float scale;                    // 65536 / keep16
};

int launch_dropout(DropoutParams p, bool grad, lemo_dtype_t dt, hipStream_t st);

}  // namespace lemo
