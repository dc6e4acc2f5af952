// The arithmetic of the loss over a vocabulary, one logit and one row at a time.
#pragma once
#include "vocab_loss.hpp"

namespace lemo {

constexpr float LOG2E = 1.4426950408889634f;

// tanh: from the exponential, but for small arguments, where the difference would lose digits, from its series (next term below 2^-22 of it)
__device__ __forceinline__ float vocab_tanh(float y) {
    const float e = __builtin_amdgcn_exp2f(2.f * LOG2E * y), far = 1.f - 2.f / (e + 1.f);
    const float q = y * y;
    const float near = y * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return q < 0.1f ? near : far;
}
__device__ __forceinline__ float vocab_cap(float x, float softcap, float inv_cap) { return softcap * vocab_tanh(x * inv_cap); }

// 2^(log2(e) (a - b)), and 1 where they are equal, infinities included
__device__ __forceinline__ float vocab_scale(float a, float b) { return a == b ? 1.f : __builtin_amdgcn_exp2f((a - b) * LOG2E); }

// (maximum, sum of exponentials) of two parts of a row.  A maximum of minus infinity goes with a sum of 0.
__device__ __forceinline__ void vocab_join(float& top, float& sum, float top2, float sum2) {
    const float t = fmaxf(top, top2);
    sum = sum * vocab_scale(top, t) + sum2 * vocab_scale(top2, t);
    top = t;
}

// Gradient of a row's logit u (capped) at column v: what the row's probabilities and label leave, times the gradient of its loss.
struct VocabRow { float neg_lse2, factor, weight; int label; bool counts; };
__device__ __forceinline__ VocabRow vocab_row(const VocabRule& r, float lse, float weight, int label) {
    // what rounding lse log2(e) leaves would be an error of all of the row's probabilities: it goes into their factor (lse 10, binary32: 6e-7 of them)
    const float neg = -lse * LOG2E, left = fmaf(-lse, LOG2E, -neg);
    return {neg, fmaf(2.f * r.z, lse, 1.f) * fmaf(left, 0.6931471805599453f, 1.f), weight, label, label >= 0 && label < r.V};
}
// row m of M (idx: of X, or null)
__device__ __forceinline__ VocabRow vocab_row_of(const VocabRule& r, const VocabSide& side, const float* lse, const int* labels, long long m) {
    const int label = labels[m];
    const bool counts = label >= 0 && label < r.V;
    return vocab_row(r, lse[m], !counts ? 0.f : side.ones ? 1.f : side.dloss[m * side.stride], label);
}
__device__ __forceinline__ void vocab_list_row(const VocabRule& r, const VocabSide& side, const int* labels, const int* idx, long long m, long long M) {
    const int label = labels[m];
    side.rows[m] = label >= 0 && label < r.V ? idx ? idx[m] : (int)m : side.past;
    if (m == M - 1) side.rows[M] = side.past;
}
__device__ __forceinline__ float vocab_grad(const VocabRule& r, const VocabRow& row, float u, int v, float inv_cap) {
    float g = fmaf(__builtin_amdgcn_exp2f(fmaf(u, LOG2E, row.neg_lse2)), row.factor, -r.all);
    g = v == row.label ? g - r.hit : g;
    if (r.softcap > 0.f) {
        const float t = u * inv_cap;
        g *= fmaf(-t, t, 1.f);
    }
    return row.counts ? g * row.weight : 0.f;  // (chosen: a row without a label may hold anything)
}

}  // namespace lemo
