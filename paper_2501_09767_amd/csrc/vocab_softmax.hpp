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

// What the gradient of a row's logits takes of the row: the probabilities' factor, smoothing's share and the label's, all times the gradient of its loss.
struct VocabRow { float neg_lse2, factor, all, hit; int label; bool counts; };
// row m
__device__ __forceinline__ VocabRow vocab_row_of(const VocabRule& r, const VocabSide& side, const float* lse, const int* labels, long long m) {
    const int label = labels[m];
    const bool counts = label >= 0 && label < r.V;
    const float weight = !counts ? 0.f : side.uniform != 0.f ? side.uniform : side.dloss[m * side.stride];
    // what rounding lse log2(e) leaves would be an error of all of the row's probabilities: it goes into their factor (lse 10, binary32: 6e-7 of them)
    const float neg = -lse[m] * LOG2E, left = fmaf(-lse[m], LOG2E, -neg);
    return {neg, weight * fmaf(2.f * r.z, lse[m], 1.f) * fmaf(left, 0.6931471805599453f, 1.f), weight * r.all, weight * r.hit, label, counts};
}
// Gradient of its logit u (capped) at a column that is not its label's, and at its label's.  A row that does not count may hold anything: what comes of it is
// replaced by zeros.
__device__ __forceinline__ float vocab_slope(const VocabRule& r, float g, float u, float inv_cap) {
    const float t = u * inv_cap;
    return r.softcap > 0.f ? g * fmaf(-t, t, 1.f) : g;
}
__device__ __forceinline__ float vocab_share(const VocabRow& row, float u) { return fmaf(__builtin_amdgcn_exp2f(fmaf(u, LOG2E, row.neg_lse2)), row.factor, -row.all); }
__device__ __forceinline__ float vocab_grad(const VocabRule& r, const VocabRow& row, float u, bool hit, float inv_cap) {
    const float g = vocab_share(row, u);
    return vocab_slope(r, hit ? g - row.hit : g, u, inv_cap);
}
__device__ __forceinline__ void vocab_list_row(const VocabRule& r, const VocabSide& side, const int* labels, const int* idx, long long m, long long M) {
    const int label = labels[m];
    const int row = label >= 0 && label < r.V ? idx ? idx[m] : (int)m : side.past;
    for (int part = 0; part < side.parts; ++part) side.rows[part * M + m] = row;
    if (m == M - 1) side.rows[side.parts * M] = side.past;
}

}  // namespace lemo
