// 16 bytes of a row as binary32 values, for the kernels that work on rows in registers.
#pragma once
#include "lemo_common.hpp"

namespace lemo {

template <typename T> struct RowPiece;
template <> struct RowPiece<bf16_t> {
    static constexpr int E = 8;
    __device__ static __forceinline__ void get(const u32x4& v, float (&x)[E]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo_to_f32(v[i]); x[2 * i + 1] = bf16hi_to_f32(v[i]); }
    }
    __device__ static __forceinline__ u32x4 put(const float (&x)[E]) {
        return u32x4{pack_bf16x2_hw(x[0], x[1]), pack_bf16x2_hw(x[2], x[3]), pack_bf16x2_hw(x[4], x[5]), pack_bf16x2_hw(x[6], x[7])};
    }
};
template <> struct RowPiece<float> {
    static constexpr int E = 4;
    __device__ static __forceinline__ void get(const u32x4& v, float (&x)[E]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
    }
    __device__ static __forceinline__ u32x4 put(const float (&x)[E]) {
        return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};
template <typename T> __device__ __forceinline__ u32x4 row_load(const void* base, long long element) {
    return *reinterpret_cast<const u32x4*>(static_cast<const char*>(base) + element * (long long)(16 / RowPiece<T>::E));
}
template <typename T> __device__ __forceinline__ void row_store(void* base, long long element, const u32x4& v) {
    *reinterpret_cast<u32x4*>(static_cast<char*>(base) + element * (long long)(16 / RowPiece<T>::E)) = v;
}

}  // namespace lemo
