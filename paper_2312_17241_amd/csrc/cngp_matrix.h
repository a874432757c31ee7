// Operands of 32 x 32 x 16 products on the matrix cores, for fp16 and fp32 values, and how an fp32 value becomes two fp16 ones.  (Linear attention,
// orthogonalised updates.)  Sums: lane l holds column l % 32; its register 4 g + e is row 8 g + 4 (l / 32) + e.
#pragma once
#include <hip/hip_runtime.h>

namespace cngp {
namespace mat {

typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float    float8_t __attribute__((ext_vector_type(8)));
typedef float    float4_t __attribute__((ext_vector_type(4)));
typedef float    acc_t __attribute__((ext_vector_type(16)));

template <typename T> struct Types;
template <> struct Types<_Float16> { using frag = half8_t; static constexpr int vec = 8, pad = 8; };
template <> struct Types<float> { using frag = float8_t; static constexpr int vec = 4, pad = 4; };
template <typename T> using frag_t = typename Types<T>::frag;

__device__ __forceinline__ acc_t zero() {
    acc_t z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.0f;
    return z;
}
// Sixteen steps of a contraction: lane l holds eight of them for row (column) l % 32, which ones is the same for a and b.
__device__ __forceinline__ acc_t mfma(const half8_t a, const half8_t b, const acc_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ acc_t mfma(const float8_t a, const float8_t b, acc_t c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// Eight neighbouring values; or four and the four that lie eight further on (the order of the state's registers).
__device__ __forceinline__ half8_t read8(const _Float16 *p) { return *reinterpret_cast<const half8_t *>(p); }
__device__ __forceinline__ float8_t read8(const float *p) {
    return __builtin_shufflevector(*reinterpret_cast<const float4_t *>(p), *reinterpret_cast<const float4_t *>(p + 4), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ half8_t read4_4(const _Float16 *p) {
    return __builtin_shufflevector(*reinterpret_cast<const half4_t *>(p), *reinterpret_cast<const half4_t *>(p + 8), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float8_t read4_4(const float *p) {
    return __builtin_shufflevector(*reinterpret_cast<const float4_t *>(p), *reinterpret_cast<const float4_t *>(p + 8), 0, 1, 2, 3, 4, 5, 6, 7);
}
// Column `col0 + lane % 32`, rows row0 + 8 (lane / 32) .. + 7 of a tile in LDS.
__device__ __forceinline__ half8_t read_column(const _Float16 *tile, const int stride, const int row0, const int col0, const int lane) {
    typedef short short4_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4_t LdsShort4;
    const int i = lane & 15;      // the transposing read: lane i of a group of 16 gets column i of four rows that the lanes 4q .. 4q + 3 name
    const _Float16 *p = tile + (row0 + 8 * (lane >> 5) + (i >> 2)) * stride + col0 + (lane & 16) + 4 * (i & 3);
    const half4_t lo = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)p));
    const half4_t hi = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(p + 4 * stride)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float8_t read_column(const float *tile, const int stride, const int row0, const int col0, const int lane) {
    const float *p = tile + (row0 + 8 * (lane >> 5)) * stride + col0 + (lane & 31);
    float8_t v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i * stride];
    return v;
}

constexpr float kLow = 2048.0f;         // the low parts are kept scaled by this: they have the range of the high ones

// x * scale as a high and a low part.
__device__ __forceinline__ void split(const float (&x)[8], const float scale, half8_t &hi, half8_t &lo) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = x[i] * scale;
        hi[i] = (_Float16)y;
        lo[i] = (_Float16)((y - (float)hi[i]) * kLow);
    }
}

}  // namespace mat
}  // namespace cngp
