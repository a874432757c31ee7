// Operands of 32 x 32 x 16 products on the matrix cores, for fp16 and fp32 values, and how an fp32 value becomes two fp16 ones.  (Linear attention,
// orthogonalised updates.)  Sums: lane l holds column l % 32; its register 4 g + e is row 8 g + 4 (l / 32) + e.
#pragma once
#include <hip/hip_runtime.h>

namespace cngp {
namespace mat {

typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float    float4_t __attribute__((ext_vector_type(4)));
typedef float    acc_t __attribute__((ext_vector_type(16)));
typedef unsigned words_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ acc_t zero() {
    acc_t z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.0f;
    return z;
}
// Sixteen steps of a contraction: lane l holds eight of them for row (column) l % 32, which ones is the same for a and b.
__device__ __forceinline__ acc_t mfma(const half8_t a, const half8_t b, const acc_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// Eight neighbouring values; or four and the four that lie eight further on (the order of sums that are used as an operand).
__device__ __forceinline__ half8_t read8(const _Float16 *p) { return *reinterpret_cast<const half8_t *>(p); }
__device__ __forceinline__ half8_t read4_4(const _Float16 *p) {
    return __builtin_shufflevector(*reinterpret_cast<const half4_t *>(p), *reinterpret_cast<const half4_t *>(p + 8), 0, 1, 2, 3, 4, 5, 6, 7);
}
// Column col0 + lane % 32 of a tile in LDS, rows row0 + 8 (lane / 32) .. + 7; SUMS: row0 + 4 (lane / 32) .. + 3 and the four eight further on.
template <bool SUMS = false>
__device__ __forceinline__ half8_t read_column(const _Float16 *tile, const int stride, const int row0, const int col0, const int lane) {
    typedef short short4_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4_t LdsShort4;
    const int i = lane & 15;      // the transposing read: lane i of a group of 16 gets column i of four rows that the lanes 4q .. 4q + 3 name
    const _Float16 *p = tile + (row0 + (SUMS ? 4 : 8) * (lane >> 5) + (i >> 2)) * stride + col0 + (lane & 16) + 4 * (i & 3);
    const half4_t lo = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)p));
    const half4_t hi = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(p + (SUMS ? 8 : 4) * stride)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// x * scale as a high and a low part.  Subnormal parts are kept: what is lost is half of 2^-24, 2^-38 of the largest value where that has been lifted to
// 2^13 (lift_of).  (As a product and sum the low part is one instruction, as a difference three.)
__device__ __forceinline__ void split(const float (&x)[8], const float scale, half8_t &hi, half8_t &lo) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi[i] = (_Float16)(x[i] * scale);
        lo[i] = (_Float16)fmaf(x[i], scale, -(float)hi[i]);
    }
}

// wave_top: the largest of a wavefront's magnitudes, as bits.  lift_of: exponent of the power of two that brings it to 2^13 .. 2^14 (0 where it is 0 or
// not finite), within +-`most`.
template <int CTRL>
__device__ __forceinline__ float max_moved(const float v) {
    return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true)));
}
__device__ __forceinline__ int lift_from(const uint32_t top, const int most) {
    const int e = (int)(top >> 23) - 127, lift = 13 - e;
    return top == 0 || e > 127 ? 0 : lift > most ? most : lift < -most ? -most : lift;
}
__device__ __forceinline__ uint32_t wave_top(float v) {
    v = max_moved<0x121>(max_moved<0x122>(max_moved<0x124>(max_moved<0x128>(v))));      // rows of 16 lanes turned by 8, 4, 2, 1
    uint32_t top = 0;
#pragma unroll
    for (int r = 0; r < 64; r += 16) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), r);
        top = top > o ? top : o;
    }
    return top;
}
__device__ __forceinline__ int lift_of(const float v, const int most = 120) { return lift_from(wave_top(v), most); }
// ... of LANES lanes side by side, for each of them.
template <int LANES>
__device__ __forceinline__ int lift_of_lanes(float v) {
    v = max_moved<0xB1>(v);                                 // neighbours; pairs; halves of eight; of sixteen
    if (LANES > 2) v = max_moved<0x4E>(v);
    if (LANES > 4) v = max_moved<0x141>(v);
    if (LANES > 8) v = max_moved<0x140>(v);
    return lift_from(__float_as_uint(v), 100);
}
__device__ __forceinline__ float power_of_two(const int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Nothing is scheduled across: operand reads hoisted into earlier stages cost registers until they spill.
__device__ __forceinline__ void apart() { __builtin_amdgcn_sched_barrier(0); }

// The same value, which the compiler takes for another one: what is computed from it in a loop is computed there, and not before it and kept in
// registers.  (Conditions on the entries of a tile are two scalar registers each.)
__device__ __forceinline__ int anew(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

}  // namespace mat
}  // namespace cngp
