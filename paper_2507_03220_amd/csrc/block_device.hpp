// Device helpers shared by the norm and key/value cache kernels: reductions over a wavefront, E4M3 and E8M0.
#pragma once
#include "symb_device.hpp"

namespace symb {

typedef __attribute__((__vector_size__(2 * sizeof(int)))) int intx2;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int intx4;
typedef __attribute__((__vector_size__(8 * sizeof(int)))) int intx8;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float floatx2;

__device__ __forceinline__ float as_float(int v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ int as_int(float v) { return __builtin_bit_cast(int, v); }
__device__ __forceinline__ float bf16_lo(unsigned v) { return as_float((int)(v << 16)); }
__device__ __forceinline__ float bf16_hi(unsigned v) { return as_float((int)(v & 0xffff0000u)); }

// f over the four rows of 16 lanes: every lane gets f of the lanes with its number mod 16.
template <class F>
__device__ __forceinline__ float across_rows(float v, F f) {
    auto a = __builtin_amdgcn_permlane16_swap(as_int(v), as_int(v), false, false);
    v = f(as_float((int)a[0]), as_float((int)a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(as_int(v), as_int(v), false, false);
    return f(as_float((int)b[0]), as_float((int)b[1]));
}
template <int ROR>
__device__ __forceinline__ float row_rotated(float v) {
    return as_float(__builtin_amdgcn_update_dpp(0, as_int(v), 0x120 + ROR, 0xf, 0xf, false));
}
// f over all 64 lanes, in a fixed order; every lane gets it.
template <class F>
__device__ __forceinline__ float across_wave(float v, F f) {
    v = f(v, row_rotated<8>(v));
    v = f(v, row_rotated<4>(v));
    v = f(v, row_rotated<2>(v));
    v = f(v, row_rotated<1>(v));
    return across_rows(v, f);
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// Four fp32 -> four E4M3 bytes, to nearest even (v_cvt_pk_fp8_f32: beyond 464, infinity and NaN become NaN).
__device__ __forceinline__ int pack4_e4m3(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
__device__ __forceinline__ floatx2 e4m3_lo(int v) { return __builtin_bit_cast(floatx2, __builtin_amdgcn_cvt_pk_f32_fp8(v, false)); }
__device__ __forceinline__ floatx2 e4m3_hi(int v) { return __builtin_bit_cast(floatx2, __builtin_amdgcn_cvt_pk_f32_fp8(v, true)); }

// 2^e, -126 <= e <= 127; 0 below.
__device__ __forceinline__ float pow2(int e) { return as_float(max(e + 127, 0) << 23); }
// |v| if it is finite, else 0.
__device__ __forceinline__ float finite_abs(float v) {
    const float a = fabsf(v);
    return a <= 3.402823466e38f ? a : 0.f;
}

}  // namespace symb
