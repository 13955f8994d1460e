// convert.h -- elements between the input types (f32, bf16) and the storage types
// (f32, bf16, OCP fp8 e4m3fn) of the cache writes (device code).
//
// bf16 rounds to nearest even (NaN kept quiet); e4m3fn from the fp32 quotient
// x / scale (IEEE division), nearest with ties to the even code, saturating at
// +-448 (infinities too), NaN -> 0x7F.
#pragma once

#include "spire_internal.h"

namespace spire {

// fp32 -> OCP e4m3fn code, round to nearest even, saturating.
__device__ __forceinline__ uint8_t f32_to_e4m3fn_sat(float x) {
    const uint32_t u = __float_as_uint(x);
    const uint32_t sign = (u >> 24) & 0x80u;
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7F;  // NaN
    const float a = __uint_as_float(u & 0x7fffffffu);
    if (a >= 448.f) return (uint8_t)(sign | 0x7Eu);
    if (a < 0x1p-6f) {
        // subnormal codes m * 2^-9 (m = 8 is the smallest normal, code 0x08)
        const uint32_t m = (uint32_t)__builtin_rintf(a * 512.f);  // exact scaling, ties to even
        return (uint8_t)(sign | m);
    }
    const uint32_t au = __float_as_uint(a);
    int e = (int)(au >> 23) - 127;        // -6 .. 8
    uint32_t m3 = (au >> 20) & 7u;        // top 3 fraction bits
    const uint32_t rem = au & 0xFFFFFu;   // the 20 bits rounded away
    if (rem > 0x80000u || (rem == 0x80000u && (m3 & 1u))) ++m3;
    if (m3 == 8u) {
        m3 = 0;
        ++e;
    }
    return (uint8_t)(sign | ((uint32_t)(e + 7) << 3) | m3);  // a < 448 never reaches 480
}

// One element, converted from the input representation to storage.
__device__ __forceinline__ float load_new(const void *src, int dtype, int64_t i) {
    if (dtype == SPIRE_BF16) return bf16_to_f32(static_cast<const uint16_t *>(src)[i]);
    return static_cast<const float *>(src)[i];
}

__device__ __forceinline__ void store_elem(uint8_t *row, int es, int d, float x, float scale) {
    if (es == 4) reinterpret_cast<float *>(row)[d] = x;
    else if (es == 2) reinterpret_cast<uint16_t *>(row)[d] = f32_to_bf16_rne(x);
    else row[d] = f32_to_e4m3fn_sat(x / scale);
}

// Four fp32 -> OCP e4m3fn codes, the same rounding: the conversion instruction
// (nearest, ties to even, subnormal codes included) takes values clamped to
// +-448; NaN becomes 0x7F afterwards.
__device__ __forceinline__ uint32_t f32x4_to_e4m3fn_sat(const float q[4]) {
    float c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = fminf(fmaxf(q[i], -448.f), 448.f);
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], v, true);
    uint32_t r = (uint32_t)v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (q[i] != q[i]) r = (r & ~(0xFFu << (8 * i))) | (0x7Fu << (8 * i));
    return r;
}

typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// elements 4q .. 4q+3 of an input row starting at element i0
__device__ __forceinline__ void load_quad(const void *src, int dtype, int64_t i0, float x[4]) {
    if (dtype == SPIRE_BF16) {
        const u32x2v v = *reinterpret_cast<const u32x2v *>(static_cast<const uint16_t *>(src) + i0);
        x[0] = __uint_as_float(v.x << 16);
        x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16);
        x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    } else {
        const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(src) + i0);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    }
}

// store 4 elements at byte `at` (4 * ES-aligned) in the storage representation
template <int ES>
__device__ __forceinline__ void store_quad(uint8_t *at, const float x[4], float scale) {
    if constexpr (ES == 4) {
        *reinterpret_cast<float4 *>(at) = make_float4(x[0], x[1], x[2], x[3]);
    } else if constexpr (ES == 2) {
        u32x2v v;
        v.x = f32_to_bf16_rne(x[0]) | ((uint32_t)f32_to_bf16_rne(x[1]) << 16);
        v.y = f32_to_bf16_rne(x[2]) | ((uint32_t)f32_to_bf16_rne(x[3]) << 16);
        *reinterpret_cast<u32x2v *>(at) = v;
    } else {
        const float q[4] = {x[0] / scale, x[1] / scale, x[2] / scale, x[3] / scale};
        *reinterpret_cast<uint32_t *>(at) = f32x4_to_e4m3fn_sat(q);
    }
}

}  // namespace spire
