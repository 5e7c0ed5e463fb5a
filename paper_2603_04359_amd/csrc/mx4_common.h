// MXFP4 helpers shared by the kernels that write the format: the scale byte
// of a block of 32 values and the conversion of eight of them.
#pragma once

#include "device_common.h"

namespace catk {

constexpr int kMxBlock = 32;               // elements per scale
constexpr int kMxByteNan = 255;            // E8M0 byte of a NaN scale
constexpr int kMxByteOne = 127;            // E8M0 byte of 2^0

// The E8M0 byte of a block from the bits of its largest magnitude: the
// biased exponent field is floor(log2 amax) + 127 (0 for zero and subnormal
// magnitudes, 255 for NaN and infinity, whose bits exceed every finite
// value's), less the element format's largest exponent 2, at least 0.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return e == 255u ? static_cast<uint32_t>(kMxByteNan) : (e > 2u ? e - 2u : 0u);
}

// 2^(127 - byte): a normal fp32 for every byte mx4_scale_byte gives but 255
// (0: 2^127; 252: 2^-125), so the division by the scale is one exact product
// (a quotient below 2^-126 becomes 0 as it would in E2M1 anyway).
__device__ __forceinline__ float mx4_inverse_scale(uint32_t byte) {
    return __uint_as_float((254u - byte) << 23);
}

// 2^(byte - 127) in fp32 (byte 0 is the subnormal 2^-127), NaN for 255.
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
    return byte == 0u ? __uint_as_float(0x00400000u)
                      : __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23);
}

// Eight scaled values to E2M1 codes, the first in the low nibble (ties to
// even, saturating at 6: v_cvt_scalef32_pk_fp4_f32 with a scale of 1).
__device__ __forceinline__ uint32_t mx4_encode8(const float* v, float inv) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * inv, v[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * inv, v[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * inv, v[5] * inv, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * inv, v[7] * inv, 1.0f, 3);
    return w;
}

// Largest of a value over groups of four consecutive lanes (quad_perm DPP).
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = static_cast<uint32_t>(
        __builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
    v = o > v ? o : v;
    o = static_cast<uint32_t>(
        __builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
    return o > v ? o : v;
}

// fp32 to bf16 bits, ties to even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, p);
}

// Eight consecutive elements at p (16-byte aligned) as fp32.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* v);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* v) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
    }
}
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float* v) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
}

// Eight consecutive elements to p (16-byte aligned), rounded to T.
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v);
template <>
__device__ __forceinline__ void store8<float>(float* p, const float* v) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
}
template <>
__device__ __forceinline__ void store8<uint16_t>(uint16_t* p, const float* v) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                                         pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}

}  // namespace catk
