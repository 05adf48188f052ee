// The 4-bit format of a compact cache (E2M1 codes, one power-of-two scale per 32 channels, see kv4.hip) on the device, and the host's
// checks of its tensors.
#pragma once

#include "kvcomm_device.h"

namespace kvc {

// Scale byte of a block whose largest magnitude has these bits: the least e with it <= 7 * 2^e, plus 127.  7 = 1.75 * 2^2: a mantissa
// above 1.75 carries into the exponent.  e >= -125 keeps every decoded value a normal bf16; e <= 125 keeps them finite (what lies above 7 * 2^125 saturates).
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t most)
{
    if (most >= 0x7f800000u) return 255;
    const int b = (int)((most + 0x1fffffu) >> 23) - 2;
    return (uint32_t)min(max(b, 2), 252);
}

// The scale as the conversion instructions read it (the exponent field is the byte itself; 255 is a NaN there too).
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// 8 channels -> their codes, channel 2 i in the low half of byte i.
__device__ __forceinline__ uint32_t fp4_encode8(const u32x4 (&raw)[1], float scale)
{
    auto pair = [&](int i) {   // (a bit cast of the vector's element itself would be one of its first element)
        const uint32_t w = raw[0][i];
        return __builtin_bit_cast(bf16x2, w);
    };
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0, pair(0), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(1), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(2), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(3), scale, 3);
}
__device__ __forceinline__ uint32_t fp4_encode8(const u32x4 (&raw)[2], float scale)
{
    auto f = [&](int i) { return __uint_as_float(raw[i >> 2][i & 3]); };
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, f(0), f(1), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f(2), f(3), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f(4), f(5), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f(6), f(7), scale, 3);
}

// 8 codes -> their values, packed bf16 (exact: a code has two significant bits) or fp32.
__device__ __forceinline__ void fp4_decode8(uint32_t codes, float scale, u32x4 (&raw)[1])
{
    raw[0][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    raw[0][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    raw[0][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    raw[0][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
}
__device__ __forceinline__ void fp4_decode8(uint32_t codes, float scale, u32x4 (&raw)[2])
{
    auto put = [&](int i, auto v) {
        raw[i >> 1][2 * (i & 1)] = __float_as_uint(v[0]);
        raw[i >> 1][2 * (i & 1) + 1] = __float_as_uint(v[1]);
    };
    put(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0));
    put(1, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1));
    put(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2));
    put(3, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3));
}

// Rows of codes are moved with 16-byte accesses, the scales of a row (2, 4 or 8 bytes) with one access.
static inline int check_tensor4(const kvcomm_tensor4 &t, int D)
{
    const kvcomm_tensor &c = t.codes, &s = t.scales;
    const int64_t row = D / 32;
    if (!c.ptr || !aligned16(c.ptr) || !s.ptr || reinterpret_cast<uintptr_t>(s.ptr) % row) return KVCOMM_EINVAL;
    for (int64_t stride : {c.stride_layer, c.stride_head, c.stride_token})
        if (stride < 0 || stride % 16) return KVCOMM_EINVAL;
    for (int64_t stride : {s.stride_layer, s.stride_head, s.stride_token})
        if (stride < 0 || stride % row) return KVCOMM_EINVAL;
    return KVCOMM_OK;
}

}  // namespace kvc
