// Codes of the quantised cache: 8-bit elements and the conversions between
// them and the compute types.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.hpp"

namespace ordermoe {

typedef __bf16 kv_bf16x2 __attribute__((ext_vector_type(2)));

template <int FMT>
constexpr float kv_code_max() { return FMT == ORDERMOE_CACHE_INT8 ? 127.f : 448.f; }

// rows of a smaller largest magnitude are stored as zeros: well above where
// the scale would lose bits to fp32's smallest exponent
constexpr float KV_TINY = 0x1p-100f;

// byte B of w as fp32
template <int FMT, int B>
__device__ inline float kv_to_f32(uint32_t w) {
    if constexpr (FMT == ORDERMOE_CACHE_INT8) return (float)(int8_t)(w >> (8 * B));
    else return __builtin_amdgcn_cvt_f32_fp8((int)w, B);
}

__device__ inline uint32_t kv_bf16_pair(float a, float b) {
    kv_bf16x2 r;
    r[0] = (__bf16)a;
    r[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, r);
}

// bytes 2H and 2H + 1 of w as a pair of bf16 (every code is a bf16 value)
template <int FMT, int H>
__device__ inline uint32_t kv_to_bf16x2(uint32_t w) {
    if constexpr (FMT == ORDERMOE_CACHE_INT8) return kv_bf16_pair(kv_to_f32<FMT, 2 * H>(w), kv_to_f32<FMT, 2 * H + 1>(w));
    else return __builtin_bit_cast(uint32_t, (kv_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, H != 0));
}

// four values in [-max, max] to codes
template <int FMT>
__device__ inline uint32_t kv_to_codes(float a, float b, float c, float d) {
    if constexpr (FMT == ORDERMOE_CACHE_INT8) {
        // 1.5 2^23 + y rounds y to the nearest integer, ties to even, and its low byte is the code
        const uint32_t m[4] = {__float_as_uint(a + 0x1.8p23f), __float_as_uint(b + 0x1.8p23f), __float_as_uint(c + 0x1.8p23f),
                               __float_as_uint(d + 0x1.8p23f)};
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(m[3], m[2], 0x0c0c0400u), __builtin_amdgcn_perm(m[1], m[0], 0x0c0c0400u),
                                     0x05040100u);
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
}

}  // namespace ordermoe
