// Operand types and products of the matrix unit that the latent and prompt
// attention share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ordermoe {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

// acc += A B, 16 x 16, for 16 bytes of A's rows and of B's columns per lane: bf16 8 inner
// indexes (8 (lane / 16) .. + 7 of 32), fp32 4 (4 (lane / 16) .. + 3 of 16).  Element i of
// a lane: row 4 (lane / 16) + i, column lane % 16.
template <bool BF>
__device__ inline f32x4 mma16(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (BF) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), acc, 0, 0, 0);
        return acc;
    }
}

// The same for long sums: fp32 in four of them, to be added at the end.  A sum of n products whose signs vary is off by about
// n / 2.4 roundings of a product's size (it grows with the square root of its terms), in four sums by half of that.  fp32 attention
// against 64 bits: 0.6 to 1.9e-6 of the outputs in one sum, 0.3 to 0.7e-6 in four, which take 0 to 3% longer.  (bf16: an
// instruction rounds once for 32 products.)
template <bool BF>
struct LongSum {
    f32x4 part[BF ? 1 : 4] = {};
    __device__ inline void add(u32x4 a, u32x4 b) {
        if constexpr (BF) {
            part[0] = mma16<true>(a, b, part[0]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                part[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), part[i], 0, 0, 0);
        }
    }
    __device__ inline f32x4 sum() const {
        if constexpr (BF) return part[0];
        else return (part[0] + part[1]) + (part[2] + part[3]);
    }
};

// The same, 32 x 32: bf16 8 inner indexes (8 (lane / 32) .. + 7 of 16), fp32 4 (4 (lane / 32) .. + 3
// of 8).  Element i of a lane: row 8 (i / 4) + 4 (lane / 32) + i % 4, column lane % 32.
template <bool BF>
__device__ inline f32x16 mma32(u32x4 a, u32x4 b, f32x16 acc) {
    if constexpr (BF) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), acc, 0, 0, 0);
        return acc;
    }
}

typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(1))) void* glob_ptr;

// 4 x 16 elements of 16 bits in LDS, turned: within each 16 lanes, lane 4 i + j gives the address of
// elements 4 j .. 4 j + 3 of row i and lane c receives column c, rows 0 .. 3.
__device__ inline u32x2 read_turned(const void* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p));
}

// 16 bytes per lane from memory straight into LDS: `to` is uniform, lane i's go to to + 16 i
__device__ inline void load_lds16(const void* from, void* to) {
    __builtin_amdgcn_global_load_lds((glob_ptr)const_cast<void*>(from), (lds_ptr)to, 16, 0, 0);
}

__device__ inline uint32_t bf16_pair(float a, float b) {
    bf16x2 r;
    r[0] = (__bf16)a;
    r[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, r);
}
// 4 values to 8 bytes of bf16 or 16 of fp32
template <bool BF>
__device__ inline void store4(void* base, int64_t at, float a, float b, float c, float d) {
    if constexpr (BF) *(u32x2*)((__bf16*)base + at) = u32x2{bf16_pair(a, b), bf16_pair(c, d)};
    else *(f32x4*)((float*)base + at) = f32x4{a, b, c, d};
}

}  // namespace ordermoe
