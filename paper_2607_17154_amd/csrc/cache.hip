// The quantised paged cache: a step's rows written, rows read back.
//
//   cache_write_kernel  every head row (query, key or value head of a token) by
//                       16 lanes, D / 16 neighbouring elements each: RMS norm
//                       (sum of squares over the 16 lanes), rotation, then
//                       queries rounded and stored, keys and values scaled by
//                       their largest magnitude and stored as codes
//   cache_read_kernel   a row of codes by 16 lanes: code * scale
// Both read and write every byte once; the memory bounds them.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "kv_codes.hpp"

namespace ordermoe {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int CW_THREADS = 256;
constexpr int CW_ROWS = CW_THREADS / 16;     // head rows per block

// reductions over the 16 lanes of a DPP row, by rotations of 8, 4, 2, 1; every
// lane ends with the same bits (each step adds the same two values in both lanes)
template <int CTRL>
__device__ inline uint32_t ror(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false); }
__device__ inline float row_sum(float v) {
    v += __uint_as_float(ror<0x128>(__float_as_uint(v)));
    v += __uint_as_float(ror<0x124>(__float_as_uint(v)));
    v += __uint_as_float(ror<0x122>(__float_as_uint(v)));
    v += __uint_as_float(ror<0x121>(__float_as_uint(v)));
    return v;
}
__device__ inline uint32_t row_max(uint32_t v) {
    uint32_t o;
    o = ror<0x128>(v); v = o > v ? o : v;
    o = ror<0x124>(v); v = o > v ? o : v;
    o = ror<0x122>(v); v = o > v ? o : v;
    o = ror<0x121>(v); v = o > v ? o : v;
    return v;
}

// N neighbouring elements of storage T as fp32, and back
template <typename T, int N>
__device__ inline void load_f32(const T* p, float* x) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const u32x4 v = ((const u32x4*)p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = __uint_as_float(v[j]);
        }
    } else {
        uint32_t w[N / 2];
        if constexpr (N == 4) {
            const u32x2 v = *(const u32x2*)p;
            w[0] = v[0]; w[1] = v[1];
        } else {
#pragma unroll
            for (int i = 0; i < N / 8; ++i) {
                const u32x4 v = ((const u32x4*)p)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
            }
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}
template <typename T, int N>
__device__ inline void store_f32(T* p, const float* x) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(x[4 * i + j]);
            ((u32x4*)p)[i] = v;
        }
    } else {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            kv_bf16x2 r;
            r[0] = (__bf16)x[2 * i];
            r[1] = (__bf16)x[2 * i + 1];
            w[i] = __builtin_bit_cast(uint32_t, r);
        }
        if constexpr (N == 4) {
            *(u32x2*)p = u32x2{w[0], w[1]};
        } else {
#pragma unroll
            for (int i = 0; i < N / 8; ++i) ((u32x4*)p)[i] = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
        }
    }
}
template <int N>
__device__ inline void load_codes(const uint8_t* p, uint32_t* w) {
    if constexpr (N == 4) {
        w[0] = *(const uint32_t*)p;
    } else if constexpr (N == 8) {
        const u32x2 v = *(const u32x2*)p;
        w[0] = v[0]; w[1] = v[1];
    } else {
        const u32x4 v = *(const u32x4*)p;
        w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; w[3] = v[3];
    }
}
template <int N>
__device__ inline void store_codes(uint8_t* p, const uint32_t* w) {
    if constexpr (N == 4) *(uint32_t*)p = w[0];
    else if constexpr (N == 8) *(u32x2*)p = u32x2{w[0], w[1]};
    else *(u32x4*)p = u32x4{w[0], w[1], w[2], w[3]};
}

// row of (slot, head) in codes; a slot's scale index is the same without D
__device__ inline int64_t cache_row(const CacheArgs& c, int64_t slot, int h) {
    return (((slot >> c.page_shift) * c.n_kv + h) << c.page_shift) + (slot & (((int64_t)1 << c.page_shift) - 1));
}

template <typename T, int D, int FMT>
__global__ void __launch_bounds__(CW_THREADS) cache_write_kernel(const CacheWriteArgs a) {
    constexpr int N = D / 16;                                   // elements per lane
    const int c = threadIdx.x & 15;
    const uint32_t heads = (uint32_t)(a.n_q + 2 * a.cache.n_kv);
    const uint32_t row = blockIdx.x * CW_ROWS + (threadIdx.x >> 4);
    if (row >= (uint32_t)a.T * heads) return;                   // whole rows leave together
    const int64_t t = row / heads;
    const int h = (int)(row - (uint32_t)t * heads);
    const int kind = h < a.n_q ? 0 : h < a.n_q + a.cache.n_kv ? 1 : 2;      // query, key, value
    const int hk = h - a.n_q - (kind == 2 ? a.cache.n_kv : 0);
    const T* src = kind == 0 ? (const T*)a.q + t * a.q_stride + h * D
                             : (kind == 1 ? (const T*)a.k + t * a.k_stride : (const T*)a.v + t * a.v_stride) + hk * D;
    float x[N];
    load_f32<T, N>(src + c * N, x);
    const T* nw = (const T*)(kind == 0 ? a.q_norm : kind == 1 ? a.k_norm : nullptr);
    if (nw) {
        float w[N], s = 0.f;
        load_f32<T, N>(nw + c * N, w);
#pragma unroll
        for (int i = 0; i < N; ++i) s = fmaf(x[i], x[i], s);
        const float r = 1.0f / sqrtf(row_sum(s) * (1.0f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = x[i] * r * w[i];
    }
    if (kind != 2 && a.rot) {
        const int half = a.rot / 2, p = a.pos[t];
        const bool in = p >= 0 && (int64_t)p < a.max_pos;
        const float* cs = a.cos_sin + (int64_t)(in ? p : 0) * a.rot;
        const float nan = __builtin_nanf("");
        if (a.interleaved) {
            const int i0 = c * (N / 2);                         // first pair of the lane
            if (i0 < half) {
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    const float co = in ? cs[i0 + i] : nan, si = in ? cs[half + i0 + i] : nan;
                    const float u = x[2 * i], v = x[2 * i + 1];
                    x[2 * i] = u * co - v * si;
                    x[2 * i + 1] = v * co + u * si;
                }
            }
        } else {
            // the partner of element i is i +- half, `half / N` lanes away (whole lanes, since half is a multiple of N)
            const int dl = half / N;
            const bool lo = c < dl, turned = c < 2 * dl;
            const int from = turned ? (lo ? c + dl : c - dl) : c;
            const int i0 = turned ? (lo ? c : c - dl) * N : 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float o = __shfl(x[i], from, 16);
                const float co = in ? cs[i0 + i] : nan, si = in ? cs[half + i0 + i] : nan;
                const float y = lo ? x[i] * co - o * si : x[i] * co + o * si;
                x[i] = turned ? y : x[i];
            }
        }
    }
    if (kind == 0) {
        store_f32<T, N>((T*)a.q_out + (t * a.n_q + h) * D + c * N, x);
        return;
    }
    // the largest magnitude on the bits, where a NaN is larger than infinity
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        big = b > big ? b : big;
    }
    big = row_max(big);
    const bool bad = big >= 0x7F800000u, none = __uint_as_float(big) < KV_TINY;
    const float scale = bad ? __builtin_nanf("") : none ? 0.f : __uint_as_float(big) / kv_code_max<FMT>();
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        w[i] = 0u;
        if (!bad && !none) {
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                y[j] = __builtin_amdgcn_fmed3f(x[4 * i + j] / scale, -kv_code_max<FMT>(), kv_code_max<FMT>());
            w[i] = kv_to_codes<FMT>(y[0], y[1], y[2], y[3]);
        }
    }
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= (a.cache.n_pages << a.cache.page_shift)) return;
    const int64_t at = cache_row(a.cache, slot, hk);
    store_codes<N>((kind == 1 ? a.cache.k_codes : a.cache.v_codes) + at * D + c * N, w);
    if (c == 0) (kind == 1 ? a.cache.k_scale : a.cache.v_scale)[at] = scale;
}

template <typename T, int D, int FMT>
__global__ void __launch_bounds__(CW_THREADS) cache_read_kernel(const CacheReadArgs a) {
    constexpr int N = D / 16;
    const int c = threadIdx.x & 15;
    const uint32_t nh = (uint32_t)a.cache.n_kv, per = 2 * nh;
    const uint32_t row = blockIdx.x * CW_ROWS + (threadIdx.x >> 4);
    if (row >= (uint32_t)a.n * per) return;
    const int64_t i = row / per;
    const int r = (int)(row - (uint32_t)i * per);
    const bool is_v = r >= (int)nh;
    const int h = is_v ? r - (int)nh : r;
    const int64_t slot = a.slots[i];
    float x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = 0.f;
    if (slot >= 0 && slot < (a.cache.n_pages << a.cache.page_shift)) {
        const int64_t at = cache_row(a.cache, slot, h);
        uint32_t w[N / 4];
        load_codes<N>((is_v ? a.cache.v_codes : a.cache.k_codes) + at * D + c * N, w);
        const float s = (is_v ? a.cache.v_scale : a.cache.k_scale)[at];
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            x[4 * j] = kv_to_f32<FMT, 0>(w[j]) * s;
            x[4 * j + 1] = kv_to_f32<FMT, 1>(w[j]) * s;
            x[4 * j + 2] = kv_to_f32<FMT, 2>(w[j]) * s;
            x[4 * j + 3] = kv_to_f32<FMT, 3>(w[j]) * s;
        }
    }
    store_f32<T, N>((T*)(is_v ? a.v_out : a.k_out) + (i * nh + h) * D + c * N, x);
}

// calls f<T, D, FMT> for the storage type, head size and format
template <typename F>
int by_type(int dtype, const CacheArgs& c, F f) {
    auto with_d = [&](auto t) {
        auto with_fmt = [&](auto d) {
            return c.format == ORDERMOE_CACHE_INT8 ? f(t, d, std::integral_constant<int, ORDERMOE_CACHE_INT8>{})
                                                   : f(t, d, std::integral_constant<int, ORDERMOE_CACHE_FP8>{});
        };
        return c.head_dim == 64    ? with_fmt(std::integral_constant<int, 64>{})
               : c.head_dim == 128 ? with_fmt(std::integral_constant<int, 128>{})
                                   : with_fmt(std::integral_constant<int, 256>{});
    };
    return dtype == ORDERMOE_BF16 ? with_d(__bf16{}) : with_d(float{});
}

}  // namespace

int launch_cache_write(const CacheWriteArgs& a, void* stream) {
    const int64_t rows = a.T * (a.n_q + 2 * a.cache.n_kv);
    if (rows == 0) return 0;
    return by_type(a.dtype, a.cache, [&](auto t, auto d, auto f) {
        KernelTimer kt_("cache_write", stream);
        cache_write_kernel<decltype(t), decltype(d)::value, decltype(f)::value>
            <<<dim3((unsigned)((rows + CW_ROWS - 1) / CW_ROWS)), dim3(CW_THREADS), 0, (hipStream_t)stream>>>(a);
        return (int)hipGetLastError();
    });
}

int launch_cache_read(const CacheReadArgs& a, void* stream) {
    const int64_t rows = a.n * 2 * a.cache.n_kv;
    if (rows == 0) return 0;
    return by_type(a.dtype, a.cache, [&](auto t, auto d, auto f) {
        KernelTimer kt_("cache_read", stream);
        cache_read_kernel<decltype(t), decltype(d)::value, decltype(f)::value>
            <<<dim3((unsigned)((rows + CW_ROWS - 1) / CW_ROWS)), dim3(CW_THREADS), 0, (hipStream_t)stream>>>(a);
        return (int)hipGetLastError();
    });
}

}  // namespace ordermoe
