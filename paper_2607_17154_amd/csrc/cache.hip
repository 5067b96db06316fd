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
#include "grid.hpp"
#include "kv_codes.hpp"

namespace ordermoe {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int CW_THREADS = 256;
constexpr int CW_ROWS = CW_THREADS / 16;     // 16-lane groups per block
constexpr int64_t CW_MANY = 1 << 16;         // head rows from which a group takes four: twice the chip's waves
constexpr int64_t CW_STREAM_BYTES = (int64_t)32 << 20;   // bytes of queries from which rows go past the caches: all L2s together

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

// N neighbouring elements of storage T: as read, and as fp32
template <typename T, int N>
struct Raw {
    static constexpr int W = N * (int)sizeof(T) / 4;
    uint32_t w[W];
    template <bool NTL = false>
    __device__ inline void load(const T* p) {
        if constexpr (W == 2) {
            u32x2 v;
            if constexpr (NTL) v = __builtin_nontemporal_load((const u32x2*)p);
            else v = *(const u32x2*)p;
            w[0] = v[0]; w[1] = v[1];
        } else {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                u32x4 v;
                if constexpr (NTL) v = __builtin_nontemporal_load((const u32x4*)p + i);
                else v = ((const u32x4*)p)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
            }
        }
    }
    __device__ inline void f32(float* x) const {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(T) == 4) {
                x[i] = __uint_as_float(w[i]);
            } else {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    }
};
template <typename T, int N>
__device__ inline void load_f32(const T* p, float* x) {
    Raw<T, N> r;
    r.load(p);
    r.f32(x);
}
template <bool NTS>
__device__ inline void store16(void* p, u32x4 v) {
    if constexpr (NTS) __builtin_nontemporal_store(v, (u32x4*)p);
    else *(u32x4*)p = v;
}
template <typename T, int N, bool NTS = false>
__device__ inline void store_f32(T* p, const float* x) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(x[4 * i + j]);
            store16<NTS>((u32x4*)p + i, v);
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
            for (int i = 0; i < N / 8; ++i) store16<NTS>((u32x4*)p + i, u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]});
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

// x / b for x of a magnitude of at most 2^30 b, rounded as an IEEE division rounds it
// where that can matter to the code: with r the correctly rounded 1 / b, q = x r is less
// than 1.5 units in the last place off, and q + r (x - b q) with fused steps is the
// correctly rounded quotient.  Its last rounding could only go wrong where x / b lies next
// to the middle of two floats; there q is one of the two, as Markstein's proof asks.  (6e8
// pairs, three quarters of them with significands next to 1 or 2: q up to 1.495 units off,
// the corrected quotient always that of the division.  The residual is exact unless x is
// below 2^-125, whose quotient is below 2^-16: code 0 either way.)  The divisions took a
// third of the kernel.
__device__ inline float quotient(float x, float b, float r) {
    const float q = x * r;
    return fmaf(fmaf(-q, b, x), r, q);
}

// row / n for row < 2^31, by a product (n >= 2)
__device__ inline uint32_t divided(uint32_t row, const Divisor& n) { return __umulhi(row, n.mul) >> n.shift; }

// One head row of N elements per lane, already read (x): all of its work.
template <typename T, int D, int FMT, bool NTS>
__device__ inline void write_head_row(const CacheWriteArgs& a, uint32_t t, int h, int pos, int64_t slot, float* x, int c) {
    constexpr int N = D / 16;                                   // elements per lane
    const int kind = h < a.n_q ? 0 : h < a.n_q + a.cache.n_kv ? 1 : 2;      // query, key, value
    const int hk = h - a.n_q - (kind == 2 ? a.cache.n_kv : 0);
    const T* nw = (const T*)(kind == 0 ? a.q_norm : kind == 1 ? a.k_norm : nullptr);
    const bool turn = kind != 2 && a.rot;
    const int half = a.rot / 2;
    const float* cs = a.cos_sin;
    bool in = true;
    // the lane's pairs (interleaved: N / 2 from c N / 2 on; else N, of its own elements or its partner's)
    const int dl = half / N;
    const bool lo = c < dl, turned = turn && (a.interleaved ? c * (N / 2) < half : c < 2 * dl);
    float co[N], si[N];
    if (turn) {
        in = pos >= 0 && (int64_t)pos < a.max_pos;
        cs += (int64_t)(in ? pos : 0) * a.rot;
        if (a.interleaved) {
            load_f32<float, N / 2 < 4 ? 4 : N / 2>(cs + (turned ? c * (N / 2) & ~3 : 0), co);
            load_f32<float, N / 2 < 4 ? 4 : N / 2>(cs + half + (turned ? c * (N / 2) & ~3 : 0), si);
            if (N == 4 && (c & 1)) {                            // (two pairs a lane, read with the neighbour's)
                co[0] = co[2]; co[1] = co[3];
                si[0] = si[2]; si[1] = si[3];
            }
        } else {
            const int i0 = turned ? (lo ? c : c - dl) * N : 0;
            load_f32<float, N>(cs + i0, co);
            load_f32<float, N>(cs + half + i0, si);
        }
    }
    if (nw) {
        float w[N], s = 0.f;
        load_f32<T, N>(nw + c * N, w);
#pragma unroll
        for (int i = 0; i < N; ++i) s = fmaf(x[i], x[i], s);
        const float r = __builtin_amdgcn_rsqf(row_sum(s) * (1.0f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = x[i] * r * w[i];
    }
    if (turn) {
        if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float u = x[2 * i], v = x[2 * i + 1];
                x[2 * i] = turned ? fmaf(u, co[i], -(v * si[i])) : u;
                x[2 * i + 1] = turned ? fmaf(v, co[i], u * si[i]) : v;
            }
        } else {
            // the partner of element i is i +- half, `half / N` lanes away (whole lanes, since half is a multiple of N)
            const int from = turned ? (lo ? c + dl : c - dl) : c;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float o = __shfl(x[i], from, 16);
                const float y = fmaf(o, lo ? -si[i] : si[i], x[i] * co[i]);
                x[i] = turned ? y : x[i];
            }
        }
        if (!in && turned)                                      // no such position
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = __builtin_nanf("");
    }
    if (kind == 0) {
        store_f32<T, N, NTS>((T*)a.q_out + ((int64_t)t * a.n_q + h) * D + c * N, x);
        return;
    }
    // the largest magnitude on the bits, where a NaN is larger than infinity
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t b = __float_as_uint(x[i]) << 1;          // (without the sign)
        big = b > big ? b : big;
    }
    big = row_max(big) >> 1;
    const bool bad = big >= 0x7F800000u, none = __uint_as_float(big) < KV_TINY;
    const float scale = bad ? __builtin_nanf("") : none ? 0.f : __uint_as_float(big) / kv_code_max<FMT>();
    const float inv = 1.0f / scale;
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = quotient(x[4 * i + j], scale, inv);
        w[i] = bad || none ? 0u : kv_to_codes<FMT>(y[0], y[1], y[2], y[3]);
    }
    if (slot < 0 || slot >= (a.cache.n_pages << a.cache.page_shift)) return;
    const int64_t at = cache_row(a.cache, slot, hk);
    store_codes<N>((kind == 1 ? a.cache.k_codes : a.cache.v_codes) + at * D + c * N, w);
    if (c == 0) (kind == 1 ? a.cache.k_scale : a.cache.v_scale)[at] = scale;
}

// U rows per 16 lanes, all read before the first is worked on: one row a lane leaves
// too few bytes on their way for a prompt's rows (16001 tokens of 16 + 16 + 16 heads of 128: one
// row 94 us, four 90, before other steps made it 79); a step's are too few to share four by
// four.  NTS: rows are read, and queries stored in 16 bytes a lane, past the caches (the same rows
// 79 us, so 74).  At the switch of 32 MiB of queries through and past, heads of 128: bf16 32 + 8 heads
// 26.8 us and 26.0, 16 + 16 50.3 and 46.5, 32 + 1 20.0 and 19.6, fp32 21.6 and 23.0, 39.1 and 37.7,
// 16.4 and 19.7; at 48 MiB bf16 40.8 and 37.0, 69.8 and 65.3, 32.9 and 28.0, fp32 33.4 and 32.5, 53.6
// and 52.7, 27.7 and 26.3.
template <typename T, int D, int FMT, int U, bool NTS>
__global__ void __launch_bounds__(CW_THREADS) cache_write_kernel(const CacheWriteArgs a) {
    constexpr int N = D / 16;
    const int c = threadIdx.x & 15;
    const uint32_t heads = (uint32_t)(a.n_q + 2 * a.cache.n_kv), rows = (uint32_t)a.T * heads;
    const uint32_t row0 = block_number() * (CW_ROWS * U) + (threadIdx.x >> 4);
    uint32_t t[U];
    int h[U], pos[U];
    int64_t slot[U];
    Raw<T, N> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t row = row0 + CW_ROWS * u < rows ? row0 + CW_ROWS * u : 0;     // (past the end: read, not worked on)
        t[u] = divided(row, a.heads);
        h[u] = (int)(row - t[u] * heads);
        const int hk = h[u] - a.n_q, hv = hk - a.cache.n_kv;
        const T* src = hk < 0 ? (const T*)a.q + (int64_t)t[u] * a.q_stride + h[u] * D
                       : hv < 0 ? (const T*)a.k + (int64_t)t[u] * a.k_stride + hk * D
                                : (const T*)a.v + (int64_t)t[u] * a.v_stride + hv * D;
        raw[u].template load<NTS>(src + c * N);
        pos[u] = hv < 0 && a.rot ? a.pos[t[u]] : 0;
        slot[u] = hk < 0 ? -1 : a.slots[t[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (row0 + CW_ROWS * u >= rows) return;                 // whole rows leave together
        float x[N];
        raw[u].f32(x);
        write_head_row<T, D, FMT, NTS>(a, t[u], h[u], pos[u], slot[u], x, c);
    }
}

// CR_U rows per 16 lanes, their reads in flight together; a store covers 256
// neighbouring bytes of a row (lane: 16 bytes of every 256).  Outputs that outgrow the
// caches are stored past them.  8 heads of 128, both outputs together, stored through and past:
// bf16 48 MiB 13.7 us and 13.9, 64 MiB 22.5 and 17.7, 128 MiB 42.5 and 33.3; fp32 48 MiB 11.7 and
// 11.1, 64 MiB 15.8 and 14.1, 128 MiB 37.1 and 26.8.
constexpr int CR_U = 4;
constexpr int64_t CR_STREAM_BYTES = (int64_t)64 << 20;
template <typename T, int D, int FMT, bool NTS>
__global__ void __launch_bounds__(CW_THREADS) cache_read_kernel(const CacheReadArgs a) {
    constexpr int N = 16 / sizeof(T);                           // elements of 16 bytes
    constexpr int C = D / (16 * N) > 0 ? D / (16 * N) : 1;      // 256-byte chunks of a row (or less than one)
    const int c = threadIdx.x & 15;
    const bool on = D >= 16 * N || c < D / N;                   // lanes with a part of the row
    const uint32_t nh = (uint32_t)a.cache.n_kv, per = 2 * nh, rows = (uint32_t)a.n * per;
    const uint32_t row0 = block_number() * (CW_ROWS * CR_U) + (threadIdx.x >> 4);
    uint32_t i[CR_U], r[CR_U];
    int64_t slot[CR_U];
#pragma unroll
    for (int u = 0; u < CR_U; ++u) {
        const uint32_t row = row0 + CW_ROWS * u;
        i[u] = divided(row < rows ? row : 0, a.per);
        r[u] = (row < rows ? row : 0) - i[u] * per;
        slot[u] = row < rows ? a.slots[i[u]] : -1;
    }
    uint32_t w[CR_U][C][N / 4];
    float s[CR_U];
    bool there[CR_U];
#pragma unroll
    for (int u = 0; u < CR_U; ++u) {
        const bool is_v = r[u] >= nh;
        there[u] = slot[u] >= 0 && slot[u] < (a.cache.n_pages << a.cache.page_shift);
        const int64_t at = cache_row(a.cache, there[u] ? slot[u] : 0, (int)(is_v ? r[u] - nh : r[u]));
        const uint8_t* p = (is_v ? a.cache.v_codes : a.cache.k_codes) + at * D + (on ? c * N : 0);
#pragma unroll
        for (int k = 0; k < C; ++k) load_codes<N>(p + 16 * N * k, w[u][k]);
        s[u] = (is_v ? a.cache.v_scale : a.cache.k_scale)[at];
    }
#pragma unroll
    for (int u = 0; u < CR_U; ++u) {
        if (row0 + CW_ROWS * u >= rows) break;
        const bool is_v = r[u] >= nh;
        T* o = (T*)(is_v ? a.v_out : a.k_out) + ((int64_t)i[u] * nh + (is_v ? r[u] - nh : r[u])) * D + c * N;
        auto chunk = [&](int k) {
            float x[N];
#pragma unroll
            for (int j = 0; j < N / 4; ++j) {
                x[4 * j] = kv_to_f32<FMT, 0>(w[u][k][j]) * s[u];
                x[4 * j + 1] = kv_to_f32<FMT, 1>(w[u][k][j]) * s[u];
                x[4 * j + 2] = kv_to_f32<FMT, 2>(w[u][k][j]) * s[u];
                x[4 * j + 3] = kv_to_f32<FMT, 3>(w[u][k][j]) * s[u];
            }
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = there[u] ? x[j] : 0.f;
            if (on) store_f32<T, N, NTS>(o + 16 * N * k, x);
        };
        // (a loop of one chunk would lose the hint that its store goes past the caches: the compiler moves the store out of it)
        if constexpr (C == 1) {
            chunk(0);
        } else {
#pragma unroll
            for (int k = 0; k < C; ++k) chunk(k);
        }
    }
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

// with 2^s the power of two from n on: row / n = (row m) / 2^(31 + s) rounded down, m = 2^(31 + s) / n rounded
// down, plus 1, for every row < 2^31 (m exceeds the quotient by at most 2^-31 of a unit of row)
Divisor divisor(int n) {
    int s = 1;
    while ((1 << s) < n) ++s;
    return Divisor{(uint32_t)(((uint64_t)1 << (31 + s)) / (uint64_t)n + 1), s - 1};
}

}  // namespace

int launch_cache_write(const CacheWriteArgs& args, void* stream) {
    CacheWriteArgs a = args;
    a.heads = divisor(a.n_q + 2 * a.cache.n_kv);
    const int64_t rows = a.T * (a.n_q + 2 * a.cache.n_kv);
    if (rows == 0) return 0;
    return by_type(a.dtype, a.cache, [&](auto t, auto d, auto f) {
        KernelTimer kt_("cache_write", stream);
        constexpr int D = decltype(d)::value, F = decltype(f)::value;
        auto blocks = [&](int u) { return grid_of((rows + CW_ROWS * u - 1) / (CW_ROWS * u)); };
        if (rows < CW_MANY)
            cache_write_kernel<decltype(t), D, F, 1, false><<<blocks(1), dim3(CW_THREADS), 0, (hipStream_t)stream>>>(a);
        else if (a.T * a.n_q * D * (int64_t)sizeof(t) < CW_STREAM_BYTES)
            cache_write_kernel<decltype(t), D, F, 4, false><<<blocks(4), dim3(CW_THREADS), 0, (hipStream_t)stream>>>(a);
        else
            cache_write_kernel<decltype(t), D, F, 4, true><<<blocks(4), dim3(CW_THREADS), 0, (hipStream_t)stream>>>(a);
        return (int)hipGetLastError();
    });
}

int launch_cache_read(const CacheReadArgs& args, void* stream) {
    CacheReadArgs a = args;
    a.per = divisor(2 * a.cache.n_kv);
    const int64_t rows = a.n * 2 * a.cache.n_kv;
    if (rows == 0) return 0;
    return by_type(a.dtype, a.cache, [&](auto t, auto d, auto f) {
        KernelTimer kt_("cache_read", stream);
        constexpr int D = decltype(d)::value, F = decltype(f)::value;
        const dim3 blocks = grid_of((rows + CW_ROWS * CR_U - 1) / (CW_ROWS * CR_U));
        if (rows * D * (int64_t)sizeof(t) >= CR_STREAM_BYTES)
            cache_read_kernel<decltype(t), D, F, true><<<blocks, dim3(CW_THREADS), 0, (hipStream_t)stream>>>(a);
        else
            cache_read_kernel<decltype(t), D, F, false><<<blocks, dim3(CW_THREADS), 0, (hipStream_t)stream>>>(a);
        return (int)hipGetLastError();
    });
}

}  // namespace ordermoe
