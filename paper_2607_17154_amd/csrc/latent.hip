// Rows of the latent cache: written (norm, rotation), and expanded to the keys and
// values of every head; queries taken through the key weights.
//
//   latent_write_kernel   three kinds of workgroups: 64 tokens x 64 ranks of one head's
//                         absorbed queries, qa[t][r] = sum_d q[t][d] W_k[d][r]; four tokens'
//                         rows, a wave each; pieces of the queries of 16 or 8 elements that are
//                         turned or copied.  Reads and writes bound it: 16001 tokens x 32 heads of
//                         192, copied, 99 us, 4.4 TB/s
//   latent_expand_kernel, latent_expand_wide_kernel  Y = C W^T for the rows C of the cache at the
//                         given slots and all of W_k and W_v, in tiles
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "grid.hpp"
#include "mfma.hpp"
#include "write_blocks.hpp"

namespace ordermoe {
namespace {

template <bool BF>
using Elem = std::conditional_t<BF, __bf16, float>;

// 8 elements as fp32, and back
template <bool BF>
__device__ inline void load8(const Elem<BF>* p, float* x) {
    if constexpr (BF) {
        const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    } else {
        const f32x4 a = ((const f32x4*)p)[0], b = ((const f32x4*)p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
    }
}
template <bool BF>
__device__ inline void store8(Elem<BF>* p, const float* x) {
    if constexpr (BF) {
        *(u32x4*)p = u32x4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
    } else {
        ((f32x4*)p)[0] = f32x4{x[0], x[1], x[2], x[3]};
        ((f32x4*)p)[1] = f32x4{x[4], x[5], x[6], x[7]};
    }
}

// 16 elements of a rotary part turned: unit u of rot / 16, pairs 8u .. 8u + 7
template <bool BF>
__device__ inline void turn16(const LatentWriteArgs& a, int64_t t, const Elem<BF>* from, Elem<BF>* to, int u) {
    const int half = a.cache.rot / 2;
    const int at0 = a.interleaved ? 16 * u : 8 * u, at1 = a.interleaved ? 16 * u + 8 : half + 8 * u;
    float x[16];
    load8<BF>(from + at0, x);
    load8<BF>(from + at1, x + 8);
    if (a.cos_sin) {
        const int64_t p = a.pos[t];
        const bool in = p >= 0 && p < a.max_pos;
        const float* cs = a.cos_sin + (in ? p : 0) * a.cache.rot + 8 * u;
        float co[8], si[8];
        load8<false>(cs, co);
        load8<false>(cs + half, si);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = in ? co[i] : __builtin_nanf(""), s = in ? si[i] : __builtin_nanf("");
            const float lo = a.interleaved ? x[2 * i] : x[i], hi = a.interleaved ? x[2 * i + 1] : x[8 + i];
            co[i] = lo * c - hi * s;
            si[i] = hi * c + lo * s;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (a.interleaved) {
                x[2 * i] = co[i];
                x[2 * i + 1] = si[i];
            } else {
                x[i] = co[i];
                x[8 + i] = si[i];
            }
        }
    }
    store8<BF>(to + at0, x);
    store8<BF>(to + at1, x + 8);
}

// One token's cache row, by one wave: 8 elements of the latent vector a lane.
template <bool BF>
__device__ inline void write_row(const LatentWriteArgs& a, int64_t t, int lane) {
    const int R = a.cache.rank, rot = a.cache.rot, row = R + rot;
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.cache.n_pages << a.cache.page_shift) return;
    const Elem<BF>* from = (const Elem<BF>*)a.kv + t * a.kv_stride;
    Elem<BF>* to = (Elem<BF>*)a.cache.rows + slot * row;
    const bool in = lane < R / 8;
    float x[8] = {};
    if (in) load8<BF>(from + 8 * lane, x);
    if (a.norm) {
        float w[8] = {};
        if (in) load8<BF>((const Elem<BF>*)a.norm + 8 * lane, w);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += x[i] * x[i];
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
        const float r = 1.0f / sqrtf(s / (float)R + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
    }
    if (in) store8<BF>(to + 8 * lane, x);
    if (lane < rot / 16) turn16<BF>(a, t, from + R, to + R, lane);
}

// qa[t][r] for 64 tokens and 64 ranks of one head: the matrix unit's rows are ranks, its
// columns tokens; a wave takes 16 ranks and every token.
template <bool BF, int D>
__device__ inline void absorb_tile(const LatentWriteArgs& a, int64_t t0, int h, int r0, char* mem) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int R = a.cache.rank, wide = R + a.cache.rot;
    const int tiles = (int)std::min<int64_t>(LW_TOK / 16, (a.T - t0 + 15) / 16);
    f32x4 acc[LW_TOK / 16] = {};
    if constexpr (BF) {
        // W_k[h]'s 64 ranks in LDS, D rows of 128 bytes; row d's pieces of 32 bytes are swapped by d % 4, so that the
        // four rows of a turned read lie on distinct banks
        const __bf16* w = (const __bf16*)a.w_k + (int64_t)h * D * R + r0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const int piece = wave * (D / 32) + i, d = piece * 8 + (lane >> 3), ch = (lane & 7) ^ ((d & 3) << 1);
            load_lds16(w + (int64_t)d * R + ch * 8, mem + piece * 1024);
        }
        u32x4 q[LW_TOK / 16][D / 32];
#pragma unroll
        for (int m = 0; m < LW_TOK / 16; ++m) {
            const int64_t t = t0 + 16 * m + c;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                q[m][s] = u32x4{0u, 0u, 0u, 0u};
                if (m < tiles && t < a.T)
                    q[m][s] = *(const u32x4*)((const __bf16*)a.q + t * a.q_stride + h * (D + a.cache.rot) + 32 * s + 8 * g);
            }
        }
        __syncthreads();
        const int i = c >> 2, j = c & 3;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            u32x2 half[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int d = 32 * s + 8 * g + 4 * p + i;
                half[p] = read_turned(mem + d * 128 + (((2 * wave + (j >> 1)) ^ ((d & 3) << 1)) * 16) + (j & 1) * 8);
            }
            const u32x4 wf = {half[0][0], half[0][1], half[1][0], half[1][1]};
#pragma unroll
            for (int m = 0; m < LW_TOK / 16; ++m) acc[m] = mma16<true>(wf, q[m][s], acc[m]);
        }
    } else {
        const float* w = (const float*)a.w_k + (int64_t)h * D * R + r0 + 16 * wave + c;
        for (int s = 0; s < D / 16; ++s) {
            u32x4 wf;
#pragma unroll
            for (int e = 0; e < 4; ++e) wf[e] = __float_as_uint(w[(int64_t)(16 * s + 4 * g + e) * R]);
#pragma unroll
            for (int m = 0; m < LW_TOK / 16; ++m) {
                const int64_t t = t0 + 16 * m + c;
                u32x4 q = {0u, 0u, 0u, 0u};
                if (m < tiles && t < a.T)
                    q = *(const u32x4*)((const float*)a.q + t * a.q_stride + h * (D + a.cache.rot) + 16 * s + 4 * g);
                acc[m] = mma16<false>(wf, q, acc[m]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < LW_TOK / 16; ++m) {
        const int64_t t = t0 + 16 * m + c;
        if (m < tiles && t < a.T)
            store4<BF>(a.q_out, (t * a.n_q + h) * wide + r0 + 16 * wave + 4 * g, acc[m][0], acc[m][1], acc[m][2], acc[m][3]);
    }
}

// blocks: absorb tiles, then rows, then the queries' pieces of 8 elements that are copied (not where they are absorbed), then
// those of 16 that are turned
template <bool BF, int D, int ROT>
__global__ void __launch_bounds__(256) latent_write_kernel(const LatentWriteArgs a, const WriteBlocks n) {
    __shared__ __attribute__((aligned(16))) char mem[BF ? D * LW_COLS * 2 : 16];
    int64_t blk = block_number();
    const WriteBlocks::Kind kind = n.kind(blk);
    if (kind == WriteBlocks::ABSORB) {
        const int slices = a.cache.rank / LW_COLS;
        const int64_t th = blk / slices;
        const int r0 = (int)(blk - th * slices) * LW_COLS, h = (int)(th % a.n_q);
        absorb_tile<BF, D>(a, th / a.n_q * LW_TOK, h, r0, mem);
        return;
    }
    if (kind == WriteBlocks::ROWS) {
        const int64_t t = blk * 4 + (threadIdx.x >> 6);
        if (t < a.T) write_row<BF>(a, t, threadIdx.x & 63);
        return;
    }
    if (kind == WriteBlocks::NONE) return;
    const uint32_t heads = (uint32_t)(a.T * a.n_q), n_q = (uint32_t)a.n_q;       // (fewer than 2^31)
    if (kind == WriteBlocks::COPY) {
        constexpr int PER = D / 8;
        float x[LW_COPIES][8];
        const int k = threadIdx.x % PER;
        const int64_t first = blk * (256 / PER * LW_COPIES) + threadIdx.x / PER;
#pragma unroll
        for (int i = 0; i < LW_COPIES; ++i) {
            const int64_t r = first + i * (256 / PER);
            if (r >= heads) continue;
            const uint32_t t = (uint32_t)r / n_q, h = (uint32_t)r - t * n_q;
            load8<BF>((const Elem<BF>*)a.q + t * a.q_stride + h * (D + ROT) + 8 * k, x[i]);
        }
#pragma unroll
        for (int i = 0; i < LW_COPIES; ++i) {
            const int64_t r = first + i * (256 / PER);
            if (r < heads) store8<BF>((Elem<BF>*)a.q_out + r * (D + ROT) + 8 * k, x[i]);
        }
        return;
    }
    constexpr int PER = ROT / 16;
    const int wide = a.absorb ? a.cache.rank : D, k = threadIdx.x % PER;
#pragma unroll
    for (int i = 0; i < LW_TURNS; ++i) {
        const int64_t r = (blk * LW_TURNS + i) * (256 / PER) + threadIdx.x / PER;
        if (r >= heads) break;
        const uint32_t t = (uint32_t)r / n_q, h = (uint32_t)r - t * n_q;
        turn16<BF>(a, t, (const Elem<BF>*)a.q + t * a.q_stride + h * (D + ROT) + D, (Elem<BF>*)a.q_out + r * (wide + ROT) + wide, k);
    }
}

template <bool BF, int D, int ROT>
int launch_write(const LatentWriteArgs& a, hipStream_t st) {
    const WriteBlocks n = write_blocks(a.T, a.n_q, D, a.cache.rank, ROT, a.q != nullptr, a.absorb != 0);
    KernelTimer kt_("latent_write", st);
    latent_write_kernel<BF, D, ROT><<<grid_of(n.absorb + n.rows + n.copies + n.turns), dim3(256), 0, st>>>(a, n);
    return (int)hipGetLastError();
}
template <bool BF>
int launch_write_dim(const LatentWriteArgs& a, hipStream_t st) {
    if (a.head_dim == 64) return a.cache.rot == 32 ? launch_write<BF, 64, 32>(a, st) : launch_write<BF, 64, 64>(a, st);
    return a.cache.rot == 32 ? launch_write<BF, 128, 32>(a, st) : launch_write<BF, 128, 64>(a, st);
}

// ------------------------------------------------------------------ expansion
constexpr int LE_SLAB = 128;                         // bytes of a row staged at a time

// The workgroup's tile; false: there is none.  spread: eight token tiles after one another on each XCD, which then go
// through all weights together
__device__ inline bool find_tile(int64_t tok_tiles, int row_tiles, int spread, int64_t& tt, int& rt) {
    const int64_t id = block_number();
    if (spread) {
        const int64_t x = id & 7, l = id >> 3, grp = l / (8 * row_tiles);
        const int in = (int)(l - grp * (8 * row_tiles));
        rt = in >> 3;
        tt = (grp * 8 + (in & 7)) * 8 + x;
    } else {
        tt = id / row_tiles;
        rt = (int)(id - tt * row_tiles);
    }
    return tt < tok_tiles;
}
// The rotary parts of a tile's tokens
template <int ES>
__device__ inline void rotary_out(const LatentExpandArgs& a, int64_t n0, int tokens, int tid) {
    const int wide = a.cache.rank + a.cache.rot, per = a.cache.rot * ES / 16;
    const int64_t slots = a.cache.n_pages << a.cache.page_shift;
    for (int u = tid; u < tokens * per; u += 256) {
        const int r = u / per, k = u - r * per;
        if (n0 + r >= a.n) break;
        const int64_t s = a.slots[n0 + r];
        u32x4 v = {0u, 0u, 0u, 0u};
        if (s >= 0 && s < slots) v = *(const u32x4*)(a.cache.rows + (s * wide + a.cache.rank) * ES + 16 * k);
        *(u32x4*)((char*)a.r_out + (n0 + r) * a.cache.rot * ES + 16 * k) = v;
    }
}
template <int N>
__device__ inline void wait_vmem() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\ns_barrier" ::: "memory"); }

// One slab's products, the loads of a later one beside them.  (Their buffers never overlap: told so, the compiler does not
// wait for the loads before the first read.)
template <bool BF, int W, class Issue>
__device__ inline __attribute__((always_inline)) void expand_step(char* __restrict behind, const char* __restrict tok, const char* __restrict wei,
                                                                  int wm, int wn, int lane, const Issue& issue, f32x4 (&acc)[W / 16][W / 16]) {
    constexpr int F = W / 16;
    const int c = lane & 15, g = lane >> 4;
    issue(behind);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        u32x4 t[F], w[F];
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int rt_ = wn * W + 16 * i + c, rw = wm * W + 16 * i + c;
            t[i] = *(const u32x4*)(tok + rt_ * LE_SLAB + (((4 * k + g) ^ (rt_ & 7)) * 16));
            w[i] = *(const u32x4*)(wei + rw * LE_SLAB + (((4 * k + g) ^ (rw & 7)) * 16));
        }
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) acc[i][j] = mma16<BF>(w[i], t[j], acc[i][j]);
    }
}

// A tile of TN tokens (the matrix unit's columns) x TN weight rows, 2 x 2 waves.  Both come in
// slabs of 128 bytes a row through LDS, two buffers, or four of fewer rows, all but one on their way; chunk c of row r
// lies at c ^ (r % 8), so that the 16-byte reads of eight rows lie on distinct banks.  (300 tokens x 8 heads of 64,
// rank 256, fp32: 8.0 us in tiles of 64, 5.9 of 32.)
template <bool BF, int TN>
__global__ void __launch_bounds__(256) latent_expand_kernel(const LatentExpandArgs a, int64_t tok_tiles, int row_tiles, int spread) {
    constexpr int ES = BF ? 2 : 4, W = TN / 2, F = W / 16, LOADS = TN / 32;     // a wave's rows, its tiles, its pieces of a slab
    constexpr int BUFS = TN < 128 ? 4 : 2, SLAB = TN * LE_SLAB;
    __shared__ __attribute__((aligned(16))) char mem[BUFS][2][SLAB];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4, wm = wave >> 1, wn = wave & 1;
    int64_t tt;
    int rt;
    if (!find_tile(tok_tiles, row_tiles, spread, tt, rt)) return;
    const int R = a.cache.rank, wide = R + a.cache.rot, half = a.n_q * a.head_dim, r0 = rt * TN;
    const int64_t n0 = tt * TN, slots = a.cache.n_pages << a.cache.page_shift;
    const char* from[2][LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int r = (wave * LOADS + i) * 8 + (lane >> 3), ch = (lane & 7) ^ (r & 7);
        int64_t s = n0 + r < a.n ? a.slots[n0 + r] : 0;
        if (s < 0 || s >= slots) s = 0;
        from[0][i] = a.cache.rows + s * wide * ES + ch * 16;
        const int wr = r0 + r < 2 * half ? r0 + r : 0;
        from[1][i] = (wr < half ? (const char*)a.w_k + (int64_t)wr * R * ES : (const char*)a.w_v + (int64_t)(wr - half) * R * ES) + ch * 16;
    }
    auto issue = [&](char* to, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int o = 0; o < 2; ++o) load_lds16(from[o][i] + s * LE_SLAB, to + o * SLAB + (wave * LOADS + i) * 1024);
    };
    f32x4 acc[F][F] = {};                            // [weight tile][token tile]
    const int slabs = R * ES / LE_SLAB;              // (2 or more)
    issue(mem[0][0], 0);
    __builtin_amdgcn_s_waitcnt(0x0F70);              // vmcnt(0), in a form that the compiler takes into account
    for (int s = 0; s < slabs; ++s) {
        if (s + BUFS - 2 < slabs) wait_vmem<(BUFS - 2) * 2 * LOADS>();
        else wait_vmem<0>();
        lds_barrier();                               // slab s has arrived, and slab s - 1 has been read
        expand_step<BF, W>(mem[0][0], mem[s % BUFS][0], mem[s % BUFS][1], wm, wn, lane, [&](char* to) __attribute__((always_inline)) {
            const int last = std::min(s + BUFS, slabs);
            for (int x = s == 0 ? 1 : s + BUFS - 1; x < last; ++x) issue(to + x % BUFS * (2 * SLAB), x);
        }, acc);
    }
#pragma unroll
    for (int j = 0; j < F; ++j) {
        const int64_t n = n0 + wn * W + 16 * j + c;
        if (n >= a.n) continue;
        const int64_t s = a.slots[n];
        const bool in = s >= 0 && s < slots;
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int wr = r0 + wm * W + 16 * i + 4 * g;
            if (wr >= 2 * half) continue;
            const f32x4 v = in ? acc[i][j] : f32x4{0.f, 0.f, 0.f, 0.f};
            if (wr < half) store4<BF>(a.k_out, n * half + wr, v[0], v[1], v[2], v[3]);
            else store4<BF>(a.v_out, n * half + wr - half, v[0], v[1], v[2], v[3]);
        }
    }
    if (rt == 0) rotary_out<ES>(a, n0, TN, tid);
}

// The same in tiles of 256 tokens x 128 weight rows, 2 x 2 waves of 128 x 64: a wave reads 12 pieces of LDS for 32 matrix
// instructions, where 64 x 64 reads 8 for 16 and LDS is what bounds it.  Slabs of 64 bytes a row, three
// buffers, two slabs on their way; chunk c of row r lies at c ^ (r / 2 % 4), so that lanes read together (0 - 3, 12 - 15,
// 20 - 27, the others of each 32) do so on distinct banks.  A workgroup takes some weight tiles of its tokens after one
// another: the next tile's loads are on their way while a tile's results go, through LDS of the wave's own, in whole
// lines to memory.  30001 tokens x 32 heads of 128, rank 512: 383 us in tiles of 128, 294 to 327 on different cards (770 to
// 857 TFLOP/s); the matrix unit is busy 39% of the time, LDS 36%, each waiting for the other at a slab's end.
constexpr int LX_TOK = 256, LX_W = 128, LX_SLAB = 64, LX_STAGE = (LX_TOK + LX_W) * LX_SLAB, LX_OUT = 16 * 128;
constexpr int LX_CHUNK = 4;                          // weight tiles of a workgroup, at most (one 332 us, two 322, four 319, eight 332)

// (The loads' buffer and the one that is read never overlap: told so, the compiler does not wait for the loads first.)
template <class Issue>
__device__ inline __attribute__((always_inline)) void expand_slab(char* __restrict behind, const char* __restrict tok,
                                                                  const char* __restrict wei, const Issue& issue, f32x4 (&acc)[4][8]) {
    issue(behind);
    __builtin_amdgcn_sched_barrier(0);
    u32x4 w[4], t[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = *(const u32x4*)(wei + 16 * i * LX_SLAB);
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = *(const u32x4*)(tok + 16 * j * LX_SLAB);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = mma16<true>(w[i], t[j], acc[i][j]);
    // three pieces of the tokens are read ahead of their products
    __builtin_amdgcn_sched_group_barrier(0x100, 7, 0);
#pragma unroll
    for (int j = 0; j < 5; ++j) {
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 12, 0);
}

__global__ void __launch_bounds__(256, 2) latent_expand_wide_kernel(const LatentExpandArgs a, int64_t tok_tiles, int row_tiles, int chunk,
                                                                    int spread) {
    constexpr int PIECES = LX_STAGE / 1024 / 4;          // of a slab, a wave: 16 rows each, the tokens' first
    constexpr int TP = LX_TOK / 64, STORES = 16;         // the tokens' pieces; a wave's stores of a whole tile
    __shared__ __attribute__((aligned(16))) char mem[3 * LX_STAGE + 4 * LX_OUT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4, wm = wave >> 1, wn = wave & 1;
    int64_t tt;
    int rc;
    if (!find_tile(tok_tiles, (row_tiles + chunk - 1) / chunk, spread, tt, rc)) return;
    const int rt0 = rc * chunk, rt1 = std::min(row_tiles, rt0 + chunk);
    const int R = a.cache.rank, wide = R + a.cache.rot, half = a.n_q * a.head_dim;
    const int64_t n0 = tt * LX_TOK, slots = a.cache.n_pages << a.cache.page_shift;
    const int row = lane >> 2, ch = (lane & 3) ^ ((lane >> 3) & 3);
    const char *tok_at[TP], *wei_at[PIECES - TP];
#pragma unroll
    for (int i = 0; i < TP; ++i) {
        const int r = (i * 4 + wave) * 16 + row;
        int64_t s = n0 + r < a.n ? a.slots[n0 + r] : 0;
        tok_at[i] = a.cache.rows + (s >= 0 && s < slots ? s : 0) * wide * 2 + ch * 16;
    }
    uint32_t there = 0;                                  // bit j: the lane's token 16 j + c of the wave's 128 lies in the cache
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t n = n0 + wn * 128 + 16 * j + c, s = n < a.n ? a.slots[n] : -1;
        there |= (uint32_t)(s >= 0 && s < slots) << j;
    }
    auto weights = [&](int rt) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PIECES - TP; ++i) {
            int wr = rt * LX_W + (i * 4 + wave) * 16 + row;
            wr = wr < 2 * half ? wr : 0;
            wei_at[i] = (wr < half ? (const char*)a.w_k + (int64_t)wr * R * 2 : (const char*)a.w_v + (int64_t)(wr - half) * R * 2) + ch * 16;
        }
    };
    const int slabs = R * 2 / LX_SLAB, place = c * LX_SLAB + (g ^ ((c >> 1) & 3)) * 16;
    const bool whole = n0 + LX_TOK <= a.n;
    char* const out = mem + 3 * LX_STAGE + wave * LX_OUT;
    int ls = 0, lt = rt0, at = 0;                        // the slab and the tile to load next; the buffer to read
    weights(lt);
    auto issue = [&](char* to) __attribute__((always_inline)) {
        if (lt >= rt1) return;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            load_lds16((i < TP ? tok_at[i] : wei_at[i < TP ? 0 : i - TP]) + ls * LX_SLAB, to + (i * 4 + wave) * 1024);
        if (++ls == slabs) {
            ls = 0;
            weights(++lt);
        }
    };
    issue(mem);
    issue(mem + LX_STAGE);
    __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0), in a form that the compiler takes into account
    for (int rt = rt0; rt < rt1; ++rt) {
        f32x4 acc[4][8] = {};                            // [weight tile][token tile]
        for (int s = 0; s < slabs; ++s) {
            // what was issued behind slab s may still be on its way: slab s + 1 and, before it, a tile's stores
            if (s + 1 == slabs && rt + 1 == rt1) wait_vmem<0>();
            else if (s < 2 && rt > rt0 && whole) wait_vmem<PIECES + STORES>();
            else wait_vmem<PIECES>();
            lds_barrier();                               // slab s has arrived, and slab s - 1 has been read
            expand_slab(mem + (at == 0 ? 2 * LX_STAGE : at - LX_STAGE), mem + at + wn * (128 * LX_SLAB) + place,
                        mem + at + (LX_TOK + wm * 64) * LX_SLAB + place, issue, acc);
            at = at == 2 * LX_STAGE ? 0 : at + LX_STAGE;
        }
        // 16 tokens at a time: token n's 128 bytes in the wave's own LDS, chunk of 16 bytes k at k ^ (n % 8)
        int l = lane;
        asm volatile("" : "+v"(l));                      // (places made anew: kept, they would take the sums' registers)
        const int oc = l & 7, on = l >> 3, wr = rt * LX_W + wm * 64 + 8 * oc;
        const int64_t first = n0 + wn * 128 + on;
        __bf16* to = (wr < half ? (__bf16*)a.k_out + wr : (__bf16*)a.v_out + (wr - half)) + first * half;
        int left = wr < 2 * half ? (int)std::min<int64_t>(a.n - first, LX_TOK) : 0;
        char* const put = out + (l & 15) * 128 + ((l >> 4) & 1) * 8;
        const int swap = ((l >> 5) ^ (l & 7)) * 16;      // (2 i + g / 2) ^ (c % 8) = 2 i ^ (g / 2 ^ c % 8)
        const char* const get = out + on * 128 + (oc ^ on) * 16;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t keep = there >> j & 1 ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(u32x2*)(put + (swap ^ (32 * i))) =
                    u32x2{bf16_pair(acc[i][j][0], acc[i][j][1]) & keep, bf16_pair(acc[i][j][2], acc[i][j][3]) & keep};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const u32x4 x = *(const u32x4*)(get + 1024 * k);
                if (left > 0) *(u32x4*)to = x;
                to += (int64_t)8 * half;
                left -= 8;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (rt0 == 0) rotary_out<2>(a, n0, LX_TOK, tid);
}

template <bool BF, int TN>
int launch_expand(const LatentExpandArgs& a, hipStream_t st) {
    const int64_t tt = (a.n + TN - 1) / TN;
    const int rt = (2 * a.n_q * a.head_dim + TN - 1) / TN;
    const bool spread = tt >= 64;
    const int64_t blocks = spread ? (tt + 63) / 64 * 64 * rt : tt * rt;
    KernelTimer kt_("latent_expand", st);
    latent_expand_kernel<BF, TN><<<grid_of(blocks), dim3(256), 0, st>>>(a, tt, rt, spread);
    return (int)hipGetLastError();
}

int launch_expand_wide(const LatentExpandArgs& a, hipStream_t st) {
    const int64_t tt = (a.n + LX_TOK - 1) / LX_TOK;
    const int rt = (2 * a.n_q * a.head_dim + LX_W - 1) / LX_W;
    const int chunk = (int)std::min<int64_t>(LX_CHUNK, std::max<int64_t>(1, tt * rt / 1024));
    const int chunks = (rt + chunk - 1) / chunk;
    const bool spread = tt >= 64;
    const int64_t blocks = spread ? (tt + 63) / 64 * 64 * chunks : tt * chunks;
    KernelTimer kt_("latent_expand", st);
    latent_expand_wide_kernel<<<grid_of(blocks), dim3(256), 0, st>>>(a, tt, rt, chunk, spread);
    return (int)hipGetLastError();
}

}  // namespace

int launch_latent_write(const LatentWriteArgs& a, void* stream) {
    if (a.T == 0) return 0;
    return a.cache.dtype == ORDERMOE_BF16 ? launch_write_dim<true>(a, (hipStream_t)stream)
                                          : launch_write_dim<false>(a, (hipStream_t)stream);
}

int launch_latent_expand(const LatentExpandArgs& a, void* stream) {
    if (a.n == 0) return 0;
    // the largest tiles that give every CU one
    auto enough = [&](int tile) { return (a.n + tile - 1) / tile * (2 * a.n_q * a.head_dim / tile) >= 256; };
    if (a.cache.dtype == ORDERMOE_BF16 && (a.n + LX_TOK - 1) / LX_TOK * (2 * a.n_q * a.head_dim / LX_W) >= 512)
        return launch_expand_wide(a, (hipStream_t)stream);
    if (a.cache.dtype == ORDERMOE_BF16)
        return enough(128) ? launch_expand<true, 128>(a, (hipStream_t)stream)
               : enough(64) ? launch_expand<true, 64>(a, (hipStream_t)stream) : launch_expand<true, 32>(a, (hipStream_t)stream);
    return enough(128) ? launch_expand<false, 128>(a, (hipStream_t)stream)
           : enough(64) ? launch_expand<false, 64>(a, (hipStream_t)stream) : launch_expand<false, 32>(a, (hipStream_t)stream);
}

}  // namespace ordermoe
