// The whole MoE layer of one server for at most ORDERMOE_MAX_FEW = 16 tokens.
//
//   few_router_kernel  logits l = x W_r^T: a workgroup per 16 experts, a wave per K
//                      slice (the slices of the split router of small batches, added in
//                      the same order: the same logits); clears the work counters
//   few_layer_kernel   everything else.  Every workgroup runs the token stage of the
//                      routing itself (a few microseconds of latency, the same in all of
//                      them; the first one writes the routing's outputs), which tells it
//                      the experts in use and their tokens.  Then the workgroups draw
//                      work items from a counter:
//     activation tiles   16 FFN columns of one expert: gate and up rows times the
//                        tokens, silu(g) u w -> the weighted activations (memory)
//     output tiles       16 output columns: the down rows of every expert in use times
//                        its weighted activations, summed over the experts in one
//                        accumulator -> y
// An output tile needs all activations.  Items are drawn in order, activation tiles
// first, and one never waits: whoever draws an output tile knows that every
// activation tile is in the hands of a running workgroup, so its wait ends without
// any assumption on which workgroups run together.  It reads its first weights
// before it waits, so that the weight stream does not stop in between.
// The weights in use are read once; they bound the time.  The 16 tokens are the
// columns of one v_mfma_f32_16x16x32_bf16 (fp32: v_mfma_f32_16x16x4_f32), the
// weights its rows, straight from memory in the lane order of the operand.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "token_pick.hpp"

namespace ordermoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int FW = ORDERMOE_MAX_FEW;
static_assert(FW == 16, "the tokens are the columns of one matrix instruction");
constexpr int FW_THREADS = 256, FW_WAVES = 4;
constexpr int FW_PER_CU = 2;                      // workgroups per CU
constexpr int FW_SLICES = 16;                     // K slices of the router, at most
constexpr uint32_t OOR = 0x80000000u;             // past every buffer: reads zeros
constexpr int NT = 2;                             // buffer load cache bit nt: non-temporal
// a layer of this many bytes of gate/up weights outgrows the caches: its weights go
// past them (as in the grouped GEMMs)
constexpr int64_t FW_STREAM_BYTES = (int64_t)64 << 20;

__device__ inline __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes, 0x00020000);
}
template <int AUX = 0>
__device__ inline u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, (int)voff, (int)soff, AUX);
}

// acc += A B for 16 bytes of A's rows and of B's columns per lane: bf16 8 inner
// indexes (8 (lane / 16) .. + 7 of 32), fp32 4 (4 (lane / 16) .. + 3 of 16)
template <bool BF>
__device__ inline f32x4 mma(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (BF) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), acc, 0, 0, 0);
        return acc;
    }
}

// ------------------------------------------------------------------ router
__global__ void __launch_bounds__(FW_SLICES * 64) few_router_kernel(const FewArgs a, int ks) {
    __shared__ double s_part[FW_SLICES][16][16];             // (bf16: floats in the same place)
    const int tid = threadIdx.x, lane = tid & 63, z = tid >> 6;
    const int r16 = lane & 15, g = lane >> 4;
    const int E = a.r.E, d = a.r.d, T = (int)a.r.T;
    const int Epad = (E + 15) & ~15;
    if (blockIdx.x == 0 && tid < 2) a.ctr[tid] = 0;
    const int kc = d / ks;                                   // a multiple of 32
    const int e = blockIdx.x * 16 + r16;
    const bool bf = a.r.dtype == ORDERMOE_BF16;
    const uint32_t esz = bf ? 2 : 4;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.r.x, (uint32_t)T * (uint32_t)d * esz);
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.r.w_router, (uint32_t)E * (uint32_t)d * esz);
    const uint32_t xo = r16 < T ? (uint32_t)r16 * (uint32_t)d * esz + 16u * g : OOR;
    const uint32_t wo = e < E ? (uint32_t)e * (uint32_t)d * esz + 16u * g : OOR;
    float* pf = (float*)s_part;
    if (z < ks) {
        if (bf) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            const int n = kc / 32;
            for (int s0 = 0; s0 < n; s0 += 8) {
                u32x4 xv[8], wv[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const uint32_t past = s0 + u < n ? 0u : OOR, so = (uint32_t)(z * kc + (s0 + u < n ? s0 + u : 0) * 32) * 2u;
                    xv[u] = load16(rx, xo | past, so);
                    wv[u] = load16(rw, wo | past, so);
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) acc = mma<true>(xv[u], wv[u], acc);
            }
            // acc[i]: token 4 g + i, expert r16
#pragma unroll
            for (int i = 0; i < 4; ++i) pf[(z * 16 + 4 * g + i) * 16 + r16] = acc[i];
        } else {
            f64x4 acc = {0.0, 0.0, 0.0, 0.0};
            const int n = kc / 16;
            for (int s0 = 0; s0 < n; s0 += 4) {
                u32x4 xv[4], wv[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t past = s0 + u < n ? 0u : OOR, so = (uint32_t)(z * kc + (s0 + u < n ? s0 + u : 0) * 16) * 4u;
                    xv[u] = load16(rx, xo | past, so);
                    wv[u] = load16(rw, wo | past, so);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)__uint_as_float(xv[u][i]),
                                                                   (double)__uint_as_float(wv[u][i]), acc, 0, 0, 0);
            }
            // acc[i]: token 4 i + g, expert r16
#pragma unroll
            for (int i = 0; i < 4; ++i) s_part[z][4 * i + g][r16] = acc[i];
        }
    }
    __syncthreads();
    if (tid < 256) {
        const int t = tid >> 4, c = tid & 15;
        float v = 0.f;
        if (bf) {
            for (int s = 0; s < ks; ++s) v += pf[(s * 16 + t) * 16 + c];
        } else {
            double w = 0.0;
            for (int s = 0; s < ks; ++s) w += s_part[s][t][c];
            v = (float)w;
        }
        if (t < T) a.logits[t * Epad + blockIdx.x * 16 + c] = v;
    }
}

// ------------------------------------------------------------------ layer
// silu(g) = g / (1 + e^-g); bf16 with the hardware reciprocal, as the result is rounded right after
template <bool BF>
__device__ inline float silu(float g) {
    if constexpr (BF) return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g));
    else return g / (1.0f + expf(-g));
}

// A matrix [N][K] of weights as the packed layout has it: byte offset of the 16
// rows that start at row0 (a multiple of 16), of lane (r = lane % 16, g = lane / 16),
// and of a step of 64 (bf16) or 32 (fp32) columns; a step is two reads 64 bytes apart.
template <bool BF>
__device__ inline uint32_t rows_offset(int row0, int K, int lane) {
    const uint32_t r = (uint32_t)(row0 + (lane & 15)), g = (uint32_t)(lane >> 4);
    if constexpr (BF) return (r / 256u) * (uint32_t)(K / 64) * 32768u + (r % 256u) * 128u + g * 16u;
    else return r * (uint32_t)K * 4u + g * 16u;
}
template <bool BF>
constexpr uint32_t STEP_BYTES = BF ? 32768u : 128u;

// the routing's outputs that need all tokens, by the first workgroup: dispatch
// list (rank of a slot: earlier destinations, then earlier slots), totals
__device__ inline void write_route_totals(const FewArgs& a, const int8_t* dst, const int32_t* cnt, int tid) {
    const int n = (int)a.r.T * a.r.k, M = a.r.M;
    if (tid < n) {
        const int m = dst[tid];
        int rank = 0, remote = 0;
        for (int i = 0; i < n; ++i) {
            const int o = dst[i];
            remote += o >= 0;
            rank += m >= 0 && o >= 0 && (o < m || (o == m && i < tid));
        }
        if (m >= 0) a.r.out.dispatch[rank] = tid;
        if (tid >= remote) a.r.out.dispatch[tid] = -1;
    }
    if (tid < M) {
        int c = 0;
        for (int i = 0; i < n; ++i) c += dst[i] == tid;
        a.r.out.dst_count[tid] = c;
    }
    if (tid < ORDERMOE_NUM_COUNTERS) a.r.out.counters[tid] = cnt[tid];
}

template <bool BF, int NBT, int AUX>
__global__ void __launch_bounds__(FW_THREADS, FW_PER_CU) few_layer_kernel(const FewArgs a) {
    constexpr int U = 4;                                     // steps per set of reads; two sets in turn
    constexpr int SK = BF ? 64 : 32;                         // columns of a step
    constexpr uint32_t ES = BF ? 2 : 4;
    __shared__ float s_logit[FW * NBT * 16];
    __shared__ int32_t s_lidx[ORDERMOE_MAX_EXPERTS];
    __shared__ float s_w[ORDERMOE_MAX_LOCAL + 1][FW];        // gate weight of (group, token)
    __shared__ uint32_t s_msk[ORDERMOE_MAX_LOCAL + 1];       // tokens of a group
    __shared__ int32_t s_grp[ORDERMOE_MAX_LOCAL + 1];        // the groups in use, the shared one first
    __shared__ int8_t s_dst[FW * ORDERMOE_MAX_TOPK];
    __shared__ int32_t s_cnt[ORDERMOE_NUM_COUNTERS];
    __shared__ __attribute__((aligned(16))) float s_red[FW_WAVES][2][16][17];
    __shared__ int32_t s_item;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g16 = lane >> 4;
    const int T = (int)a.r.T, E = a.r.E, k = a.r.k, d = a.r.d, n_local = a.n_local;
    const int Epad = (E + 15) & ~15;
    const bool first = blockIdx.x == 0;
    int next = 0;
    if (tid == 0) next = __hip_atomic_fetch_add(a.ctr, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

    // ---- token stage: lanes 16 t .. 16 t + 15 of the block hold token t
    const int t = tid >> 4, j = tid & 15;
    const bool valid = t < T;
    const int loc = valid ? a.r.loc_in[t] : 0;
    const float qhat = valid ? a.r.qhat_in[t] : 0.f;
    for (int i = tid; i < T * Epad; i += FW_THREADS) s_logit[i] = a.logits[i];
    for (int i = tid; i < E; i += FW_THREADS) s_lidx[i] = a.lidx[i];
    for (int i = tid; i < (ORDERMOE_MAX_LOCAL + 1) * FW; i += FW_THREADS) (&s_w[0][0])[i] = 0.f;
    if (tid <= ORDERMOE_MAX_LOCAL) s_msk[tid] = 0u;
    if (tid < ORDERMOE_NUM_COUNTERS) s_cnt[tid] = 0;
    __syncthreads();
    if (4 * wave < T) {
        const TokenPick p = pick_token<NBT, ORDERMOE_MAX_TOPK>(a.r, s_logit + (valid ? t : 0) * Epad, a.r.t1_k, a.r.t1_q,
                                                               a.r.t1_n, a.r.srvmask, a.r.S, j, loc, qhat);
        const bool mine = valid && j < k;
        const float w = expf(p.v - p.top) / p.den;
        // the slots that run here; those of one expert merged, weights added in slot order
        const int ls = mine && p.loc_ok && p.m == a.server && p.k >= 0 && p.k < E ? s_lidx[p.k] : -1;
        float sum = w;
        bool again = false;
#pragma unroll
        for (int i = 0; i < ORDERMOE_MAX_TOPK; ++i) {
            const float wi = __shfl(w, i, 16);
            const bool same = __shfl(ls, i, 16) == ls;
            again |= same && i < j;
            if (same && i > j) sum = sum + wi;           // (a slot past k has ls = -1)
        }
        if (ls >= 0 && !again) {
            s_w[ls][t] = sum;
            atomicOr(&s_msk[ls], 1u << t);
        }
        if (valid && j == 0 && loc == a.server && a.n_shared > 0) {
            s_w[n_local][t] = 1.0f;
            atomicOr(&s_msk[n_local], 1u << t);
        }
        if (first) {
            const bool remote = p.m != loc;
            const int c = ((int)remote << 1) | (int)(p.k != p.r);
            const bool placed = mine && p.loc_ok;
            if (mine) {
                const int o = t * k + j;
                a.r.out.idx[o] = p.r;
                a.r.out.w[o] = w;
                a.r.out.exec_k[o] = p.loc_ok ? p.k : -1;
                a.r.out.exec_m[o] = p.loc_ok ? (uint8_t)p.m : 255;
                a.r.out.cls[o] = p.loc_ok ? (uint8_t)c : 255;
                s_dst[o] = placed && remote ? (int8_t)p.m : (int8_t)-1;
                if (placed) {
                    atomicAdd(&s_cnt[c], 1);
                    if (remote) atomicAdd(&s_cnt[ORDERMOE_CNT_REMOTE_SLOTS], 1);
                }
            }
            if (valid && j == 0) {
                const int fl = p.margin < ORDERMOE_MARGIN_FLAG;
                a.r.out.margin[t] = p.margin;
                a.r.out.flag[t] = (uint8_t)fl;
                a.r.out.qhat_out[t] = p.loc_ok ? p.qhat : qhat;
                a.r.out.loc_out[t] = p.loc_ok ? (uint8_t)p.first_m : (uint8_t)loc;
                if (fl) atomicAdd(&s_cnt[ORDERMOE_CNT_FLAGGED], 1);
                if (p.loc_ok) atomicAdd(&s_cnt[ORDERMOE_CNT_TRANSFERS], __builtin_popcount(p.dstmask));
                else atomicAdd(&s_cnt[ORDERMOE_CNT_INVALID], 1);
            }
        }
    }
    __syncthreads();
    if (first) write_route_totals(a, s_dst, s_cnt, tid);

    // ---- the groups in use
    const uint64_t used = __builtin_amdgcn_ballot_w64(lane < n_local && s_msk[lane < n_local ? lane : 0] != 0u);
    const int sh = a.n_shared > 0 && s_msk[n_local] != 0u ? 1 : 0;
    const int nu = __popcll(used);
    if (wave == 0) {
        if (lane == 0 && sh) s_grp[0] = n_local;
        if ((used >> lane) & 1) s_grp[sh + __popcll(used & ((1ull << lane) - 1ull))] = lane;
    }
    const int per = a.f / 16, per_sh = sh * a.n_shared * per;
    const int n_act = per_sh + nu * per, n_items = T > 0 ? n_act + d / 16 : 0;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.r.x, (uint32_t)T * (uint32_t)d * ES);
    bool ready = false;
    for (;;) {
        __syncthreads();
        if (tid == 0) s_item = next;
        __syncthreads();
        const int item = __builtin_amdgcn_readfirstlane(s_item);
        if (item >= n_items) break;
        // the following item is drawn now, its latency behind this one
        if (tid == 0) next = __hip_atomic_fetch_add(a.ctr, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (item < n_act) {
            // ---- activation tile: FFN columns c0 .. c0 + 15 of group grp
            const bool shared = item < per_sh;
            const int q = shared ? 0 : (item - per_sh) / per;
            const int c0 = 16 * (shared ? item : item - per_sh - q * per);
            const int grp = __builtin_amdgcn_readfirstlane(shared ? n_local : s_grp[sh + q]);
            const int F = shared ? a.n_shared * a.f : a.f;
            const char* W = shared ? (const char*)a.w_sh_gu : (const char*)a.w_gu + (size_t)grp * 2 * a.f * d * ES;
            const __amdgpu_buffer_rsrc_t rw = make_rsrc(W, (uint32_t)((size_t)2 * F * d * ES));
            // packed rows: gate columns in blocks of 32, each followed by its up columns
            const int row0 = 64 * (c0 / 32) + c0 % 32;
            const uint32_t wg = rows_offset<BF>(row0, d, lane), wu = rows_offset<BF>(row0 + 32, d, lane);
            const uint32_t msk = s_msk[grp];
            const uint32_t xo = (msk >> r16) & 1 ? (uint32_t)r16 * (uint32_t)d * ES + 16u * g16 : OOR;
            const int n = d / SK, ns = (n - wave + FW_WAVES - 1) / FW_WAVES;     // steps wave, wave + 4, ...
            u32x4 vg[2][U][2], vu[2][U][2], vx[2][U][2];
            auto load = [&](int b, int i0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t past = i0 + u < ns ? 0u : OOR;
                    const uint32_t s = (uint32_t)(i0 + u < ns ? wave + FW_WAVES * (i0 + u) : 0);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        vg[b][u][h] = load16<AUX>(rw, wg | past, s * STEP_BYTES<BF> + 64u * h);
                        vu[b][u][h] = load16<AUX>(rw, wu | past, s * STEP_BYTES<BF> + 64u * h);
                        vx[b][u][h] = load16(rx, xo | past, s * 128u + 64u * h);
                    }
                }
            };
            f32x4 ag = {0.f, 0.f, 0.f, 0.f}, au = {0.f, 0.f, 0.f, 0.f};
            auto mul = [&](int b) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        ag = mma<BF>(vg[b][u][h], vx[b][u][h], ag);
                        au = mma<BF>(vu[b][u][h], vx[b][u][h], au);
                    }
            };
            load(0, 0);
            for (int i = 0; i < ns; i += 2 * U) {
                load(1, i + U);
                __builtin_amdgcn_sched_barrier(0);
                mul(0);
                __builtin_amdgcn_sched_barrier(0);
                load(0, i + 2 * U);
                __builtin_amdgcn_sched_barrier(0);
                mul(1);
                __builtin_amdgcn_sched_barrier(0);
            }
            // element i of a lane: column 4 g16 + i of the tile, token r16
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s_red[wave][0][4 * g16 + i][r16] = ag[i];
                s_red[wave][1][4 * g16 + i][r16] = au[i];
            }
            __syncthreads();
            const int col = tid & 15, tok = tid >> 4;
            if ((msk >> tok) & 1) {
                float gv = 0.f, uv = 0.f;
#pragma unroll
                for (int w = 0; w < FW_WAVES; ++w) { gv += s_red[w][0][col][tok]; uv += s_red[w][1][col][tok]; }
                const float v = silu<BF>(gv) * uv * s_w[grp][tok];
                const size_t o = shared ? (size_t)tok * F + c0 + col : ((size_t)grp * FW + tok) * F + c0 + col;
                if constexpr (BF) ((__bf16*)(shared ? a.act_s : a.act_r))[o] = (__bf16)v;
                else ((float*)(shared ? a.act_s : a.act_r))[o] = v;
            }
            // every wave's activations are in memory for every XCD before the tile counts as finished
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
            __syncthreads();
            if (tid == 0) __hip_atomic_fetch_add(a.ctr + 1, 1, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_AGENT);
            continue;
        }
        // ---- output tile: columns d0 .. d0 + 15 of y
        const int d0 = 16 * (item - n_act), ng = sh + nu;
        const int n_r = a.f / SK, n_s = a.n_shared * n_r;    // steps of a routed group, of the shared one
        // this wave's steps wave, wave + 4, ... of the groups' steps one after the other
        struct Pos { int q, s; };                            // group (of those in use), step in it
        auto norm = [&](Pos& p) {
            while (p.q < ng) {
                const int n = p.q < sh ? n_s : n_r;
                if (p.s < n) break;
                p.s -= n;
                ++p.q;
            }
        };
        u32x4 vw[2][U][2], va[2][U][2];
        Pos pw{0, wave}, pa{0, wave};
        auto load_w = [&](int b) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                norm(pw);
                const bool in = pw.q < ng;
                const int grp = __builtin_amdgcn_readfirstlane(s_grp[in ? pw.q : 0]);
                const bool shared = in && pw.q < sh;
                const int F = shared ? a.n_shared * a.f : a.f;
                const char* W = shared ? (const char*)a.w_sh_dn : (const char*)a.w_dn + (size_t)(in ? grp : 0) * a.f * d * ES;
                const __amdgpu_buffer_rsrc_t rw = make_rsrc(W, (uint32_t)((size_t)F * d * ES));
                const uint32_t wo = in ? rows_offset<BF>(d0, F, lane) : OOR;
#pragma unroll
                for (int h = 0; h < 2; ++h) vw[b][u][h] = load16<AUX>(rw, wo, (uint32_t)(in ? pw.s : 0) * STEP_BYTES<BF> + 64u * h);
                pw.s += FW_WAVES;
            }
        };
        auto load_a = [&](int b) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                norm(pa);
                const bool in = pa.q < ng;
                const int grp = __builtin_amdgcn_readfirstlane(s_grp[in ? pa.q : 0]);
                const bool shared = in && pa.q < sh;
                const int F = shared ? a.n_shared * a.f : a.f;
                const char* A = shared ? (const char*)a.act_s : (const char*)a.act_r + (size_t)(in ? grp : 0) * FW * a.f * ES;
                const __amdgpu_buffer_rsrc_t ra = make_rsrc(A, (uint32_t)FW * (uint32_t)F * ES);
                const bool has = in && ((s_msk[grp] >> r16) & 1);
                const uint32_t ao = has ? (uint32_t)r16 * (uint32_t)F * ES + 16u * g16 : OOR;
#pragma unroll
                for (int h = 0; h < 2; ++h) va[b][u][h] = load16(ra, ao, (uint32_t)(in ? pa.s : 0) * 128u + 64u * h);
                pa.s += FW_WAVES;
            }
        };
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        auto mul = [&](int b) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc = mma<BF>(vw[b][u][h], va[b][u][h], acc);
        };
        const int total = sh * n_s + nu * n_r, ns = (total - wave + FW_WAVES - 1) / FW_WAVES;
        load_w(0);
        load_w(1);
        if (!ready) {
            // all activation tiles have been drawn by running workgroups (they precede
            // this item on the counter) and wait for nothing: this ends
            if (tid == 0) {
                while (__hip_atomic_load(a.ctr + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < n_act) __builtin_amdgcn_s_sleep(1);
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
            }
            __syncthreads();
            ready = true;
        }
        load_a(0);
        for (int i = 0; i < ns; i += 2 * U) {
            load_a(1);
            __builtin_amdgcn_sched_barrier(0);
            mul(0);
            __builtin_amdgcn_sched_barrier(0);
            load_w(0);
            load_a(0);
            __builtin_amdgcn_sched_barrier(0);
            mul(1);
            __builtin_amdgcn_sched_barrier(0);
            load_w(1);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s_red[wave][0][4 * g16 + i][r16] = acc[i];
        __syncthreads();
        const int col = tid & 15, tok = tid >> 4;
        if (tok < T) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < FW_WAVES; ++w) v += s_red[w][0][col][tok];
            const size_t o = (size_t)tok * d + d0 + col;
            if constexpr (BF) ((__bf16*)a.y)[o] = (__bf16)v;
            else ((float*)a.y)[o] = v;
        }
    }
}

template <bool BF, int NBT, int AUX>
int launch_layer(const FewArgs& a, hipStream_t st) {
    // never more workgroups than items: a tile of every group that can be in use
    const int64_t groups = a.r.T * (a.r.k < a.n_local ? a.r.k : a.n_local);
    const int64_t act = ((groups < a.n_local ? groups : a.n_local) + a.n_shared) * (a.f / 16);
    const int64_t items = a.r.T > 0 ? act + a.r.d / 16 : 1;
    const int64_t most = 256 * FW_PER_CU;
    KernelTimer kt_("few_layer", st);
    few_layer_kernel<BF, NBT, AUX><<<dim3((unsigned)(items < most ? items : most)), dim3(FW_THREADS), 0, st>>>(a);
    return (int)hipGetLastError();
}

template <bool BF, int AUX>
int launch_experts(const FewArgs& a, hipStream_t st) {
    const int nb = (a.r.E + 15) / 16;
    if (nb <= 1) return launch_layer<BF, 1, AUX>(a, st);
    if (nb <= 4) return launch_layer<BF, 4, AUX>(a, st);
    if (nb <= 8) return launch_layer<BF, 8, AUX>(a, st);
    return launch_layer<BF, 16, AUX>(a, st);
}

}  // namespace

int launch_few_layer(const FewArgs& a, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    const int nb = (a.r.E + 15) / 16;
    {
        KernelTimer kt_("few_router", st);
        few_router_kernel<<<dim3((unsigned)nb), dim3(FW_SLICES * 64), 0, st>>>(a, route_ksplit(1, nb, a.r.d));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    if (a.r.dtype != ORDERMOE_BF16) return launch_experts<false, 0>(a, st);
    const bool stream_w = (int64_t)a.n_local * 2 * a.f * a.r.d * 2 >= FW_STREAM_BYTES;
    return stream_w ? launch_experts<true, NT>(a, st) : launch_experts<true, 0>(a, st);
}

}  // namespace ordermoe
