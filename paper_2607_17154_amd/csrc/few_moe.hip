// The whole MoE layer of one server for at most ORDERMOE_MAX_FEW = 16 tokens:
//   l = x W_r^T, the routing decisions of route_select on l, and
//   y[t] = sum over the slots of t executed here of w (silu(x G^T) * x U^T) D^T
//          + the shared experts of the tokens that are at home here.
//
//   few_router_kernel  sums of l over K slices: a wave per (16 experts, slice), the
//                      slices of the split router of small batches, so that added in
//                      the same order they are the same logits; clears the counters
//   few_layer_kernel   everything else, in at most FW_SHARES workgroups.  Each adds the
//                      router's slices and runs the token stage of the routing itself (about
//                      5 us of latency, side by side; the first one writes the routing's
//                      outputs), which tells it the experts in use and their tokens.
//                      Then it works through its share of two lists:
//     activation tiles   32 FFN columns of one expert: gate and up rows times the
//                        tokens, silu(g) u w -> the weighted activations (memory)
//     output tiles       64 output columns: the down rows of every expert in use times
//                        its weighted activations, summed over the experts in one
//                        accumulator, in up to 16 pieces along the experts' columns whose
//                        sums the last one to finish adds in order -> y
// An output tile needs all activations.  A workgroup waits for them only after its own
// share's activation tiles and those of every share that no workgroup has drawn yet,
// so all waits end whatever else runs on the GPU.  It reads the first weights of its
// output tile before it waits, so that the weight stream does not stop in between.
// The 16 tokens are the columns of one v_mfma_f32_16x16x32_bf16 (fp32:
// v_mfma_f32_16x16x4_f32), the weights its rows, read in whole cache lines and turned
// into the operand's lane order through LDS.
// Bound: the weights in use, read once; below some 100 MB of them the latency of router,
// token stage and hand-over and of the weight stream's start.  d 4096, f 1536, bf16, both
// kernels: 16 tokens with 24 experts in use (906 MB) 170 us, 5.3 TB/s; 1 token with 2 (75 MB)
// 36.7 us.  The layer kernel's workgroups by their clocks, us from their start (the router's
// kernel takes 2.6 before):
//                                  logits  token stage  activations  all done  outputs  end
//   1 token                          2.7       5.2        1 to 18       26      4.7-7     35
//   16 tokens                        4.3       7.9       66 to 103     113      35-47    161
//   5, f 1408, two shared experts    2.5       4.5       10 to 20       27      3.7-7     37
//   8, fp32, d 512, f 1024           2.6       2.6        1 to 8        14      4.8-6     20
// route_select and local_moe_forward in turn on the same card: 184 and 51 us (16 tokens, 1),
// 57 for 36.9 and 45 for 24 (the last two).
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
constexpr int FW_WAVES = 8, FW_THREADS = 64 * FW_WAVES;
constexpr int FW_ITEMS = 256;                     // output items wished for
constexpr int FW_PIECES = 16;                     // pieces of an output tile, at most
constexpr int FW_XCDS = 8;
// shares of the work, at most: a workgroup of 8 waves per CU (512 of 4 waves: 16 tokens 183 us, these 172)
constexpr int FW_SHARES = 256;
// Counters, each in a cache line of its own: atomics on one line take turns, 50 ns each here (drawing every
// item from one counter cost 24 us with 768 workgroups).  Per XCD: shares drawn, shares whose activations are
// done, the signal that all are; then the XCDs that are done, and the finished pieces of each output tile.
constexpr int LINE = 16;
constexpr int CTR_DRAWN = 0, CTR_DONE = FW_XCDS, CTR_ALL = 2 * FW_XCDS, CTR_XCDS = 3 * FW_XCDS, CTR_TILE = 3 * FW_XCDS + 1;
constexpr int FW_SLICES = 16;                     // K slices of the router, at most
constexpr uint32_t OOR = 0x80000000u;             // past every buffer: reads zeros
constexpr int NT = 2;                             // buffer load cache bit nt: non-temporal
constexpr int SC1 = 16;                           // buffer store cache bit sc1: through to where every XCD reads
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
// Partial logits of 16 experts over the K slice [z kc, (z + 1) kc), by one wave:
// bf16 v_mfma_f32_16x16x32_bf16 (element i of a lane: token 4 g + i), fp32
// v_mfma_f64_16x16x4_f64 (token 4 i + g, exact products); expert lane % 16.
template <bool BF>
__device__ inline auto router_slice(const FewArgs& a, int eb, int z, int kc, int lane) {
    constexpr uint32_t ES = BF ? 2 : 4;
    constexpr int U = BF ? 8 : 4, SK = BF ? 32 : 16;         // steps in flight, columns of a step
    const int r16 = lane & 15, g = lane >> 4;
    const int E = a.r.E, d = a.r.d, T = (int)a.r.T, e = eb * 16 + r16;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.r.x, (uint32_t)T * (uint32_t)d * ES);
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.r.w_router, (uint32_t)E * (uint32_t)d * ES);
    const uint32_t xo = r16 < T ? (uint32_t)r16 * (uint32_t)d * ES + 16u * g : OOR;
    const uint32_t wo = e < E ? (uint32_t)e * (uint32_t)d * ES + 16u * g : OOR;
    std::conditional_t<BF, f32x4, f64x4> acc = {};
    const int n = kc / SK;
    for (int s0 = 0; s0 < n; s0 += U) {
        u32x4 xv[U], wv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t past = s0 + u < n ? 0u : OOR, so = (uint32_t)(z * kc + (s0 + u < n ? s0 + u : 0) * SK) * ES;
            xv[u] = load16(rx, xo | past, so);
            wv[u] = load16(rw, wo | past, so);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (BF) {
                acc = mma<true>(xv[u], wv[u], acc);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)__uint_as_float(xv[u][i]), (double)__uint_as_float(wv[u][i]),
                                                               acc, 0, 0, 0);
            }
        }
    }
    return acc;
}

// a wave per (16 experts, slice); workgroup 0 clears the layer kernel's counters
template <bool BF>
__global__ void __launch_bounds__(64) few_router_kernel(const FewArgs a, int ks) {
    using V = std::conditional_t<BF, float, double>;
    const int lane = threadIdx.x, r16 = lane & 15, g = lane >> 4, Epad = (a.r.E + 15) & ~15;
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = lane; i < (CTR_TILE + a.r.d / 64) * LINE; i += 64) a.ctr[i] = 0;
    const auto acc = router_slice<BF>(a, blockIdx.x, blockIdx.y, a.r.d / ks, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = BF ? 4 * g + i : 4 * i + g;
        if (t < a.r.T) ((V*)a.logits)[((int)blockIdx.y * FW + t) * Epad + blockIdx.x * 16 + r16] = acc[i];
    }
}

// ------------------------------------------------------------------ layer
// silu(g) = g / (1 + e^-g); bf16 with the hardware reciprocal, as the result is rounded right after
template <bool BF>
__device__ inline float silu(float g) {
    if constexpr (BF) return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g));
    else return g / (1.0f + expf(-g));
}

// A matrix [N][K] of weights as the packed layout has it, read in steps of 64 (bf16)
// or 32 (fp32) columns, 128 bytes of a row: one read of a wave covers 8 rows, whole
// cache lines (lane: row lane / 8, 16 bytes at 16 (lane % 8)).  Byte offset of the
// lane's part of the 8 rows from row0 (a multiple of 8), and of a step.
template <bool BF>
__device__ inline uint32_t rows_offset(int row0, int K, int lane) {
    const uint32_t r = (uint32_t)(row0 + (lane >> 3)), ch = (uint32_t)(lane & 7);
    if constexpr (BF) return (r / 256u) * (uint32_t)(K / 64) * 32768u + (r % 256u) * 128u + ch * 16u;
    else return r * (uint32_t)K * 4u + ch * 16u;
}
template <bool BF>
constexpr uint32_t STEP_BYTES = BF ? 32768u : 128u;

// From that order to the operand's (lane: row lane % 16, 16 bytes at 16 (lane / 16)
// of either half of the row's 128) through the wave's own LDS rows, padded so that
// 8 rows' reads fall on distinct banks.  (Reading memory in the operand's order asks
// for half a line at a time, and a CU has so many requests in flight: 16 tokens of the
// 128-expert layer took 312 us.)
constexpr int ROW_LD = 144;

// The candidate tables in LDS, in the place of the staging rows, which are not in use yet: the selection reads them in
// a chain (an expert's row, its substitutes' servers, each server's cost).
constexpr int TAB_T1 = ORDERMOE_MAX_EXPERTS * ORDERMOE_MAX_SUBS, TAB_S = 8192;      // words of t1_k, t1_q; of S at most
constexpr int TAB_READS = (TAB_T1 / 4 + FW_THREADS - 1) / FW_THREADS, TAB_S_READS = TAB_S / 4 / FW_THREADS;
static_assert((2 * TAB_T1 + 2 * ORDERMOE_MAX_EXPERTS + TAB_S) * 4 <= FW_WAVES * 64 * ROW_LD, "the tables fit in the staging rows");
// where the selection reads them: there or in memory
struct Tables {
    const int32_t* k;
    const float* q;
    const int32_t* n;
    const uint32_t* mask;
    const float* S;
};

// pick_token's decisions, bit for bit, in loops that are not unrolled and with the slots' searches side by side: the
// kernel runs this code once, so that fetching its instructions counts (one token of 128 experts, top-8: pick_token,
// 20 KB of instructions, 7.6 us; this, with the tables in LDS, 5.3).  Three parts, with the workgroup's barriers
// between them: targets, searches, and the choice (in the kernel).
struct FewPick {
    int r;                   // lane j: slot j's target
    float v, top, den, margin;
};
// by the 16 lanes of a token: the targets in rank order, gates and margin
template <int NBT>
__device__ inline FewPick few_top(const RouteArgs& a, const float* lg, int j) {
    const int E = a.E, k = a.k, kk1 = k + 1 < E ? k + 1 : E;
    uint32_t okey[NBT];
#pragma unroll
    for (int i = 0; i < NBT; ++i) {
        const int e = j + 16 * i;
        const uint32_t o = f2ord(lg[e < E ? e : E - 1]);
        okey[i] = e < E ? (o > 1u ? o : 1u) : 0u;
    }
    FewPick p{0, 0.f, 0.f, 0.f, __builtin_inff()};
    float last = 0.f;
#pragma unroll 1
    for (int r = 0; r < kk1; ++r) {
        uint32_t mx = okey[0];
#pragma unroll
        for (int i = 1; i < NBT; ++i) mx = okey[i] > mx ? okey[i] : mx;
        mx = row_max_u32(mx);
        uint32_t e = 0xFFFFu;
#pragma unroll
        for (int i = NBT - 1; i >= 0; --i) e = okey[i] == mx ? (uint32_t)(j + 16 * i) : e;
        e = row_min_u32(e);
#pragma unroll
        for (int i = 0; i < NBT; ++i) okey[i] = e == (uint32_t)(j + 16 * i) ? 0u : okey[i];
        const float v = ord2f(mx);
        if (r == 0) p.top = v;
        else p.margin = last - v < p.margin ? last - v : p.margin;
        last = v;
        if (r < k && a.renorm) p.den += expf(v - p.top);
        if (j == r) { p.r = (int)e; p.v = v; }
    }
    if (!a.renorm) {
#pragma unroll 1
        for (int e = j; e < E; e += 16) p.den += expf(lg[e] - p.top);
        p.den = __shfl(row_sum_f32(p.den), 0, 16);
    }
    return p;
}
// by 16 lanes per (token, slot): the best server of each candidate (lane j: candidate j) of target r; false: no search,
// the target runs where the token is
__device__ inline bool few_search(const RouteArgs& a, const Tables& tb, int r, int loc, int j, uint64_t& key, float& q) {
    const int E = a.E, M = a.M;
    const bool subs_on = a.allow_sub && a.Qbar > 0.f;
    const uint32_t mmask = M >= 32 ? 0xFFFFFFFFu : ((1u << M) - 1u);
    const int jm1 = j >= 1 && j - 1 < a.gmax ? j - 1 : 0;
    const uint32_t rmask = tb.mask[r];
    const int nsub = tb.n[r], tk = tb.k[r * a.gmax + jm1];
    const float tq = tb.q[r * a.gmax + jm1];
    const bool search = loc < M && !(a.pin && ((rmask >> loc) & 1u)), sub = j >= 1 && subs_on && j - 1 < nsub;
    int kc = j == 0 ? r : (sub ? tk : -1);
    if (kc < 0 || kc >= E) kc = -1;
    q = sub ? tq : 0.f;
    key = ~0ull;
    const uint32_t lmask = a.allow_sub == 2 && j >= 1 ? 1u << (loc & 31) : ~0u;
    uint32_t on = search && kc >= 0 ? tb.mask[kc] & mmask & lmask : 0u;
#pragma unroll 1
    while (__builtin_amdgcn_ballot_w64(on != 0)) {
        if (on) {
            const int m = __builtin_ctz(on);
            on &= on - 1;
            const float J = fmaf(a.cq, q, tb.S[((int64_t)loc * M + m) * E + kc]);
            const uint64_t cand = ((uint64_t)f2ord(J == 0.f ? 0.f : J) << 32) | ((uint32_t)j << 16) | ((uint32_t)(m != loc) << 15) |
                                  ((uint32_t)m << 8) | (uint32_t)kc;
            key = cand < key ? cand : key;
        }
    }
    return search;
}

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
__global__ void __launch_bounds__(FW_THREADS) few_layer_kernel(const FewArgs a, int ks, int tables) {
    constexpr int SK = BF ? 64 : 32;                         // columns of a step
    constexpr uint32_t ES = BF ? 2 : 4;
    __shared__ float s_logit[FW * NBT * 16];
    __shared__ int32_t s_lidx[ORDERMOE_MAX_EXPERTS];
    __shared__ float s_w[ORDERMOE_MAX_LOCAL + 1][FW];        // gate weight of (group, token)
    __shared__ uint32_t s_msk[ORDERMOE_MAX_LOCAL + 1];       // tokens of a group
    __shared__ int32_t s_grp[ORDERMOE_MAX_LOCAL + 1];        // the groups in use, the shared one first
    __shared__ int8_t s_dst[FW * ORDERMOE_MAX_TOPK];
    __shared__ int32_t s_cnt[ORDERMOE_NUM_COUNTERS];
    __shared__ __attribute__((aligned(16))) float s_red[FW_WAVES][4][16][17];
    __shared__ __attribute__((aligned(16))) char s_stage[FW_WAVES][64 * ROW_LD];
    __shared__ int32_t s_item;
    __shared__ int32_t s_share[FW_SHARES];                   // shares of this workgroup: XCD << 16 | number
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g16 = lane >> 4;
    const int T = (int)a.r.T, E = a.r.E, k = a.r.k, d = a.r.d, n_local = a.n_local;
    const int Epad = (E + 15) & ~15;
    const bool first = blockIdx.x == 0;
    auto add = [&](int c) { return __hip_atomic_fetch_add(a.ctr + c * LINE, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    auto look = [&](int c) { return __hip_atomic_load(a.ctr + c * LINE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    // this workgroup's share, drawn among those of its XCD (workgroups go to the XCDs in turn; where they do not,
    // only locality is lost)
    const int grid = (int)gridDim.x, per_xcd = grid / FW_XCDS;
    int drawn = 0;
    if (tid == 0) drawn = add(CTR_DRAWN + (int)(blockIdx.x % FW_XCDS));

    // ---- token stage: lanes 16 t .. 16 t + 15 of the block hold token t
    const int t = tid >> 4, j = tid & 15;
    const bool valid = t < T;
    const int loc = valid ? a.r.loc_in[t] : 0;
    const float qhat = valid ? a.r.qhat_in[t] : 0.f;
    // tables: 16-byte reads of each (tables & 2: of S too), on their way while the logits are added
    const int n_t1 = E * a.r.gmax, n_S = tables & 2 ? a.r.M * a.r.M * E : 0;
    u32x4 vk[TAB_READS] = {}, vq[TAB_READS] = {}, vS[TAB_S_READS] = {}, vn = {}, vm = {};
    if (tables) {
#pragma unroll
        for (int u = 0; u < TAB_READS; ++u) {
            const int i = 4 * (tid + FW_THREADS * u);
            if (i < n_t1) {
                vk[u] = *(const u32x4*)(a.r.t1_k + i);
                vq[u] = *(const u32x4*)(a.r.t1_q + i);
            }
        }
        if (4 * tid < E) {
            vn = *(const u32x4*)(a.r.t1_n + 4 * tid);
            vm = *(const u32x4*)(a.r.srvmask + 4 * tid);
        }
#pragma unroll
        for (int u = 0; u < TAB_S_READS; ++u) {
            const int i = 4 * (tid + FW_THREADS * u);
            if (i < n_S) vS[u] = *(const u32x4*)(a.r.S + i);
        }
    }
    for (int i = tid; i < T * Epad; i += FW_THREADS) {       // logits: the router's slices, added in order
        using V = std::conditional_t<BF, float, double>;
        const V* q = (const V*)a.logits + i;
        V part[FW_SLICES], v = 0;
#pragma unroll
        for (int z = 0; z < FW_SLICES; ++z) part[z] = q[(z < ks ? z : 0) * FW * Epad];
#pragma unroll
        for (int z = 0; z < FW_SLICES; ++z)
            if (z < ks) v += part[z];
        s_logit[i] = (float)v;
    }
    for (int i = tid; i < E; i += FW_THREADS) s_lidx[i] = a.lidx[i];
    for (int i = tid; i < (ORDERMOE_MAX_LOCAL + 1) * FW; i += FW_THREADS) (&s_w[0][0])[i] = 0.f;
    if (tid <= ORDERMOE_MAX_LOCAL) s_msk[tid] = 0u;
    if (tid < ORDERMOE_NUM_COUNTERS) s_cnt[tid] = 0;
    Tables tb{a.r.t1_k, a.r.t1_q, a.r.t1_n, a.r.srvmask, a.r.S};
    if (tables) {
        int32_t* const l_k = (int32_t*)&s_stage[0][0];
        float* const l_q = (float*)(l_k + TAB_T1);
        int32_t* const l_n = (int32_t*)(l_q + TAB_T1);
        uint32_t* const l_m = (uint32_t*)(l_n + ORDERMOE_MAX_EXPERTS);
        float* const l_S = (float*)(l_m + ORDERMOE_MAX_EXPERTS);
#pragma unroll
        for (int u = 0; u < TAB_READS; ++u) {
            const int i = 4 * (tid + FW_THREADS * u);
            if (i < n_t1) {
                *(u32x4*)(l_k + i) = vk[u];
                *(u32x4*)(l_q + i) = vq[u];
            }
        }
        if (4 * tid < E) {
            *(u32x4*)(l_n + 4 * tid) = vn;
            *(u32x4*)(l_m + 4 * tid) = vm;
        }
#pragma unroll
        for (int u = 0; u < TAB_S_READS; ++u) {
            const int i = 4 * (tid + FW_THREADS * u);
            if (i < n_S) *(u32x4*)(l_S + i) = vS[u];
        }
        tb = Tables{l_k, l_q, l_n, l_m, tables & 2 ? l_S : a.r.S};
    }
    // (targets, and what the searches find, in the place of the partial sums)
    uint64_t* const s_key = (uint64_t*)&s_red[0][0][0][0];       // [slot of a token][16]
    float* const s_q = (float*)(s_key + FW * ORDERMOE_MAX_TOPK * 16);
    int32_t* const s_sel = (int32_t*)(s_q + FW * ORDERMOE_MAX_TOPK * 16);
    uint8_t* const s_try = (uint8_t*)(s_sel + FW * ORDERMOE_MAX_TOPK);
    uint8_t* const s_loc = s_try + FW * ORDERMOE_MAX_TOPK;
    static_assert(FW * ORDERMOE_MAX_TOPK * (16 * 12 + 5) + FW <= (int)sizeof(s_red), "the searches fit");
    __syncthreads();
    FewPick f{};
    if (4 * wave < T) {
        f = few_top<NBT>(a.r, s_logit + (valid ? t : 0) * Epad, j);
        if (valid && j < k) s_sel[t * k + j] = f.r;
        if (valid && j == 0) s_loc[t] = (uint8_t)loc;
    }
    __syncthreads();
#pragma unroll 1
    for (int i = t; i < T * k; i += FW_THREADS / 16) {
        uint64_t key;
        float q;
        const bool search = few_search(a.r, tb, s_sel[i], s_loc[i / k], j, key, q);
        s_key[i * 16 + j] = key;
        s_q[i * 16 + j] = q;
        if (j == 0) s_try[i] = search;
    }
    __syncthreads();
    if (4 * wave < T) {
        TokenPick p;
        p.r = f.r; p.k = 0; p.m = loc;
        p.v = f.v; p.top = f.top; p.den = f.den; p.margin = f.margin;
        p.qhat = qhat; p.first_m = loc; p.dstmask = 0; p.loc_ok = loc < a.r.M;
        // the slots in rank order: eq (40)'s budget, the choice of eq (43), the update of eq (44)
#pragma unroll 1
        for (int slot = 0; slot < k; ++slot) {
            const int i = (valid ? t : 0) * k + slot;
            int km = __shfl(f.r, slot, 16), mm = loc;
            float qsel = 0.f;
            if (s_try[i]) {
                const float q = s_q[i * 16 + j];
                uint64_t kk = (j == 0 || p.qhat + q <= a.r.Qbar) ? s_key[i * 16 + j] : ~0ull;
                kk = row_min_u64(kk);
                const int pos = (int)((kk >> 16) & 15u);
                mm = (int)((kk >> 8) & 31u);
                km = (int)(kk & 0xFFu);
                qsel = row_sum_f32(j == pos ? q : 0.f);
            }
            p.qhat += qsel;
            if (slot == 0) p.first_m = mm;
            if (mm != loc) p.dstmask |= 1u << mm;
            if (j == slot) { p.k = km; p.m = mm; }
        }
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
    const int per = a.f / 32, per_sh = sh * a.n_shared * per;
    const int n_r = a.f / SK, n_s = a.n_shared * n_r;        // steps of a routed group's down rows, of the shared one's
    const int total = sh * n_s + nu * n_r;
    // output tiles are cut into pieces along the groups' columns, enough for the chip but of FW_WAVES steps at least
    const int tiles = d / 64;
    const int n_act = per_sh + nu * per;
    int pieces = FW_ITEMS / tiles;
    pieces = pieces > FW_PIECES ? FW_PIECES : pieces;
    pieces = pieces > total / FW_WAVES ? total / FW_WAVES : pieces;
    pieces = pieces < 1 ? 1 : pieces;
    const int n_out = T > 0 ? tiles * pieces : 0;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.r.x, (uint32_t)T * (uint32_t)d * ES);
    char* const put = s_stage[wave] + (lane >> 3) * ROW_LD + (lane & 7) * 16;
    const char* const get = s_stage[wave] + r16 * ROW_LD + g16 * 16;
    // item `round` of share (x, j) among n: every XCD's shares get neighbouring items; the last, partial round is
    // spread evenly over the XCDs
    auto item_of = [&](int x, int j, int round, int n) {
        const int left = n - round * grid;
        if (left >= grid) return round * grid + x * per_xcd + j;
        const int lo = x * (left > 0 ? left : 0) / FW_XCDS, hi = (x + 1) * (left > 0 ? left : 0) / FW_XCDS;
        return j < hi - lo ? round * grid + lo + j : -1;
    };
    // Activation tiles of this workgroup's share, then of shares that nobody has drawn (their workgroups have not
    // started: they will find no share left and leave).  So when a workgroup begins to wait, every share is in the
    // hands of a running workgroup that finishes its activation tiles before it waits for anything: all waits end,
    // whatever else runs on the GPU.
    int own = 0;
    if (tid == 0) s_item = drawn < per_xcd ? (int)(blockIdx.x % FW_XCDS) << 16 | drawn : -1;
    __syncthreads();
    int share = __builtin_amdgcn_readfirstlane(s_item);
    for (;;) {
        if (share >= 0) {
            if (tid == 0) s_share[own] = share;
            ++own;
            const int sx = share >> 16, sj = share & 0xFFFF;
            int item = item_of(sx, sj, 0, n_act);
            const bool some = item >= 0;
            for (int round = 1; item >= 0; item = item_of(sx, sj, round++, n_act)) {
            // ---- activation tile: FFN columns c0 .. c0 + 31 of group grp
            constexpr int UA = 1;                            // steps per set of reads
            const bool shared = item < per_sh;
            const int q = shared ? 0 : (item - per_sh) / per;
            const int c0 = 32 * (shared ? item : item - per_sh - q * per);
            const int grp = __builtin_amdgcn_readfirstlane(shared ? n_local : s_grp[sh + q]);
            const int F = shared ? a.n_shared * a.f : a.f;
            const char* W = shared ? (const char*)a.w_sh_gu : (const char*)a.w_gu + (size_t)grp * 2 * a.f * d * ES;
            const __amdgpu_buffer_rsrc_t rw = make_rsrc(W, (uint32_t)((size_t)2 * F * d * ES));
            // packed rows: gate columns in blocks of 32, each followed by its up columns
            uint32_t wo[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) wo[i] = rows_offset<BF>(2 * c0 + 8 * i, d, lane);
            const uint32_t msk = s_msk[grp];
            const uint32_t xo = (msk >> r16) & 1 ? (uint32_t)r16 * (uint32_t)d * ES + 16u * g16 : OOR;
            const int n = d / SK, ns = (n - wave + FW_WAVES - 1) / FW_WAVES;     // steps wave, wave + 8, ...
            u32x4 vw[2][UA][8], vx[2][UA][2];
            auto load = [&](int b, int i0) {
#pragma unroll
                for (int u = 0; u < UA; ++u) {
                    const uint32_t past = i0 + u < ns ? 0u : OOR;
                    const uint32_t s = (uint32_t)(i0 + u < ns ? wave + FW_WAVES * (i0 + u) : 0);
#pragma unroll
                    for (int i = 0; i < 8; ++i) vw[b][u][i] = load16<AUX>(rw, wo[i] | past, s * STEP_BYTES<BF>);
#pragma unroll
                    for (int h = 0; h < 2; ++h) vx[b][u][h] = load16(rx, xo | past, s * 128u + 64u * h);
                }
            };
            f32x4 acc[4] = {};                               // gate columns 0-15, 16-31, up columns 0-15, 16-31
            auto mul = [&](int b) {
#pragma unroll
                for (int u = 0; u < UA; ++u) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) *(u32x4*)(put + 8 * i * ROW_LD) = vw[b][u][i];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            acc[r] = mma<BF>(*(const u32x4*)(get + 16 * r * ROW_LD + 64 * h), vx[b][u][h], acc[r]);
                }
            };
            load(0, 0);
            for (int i = 0; i < ns; i += 2 * UA) {
                load(1, i + UA);
                __builtin_amdgcn_sched_barrier(0);
                mul(0);
                __builtin_amdgcn_sched_barrier(0);
                load(0, i + 2 * UA);
                __builtin_amdgcn_sched_barrier(0);
                mul(1);
                __builtin_amdgcn_sched_barrier(0);
            }
            // element i of a lane: column 4 g16 + i of the 16, token r16
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) s_red[wave][r][4 * g16 + i][r16] = acc[r][i];
            __syncthreads();
            const __amdgpu_buffer_rsrc_t ra = make_rsrc(shared ? (char*)a.act_s : (char*)a.act_r + (size_t)grp * FW * F * ES,
                                                        (uint32_t)FW * (uint32_t)F * ES);
            const int col = tid & 15, r = (tid >> 4) & 1, tok = tid >> 5;
            if ((msk >> tok) & 1) {
                float gv = 0.f, uv = 0.f;
#pragma unroll
                for (int w = 0; w < FW_WAVES; ++w) { gv += s_red[w][r][col][tok]; uv += s_red[w][2 + r][col][tok]; }
                const float v = silu<BF>(gv) * uv * s_w[grp][tok];
                const uint32_t o = ((uint32_t)tok * (uint32_t)F + c0 + 16 * r + col) * ES;
                if constexpr (BF)
                    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (__bf16)v), ra, (int)o, 0, SC1);
                else
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), ra, (int)o, 0, SC1);
            }
            // every wave's stores have been acknowledged before the tile counts as finished
            // (written through: a release fence would write back the whole L2 for them)
            __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0)
            __syncthreads();
            }
            if (some && tid == 0) {
                // shares of the XCD that have activation tiles
                auto with = [&](int x) { return n_act >= grid ? per_xcd : (x + 1) * n_act / FW_XCDS - x * n_act / FW_XCDS; };
                if (add(CTR_DONE + sx) == with(sx) - 1) {
                    int xcds = 0;
                    for (int x = 0; x < FW_XCDS; ++x) xcds += with(x) > 0;
                    if (add(CTR_XCDS) == xcds - 1)
                        for (int x = 0; x < FW_XCDS; ++x)
                            __hip_atomic_store(a.ctr + (CTR_ALL + x) * LINE, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
            }
        }
        // a share that nobody has drawn
        __syncthreads();
        if (wave == 0) {
            const uint64_t open = __builtin_amdgcn_ballot_w64(lane < FW_XCDS && look(CTR_DRAWN + (lane < FW_XCDS ? lane : 0)) < per_xcd);
            int f = open ? -2 : -1;
            if (open && lane == 0) {
                const int x = __builtin_ctzll(open), t = add(CTR_DRAWN + x);
                if (t < per_xcd) f = x << 16 | t;
            }
            if (lane == 0) s_item = f;
        }
        __syncthreads();
        share = __builtin_amdgcn_readfirstlane(s_item);
        if (share == -1) break;                              // (-2: another workgroup was first, look again)
    }
    bool ready = n_act == 0;
    for (int o = 0; o < own; ++o) {
      const int sh_o = __builtin_amdgcn_readfirstlane(s_share[o]);
      // (from the other end: shares without activation tiles take output items first)
      const int ox = sh_o >> 16, oj = per_xcd - 1 - (sh_o & 0xFFFF);
      int item = item_of(ox, oj, 0, n_out);
      for (int round = 1; item >= 0; item = item_of(ox, oj, round++, n_out)) {
        // ---- output tile: columns d0 .. d0 + 63 of y, piece sp of the groups' steps one after the other
        constexpr int UD = 1;
        const int tile = item % tiles, sp = item / tiles;
        const int d0 = 64 * tile;
        const int lo = (int)((int64_t)total * sp / pieces), hi = (int)((int64_t)total * (sp + 1) / pieces);
        const int ns = (hi - lo - wave + FW_WAVES - 1) / FW_WAVES;               // steps lo + wave, lo + wave + 8, ...
        struct Pos { int q, s, left; };                      // group (of those in use), step in it, steps left
        auto norm = [&](Pos& p) {
            while (p.left > 0) {
                const int n = p.q < sh ? n_s : n_r;
                if (p.s < n) break;
                p.s -= n;
                ++p.q;
            }
        };
        u32x4 vw[2][UD][8], va[2][UD][2];
        bool runs[2][UD];                                    // the lane's token runs in the step's group
        Pos pw{0, lo + wave, ns}, pa = pw;
        auto load_w = [&](int b) {
#pragma unroll
            for (int u = 0; u < UD; ++u) {
                norm(pw);
                const bool in = pw.left > 0;
                const int grp = __builtin_amdgcn_readfirstlane(s_grp[in ? pw.q : 0]);
                const bool shared = in && pw.q < sh;
                const int F = shared ? a.n_shared * a.f : a.f;
                const char* W = shared ? (const char*)a.w_sh_dn : (const char*)a.w_dn + (size_t)(in ? grp : 0) * a.f * d * ES;
                const __amdgpu_buffer_rsrc_t rw = make_rsrc(W, (uint32_t)((size_t)F * d * ES));
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    vw[b][u][i] = load16<AUX>(rw, in ? rows_offset<BF>(d0 + 8 * i, F, lane) : OOR, (uint32_t)(in ? pw.s : 0) * STEP_BYTES<BF>);
                pw.s += FW_WAVES;
                --pw.left;
            }
        };
        auto load_a = [&](int b) {
#pragma unroll
            for (int u = 0; u < UD; ++u) {
                norm(pa);
                const bool in = pa.left > 0;
                const int grp = __builtin_amdgcn_readfirstlane(s_grp[in ? pa.q : 0]);
                const bool shared = in && pa.q < sh;
                const int F = shared ? a.n_shared * a.f : a.f;
                const char* A = shared ? (const char*)a.act_s : (const char*)a.act_r + (size_t)(in ? grp : 0) * FW * a.f * ES;
                const __amdgpu_buffer_rsrc_t ra = make_rsrc(A, (uint32_t)FW * (uint32_t)F * ES);
                const bool has = in && ((s_msk[grp] >> r16) & 1);
                runs[b][u] = has;
                const uint32_t ao = has ? (uint32_t)r16 * (uint32_t)F * ES + 16u * g16 : OOR;
#pragma unroll
                for (int h = 0; h < 2; ++h) va[b][u][h] = load16(ra, ao, (uint32_t)(in ? pa.s : 0) * 128u + 64u * h);
                pa.s += FW_WAVES;
                --pa.left;
            }
        };
        f32x4 acc[4] = {};
        auto mul = [&](int b) {
#pragma unroll
            for (int u = 0; u < UD; ++u) {
#pragma unroll
                for (int i = 0; i < 8; ++i) *(u32x4*)(put + 8 * i * ROW_LD) = vw[b][u][i];
                f32x4 sum[4] = {acc[0], acc[1], acc[2], acc[3]};
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        sum[r] = mma<BF>(*(const u32x4*)(get + 16 * r * ROW_LD + 64 * h), va[b][u][h], sum[r]);
                // a group's weights reach its own tokens only (to the others' zeros one that is no number would add a NaN)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[r][i] = runs[b][u] ? sum[r][i] : acc[r][i];
            }
        };
        load_w(0);
        load_w(1);
        if (!ready) {
            if (tid == 0) {
                while (look(CTR_ALL + (int)(blockIdx.x % FW_XCDS)) == 0) __builtin_amdgcn_s_sleep(8);
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
            }
            __syncthreads();
            ready = true;
        }
        load_a(0);
        for (int i = 0; i < ns; i += 2 * UD) {
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
        __syncthreads();                                     // (the sums of the item before have been read)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) s_red[wave][r][4 * g16 + i][r16] = acc[r][i];
        __syncthreads();
        // two of the 64 columns per thread, 32 apart
        const int col = tid & 31, tok = tid >> 5;
        float v[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            v[r] = 0.f;
#pragma unroll
            for (int w = 0; w < FW_WAVES; ++w) v[r] += s_red[w][2 * r + (col >> 4)][col & 15][tok];
        }
        if (pieces > 1) {
            // the pieces' sums meet in memory; the last piece to arrive adds them in order
            const __amdgpu_buffer_rsrc_t rp = make_rsrc(a.part + (size_t)tile * FW_PIECES * FW * 64, FW_PIECES * FW * 64 * 4);
            const uint32_t at = (uint32_t)(tok * 64 + col) * 4u;
            if (tok < T)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[r]), rp, (int)(at + 128u * r), sp * FW * 64 * 4, SC1);
            __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0)
            __syncthreads();
            if (tid == 0) s_item = add(CTR_TILE + tile);
            __syncthreads();
            if (s_item != pieces - 1) continue;
            if (tok < T) {
                float pv[FW_PIECES][2];
#pragma unroll
                for (int p = 0; p < FW_PIECES; ++p)          // (past the pieces: the last one again, not added)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        pv[p][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                            rp, (int)(at + 128u * r), (p < pieces ? p : pieces - 1) * FW * 64 * 4, SC1));
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    v[r] = pv[0][r];
#pragma unroll
                    for (int p = 1; p < FW_PIECES; ++p)
                        if (p < pieces) v[r] += pv[p][r];
                }
            }
        }
        if (tok < T) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const size_t o = (size_t)tok * d + d0 + 32 * r + col;
                if constexpr (BF) ((__bf16*)a.y)[o] = (__bf16)v[r];
                else ((float*)a.y)[o] = v[r];
            }
        }
      }
    }
}

template <bool BF, int NBT, int AUX>
int launch_layer(const FewArgs& a, int ks, hipStream_t st) {
    // never more workgroups than items: a tile of every group that can be in use
    const int64_t groups = a.r.T * (a.r.k < a.n_local ? a.r.k : a.n_local);
    const int64_t act = ((groups < a.n_local ? groups : a.n_local) + a.n_shared) * (a.f / 32);
    const int64_t items = a.r.T > 0 ? act + a.r.d / 64 * FW_PIECES : 1;
    const int64_t most = FW_SHARES, shares = (items + FW_XCDS - 1) / FW_XCDS * FW_XCDS;
    // (tables of other sizes and alignments are read where they are)
    auto vec = [](const void* p, int64_t n) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && n % 4 == 0; };
    const int64_t n_t1 = (int64_t)a.r.E * a.r.gmax, n_S = (int64_t)a.r.M * a.r.M * a.r.E;
    int tables = vec(a.r.t1_k, n_t1) && vec(a.r.t1_q, n_t1) && vec(a.r.t1_n, a.r.E) && vec(a.r.srvmask, a.r.E) ? 1 : 0;
    if (tables && vec(a.r.S, n_S) && n_S <= TAB_S) tables |= 2;
    KernelTimer kt_("few_layer", st);
    few_layer_kernel<BF, NBT, AUX><<<dim3((unsigned)(shares < most ? shares : most)), dim3(FW_THREADS), 0, st>>>(a, ks, tables);
    return (int)hipGetLastError();
}

template <bool BF, int AUX>
int launch_experts(const FewArgs& a, int ks, hipStream_t st) {
    const int nb = (a.r.E + 15) / 16;
    if (nb <= 1) return launch_layer<BF, 1, AUX>(a, ks, st);
    if (nb <= 4) return launch_layer<BF, 4, AUX>(a, ks, st);
    if (nb <= 8) return launch_layer<BF, 8, AUX>(a, ks, st);
    return launch_layer<BF, 16, AUX>(a, ks, st);
}

}  // namespace

size_t few_counters(int d) { return (size_t)(CTR_TILE + d / 64) * LINE; }

int launch_few_layer(const FewArgs& a, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    const bool bf = a.r.dtype == ORDERMOE_BF16;
    const int nb = (a.r.E + 15) / 16, ks = route_ksplit(1, nb, a.r.d);
    {
        KernelTimer kt_("few_router", st);
        const dim3 blocks((unsigned)nb, (unsigned)ks);
        if (bf) few_router_kernel<true><<<blocks, dim3(64), 0, st>>>(a, ks);
        else few_router_kernel<false><<<blocks, dim3(64), 0, st>>>(a, ks);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    if (!bf) return launch_experts<false, 0>(a, ks, st);
    const bool stream_w = (int64_t)a.n_local * 2 * a.f * a.r.d * 2 >= FW_STREAM_BYTES;
    return stream_w ? launch_experts<true, NT>(a, ks, st) : launch_experts<true, 0>(a, ks, st);
}

}  // namespace ordermoe
