// Attention of drafted tokens over the latent cache: every head's absorbed query on the
// same rows [c_p | r_p], of which the first part is the value too.
//
//   latent_attention_kernel  one workgroup per (work item, block of 16 RW query rows).  A work
//                            item is a piece of one sequence's cache.  RW waves that take 16 rows
//                            each share a tile of its tokens in LDS; the tiles go round the groups of
//                            such waves, every group with a running maximum, sum and output of its
//                            own, joined in LDS at the end -> partial sums (memory)
//   latent_out_kernel        the pieces' sums added in order, relative to their largest maximum,
//                            divided, and taken through W_v: 16 tokens of one head
//   latent_mass_kernel       the weight that each position got, from the scores that the first
//                            kernel wrote and the rows' final maximum and sum
// The query rows of a sequence are its n_b tokens times the heads: row = token * n_q + head.
//
// A tile (bf16; c = lane % 16, g = lane / 16):
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16; rows: 16 tokens, columns: 16 query rows.  Maximum and sum belong
//                 to a column, that is to a lane.
//   O^T = C^T P^T v_mfma_f32_16x16x32_bf16, or 16x16x16 where a tile has 16 tokens; rows: 16 elements of the latent
//                 vector, columns: 16 query rows.  S^T leaves lane (c, g) the weights of query row c for tokens
//                 4g .. 4g + 3 of each 16: the inner indexes of its P^T operand, when C^T's lanes hold the
//                 same tokens, which turned reads of the rows in LDS give them.  So the weights never
//                 leave their registers.
// fp32 runs the same tile with v_mfma_f32_16x16x4_f32.  Rows go straight from memory into LDS, a group's next tile
// while it attends to one.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "grid.hpp"
#include "mfma.hpp"

namespace ordermoe {
namespace {

constexpr int LA_TARGET = 512;                       // workgroups that a large batch is split into
constexpr int LA_MIN_PIECE = 64;                     // tokens
constexpr int LO_GROUPS = 256;                       // workgroups of the last product wished for
constexpr float LA_LAG = 8.0f;                       // see attend_tile

// waves that share a tile, for sequences of up to `rows` query rows: 16 rows each
__host__ __device__ inline int row_waves(int dtype, int rows) {
    return dtype != ORDERMOE_BF16 || rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : 8;
}
__host__ __device__ inline int row_blocks(int rows, int rw) { return (rows + 16 * rw - 1) / (16 * rw); }

struct Seq {
    int first, n, ctx, len;     // first token, drafted tokens, cached tokens before them, positions
};
__device__ inline Seq sequence(const LatentAttentionArgs& a, int b) {
    Seq s;
    const int T = (int)a.T, cap = a.max_pages << a.cache.page_shift;
    int s0 = a.q_start[b], s1 = a.q_start[b + 1], ctx = a.ctx_len[b];
    s0 = s0 < 0 ? 0 : s0 > T ? T : s0;
    s1 = s1 < s0 ? s0 : s1 > T ? T : s1;
    ctx = ctx < 0 ? 0 : ctx > cap ? cap : ctx;
    s.first = s0;
    s.n = s1 - s0 < a.max_q ? s1 - s0 : a.max_q;
    s.ctx = ctx;
    s.len = s.n < cap - ctx ? ctx + s.n : cap;
    return s;
}
__device__ inline Seq uniform(const Seq& s, int l) {
    return Seq{__builtin_amdgcn_readlane(s.first, l), __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.ctx, l),
               __builtin_amdgcn_readlane(s.len, l)};
}

__device__ inline int64_t first_lane(int64_t x) {
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) | (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// The tokens of a piece, by one wave: as many, a multiple of a round of the waves, as give about LA_TARGET
// workgroups in all, but at least total * rb_n / (2 LA_TARGET): that bounds the pieces by 2 LA_TARGET / rb_n + B.
__device__ inline int piece_tokens(const LatentAttentionArgs& a, int rb_n, int rw, int round, const Seq& mine, int lane) {
    int64_t total = 0, blocks = 0;
    for (int b = lane; b < a.B; b += 64) {
        const Seq s = b < 64 ? mine : sequence(a, b);
        total += s.n > 0 ? s.len : 0;
        blocks += s.n > 0 ? (int64_t)s.len * row_blocks(s.n * a.n_q, rw) : 0;
    }
    // (to lane 0, from as many lanes as there are sequences)
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        if (o >= a.B) continue;
        total += __shfl_xor(total, o);
        if (rb_n > 1) blocks += __shfl_xor(blocks, o);
    }
    total = first_lane(total);
    blocks = rb_n > 1 ? first_lane(blocks) : total;
    int64_t p = (blocks + LA_TARGET - 1) / LA_TARGET;
    const int64_t least = (total * rb_n + 2 * LA_TARGET - 1) / (2 * LA_TARGET);
    p = p < least ? least : p;
    p = p < LA_MIN_PIECE ? LA_MIN_PIECE : p;
    p = (p + round - 1) / round * round;
    return (int)(p > (1 << 30) ? 1 << 30 : p);
}
__device__ inline int pieces_of(const Seq& s, int piece) {
    // a sequence without positions still writes its rows (zeros)
    return s.n <= 0 ? 0 : s.len <= piece ? 1 : (s.len + piece - 1) / piece;
}
// sequence (of number b, < 0: none) and piece j of a work item, by one wave.
// write_plan: every sequence's first item and pieces to a.plan.
__device__ inline Seq find_item(const LatentAttentionArgs& a, int piece, int item, int lane, bool write_plan, const Seq& mine, int& b,
                                int& j) {
    Seq found = {0, 0, 0, 0};
    int base = 0;
    b = -1;
    j = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        Seq s = mine;
        if (b0 > 0 && b0 + lane < a.B) s = sequence(a, b0 + lane);
        const int cnt = b0 + lane < a.B ? pieces_of(s, piece) : 0;
        int inc = cnt;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            if (o >= a.B) continue;
            const int v = __shfl_up(inc, o);
            if (lane >= o) inc += v;
        }
        const int first = base + inc - cnt;
        if (write_plan && b0 + lane < a.B) {
            a.plan[2 * (b0 + lane)] = first;
            a.plan[2 * (b0 + lane) + 1] = cnt;
        }
        const uint64_t hit = __builtin_amdgcn_ballot_w64(item >= first && item < first + cnt);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            b = b0 + l;
            j = item - __builtin_amdgcn_readlane(first, l);
            found = uniform(s, l);
            if (!write_plan) break;
        }
        base += __builtin_amdgcn_readlane(inc, 63);
    }
    return found;
}

// A tile of TILE rows of RB bytes in LDS: panels of 128 bytes of every row, chunk (of 16 bytes) ch of row r at ch ^ r % 8, so
// that the reads of one chunk of eight rows lie on distinct banks; and what is left over, 64 bytes, as rows of their own,
// at ch ^ r / 2 % 4.  A wave's load of 1 KB is eight rows of a panel: one offset per lane serves all of them.
template <bool BF, int R, int ROT, int RW>
struct Config {
    static constexpr int ES = BF ? 2 : 4, RB = (R + ROT) * ES;
    static constexpr int NW = RW > 1 ? 8 : BF ? 4 : 2, GROUPS = NW / RW;     // waves, groups of them
    static constexpr int TILE = RW > 1 ? 8 * RW : 16;                        // tokens of a group's tile
    static constexpr int SUB = TILE < 32 ? 16 : 32;                          // tokens that are attended to at a time
    static constexpr int PANELS = RB / 128, TAIL = PANELS * TILE * 128;      // whole panels, where the rest begins
    static constexpr bool HAS_TAIL = RB % 128 != 0;
    static constexpr int STAGE = TILE * RB, OCTETS = TILE / 8 / RW;          // bytes of a tile, a wave's eights of its rows
    static constexpr int LOADS = OCTETS * (PANELS + HAS_TAIL);               // of a wave for a tile
    static constexpr int KS = RB / 64;                                       // steps of the first product
    static constexpr int LD = R + 4;                                         // floats of a row of sums in LDS
    static_assert(RB % 64 == 0 && R * ES % 128 == 0 && GROUPS * 16 * LD * 4 <= GROUPS * 2 * STAGE, "whole chunks, the sums fit");
};

// page of the tile at t0 (16 tokens never cross a page), -1: none; uniform, through the scalar cache
__device__ inline int tile_page(const LatentAttentionArgs& a, const int32_t* table, int t0, int len) {
    const __attribute__((address_space(4))) int32_t* t = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)table;
    return t0 < len ? t[t0 >> a.cache.page_shift] : -1;
}

template <int N>
__device__ inline void wait_loads() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The bare barrier: what waves have waited for themselves is there for all behind it (__syncthreads() would wait for
// every load that is on its way)
__device__ inline void lds_barrier() { asm volatile("s_barrier" ::: "memory"); }

// of SUB tokens from row r0 of a tile on, those whose row holds an infinity or a NaN, a bit each, by one wave
template <bool BF, typename Cf>
__device__ inline uint32_t not_finite(const char* st, int r0, int lane) {
    uint32_t m = 0;
    auto look = [&](const char* p, int row) {
        const u32x4 x = *(const u32x4*)p;
        bool bad = false;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            bad |= BF ? (x[w] & 0x7F80u) == 0x7F80u || (x[w] & 0x7F800000u) == 0x7F800000u : (x[w] & 0x7F800000u) == 0x7F800000u;
        if (bad) m |= 1u << row;
    };
#pragma unroll 2
    for (int p = 0; p < Cf::PANELS; ++p)
#pragma unroll
        for (int o = 0; o < Cf::SUB; o += 8) look(st + p * (Cf::TILE * 128) + (r0 + o) * 128 + lane * 16, o + (lane >> 3));
    if constexpr (Cf::HAS_TAIL)
#pragma unroll
        for (int o = 0; o < Cf::SUB; o += 16) look(st + Cf::TAIL + (r0 + o) * 64 + lane * 16, o + (lane >> 2));
    if (!__builtin_amdgcn_ballot_w64(m != 0)) return 0;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m |= __shfl_xor(m, o);
    return m;
}

// The running state of a wave: lane (c, g) has row c's maximum (in units of log 2; a shared reference that may
// lag behind the true one) and its own tokens' share of the sum; o[j] holds row c's elements 16 j + 4 g + i, i = 0 .. 3.
template <int R>
struct State {
    float m, l;
    f32x4 o[R / 16];
};

__device__ inline u32x2 only_finite(u32x2 v) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        if ((v[w] & 0x7F80u) == 0x7F80u) v[w] &= 0xFFFF0000u;
        if ((v[w] & 0x7F800000u) == 0x7F800000u) v[w] &= 0xFFFFu;
    }
    return v;
}

// O^T += C^T P^T over SUB tokens from row r0 of a tile on; CLEAN: what is no number counts as 0.  The reads of a few
// elements' rows are on their way during the products of the ones before.
template <int R, typename Cf, bool FINE, bool CLEAN>
__device__ inline __attribute__((always_inline)) void add_weighted(const char* st, int r0, const u32x2* pf, const u32x2* pl, int lane,
                                                                   State<R>& state) {
    constexpr int NB = Cf::SUB / 16, PANEL = Cf::TILE * 128, AHEAD = 4 / NB, STEPS = R / 16 / AHEAD;
    const int c = lane & 15, row = 4 * (lane >> 4) + (c >> 2);
    const char* at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = st + (r0 + row) * 128 + (((2 * j + ((c >> 1) & 1)) ^ (row & 7)) * 16) + (c & 1) * 8;
    u32x2 v[2][AHEAD][NB];
    auto read = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < AHEAD; ++e)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int j = i * AHEAD + e;
                v[i & 1][e][n] = read_turned(at[j % 4] + j / 4 * PANEL + 16 * n * 128);
            }
    };
    read(0);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (i + 1 < STEPS) read(i + 1);
        if constexpr (CLEAN)
#pragma unroll
            for (int e = 0; e < AHEAD; ++e)
#pragma unroll
                for (int n = 0; n < NB; ++n) v[i & 1][e][n] = only_finite(v[i & 1][e][n]);
#pragma unroll
        for (int part = 0; part < (FINE ? 2 : 1); ++part) {
            const u32x2* p = part ? pl : pf;
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int j = i * AHEAD + e;
                const u32x2* x = v[i & 1][e];
                if constexpr (NB == 1)
                    state.o[j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, x[0]), __builtin_bit_cast(s16x4, p[0]),
                                                                           state.o[j], 0, 0, 0);
                else
                    state.o[j] = mma16<true>(u32x4{x[0][0], x[0][1], x[1][0], x[1][1]}, u32x4{p[0][0], p[0][1], p[1][0], p[1][1]}, state.o[j]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// SUB tokens from t0 on, rows r0 .. of the tile staged at st.  A maximum is taken over only when some score passes it by
// LA_LAG (a factor of 256 in the weights, which fp32 sums and bf16 weights hold as well as 1): most tiles then need no
// exchange between lanes and no rescaling of the outputs.  FINE: the second product takes what the rounding of the
// weights to bf16 leaves out as well.
template <bool BF, int R, typename Cf, bool FINE, bool WEIGHS>
__device__ inline __attribute__((always_inline)) void attend_tile(const char* st, int r0, const u32x4* q, uint32_t ok, int t0, const Seq& s,
                                                                  uint64_t word, bool in, float scale2, float* score, int lane,
                                                                  State<R>& state) {
    constexpr int SUB = Cf::SUB, NB = SUB / 16, KS = Cf::KS, PANEL = Cf::TILE * 128;
    const int c = lane & 15, g = lane >> 4;
    const float ninf = -__builtin_inff();
    f32x4 sc[NB] = {};
    {
        constexpr int RING = NB == 1 ? 5 : 3;                    // steps whose reads are in registers or on their way
        const char* at[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) at[k] = st + (r0 + c) * 128 + (((4 * k + g) ^ (c & 7)) * 16);
        const char* tail = st + Cf::TAIL + (r0 + c) * 64 + ((g ^ ((c >> 1) & 3)) * 16);
        u32x4 x[RING][NB];
        auto read = [&](int k) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
                x[k % RING][n] = *(const u32x4*)(k / 2 < Cf::PANELS ? at[k % 2] + k / 2 * PANEL + 16 * n * 128 : tail + 16 * n * 64);
        };
#pragma unroll
        for (int k = 0; k < RING - 1; ++k) read(k);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            if (k + RING - 1 < KS) read(k + RING - 1);
#pragma unroll
            for (int n = 0; n < NB; ++n) sc[n] = mma16<BF>(x[k % RING][n], q[k], sc[n]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    const bool edge = t0 + SUB > s.ctx || (~ok & ((1u << NB) - 1u));
#pragma unroll
    for (int n = 0; n < NB; ++n) sc[n] = sc[n] * scale2;
    uint32_t bad = 0;
    if (edge) {
        // (places past the end hold the last token's row, see issue: what all rows see keeps nothing from any)
        uint32_t seen = 0, there = 0;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int p = t0 + 16 * n + 4 * g + i, j = p - s.ctx;
                const bool see = ((ok >> n) & 1) && p < s.len && (j < 0 || ((word >> (j & 63)) & 1));
                seen |= (uint32_t)see << (16 * n + 4 * g + i);
                there |= (uint32_t)(p < s.len) << (16 * n + 4 * g + i);
                sc[n][i] = see ? sc[n][i] : ninf;
            }
        if (__builtin_amdgcn_ballot_w64(in && seen != there)) {
            bad = not_finite<BF, Cf>(st, r0, lane);
            if (bad & seen) state.l = __builtin_nanf("");    // (what is no number is taken as 0 below)
        }
    }
    if constexpr (WEIGHS) {
        if (score) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
                if (t0 + 16 * n < s.len) *(f32x4*)(score + t0 + 16 * n + 4 * g) = sc[n];     // (a table holds whole 16s)
        }
    }
    float top = ninf;
#pragma unroll
    for (int n = 0; n < NB; ++n) top = fmaxf(top, fmaxf(fmaxf(sc[n][0], sc[n][1]), fmaxf(sc[n][2], sc[n][3])));
    if (__builtin_amdgcn_ballot_w64(top > state.m + LA_LAG)) {
        float x = fmaxf(top, __shfl_xor(top, 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        const float m = x > state.m + LA_LAG ? x : state.m;      // by the row alone, whatever the others do
        const float al = state.m == m ? 1.0f : __builtin_amdgcn_exp2f(state.m - m);
        state.m = m;
        state.l *= al;
#pragma unroll
        for (int j = 0; j < R / 16; ++j) state.o[j] = state.o[j] * al;
    }
    // weights exp2(score - maximum), 0 where nothing has been seen yet
    const float m = state.m == ninf ? 0.f : state.m;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sc[n][i] = __builtin_amdgcn_exp2f(sc[n][i] - m);
            state.l += sc[n][i];
        }
    if constexpr (BF) {
        u32x2 pf[NB], pl[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            bf16x4 hi, lo;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi[i] = (__bf16)sc[n][i];
                if constexpr (FINE) lo[i] = (__bf16)(sc[n][i] - (float)hi[i]);
            }
            pf[n] = __builtin_bit_cast(u32x2, hi);
            if constexpr (FINE) pl[n] = __builtin_bit_cast(u32x2, lo);
        }
        if (bad) add_weighted<R, Cf, FINE, true>(st, r0, pf, pl, lane, state);
        else add_weighted<R, Cf, FINE, false>(st, r0, pf, pl, lane, state);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * g + i;
            const char* at[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) at[j] = st + (r0 + row) * 128 + (((4 * j + (c >> 2)) ^ (row & 7)) * 16) + (c & 3) * 4;
#pragma unroll
            for (int j = 0; j < R / 16; ++j) {
                float v = *(const float*)(at[j % 2] + j / 2 * PANEL);
                if (bad) v = (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u ? 0.f : v;
                state.o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, sc[0][i], state.o[j], 0, 0, 0);
            }
        }
    }
}

template <bool BF, int R, int ROT, int RW, bool FINE, bool WEIGHS>
__global__ void __launch_bounds__((64 * Config<BF, R, ROT, RW>::NW), (BF || R < 512 ? 2 : 1))
latent_attention_kernel(const LatentAttentionArgs a, int items, int rb_n) {
    using Cf = Config<BF, R, ROT, RW>;
    constexpr int NW = Cf::NW, GROUPS = Cf::GROUPS, ROUND = GROUPS * Cf::TILE, NB = Cf::TILE / 16;
    __shared__ __attribute__((aligned(16))) char s_mem[GROUPS * 2 * Cf::STAGE];
    __shared__ float s_m[NW][16], s_l[NW][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4, rw = wave % RW, grp = wave / RW;
    // the row blocks of one piece on one XCD, where its rows are in L2
    const int idx = (int)block_number(), jx = idx >> 3;
    const int item = (jx / rb_n) * 8 + (idx & 7), rb = jx % rb_n;
    if (item >= items) return;
    Seq mine = {0, 0, 0, 0};
    if (lane < a.B) mine = sequence(a, lane);
    const int piece = __builtin_amdgcn_readfirstlane(piece_tokens(a, rb_n, RW, ROUND, mine, lane));
    int b, j;
    const Seq s = find_item(a, piece, item, lane, idx == 0 && wave == 0, mine, b, j);
    if (b < 0) return;
    const int rows = s.n * a.n_q, row0 = rb * 16 * RW, rows_max = a.max_q * a.n_q;
    if (row0 >= rows) return;
    const int t_lo = j * piece, t_hi = s.len - t_lo < piece ? s.len : t_lo + piece;
    const int32_t* table = a.page_table + (int64_t)b * a.max_pages;
    const float scale2 = a.scale * LOG2E;            // scores in units of log 2
    const int row = row0 + 16 * rw + c;
    const bool in = row < rows;                      // rows past the end are zeros and see nothing
    const int i_tok = in ? row / a.n_q : 0;
    const uint64_t word = !in ? 0ull : a.tree ? a.tree[s.first + i_tok] : ~0ull >> (63 - i_tok);
    float* const score = WEIGHS && in ? a.score + ((int64_t)b * rows_max + row) * ((int64_t)a.max_pages << a.cache.page_shift) : nullptr;
    u32x4 q[Cf::KS];
    {
        const char* from = (const char*)a.q + ((int64_t)s.first * a.n_q + (in ? row : 0)) * Cf::RB + 16 * g;
#pragma unroll
        for (int k = 0; k < Cf::KS; ++k) {
            q[k] = u32x4{0u, 0u, 0u, 0u};
            if (in) q[k] = *(const u32x4*)(from + 64 * k);
        }
    }
    State<R> st;
    st.m = -__builtin_inff();
    st.l = 0.f;
#pragma unroll
    for (int e = 0; e < R / 16; ++e) st.o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
    char* const stage = s_mem + grp * 2 * Cf::STAGE;
    const int sh = a.cache.page_shift;
    // a tile's pages, 16 tokens each
    struct Pages { int p[NB]; };
    auto pages = [&](int t0) __attribute__((always_inline)) {
        Pages r;
#pragma unroll
        for (int n = 0; n < NB; ++n) r.p[n] = tile_page(a, table, t0 + 16 * n, t_hi);
        return r;
    };
    const uint32_t voff = (lane >> 3) * Cf::RB + (((lane & 7) ^ (lane >> 3)) * 16);
    const uint32_t voff_tail = ((lane >> 2) & 7) * Cf::RB + (((lane & 3) ^ ((lane >> 3) & 3)) * 16);
    auto issue = [&](const Pages& pg, int t0, char* to) __attribute__((always_inline)) {
        uint32_t ok = 0;                             // a bit each
#pragma unroll
        for (int n = 0; n < NB; ++n) ok |= (uint32_t)(pg.p[n] >= 0 && pg.p[n] < a.cache.n_pages) << n;
#pragma unroll
        for (int e = 0; e < Cf::OCTETS; ++e) {
            // eight rows; tokens without a page read page 0
            const int o = rw * Cf::OCTETS + e;
            int pid = pg.p[0];
#pragma unroll
            for (int n = 1; n < NB; ++n) pid = o >= 2 * n ? pg.p[n] : pid;
            const bool there = (ok >> (o / 2)) & 1;
            const char* base = a.cache.rows + (there ? ((int64_t)pid << sh) + ((t0 + 8 * o) & ((1 << sh) - 1)) : 0) * Cf::RB;
            const int last = s.len - 1 - (t0 + 8 * o);
            if (last >= 7) {
#pragma unroll
                for (int i = 0; i < Cf::PANELS; ++i) load_lds16(base + i * 128 + voff, to + (i * Cf::TILE + 8 * o) * 128);
                if constexpr (Cf::HAS_TAIL)
                    if (lane < 32) load_lds16(base + Cf::PANELS * 128 + voff_tail, to + Cf::TAIL + 8 * o * 64);
            } else {
                // places past the end, which nothing may have been written to, take the last token's row
                const int end = s.len - 1 - t0, e16 = end >> 4;
                int pe = pg.p[0];
#pragma unroll
                for (int n = 1; n < NB; ++n) pe = e16 == n ? pg.p[n] : pe;
                const char* row = a.cache.rows + (((ok >> e16) & 1) ? ((int64_t)pe << sh) + ((s.len - 1) & ((1 << sh) - 1)) : 0) * Cf::RB;
                const int r = lane >> 3, rt = (lane >> 2) & 7;
                const char* f = r <= last ? base + voff : row + (voff - r * Cf::RB);
                const char* ft = rt <= last ? base + voff_tail : row + (voff_tail - rt * Cf::RB);
#pragma unroll
                for (int i = 0; i < Cf::PANELS; ++i) load_lds16(f + i * 128, to + (i * Cf::TILE + 8 * o) * 128);
                if constexpr (Cf::HAS_TAIL)
                    if (lane < 32) load_lds16(ft + Cf::PANELS * 128, to + Cf::TAIL + 8 * o * 64);
            }
        }
        return ok;
    };
    int p = t_lo + grp * Cf::TILE;
    const int rounds = (t_hi - t_lo + ROUND - 1) / ROUND;
    uint32_t ok = 0, next = 0;
    Pages pg = pages(p);
    if (p < t_hi) ok = issue(pg, p, stage);
    pg = pages(p + ROUND);
    for (int k = 0, buf = 0; k < rounds; ++k, p += ROUND, buf ^= 1) {
        if constexpr (RW > 1)
            if (k > 0) {
                wait_loads<0>();
                __syncthreads();                     // the tile has arrived, and the one before has been read
            }
        if (p + ROUND < t_hi) {
            next = issue(pg, p + ROUND, stage + (buf ^ 1) * Cf::STAGE);
            pg = pages(p + 2 * ROUND);
            if (RW == 1 || k == 0) wait_loads<Cf::LOADS>();      // all but the next tile's
        } else if (RW == 1 || k == 0) {
            wait_loads<0>();
        }
        if constexpr (RW > 1)
            if (k == 0) lds_barrier();               // the first tile has arrived
        if (p < t_hi) {
#pragma unroll 1
            for (int n = 0; n < Cf::TILE / Cf::SUB; ++n) {
                if (p + n * Cf::SUB >= t_hi) break;
                attend_tile<BF, R, Cf, FINE, WEIGHS>(stage + buf * Cf::STAGE, n * Cf::SUB, q, ok >> (n * (Cf::SUB / 16)),
                                                                  p + n * Cf::SUB, s, word, in, scale2, score, lane, st);
            }
        }
        ok = next;
    }
    // the groups' states joined, the rows of one of their waves at a time
    float l = st.l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) { s_m[wave][c] = st.m; s_l[wave][c] = l; }
    __syncthreads();                                 // the staged rows become the place of the sums
    float(*const s_o)[16][Cf::LD] = (float(*)[16][Cf::LD])s_mem;
    constexpr int PER = NW * 4, PART = R / PER;      // threads a row, their elements
    const int64_t prow = (int64_t)item * rows_max;
    float m = s_m[rw][c];
#pragma unroll
    for (int w = 1; w < GROUPS; ++w) m = fmaxf(m, s_m[w * RW + rw][c]);
    const float f = st.m == m ? 1.0f : __builtin_amdgcn_exp2f(st.m - m);
#pragma unroll 1
    for (int r = 0; r < RW; ++r) {
        if (row0 + 16 * r >= rows) break;
        if (r == rw) {
#pragma unroll
            for (int e = 0; e < R / 16; ++e) *(f32x4*)&s_o[grp][c][16 * e + 4 * g] = st.o[e] * f;
        }
        __syncthreads();
        const int rt = tid / PER, rr = row0 + 16 * r + rt, u = tid % PER;
        if (rr < rows) {
            float* po = a.part_o + (prow + rr) * R;
#pragma unroll
            for (int e = 0; e < PART; e += 4) {
                f32x4 v = *(const f32x4*)&s_o[0][rt][4 * u + PER * e];
#pragma unroll
                for (int w = 1; w < GROUPS; ++w) v += *(const f32x4*)&s_o[w][rt][4 * u + PER * e];
                *(f32x4*)(po + 4 * u + PER * e) = v;
            }
            if (u == 0) {
                float mm = s_m[r][rt], ll = 0.f;
#pragma unroll
                for (int w = 1; w < GROUPS; ++w) mm = fmaxf(mm, s_m[w * RW + r][rt]);
#pragma unroll
                for (int w = 0; w < GROUPS; ++w) {
                    const float mw = s_m[w * RW + r][rt];
                    ll += s_l[w * RW + r][rt] * (mw == mm ? 1.0f : __builtin_amdgcn_exp2f(mw - mm));
                }
                a.part_ml[2 * (prow + rr)] = mm;
                a.part_ml[2 * (prow + rr) + 1] = ll;
            }
        }
        __syncthreads();
    }
}

// 16 / S tokens (of the batch) of one head, DS of the head's elements: the rows' pieces added in order, divided, and
// out = o W_v^T.  A row has S sets of 16 lanes: set z adds pieces z, z + S, .., then the sets' sums are added.  The matrix
// unit's rows are elements, its columns tokens.  DS / 32 pairs of element tiles go round the waves; where they are fewer
// than the waves, the waves share the inner index, and their weights are on their way during the additions.
template <bool BF, int R, int D, int DS, int S>
__global__ void __launch_bounds__(256) latent_out_kernel(const LatentAttentionArgs a, int slices) {
    constexpr int ES = BF ? 2 : 4, PITCH = R * ES + 16, U = 4, TOK = 16 / S;     // bytes of a row in LDS; pieces whose reads are in flight; tokens
    constexpr int PAIRS = DS / 32, SHARE = 4 / PAIRS, KS = R * ES / 64 / SHARE, EARLY = SHARE > 1 ? KS : 4;
    __shared__ __attribute__((aligned(16))) char s_o[BF ? 2 : 1][16 * PITCH];
    __shared__ f32x4 s_acc[SHARE > 1 ? 4 : 1][2][64];
    __shared__ float s_x[S == 16 ? 4 : 1][S == 16 ? R : 1], s_m[4], s_l[4];
    __shared__ int s_in[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t id = block_number(), rest = id / slices;
    const int d0 = (int)(id - rest * slices) * DS, h = (int)(rest % a.n_q);
    const int64_t tb = rest / a.n_q * TOK;
    if (tb >= a.T) return;
    const int c = lane & 15, g = lane >> 4, pair = wave % PAIRS, share = wave / PAIRS;
    const char* w = (const char*)a.w_v + ((int64_t)(h * D + d0 + 32 * pair + c) * R) * ES + (share * KS * 4 + g) * 16;
    u32x4 early[EARLY][2];
#pragma unroll
    for (int k = 0; k < EARLY; ++k) {
        early[k][0] = *(const u32x4*)(w + 64 * k);
        early[k][1] = *(const u32x4*)(w + 16 * R * ES + 64 * k);
    }
    // the token's sequence: the number of sequences that end at or before it
    const int slot = (tid >> 4) / S, z = (tid >> 4) % S, u = tid & 15, t = (int)std::min<int64_t>(tb + slot, a.T);
    int b = 0;
    for (int b0 = 0; b0 < a.B; b0 += 16) {
        const bool past = b0 + u < a.B && a.q_start[b0 + u + 1] <= t;
        const uint32_t m = (uint32_t)(__builtin_amdgcn_ballot_w64(past) >> (lane & 48)) & 0xFFFFu;
        b += __builtin_popcount(m);
    }
    bool in = tb + slot < a.T && b < a.B;
    Seq s = {0, 0, 0, 0};
    if (in) s = sequence(a, b);
    const int i = t - s.first;
    in = in && i >= 0 && i < s.n;
    const int row = i * a.n_q + h, rows_max = a.max_q * a.n_q;
    if (tid < 16) s_in[tid] = 0;
    const int pieces = in ? a.plan[2 * b + 1] : 0;
    const int64_t at = in ? (int64_t)a.plan[2 * b] * rows_max + row : 0;
    const f32x2* ml = (const f32x2*)a.part_ml;
    float m = -__builtin_inff(), l = 0.f, x[R / 16] = {};
    for (int p = z; p < pieces; p += U * S) {
        f32x2 q[U];
        f32x4 v[U][R / 64];
        float top = m;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t pr = at + (int64_t)(p + k * S < pieces ? p + k * S : p) * rows_max;
            q[k] = ml[pr];
#pragma unroll
            for (int e = 0; e < R / 64; ++e) v[k][e] = *(const f32x4*)(a.part_o + pr * R + 4 * u + 64 * e);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) top = fmaxf(top, q[k][0]);
        const float al = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= al;
#pragma unroll
        for (int e = 0; e < R / 16; ++e) x[e] *= al;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (p + k * S >= pieces) break;
            const float f = q[k][0] == m ? 1.0f : __builtin_amdgcn_exp2f(q[k][0] - m);
            l += q[k][1] * f;
#pragma unroll
            for (int e = 0; e < R / 16; ++e) x[e] += v[k][e / 4][e % 4] * f;
        }
    }
    // four sets of a wave, then (S = 16) the waves'
    if constexpr (S > 1) {
        float top = fmaxf(m, __shfl_xor(m, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float f = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= f;
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
#pragma unroll
        for (int e = 0; e < R / 16; ++e) {
            x[e] *= f;
            x[e] += __shfl_xor(x[e], 16);
            x[e] += __shfl_xor(x[e], 32);
        }
    }
    __syncthreads();                                 // s_in is clear
    if constexpr (S == 16) {
        if (lane < 16) {
#pragma unroll
            for (int e = 0; e < R / 64; ++e) *(f32x4*)&s_x[wave][4 * u + 64 * e] = f32x4{x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]};
        }
        if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
        __syncthreads();
        m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
        l = 0.f;
#pragma unroll
        for (int e = 0; e < R / 16; ++e) x[e] = 0.f;
        if (tid < 16) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = s_m[k] == m ? 1.0f : __builtin_amdgcn_exp2f(s_m[k] - m);
                l += s_l[k] * f;
#pragma unroll
                for (int e = 0; e < R / 16; ++e) x[e] += s_x[k][4 * u + 64 * (e / 4) + e % 4] * f;
            }
        }
    }
    if (z == 0) {
        const float r = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
        for (int e = 0; e < R / 64; ++e) {
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = x[4 * e + k] * r;
            char* o = &s_o[0][slot * PITCH + (4 * u + 64 * e) * ES];
            if constexpr (BF) {
                float d[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) d[k] = y[k] - (float)(__bf16)y[k];
                *(u32x2*)o = u32x2{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
                *(u32x2*)&s_o[BF ? 1 : 0][slot * PITCH + (4 * u + 64 * e) * ES] = u32x2{bf16_pair(d[0], d[1]), bf16_pair(d[2], d[3])};
            } else {
                *(f32x4*)o = f32x4{y[0], y[1], y[2], y[3]};
            }
        }
        if (in && u == 0) {
            s_in[slot] = 1;
            if (d0 == 0) {
                if (a.lse) a.lse[(int64_t)t * a.n_q + h] = l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * LN2;
                if (a.mass_out) ((f32x2*)a.stat)[(int64_t)b * rows_max + row] = f32x2{m == -__builtin_inff() ? 0.f : m, r};
            }
        }
    }
    __syncthreads();
    f32x4 acc[2] = {};
    // (tokens past TOK: a row that is there, for columns that nobody reads)
    const char* o = &s_o[0][(c < TOK ? c : 0) * PITCH + (share * KS * 4 + g) * 16];
    const char* o_lo = &s_o[BF ? 1 : 0][(c < TOK ? c : 0) * PITCH + (share * KS * 4 + g) * 16];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        const u32x4 w0 = k < EARLY ? early[k < EARLY ? k : 0][0] : *(const u32x4*)(w + 64 * k);
        const u32x4 w1 = k < EARLY ? early[k < EARLY ? k : 0][1] : *(const u32x4*)(w + 16 * R * ES + 64 * k);
        const u32x4 hi = *(const u32x4*)(o + 64 * k);
        acc[0] = mma16<BF>(w0, hi, acc[0]);
        acc[1] = mma16<BF>(w1, hi, acc[1]);
        if constexpr (BF) {
            const u32x4 lo = *(const u32x4*)(o_lo + 64 * k);
            acc[0] = mma16<BF>(w0, lo, acc[0]);
            acc[1] = mma16<BF>(w1, lo, acc[1]);
        }
    }
    if constexpr (SHARE > 1) {
        s_acc[wave][0][lane] = acc[0];
        s_acc[wave][1][lane] = acc[1];
        __syncthreads();
        if (share != 0) return;
#pragma unroll
        for (int k = 1; k < SHARE; ++k) {
            acc[0] += s_acc[pair + k * PAIRS][0][lane];
            acc[1] += s_acc[pair + k * PAIRS][1][lane];
        }
    }
    // (a token of no sequence, or past its sequence's first max_q, is not written)
    if (!s_in[c]) return;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        store4<BF>(a.out, ((tb + c) * a.n_q + h) * D + d0 + 32 * pair + 16 * k + 4 * g, acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
}

// 256 positions of a sequence: the weights of its rows, exp2(score - maximum) / sum, added up; the waves share the rows
__global__ void __launch_bounds__(256) latent_mass_kernel(const LatentAttentionArgs a, int per_seq) {
    __shared__ f32x4 s_w[4][64];
    const int64_t id = block_number();
    const int b = (int)(id / per_seq), p0 = (int)(id - (int64_t)b * per_seq) * 256;
    if (b >= a.B) return;
    const Seq s = sequence(a, b);
    if (s.n <= 0 || p0 >= s.len) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = p0 + 4 * lane;
    const int rows = s.n * a.n_q, rows_max = a.max_q * a.n_q;
    const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
    const f32x2* stat = (const f32x2*)a.stat + (int64_t)b * rows_max;
    f32x4 w = {0.f, 0.f, 0.f, 0.f};
    if (p < s.len) {
        const float* score = a.score + (int64_t)b * rows_max * cap + p;
#pragma unroll 4
        for (int r = wave; r < rows; r += 4) {
            const f32x4 x = *(const f32x4*)(score + r * cap);
            const f32x2 q = stat[r];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] += x[k] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(x[k] - q[0]) * q[1];
        }
    }
    s_w[wave][lane] = w;
    __syncthreads();
    if (wave != 0) return;
    w = s_w[0][lane] + s_w[1][lane] + s_w[2][lane] + s_w[3][lane];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (p + k >= s.len || p + k >= a.mass_stride) break;
        const int64_t at = b * a.mass_stride + p + k;
        a.mass_out[at] = p + k < s.ctx && a.mass ? a.decay * a.mass[at] + w[k] : w[k];
    }
}

template <bool BF, int R, int ROT, int RW, bool FINE>
int launch_rows(const LatentAttentionArgs& a, hipStream_t st) {
    const int rb = row_blocks(a.max_q * a.n_q, RW);
    const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
    {
        const int64_t items = std::min<int64_t>(latent_items(a.cache.dtype, a.n_q, a.B, a.max_q),
                                                a.B * ((cap + LA_MIN_PIECE - 1) / LA_MIN_PIECE));
        const dim3 grid = grid_of((items + 7) / 8 * 8 * rb), block((64 * Config<BF, R, ROT, RW>::NW));
        KernelTimer kt_("latent_attention", st);
        if (a.mass_out) latent_attention_kernel<BF, R, ROT, RW, FINE, true><<<grid, block, 0, st>>>(a, (int)items, rb);
        else latent_attention_kernel<BF, R, ROT, RW, FINE, false><<<grid, block, 0, st>>>(a, (int)items, rb);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    {
        KernelTimer kt_("latent_out", st);
        // as few sets a row as give every CU a workgroup; few rows: slices of the head's elements too
        auto go = [&](auto d, auto ds, auto sets) {
            constexpr int D = decltype(d)::value, DS = decltype(ds)::value, S = decltype(sets)::value, TOK = 16 / S;
            latent_out_kernel<BF, R, D, DS, S><<<grid_of((a.T + TOK - 1) / TOK * a.n_q * (D / DS)), dim3(256), 0, st>>>(a, D / DS);
        };
        auto of = [&](auto d) {
            using N1 = std::integral_constant<int, 1>;
            using N4 = std::integral_constant<int, 4>;
            using N16 = std::integral_constant<int, 16>;
            if ((a.T + 15) / 16 * a.n_q >= LO_GROUPS) go(d, d, N1{});
            else if ((a.T + 3) / 4 * a.n_q >= LO_GROUPS) go(d, d, N4{});
            else if ((a.T + 3) / 4 * a.n_q * (decltype(d)::value / 32) >= LO_GROUPS) go(d, std::integral_constant<int, 32>{}, N4{});
            else go(d, std::integral_constant<int, 32>{}, N16{});
        };
        if (a.head_dim == 64) of(std::integral_constant<int, 64>{});
        else of(std::integral_constant<int, 128>{});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    if (!a.mass_out) return 0;
    const int per = (int)((cap + 255) / 256);
    KernelTimer kt_("latent_mass", st);
    latent_mass_kernel<<<grid_of((int64_t)a.B * per), dim3(256), 0, st>>>(a, per);
    return (int)hipGetLastError();
}
template <bool BF, int R, int ROT>
int launch_tiles(const LatentAttentionArgs& a, hipStream_t st) {
    if constexpr (BF) {
        static_assert(ORDERMOE_LATENT_FINE_ROWS == 64, "the waves that share a tile where the weights keep 16 bits");
        switch (row_waves(ORDERMOE_BF16, a.max_q * a.n_q)) {
            case 2: return launch_rows<BF, R, ROT, 2, true>(a, st);
            case 4: return launch_rows<BF, R, ROT, 4, true>(a, st);
            case 8: return launch_rows<BF, R, ROT, 8, false>(a, st);
        }
    }
    return launch_rows<BF, R, ROT, 1, BF>(a, st);
}
template <bool BF, int R>
int launch_rot(const LatentAttentionArgs& a, hipStream_t st) {
    return a.cache.rot == 32 ? launch_tiles<BF, R, 32>(a, st) : launch_tiles<BF, R, 64>(a, st);
}
template <bool BF>
int launch_rank(const LatentAttentionArgs& a, hipStream_t st) {
    return a.cache.rank == 128 ? launch_rot<BF, 128>(a, st) : a.cache.rank == 256 ? launch_rot<BF, 256>(a, st) : launch_rot<BF, 512>(a, st);
}

}  // namespace

int64_t latent_items(int dtype, int n_q, int B, int max_q) {
    const int rows = max_q * n_q, rb = row_blocks(rows, row_waves(dtype, rows));
    return (2 * LA_TARGET + rb - 1) / rb + B;
}

int launch_latent_attention(const LatentAttentionArgs& a, void* stream) {
    if (a.B == 0 || a.T == 0) return 0;
    return a.cache.dtype == ORDERMOE_BF16 ? launch_rank<true>(a, (hipStream_t)stream) : launch_rank<false>(a, (hipStream_t)stream);
}

}  // namespace ordermoe
