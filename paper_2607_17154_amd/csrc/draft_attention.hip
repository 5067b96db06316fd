// Attention of drafted tokens over the quantised paged cache.
//
//   draft_attention_kernel  one workgroup per (work item, key/value head, block of
//                           16 RT query rows).  A work item is a piece of one
//                           sequence's cache; its 32-token tiles go round the
//                           workgroup's waves, every wave with a running maximum,
//                           sum and output of its own, joined in LDS at the end.
//   draft_join_kernel       sequences of several pieces: the pieces' sums added in
//                           order, relative to their largest maximum
// The query rows of a key/value head are its n_b tokens times the n_q / n_kv query
// heads that share it, so that one read of the codes serves them all.
//
// A tile (bf16; v_mfma_f32_16x16x32_bf16, c = lane % 16, g = lane / 16):
//   S^T = K Q^T   rows: 16 tokens, columns: 16 query rows.  The inner index may be
//                 taken in any order common to both sides, so lane (c, g) reads, of
//                 token c, the 16 neighbouring codes from 64 i + 16 g on for i = 0, 1, ..,
//                 and Q in the same order.
//   O^T = V^T P^T rows: 16 elements of the head, columns: 16 query rows.  Two S^T
//                 blocks leave lane (c, g) the weights of query row c for tokens
//                 4g .. 4g + 3 of each: exactly the 8 inner indexes of its P^T operand
//                 when V^T's lanes hold the same tokens.  So the weights never leave
//                 their registers, and neither do maximum and sum: they belong to a
//                 column, that is to a lane.
//   V             lane (c, g) reads D/16 neighbouring codes of its 8 tokens; matrix
//                 instruction j takes element c D/16 + j of each, whose codes are
//                 paired across tokens (e4m3: by byte permutes).
// Codes come from memory in whole cache lines, 16 bytes a lane, two tiles on their way,
// and get into these orders through the wave's own LDS rows (read in operand order
// straight from memory, 64 single tokens took 149 us for 119).
// Keys' scales multiply the scores, values' scales the weights, so codes enter the
// matrix unit as they are (8-bit codes are exact in bf16).  In bf16 the weights are
// rounded to bf16 for the second product, as its operands are; for blocks of up to 16 rows
// and heads of 256 what the rounding leaves out goes through it as well (one token over 777
// cached: error 0.0028 of the output's size without, 0.0017 with, which is the output's own
// rounding; 64 single tokens 100 -> 101 us; for all rows trees of 64 would take 361 us for 317
// and trees of 33 42.4 for 40.7, error 0.0024 as it is).  Sums stay in fp32.
// fp32 runs the same tile with v_mfma_f32_16x16x4_f32.
//
// Bound: one query row block, the codes: 64 sequences of 200-8000 tokens, 32 query and 8
// key/value heads of 128, 101 us with the join, 5.5 TB/s.  64 drafted tokens (16 rows
// of 16 a head), the vector instructions of a tile (some 230 a wave next to 40 matrix
// instructions, hardly at the same time): 4 sequences of 30000-100000 tokens 317 us, 560
// TFLOP/s.  Trees of 33 over 1-5000 tokens, eight sequences of 16 heads, 40.7 us: by the
// workgroups' clocks 2.6 us of plan, 12 (3 to 21) of tiles, 1 to 4 of sums; those that do not
// start with the first 512 start at 18 to 20 and the last ends at 35; then the join.  One
// sequence of 778 tokens 10.5 us: by the same clocks 1 to the first read, 6.5 for up to four
// tiles a wave one after the other, 2 for the waves' sums.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "grid.hpp"
#include "kv_codes.hpp"

namespace ordermoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int DA_WAVES = 4, DA_WAVES_WIDE = 8;       // waves of a workgroup (wide: see launch_type)
constexpr int DA_TILE = 32;                          // tokens of a tile
// Tokens of a piece.  DA_FULL at least, where that gives DA_ONE_EACH workgroups or more
// (pieces of 512: trees of 33 over 1-5000, eight sequences, 47 us for 40.5); else as many
// fewer as give about that many, but DA_MIN_PIECE at least (one sequence of 8000 tokens:
// 1024 19.8 us, 512 15.9, 256 15.3, with the second kernel; 128 is one round of the waves).
constexpr int DA_FULL = 1024, DA_MIN_PIECE = 256, DA_ONE_EACH = 256;
// Tokens of a table up to which sequences are not split: see launch_type
constexpr int DA_WHOLE_WIDE = 1024, DA_WHOLE = 512;
// Workgroups that a large batch is split into: two rounds of the 512 that run together
// (64 tokens over 200-8000 cached: 1024 101 us, 1536 102; trees of 33 over 1-5000: 1024 40.5,
// 1536 43; trees of 64 over 30000-100000: 312, 312)
constexpr int DA_TARGET = 1024;

// 16-row tiles of query rows per workgroup
__host__ __device__ inline int row_tiles(int dtype, int head_dim, int rows) {
    const int most = dtype == ORDERMOE_BF16 ? (head_dim == 256 ? 1 : 2) : 1;
    return rows <= 16 ? 1 : most;
}
__host__ __device__ inline int row_blocks(int rows, int rt) { return (rows + 16 * rt - 1) / (16 * rt); }

struct SeqInfo {
    int first, n, ctx, len;     // first token, drafted tokens, cached tokens before them, positions
};
__device__ inline SeqInfo sequence(const DraftArgs& a, int b) {
    SeqInfo s;
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

// The pieces of the batch, by one wave.  A workgroup's work is a piece of one
// sequence's tokens for one key/value head and one block of its rows; pieces have as
// many tokens, a multiple of `round`, as give about DA_TARGET workgroups in all, but at
// least half of what the batch would ask for with every sequence at max_q: that bounds
// the pieces by 2 DA_TARGET / (n_kv rb_n) + B, since each sequence ends in one short one.
__device__ inline int piece_tokens(const DraftArgs& a, int rb_n, int rt, int round, const SeqInfo& mine, int lane) {
    constexpr int target = DA_TARGET;
    const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
    int64_t total = 0, blocks = 0;
    int ends = 0;                                    // row blocks in all
    for (int b = lane; b < a.B; b += 64) {
        const SeqInfo s = b < 64 ? mine : sequence(a, b);
        const int rb = s.n > 0 ? row_blocks(s.n * G, rt) : 0;
        total += s.n > 0 ? s.len : 0;
        blocks += (int64_t)s.len * rb;
        ends += rb;
    }
    if (a.B > 1) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            total += __shfl_xor(total, o);
            ends += __shfl_xor(ends, o);
            if (rb_n > 1) blocks += __shfl_xor(blocks, o);
        }
    } else {
        total = __shfl(total, 0);
        blocks = __shfl(blocks, 0);
        ends = __shfl(ends, 0);
    }
    if (rb_n == 1) blocks = total;
    // (a sequence's last piece is half a piece on average)
    const int64_t half = (int64_t)ends * n_kv / 2, want = half < target / 2 ? target - half : target / 2;
    int64_t p = (blocks * n_kv + want - 1) / want, few = (blocks * n_kv + DA_ONE_EACH - 1) / DA_ONE_EACH;
    p = p < DA_FULL ? DA_FULL : p;
    few = few < DA_MIN_PIECE ? DA_MIN_PIECE : few;
    p = p < few ? p : few;
    const int64_t least = (total * n_kv * rb_n + 2 * target - 1) / (2 * target);
    p = p < least ? least : p;
    p = (p + round - 1) / round * round;
    return (int)(p > (1 << 30) ? 1 << 30 : p);
}
__device__ inline int pieces_of(const SeqInfo& s, int piece) {
    // a sequence without positions still writes its rows (zeros)
    return s.n <= 0 ? 0 : s.len <= piece ? 1 : (s.len + piece - 1) / piece;
}
// sequence (of number b, < 0: none) and piece j of a work item, by one wave.
// write_plan: every sequence's first item and pieces to a.plan.
__device__ inline SeqInfo find_item(const DraftArgs& a, int piece, int item, int lane, bool write_plan, const SeqInfo& mine, int& b,
                                    int& j) {
    SeqInfo found = {0, 0, 0, 0};
    int base = 0;
    b = -1;
    j = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        SeqInfo s = mine;
        if (b0 > 0 && b0 + lane < a.B) s = sequence(a, b0 + lane);
        const int cnt = b0 + lane < a.B ? pieces_of(s, piece) : 0;
        int inc = cnt;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
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
            found = SeqInfo{__builtin_amdgcn_readlane(s.first, l), __builtin_amdgcn_readlane(s.n, l),
                            __builtin_amdgcn_readlane(s.ctx, l), __builtin_amdgcn_readlane(s.len, l)};
            if (!write_plan) break;
        }
        base += __builtin_amdgcn_readlane(inc, 63);
    }
    return found;
}

// A tile's codes and scales on their way: whole cache lines, 16 bytes a lane (a
// 16-token block is 16 D bytes in a row), and one scale a lane (K's of the 32 tokens,
// then V's).  They go through the wave's own LDS rows into the lane order of the
// operands; rows PITCH = D + 32 bytes apart put the reads of both on distinct banks.
template <int D>
struct Tile {
    u32x4 k[2][D / 64], v[2][D / 64];
    float s;
    bool ok[2];                 // uniform: the block's page is in the cache
};
template <int D>
constexpr int PITCH = D + 32;
template <int D>
constexpr int STAGE = 64 * PITCH<D> + 64 * 4;        // bytes of a wave: 32 rows of K, 32 of V, 64 scales

// pages of the tile's two 16-token blocks (16 tokens never cross a page), -1: none; uniform, through the
// scalar cache
struct Pages { int p[2]; };
__device__ inline Pages tile_pages(const DraftArgs& a, const int32_t* table, int t0, int len) {
    const __attribute__((address_space(4))) int32_t* t = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)table;
    Pages r;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const int p = t0 + 16 * tb;
        r.p[tb] = p < len ? t[p >> a.cache.page_shift] : -1;
    }
    return r;
}

// NTL: past the caches (see launch_rows)
template <bool NTL>
__device__ inline u32x4 load_codes(const uint8_t* p) {
    if constexpr (NTL) return __builtin_nontemporal_load((const u32x4*)p);
    else return *(const u32x4*)p;
}

template <int D, bool NTL>
__device__ inline void load_tile(const DraftArgs& a, const Pages& pg, int kvh, int t0, int lane, Tile<D>& t) {
    const int sh = a.cache.page_shift;
    int64_t row[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const int pid = pg.p[tb];
        t.ok[tb] = pid >= 0 && pid < a.cache.n_pages;
        // a block without a page reads page 0
        row[tb] = t.ok[tb] ? ((((int64_t)pid * a.cache.n_kv + kvh) << sh) + ((t0 + 16 * tb) & ((1 << sh) - 1))) : 0;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            t.k[tb][i] = load_codes<NTL>(a.cache.k_codes + row[tb] * D + (uint32_t)(lane * 16 + 1024 * i));
            t.v[tb][i] = load_codes<NTL>(a.cache.v_codes + row[tb] * D + (uint32_t)(lane * 16 + 1024 * i));
        }
    }
    const float* sc = lane < 32 ? a.cache.k_scale : a.cache.v_scale;
    t.s = sc[(lane & 16 ? row[1] : row[0]) + (lane & 15)];
}
// edge: some row may not see some token.  A weight of 0 would not keep a code that is no number (e4m3; a place
// that was never written may hold one) out of that row's sums, so V's become zeros and the token's scale a NaN:
// the rows that see it are no numbers all the same.  (In other tiles every row sees every token.)
template <int D, int FMT>
__device__ inline void stage_tile(const Tile<D>& t, char* st, int lane, float scale2, bool edge) {
    constexpr int CH = D / 16;                       // 16-byte chunks of a row
    char* p = st + (lane / CH) * PITCH<D> + (lane % CH) * 16;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            *(u32x4*)(p + (16 * tb + 64 / CH * i) * PITCH<D>) = t.k[tb][i];
            *(u32x4*)(p + (32 + 16 * tb + 64 / CH * i) * PITCH<D>) = t.v[tb][i];
        }
    *(float*)(st + 64 * PITCH<D> + 4 * lane) = lane < 32 ? t.s * scale2 : t.s;   // (K's in units of the scores)
    if constexpr (FMT == ORDERMOE_CACHE_FP8) {
        if (edge) {
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    uint32_t nan = 0u;                           // the top bits of the bytes that are 0x7F but for their sign
#pragma unroll
                    for (int w = 0; w < 4; ++w) nan |= ~((~t.v[tb][i][w] & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) & 0x80808080u;
                    if (nan) {
                        const int row = 32 + 16 * tb + 64 / CH * i;
                        *(u32x4*)(p + row * PITCH<D>) = u32x4{0u, 0u, 0u, 0u};
                        *(float*)(st + 64 * PITCH<D> + 4 * (row + lane / CH)) = __builtin_nanf("");
                    }
                }
        }
    }
}

// The running state of a wave: per row tile, lane (c, g) has row c's maximum (in
// units of log 2; a shared reference that may lag behind the true one, see
// below) and its own tokens' share of the sum; o[j] holds rows' elements
// (4g + i) D/16 + j, i = 0 .. 3.
template <int D, int RT>
struct State {
    float m[RT], l[RT];
    f32x4 o[D / 16][RT];
};
// A maximum is taken over only when some score passes it by 8 (a factor of 256 in
// the weights, which fp32 sums and bf16 weights hold as well as 1): most tiles then
// need no exchange between lanes and no rescaling of the outputs.
constexpr float DA_LAG = 8.0f;

template <int N>
struct Queries { bf16x8 b[N]; };

// FINE: the second product takes what the rounding of the weights to bf16 leaves out as well
template <bool BF, int D, int FMT, int RT, bool FINE>
__device__ inline __attribute__((always_inline)) void attend_tile(const char* stage, const bool* ok, const void* qv, const uint64_t* word,
                                   int t0, const SeqInfo& s, int lane, State<D, RT>& st) {
    const int c = lane & 15, g = lane >> 4;
    const f32x4* scales = (const f32x4*)(stage + 64 * PITCH<D>) + g;     // of tokens 4g .. 4g + 3
    f32x4 sc[2][RT] = {};
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            // K: token c, elements 64 i + 16 g .. + 15
            const u32x4 kc = *(const u32x4*)(stage + (16 * tb + c) * PITCH<D> + 64 * i + 16 * g);
            if constexpr (BF) {
                const Queries<RT * D / 32>& q = *(const Queries<RT * D / 32>*)qv;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x4 kf;
                    kf[0] = kv_to_bf16x2<FMT, 0>(kc[2 * h]);
                    kf[1] = kv_to_bf16x2<FMT, 1>(kc[2 * h]);
                    kf[2] = kv_to_bf16x2<FMT, 0>(kc[2 * h + 1]);
                    kf[3] = kv_to_bf16x2<FMT, 1>(kc[2 * h + 1]);
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        sc[tb][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf),
                                                                            q.b[r * (D / 32) + 2 * i + h], sc[tb][r], 0, 0, 0);
                }
            } else {
                const float* q = (const float*)qv;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const uint32_t w = kc[h];
                    const float kf[4] = {kv_to_f32<FMT, 0>(w), kv_to_f32<FMT, 1>(w), kv_to_f32<FMT, 2>(w), kv_to_f32<FMT, 3>(w)};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        sc[tb][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], q[16 * i + 4 * h + e], sc[tb][0], 0, 0, 0);
                }
            }
        }
    }
    const float ninf = -__builtin_inff();
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const f32x4 ks = scales[4 * tb];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[tb][r][i] *= ks[i];
    }
    const bool edge = t0 + DA_TILE > s.ctx || !ok[0] || !ok[1];
    uint32_t hidden[RT];                                         // the lane's 8 tokens, a bit each
    if (edge) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            hidden[r] = 0u;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int p = t0 + 16 * (u >> 2) + 4 * g + (u & 3), j = p - s.ctx;
                const bool seen = ok[u >> 2] && p < s.len && (j < 0 || ((word[r] >> (j & 63)) & 1));
                hidden[r] |= (uint32_t)!seen << u;
                sc[u >> 2][r][u & 3] = seen ? sc[u >> 2][r][u & 3] : ninf;
            }
        }
    }
    float top[RT];
    bool past = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        top[r] = ninf;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[r] = fmaxf(top[r], sc[tb][r][i]);
        past |= top[r] > st.m[r] + DA_LAG;
    }
    if (__builtin_amdgcn_ballot_w64(past)) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float x = fmaxf(top[r], __shfl_xor(top[r], 16));
            x = fmaxf(x, __shfl_xor(x, 32));
            const float m = x > st.m[r] + DA_LAG ? x : st.m[r];      // by the row alone, whatever the others do
            const float al = st.m[r] == m ? 1.0f : __builtin_amdgcn_exp2f(st.m[r] - m);
            st.m[r] = m;
            st.l[r] *= al;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) st.o[j][r] = st.o[j][r] * al;
        }
    }
    // weights exp2(score - maximum), 0 where nothing has been seen yet
    float pw[RT][8];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float m = st.m[r] == ninf ? 0.f : st.m[r];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const f32x4 vs = scales[8 + 4 * tb];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(sc[tb][r][i] - m);
                st.l[r] += p;
                pw[r][4 * tb + i] = p * vs[i];
            }
        }
    }
    if (edge) {
        // an unseen token's scale may be no number
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int u = 0; u < 8; ++u) pw[r][u] = (hidden[r] >> u) & 1 ? 0.f : pw[r][u];
    }
    __builtin_amdgcn_sched_barrier(0);               // (V's registers only from here on)
    // V: tokens 4g .. 4g + 3 of each block, elements [c D/16, (c + 1) D/16)
    uint32_t v[8][D / 64];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const char* r = stage + (32 + 16 * (u >> 2) + 4 * g + (u & 3)) * PITCH<D> + c * (D / 16);
        if constexpr (D == 64) {
            v[u][0] = *(const uint32_t*)r;
        } else if constexpr (D == 128) {
            const u32x2 w = *(const u32x2*)r;
            v[u][0] = w[0]; v[u][1] = w[1];
        } else {
            const u32x4 w = *(const u32x4*)r;
            v[u][0] = w[0]; v[u][1] = w[1]; v[u][2] = w[2]; v[u][3] = w[3];
        }
    }
    if constexpr (BF) {
        // a kernel of one row tile has the matrix unit's time for it (the codes' reads bound it)
        bf16x8 pf[RT], pl = {};
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                pf[r][u] = (__bf16)pw[r][u];
                if constexpr (FINE) pl[u] = (__bf16)(pw[r][u] - (float)pf[r][u]);
            }
#pragma unroll
        for (int w = 0; w < D / 64; ++w) {
            u32x4 vf[4];                                         // elements 4w .. 4w + 3, tokens in pairs
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if constexpr (FMT == ORDERMOE_CACHE_INT8) {
                    vf[0][u] = kv_bf16_pair(kv_to_f32<FMT, 0>(v[2 * u][w]), kv_to_f32<FMT, 0>(v[2 * u + 1][w]));
                    vf[1][u] = kv_bf16_pair(kv_to_f32<FMT, 1>(v[2 * u][w]), kv_to_f32<FMT, 1>(v[2 * u + 1][w]));
                    vf[2][u] = kv_bf16_pair(kv_to_f32<FMT, 2>(v[2 * u][w]), kv_to_f32<FMT, 2>(v[2 * u + 1][w]));
                    vf[3][u] = kv_bf16_pair(kv_to_f32<FMT, 3>(v[2 * u][w]), kv_to_f32<FMT, 3>(v[2 * u + 1][w]));
                } else {
                    // bytes b of tokens 2u and 2u + 1 side by side: b = 0, 1 and b = 2, 3
                    const uint32_t lo = __builtin_amdgcn_perm(v[2 * u + 1][w], v[2 * u][w], 0x05010400u);
                    const uint32_t hi = __builtin_amdgcn_perm(v[2 * u + 1][w], v[2 * u][w], 0x07030602u);
                    vf[0][u] = kv_to_bf16x2<FMT, 0>(lo);
                    vf[1][u] = kv_to_bf16x2<FMT, 1>(lo);
                    vf[2][u] = kv_to_bf16x2<FMT, 0>(hi);
                    vf[3][u] = kv_to_bf16x2<FMT, 1>(hi);
                }
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    st.o[4 * w + b][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[b]), pf[r],
                                                                                 st.o[4 * w + b][r], 0, 0, 0);
                if constexpr (FINE)
                    st.o[4 * w + b][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[b]), pl,
                                                                                 st.o[4 * w + b][0], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int w = 0; w < D / 64; ++w)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t x = v[u][w];
                const float vf[4] = {kv_to_f32<FMT, 0>(x), kv_to_f32<FMT, 1>(x), kv_to_f32<FMT, 2>(x), kv_to_f32<FMT, 3>(x)};
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    st.o[4 * w + b][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[b], pw[0][u], st.o[4 * w + b][0], 0, 0, 0);
            }
    }
}

// out = sum / l (0 where nothing was seen), N elements of a row
template <bool BF, int N>
__device__ inline void write_row(void* out, int64_t at, const float* x, float l) {
    const float r = l == 0.f ? 0.f : 1.0f / l;
    if constexpr (BF) {
        __bf16* o = (__bf16*)out + at;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            kv_bf16x2 u, v;
            u[0] = (__bf16)(x[i] * r); u[1] = (__bf16)(x[i + 1] * r);
            v[0] = (__bf16)(x[i + 2] * r); v[1] = (__bf16)(x[i + 3] * r);
            *(u32x2*)(o + i) = u32x2{__builtin_bit_cast(uint32_t, u), __builtin_bit_cast(uint32_t, v)};
        }
    } else {
        float* o = (float*)out + at;
#pragma unroll
        for (int i = 0; i < N; i += 4) *(f32x4*)(o + i) = f32x4{x[i] * r, x[i + 1] * r, x[i + 2] * r, x[i + 3] * r};
    }
}
constexpr float LN2 = 0.69314718055994531f;
__device__ inline float row_lse(float m, float l) {
    return l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// waves per SIMD that the registers leave room for (two tiles on their way take 66,
// the outputs D / 4 per row tile; four row tiles at one wave per SIMD took 932 us where
// two at two take 360)
template <int D>
constexpr int OCC = D == 256 ? 1 : 2;

// What a workgroup's rows are attended to with: LDS for the codes' staging rows, then the waves' sums (in one place),
// and for their maxima and sums
template <int D, int NW>
constexpr int SUMS = NW * 16 * (D + 4) * 4;
template <int D, int RT, int NW>
struct Shared {
    __attribute__((aligned(16))) char mem[NW * STAGE<D> > SUMS<D, NW> ? NW * STAGE<D> : SUMS<D, NW>];
    float m[NW][RT * 16], l[NW][RT * 16];
};

// rows row0 .. row0 + 16 RT - 1 (of `rows`) of key/value head kvh over tokens [t_lo, t_hi) of a sequence.  NTL: see
// load_codes, FINE: see attend_tile
template <bool BF, int D, int FMT, int RT, int NW, bool FINE, bool NTL>
__device__ inline __attribute__((always_inline)) void attend_rows(const DraftArgs& a, const SeqInfo& s, int item, int kvh, int row0,
                                                                  int rows, int pieces, int t_lo, int t_hi, const int32_t* table,
                                                                  char* s_mem, float (*s_m)[RT * 16], float (*s_l)[RT * 16]) {
    constexpr int LD = D + 4, ROUND = NW * DA_TILE;
    float (*const s_o)[16][LD] = (float (*)[16][LD])s_mem;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
    // query rows: row = token * G + head; rows past the end are zeros and see nothing
    constexpr int NQ = BF ? RT * D / 32 : 1;
    Queries<NQ> qb;
    float qf[BF ? 1 : D / 4];
    uint64_t word[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = row0 + 16 * r + c;
        const bool in = row < rows;
        const int i = in ? row / G : 0, h = kvh * G + (in ? row - i * G : 0);
        // lane group g holds elements 16 g .. 16 g + 15 of every 64
        const int64_t at = ((int64_t)(s.first + i) * a.n_q + h) * D + 16 * g;
        // a chain's word: bits 0 .. i
        word[r] = !in ? 0ull : a.tree ? a.tree[s.first + i] : ~0ull >> (63 - i);
        if constexpr (BF) {
#pragma unroll
            for (int e = 0; e < D / 32; ++e) {
                bf16x8 v = {};
                if (in) v = *(const bf16x8*)((const __bf16*)a.q + at + 64 * (e >> 1) + 8 * (e & 1));
                qb.b[r * (D / 32) + e] = v;
            }
        } else {
#pragma unroll
            for (int e = 0; e < D / 16; ++e) {
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
                if (in) v = *(const f32x4*)((const float*)a.q + at + 64 * (e >> 2) + 4 * (e & 3));
#pragma unroll
                for (int f = 0; f < 4; ++f) qf[4 * e + f] = v[f];
            }
        }
    }
    const void* qv = BF ? (const void*)&qb : (const void*)qf;
    State<D, RT> st;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.m[r] = -__builtin_inff();
        st.l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) st.o[e][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = a.scale * 1.44269504088896341f;        // scores in units of log 2
    // two tiles are on their way while one is attended to
    Tile<D> t[2];
    char* const stage = s_mem + wave * STAGE<D>;
    int p = t_lo + wave * DA_TILE;
    Pages pg = tile_pages(a, table, p, t_hi);
    load_tile<D, NTL>(a, pg, kvh, p, lane, t[0]);
    pg = tile_pages(a, table, p + ROUND, t_hi);
    load_tile<D, NTL>(a, pg, kvh, p + ROUND, lane, t[1]);
    pg = tile_pages(a, table, p + 2 * ROUND, t_hi);
    auto step = [&](Tile<D>& u) __attribute__((always_inline)) {
        const bool ok[2] = {u.ok[0], u.ok[1]};
        stage_tile<D, FMT>(u, stage, lane, scale2, p + DA_TILE > s.ctx || !ok[0] || !ok[1]);
        load_tile<D, NTL>(a, pg, kvh, p + 2 * ROUND, lane, u);
        pg = tile_pages(a, table, p + 3 * ROUND, t_hi);
        attend_tile<BF, D, FMT, RT, FINE>(stage, ok, qv, word, p, s, lane, st);
        p += ROUND;
    };
    while (p < t_hi) {
        step(t[0]);
        if (p >= t_hi) break;
        step(t[1]);
    }

    __syncthreads();                                 // the staging rows become the place of the sums
    // the waves' states joined, a row tile at a time
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float l = st.l[r];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) { s_m[wave][16 * r + c] = st.m[r]; s_l[wave][16 * r + c] = l; }
    }
    __syncthreads();
    const int64_t prow = ((int64_t)item * n_kv + kvh) * (a.max_q * G);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (row0 + 16 * r >= rows) break;
        float m = s_m[0][16 * r + c];
#pragma unroll
        for (int w = 1; w < NW; ++w) m = fmaxf(m, s_m[w][16 * r + c]);
        const float f = st.m[r] == m ? 1.0f : __builtin_amdgcn_exp2f(st.m[r] - m);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < D / 16; e += 4)
                *(f32x4*)&s_o[wave][c][(4 * g + i) * (D / 16) + e] =
                    f32x4{st.o[e][r][i], st.o[e + 1][r][i], st.o[e + 2][r][i], st.o[e + 3][r][i]} * f;
        __syncthreads();
        // 16 threads a row, D / 16 elements each
        const int row = tid >> 4, rr = row0 + 16 * r + row, d0 = (tid & 15) * (D / 16);
        if (row < 16 && rr < rows) {
            float mm = s_m[0][16 * r + row], l = 0.f;
#pragma unroll
            for (int w = 1; w < NW; ++w) mm = fmaxf(mm, s_m[w][16 * r + row]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float mw = s_m[w][16 * r + row];
                l += s_l[w][16 * r + row] * (mw == mm ? 1.0f : __builtin_amdgcn_exp2f(mw - mm));
            }
            float x[D / 16];
#pragma unroll
            for (int e = 0; e < D / 16; e += 4) {
                f32x4 v = *(const f32x4*)&s_o[0][row][d0 + e];
#pragma unroll
                for (int w = 1; w < NW; ++w) v += *(const f32x4*)&s_o[w][row][d0 + e];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[e + k] = v[k];
            }
            if (pieces > 1) {
                float* po = a.part_o + (prow + rr) * D + d0;
#pragma unroll
                for (int e = 0; e < D / 16; e += 4) *(f32x4*)(po + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
                if ((tid & 15) == 0) {
                    a.part_ml[2 * (prow + rr)] = mm;
                    a.part_ml[2 * (prow + rr) + 1] = l;
                }
            } else {
                const int i = rr / G, h = kvh * G + rr - i * G;
                const int64_t at = (int64_t)(s.first + i) * a.n_q + h;
                write_row<BF, D / 16>(a.out, at * D + d0, x, l);
                if (a.lse && (tid & 15) == 0) a.lse[at] = row_lse(mm, l);
            }
        }
        __syncthreads();
    }
}

template <bool BF, int D, int FMT, int RT, int NW, bool NTL>
__global__ void __launch_bounds__(64 * NW, OCC<D>) draft_attention_kernel(const DraftArgs a, int items, int rb_n, int whole) {
    constexpr int ROUND = NW * DA_TILE;
    __shared__ Shared<D, RT, NW> sh;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the row blocks of one piece and head on one XCD, where its codes are in L2
    const int idx = (int)block_number(), jx = idx >> 3;
    const int unit = (jx / rb_n) * 8 + (idx & 7), rb = jx % rb_n;
    const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
    if (unit >= items * n_kv) return;
    const int item = unit / n_kv, kvh = unit - item * n_kv;
    int piece = 1 << 30, b = item, j = 0;
    SeqInfo s;
    if (whole) {
        s = sequence(a, b);                          // every sequence is one piece
    } else {
        SeqInfo mine = {0, 0, 0, 0};
        if (lane < a.B) mine = sequence(a, lane);
        // (the same in every lane, and in scalar registers from here on: addresses and branches below rest on it)
        piece = __builtin_amdgcn_readfirstlane(piece_tokens(a, rb_n, RT, ROUND, mine, lane));
        s = find_item(a, piece, item, lane, idx == 0 && wave == 0, mine, b, j);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    j = __builtin_amdgcn_readfirstlane(j);
    s = SeqInfo{__builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.n), __builtin_amdgcn_readfirstlane(s.ctx),
                __builtin_amdgcn_readfirstlane(s.len)};
    if (b < 0) return;
    const int rows = s.n * G, row0 = rb * 16 * RT;
    if (row0 >= rows) return;
    const int pieces = pieces_of(s, piece);
    const int t_lo = j * piece, t_hi = s.len - t_lo < piece ? s.len : t_lo + piece;
    const int32_t* table = a.page_table + (int64_t)b * a.max_pages;
    if constexpr (RT > 1) {
        // A last block of up to 16 rows, or a sequence of no more (ragged trees of 33 44 -> 41 us, of 64 325 -> 312).  FINE,
        // as with one row tile: a token's bits do not go with how many its neighbours in the batch have drafted
        // (trees of 33 40.0 -> 40.7 us, of 64 312 -> 317).
        if (rows - row0 <= 16) {
            attend_rows<BF, D, FMT, 1, NW, true, false>(a, s, item, kvh, row0, rows, pieces, t_lo, t_hi, table, sh.mem,
                                                  (float (*)[16])sh.m, (float (*)[16])sh.l);
            return;
        }
    }
    attend_rows<BF, D, FMT, RT, NW, RT == 1, NTL>(a, s, item, kvh, row0, rows, pieces, t_lo, t_hi, table, sh.mem, sh.m, sh.l);
}

// 16 / S (token, head) rows of a sequence per workgroup, S sets of 16 lanes a row: set z
// adds pieces z, z + S, .., and the sets' sums are added in order
template <bool BF, int D, int S>
__global__ void __launch_bounds__(256) draft_join_kernel(const DraftArgs a, int rows_n) {
    constexpr int R = 16 / S, U = 4;                             // rows; pieces whose reads are in flight
    __shared__ __attribute__((aligned(16))) float s_x[16][D + 4];
    __shared__ float s_m[16], s_l[16];
    const int idx = (int)block_number(), b = idx / rows_n;
    if (b >= a.B) return;
    const int pieces = a.plan[2 * b + 1];
    if (pieces <= 1) return;
    const SeqInfo s = sequence(a, b);
    const int slot = threadIdx.x >> 4, z = slot % S, rows = s.n * a.n_q;
    const int r = (idx - b * rows_n) * R + slot / S;
    const int item = a.plan[2 * b], n_kv = a.cache.n_kv, G = a.n_q / n_kv;
    const int i = r / a.n_q, h = r - i * a.n_q, kvh = h / G;
    const int64_t stride = (int64_t)n_kv * a.max_q * G;          // rows of a piece
    const int64_t row = ((int64_t)item * n_kv + kvh) * (a.max_q * G) + i * G + (h - kvh * G);
    const int d0 = (threadIdx.x & 15) * (D / 16);
    const f32x2* ml = (const f32x2*)a.part_ml;
    float m = -__builtin_inff(), l = 0.f, x[D / 16] = {};
    for (int p = r < rows ? z : pieces; p < pieces; p += U * S) {
        f32x2 q[U];
        f32x4 v[U][D / 64];
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = row + (p + u * S < pieces ? p + u * S : p) * stride;
            q[u] = ml[at];
#pragma unroll
            for (int e = 0; e < D / 64; ++e) v[u][e] = *(const f32x4*)(a.part_o + at * D + d0 + 4 * e);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, q[u][0]);
        const float al = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= al;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) x[e] *= al;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * S >= pieces) break;
            const float f = q[u][0] == m ? 1.0f : __builtin_amdgcn_exp2f(q[u][0] - m);
            l += q[u][1] * f;
#pragma unroll
            for (int e = 0; e < D / 16; ++e) x[e] += v[u][e / 4][e % 4] * f;
        }
    }
    if constexpr (S > 1) {
        if ((threadIdx.x & 15) == 0) { s_m[slot] = m; s_l[slot] = l; }
#pragma unroll
        for (int e = 0; e < D / 16; e += 4) *(f32x4*)&s_x[slot][d0 + e] = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        __syncthreads();
        if (z != 0) return;
        float mm = m;
#pragma unroll
        for (int u = 1; u < S; ++u) mm = fmaxf(mm, s_m[slot + u]);
        const float al = m == mm ? 1.0f : __builtin_amdgcn_exp2f(m - mm);
        m = mm;
        l *= al;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) x[e] *= al;
        for (int u = 1; u < S && u < pieces; ++u) {
            const float f = s_m[slot + u] == m ? 1.0f : __builtin_amdgcn_exp2f(s_m[slot + u] - m);
            l += s_l[slot + u] * f;
#pragma unroll
            for (int e = 0; e < D / 16; ++e) x[e] += s_x[slot + u][d0 + e] * f;
        }
    }
    if (r >= rows) return;
    const int64_t at = (int64_t)(s.first + i) * a.n_q + h;
    write_row<BF, D / 16>(a.out, at * D + d0, x, l);
    if (a.lse && (threadIdx.x & 15) == 0) a.lse[at] = row_lse(m, l);
}

// rows (of all sequences) up to which a row gets 16 sets of lanes, or 4: 40 pieces of
// 32 rows 16 sets 7 us, one 21; 6 of 8192 rows 4 sets 9 us, one 12
constexpr int64_t JOIN_16 = 1024, JOIN_4 = 16384;

int64_t table_tokens(const DraftArgs& a) { return (int64_t)a.max_pages << a.cache.page_shift; }

template <bool BF, int D, int FMT, int RT, int NW>
int launch_rows(const DraftArgs& a, int rows, bool whole, hipStream_t st) {
    const int rb = row_blocks(rows, RT);
    // (workgroups without a piece are not free: a sequence has no more of them than its table holds)
    const int64_t most = whole ? a.B : (int64_t)a.B * ((table_tokens(a) + DA_MIN_PIECE - 1) / DA_MIN_PIECE);
    const int64_t items = std::min(most, draft_items(a.n_q, a.cache.n_kv, D, a.dtype, a.B, a.max_q));
    const int64_t units = (items * a.cache.n_kv + 7) / 8 * 8;
    {
        KernelTimer kt_("draft_attention", st);
        auto attend = [&](auto ntl) {
            draft_attention_kernel<BF, D, FMT, RT, NW, decltype(ntl)::value>
                <<<grid_of(units * rb), dim3(64 * NW), 0, st>>>(a, (int)items, rb, whole);
        };
        // Codes are read past the caches unless several row blocks share them: with two row tiles, and with heads of 256
        // (four sequences, trees of 16 and 64: 4000 tokens 48.3 -> 43.6 us and 89.7 -> 81.7, 30000 204 -> 194 and 419 -> 400).
        // Not in fp32, whose blocks wait for the matrix unit (the same with heads of 128: 58.4, 58.7; 144, 142; 328, 330; 869, 869).
        if constexpr (BF && D == 256)
            if (rb > 1) attend(std::false_type{});
            else attend(std::true_type{});
        else
            attend(std::bool_constant<RT == 1>{});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    if (whole) return 0;
    KernelTimer kt_("draft_join", st);
    const int64_t all = (int64_t)a.B * a.max_q * a.n_q;
    auto join = [&](auto sets) {
        constexpr int S = decltype(sets)::value;
        const int rows_n = (a.max_q * a.n_q + 16 / S - 1) / (16 / S);
        draft_join_kernel<BF, D, S><<<grid_of((int64_t)a.B * rows_n), dim3(256), 0, st>>>(a, rows_n);
    };
    if (all <= JOIN_16) join(std::integral_constant<int, 16>{});
    else if (all <= JOIN_4) join(std::integral_constant<int, 4>{});
    else join(std::integral_constant<int, 1>{});
    return (int)hipGetLastError();
}

template <bool BF, int D, int FMT>
int launch_type(const DraftArgs& a, hipStream_t st) {
    const int rows = a.max_q * (a.n_q / a.cache.n_kv), rt = row_tiles(a.dtype, D, rows);
    const int64_t table = table_tokens(a);
    // Sequences that the host knows to be short are not split, which saves the second
    // kernel.  With a workgroup per compute unit all the same: those of a whole piece; else
    // as long as one workgroup takes less time than pieces and join (one sequence, whole and
    // split: bf16 500 tokens 9.3 and 12.8 us, 1000 13.0 and 12.7; fp32 500 17.4 and 16.8;
    // heads of 256, 500 15.9 and 16.3; trees of 33, 470 12.3 and 15.3, 900 17.8 and 15.4).
    const bool many = (int64_t)a.B * a.cache.n_kv * row_blocks(rows, rt) >= DA_ONE_EACH;
    if (many || rt > 1 || D == 256) {
        const bool whole = table <= (many ? DA_FULL : DA_WHOLE);
        if constexpr (BF && D != 256)
            if (rt == 2) return launch_rows<BF, D, FMT, 2, DA_WAVES>(a, rows, whole, st);
        return launch_rows<BF, D, FMT, 1, DA_WAVES>(a, rows, whole, st);
    }
    // one row tile, eight waves (not with heads of 256, whose registers eight waves do not have)
    if constexpr (D != 256)
        if (table <= (BF ? DA_WHOLE_WIDE : DA_WHOLE)) return launch_rows<BF, D, FMT, 1, DA_WAVES_WIDE>(a, rows, true, st);
    return launch_rows<BF, D, FMT, 1, DA_WAVES>(a, rows, false, st);
}
template <bool BF, int D>
int launch_fmt(const DraftArgs& a, hipStream_t st) {
    return a.cache.format == ORDERMOE_CACHE_INT8 ? launch_type<BF, D, ORDERMOE_CACHE_INT8>(a, st)
                                                 : launch_type<BF, D, ORDERMOE_CACHE_FP8>(a, st);
}
template <bool BF>
int launch_dim(const DraftArgs& a, hipStream_t st) {
    return a.cache.head_dim == 64    ? launch_fmt<BF, 64>(a, st)
           : a.cache.head_dim == 128 ? launch_fmt<BF, 128>(a, st)
                                     : launch_fmt<BF, 256>(a, st);
}

}  // namespace

int64_t draft_items(int n_q, int n_kv, int head_dim, int dtype, int B, int max_q) {
    const int rows = max_q * (n_q / n_kv);
    const int rb = row_blocks(rows, row_tiles(dtype, head_dim, rows));
    const int64_t units = (int64_t)n_kv * rb;
    return (2 * DA_TARGET + units - 1) / units + B;
}

int launch_draft_attention(const DraftArgs& a, void* stream) {
    if (a.B == 0 || a.T == 0) return 0;
    return a.dtype == ORDERMOE_BF16 ? launch_dim<true>(a, (hipStream_t)stream) : launch_dim<false>(a, (hipStream_t)stream);
}

}  // namespace ordermoe
