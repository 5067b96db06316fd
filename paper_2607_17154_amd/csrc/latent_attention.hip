// Attention of drafted tokens over the latent cache: every head's absorbed query on the
// same rows [c_p | r_p], of which the first part is the value too.
//
//   latent_attention_kernel  one workgroup per (work item, block of 16 or 32 query rows).  A work
//                            item is a piece of one sequence's cache, gone through in tiles that all
//                            waves share -> sums relative to the piece's maximum (memory)
//   latent_rows_kernel       the same for sequences of many query rows: blocks of 128, 16 of them
//                            a wave
//   latent_out_kernel        the pieces' sums added in order, relative to their largest maximum,
//                            divided, and taken through W_v: 16 tokens of one head
//   latent_mass_kernel       the weight that each position got, from the scores that the first
//                            kernel wrote and the rows' final maximum and sum
// The query rows of a sequence are its n_b tokens times the heads: row = token * n_q + head.
//
// A tile of 32 tokens (latent_rows_kernel: 64; c = lane % 16, g = lane / 16; fp32 v_mfma_f32_16x16x4_f32 for each):
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16; rows: 16 tokens, columns: 16 query rows.  Maximum and sum belong to a
//                 column, that is to a lane.
//   O^T = C^T P^T rows: 16 elements of the latent vector, columns: 16 query rows, tokens the inner index; C^T by turned
//                 reads of the rows in LDS (where tokens lie apart).
// latent_attention_kernel: a wave forms the scores of 16 tokens and 16 query rows, and the sums of its share of the
// elements, so that every row in LDS is read once for them and the outputs take few registers.  The maxima of a tile
// go through LDS, so that all waves come to the same reference, and so do the weights: three barriers a tile.
// latent_rows_kernel: a wave has 16 rows and all elements; the weights of two score blocks (tokens 4g .. 4g + 3 of each in
// lane (c, g)) are the inner indexes of its second product when C^T's lanes hold the same tokens, so they never leave their
// registers: one barrier a tile.  It reads each row in LDS eight times for 128 query rows, which bounds it (128 bytes a
// cycle); blocks of 64 rows in the first way read it less than half as often but waited for each other: trees of 64 over
// 30000-100000 tokens 993 us for 513, before loads were told apart from reads (482).
// Rows go straight from memory into LDS, the next tile while one is attended to.  64 sequences of 200 to 8000 tokens, one token
// of 32 heads, rank 512: 67 us, 4.6 TB/s, by the rows on their way; trees of 64 482 (790 TFLOP/s).
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
// Tokens of a piece, at least: 64, and a tile of 32 alone in fp32 and for batches of up to LA_SHORT tokens, whose latency it
// shortens (200 tokens 12.6 -> 11.6 us, two fp32 sequences of 800 22.4 -> 18.2; 4 of 1000 15.5 -> 17.1, 16 of 300 16.5 -> 19.3)
constexpr int LA_MIN_PIECE = 64, LA_SHORT = 1024;
constexpr int LA_FEW = 32;                           // query rows up to which latent_attention_kernel takes a batch
constexpr int LO_PIECES = 32;                        // pieces of a sequence, as expected, past which 16 sets of lanes add them
constexpr int LO_GROUPS = 256;                       // workgroups of the last product wished for
constexpr float LA_LAG = 8.0f;                       // see latent_attention_kernel

// 16-row tiles of query rows per workgroup, for sequences of up to `rows` query rows (8: latent_rows_kernel)
__host__ __device__ inline int row_tiles(int dtype, int rows) { return rows <= 16 ? 1 : rows <= LA_FEW || dtype != ORDERMOE_BF16 ? 2 : 8; }
__host__ __device__ inline int row_blocks(int rows, int mt) { return (rows + 16 * mt - 1) / (16 * mt); }

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
__device__ inline int piece_tokens(const LatentAttentionArgs& a, int rb_n, int mt, int round, const Seq& mine, int lane) {
    int64_t total = 0, blocks = 0;
    for (int b = lane; b < a.B; b += 64) {
        const Seq s = b < 64 ? mine : sequence(a, b);
        total += s.n > 0 ? s.len : 0;
        blocks += s.n > 0 ? (int64_t)s.len * row_blocks(s.n * a.n_q, mt) : 0;
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
    // One round of the workgroups that run together, each sequence's short last piece counted in (64 sequences of 200 to 8000
    // tokens: 32 heads 111 us without, 84); blocks of 128 rows take two rounds (157 us in one, 128 heads, 139)
    const int64_t ends = mt == 8 ? 0 : (int64_t)a.B * rb_n, want = ends < LA_TARGET / 2 ? LA_TARGET - ends : LA_TARGET / 2;
    int64_t p = (blocks + want - 1) / want;
    const int64_t least = (total * rb_n + 2 * LA_TARGET - 1) / (2 * LA_TARGET);
    p = p < least ? least : p;
    const int min_piece = a.cache.dtype == ORDERMOE_F32 || total <= LA_SHORT ? LA_MIN_PIECE / 2 : LA_MIN_PIECE;
    p = p < min_piece ? min_piece : p;
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
template <bool BF, int R_, int ROT, int MT>
struct Config {
    static constexpr int ES = BF ? 2 : 4, R = R_, RB = (R + ROT) * ES;
    static constexpr int NW = MT == 8 ? 8 : 4;                               // waves
    static constexpr int QT = MT == 8 ? 4 : 2, TILE = 16 * QT;               // 16-token blocks, tokens of a tile
    static constexpr int CT = R / 16 / NW;                                   // 16-element tiles whose sums a wave holds
    static constexpr int PANELS = RB / 128, TAIL = PANELS * TILE * 128;      // whole panels, where the rest begins
    static constexpr bool HAS_TAIL = RB % 128 != 0;
    static constexpr int STAGE = TILE * RB, OCTETS = TILE / 8 / NW;          // bytes of a tile, a wave's eights of its rows
    static constexpr int KS = RB / 64;                                       // steps of the first product
    static constexpr int PP = TILE * ES + 16;                                // bytes of a row of weights in LDS
    static constexpr int LD = R + 4;                                         // floats of a row of sums in LDS
    static_assert(RB % 64 == 0 && R * ES % 128 == 0 && OCTETS * 8 * NW == TILE && (MT == 8 || CT * 16 * NW == R), "whole shares");
};

// The pages of a piece's tiles, 16 tokens each (they never cross a page), -1: none.  Lane i holds the page of block 64 j + i,
// so that the loop has no loads through the scalar cache: those return in no order with reads of LDS, which would all wait
// for them.
template <int QT>
struct Pages {
    const int32_t* table;
    int t_lo, t_hi, shift, now, after;
    __device__ int load(int j, int lane) const {
        const int64_t t = t_lo + 16 * (64 * (int64_t)j + lane);
        return t < t_hi ? table[t >> shift] : -1;
    }
    __device__ void start(const LatentAttentionArgs& a, int b, int lo, int hi, int lane) {
        table = a.page_table + (int64_t)b * a.max_pages;
        t_lo = lo;
        t_hi = hi;
        shift = a.cache.page_shift;
        now = load(0, lane);
        after = load(1, lane);
    }
    struct Tile { int p[QT]; };
    // of tile k; to be called for one tile after the other
    __device__ Tile tile(int k, int lane) {
        const int i = k * QT;
        if (i > 0 && (i & 63) == 0) {
            now = after;
            after = load(i / 64 + 1, lane);
        }
        Tile t;
#pragma unroll
        for (int n = 0; n < QT; ++n) t.p[n] = __builtin_amdgcn_readlane(now, (i & 63) + n);
        return t;
    }
};

// All loads of the wave, in a form that the compiler takes into account
__device__ inline void wait_loads() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0F70);              // vmcnt(0)
    asm volatile("" ::: "memory");                   // (no read of LDS moves before it)
    __builtin_amdgcn_sched_barrier(0);
}
// load(ahead) and then work(tile), which touch different memory: the compiler would wait for the loads into LDS before work's
// first read there (trees of 64 over 30000 to 100000 tokens: 517 us with that wait, 482 without)
template <class Load, class Work>
__device__ inline __attribute__((always_inline)) void beside(char* __restrict ahead, char* __restrict tile, const Load& load, const Work& work) {
    load(ahead);
    work(tile);
}

// A barrier behind which the waves' LDS writes, and the loads that they have waited for, are there for all
// (__syncthreads() would wait for every load that is on its way)
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The wave's rows of the tile at t0 on their way into LDS; returns a bit for each 16 tokens: their page is in the cache
template <typename Cf>
__device__ inline __attribute__((always_inline)) uint32_t issue_tile(const LatentAttentionArgs& a, const Seq& s, const typename Pages<Cf::QT>::Tile& pg,
                                                                     int t0, char* to, int wave, int lane) {
    constexpr int QT = Cf::QT, TILE = Cf::TILE;
    const uint32_t voff = (lane >> 3) * Cf::RB + (((lane & 7) ^ (lane >> 3)) * 16);
    const uint32_t voff_tail = ((lane >> 2) & 7) * Cf::RB + (((lane & 3) ^ ((lane >> 3) & 3)) * 16);
    const int sh = a.cache.page_shift;
    uint32_t ok = 0;
#pragma unroll
    for (int n = 0; n < QT; ++n) ok |= (uint32_t)(pg.p[n] >= 0 && pg.p[n] < a.cache.n_pages) << n;
#pragma unroll
    for (int e = 0; e < Cf::OCTETS; ++e) {
        // eight rows; tokens without a page read page 0
        const int o = wave * Cf::OCTETS + e;
        int pid = pg.p[0];
#pragma unroll
        for (int n = 1; n < QT; ++n) pid = o >= 2 * n ? pg.p[n] : pid;
        const bool there = (ok >> (o / 2)) & 1;
        const char* base = a.cache.rows + (there ? ((int64_t)pid << sh) + ((t0 + 8 * o) & ((1 << sh) - 1)) : 0) * Cf::RB;
        const int last = s.len - 1 - (t0 + 8 * o);
        if (last >= 7) {
#pragma unroll
            for (int i = 0; i < Cf::PANELS; ++i) load_lds16(base + i * 128 + voff, to + (i * TILE + 8 * o) * 128);
            if constexpr (Cf::HAS_TAIL)
                if (lane < 32) load_lds16(base + Cf::PANELS * 128 + voff_tail, to + Cf::TAIL + 8 * o * 64);
        } else {
            // places past the end, which nothing may have been written to, take the last token's row: what all rows see
            // keeps nothing from any
            const int e16 = (s.len - 1 - t0) >> 4;
            int pe = pg.p[0];
#pragma unroll
            for (int n = 1; n < QT; ++n) pe = e16 == n ? pg.p[n] : pe;
            const char* row = a.cache.rows + (((ok >> e16) & 1) ? ((int64_t)pe << sh) + ((s.len - 1) & ((1 << sh) - 1)) : 0) * Cf::RB;
            const int r = lane >> 3, rt = (lane >> 2) & 7;
            const char* f = r <= last ? base + voff : row + (voff - r * Cf::RB);
            const char* ft = rt <= last ? base + voff_tail : row + (voff_tail - rt * Cf::RB);
#pragma unroll
            for (int i = 0; i < Cf::PANELS; ++i) load_lds16(f + i * 128, to + (i * TILE + 8 * o) * 128);
            if constexpr (Cf::HAS_TAIL)
                if (lane < 32) load_lds16(ft + Cf::PANELS * 128, to + Cf::TAIL + 8 * o * 64);
        }
    }
    return ok;
}

// Eight rows of a tile, by the wave that has loaded them: 16 bytes of the latent part that hold an infinity or a NaN become
// zeros (a weight of 0 would not keep them out of the sums of the tokens that do not see the row), and the row's rotary part
// a NaN: its scores are no numbers, whatever else it holds, for the tokens that do.
template <bool BF, typename Cf>
__device__ inline void clean_rows(char* tile, int o, int lane) {
    constexpr int LATENT = Cf::R * Cf::ES / 128;
    bool bad = false;
#pragma unroll 4
    for (int p = 0; p < LATENT; ++p) {
        u32x4* at = (u32x4*)(tile + (p * Cf::TILE + 8 * o) * 128 + lane * 16);
        const u32x4 x = *at;
        bool no = false;
#pragma unroll
        for (int w = 0; w < 4; ++w) no |= (BF && (x[w] & 0x7F80u) == 0x7F80u) || (x[w] & 0x7F800000u) == 0x7F800000u;
        if (no) *at = u32x4{0u, 0u, 0u, 0u};
        bad |= no;
    }
    const uint64_t rows = __builtin_amdgcn_ballot_w64(bad);
    if ((lane & 7) == 0 && ((rows >> lane) & 0xFF)) {
        const uint32_t nan = BF ? 0x7FC07FC0u : 0x7FC00000u;
        char* at = Cf::PANELS > LATENT ? tile + (LATENT * Cf::TILE + 8 * o) * 128 + lane * 16 : tile + Cf::TAIL + (8 * o + (lane >> 3)) * 64;
        *(u32x4*)at = u32x4{nan, nan, nan, nan};
    }
}

// Rows of a tile that hold what is no number and that some token may not see are cleaned by the wave that has loaded them.
// careful: not a token alone that sees itself, which sees all that is there
template <bool BF, typename Cf>
__device__ inline void clean_tile(const Seq& s, char* tile, int t0, int t_hi, uint32_t ok, bool careful, int wave, int lane) {
    const int blocks = t_hi - t0 < Cf::TILE ? (t_hi - t0 + 15) / 16 : Cf::QT;
    if ((careful && t0 + Cf::TILE > s.ctx) || (~ok & ((1u << blocks) - 1u)))
#pragma unroll
        for (int e = 0; e < Cf::OCTETS; ++e) clean_rows<BF, Cf>(tile, wave * Cf::OCTETS + e, lane);
}

// whether a row with this word sees position p, whose page is there.  (No branches: with && and || in one of these loops the
// compiler lost the score of one of the four places.)
__device__ inline bool sees(const Seq& s, bool there, uint64_t word, int p) {
    const int d = p - s.ctx;
    return ((uint32_t)there & (uint32_t)(p < s.len) & ((uint32_t)(d < 0) | (uint32_t)(word >> (d & 63)))) & 1u;
}

// FINE: the second product takes what the rounding of the weights to bf16 leaves out as well
template <bool BF, int R, int ROT, int MT, bool FINE, bool WEIGHS>
__global__ void __launch_bounds__((64 * Config<BF, R, ROT, MT>::NW), (BF ? 2 : 1))
latent_attention_kernel(const LatentAttentionArgs a, int items, int rb_n) {
    using Cf = Config<BF, R, ROT, MT>;
    constexpr int NW = Cf::NW, TILE = Cf::TILE, QT = Cf::QT, CT = Cf::CT, KS = Cf::KS, PANEL = TILE * 128;
    constexpr int ROWS = 16 * MT, SUMS = ROWS * Cf::LD * 4, MEM = 2 * Cf::STAGE > SUMS ? 2 * Cf::STAGE : SUMS;
    __shared__ __attribute__((aligned(16))) char s_mem[MEM];
    __shared__ __attribute__((aligned(16))) char s_p[FINE ? 2 : 1][ROWS * Cf::PP];
    __shared__ float s_top[QT][ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    // the row blocks of one piece on one XCD, where its rows are in L2
    const int idx = (int)block_number(), jx = idx >> 3;
    const int item = (jx / rb_n) * 8 + (idx & 7), rb = jx % rb_n;
    if (item >= items) return;
    Seq mine = {0, 0, 0, 0};
    if (lane < a.B) mine = sequence(a, lane);
    const int piece = __builtin_amdgcn_readfirstlane(piece_tokens(a, rb_n, MT, TILE, mine, lane));
    int b, j;
    const Seq s = find_item(a, piece, item, lane, idx == 0 && wave == 0, mine, b, j);
    if (b < 0) return;
    const int rows = s.n * a.n_q, row0 = rb * ROWS, rows_max = a.max_q * a.n_q;
    if (row0 >= rows) return;
    const int t_lo = j * piece, t_hi = s.len - t_lo < piece ? s.len : t_lo + piece;
    const float scale2 = a.scale * LOG2E, ninf = -__builtin_inff();      // scores in units of log 2
    const int sh = a.cache.page_shift;
    Pages<QT> pages;
    pages.start(a, b, t_lo, t_hi, lane);
    int p = t_lo, k_tile = 0;
    uint32_t ok = 0, next = 0;
    if (p < t_hi) ok = issue_tile<Cf>(a, s, pages.tile(0, lane), p, s_mem, wave, lane);
    // the wave's tokens and query rows of the first product
    const int tt = wave % QT, r0 = wave / QT;
    const bool scores = r0 < MT;
    u32x4 q[KS];
    {
        const int row = row0 + 16 * r0 + c;
        const bool in = scores && row < rows;        // rows past the end are zeros and see nothing
        const char* from = (const char*)a.q + ((int64_t)s.first * a.n_q + (in ? row : 0)) * Cf::RB + 16 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            q[k] = u32x4{0u, 0u, 0u, 0u};
            if (in) q[k] = *(const u32x4*)(from + 64 * k);
        }
    }
    const bool careful = s.n > 1 || (a.tree && !(a.tree[s.first] & 1));
    // Lane (c, g): the reference of row c of every row tile, in units of log 2; its own tokens' share of the sum of its
    // row tile; row c's elements 16 (CT wave + t) + 4 g + i of every row tile.  The reference is the maximum, taken
    // over only when some score passes it by LA_LAG (a factor of 256 in the weights, which fp32 sums and bf16 weights
    // hold as well as 1): most tiles need no rescaling.
    float m[MT], l = 0.f;
    f32x4 o[CT][MT] = {};
#pragma unroll
    for (int r = 0; r < MT; ++r) m[r] = ninf;
    for (int buf = 0; p < t_hi; p += TILE, buf ^= 1) {
        char* const staged = s_mem + buf * Cf::STAGE;
        wait_loads();
        clean_tile<BF, Cf>(s, staged, p, t_hi, ok, careful, wave, lane);
        lds_barrier();                               // the tile has arrived, the one before has been read
        auto load = [&](char* to) __attribute__((always_inline)) {
            if (p + TILE < t_hi) next = issue_tile<Cf>(a, s, pages.tile(++k_tile, lane), p + TILE, to, wave, lane);
        };
        auto work = [&](char* tile) __attribute__((always_inline)) {
        f32x4 sc = {};
        if (scores) {
            LongSum<BF> dot;
            constexpr int RING = 6;    // steps whose reads are in registers or on their way
            const char* at[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) at[k] = tile + (16 * tt + c) * 128 + (((4 * k + g) ^ (c & 7)) * 16);
            const char* tail = tile + Cf::TAIL + (16 * tt + c) * 64 + ((g ^ ((c >> 1) & 3)) * 16);
            u32x4 x[RING];
            auto read = [&](int k) __attribute__((always_inline)) {
                x[k % RING] = *(const u32x4*)(k / 2 < Cf::PANELS ? at[k % 2] + k / 2 * PANEL : tail);
            };
#pragma unroll
            for (int k = 0; k < RING - 1; ++k) read(k);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                if (k + RING - 1 < KS) read(k + RING - 1);
                dot.add(x[k % RING], q[k]);
                __builtin_amdgcn_sched_barrier(0);
            }
            sc = dot.sum();
            const int t0 = p + 16 * tt;              // the wave's tokens
            const bool there = (ok >> tt) & 1, edge = t0 + 16 > s.ctx || !there;
            sc = sc * scale2;
            const int row = row0 + 16 * r0 + c;
            if (edge) {
                const int i_tok = row / a.n_q;
                const uint64_t word = row >= rows ? 0ull : a.tree ? a.tree[s.first + i_tok] : ~0ull >> (63 - i_tok);
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[i] = sees(s, there, word, t0 + 4 * g + i) ? sc[i] : ninf;
            }
            if constexpr (WEIGHS)
                if (row < rows && t0 < s.len)        // (a table holds whole 16s)
                    *(f32x4*)(a.score + ((int64_t)b * rows_max + row) * ((int64_t)a.max_pages << sh) + t0 + 4 * g) = sc;
            float top = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3]));
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (g == 0) s_top[tt][16 * r0 + c] = top;
        }
        lds_barrier();
        // the same in all waves
        float al[MT];
        bool change = false;
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            float top = s_top[0][16 * r + c];
#pragma unroll
            for (int k = 1; k < QT; ++k) top = fmaxf(top, s_top[k][16 * r + c]);
            const float was = m[r];
            m[r] = top > was + LA_LAG ? top : was;
            al[r] = was == m[r] ? 1.0f : __builtin_amdgcn_exp2f(was - m[r]);
            change |= was != m[r] && was != ninf;    // (nothing to rescale before the first weights)
        }
        if (scores) {
            float mr = m[0], ar = al[0];             // of the wave's row tile
            if (MT > 1 && r0 > 0) { mr = m[MT - 1]; ar = al[MT - 1]; }
            mr = mr == ninf ? 0.f : mr;              // (weights of 0 where nothing has been seen yet)
            l *= ar;
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = __builtin_amdgcn_exp2f(sc[i] - mr);
                l += w[i];
            }
            char* to = &s_p[0][(16 * r0 + c) * Cf::PP + (16 * tt + 4 * g) * Cf::ES];
            if constexpr (BF) {
                *(u32x2*)to = u32x2{bf16_pair(w[0], w[1]), bf16_pair(w[2], w[3])};
                if constexpr (FINE) {
                    float d[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[i] = w[i] - (float)(__bf16)w[i];
                    *(u32x2*)(to + ROWS * Cf::PP) = u32x2{bf16_pair(d[0], d[1]), bf16_pair(d[2], d[3])};
                }
            } else {
                *(f32x4*)to = f32x4{w[0], w[1], w[2], w[3]};
            }
        }
        if (__builtin_amdgcn_ballot_w64(change)) {
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int t = 0; t < CT; ++t) o[t][r] = o[t][r] * al[r];
        }
        lds_barrier();
        if constexpr (BF) {
            // inner indexes 8 g .. 8 g + 7 of each 32 tokens
            constexpr int STEPS = TILE / 32 * CT, RING = 4;
            const int row = 8 * g + (c >> 2);
            const int e0 = (2 * CT * wave) & 7;      // the wave's first chunk of a panel
            const char* base = tile + (2 * CT * wave) / 8 * PANEL + row * 128 + (c & 1) * 8;
            const int half = (c >> 1) & 1;
            u32x2 v[RING][2];
            auto read = [&](int i) __attribute__((always_inline)) {
                const int s2 = i / CT, t = i % CT;
                const int ch = e0 + 2 * t;           // (a wave's elements end within a panel, or are whole panels)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    v[i % RING][u] = read_turned(base + (ch >> 3) * PANEL + (32 * s2 + 4 * u) * 128 +
                                                 ((((ch & 7) + half) ^ ((row + 4 * u) & 7)) * 16));
            };
            u32x4 pf[MT], pl[MT];
#pragma unroll
            for (int i = 0; i < RING - 1; ++i) read(i);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (i % CT == 0) {
#pragma unroll
                    for (int r = 0; r < MT; ++r) {
                        const char* at = &s_p[0][(16 * r + c) * Cf::PP + i / CT * 64 + 16 * g];
                        pf[r] = *(const u32x4*)at;
                        if constexpr (FINE) pl[r] = *(const u32x4*)(at + ROWS * Cf::PP);
                    }
                }
                if (i + RING - 1 < STEPS) read(i + RING - 1);
                const u32x2* x = v[i % RING];
                const u32x4 vf = {x[0][0], x[0][1], x[1][0], x[1][1]};
#pragma unroll
                for (int r = 0; r < MT; ++r) o[i % CT][r] = mma16<true>(vf, pf[r], o[i % CT][r]);
                if constexpr (FINE)
#pragma unroll
                    for (int r = 0; r < MT; ++r) o[i % CT][r] = mma16<true>(vf, pl[r], o[i % CT][r]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int n = 0; n < QT; ++n) {
                f32x4 pf[MT];
#pragma unroll
                for (int r = 0; r < MT; ++r) pf[r] = *(const f32x4*)&s_p[0][(16 * r + c) * Cf::PP + (16 * n + 4 * g) * 4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * n + 4 * g + i;
#pragma unroll
                    for (int t = 0; t < CT; ++t) {
                        const int ch = 4 * (CT * wave + t) + (c >> 2);       // (of 16 bytes)
                        const float v = *(const float*)(tile + (ch >> 3) * PANEL + row * 128 + (((ch & 7) ^ (row & 7)) * 16) + (c & 3) * 4);
#pragma unroll
                        for (int r = 0; r < MT; ++r) o[t][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, pf[r][i], o[t][r], 0, 0, 0);
                    }
                }
            }
        }
        };
        beside(s_mem + (buf ^ 1) * Cf::STAGE, staged, load, work);
        ok = next;
    }
    // the sums in rows
    __syncthreads();                                 // the staged rows become their place
    int tid2 = tid;
    asm volatile("" : "+v"(tid2));                   // (what follows needs no registers before)
    const int c2 = tid2 & 15, g2 = (tid2 & 63) >> 4;
    float(*const s_o)[Cf::LD] = (float(*)[Cf::LD])s_mem;
#pragma unroll
    for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int t = 0; t < CT; ++t) *(f32x4*)&s_o[16 * r + c2][16 * (CT * wave + t) + 4 * g2] = o[t][r];
    if (scores) {
        float x = l;
        x += __shfl_xor(x, 16);
        x += __shfl_xor(x, 32);
        if (g2 == 0) s_top[tt][16 * r0 + c2] = x;
    }
    __syncthreads();
    const int64_t at = (int64_t)item * rows_max + row0;
    const int here = rows - row0 < ROWS ? rows - row0 : ROWS;
    for (int u = tid2; u < here * (R / 4); u += 64 * NW) {
        const int r = u / (R / 4), e = u % (R / 4) * 4;
        *(f32x4*)(a.part_o + (at + r) * R + e) = *(const f32x4*)&s_o[r][e];
    }
    if (wave == 0 && g2 == 0) {
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            if (16 * r + c2 >= here) continue;
            float x = s_top[0][16 * r + c2];
#pragma unroll
            for (int k = 1; k < QT; ++k) x += s_top[k][16 * r + c2];
            ((f32x2*)a.part_ml)[at + 16 * r + c2] = f32x2{m[r], x};
        }
    }
}

// Sequences of many query rows: blocks of 128.  The weights are rounded to bf16: over many positions their errors mostly
// cancel (trees of 64 over 30000-100000 tokens: 0.0017 of the outputs, as by the outputs' own rounding alone), and two parts
// would double the second product of a kernel that the matrix unit and LDS bound.
template <int R, int ROT, bool WEIGHS>
__global__ void __launch_bounds__(512, 2) latent_rows_kernel(const LatentAttentionArgs a, int items, int rb_n) {
    using Cf = Config<true, R, ROT, 8>;
    constexpr int TILE = Cf::TILE, QT = Cf::QT, KS = Cf::KS, PANEL = TILE * 128, ET = R / 16;    // elements' tiles
    static_assert(Cf::NW == 8 && Cf::OCTETS == 1 && TILE == 64, "a wave an eight of a tile's rows");
    __shared__ __attribute__((aligned(16))) char s_mem[2 * Cf::STAGE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int idx = (int)block_number(), jx = idx >> 3;
    const int item = (jx / rb_n) * 8 + (idx & 7), rb = jx % rb_n;
    if (item >= items) return;
    Seq mine = {0, 0, 0, 0};
    if (lane < a.B) mine = sequence(a, lane);
    const int piece = __builtin_amdgcn_readfirstlane(piece_tokens(a, rb_n, 8, TILE, mine, lane));
    int b, j;
    const Seq s = find_item(a, piece, item, lane, idx == 0 && wave == 0, mine, b, j);
    if (b < 0) return;
    const int rows = s.n * a.n_q, row0 = rb * 128, rows_max = a.max_q * a.n_q;
    if (row0 >= rows) return;
    const int t_lo = j * piece, t_hi = s.len - t_lo < piece ? s.len : t_lo + piece;
    const float scale2 = a.scale * LOG2E, ninf = -__builtin_inff();      // scores in units of log 2
    const int sh = a.cache.page_shift;
    Pages<QT> pages;
    pages.start(a, b, t_lo, t_hi, lane);
    int p = t_lo, k_tile = 0;
    uint32_t ok = 0, next = 0;
    if (p < t_hi) ok = issue_tile<Cf>(a, s, pages.tile(0, lane), p, s_mem, wave, lane);
    const int wrow = row0 + 16 * wave;
    u32x4 q[KS];
    {
        const bool in = wrow + c < rows;             // rows past the end are zeros and see nothing
        const char* from = (const char*)a.q + ((int64_t)s.first * a.n_q + (in ? wrow + c : 0)) * Cf::RB + 16 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            q[k] = u32x4{0u, 0u, 0u, 0u};
            if (in) q[k] = *(const u32x4*)(from + 64 * k);
        }
    }
    // Lane (c, g): row c's maximum (a reference that may lag, as above) and its own tokens' share of the sum; row c's elements
    // 16 j + 4 g + i
    float m = ninf, l = 0.f;
    f32x4 o[ET];
#pragma unroll
    for (int e = 0; e < ET; ++e) o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int buf = 0; p < t_hi; p += TILE, buf ^= 1) {
        char* const staged = s_mem + buf * Cf::STAGE;
        wait_loads();
        clean_tile<true, Cf>(s, staged, p, t_hi, ok, true, wave, lane);
        lds_barrier();                               // the tile has arrived, the one before has been read
        auto load = [&](char* to) __attribute__((always_inline)) {
            if (p + TILE < t_hi) next = issue_tile<Cf>(a, s, pages.tile(++k_tile, lane), p + TILE, to, wave, lane);
        };
        auto work = [&](char* tile) __attribute__((always_inline)) {
#pragma unroll 1
        for (int n0 = 0; n0 < 2; ++n0) {             // 32 tokens at a time
            const int t0 = p + 32 * n0;
            if (t0 >= t_hi) break;
            f32x4 sc[2] = {};
            {
                constexpr int RING = 3;              // steps whose reads are in registers or on their way
                const char* at[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) at[k] = tile + (32 * n0 + c) * 128 + (((4 * k + g) ^ (c & 7)) * 16);
                const char* tail = tile + Cf::TAIL + (32 * n0 + c) * 64 + ((g ^ ((c >> 1) & 3)) * 16);
                u32x4 x[RING][2];
                auto read = [&](int k) __attribute__((always_inline)) {
#pragma unroll
                    for (int n = 0; n < 2; ++n)
                        x[k % RING][n] = *(const u32x4*)(k / 2 < Cf::PANELS ? at[k % 2] + k / 2 * PANEL + 16 * n * 128 : tail + 16 * n * 64);
                };
#pragma unroll
                for (int k = 0; k < RING - 1; ++k) read(k);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    if (k + RING - 1 < KS) read(k + RING - 1);
#pragma unroll
                    for (int n = 0; n < 2; ++n) sc[n] = mma16<true>(x[k % RING][n], q[k], sc[n]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            const uint32_t there = (ok >> (2 * n0)) & 3u;
#pragma unroll
            for (int n = 0; n < 2; ++n) sc[n] = sc[n] * scale2;
            if (WEIGHS || t0 + 32 > s.ctx || there != 3u) {
                // (the row's number is made again here, not held in registers)
                int lane2 = lane;
                asm volatile("" : "+v"(lane2));
                const int row = wrow + (lane2 & 15), g2 = lane2 >> 4;
                if (t0 + 32 > s.ctx || there != 3u) {
                    const int i_tok = row / a.n_q;
                    const uint64_t word = row >= rows ? 0ull : a.tree ? a.tree[s.first + i_tok] : ~0ull >> (63 - i_tok);
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sc[n][i] = sees(s, (there >> n) & 1u, word, t0 + 16 * n + 4 * g2 + i) ? sc[n][i] : ninf;
                }
                if constexpr (WEIGHS) {
                    if (row < rows) {
                        float* to = a.score + ((int64_t)b * rows_max + row) * ((int64_t)a.max_pages << sh) + t0 + 4 * g2;
#pragma unroll
                        for (int n = 0; n < 2; ++n)
                            if (t0 + 16 * n < s.len) *(f32x4*)(to + 16 * n) = sc[n];     // (a table holds whole 16s)
                    }
                }
            }
            float top = ninf;
#pragma unroll
            for (int n = 0; n < 2; ++n) top = fmaxf(top, fmaxf(fmaxf(sc[n][0], sc[n][1]), fmaxf(sc[n][2], sc[n][3])));
            if (__builtin_amdgcn_ballot_w64(top > m + LA_LAG)) {
                float x = fmaxf(top, __shfl_xor(top, 16));
                x = fmaxf(x, __shfl_xor(x, 32));
                x = x > m + LA_LAG ? x : m;          // by the row alone, whatever the others do
                const float al = m == x ? 1.0f : __builtin_amdgcn_exp2f(m - x);
                m = x;
                l *= al;
#pragma unroll
                for (int e = 0; e < ET; ++e) o[e] = o[e] * al;
            }
            const float mr = m == ninf ? 0.f : m;    // (weights of 0 where nothing has been seen yet)
            u32x4 pf;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sc[n][i] = __builtin_amdgcn_exp2f(sc[n][i] - mr);
                    l += sc[n][i];
                }
                pf[2 * n] = bf16_pair(sc[n][0], sc[n][1]);
                pf[2 * n + 1] = bf16_pair(sc[n][2], sc[n][3]);
            }
            const int vrow = 4 * g + (c >> 2);
            const char* at[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) at[e] = tile + (32 * n0 + vrow) * 128 + (((2 * e + ((c >> 1) & 1)) ^ (vrow & 7)) * 16) + (c & 1) * 8;
            u32x2 v[2][2][2];
            auto read = [&](int i) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const int t = 2 * i + e;
                        v[i & 1][e][n] = read_turned(at[t % 4] + t / 4 * PANEL + 16 * n * 128);
                    }
            };
            read(0);
#pragma unroll
            for (int i = 0; i < ET / 2; ++i) {
                if (i + 1 < ET / 2) read(i + 1);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2* x = v[i & 1][e];
                    o[2 * i + e] = mma16<true>(u32x4{x[0][0], x[0][1], x[1][0], x[1][1]}, pf, o[2 * i + e]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        };
        beside(s_mem + (buf ^ 1) * Cf::STAGE, staged, load, work);
        ok = next;
    }
    // the sums through LDS, so that they are written in whole cache lines: two waves' rows at a time
    int tid2 = tid;
    asm volatile("" : "+v"(tid2));                   // (what follows needs no registers before)
    const int c2 = tid2 & 15, g2 = (tid2 & 63) >> 4;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const int64_t at = (int64_t)item * rows_max;
    if (g2 == 0 && wrow + c2 < rows) ((f32x2*)a.part_ml)[at + wrow + c2] = f32x2{m, l};
    constexpr int AT_ONCE = 2 * Cf::STAGE / (16 * Cf::LD * 4) >= 4 ? 4 : 2;
    float(*const s_o)[Cf::LD] = (float(*)[Cf::LD])s_mem;
#pragma unroll 1
    for (int w0 = 0; w0 < 8; w0 += AT_ONCE) {
        if (row0 + 16 * w0 >= rows) break;
        __syncthreads();
        if (wave / AT_ONCE * AT_ONCE == w0) {
#pragma unroll
            for (int e = 0; e < ET; ++e) *(f32x4*)&s_o[16 * (wave - w0) + c2][16 * e + 4 * g2] = o[e];
        }
        __syncthreads();
        const int left = rows - row0 - 16 * w0, here = left < 16 * AT_ONCE ? left : 16 * AT_ONCE;
        for (int u = tid2; u < here * (R / 4); u += 512) {
            const int r = u / (R / 4), e = u % (R / 4) * 4;
            *(f32x4*)(a.part_o + (at + row0 + 16 * w0 + r) * R + e) = *(const f32x4*)&s_o[r][e];
        }
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
    __shared__ __attribute__((aligned(16))) char s_o[BF ? 2 : 1][TOK * PITCH];
    __shared__ f32x4 s_acc[SHARE > 1 ? 4 : 1][2][64];
    __shared__ __attribute__((aligned(16))) float s_x[S > 1 ? 16 : 1][S > 1 ? R + 4 : 4];
    __shared__ float s_m[16], s_l[16];
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
    int first = 0, pieces = 0;
    if (in) {
        s = sequence(a, b);
        first = a.plan[2 * b];
        pieces = a.plan[2 * b + 1];
    }
    const int i = t - s.first;
    in = in && i >= 0 && i < s.n;
    pieces = in ? pieces : 0;
    const int row = i * a.n_q + h, rows_max = a.max_q * a.n_q;
    if (tid < 16) s_in[tid] = 0;
    const int64_t at = in ? (int64_t)first * rows_max + row : 0;
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
    // Four elements of a token's sums, relative to its maximum, divided and put into the operand's two parts
    auto put = [&](int to, int e, const f32x4& sum, float r) __attribute__((always_inline)) {
        const f32x4 y = sum * r;
        char* o = &s_o[0][to * PITCH + e * ES];
        if constexpr (BF) {
            float d[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) d[k] = y[k] - (float)(__bf16)y[k];
            *(u32x2*)o = u32x2{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
            *(u32x2*)&s_o[BF ? 1 : 0][to * PITCH + e * ES] = u32x2{bf16_pair(d[0], d[1]), bf16_pair(d[2], d[3])};
        } else {
            *(f32x4*)o = y;
        }
    };
    if constexpr (S > 1) {
        // the sets of a token through LDS, in order.  (By exchanges between the lanes that hold them 6500 cycles, of 13000 in
        // all for one token over 777.)
#pragma unroll
        for (int e = 0; e < R / 64; ++e) *(f32x4*)&s_x[tid >> 4][4 * u + 64 * e] = f32x4{x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]};
        if (u == 0) { s_m[tid >> 4] = m; s_l[tid >> 4] = l; }
        __syncthreads();
        auto whole = [&](int to, float (&f)[S]) __attribute__((always_inline)) {        // m, l and the sets' factors
            m = s_m[to * S];
#pragma unroll
            for (int k = 1; k < S; ++k) m = fmaxf(m, s_m[to * S + k]);
            l = 0.f;
#pragma unroll
            for (int k = 0; k < S; ++k) {
                f[k] = s_m[to * S + k] == m ? 1.0f : __builtin_amdgcn_exp2f(s_m[to * S + k] - m);
                l += s_l[to * S + k] * f[k];
            }
        };
        float f[S];
        for (int v = tid; v < TOK * (R / 4); v += 256) {
            const int to = v / (R / 4), e = v % (R / 4) * 4;
            whole(to, f);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < S; ++k) sum = sum + *(const f32x4*)&s_x[to * S + k][e] * f[k];
            put(to, e, sum, l == 0.f ? 0.f : 1.0f / l);
        }
        if (z == 0) whole(slot, f);
    } else {
        __syncthreads();                             // s_in is clear
        const float r = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
        for (int e = 0; e < R / 64; ++e) put(slot, 4 * u + 64 * e, f32x4{x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]}, r);
    }
    if (z == 0 && in && u == 0) {
        s_in[slot] = 1;
        if (d0 == 0) {
            if (a.lse) a.lse[(int64_t)t * a.n_q + h] = l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * LN2;
            if (a.mass_out) ((f32x2*)a.stat)[(int64_t)b * rows_max + row] = f32x2{m == -__builtin_inff() ? 0.f : m, l == 0.f ? 0.f : 1.0f / l};
        }
    }
    __syncthreads();
    LongSum<BF> sums[2];
    // (tokens past TOK: a row that is there, for columns that nobody reads)
    const char* o = &s_o[0][(c < TOK ? c : 0) * PITCH + (share * KS * 4 + g) * 16];
    const char* o_lo = &s_o[BF ? 1 : 0][(c < TOK ? c : 0) * PITCH + (share * KS * 4 + g) * 16];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        const u32x4 w0 = k < EARLY ? early[k < EARLY ? k : 0][0] : *(const u32x4*)(w + 64 * k);
        const u32x4 w1 = k < EARLY ? early[k < EARLY ? k : 0][1] : *(const u32x4*)(w + 16 * R * ES + 64 * k);
        const u32x4 hi = *(const u32x4*)(o + 64 * k);
        sums[0].add(w0, hi);
        sums[1].add(w1, hi);
        if constexpr (BF) {
            const u32x4 lo = *(const u32x4*)(o_lo + 64 * k);
            sums[0].add(w0, lo);
            sums[1].add(w1, lo);
        }
    }
    f32x4 acc[2] = {sums[0].sum(), sums[1].sum()};
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

template <bool BF, int R, int ROT, int MT, bool FINE>
int launch_rows(const LatentAttentionArgs& a, hipStream_t st) {
    const int rb = row_blocks(a.max_q * a.n_q, MT);
    const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
    {
        const int64_t items = a.items;
        const dim3 grid = grid_of((items + 7) / 8 * 8 * rb), block((64 * Config<BF, R, ROT, MT>::NW));
        KernelTimer kt_("latent_attention", st);
        if constexpr (MT == 8) {
            if (a.mass_out) latent_rows_kernel<R, ROT, true><<<grid, block, 0, st>>>(a, (int)items, rb);
            else latent_rows_kernel<R, ROT, false><<<grid, block, 0, st>>>(a, (int)items, rb);
        } else {
            if (a.mass_out) latent_attention_kernel<BF, R, ROT, MT, FINE, true><<<grid, block, 0, st>>>(a, (int)items, rb);
            else latent_attention_kernel<BF, R, ROT, MT, FINE, false><<<grid, block, 0, st>>>(a, (int)items, rb);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    // About how many pieces a sequence has where they are of like length.  (One long sequence among many short ones has more,
    // up to 2 LA_TARGET / rb, and fewer sets to add them than it could use.)
    const bool many = std::min<int64_t>((cap + LA_MIN_PIECE - 1) / LA_MIN_PIECE, LA_TARGET / ((int64_t)a.B * rb) + 1) > LO_PIECES;
    {
        KernelTimer kt_("latent_out", st);
        // As few sets a row as give every CU a workgroup, and all 16 for many pieces (two sequences of 8000, 128 heads: 47 us
        // with 4 sets, 21 with 16); few rows: slices of the head's elements too
        auto go = [&](auto d, auto ds, auto sets) {
            constexpr int D = decltype(d)::value, DS = decltype(ds)::value, S = decltype(sets)::value, TOK = 16 / S;
            latent_out_kernel<BF, R, D, DS, S><<<grid_of((a.T + TOK - 1) / TOK * a.n_q * (D / DS)), dim3(256), 0, st>>>(a, D / DS);
        };
        auto of = [&](auto d) {
            using N1 = std::integral_constant<int, 1>;
            using N4 = std::integral_constant<int, 4>;
            using N16 = std::integral_constant<int, 16>;
            using N32 = std::integral_constant<int, 32>;
            const int64_t one = (a.T + 15) / 16 * a.n_q, four = (a.T + 3) / 4 * a.n_q;
            if (many) a.T * a.n_q >= LO_GROUPS ? go(d, d, N16{}) : go(d, N32{}, N16{});
            else if (one >= LO_GROUPS) go(d, d, N1{});
            else if (four >= LO_GROUPS) go(d, d, N4{});
            else if (four * (decltype(d)::value / 32) >= LO_GROUPS) go(d, N32{}, N4{});
            else go(d, N32{}, N16{});
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
    static_assert(ORDERMOE_LATENT_FINE_ROWS == LA_FEW, "the batches whose weights keep 16 bits");
    const int mt = row_tiles(a.cache.dtype, a.max_q * a.n_q);
    if constexpr (BF)
        if (mt == 8) return launch_rows<BF, R, ROT, 8, false>(a, st);
    return mt == 2 ? launch_rows<BF, R, ROT, 2, BF>(a, st) : launch_rows<BF, R, ROT, 1, BF>(a, st);
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

int64_t latent_items(int dtype, int n_q, int B, int max_q, int64_t cap) {
    const int rows = max_q * n_q, rb = row_blocks(rows, row_tiles(dtype, rows));
    constexpr int LEAST = LA_MIN_PIECE / 2;
    return std::min<int64_t>((2 * LA_TARGET + rb - 1) / rb + B, B * ((cap + LEAST - 1) / LEAST));
}

int launch_latent_attention(const LatentAttentionArgs& a, void* stream) {
    if (a.B == 0 || a.T == 0) return 0;
    return a.cache.dtype == ORDERMOE_BF16 ? launch_rank<true>(a, (hipStream_t)stream) : launch_rank<false>(a, (hipStream_t)stream);
}

}  // namespace ordermoe
