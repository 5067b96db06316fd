// Causal attention of prompts over keys and values in rows.
//
//   prompt_attention_kernel  one workgroup per (128 query rows of a sequence, key/value
//                            head): its four waves take 32 rows each and go through the
//                            positions together, a tile at a time
//   prompt_join_kernel       few rows: their positions are split over workgroups, and this
//                            adds up the pieces in order
// The query rows of a key/value head are its n_b tokens times the n_q / n_kv query heads
// that share it (row = token * (n_q / n_kv) + head).
//
// A tile (v_mfma_f32_32x32x16_bf16, c = lane % 32, h = lane / 32; fp32 the same with
// v_mfma_f32_32x32x2_f32):
//   S^T = K Q^T   rows: 32 positions, columns: 32 query rows.  Maximum and sum belong to a
//                 column, that is to two lanes.
//   O^T = V^T P^T rows: 32 elements of the head, columns: the query rows.  S^T leaves lane (c, h)
//                 the weights of query row c for positions 8 j + 4 h .. + 3, j = 0 .. 3: in pairs of
//                 j the 8 inner indexes of its P^T operand, when V^T's lanes hold the same positions,
//                 which a turned read of V's rows in LDS gives them.  So the weights never leave their
//                 registers.
// K, the shared rotary part and V go straight from memory into LDS, keys two tiles ahead, values one: a tile's weights are
// made beside the scores of the next.  Two waves a SIMD share the matrix unit and the vector instructions of the softmax,
// which are busy 51% and 43% of the time: 12001 tokens x 32 heads of 128 + 64 1390 to 1510 us on different cards (970 to 1060
// TFLOP/s of the part that is seen), 8 prompts of up to 4000 tokens, 32 heads over 8 of 128, 474 to 536.  A comparison and a
// selection more per weight cost 7%.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "grid.hpp"
#include "mfma.hpp"

namespace ordermoe {
namespace {

constexpr int PA_WAVES = 4, PA_ROWS = 32 * PA_WAVES;     // query rows of a workgroup
template <bool BF>
constexpr int PA_TILE = BF ? 64 : 32;                    // positions of a tile
// A maximum is taken over only when some score passes it by 8 (a factor of 256 in the weights, which fp32 sums
// and bf16 weights hold as well as 1): most tiles then need no exchange between lanes and no rescaling.
constexpr float PA_LAG = 8.0f;

// Blocks of rows that leave the card empty: their positions are split into pieces, so many that the workgroups fill it, of
// PA_LEAST tiles or more of the longest sequence there can be.  (16 tokens behind 8000, 8 key heads: 152 us whole, 27 in
// pieces of 8 tiles or more, 28 of 4, 33 of 16; 300 tokens of 16 heads: 18 whole or of 8, 20 of 4.)
constexpr int PA_FEW = 128, PA_FILL = 512, PA_LEAST = 8;

__host__ __device__ inline int64_t row_blocks(int64_t rows) { return (rows + PA_ROWS - 1) / PA_ROWS; }

struct Seq {
    int q0, n, k0, len;      // first token, tokens, first position, positions
};
__device__ inline Seq sequence(const PromptArgs& a, int b) {
    const int T = (int)a.T, L = (int)a.L;
    int q0 = a.q_start[b], q1 = a.q_start[b + 1], k0 = a.kv_start[b], k1 = a.kv_start[b + 1];
    q0 = q0 < 0 ? 0 : q0 > T ? T : q0;
    q1 = q1 < q0 ? q0 : q1 > T ? T : q1;
    k0 = k0 < 0 ? 0 : k0 > L ? L : k0;
    k1 = k1 < k0 ? k0 : k1 > L ? L : k1;
    return Seq{q0, q1 - q0, k0, k1 - k0};
}

// sequence and row block of an item, by one wave; false: there are not so many.  A sequence's last row blocks,
// which see the most, come first.
__device__ inline bool find_block(const PromptArgs& a, int64_t item, int lane, Seq& s, int& rb) {
    const int G = a.n_q / a.n_kv;
    int64_t base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        Seq m = {0, 0, 0, 0};
        if (b0 + lane < a.B) m = sequence(a, b0 + lane);
        const int cnt = (int)row_blocks((int64_t)m.n * G);
        int inc = cnt;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            if (o >= a.B) continue;
            const int v = __shfl_up(inc, o);
            if (lane >= o) inc += v;
        }
        const int64_t first = base + inc - cnt;
        const uint64_t hit = __builtin_amdgcn_ballot_w64(item >= first && item < first + cnt);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            s = Seq{__builtin_amdgcn_readlane(m.q0, l), __builtin_amdgcn_readlane(m.n, l), __builtin_amdgcn_readlane(m.k0, l),
                    __builtin_amdgcn_readlane(m.len, l)};
            rb = __builtin_amdgcn_readlane((int)(first + cnt - 1 - item), l);
            return true;
        }
        base += __builtin_amdgcn_readlane(inc, 63);
    }
    return false;
}

// Rows of RB bytes in LDS, as 16-byte chunks: chunk c of row r lies at c ^ swap(r), so that what the lanes of a read
// take together lies on distinct banks: lanes 0 - 3, 12 - 15, 20 - 27 and the others of each 32, 256 bytes.  K and the rotary
// part: one chunk of 16 rows; V: four rows of two chunks (bf16, turned) or two rows, four apart, of eight (fp32).
template <int RB>
__device__ inline int swap_k(int r) {
    return RB >= 256 ? r & 15 : RB == 128 ? (r >> 1) & 7 : (r >> 2) & 3;
}
template <bool BF, int RB>
__device__ inline int swap_v(int r) {
    if constexpr (BF) return RB >= 256 ? (r & 3) << 2 : (r & 3) << 1;
    else return ((r >> 2) & 1) << 3;
}

template <bool BF, int D, int ROT>
struct Layout {
    static constexpr int ES = BF ? 2 : 4, TILE = PA_TILE<BF>, RBD = D * ES, RBR = ROT * ES;
    static constexpr int R = TILE * RBD, KEYS = R + TILE * RBR, VALUES = TILE * RBD;      // a tile's keys, rotary part behind them
    static constexpr int V = 2 * KEYS, BYTES = V + 2 * VALUES;                           // two tiles' keys, two tiles' values
    static constexpr int QN = (D + ROT) * ES / 32;       // 16-byte pieces of a query that a lane holds
};

// TILE rows of RB bytes, `stride` bytes apart in memory, into LDS by pieces of 1024 bytes, N of them a wave; where a lane's
// 16 bytes of a piece lie is kept.  Rows behind the last of `left` take the last one's.
template <bool BF, int RB, int KIND>
__device__ inline uint32_t lane_place(int row, int lane, uint32_t stride, int last) {
    constexpr int CH = RB / 16;
    const int swap = KIND == 0 ? swap_k<RB>(row) : swap_v<BF, RB>(row);
    return std::min(row, last) * stride + ((lane % CH) ^ swap) * 16;
}
template <bool BF, int RB, int KIND, int N>
__device__ inline void lane_places(uint32_t (&o)[N], uint32_t stride, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        o[i] = lane_place<BF, RB, KIND>((wave * N + i) * (1024 / RB) + lane / (RB / 16), lane, stride, 0x7FFF);
}
template <bool BF, int RB, int KIND, int N>
__device__ inline __attribute__((always_inline)) void issue_rows(const uint32_t (&o)[N], const char* from, int left, uint32_t stride, char* to,
                                                                 int wave, int lane) {
    if (left >= N * PA_WAVES * 1024 / RB) {
#pragma unroll
        for (int i = 0; i < N; ++i) load_lds16(from + o[i], to + (wave * N + i) * 1024);
    } else {
#pragma unroll 1
        for (int i = 0; i < N; ++i)
            load_lds16(from + lane_place<BF, RB, KIND>((wave * N + i) * (1024 / RB) + lane / (RB / 16), lane, stride, left - 1),
                       to + (wave * N + i) * 1024);
    }
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

// The largest exponents of 16 bytes, taken up in `top`
template <bool BF>
__device__ inline void exponents(const u32x4& x, u32x4& top) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if constexpr (BF) {
            const uint32_t now = x[w] & 0x7F807F80u, was = top[w];      // (a cast of a vector's element would take its first)
            top[w] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, now), __builtin_bit_cast(u16x2, was)));
        } else {
            top[w] = std::max<uint32_t>(x[w] & 0x7F800000u, top[w]);
        }
    }
}
template <bool BF>
__device__ inline bool no_number(const u32x4& top) {
    bool r = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) r |= (top[w] >= 0x7F800000u) | (BF && (top[w] & 0xFFFFu) >= 0x7F80u);
    return r;
}
// the elements of 16 bytes that are no numbers, as they are (NUMBERS: those that are), the others as zeros
template <bool BF, bool NUMBERS>
__device__ inline uint32_t parted(uint32_t x) {
    if constexpr (BF) {
        const bool lo = (x & 0x7F80u) == 0x7F80u, hi = (x & 0x7F800000u) == 0x7F800000u;
        return (lo == NUMBERS ? 0u : x & 0xFFFFu) | (hi == NUMBERS ? 0u : x & 0xFFFF0000u);
    } else {
        return ((x & 0x7F800000u) == 0x7F800000u) == NUMBERS ? 0u : x;
    }
}
// Infinities and NaNs of a tile's values become zeros: a weight of 0 would not keep what is no number out of a row's sums.
// A lane's row that sees such a value (positions of the tile up to `see`) gets it added to the sums of its own element here.
// Every wave looks through the whole tile, so that they meet the barriers together.
template <bool BF, int D>
__device__ inline __attribute__((always_inline)) void clean_values(char* v, int see, int wave, int lane, f32x16 (&o)[D / 32]) {
    constexpr int RB = D * (BF ? 2 : 4), CH = RB / 16, PIECES = PA_TILE<BF> * CH / 64;
    u32x4 top = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < PIECES; ++i) exponents<BF>(*(const u32x4*)(v + (i * 64 + lane) * 16), top);
    if (!__builtin_amdgcn_ballot_w64(no_number<BF>(top))) return;       // (alike in all waves)
    const int h = lane >> 5;
    uint64_t m = 0;                                      // positions
#pragma unroll 1
    for (int i = 0; i < PIECES; ++i) {
        u32x4 t = {0u, 0u, 0u, 0u};
        exponents<BF>(*(const u32x4*)(v + (i * 64 + lane) * 16), t);
        if (no_number<BF>(t)) m |= 1ull << ((i * 64 + lane) / CH);
    }
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) m |= __shfl_xor((unsigned long long)m, x);
    uint64_t left = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)m) |
                    (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(m >> 32)) << 32;
    for (; left; left &= left - 1) {
        const int p = __builtin_ctzll(left);
        const char* row = v + p * RB;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // elements 32 d + 8 j + 4 h .. + 3
                const int ch = (BF ? 4 * d + j : 8 * d + 2 * j + h) ^ swap_v<BF, RB>(p);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x;
                    if constexpr (BF) {
                        const uint32_t w = parted<BF, false>(*(const uint32_t*)(row + ch * 16 + 8 * h + 4 * (e / 2)));
                        x = __uint_as_float(e % 2 ? w & 0xFFFF0000u : w << 16);
                    } else {
                        x = __uint_as_float(parted<BF, false>(*(const uint32_t*)(row + ch * 16 + 4 * e)));
                    }
                    if (p <= see) o[d][4 * j + e] += x;
                }
                __builtin_amdgcn_sched_barrier(0);       // (few registers: most tiles hold numbers alone)
            }
    }
    __syncthreads();
    for (int i = wave; i < PIECES; i += PA_WAVES) {
        u32x4* at = (u32x4*)(v + (i * 64 + lane) * 16);
        u32x4 x = *at;
#pragma unroll
        for (int w = 0; w < 4; ++w) x[w] = parted<BF, true>(x[w]);
        *at = x;
    }
    __syncthreads();
}

template <bool BF, int D, int ROT>
struct State {
    float m, l;                  // of the lane's query row: maximum in units of log 2 (may lag), its positions' share of the sum
    f32x16 o[D / 32];
};

// A lane's chunk of keys for block tb, inner step k.  (2 k + h) ^ swap = (h ^ swap) ^ 2 k
template <bool BF, int D, int ROT>
__device__ inline __attribute__((always_inline)) u32x4 key_part(const char* keys, int tb, int k, int lane) {
    using Lay = Layout<BF, D, ROT>;
    constexpr int KN = Lay::RBD / 32, RBR = ROT ? Lay::RBR : 64;
    const int c = lane & 31, h = lane >> 5;
    if (k < KN) return *(const u32x4*)(keys + 32 * tb * Lay::RBD + ((c * Lay::RBD + (h ^ swap_k<Lay::RBD>(c)) * 16) ^ (32 * k)));
    return *(const u32x4*)(keys + Lay::R + 32 * tb * RBR + ((c * RBR + (h ^ swap_k<RBR>(c)) * 16) ^ (32 * (k - KN))));
}

// One tile by one wave, its scores in sc; NEXT: the scores of the tile behind it are made meanwhile.  edge: some row of the
// workgroup does not see all of the tile; the lane's row sees positions up to see.
template <bool BF, int D, int ROT, bool NEXT, class Load>
__device__ inline __attribute__((always_inline)) void attend_tile(char* __restrict k0, const char* __restrict keys,
                                                                  const char* __restrict values, char* __restrict v1, const Load& load, const u32x4* q, float scale2, bool edge,
                                                                  int see, int lane, f32x16 (&sc)[PA_TILE<BF> / 32],
                                                                  f32x16 (&nx)[PA_TILE<BF> / 32], State<BF, D, ROT>& s) {
    using Lay = Layout<BF, D, ROT>;
    constexpr int NB = Lay::TILE / 32, QN = Lay::QN, STEPS = NB * QN;
    if constexpr (NEXT) load(k0, v1);
    const int c = lane & 31, h = lane >> 5;
    const float ninf = -__builtin_inff();
    if (edge) {
#pragma unroll
        for (int tb = 0; tb < NB; ++tb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int p = 32 * tb + 8 * (i >> 2) + 4 * h + (i & 3);
                sc[tb][i] = p <= see ? sc[tb][i] : ninf;
            }
    }
    float top = ninf;
#pragma unroll
    for (int tb = 0; tb < NB; ++tb)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[tb][i]);
    top *= scale2;                                       // (scale2 > 0)
    if (__builtin_amdgcn_ballot_w64(top > s.m + PA_LAG)) {
        const float x = fmaxf(top, __shfl_xor(top, 32));
        const float m = x > s.m + PA_LAG ? x : s.m;
        const float al = s.m == m ? 1.0f : __builtin_amdgcn_exp2f(s.m - m);
        s.m = m;
        s.l *= al;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) s.o[d] = s.o[d] * al;
    }
    const float m = s.m == ninf ? 0.f : s.m;
    constexpr int AHEAD = 4;
    u32x4 kf[AHEAD];
    if constexpr (NEXT) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) kf[i] = key_part<BF, D, ROT>(keys, i % NB, i / NB, lane);
#pragma unroll
        for (int tb = 0; tb < NB; ++tb) nx[tb] = f32x16{};
    }
    int done = 0;
#pragma unroll
    for (int i = 0; i < (NEXT ? STEPS : 1); ++i) {
        if constexpr (NEXT) {
            nx[i % NB] = mma32<BF>(kf[i % AHEAD], q[i / NB], nx[i % NB]);
            if (i + AHEAD < STEPS) kf[i % AHEAD] = key_part<BF, D, ROT>(keys, (i + AHEAD) % NB, (i + AHEAD) / NB, lane);
        }
        const int to = NEXT ? 16 * NB * (i + 1) / STEPS : 16 * NB;
#pragma unroll
        for (int e = 0; e < 16 * NB; ++e) {
            if (e < done || e >= to) continue;
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e / 16][e % 16], scale2, -m));   // (of -infinity: 0)
            sc[e / 16][e % 16] = p;
            s.l += p;
        }
        done = to;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int tb = 0; tb < NB; ++tb) {
        if constexpr (BF) {
            // row 4 h + i of eight, elements col .. col + 3 of 32
            const int i = (lane >> 2) & 3, col = ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
            const int at = (4 * h + i) * Lay::RBD + (((col >> 3) ^ swap_v<BF, Lay::RBD>(i)) * 16) + (col & 7) * 2;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                // The weights in bf16: as large an error as the outputs' own rounding (0.0019 to 0.0023 of the outputs with both,
                // 0.0017 with that alone); two parts of 16 bits together would double this product
                u32x4 pf;
#pragma unroll
                for (int e = 0; e < 4; ++e) pf[e] = bf16_pair(sc[tb][8 * k + 2 * e], sc[tb][8 * k + 2 * e + 1]);
#pragma unroll
                for (int d = 0; d < D / 32; ++d) {
                    u32x4 vf;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const u32x2 t = read_turned(values + (32 * tb + 16 * k + 8 * u) * Lay::RBD + (at ^ (64 * d)));
                        vf[2 * u] = t[0];
                        vf[2 * u + 1] = t[1];
                    }
                    s.o[d] = mma32<true>(vf, pf, s.o[d]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 32 * tb + 8 * (i >> 2) + 4 * h + (i & 3);
#pragma unroll
                for (int d = 0; d < D / 32; ++d) {
                    const int e = 32 * d + c;
                    const float v = *(const float*)(values + row * Lay::RBD + (((e >> 2) ^ swap_v<BF, Lay::RBD>(row)) * 16) + (e & 3) * 4);
                    s.o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, sc[tb][i], s.o[d], 0, 0, 0);
                }
            }
        }
    }
}

template <bool BF, int D, int ROT, bool SPLIT>
__global__ void __launch_bounds__(64 * PA_WAVES, 2) prompt_attention_kernel(const PromptArgs a, int64_t items, int64_t per_xcd, int pieces) {
    using Lay = Layout<BF, D, ROT>;
    constexpr int ES = Lay::ES, TILE = Lay::TILE;
    __shared__ __attribute__((aligned(16))) char mem[Lay::BYTES];
    const int tid = threadIdx.x, lane_ = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane_ & 31, h = lane_ >> 5;
    // a key/value head's row blocks after one another on one XCD, where its rows are in L2
    const int64_t id = block_number();
    int64_t unit = (id & 7) * per_xcd + (id >> 3);
    int piece = 0;
    if constexpr (SPLIT) {
        piece = (int)(unit % pieces);
        unit /= pieces;
    }
    if ((id >> 3) >= per_xcd || unit >= items * a.n_kv) return;
    const int kvh = (int)(unit / items);
    Seq s;
    int rb;
    if (!find_block(a, unit - kvh * items, lane_, s, rb)) return;
    const int G = a.n_q / a.n_kv;
    const int64_t rows = (int64_t)s.n * G, row0 = (int64_t)rb * PA_ROWS, row = row0 + 32 * wave + c;
    const bool in = row < rows;
    const int i = in ? (int)(row / G) : 0, hq = kvh * G + (in ? (int)(row - (int64_t)i * G) : 0);
    const int before = s.len - s.n;                      // (may be negative)
    const int lim = in ? before + i : -1;                // the last position that the lane's row sees
    // positions that some row of the workgroup sees, and that all of them do
    const int last = (int)((std::min(rows, row0 + PA_ROWS) - 1) / G);
    int start = 0, end = std::max(0, std::min(s.len, before + last + 1));
    if constexpr (SPLIT) {
        const int tiles = (end + TILE - 1) / TILE;
        start = (int)((int64_t)tiles * piece / pieces) * TILE;
        end = std::min(end, (int)((int64_t)tiles * (piece + 1) / pieces) * TILE);
    }
    const int all = before + (int)(row0 / G) + 1;
    // scores times scale2 > 0: a negative scale's sign goes to the query, a scale of 0 makes it zeros
    const float scale2 = a.scale == 0.f ? 1.0f : std::fabs(a.scale) * LOG2E;
    u32x4 q[Lay::QN];
    {
        const char* from = (const char*)a.q + ((int64_t)(s.q0 + i) * a.n_q + hq) * ((D + ROT) * ES) + 16 * h;
        const uint32_t flip = a.scale < 0.f ? (BF ? 0x80008000u : 0x80000000u) : 0u, keep = a.scale == 0.f ? 0u : ~0u;
#pragma unroll
        for (int k = 0; k < Lay::QN; ++k) {
            q[k] = u32x4{0u, 0u, 0u, 0u};
            if (in) q[k] = *(const u32x4*)(from + 32 * k);
#pragma unroll
            for (int w = 0; w < 4; ++w) q[k][w] = (q[k][w] & keep) ^ flip;
        }
    }
    State<BF, D, ROT> st;
    st.m = -__builtin_inff();
    st.l = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) st.o[d] = f32x16{};
    const uint32_t stride = (uint32_t)a.n_kv * D * ES;
    constexpr int NK = TILE * Lay::RBD / 1024 / PA_WAVES, NR = ROT ? TILE * Lay::RBR / 1024 / PA_WAVES : 1;
    static_assert(NK * 1024 * PA_WAVES == TILE * Lay::RBD && (!ROT || NR * 1024 * PA_WAVES == TILE * Lay::RBR), "whole pieces a wave");
    uint32_t ko[NK], ro[NR], vo[NK];
    lane_places<BF, Lay::RBD, 0>(ko, stride, wave, lane_);
    lane_places<BF, Lay::RBD, 1>(vo, stride, wave, lane_);
    if constexpr (ROT > 0) lane_places<BF, Lay::RBR, 0>(ro, Lay::RBR, wave, lane_);
    const char *const kb = (const char*)a.k + (int64_t)s.k0 * stride + kvh * (D * ES), *const vb = (const char*)a.v + (kb - (const char*)a.k),
               *const rb_ = ROT ? (const char*)a.r + (int64_t)s.k0 * Lay::RBR : nullptr;
    auto keys = [&](int t0, char* to, int lane) __attribute__((always_inline)) {
        issue_rows<BF, Lay::RBD, 0>(ko, kb + (int64_t)t0 * stride, s.len - t0, stride, to, wave, lane);
        if constexpr (ROT > 0) issue_rows<BF, Lay::RBR, 0>(ro, rb_ + (int64_t)t0 * Lay::RBR, s.len - t0, Lay::RBR, to + Lay::R, wave, lane);
    };
    auto values = [&](int t0, char* to, int lane) __attribute__((always_inline)) {
        issue_rows<BF, Lay::RBD, 1>(vo, vb + (int64_t)t0 * stride, s.len - t0, stride, to, wave, lane);
    };
    // Tile t's weights and its product with V run beside tile t + 1's scores: the keys are a tile ahead of the values.
    // What lies in k0 and v1 has been read, k1 and v0 are on their way.
    auto step = [&](auto next, int t0, char* k0, char* k1, char* v0, char* v1, f32x16 (&sc)[TILE / 32],
                    f32x16 (&nx)[TILE / 32]) __attribute__((always_inline)) {
        const bool edge = t0 + TILE > all;
        int lane = lane_;
        asm volatile("" : "+v"(lane));                   // (addresses made anew for each tile: kept, they would take the sums' registers)
        wait_loads<0>();
        __syncthreads();
        if (edge) clean_values<BF, D>(v0, lim - t0, wave, lane, st.o);
        auto load = [&](char* k, char* v) __attribute__((always_inline)) {
            if (t0 + 2 * TILE < end) keys(t0 + 2 * TILE, k, lane);
            values(t0 + TILE, v, lane);
        };
        attend_tile<BF, D, ROT, decltype(next)::value>(k0, k1, v0, v1, load, q, scale2, edge, lim - t0, lane, sc, nx, st);
    };
    if (start < end) {
        char *const k0 = mem, *const k1 = mem + Lay::KEYS, *const v0 = mem + Lay::V, *const v1 = v0 + Lay::VALUES;
        f32x16 s0[TILE / 32], s1[TILE / 32];
        keys(start, k0, lane_);
        if (start + TILE < end) keys(start + TILE, k1, lane_);
        values(start, v0, lane_);
        if (start + TILE < end) wait_loads<(Lay::KEYS + Lay::VALUES) / 1024 / PA_WAVES>();
        else wait_loads<Lay::VALUES / 1024 / PA_WAVES>();
        lds_barrier();
#pragma unroll
        for (int tb = 0; tb < TILE / 32; ++tb) {
            s0[tb] = f32x16{};
#pragma unroll
            for (int k = 0; k < Lay::QN; ++k) s0[tb] = mma32<BF>(key_part<BF, D, ROT>(k0, tb, k, lane_), q[k], s0[tb]);
        }
        int t0 = start;
        for (; t0 + 2 * TILE < end; t0 += 2 * TILE) {
            step(std::true_type{}, t0, k0, k1, v0, v1, s0, s1);
            step(std::true_type{}, t0 + TILE, k1, k0, v1, v0, s1, s0);
        }
        char* v = v0;
        if (t0 + TILE < end) {
            step(std::true_type{}, t0, k0, k1, v0, v1, s0, s1);
#pragma unroll
            for (int tb = 0; tb < TILE / 32; ++tb) s0[tb] = s1[tb];
            v = v1;
            t0 += TILE;
        }
        step(std::false_type{}, t0, k0, k1, v, v1, s0, s1);
    }
    if (!in) return;
    const float l = st.l + __shfl_xor(st.l, 32);
    const int64_t at = (int64_t)(s.q0 + i) * a.n_q + hq;
    if constexpr (SPLIT) {
        const int64_t pr = (int64_t)piece * a.T * a.n_q + at;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(f32x4*)(a.part_o + pr * D + 32 * d + 8 * j + 4 * h) =
                    f32x4{st.o[d][4 * j], st.o[d][4 * j + 1], st.o[d][4 * j + 2], st.o[d][4 * j + 3]};
        if (h == 0) ((f32x2*)a.part_ml)[pr] = f32x2{st.m, l};
        return;
    }
    const float r = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            store4<BF>(a.out, at * D + 32 * d + 8 * j + 4 * h, st.o[d][4 * j] * r, st.o[d][4 * j + 1] * r, st.o[d][4 * j + 2] * r,
                       st.o[d][4 * j + 3] * r);
    if (a.lse && h == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (st.m + __builtin_amdgcn_logf(l)) * LN2;
}

// The pieces of a row's positions, in order: a workgroup has 1024 / D rows of a block, a thread four elements
template <bool BF, int D>
__global__ void __launch_bounds__(256) prompt_join_kernel(const PromptArgs a, int64_t items, int pieces) {
    constexpr int ROWS = 1024 / D, PER = PA_ROWS / ROWS;
    const int tid = threadIdx.x;
    const int64_t id = block_number(), unit = id / PER;
    if (unit >= items * a.n_kv) return;
    const int kvh = (int)(unit / items);
    Seq s;
    int rb;
    if (!find_block(a, unit - kvh * items, tid & 63, s, rb)) return;
    const int G = a.n_q / a.n_kv, e = tid % (D / 4) * 4;
    const int64_t row = (int64_t)rb * PA_ROWS + (id % PER) * ROWS + tid / (D / 4);
    if (row >= (int64_t)s.n * G) return;
    const int i = (int)(row / G), hq = kvh * G + (int)(row - (int64_t)i * G);
    const int64_t at = (int64_t)(s.q0 + i) * a.n_q + hq, step = a.T * a.n_q;
    constexpr int U = 4;
    float m = -__builtin_inff(), l = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < pieces; p += U) {
        f32x2 q[U];
        f32x4 v[U];
        float top = m;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t pr = at + std::min(p + k, pieces - 1) * step;
            q[k] = ((const f32x2*)a.part_ml)[pr];
            v[k] = *(const f32x4*)(a.part_o + pr * D + e);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) top = fmaxf(top, q[k][0]);
        const float al = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= al;
        x = x * al;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (p + k >= pieces) break;
            const float f = q[k][0] == m ? 1.0f : __builtin_amdgcn_exp2f(q[k][0] - m);
            l += q[k][1] * f;
            x = x + v[k] * f;
        }
    }
    const float r = l == 0.f ? 0.f : 1.0f / l;
    store4<BF>(a.out, at * D + e, x[0] * r, x[1] * r, x[2] * r, x[3] * r);
    if (a.lse && e == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// row blocks: every sequence ends in one that is not full, at most
int64_t blocks_at_most(int n_q, int n_kv, int64_t T, int B) {
    const int64_t rows = T * (n_q / n_kv);
    return std::min(rows, rows / PA_ROWS + B);
}

template <bool BF, int D, int ROT>
int launch_rows(const PromptArgs& a, hipStream_t st) {
    const int64_t items = blocks_at_most(a.n_q, a.n_kv, a.T, a.B), least = (int64_t)PA_LEAST * PA_TILE<BF>;
    const int pieces = (int)std::min<int64_t>(prompt_pieces(a.n_q, a.n_kv, a.T, a.B), (a.L + least - 1) / least);
    const int64_t per = (items * a.n_kv * std::max(pieces, 1) + 7) / 8;
    {
        KernelTimer kt_("prompt_attention", st);
        if (pieces > 1) prompt_attention_kernel<BF, D, ROT, true><<<grid_of(per * 8), dim3(64 * PA_WAVES), 0, st>>>(a, items, per, pieces);
        else prompt_attention_kernel<BF, D, ROT, false><<<grid_of(per * 8), dim3(64 * PA_WAVES), 0, st>>>(a, items, per, 1);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || pieces <= 1) return (int)e;
    }
    KernelTimer kt_("prompt_join", st);
    prompt_join_kernel<BF, D><<<grid_of(items * a.n_kv * (PA_ROWS * D / 1024)), dim3(256), 0, st>>>(a, items, pieces);
    return (int)hipGetLastError();
}
template <bool BF, int D>
int launch_rot(const PromptArgs& a, hipStream_t st) {
    return a.rot == 0 ? launch_rows<BF, D, 0>(a, st) : a.rot == 32 ? launch_rows<BF, D, 32>(a, st) : launch_rows<BF, D, 64>(a, st);
}

}  // namespace

int prompt_pieces(int n_q, int n_kv, int64_t T, int B) {
    const int64_t blocks = blocks_at_most(n_q, n_kv, T, B) * n_kv;
    return B == 0 || blocks == 0 || blocks > PA_FEW ? 1 : (int)(PA_FILL / blocks);
}

// `pieces` workgroups of a block hold PA_ROWS rows each, or what few tokens have, and there are PA_FILL of them at most
int64_t prompt_rows_at_most(int n_q, int n_kv, int64_t T) {
    return n_kv > PA_FEW ? 0 : std::min<int64_t>(PA_ROWS, T * (n_q / n_kv)) * PA_FILL;
}

int launch_prompt_attention(const PromptArgs& a, void* stream) {
    if (a.B == 0 || a.T == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    if (a.dtype == ORDERMOE_BF16) return a.head_dim == 64 ? launch_rot<true, 64>(a, st) : launch_rot<true, 128>(a, st);
    return a.head_dim == 64 ? launch_rot<false, 64>(a, st) : launch_rot<false, 128>(a, st);
}

}  // namespace ordermoe
