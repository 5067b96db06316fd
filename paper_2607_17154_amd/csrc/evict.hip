// Sequences of the latent cache cut to a budget of tokens.
//
//   evict_select_kernel  one workgroup per sequence: the keep-th largest key of its places (mass,
//                        or above all masses where the token is protected) by three histograms
//                        of the keys' bits, then the places that stay, go or move; few rows move here
//   evict_digit_kernel, evict_mark_kernel  the same where tables are long, a workgroup per slice of a
//                        sequence: a slice's histogram of the next digit (three launches; every
//                        workgroup finds the digits before from all the slices' histograms), then its places
//   evict_move_kernel    the i-th kept row past the budget into the i-th place that came free
//                        before it: as few rows move as can
// Masses and positions are 8 bytes a place, little beside a row: barriers and launches bound the selection (16 of 1016 places
// 10 us, of which 7 to 8 select; 20000 to 60000 places of 8 sequences 40), what the card copies the moves (5.5 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "common.hpp"
#include "grid.hpp"
#include "mfma.hpp"

namespace ordermoe {
namespace {

constexpr int EV_CHUNK = 8192, EV_WORDS = EV_CHUNK / 64;      // places gone through together
constexpr int EV_BINS = 2048;                        // of a histogram: digits of 11, 11 and 10 bits
constexpr int EV_SLICES = 64;                        // of a sequence, at most, and one more
constexpr int EV_MOVES = 256;                        // rows of a sequence that the workgroup which finds them moves
constexpr uint32_t EV_SAFE = 0xFFFFFFFFu;
__device__ inline int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ inline int digit_bits(int pass) { return pass == 2 ? 10 : 11; }

// a mass as an integer of the same order; NaN below all
__device__ inline uint32_t mass_key(float m) {
    if (m != m) return 0u;
    const uint32_t u = __float_as_uint(m + 0.0f);    // (-0 as 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A sequence's places
struct Places {
    int n;                   // of them
    const float* mass;
    const int32_t* pos;
    float* mass_out;
    int32_t* pos_out;
    int32_t* kept;
    int first;
    int64_t recent;          // positions from here on are protected
    __device__ uint32_t key(int q, float m) const { return q < first || q >= recent ? EV_SAFE : mass_key(m); }
};
__host__ __device__ inline int64_t most_places(const EvictArgs& a) {
    const int64_t table = (int64_t)a.max_pages << a.cache.page_shift;
    return table < a.stride ? table : a.stride;
}
__device__ inline Places places_of(const EvictArgs& a, int b) {
    const int64_t cap = most_places(a);
    const int ctx = a.ctx_len[b];
    return Places{(int)(ctx < 0 ? 0 : ctx < cap ? ctx : cap), a.mass + b * a.stride, a.pos + b * a.stride, a.mass_out + b * a.stride,
                  a.pos_out + b * a.stride, a.kept + (int64_t)b * a.keep, a.first, (int64_t)a.seq_len[b] - a.recent};
}
// a sequence that keeps all of its tokens
template <int NT>
__device__ inline void keep_all(const EvictArgs& a, const Places& pl, int b, int tid) {
    every(tid, a.keep, NT, [&](int p) {
        pl.kept[p] = p < pl.n ? p : -1;
        if (p < pl.n) {
            if (pl.mass_out != pl.mass) pl.mass_out[p] = pl.mass[p];
            if (pl.pos_out != pl.pos) pl.pos_out[p] = pl.pos[p];
        }
    });
    if (tid == 0) { a.moves[b] = -1; a.len_out[b] = pl.n; }
}

// the sum over the threads before this one; all: over every thread
template <int NT>
__device__ inline uint32_t sum_before(uint32_t own, uint32_t* s_wave, int tid, uint32_t& all) {
    const int lane = tid & 63, wave = tid >> 6;
    uint32_t inc = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(inc, o);
        if (lane >= o) inc += v;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = inc;
    __syncthreads();
    uint32_t base = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        base += w < wave ? s_wave[w] : 0u;
        all += s_wave[w];
    }
    return base + inc - own;
}
__device__ inline uint32_t bits_below(uint64_t m) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
}
// the lowest k set bits of m
__device__ inline uint64_t lowest(uint64_t m, int k) {
    if (k >= __builtin_popcountll(m)) return m;
    uint64_t r = 0;
    for (; k > 0; --k) {
        r |= m & (0 - m);
        m &= m - 1;
    }
    return r;
}
// bits of the 64 places from p on that lie below n
__device__ inline uint64_t below(int p, int n) { return n <= p ? 0ull : n - p >= 64 ? ~0ull : (1ull << (n - p)) - 1; }

// The bin of s_hist in which the `more`-th largest key lies; `more` becomes its rank there.  s_found: two words of LDS
template <int NT>
__device__ inline uint32_t find_bin(const uint32_t* s_hist, uint32_t* s_wave, uint32_t* s_found, uint32_t& more, int tid) {
    constexpr int PER = EV_BINS / NT;
    // from the top: thread t holds bins PER (NT - 1 - t) .. + PER - 1
    const int lo = PER * (NT - 1 - tid);
    uint32_t h[PER], own = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) own += h[i] = s_hist[lo + i];
    uint32_t above = sum_before<NT>(own, s_wave, tid, all);
    if (above < more && above + own >= more) {
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) {
            if (above < more && above + h[i] >= more) { s_found[0] = (uint32_t)(lo + i); s_found[1] = more - above; }
            above += h[i];
        }
    }
    __syncthreads();
    more = s_found[1];
    return s_found[0];
}

struct Marks {
    uint64_t stay[EV_WORDS], equal[EV_WORDS];
    uint32_t off[EV_WORDS];
};
// positions and masses of a chunk's places, p0 + thread + i * NT
template <int NT>
struct Chunk {
    static constexpr int PER = EV_CHUNK / NT;
    int32_t pos[PER];
    float mass[PER];
    __device__ void read(const Places& pl, int64_t p0, int64_t hi, int tid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int64_t p = std::min<int64_t>(p0 + tid + i * NT, hi - 1);
            pos[i] = pl.pos[p];
            mass[i] = pl.mass[p];
        }
    }
};
// Of the chunk of places [p0, hi) those stay whose key is larger than `limit`, and the first `more` of all whose key is
// equal; the places that go and the rows that move, after `holes` and `fills` of them.  `equal` keys lie before.
template <int NT>
__device__ inline void mark_chunk(const EvictArgs& a, const Places& pl, int b, int64_t p0, int64_t hi, const Chunk<NT>& ch, uint32_t limit,
                                  uint32_t more, uint32_t& equal, uint32_t& holes, uint32_t& fills, Marks& s, uint32_t* s_wave, int tid) {
    static_assert(EV_WORDS <= NT && EV_CHUNK < 1 << 16, "a thread a word, two counts in 32 bits");
    constexpr int WAVES = NT / 64;
    const int lane = tid & 63, wave = tid >> 6, keep = a.keep;
    const int words = (int)std::min<int64_t>(EV_WORDS, (hi - p0 + 63) / 64);
#pragma unroll
    for (int i = 0; i < Chunk<NT>::PER; ++i) {
        const int w = wave + i * WAVES;
        if (w >= words) break;
        const uint32_t key = pl.key(ch.pos[i], ch.mass[i]);
        const bool in = p0 + w * 64 + lane < hi;
        const uint64_t gt = __builtin_amdgcn_ballot_w64(in && key > limit), eq = __builtin_amdgcn_ballot_w64(in && key == limit);
        if (lane == 0) { s.stay[w] = gt; s.equal[w] = eq; }
    }
    __syncthreads();
    uint32_t all;
    const uint64_t eq = tid < words ? s.equal[tid] : 0ull;
    const uint32_t before = equal + sum_before<NT>((uint32_t)__builtin_popcountll(eq), s_wave, tid, all);
    equal += all;
    uint64_t stay = 0ull, front = 0ull;
    if (tid < words) {
        stay = s.stay[tid] | (before < more ? lowest(eq, (int)(more - before)) : 0ull);
        front = below((int)p0 + tid * 64, keep);
    }
    const uint64_t there = below((int)p0 + tid * 64, (int)hi);
    const uint32_t own = (uint32_t)__builtin_popcountll(front & there & ~stay) | (uint32_t)__builtin_popcountll(stay & ~front) << 16;
    const uint32_t off = sum_before<NT>(own, s_wave, tid, all);
    if (tid < words) { s.stay[tid] = stay; s.off[tid] = off; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < Chunk<NT>::PER; ++i) {
        const int w = wave + i * WAVES, q0 = (int)p0 + w * 64, at = q0 + lane;
        if (w >= words) break;
        const uint64_t st = s.stay[w], fr = below(q0, keep) & below(q0, (int)hi), hm = fr & ~st, fm = st & ~fr;
        const uint32_t o = s.off[w];
        if ((hm >> lane) & 1) a.holes[(int64_t)b * a.holes_max + holes + (o & 0xFFFFu) + bits_below(hm)] = at;
        if ((fm >> lane) & 1) a.fills[(int64_t)b * a.holes_max + fills + (o >> 16) + bits_below(fm)] = at;
        if ((fr & st) >> lane & 1) {
            pl.kept[at] = at;
            if (pl.mass_out != pl.mass) pl.mass_out[at] = ch.mass[i];
            if (pl.pos_out != pl.pos) pl.pos_out[at] = ch.pos[i];
        }
    }
    holes += all & 0xFFFFu;
    fills += all >> 16;
}

// one more for the digit of a key that shares the digits before
__device__ inline void count_key(uint32_t* s_hist, uint32_t key, int pass, uint32_t prefix) {
    const int shift = digit_shift(pass), bits = digit_bits(pass);
    if (pass == 0 || (key >> (shift + bits)) == prefix) atomicAdd(&s_hist[(key >> shift) & ((1u << bits) - 1u)], 1u);
}

// Up to ROWS moves of a sequence from the x0-th on, by a workgroup
template <int NT, int ROWS>
struct Move { const char* from[ROWS]; char* to[ROWS]; };
template <int NT, int ROWS>
__device__ inline void move_rows(const EvictArgs& a, int b, int64_t x0, int rows, int chunks, Move<NT, ROWS>& s, int tid) {
    if (tid < rows) {
        const int to = a.holes[(int64_t)b * a.holes_max + x0 + tid], from = a.fills[(int64_t)b * a.holes_max + x0 + tid];
        a.kept[(int64_t)b * a.keep + to] = from;
        a.mass_out[b * a.stride + to] = a.mass[b * a.stride + from];
        a.pos_out[b * a.stride + to] = a.pos[b * a.stride + from];
        const int sh = a.cache.page_shift, in = (1 << sh) - 1;
        const int32_t* table = a.page_table + (int64_t)b * a.max_pages;
        const int64_t pt = table[to >> sh], pf = table[from >> sh], row = (int64_t)chunks * 16;
        s.from[tid] = pf >= 0 && pf < a.cache.n_pages ? a.cache.rows + ((pf << sh) + (from & in)) * row : nullptr;
        s.to[tid] = pt >= 0 && pt < a.cache.n_pages ? a.cache.rows + ((pt << sh) + (to & in)) * row : nullptr;
    }
    __syncthreads();
    for (int u = tid; u < rows * chunks; u += NT) {
        const int r = u / chunks, c = u - r * chunks;
        u32x4 v = {0u, 0u, 0u, 0u};
        if (s.from[r]) v = *(const u32x4*)(s.from[r] + 16 * c);
        if (s.to[r]) *(u32x4*)(s.to[r] + 16 * c) = v;
    }
}

// tables of up to EV_CHUNK places: a sequence in registers
// chunks > 0: the rows, of so many pieces of 16 bytes, move here too
__global__ void __launch_bounds__(1024) evict_select_kernel(const EvictArgs a, int chunks) {
    constexpr int NT = 1024;
    __shared__ Move<NT, EV_MOVES> s_move;
    __shared__ uint32_t s_hist[EV_BINS], s_wave[NT / 64], s_found[2];
    __shared__ Marks s_marks;
    const int tid = threadIdx.x, b = (int)block_number();
    if (b >= a.B) return;
    const Places pl = places_of(a, b);
    if (pl.n <= a.keep) {
        keep_all<NT>(a, pl, b, tid);
        return;
    }
    Chunk<NT> ch;
    ch.read(pl, 0, pl.n, tid);
    for (int i = tid; i < EV_BINS; i += NT) s_hist[i] = 0u;
    __syncthreads();
    uint32_t prefix = 0u, more = (uint32_t)a.keep;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
#pragma unroll
        for (int i = 0; i < Chunk<NT>::PER; ++i) {
            if (i * NT >= pl.n) break;
            if (tid + i * NT < pl.n) count_key(s_hist, pl.key(ch.pos[i], ch.mass[i]), pass, prefix);
        }
        __syncthreads();
        const uint32_t bin = find_bin<NT>(s_hist, s_wave, s_found, more, tid);
        prefix = (prefix << digit_bits(pass)) | bin;
        for (int i = tid; i < EV_BINS; i += NT) s_hist[i] = 0u;
        __syncthreads();
    }
    uint32_t equal = 0, holes = 0, fills = 0;
    mark_chunk<NT>(a, pl, b, 0, pl.n, ch, prefix, more, equal, holes, fills, s_marks, s_wave, tid);
    if (tid == 0) a.moves[b] = (int32_t)holes;
    if (chunks == 0) return;
    __syncthreads();                                 // the places are written
    if (tid == 0) a.len_out[b] = a.keep;
    move_rows<NT, EV_MOVES>(a, b, 0, (int)holes, chunks, s_move, tid);
}

// Slices of `slice` places: those before the budget, then those from it on, so that a slice is all front or all back.
struct Slices {
    int front, all;          // slices of a sequence before the budget, in all
};
__device__ inline Slices slices_of(int n, int keep, int64_t slice) {
    const int f = (int)((keep + slice - 1) / slice);
    return Slices{f, f + (int)((n - keep + slice - 1) / slice)};
}
// what the passes leave behind for the ones after, per sequence and pass
struct Found { uint32_t prefix, more; };

// Sums all slices' histograms of a pass into s_hist.  They are EV_BINS counts each.
template <int NT>
__device__ inline void sum_slices(const uint32_t* part, int slices, uint32_t* s_hist, int tid) {
    u32x4 s = {0u, 0u, 0u, 0u};
#pragma unroll 8
    for (int k = 0; k < slices; ++k) s += *(const u32x4*)(part + (int64_t)k * EV_BINS + 4 * tid);
    *(u32x4*)(s_hist + 4 * tid) = s;
    static_assert(4 * NT == EV_BINS, "four bins a thread");
}
constexpr int ES_THREADS = 512;

// pass 0, 1, 2: the slice's histogram of digit `pass` to a.part, after its number of keys that are larger by the digit
// before to a.above
__global__ void __launch_bounds__(ES_THREADS) evict_digit_kernel(const EvictArgs a, int slices, int64_t slice, int pass) {
    constexpr int NT = ES_THREADS;
    __shared__ __attribute__((aligned(16))) uint32_t s_hist[EV_BINS];
    __shared__ uint32_t s_wave[NT / 64], s_found[2];
    const int64_t id = block_number();
    const int b = (int)(id / slices), k = (int)(id - (int64_t)b * slices), tid = threadIdx.x;
    if (b >= a.B) return;
    const Places pl = places_of(a, b);
    if (pl.n <= a.keep) {
        if (pass == 0 && k == 0) keep_all<NT>(a, pl, b, tid);
        return;
    }
    const Slices sl = slices_of(pl.n, a.keep, slice);
    if (k >= sl.all) return;
    uint32_t* part = a.part + ((int64_t)pass * a.B + b) * slices * EV_BINS;
    uint32_t prefix = 0u, more = (uint32_t)a.keep;
    if (pass > 0) {
        const uint32_t* before = part - (int64_t)a.B * slices * EV_BINS;
        Found* found = (Found*)a.found + b;
        if (pass > 1) { prefix = found->prefix; more = found->more; }
        sum_slices<NT>(before, sl.all, s_hist, tid);
        __syncthreads();
        const uint32_t bin = find_bin<NT>(s_hist, s_wave, s_found, more, tid);
        prefix = (prefix << digit_bits(pass - 1)) | bin;
        if (k == 0 && tid == 0) found[pass == 1 ? 0 : a.B] = Found{prefix, more};
        uint32_t larger = 0, all;
#pragma unroll
        for (int i = 0; i < EV_BINS / NT; ++i)
            if ((uint32_t)(tid + i * NT) > bin) larger += before[(int64_t)k * EV_BINS + tid + i * NT];
        sum_before<NT>(larger, s_wave, tid, all);
        if (tid == 0) a.above[(((int64_t)pass - 1) * a.B + b) * slices + k] = all;
    }
    for (int i = tid; i < EV_BINS; i += NT) s_hist[i] = 0u;
    __syncthreads();
    const int64_t lo = k < sl.front ? k * slice : a.keep + (k - sl.front) * slice;
    const int64_t hi = std::min<int64_t>(lo + slice, k < sl.front ? a.keep : pl.n);
    for (int64_t p0 = lo; p0 < hi; p0 += EV_CHUNK) {
        Chunk<NT> ch;
        ch.read(pl, p0, hi, tid);
#pragma unroll
        for (int i = 0; i < Chunk<NT>::PER; ++i)
            if (p0 + tid + i * NT < hi) count_key(s_hist, pl.key(ch.pos[i], ch.mass[i]), pass, prefix);
    }
    __syncthreads();
    *(u32x4*)(part + (int64_t)k * EV_BINS + 4 * tid) = *(const u32x4*)(s_hist + 4 * tid);
}

__global__ void __launch_bounds__(ES_THREADS) evict_mark_kernel(const EvictArgs a, int slices, int64_t slice) {
    constexpr int NT = ES_THREADS;
    __shared__ __attribute__((aligned(16))) uint32_t s_hist[EV_BINS];
    __shared__ uint32_t s_wave[NT / 64], s_found[2], s_larger[EV_SLICES + 2];
    __shared__ Marks s_marks;
    const int64_t id = block_number();
    const int b = (int)(id / slices), k = (int)(id - (int64_t)b * slices), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (b >= a.B) return;
    const Places pl = places_of(a, b);
    if (pl.n <= a.keep) return;
    const Slices sl = slices_of(pl.n, a.keep, slice);
    if (k >= sl.all) return;
    const uint32_t* part = a.part + ((int64_t)2 * a.B + b) * slices * EV_BINS;
    const Found f = ((const Found*)a.found)[a.B + b];
    uint32_t more = f.more;
    sum_slices<NT>(part, sl.all, s_hist, tid);
    __syncthreads();
    const uint32_t bin = find_bin<NT>(s_hist, s_wave, s_found, more, tid), limit = (f.prefix << digit_bits(2)) | bin;
    // the slices before: how many of their keys are larger, a wave a slice
    for (int j = wave; j < k; j += NT / 64) {
        uint32_t larger = 0;
        for (int i = lane; i < 1 << digit_bits(2); i += 64)
            if ((uint32_t)i > bin) larger += part[(int64_t)j * EV_BINS + i];
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) larger += __shfl_xor(larger, o);
        if (lane == 0) s_larger[j] = larger + a.above[((int64_t)0 * a.B + b) * slices + j] + a.above[((int64_t)1 * a.B + b) * slices + j];
    }
    __syncthreads();
    uint32_t equal = 0, holes = 0, fills = 0;
    for (int j = 0; j < k; ++j) {
        const uint32_t eq = part[(int64_t)j * EV_BINS + bin], take = equal >= more ? 0u : std::min(eq, more - equal), stay = s_larger[j] + take;
        equal += eq;
        if (j < sl.front) holes += (uint32_t)(std::min<int64_t>(a.keep, (j + 1) * slice) - j * slice) - stay;
        else fills += stay;
    }
    const int64_t lo = k < sl.front ? k * slice : a.keep + (k - sl.front) * slice;
    const int64_t hi = std::min<int64_t>(lo + slice, k < sl.front ? a.keep : pl.n);
    for (int64_t p0 = lo; p0 < hi; p0 += EV_CHUNK) {
        Chunk<NT> ch;
        ch.read(pl, p0, hi, tid);
        mark_chunk<NT>(a, pl, b, p0, hi, ch, limit, more, equal, holes, fills, s_marks, s_wave, tid);
        __syncthreads();
    }
    // (the last slice before the budget has come to all of the places that go)
    if (k == sl.front - 1 && tid == 0) a.moves[b] = (int32_t)holes;
}

constexpr int EM_ROWS = 32;                          // rows that a workgroup moves

__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs a, int per_seq, int chunks) {
    __shared__ Move<256, EM_ROWS> s_move;
    const int64_t id = block_number();
    const int b = (int)(id / per_seq), x0 = (int)(id - (int64_t)b * per_seq) * EM_ROWS, tid = threadIdx.x;
    if (b >= a.B) return;
    const int moves = a.moves[b], rows = std::min(EM_ROWS, moves - x0);
    if (x0 == 0 && tid == 0 && moves >= 0) a.len_out[b] = a.keep;        // (it may be ctx_len: read by no kernel from here on)
    if (rows > 0) move_rows<256, EM_ROWS>(a, b, x0, rows, chunks, s_move, tid);
}

}  // namespace

int evict_slices(int64_t places) { return (int)std::min<int64_t>(EV_SLICES + 1, places / EV_CHUNK + 2); }
size_t evict_slice_words(int64_t places) { return places <= EV_CHUNK ? 0 : (size_t)evict_slices(places) * (3 * EV_BINS + 2) + 4; }

int launch_latent_evict(const EvictArgs& a, void* stream) {
    if (a.B == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    const int64_t cap = most_places(a);
    const int chunks = (a.cache.rank + a.cache.rot) * (a.cache.dtype == ORDERMOE_BF16 ? 2 : 4) / 16;
    // One workgroup per sequence goes through a thousand places a microsecond; slices take four more launches (one sequence of
    // 8000 places 18 us in one kernel).  Few rows move there and then (16 of 1016 places: 12.0 us with a kernel for them, 10.0; 128
    // of 1128 in 64 sequences: 15.9 and 14.2).
    if (cap <= EV_CHUNK) {
        const bool here = a.holes_max <= EV_MOVES;
        KernelTimer kt_("evict_select", st);
        evict_select_kernel<<<grid_of(a.B), dim3(1024), 0, st>>>(a, here ? chunks : 0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || here) return (int)e;
    } else {
        const int64_t slice = std::max<int64_t>(EV_CHUNK, (cap + EV_SLICES - 2) / (EV_SLICES - 1));
        const int slices = (int)std::min<int64_t>(evict_slices(cap), cap / slice + 2);
        const dim3 grid = grid_of((int64_t)a.B * slices);
        for (int pass = 0; pass < 3; ++pass) {
            KernelTimer kt_("evict_digit", st);
            evict_digit_kernel<<<grid, dim3(ES_THREADS), 0, st>>>(a, slices, slice, pass);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return (int)e;
        }
        KernelTimer kt_("evict_mark", st);
        evict_mark_kernel<<<grid, dim3(ES_THREADS), 0, st>>>(a, slices, slice);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    if (a.holes_max == 0) return 0;
    const int per = (int)((a.holes_max + EM_ROWS - 1) / EM_ROWS);
    KernelTimer kt_("evict_move", st);
    evict_move_kernel<<<grid_of((int64_t)a.B * per), dim3(256), 0, st>>>(a, per, chunks);
    return (int)hipGetLastError();
}

}  // namespace ordermoe
