// Sequences of the latent cache cut to a budget of tokens.
//
//   evict_select_kernel  one workgroup per sequence: the keep-th largest key of its places (mass,
//                        or above all masses where the token is protected) by three histograms
//                        of the keys' bits, then the places that stay, go or move
//   evict_move_kernel    the i-th kept row past the budget into the i-th place that came free
//                        before it: as few rows move as can
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "common.hpp"
#include "grid.hpp"
#include "mfma.hpp"

namespace ordermoe {
namespace {

constexpr int EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64;
constexpr int EV_BLOCK = 32768;                      // places whose keys LDS holds; those of longer sequences are made again
constexpr int EV_WORDS = EV_BLOCK / 64;
static_assert(EV_WORDS <= EV_THREADS && EV_BLOCK <= 1 << 15, "a thread a word, two counts in 32 bits");
constexpr int EV_AHEAD = 8;                          // places of a thread whose reads are in flight together
constexpr int EV_BINS = 2048;                        // of a histogram: 11 bits, 11 bits, 10 bits
constexpr uint32_t EV_SAFE = 0xFFFFFFFFu;

// a mass as an integer of the same order; NaN below all
__device__ inline uint32_t mass_key(float m) {
    if (m != m) return 0u;
    const uint32_t u = __float_as_uint(m + 0.0f);    // (-0 as 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// the sum over the threads before this one; all: over every thread
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
    for (int w = 0; w < EV_WAVES; ++w) {
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

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const EvictArgs a) {
    __shared__ uint32_t s_key[EV_BLOCK], s_hist[EV_BINS], s_off[EV_WORDS], s_wave[EV_WAVES];
    __shared__ uint64_t s_stay[EV_WORDS], s_equal[EV_WORDS];
    __shared__ uint32_t s_bin, s_more;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = (int)block_number();
    if (b >= a.B) return;
    const int64_t cap = std::min<int64_t>((int64_t)a.max_pages << a.cache.page_shift, a.stride);
    const int ctx = a.ctx_len[b], n = (int)std::min<int64_t>(ctx < 0 ? 0 : ctx, cap), keep = a.keep;
    const float* mass = a.mass + b * a.stride;
    const int32_t* pos = a.pos + b * a.stride;
    float* mass_out = a.mass_out + b * a.stride;
    int32_t* pos_out = a.pos_out + b * a.stride;
    int32_t* kept = a.kept + (int64_t)b * keep;
    if (n <= keep) {
        for (int p = tid; p < keep; p += EV_THREADS) {
            kept[p] = p < n ? p : -1;
            if (p < n) {
                if (mass_out != mass) mass_out[p] = mass[p];
                if (pos_out != pos) pos_out[p] = pos[p];
            }
        }
        if (tid == 0) { a.moves[b] = 0; a.len_out[b] = n; }
        return;
    }
    const int64_t recent = (int64_t)a.seq_len[b] - a.recent;
    const bool cached = n <= EV_BLOCK;
    // the keep-th largest key, a digit at a time: `prefix` its digits so far, `more` of the keys that share them to keep
    uint32_t prefix = 0u, more = (uint32_t)keep;
    for (int i = tid; i < EV_BINS; i += EV_THREADS) s_hist[i] = 0u;
    __syncthreads();
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        const bool again = pass > 0 && cached;
        for (int64_t p0 = tid; p0 < n; p0 += EV_THREADS * EV_AHEAD) {
            uint32_t key[EV_AHEAD];
            if (again) {
#pragma unroll
                for (int e = 0; e < EV_AHEAD; ++e) key[e] = s_key[(p0 + e * EV_THREADS) & (EV_BLOCK - 1)];
            } else {
                int32_t q[EV_AHEAD];
                float m[EV_AHEAD];
#pragma unroll
                for (int e = 0; e < EV_AHEAD; ++e) {
                    const int64_t p = p0 + e * EV_THREADS < n ? p0 + e * EV_THREADS : p0;
                    q[e] = pos[p];
                    m[e] = mass[p];
                }
#pragma unroll
                for (int e = 0; e < EV_AHEAD; ++e) {
                    key[e] = q[e] < a.first || q[e] >= recent ? EV_SAFE : mass_key(m[e]);
                    if (cached && p0 + e * EV_THREADS < n) s_key[p0 + e * EV_THREADS] = key[e];
                }
            }
#pragma unroll
            for (int e = 0; e < EV_AHEAD; ++e)
                if (p0 + e * EV_THREADS < n && (pass == 0 || (key[e] >> (shift + bits)) == prefix))
                    atomicAdd(&s_hist[(key[e] >> shift) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // from the top: thread t holds bins 2 (1023 - t) and the one above
        const int hi = EV_BINS - 1 - 2 * tid;
        const uint32_t h1 = s_hist[hi], h0 = s_hist[hi - 1];
        s_hist[hi] = s_hist[hi - 1] = 0u;
        uint32_t all;
        const uint32_t above = sum_before(h1 + h0, s_wave, tid, all);
        if (above < more && above + h1 >= more) { s_bin = (uint32_t)hi; s_more = more - above; }
        else if (above + h1 < more && above + h1 + h0 >= more) { s_bin = (uint32_t)(hi - 1); s_more = more - above - h1; }
        __syncthreads();
        prefix = (prefix << bits) | s_bin;
        more = s_more;
    }
    // places stay whose key is larger, and the first `more` of those whose key is equal
    uint32_t equal = 0, holes = 0, fills = 0;
    for (int64_t p0 = 0; p0 < n; p0 += EV_BLOCK) {
        const int words = (int)std::min<int64_t>(EV_WORDS, (n - p0 + 63) / 64);
        for (int w = wave; w < words; w += EV_WAVES) {
            const int64_t p = p0 + w * 64 + lane;
            uint32_t key = 0u;
            if (p < n) {
                if (cached) {
                    key = s_key[p & (EV_BLOCK - 1)];
                } else {
                    const int q = pos[p];
                    key = q < a.first || q >= recent ? EV_SAFE : mass_key(mass[p]);
                }
            }
            const uint64_t gt = __builtin_amdgcn_ballot_w64(p < n && key > prefix), eq = __builtin_amdgcn_ballot_w64(p < n && key == prefix);
            if (lane == 0) { s_stay[w] = gt; s_equal[w] = eq; }
        }
        __syncthreads();
        uint32_t all;
        const uint64_t eq = tid < words ? s_equal[tid] : 0ull;
        const uint32_t before = equal + sum_before((uint32_t)__builtin_popcountll(eq), s_wave, tid, all);
        equal += all;
        const int p = (int)p0 + tid * 64;
        uint64_t stay = 0ull;
        if (tid < words) {
            stay = s_stay[tid] | (before < more ? lowest(eq, (int)(more - before)) : 0ull);
            s_stay[tid] = stay;
        }
        const uint64_t front = tid < words ? below(p, keep) : 0ull;
        const uint32_t own = (uint32_t)__builtin_popcountll(front & ~stay) | (uint32_t)__builtin_popcountll(stay & ~front) << 16;
        const uint32_t off = sum_before(own, s_wave, tid, all);
        if (tid < words) s_off[tid] = off;
        __syncthreads();
        for (int w = wave; w < words; w += EV_WAVES) {
            const int q = (int)p0 + w * 64 + lane;
            const uint64_t st = s_stay[w], fr = below((int)p0 + w * 64, keep), hm = fr & ~st, fm = st & ~fr;
            const uint32_t o = s_off[w];
            if ((hm >> lane) & 1) a.holes[(int64_t)b * a.holes_max + holes + (o & 0xFFFFu) + bits_below(hm)] = q;
            if ((fm >> lane) & 1) a.fills[(int64_t)b * a.holes_max + fills + (o >> 16) + bits_below(fm)] = q;
            if ((fr & st) >> lane & 1) {
                kept[q] = q;
                if (mass_out != mass) mass_out[q] = mass[q];
                if (pos_out != pos) pos_out[q] = pos[q];
            }
        }
        holes += all & 0xFFFFu;
        fills += all >> 16;
    }
    if (tid == 0) { a.moves[b] = (int32_t)holes; a.len_out[b] = keep; }
}

constexpr int EM_ROWS = 32;                          // rows that a workgroup moves

__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs a, int per_seq, int chunks) {
    __shared__ const char* s_from[EM_ROWS];
    __shared__ char* s_to[EM_ROWS];
    const int64_t id = block_number();
    const int b = (int)(id / per_seq), x0 = (int)(id - (int64_t)b * per_seq) * EM_ROWS, tid = threadIdx.x;
    if (b >= a.B) return;
    const int rows = std::min(EM_ROWS, a.moves[b] - x0);
    if (rows <= 0) return;
    if (tid < rows) {
        const int to = a.holes[(int64_t)b * a.holes_max + x0 + tid], from = a.fills[(int64_t)b * a.holes_max + x0 + tid];
        a.kept[(int64_t)b * a.keep + to] = from;
        a.mass_out[b * a.stride + to] = a.mass[b * a.stride + from];
        a.pos_out[b * a.stride + to] = a.pos[b * a.stride + from];
        const int sh = a.cache.page_shift, in = (1 << sh) - 1;
        const int32_t* table = a.page_table + (int64_t)b * a.max_pages;
        const int64_t pt = table[to >> sh], pf = table[from >> sh], row = (int64_t)chunks * 16;
        s_from[tid] = pf >= 0 && pf < a.cache.n_pages ? a.cache.rows + ((pf << sh) + (from & in)) * row : nullptr;
        s_to[tid] = pt >= 0 && pt < a.cache.n_pages ? a.cache.rows + ((pt << sh) + (to & in)) * row : nullptr;
    }
    __syncthreads();
    for (int u = tid; u < rows * chunks; u += 256) {
        const int r = u / chunks, c = u - r * chunks;
        u32x4 v = {0u, 0u, 0u, 0u};
        if (s_from[r]) v = *(const u32x4*)(s_from[r] + 16 * c);
        if (s_to[r]) *(u32x4*)(s_to[r] + 16 * c) = v;
    }
}

}  // namespace

int launch_latent_evict(const EvictArgs& a, void* stream) {
    if (a.B == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    {
        KernelTimer kt_("evict_select", st);
        evict_select_kernel<<<grid_of(a.B), dim3(EV_THREADS), 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    if (a.holes_max == 0) return 0;
    const int per = (int)((a.holes_max + EM_ROWS - 1) / EM_ROWS);
    const int chunks = (a.cache.rank + a.cache.rot) * (a.cache.dtype == ORDERMOE_BF16 ? 2 : 4) / 16;
    KernelTimer kt_("evict_move", st);
    evict_move_kernel<<<grid_of((int64_t)a.B * per), dim3(256), 0, st>>>(a, per, chunks);
    return (int)hipGetLastError();
}

}  // namespace ordermoe
