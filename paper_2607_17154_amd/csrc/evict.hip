// Sequences of the latent cache cut to a budget of tokens.
//
//   evict_select_kernel  one workgroup per sequence: the keys of its places (mass, or above
//                        all masses where the token is protected) in registers, the keep-th
//                        largest by three histograms of their bits, then the places that
//                        stay, go or move
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
constexpr int EV_KEYS = 32;                          // keys a thread holds
constexpr int EV_BLOCK = EV_THREADS * EV_KEYS;       // places whose keys the registers hold
static_assert(EV_KEYS * EV_WAVES <= EV_THREADS && EV_KEYS <= 32, "a count a thread, a bit a key");
constexpr int EV_BITS = 11, EV_BINS = 1 << EV_BITS;  // of a histogram; shifts 21, 10 and (10 bits) 0
constexpr uint32_t EV_SAFE = 0xFFFFFFFFu;

// a mass as an integer of the same order; NaN below all
__device__ inline uint32_t mass_key(float m) {
    if (m != m) return 0u;
    const uint32_t u = __float_as_uint(m + 0.0f);    // (-0 as 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Scan {
    uint32_t cnt[EV_THREADS], wave[EV_WAVES];
};
// cnt[] becomes the sum before each entry; returns the sum of all
__device__ inline uint32_t scan(Scan& s, int tid) {
    __syncthreads();
    const int lane = tid & 63;
    const uint32_t own = s.cnt[tid];
    uint32_t inc = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(inc, o);
        if (lane >= o) inc += v;
    }
    if (lane == 63) s.wave[tid >> 6] = inc;
    __syncthreads();
    uint32_t base = 0, all = 0;
#pragma unroll
    for (int w = 0; w < EV_WAVES; ++w) {
        base += w < (tid >> 6) ? s.wave[w] : 0u;
        all += s.wave[w];
    }
    s.cnt[tid] = base + inc - own;
    __syncthreads();
    return all;
}
__device__ inline uint32_t lanes_below(uint64_t m) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const EvictArgs a) {
    __shared__ uint32_t s_hist[EV_BINS];
    __shared__ Scan s_a, s_b;
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
    const int blocks = (n + EV_BLOCK - 1) / EV_BLOCK;
    uint32_t key[EV_KEYS];
    auto load = [&](int p0) {
#pragma unroll
        for (int j = 0; j < EV_KEYS; ++j) {
            key[j] = 0u;
            if (p0 + j * EV_THREADS >= n) continue;
            const int p = p0 + j * EV_THREADS + tid;
            if (p < n) {
                const int q = pos[p];
                key[j] = q < a.first || q >= recent ? EV_SAFE : mass_key(mass[p]);
            }
        }
    };
    if (blocks == 1) load(0);
    // the keep-th largest key, a digit at a time: `prefix` its digits so far, `more` of the keys that share them to keep
    uint32_t prefix = 0u, more = (uint32_t)keep;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : EV_BITS;
        for (int i = tid; i < EV_BINS; i += EV_THREADS) s_hist[i] = 0u;
        __syncthreads();
        for (int k = 0; k < blocks; ++k) {
            const int p0 = k * EV_BLOCK;
            if (blocks > 1) load(p0);
#pragma unroll
            for (int j = 0; j < EV_KEYS; ++j) {
                if (p0 + j * EV_THREADS >= n) continue;
                const bool in = p0 + j * EV_THREADS + tid < n && (pass == 0 || (key[j] >> (shift + bits)) == prefix);
                if (in) atomicAdd(&s_hist[(key[j] >> shift) & ((1u << bits) - 1u)], 1u);
            }
        }
        __syncthreads();
        // from the top: thread t holds bins 2 (1023 - t) and the one above
        const int hi = EV_BINS - 1 - 2 * tid;
        const uint32_t h1 = s_hist[hi], h0 = s_hist[hi - 1];
        s_a.cnt[tid] = h1 + h0;
        scan(s_a, tid);
        const uint32_t above = s_a.cnt[tid];
        if (above < more && above + h1 >= more) { s_bin = (uint32_t)hi; s_more = more - above; }
        else if (above + h1 < more && above + h1 + h0 >= more) { s_bin = (uint32_t)(hi - 1); s_more = more - above - h1; }
        __syncthreads();
        prefix = (prefix << bits) | s_bin;
        more = s_more;
        __syncthreads();
    }
    // places stay whose key is larger, and the first `more` of those whose key is equal
    uint32_t equal = 0, holes = 0, fills = 0;
    for (int k = 0; k < blocks; ++k) {
        const int p0 = k * EV_BLOCK;
        if (blocks > 1) load(p0);
        s_a.cnt[tid] = 0u;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < EV_KEYS; ++j) {
            if (p0 + j * EV_THREADS >= n) continue;
            const uint64_t m = __builtin_amdgcn_ballot_w64(p0 + j * EV_THREADS + tid < n && key[j] == prefix);
            if (lane == 0) s_a.cnt[j * EV_WAVES + wave] = (uint32_t)__builtin_popcountll(m);
        }
        const uint32_t eq_all = scan(s_a, tid);
        uint32_t stay_bits = 0;
#pragma unroll
        for (int j = 0; j < EV_KEYS; ++j) {
            if (p0 + j * EV_THREADS >= n) continue;
            const int p = p0 + j * EV_THREADS + tid;
            const bool eq = p < n && key[j] == prefix;
            const uint64_t m = __builtin_amdgcn_ballot_w64(eq);
            const bool stay = p < n && (key[j] > prefix || (eq && equal + s_a.cnt[j * EV_WAVES + wave] + lanes_below(m) < more));
            stay_bits |= (uint32_t)stay << j;
        }
        equal += eq_all;
        __syncthreads();                             // s_a has been read
        s_a.cnt[tid] = 0u;
        s_b.cnt[tid] = 0u;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < EV_KEYS; ++j) {
            if (p0 + j * EV_THREADS >= n) continue;
            const int p = p0 + j * EV_THREADS + tid;
            const bool stay = (stay_bits >> j) & 1;
            const uint64_t hm = __builtin_amdgcn_ballot_w64(p < keep && !stay), fm = __builtin_amdgcn_ballot_w64(p >= keep && stay);
            if (lane == 0) {
                s_a.cnt[j * EV_WAVES + wave] = (uint32_t)__builtin_popcountll(hm);
                s_b.cnt[j * EV_WAVES + wave] = (uint32_t)__builtin_popcountll(fm);
            }
        }
        const uint32_t h_all = scan(s_a, tid), f_all = scan(s_b, tid);
#pragma unroll
        for (int j = 0; j < EV_KEYS; ++j) {
            if (p0 + j * EV_THREADS >= n) continue;
            const int p = p0 + j * EV_THREADS + tid;
            const bool stay = (stay_bits >> j) & 1, hole = p < keep && !stay, fill = p >= keep && stay;
            const uint64_t hm = __builtin_amdgcn_ballot_w64(hole), fm = __builtin_amdgcn_ballot_w64(fill);
            if (hole) a.holes[(int64_t)b * a.holes_max + holes + s_a.cnt[j * EV_WAVES + wave] + lanes_below(hm)] = p;
            if (fill) a.fills[(int64_t)b * a.holes_max + fills + s_b.cnt[j * EV_WAVES + wave] + lanes_below(fm)] = p;
            if (p < keep && stay) {
                kept[p] = p;
                if (mass_out != mass) mass_out[p] = mass[p];
                if (pos_out != pos) pos_out[p] = pos[p];
            }
        }
        holes += h_all;
        fills += f_all;
        __syncthreads();
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
