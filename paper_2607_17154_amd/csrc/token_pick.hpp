// The token stage of the routing: top-k, gates, margin and server-expert selection of
// one token by 16 lanes (one DPP row).  The layer kernel for a few tokens shares the
// order of logits, the reductions and the result, and makes the same decisions in loops.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.hpp"

namespace ordermoe {

// order-preserving map of fp32 onto uint32
__device__ inline uint32_t f2ord(float v) {
    uint32_t u = __float_as_uint(v);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ inline float ord2f(uint32_t o) {
    uint32_t u = (o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o;
    return __uint_as_float(u);
}

// Reductions over each row of 16 lanes (one token's lanes) with DPP row
// rotations by 8, 4, 2, 1: after the four steps every lane of the row holds
// the result.  Max and min are exact in any order; of a float sum of several
// terms only lane 0's is used.
template <int CTRL>
__device__ inline uint32_t dpp_u32(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ inline uint64_t dpp_u64(uint64_t v) {
    const uint32_t lo = dpp_u32<CTRL>((uint32_t)v), hi = dpp_u32<CTRL>((uint32_t)(v >> 32));
    return ((uint64_t)hi << 32) | lo;
}
constexpr int DPP_ROR8 = 0x128, DPP_ROR4 = 0x124, DPP_ROR2 = 0x122, DPP_ROR1 = 0x121;
__device__ inline uint32_t row_max_u32(uint32_t v) {
    uint32_t o;
    o = dpp_u32<DPP_ROR8>(v); v = o > v ? o : v;
    o = dpp_u32<DPP_ROR4>(v); v = o > v ? o : v;
    o = dpp_u32<DPP_ROR2>(v); v = o > v ? o : v;
    o = dpp_u32<DPP_ROR1>(v); v = o > v ? o : v;
    return v;
}
__device__ inline uint32_t row_min_u32(uint32_t v) {
    uint32_t o;
    o = dpp_u32<DPP_ROR8>(v); v = o < v ? o : v;
    o = dpp_u32<DPP_ROR4>(v); v = o < v ? o : v;
    o = dpp_u32<DPP_ROR2>(v); v = o < v ? o : v;
    o = dpp_u32<DPP_ROR1>(v); v = o < v ? o : v;
    return v;
}
__device__ inline uint64_t row_min_u64(uint64_t v) {
    uint64_t o;
    o = dpp_u64<DPP_ROR8>(v); v = o < v ? o : v;
    o = dpp_u64<DPP_ROR4>(v); v = o < v ? o : v;
    o = dpp_u64<DPP_ROR2>(v); v = o < v ? o : v;
    o = dpp_u64<DPP_ROR1>(v); v = o < v ? o : v;
    return v;
}
__device__ inline float row_sum_f32(float v) {
    v += __uint_as_float(dpp_u32<DPP_ROR8>(__float_as_uint(v)));
    v += __uint_as_float(dpp_u32<DPP_ROR4>(__float_as_uint(v)));
    v += __uint_as_float(dpp_u32<DPP_ROR2>(__float_as_uint(v)));
    v += __uint_as_float(dpp_u32<DPP_ROR1>(__float_as_uint(v)));
    return v;
}

// What the 16 lanes of a token find: lane j its slot j, every lane the rest.
struct TokenPick {
    int r, k, m;             // slot j: target, executed expert, execution server
    float v;                 // slot j: the target's logit
    float top, den;          // the largest logit, the gates' denominator: w = exp(v - top) / den
    float margin, qhat;      // margin, accumulated loss after the layer
    int first_m;             // slot 0's execution server
    uint32_t dstmask;        // remote servers of the token's slots
    bool loc_ok;             // the token's location is a server
};

// lg: the token's E logits; s_t1k, s_t1q [E][gmax], s_t1n, s_mask [E]: the candidate
// tables (in LDS or memory, as Stab [M][M][E]); s_loc, qhat_in: the token's location and
// loss so far.  Slots up to KM >= k.
template <int NBT, int KM>
__device__ inline TokenPick pick_token(const RouteArgs& a, const float* lg, const int32_t* s_t1k, const float* s_t1q,
                                       const int32_t* s_t1n, const uint32_t* s_mask, const float* Stab, int j, int s_loc,
                                       float qhat_in) {
    const int E = a.E, k = a.k, M = a.M;
    // top-(k+1) selection by (logit desc, index asc); this lane's logits (experts
    // j + 16 i) are read once and kept as order-preserving keys
    const int kk1 = (k + 1 < E) ? k + 1 : E;
    // (reads at clamped addresses and selects instead of branches, so that the
    // LDS reads issue together and no per-element branch splits the wave)
    // Each rank takes the row's largest key with 32-bit maxima, then the lowest
    // expert that has it (64-bit (logit, expert) keys took 900 cycles a rank, this
    // about 300); a taken key becomes 0, below every key in play (at least 1).
    uint32_t okey[NBT];
#pragma unroll
    for (int i = 0; i < NBT; ++i) {
        const int e = j + 16 * i;
        const uint32_t o = f2ord(lg[e < E ? e : E - 1]);
        okey[i] = e < E ? (o > 1u ? o : 1u) : 0u;
    }
    int sel_e[KM + 1];
    float sel_v[KM + 1];
#pragma unroll
    for (int r = 0; r < KM + 1; ++r) {
        if (r < kk1) {
            uint32_t mx = okey[0];
#pragma unroll
            for (int i = 1; i < NBT; ++i) mx = okey[i] > mx ? okey[i] : mx;
            mx = row_max_u32(mx);
            uint32_t e = 0xFFFFu;
#pragma unroll
            for (int i = NBT - 1; i >= 0; --i) e = okey[i] == mx ? (uint32_t)(j + 16 * i) : e;
            e = row_min_u32(e);
            sel_e[r] = (int)e;
            sel_v[r] = ord2f(mx);
#pragma unroll
            for (int i = 0; i < NBT; ++i) okey[i] = e == (uint32_t)(j + 16 * i) ? 0u : okey[i];
        }
    }
    float mg = __builtin_inff();
#pragma unroll
    for (int r = 0; r < KM; ++r) {
        if (r + 1 < kk1) {
            float gap = sel_v[r] - sel_v[r + 1];
            mg = gap < mg ? gap : mg;
        }
    }
    // gates: softmax renormalised over the top-k, or over all experts
    float den = 0.f;
    if (a.renorm) {
#pragma unroll
        for (int r = 0; r < KM; ++r)
            if (r < k) den += expf(sel_v[r] - sel_v[0]);
    } else {
        for (int e = j; e < E; e += 16) den += expf(lg[e] - sel_v[0]);
        // (the rotations add in another order in every lane: all take lane 0's sum)
        den = __shfl(row_sum_f32(den), 0, 16);
    }

    // server-expert selection.  Lane j holds candidate j of every slot: j = 0
    // the exact target, j >= 1 its (j-1)-th substitute in the LDS-staged table.
    // The search does not depend on the budget, so it runs for all slots at
    // once: each lane keeps, per slot, the smallest 64-bit key (J, position,
    // remote, server, expert) over the servers holding its expert.  Then the
    // slots are taken in rank order: the budget test of eq (40) masks the
    // substitutes, a min over the row picks (m*, k*) (eq 43) and the budget is
    // updated as eq (44).
    const bool loc_ok = s_loc < M;
    float qhat = qhat_in;
    const bool subs_on = a.allow_sub && a.Qbar > 0.f;
    const uint32_t mmask = M >= 32 ? 0xFFFFFFFFu : ((1u << M) - 1u);   // servers that exist
    const int jm1 = j >= 1 && j - 1 < a.gmax ? j - 1 : 0;    // (in the table's row; past its entries it is not used)
    int ke[KM];
    float qe[KM];
    uint32_t msv[KM];
    uint64_t key[KM];
    bool search[KM];
    // every slot's table reads are issued (slots past k read slot 0's entries,
    // discarded), then masked, so that no per-slot branch serialises them
#pragma unroll
    for (int slot = 0; slot < KM; ++slot) {
        const bool on = slot < k;
        const int r = sel_e[on ? slot : 0];
        const uint32_t rmask = s_mask[r];
        const int nsub = s_t1n[r];
        const int tk = s_t1k[r * a.gmax + jm1];
        const float tq = s_t1q[r * a.gmax + jm1];
        // uniform over the token's row: the reductions below read only lanes of the row
        search[slot] = on && loc_ok && !(a.pin && ((rmask >> s_loc) & 1u));
        const bool sub = j >= 1 && subs_on && j - 1 < nsub;
        int kc = j == 0 ? r : (sub ? tk : -1);
        if (!on || kc < 0 || kc >= E) kc = -1;
        ke[slot] = kc;
        qe[slot] = on && sub ? tq : 0.f;
        key[slot] = ~0ull;
    }
    // the servers holding each candidate (a substitute only on the token's
    // server in the Local Substitute Only mode)
    const uint32_t lmask = a.allow_sub == 2 && j >= 1 ? 1u << (s_loc & 31) : ~0u;
#pragma unroll
    for (int slot = 0; slot < KM; ++slot) {
        const uint32_t hm = s_mask[ke[slot] >= 0 ? ke[slot] : 0];
        msv[slot] = search[slot] && ke[slot] >= 0 ? hm & mmask & lmask : 0u;
    }
    // servers holding each candidate, one per round for every slot together
    for (;;) {
        uint32_t any = 0;
#pragma unroll
        for (int slot = 0; slot < KM; ++slot) any |= msv[slot];
        if (!__builtin_amdgcn_ballot_w64(any != 0)) break;
#pragma unroll
        for (int slot = 0; slot < KM; ++slot) {
            if (msv[slot]) {
                const int m = __builtin_ctz(msv[slot]);
                msv[slot] &= msv[slot] - 1;
                const float J = fmaf(a.cq, qe[slot], Stab[((int64_t)s_loc * M + m) * E + ke[slot]]);
                // J's order as a float (negative costs included; -0 counts as +0)
                const uint64_t cand = ((uint64_t)f2ord(J == 0.f ? 0.f : J) << 32) | ((uint32_t)j << 16) |
                                      ((uint32_t)(m != s_loc) << 15) | ((uint32_t)m << 8) |
                                      (uint32_t)ke[slot];
                key[slot] = cand < key[slot] ? cand : key[slot];
            }
        }
    }
    // Only the choice is serial over the slots; lane j keeps slot j's, and the
    // lanes write the token's slots together (lane 0 writing them one after the
    // other took 5.6 of 19 us at 64 tokens of 128 experts, top-8).
    int first_m = s_loc, my_r = 0, my_k = 0, my_m = s_loc;
    float my_v = 0.f;
    uint32_t dstmask = 0;
#pragma unroll
    for (int slot = 0; slot < KM; ++slot) {
        if (slot >= k) break;
        const int r = sel_e[slot];
        int km = r, mm = s_loc;
        float qsel = 0.f;
        if (search[slot]) {
            // eq (40): a substitute must fit the remaining budget; the exact target always does
            uint64_t kk = (j == 0 || qhat + qe[slot] <= a.Qbar) ? key[slot] : ~0ull;
            kk = row_min_u64(kk);
            const int pos = (int)((kk >> 16) & 15u);
            mm = (int)((kk >> 8) & 31u);
            km = (int)(kk & 0xFFu);
            // the chosen candidate's loss, from its lane (a sum of one term: exact)
            qsel = row_sum_f32(j == pos ? qe[slot] : 0.f);
        }
        qhat = qhat + qsel;
        if (slot == 0) first_m = mm;
        if (mm != s_loc) dstmask |= 1u << mm;
        if (j == slot) { my_r = r; my_k = km; my_m = mm; my_v = sel_v[slot]; }
    }
    TokenPick o;
    o.r = my_r; o.k = my_k; o.m = my_m;
    o.v = my_v; o.top = sel_v[0]; o.den = den;
    o.margin = mg; o.qhat = qhat;
    o.first_m = first_m; o.dstmask = dstmask; o.loc_ok = loc_ok;
    return o;
}

}  // namespace ordermoe
