// C ABI entry points of the latent and prompt attention and of the eviction:
// validation, workspace carving and kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "common.hpp"

namespace ordermoe {
namespace {

constexpr int64_t INT_LIMIT = (int64_t)1 << 31;
// (scores are taken in units of log 2: the factor has to be finite too)
bool good_scale(float scale) { return std::isfinite(scale * 1.44269504f); }

int hip_fail(int e, const char* where) {
    return fail(ORDERMOE_EHIP, std::string(where) + ": " + hipGetErrorString((hipError_t)e));
}
int bad(const std::string& who, const char* what) { return fail(ORDERMOE_EINVAL, who + ": " + what); }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool good16(const void* p) { return p && aligned16(p); }

int check_cache(const ordermoe_latent_cache* C, const std::string& who) {
    if (!C) return bad(who, "null cache");
    if (C->dtype != ORDERMOE_F32 && C->dtype != ORDERMOE_BF16) return fail(ORDERMOE_EDTYPE, who + ": dtype");
    if (C->rank != 128 && C->rank != 256 && C->rank != 512) return bad(who, "rank must be 128, 256 or 512");
    if (C->rotary_dim != 32 && C->rotary_dim != 64) return bad(who, "rotary_dim must be 32 or 64");
    if (C->page_size < 16 || C->page_size > 1024 || (C->page_size & (C->page_size - 1)))
        return bad(who, "page_size must be a power of two from 16 to 1024");
    if (C->n_pages < 1 || C->n_pages >= INT_LIMIT) return bad(who, "n_pages out of range");
    if (!good16(C->rows)) return bad(who, "rows must be 16-byte aligned");
    return ORDERMOE_OK;
}
int check_heads(const ordermoe_latent_heads* H, const std::string& who) {
    if (!H) return bad(who, "null heads");
    if (H->n_q < 1 || H->n_q > 128) return bad(who, "n_q must lie in [1, 128]");
    if (H->head_dim != 64 && H->head_dim != 128) return bad(who, "head_dim must be 64 or 128");
    if (!good16(H->w_k) || !good16(H->w_v)) return bad(who, "w_k and w_v must be 16-byte aligned");
    return ORDERMOE_OK;
}
int check_table(const ordermoe_latent_cache* C, int32_t B, int32_t max_pages, const std::string& who) {
    if (B < 0 || B > 65535) return bad(who, "B must lie in [0, 65535]");
    if (max_pages < 1 || (int64_t)max_pages * C->page_size > (int64_t)1 << 30)
        return bad(who, "max_pages * page_size must lie in [1, 2^30]");
    return ORDERMOE_OK;
}

LatentArgs cache_args(const ordermoe_latent_cache* C) {
    return LatentArgs{C->dtype, C->rank, C->rotary_dim, __builtin_ctz((unsigned)C->page_size), C->n_pages, (char*)C->rows};
}

int check_attention(const ordermoe_latent_cache* C, const ordermoe_latent_heads* H, int32_t B, int32_t max_q, int32_t max_pages,
                    const std::string& who) {
    int rc = check_cache(C, who);
    if (rc || (rc = check_heads(H, who)) || (rc = check_table(C, B, max_pages, who))) return rc;
    if (max_q < 1 || max_q > ORDERMOE_MAX_DRAFT)
        return fail(ORDERMOE_EINVAL, who + ": max_q must lie in [1, " + std::to_string(ORDERMOE_MAX_DRAFT) + "]");
    return ORDERMOE_OK;
}
// Each workspace is carved by the call's own sizes; its size function asks for the most that a call of the same or of smaller
// sizes carves, so that one buffer serves them all.
int64_t attention_rows(const ordermoe_latent_cache* C, const ordermoe_latent_heads* H, int32_t B, int32_t max_q, int32_t max_pages) {
    return latent_items(C->dtype, H->n_q, B, max_q, (int64_t)max_pages * C->page_size) * max_q * H->n_q;
}
size_t attention_ws(const ordermoe_latent_cache* C, const ordermoe_latent_heads* H, int32_t B, int32_t max_q, int32_t max_pages,
                    int64_t parts, bool weighs, Carver& c, LatentAttentionArgs* a) {
    const size_t rows = (size_t)max_q * H->n_q;
    int32_t* pl = c.take<int32_t>((size_t)std::max(B, 1) * 2);
    float* ml = c.take<float>((size_t)parts * 2);
    float* po = c.take<float>((size_t)parts * C->rank);
    float* st = c.take<float>(weighs ? B * rows * 2 : 0);
    float* sc = c.take<float>(weighs ? B * rows * max_pages * C->page_size : 0);
    if (a) { a->items = parts / (int64_t)rows; a->plan = pl; a->part_ml = ml; a->part_o = po; a->stat = st; a->score = sc; }
    return c.size();
}

// rows of a sequence that move at most, out of the places past the budget into those before it
int64_t evict_moves(int64_t cap, int32_t keep) { return std::max<int64_t>(0, std::min<int64_t>(keep, cap - keep)); }
size_t evict_ws(const ordermoe_latent_cache* C, int32_t B, int32_t max_pages, int64_t most, Carver& c, EvictArgs* a) {
    const int64_t cap = (int64_t)max_pages * C->page_size;
    int32_t* m = c.take<int32_t>((size_t)std::max(B, 1));
    int32_t* h = c.take<int32_t>((size_t)B * most);
    int32_t* f = c.take<int32_t>((size_t)B * most);
    // (one taking for the three of them: the sizes go with the places that there are, which may be fewer than the table's)
    uint32_t* w = c.take<uint32_t>((size_t)B * evict_slice_words(cap));
    if (a) {
        a->moves = m; a->holes = h; a->fills = f; a->holes_max = most;
        const size_t slices = (size_t)evict_slices(cap);
        a->part = w; a->above = w + 3 * (size_t)B * slices * 2048; a->found = a->above + 2 * (size_t)B * slices;
    }
    return c.size();
}

int check_prompt(int32_t dtype, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t rotary_dim, int64_t T, int32_t B,
                 const std::string& who) {
    if (dtype != ORDERMOE_F32 && dtype != ORDERMOE_BF16) return fail(ORDERMOE_EDTYPE, who + ": dtype");
    if (n_kv < 1 || n_q < 1 || n_q > 1024 || n_q % n_kv != 0) return bad(who, "n_q must be a multiple of n_kv, at most 1024");
    if (head_dim != 64 && head_dim != 128) return bad(who, "head_dim must be 64 or 128");
    if (rotary_dim != 0 && rotary_dim != 32 && rotary_dim != 64) return bad(who, "rotary_dim must be 0, 32 or 64");
    if (B < 0 || B > 65535) return bad(who, "B must lie in [0, 65535]");
    if (T < 0 || T > (INT_LIMIT - 1) / n_q) return bad(who, "T * n_q must lie in [0, 2^31)");
    return ORDERMOE_OK;
}
size_t prompt_ws(int32_t head_dim, int64_t rows, Carver& c, PromptArgs* a) {
    float* ml = c.take<float>((size_t)rows * 2);
    float* po = c.take<float>((size_t)rows * head_dim);
    if (a) { a->part_ml = ml; a->part_o = po; }
    return c.size();
}

}  // namespace
}  // namespace ordermoe

using namespace ordermoe;

extern "C" int ordermoe_latent_write(const ordermoe_latent_cache* C, const ordermoe_latent_heads* H, const void* q, int64_t q_stride,
                                     const void* kv, int64_t kv_stride, int64_t T, const int32_t* pos, const int64_t* slots,
                                     int32_t absorb, void* q_out, void* stream) {
    const char* who = "latent_write";
    int rc = check_cache(C, who);
    if (rc || (rc = check_heads(H, who))) return rc;
    if (absorb != 0 && absorb != 1) return bad(who, "absorb must be 0 or 1");
    if (H->interleaved != 0 && H->interleaved != 1) return bad(who, "interleaved must be 0 or 1");
    if (!(H->eps >= 0.0f) || std::isinf(H->eps)) return bad(who, "eps must be finite and >= 0");
    if ((H->norm && !aligned16(H->norm)) || (H->cos_sin && !aligned16(H->cos_sin)))
        return bad(who, "norm and cos_sin must be 16-byte aligned");
    if (T < 0 || T > (INT_LIMIT - 1) / H->n_q) return bad(who, "T * n_q must lie in [0, 2^31)");
    if (H->cos_sin && (H->max_pos < 1 || (T > 0 && !pos))) return bad(who, "rotation needs max_pos >= 1 and pos");
    if (T > 0 && (!good16(kv) || !slots || (q && (!aligned16(q) || !good16(q_out)))))
        return bad(who, "kv, slots, and q_out with q, are needed; q, kv and q_out 16-byte aligned");
    const int64_t per = C->dtype == ORDERMOE_BF16 ? 8 : 4;         // elements of 16 bytes
    if (kv_stride < C->rank + C->rotary_dim || kv_stride % per ||
        (q && (q_stride < (int64_t)H->n_q * (H->head_dim + C->rotary_dim) || q_stride % per)))
        return bad(who, "strides must hold a token's elements and be multiples of 16 bytes");
    LatentWriteArgs a{};
    a.cache = cache_args(C);
    a.n_q = H->n_q; a.head_dim = H->head_dim; a.interleaved = H->interleaved; a.absorb = absorb;
    a.eps = H->eps; a.max_pos = H->max_pos; a.norm = H->norm; a.cos_sin = H->cos_sin; a.w_k = H->w_k;
    a.q = q; a.kv = kv; a.q_stride = q_stride; a.kv_stride = kv_stride; a.T = T; a.pos = pos; a.slots = slots; a.q_out = q_out;
    const int e = launch_latent_write(a, stream);
    if (e) return hip_fail(e, "latent_write launch");
    clear_error();
    return ORDERMOE_OK;
}

extern "C" size_t ordermoe_latent_attention_workspace_size(const ordermoe_latent_cache* C, const ordermoe_latent_heads* H, int32_t B,
                                                           int32_t max_q, int32_t max_pages, int32_t weighs) {
    if (check_attention(C, H, B, max_q, max_pages, "latent_attention") != ORDERMOE_OK) return 0;
    int64_t parts = 0;
    for (int32_t q = 1; q <= max_q; ++q) parts = std::max(parts, attention_rows(C, H, B, q, max_pages));
    Carver c(nullptr);
    return attention_ws(C, H, B, max_q, max_pages, parts, weighs != 0, c, nullptr);
}

extern "C" int ordermoe_latent_attention(const ordermoe_latent_cache* C, const ordermoe_latent_heads* H, const void* q, int64_t T,
                                         int32_t B, int32_t max_q, const int32_t* q_start, const int32_t* ctx_len,
                                         const int32_t* page_table, int32_t max_pages, const uint64_t* tree, float scale, void* out,
                                         float* lse, const float* mass, float* mass_out, int64_t mass_stride, float decay, void* ws,
                                         size_t ws_bytes, void* stream) {
    const char* who = "latent_attention";
    const int rc = check_attention(C, H, B, max_q, max_pages, who);
    if (rc) return rc;
    if (T < 0 || T > (INT_LIMIT - 1) / H->n_q) return bad(who, "T * n_q must lie in [0, 2^31)");
    if (!good_scale(scale) || !std::isfinite(decay)) return bad(who, "scale (times log2 e) and decay must be finite");
    if (T > 0 && B > 0 && (!good16(q) || !q_start || !ctx_len || !page_table || !good16(out)))
        return bad(who, "null pointer, or q or out not 16-byte aligned");
    if (mass_out ? mass_stride < 1 || (B > 0 && mass_stride > ((int64_t)1 << 40) / B) : mass != nullptr)
        return bad(who, "mass_stride must lie in [1, 2^40 / B] where mass_out is given; mass needs mass_out");
    const int64_t parts = attention_rows(C, H, B, max_q, max_pages);
    Carver sized(nullptr);
    const size_t need = attention_ws(C, H, B, max_q, max_pages, parts, mass_out != nullptr, sized, nullptr);
    if (!ws || ws_bytes < need) return fail(ORDERMOE_EWORKSPACE, std::string(who) + ": workspace needs " + std::to_string(need) + " bytes");
    LatentAttentionArgs a{};
    a.cache = cache_args(C);
    a.n_q = H->n_q; a.head_dim = H->head_dim; a.B = B; a.max_q = max_q; a.max_pages = max_pages; a.T = T;
    a.q = q; a.w_v = H->w_v; a.q_start = q_start; a.ctx_len = ctx_len; a.page_table = page_table; a.tree = tree;
    a.scale = scale; a.decay = decay; a.out = out; a.lse = lse; a.mass = mass; a.mass_out = mass_out; a.mass_stride = mass_stride;
    Carver c(ws);
    attention_ws(C, H, B, max_q, max_pages, parts, mass_out != nullptr, c, &a);
    const int e = launch_latent_attention(a, stream);
    if (e) return hip_fail(e, "latent_attention launch");
    clear_error();
    return ORDERMOE_OK;
}

extern "C" int ordermoe_latent_expand(const ordermoe_latent_cache* C, const ordermoe_latent_heads* H, const int64_t* slots, int64_t n,
                                      void* k_out, void* r_out, void* v_out, void* stream) {
    const char* who = "latent_expand";
    int rc = check_cache(C, who);
    if (rc || (rc = check_heads(H, who))) return rc;
    if (n < 0 || n > (INT_LIMIT - 1) / H->n_q) return bad(who, "n * n_q must lie in [0, 2^31)");
    if (n > 0 && (!slots || !good16(k_out) || !good16(r_out) || !good16(v_out)))
        return bad(who, "null pointer, or an output not 16-byte aligned");
    LatentExpandArgs a{};
    a.cache = cache_args(C);
    a.n_q = H->n_q; a.head_dim = H->head_dim; a.w_k = H->w_k; a.w_v = H->w_v;
    a.slots = slots; a.n = n; a.k_out = k_out; a.r_out = r_out; a.v_out = v_out;
    const int e = launch_latent_expand(a, stream);
    if (e) return hip_fail(e, "latent_expand launch");
    clear_error();
    return ORDERMOE_OK;
}

extern "C" size_t ordermoe_prompt_attention_workspace_size(int32_t dtype, int32_t n_q, int32_t n_kv, int32_t head_dim,
                                                           int32_t rotary_dim, int64_t T, int32_t B) {
    if (check_prompt(dtype, n_q, n_kv, head_dim, rotary_dim, T, B, "prompt_attention") != ORDERMOE_OK) return 0;
    Carver c(nullptr);
    return prompt_ws(head_dim, prompt_rows_at_most(n_q, n_kv, T), c, nullptr);
}

extern "C" int ordermoe_prompt_attention(int32_t dtype, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t rotary_dim, const void* q,
                                         int64_t T, const void* k, const void* r, const void* v, int64_t L, int32_t B,
                                         const int32_t* q_start, const int32_t* kv_start, float scale, void* out, float* lse, void* ws,
                                         size_t ws_bytes, void* stream) {
    const char* who = "prompt_attention";
    const int rc = check_prompt(dtype, n_q, n_kv, head_dim, rotary_dim, T, B, who);
    if (rc) return rc;
    // (the kernel counts positions in 32 bits and looks up to two tiles of 64 past the last one)
    if (L < 0 || L > INT_LIMIT - 128) return bad(who, "L must lie in [0, 2^31 - 128]");
    if (!good_scale(scale)) return bad(who, "scale (times log2 e) must be finite");
    if (T > 0 && B > 0 && (!good16(q) || !q_start || !kv_start || !good16(out) ||
                           (L > 0 && (!good16(k) || !good16(v) || (rotary_dim > 0 && !good16(r))))))
        return bad(who, "null pointer, or q, k, r, v or out not 16-byte aligned");
    const int64_t pieces = prompt_pieces(n_q, n_kv, T, B), rows = pieces > 1 ? pieces * T * n_q : 0;
    Carver sized(nullptr);
    const size_t need = prompt_ws(head_dim, rows, sized, nullptr);
    if (need > 0 && (!ws || ws_bytes < need))
        return fail(ORDERMOE_EWORKSPACE, std::string(who) + ": workspace needs " + std::to_string(need) + " bytes");
    PromptArgs a{};
    a.dtype = dtype; a.n_q = n_q; a.n_kv = n_kv; a.head_dim = head_dim; a.rot = rotary_dim; a.B = B;
    a.q = q; a.k = k; a.r = r; a.v = v; a.T = T; a.L = L; a.q_start = q_start; a.kv_start = kv_start;
    a.scale = scale; a.out = out; a.lse = lse;
    Carver c(ws);
    prompt_ws(head_dim, rows, c, &a);
    const int e = launch_prompt_attention(a, stream);
    if (e) return hip_fail(e, "prompt_attention launch");
    clear_error();
    return ORDERMOE_OK;
}

extern "C" size_t ordermoe_latent_evict_workspace_size(const ordermoe_latent_cache* C, int32_t B, int32_t max_pages, int32_t keep) {
    const char* who = "latent_evict";
    if (check_cache(C, who) != ORDERMOE_OK || check_table(C, B, max_pages, who) != ORDERMOE_OK) return 0;
    if (keep < 1) { bad(who, "keep must be at least 1"); return 0; }
    const int64_t cap = (int64_t)max_pages * C->page_size;
    Carver c(nullptr);
    return evict_ws(C, B, max_pages, std::min<int64_t>(keep, cap / 2), c, nullptr);      // (the most moves of any budget up to keep)
}

extern "C" int ordermoe_latent_evict(const ordermoe_latent_cache* C, int32_t B, const int32_t* ctx_len, const int32_t* seq_len,
                                     const int32_t* page_table, int32_t max_pages, int32_t keep, int32_t first, int32_t recent,
                                     const float* mass, const int32_t* pos, int64_t stride, int32_t* kept, int32_t* len_out,
                                     float* mass_out, int32_t* pos_out, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "latent_evict";
    int rc = check_cache(C, who);
    if (rc || (rc = check_table(C, B, max_pages, who))) return rc;
    if (keep < 1 || first < 0 || recent < 0 || (int64_t)first + recent > keep)
        return bad(who, "keep must be at least 1, first and recent at least 0 and no more than keep together");
    if (stride < 1 || (B > 0 && (stride > ((int64_t)1 << 40) / B || keep > ((int64_t)1 << 40) / B)))
        return bad(who, "stride must be at least 1, B * stride and B * keep at most 2^40");
    if (B > 0 && (!ctx_len || !seq_len || !page_table || !mass || !pos || !kept || !len_out || !mass_out || !pos_out))
        return bad(who, "null pointer");
    const int64_t most = evict_moves((int64_t)max_pages * C->page_size, keep);
    Carver sized(nullptr);
    const size_t need = evict_ws(C, B, max_pages, most, sized, nullptr);
    if (!ws || ws_bytes < need) return fail(ORDERMOE_EWORKSPACE, std::string(who) + ": workspace needs " + std::to_string(need) + " bytes");
    EvictArgs a{};
    a.cache = cache_args(C);
    a.B = B; a.max_pages = max_pages; a.keep = keep; a.first = first; a.recent = recent;
    a.ctx_len = ctx_len; a.seq_len = seq_len; a.page_table = page_table; a.mass = mass; a.pos = pos; a.stride = stride;
    a.kept = kept; a.len_out = len_out; a.mass_out = mass_out; a.pos_out = pos_out;
    Carver c(ws);
    evict_ws(C, B, max_pages, most, c, &a);
    const int e = launch_latent_evict(a, stream);
    if (e) return hip_fail(e, "latent_evict launch");
    clear_error();
    return ORDERMOE_OK;
}
