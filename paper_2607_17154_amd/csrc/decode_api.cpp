// C ABI entry points of the decode-step operators: validation, workspace
// carving and kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "common.hpp"

namespace ordermoe {
namespace {

int hip_fail(int e, const char* where) {
    return fail(ORDERMOE_EHIP, std::string(where) + ": " + hipGetErrorString((hipError_t)e));
}
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_dtype(int32_t dtype, const char* who) {
    return dtype == ORDERMOE_F32 || dtype == ORDERMOE_BF16 ? ORDERMOE_OK : fail(ORDERMOE_EDTYPE, std::string(who) + ": dtype");
}

int check_cache(const ordermoe_cache* C) {
    if (!C) return fail(ORDERMOE_EINVAL, "cache: null");
    if (C->format != ORDERMOE_CACHE_INT8 && C->format != ORDERMOE_CACHE_FP8) return fail(ORDERMOE_EDTYPE, "cache: format");
    if (C->n_kv < 1 || C->n_kv > 1024) return fail(ORDERMOE_EINVAL, "cache: n_kv must lie in [1, 1024]");
    if (C->head_dim != 64 && C->head_dim != 128 && C->head_dim != 256)
        return fail(ORDERMOE_EINVAL, "cache: head_dim must be 64, 128 or 256");
    if (C->page_size < 16 || C->page_size > 1024 || (C->page_size & (C->page_size - 1)))
        return fail(ORDERMOE_EINVAL, "cache: page_size must be a power of two from 16 to 1024");
    if (C->n_pages < 1 || C->n_pages > ((int64_t)1 << 31) - 1) return fail(ORDERMOE_EINVAL, "cache: n_pages out of range");
    if (!C->k_codes || !C->v_codes || !C->k_scale || !C->v_scale) return fail(ORDERMOE_EINVAL, "cache: null pointer");
    if (!aligned16(C->k_codes) || !aligned16(C->v_codes) || !aligned16(C->k_scale) || !aligned16(C->v_scale))
        return fail(ORDERMOE_EINVAL, "cache: pointers must be 16-byte aligned");
    return ORDERMOE_OK;
}

CacheArgs cache_args(const ordermoe_cache* C) {
    CacheArgs c{};
    c.format = C->format; c.n_kv = C->n_kv; c.head_dim = C->head_dim;
    c.page_shift = __builtin_ctz((unsigned)C->page_size);
    c.n_pages = C->n_pages;
    c.k_codes = C->k_codes; c.v_codes = C->v_codes; c.k_scale = C->k_scale; c.v_scale = C->v_scale;
    return c;
}

int check_draft_sizes(const ordermoe_cache* C, int32_t dtype, int32_t n_q, int32_t B, int32_t max_q) {
    int rc = check_cache(C);
    if (rc) return rc;
    if ((rc = check_dtype(dtype, "draft_attention"))) return rc;
    if (n_q < 1 || n_q > 1024 || n_q % C->n_kv != 0)
        return fail(ORDERMOE_EINVAL, "draft_attention: n_q must be a multiple of n_kv, at most 1024");
    if (B < 0 || B > 65535) return fail(ORDERMOE_EINVAL, "draft_attention: B must lie in [0, 65535]");
    if (max_q < 1 || max_q > ORDERMOE_MAX_DRAFT)
        return fail(ORDERMOE_EINVAL, "draft_attention: max_q must lie in [1, " + std::to_string(ORDERMOE_MAX_DRAFT) + "]");
    return ORDERMOE_OK;
}

size_t draft_ws(const ordermoe_cache* C, int32_t dtype, int32_t n_q, int32_t B, int32_t max_q, Carver& c, DraftArgs* a) {
    const int64_t items = draft_items(n_q, C->n_kv, C->head_dim, dtype, B, max_q);
    const size_t rows = (size_t)items * max_q * n_q;
    int32_t* pl = c.take<int32_t>((size_t)std::max(B, 1) * 2);
    float* ml = c.take<float>(rows * 2);
    float* po = c.take<float>(rows * C->head_dim);
    if (a) { a->plan = pl; a->part_ml = ml; a->part_o = po; }
    return c.size();
}

}  // namespace
}  // namespace ordermoe

using namespace ordermoe;

extern "C" int ordermoe_cache_write(const ordermoe_cache* C, const ordermoe_heads* H, const void* q, int64_t q_stride,
                                    const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t T,
                                    const int32_t* pos, const int64_t* slots, void* q_out, void* stream) {
    int rc = check_cache(C);
    if (rc) return rc;
    if (!H) return fail(ORDERMOE_EINVAL, "cache_write: null heads");
    if ((rc = check_dtype(H->dtype, "cache_write"))) return rc;
    const int D = C->head_dim;
    if (H->n_q < 1 || H->n_q > 1024 || H->n_q % C->n_kv != 0)
        return fail(ORDERMOE_EINVAL, "cache_write: n_q must be a multiple of n_kv, at most 1024");
    if (H->rotary_dim < 0 || H->rotary_dim > D || H->rotary_dim % (D / 8) != 0)
        return fail(ORDERMOE_EINVAL, "cache_write: rotary_dim must be a multiple of head_dim / 8, at most head_dim");
    if (H->interleaved != 0 && H->interleaved != 1) return fail(ORDERMOE_EINVAL, "cache_write: interleaved must be 0 or 1");
    if (!(H->eps >= 0.0f) || std::isinf(H->eps)) return fail(ORDERMOE_EINVAL, "cache_write: eps must be finite and >= 0");
    if (T < 0 || T > (((int64_t)1 << 31) - 1) / (H->n_q + 2 * C->n_kv))
        return fail(ORDERMOE_EINVAL, "cache_write: T * (n_q + 2 n_kv) must lie in [0, 2^31)");
    if (H->rotary_dim > 0 && (H->max_pos < 1 || !H->cos_sin || (T > 0 && !pos)))
        return fail(ORDERMOE_EINVAL, "cache_write: rotation needs cos_sin, max_pos >= 1 and pos");
    if (T > 0 && (!q || !k || !v || !slots || !q_out)) return fail(ORDERMOE_EINVAL, "cache_write: null pointer");
    const int64_t per = H->dtype == ORDERMOE_BF16 ? 8 : 4;         // elements of 16 bytes
    if (q_stride < (int64_t)H->n_q * D || k_stride < (int64_t)C->n_kv * D || v_stride < (int64_t)C->n_kv * D ||
        q_stride % per || k_stride % per || v_stride % per)
        return fail(ORDERMOE_EINVAL, "cache_write: strides must hold the heads and be multiples of 16 bytes");
    if (T > 0 && (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out)))
        return fail(ORDERMOE_EINVAL, "cache_write: q, k, v and q_out must be 16-byte aligned");
    if ((H->q_norm && !aligned16(H->q_norm)) || (H->k_norm && !aligned16(H->k_norm)) || (H->rotary_dim > 0 && !aligned16(H->cos_sin)))
        return fail(ORDERMOE_EINVAL, "cache_write: norm weights and cos_sin must be 16-byte aligned");
    CacheWriteArgs a{};
    a.cache = cache_args(C);
    a.dtype = H->dtype; a.n_q = H->n_q; a.rot = H->rotary_dim; a.interleaved = H->interleaved;
    a.eps = H->eps; a.max_pos = H->max_pos; a.q_norm = H->q_norm; a.k_norm = H->k_norm; a.cos_sin = H->cos_sin;
    a.q = q; a.k = k; a.v = v; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.T = T; a.pos = pos; a.slots = slots; a.q_out = q_out;
    const int e = launch_cache_write(a, stream);
    if (e) return hip_fail(e, "cache_write launch");
    clear_error();
    return ORDERMOE_OK;
}

extern "C" int ordermoe_cache_read(const ordermoe_cache* C, int32_t dtype, const int64_t* slots, int64_t n, void* k_out,
                                   void* v_out, void* stream) {
    int rc = check_cache(C);
    if (rc) return rc;
    if ((rc = check_dtype(dtype, "cache_read"))) return rc;
    if (n < 0 || n > (((int64_t)1 << 31) - 1) / (2 * C->n_kv))
        return fail(ORDERMOE_EINVAL, "cache_read: 2 n n_kv must lie in [0, 2^31)");
    if (n > 0 && (!slots || !k_out || !v_out)) return fail(ORDERMOE_EINVAL, "cache_read: null pointer");
    if (n > 0 && (!aligned16(k_out) || !aligned16(v_out)))
        return fail(ORDERMOE_EINVAL, "cache_read: outputs must be 16-byte aligned");
    CacheReadArgs a{};
    a.cache = cache_args(C);
    a.dtype = dtype; a.slots = slots; a.n = n; a.k_out = k_out; a.v_out = v_out;
    const int e = launch_cache_read(a, stream);
    if (e) return hip_fail(e, "cache_read launch");
    clear_error();
    return ORDERMOE_OK;
}

extern "C" size_t ordermoe_draft_attention_workspace_size(const ordermoe_cache* C, int32_t dtype, int32_t n_q, int32_t B,
                                                          int32_t max_q) {
    if (check_draft_sizes(C, dtype, n_q, B, max_q) != ORDERMOE_OK) return 0;
    Carver c(nullptr);
    return draft_ws(C, dtype, n_q, B, max_q, c, nullptr);
}

extern "C" int ordermoe_draft_attention(const ordermoe_cache* C, int32_t dtype, int32_t n_q, const void* q, int64_t T,
                                        int32_t B, int32_t max_q, const int32_t* q_start, const int32_t* ctx_len,
                                        const int32_t* page_table, int32_t max_pages, const uint64_t* tree, float scale,
                                        void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    const int rc = check_draft_sizes(C, dtype, n_q, B, max_q);
    if (rc) return rc;
    if (T < 0 || T > ((int64_t)1 << 31) - 1) return fail(ORDERMOE_EINVAL, "draft_attention: T out of range");
    if (max_pages < 1 || (int64_t)max_pages * C->page_size > (int64_t)1 << 30)
        return fail(ORDERMOE_EINVAL, "draft_attention: max_pages * page_size must lie in [1, 2^30]");
    if (!std::isfinite(scale)) return fail(ORDERMOE_EINVAL, "draft_attention: scale must be finite");
    if (T > 0 && B > 0 && (!q || !q_start || !ctx_len || !page_table || !out))
        return fail(ORDERMOE_EINVAL, "draft_attention: null pointer");
    if (T > 0 && (!aligned16(q) || !aligned16(out)))
        return fail(ORDERMOE_EINVAL, "draft_attention: q and out must be 16-byte aligned");
    const size_t need = ordermoe_draft_attention_workspace_size(C, dtype, n_q, B, max_q);
    if (!ws || ws_bytes < need)
        return fail(ORDERMOE_EWORKSPACE, "draft_attention: workspace needs " + std::to_string(need) + " bytes");
    DraftArgs a{};
    a.cache = cache_args(C);
    a.dtype = dtype; a.n_q = n_q; a.B = B; a.max_q = max_q; a.max_pages = max_pages; a.T = T;
    a.q = q; a.q_start = q_start; a.ctx_len = ctx_len; a.page_table = page_table; a.tree = tree;
    a.scale = scale; a.out = out; a.lse = lse;
    Carver c(ws);
    draft_ws(C, dtype, n_q, B, max_q, c, &a);
    const int e = launch_draft_attention(a, stream);
    if (e) return hip_fail(e, "draft_attention launch");
    clear_error();
    return ORDERMOE_OK;
}
