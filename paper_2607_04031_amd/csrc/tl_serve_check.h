// Checks of arguments that the entry points of the serving step share.
#pragma once

#include <cstdint>

#include "tl_internal.h"
#include "tl_serve.h"

namespace tl {

constexpr int64_t kMaxInt = 0x7fffffff;

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool bad_pointer(const void* p, uintptr_t to) { return !p || !aligned(p, to); }

struct Range {
    const void* p;
    int64_t bytes;
};
inline bool overlap(const Range& a, const Range& b) {
    if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
    const auto x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x < y + uintptr_t(b.bytes) && y < x + uintptr_t(a.bytes);
}

// The cache's sizes; data and exps: bytes of k (v) and of k_exp (v_exp).
inline int check_sizes(const tl_kv_cache* c, int64_t* data, int64_t* exps) {
    if (!c || c->num_pages < 1 || !is_pow2(c->page_tokens) || c->page_tokens < 64 || c->page_tokens > 4096) return TL_EINVAL;
    if (c->kv_heads < 1 || c->kv_heads > 1024 || (c->elem_bytes != 1 && c->elem_bytes != 2 && c->elem_bytes != TL_KV_E2M1)) return TL_EINVAL;
    if (c->num_pages > kMaxInt / c->page_tokens) return TL_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128) return TL_EUNSUPPORTED;
    const int64_t tokens = c->num_pages * c->page_tokens * c->kv_heads;
    const bool four = c->elem_bytes == TL_KV_E2M1;
    *data = four ? tokens * c->head_dim / 2 : tokens * c->head_dim * c->elem_bytes;
    *exps = four ? tokens * c->head_dim / 32 : c->elem_bytes == 1 ? tokens : 0;
    return TL_OK;
}

inline int check_cache(const tl_kv_cache* c, int64_t* data, int64_t* exps, KvView* view) {
    const int rc = check_sizes(c, data, exps);
    if (rc != TL_OK) return rc;
    if (bad_pointer(c->k, 16) || bad_pointer(c->v, 16)) return TL_EINVAL;
    if (*exps && (bad_pointer(c->k_exp, 16) || bad_pointer(c->v_exp, 16))) return TL_EINVAL;
    *view = KvView{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_exp, c->v_exp, c->num_pages,
                   ilog2(c->page_tokens), c->kv_heads};
    return TL_OK;
}

inline bool hits_cache(const tl_kv_cache* c, int64_t data, int64_t exps, const Range& r) {
    return overlap(r, {c->k, data}) || overlap(r, {c->v, data}) || overlap(r, {c->k_exp, exps}) || overlap(r, {c->v_exp, exps});
}

inline int done(hipError_t e) { return e == hipSuccess ? TL_OK : TL_EHIP; }

}  // namespace tl
