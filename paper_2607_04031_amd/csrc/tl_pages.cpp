// C ABI of the calls on a pool of pages: argument validation, dispatch.  Nothing
// is enqueued unless every check passes.
#include <initializer_list>

#include "tl_internal.h"
#include "tl_serve.h"
#include "tl_serve_check.h"

namespace tl {
namespace {

// A pool's sizes and pointers, and lists of n entries each (not looked at where n is 0).
int check_pages(const tl_kv_pages* p, int64_t n, std::initializer_list<const int32_t*> lists, PagesLaunch* a) {
    if (!p || p->num_pages < 1 || p->num_rows < 1 || p->max_pages < 1 || n < 0) return TL_EINVAL;
    if (!is_pow2(p->page_tokens) || p->page_tokens < 64 || p->page_tokens > 4096 || p->num_pages > kMaxInt / p->page_tokens) return TL_EINVAL;
    if (bad_pointer(p->refs, 4) || bad_pointer(p->page_table, 4)) return TL_EINVAL;
    for (const int32_t* list : lists)
        if (n > 0 && bad_pointer(list, 4)) return TL_EINVAL;
    if (p->max_pages > kMostRowPages || p->num_rows > kMostEntries / p->max_pages || n > kMostPageRows) return TL_EUNSUPPORTED;
    if (overlap({p->refs, p->num_pages * 4}, {p->page_table, p->max_pages * p->num_rows * 4})) return TL_EINVAL;
    a->refs = p->refs;
    a->table = p->page_table;
    a->num_pages = p->num_pages;
    a->max_pages = p->max_pages;
    a->num_rows = p->num_rows;
    a->log2_page = ilog2(p->page_tokens);
    a->n = n;
    a->blocks = (p->num_pages + kPageBlock - 1) / kPageBlock;
    return TL_OK;
}

// whether outputs overlap the pool, lists of n entries or one another, or lists the pool
bool hits(const tl_kv_pages* p, int64_t n, std::initializer_list<const int32_t*> lists, std::initializer_list<Range> outs) {
    const Range refs = {p->refs, p->num_pages * 4}, table = {p->page_table, p->max_pages * p->num_rows * 4};
    for (const Range* r = outs.begin(); r != outs.end(); ++r) {
        if (overlap(*r, refs) || overlap(*r, table)) return true;
        for (const int32_t* list : lists)
            if (overlap(*r, {list, n * 4})) return true;
        for (const Range* other = outs.begin(); other != r; ++other)
            if (overlap(*r, *other)) return true;
    }
    for (const int32_t* list : lists)
        if (overlap({list, n * 4}, refs) || overlap({list, n * 4}, table)) return true;
    return false;
}

int pages_workspace(PagesLaunch* a, int64_t n, StreamHold* hold, void* stream) {
    void* ws = nullptr;
    const int st = stream_workspace((hipStream_t)stream, size_t(a->blocks * (64 * 12 + 4) + n * 8), hold, &ws);
    if (st != TL_OK) return st;
    a->map = static_cast<unsigned long long*>(ws);
    a->before = reinterpret_cast<int32_t*>(a->map + a->blocks * 64);
    a->free = a->before + a->blocks * 64;
    a->want = a->free + a->blocks;
    a->first = a->want + n;
    return TL_OK;
}

}  // namespace
}  // namespace tl

using namespace tl;

extern "C" {

int tl_kv_grow(const tl_kv_pages* pages, const int32_t* rows, const int32_t* lens, int32_t n, int32_t* missing, void* stream) {
    PagesLaunch a{};
    const int rc = check_pages(pages, n, {rows, lens}, &a);
    if (rc != TL_OK) return rc;
    if (bad_pointer(missing, 4) || hits(pages, n, {rows, lens}, {{missing, 4}})) return TL_EINVAL;
    a.rows = rows;
    a.lens = lens;
    a.count = missing;
    StreamHold hold;
    const int st = pages_workspace(&a, n, &hold, stream);
    return st != TL_OK ? st : done(launch_pages_grow(a, (hipStream_t)stream));
}

int tl_kv_free(const tl_kv_pages* pages, const int32_t* rows, const int32_t* lens, int32_t n, void* stream) {
    PagesLaunch a{};
    const int rc = check_pages(pages, n, {rows, lens ? lens : rows}, &a);
    if (rc != TL_OK) return rc;
    if (hits(pages, n, {rows, lens}, {})) return TL_EINVAL;
    a.rows = rows;
    a.lens = lens;
    return n == 0 ? TL_OK : done(launch_pages_free(a, (hipStream_t)stream));
}

int tl_kv_fork(const tl_kv_pages* pages, const int32_t* parents, const int32_t* children, const int32_t* lens, int32_t n,
               int32_t* src, int32_t* dst, int32_t* tokens, int32_t* count, void* stream) {
    PagesLaunch a{};
    const int rc = check_pages(pages, n, {parents, children, lens}, &a);
    if (rc != TL_OK) return rc;
    if (bad_pointer(count, 4) || (n > 0 && (bad_pointer(src, 4) || bad_pointer(dst, 4) || bad_pointer(tokens, 4)))) return TL_EINVAL;
    const int64_t list = int64_t(n) * 4;
    if (hits(pages, n, {parents, children, lens}, {{src, list}, {dst, list}, {tokens, list}, {count, 8}})) return TL_EINVAL;
    a.parents = parents;
    a.rows = children;
    a.lens = lens;
    a.src = src;
    a.dst = dst;
    a.tokens = tokens;
    a.count = count;
    StreamHold hold;
    const int st = pages_workspace(&a, n, &hold, stream);
    return st != TL_OK ? st : done(launch_pages_fork(a, (hipStream_t)stream));
}

int tl_kv_compact(const tl_kv_pages* pages, int64_t max_moves, int32_t* src, int32_t* dst, int32_t* count, void* stream) {
    PagesLaunch a{};
    const int rc = check_pages(pages, 0, {}, &a);
    if (rc != TL_OK) return rc;
    if (max_moves < 0 || bad_pointer(count, 4) || (max_moves > 0 && (bad_pointer(src, 4) || bad_pointer(dst, 4)))) return TL_EINVAL;
    if (max_moves > kMaxInt) return TL_EUNSUPPORTED;
    if (hits(pages, 0, {}, {{src, max_moves * 4}, {dst, max_moves * 4}, {count, 8}})) return TL_EINVAL;
    a.n = max_moves;
    a.src = src;
    a.dst = dst;
    a.count = count;
    StreamHold hold;
    const int st = pages_workspace(&a, 0, &hold, stream);
    return st != TL_OK ? st : done(launch_pages_compact(a, (hipStream_t)stream));
}

int tl_kv_copy(const tl_kv_cache* cache, const int32_t* src, const int32_t* dst, const int32_t* tokens, const int32_t* count,
               int64_t max_pairs, void* stream) {
    int64_t data, exps;
    PagesCopyLaunch a{};
    const int rc = check_cache(cache, &data, &exps, &a.c);
    if (rc != TL_OK) return rc;
    if (max_pairs < 0 || !aligned(tokens, 4) || !aligned(count, 4)) return TL_EINVAL;
    if (max_pairs == 0) return TL_OK;
    if (bad_pointer(src, 4) || bad_pointer(dst, 4)) return TL_EINVAL;
    if (max_pairs > kMaxInt) return TL_EUNSUPPORTED;
    const Range lists[4] = {{src, max_pairs * 4}, {dst, max_pairs * 4}, {tokens, max_pairs * 4}, {count, 4}};
    for (const Range& r : lists)
        if (hits_cache(cache, data, exps, r)) return TL_EINVAL;
    const Range arrays[4] = {{cache->k, data}, {cache->v, data}, {cache->k_exp, exps}, {cache->v_exp, exps}};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(arrays[i], arrays[j])) return TL_EINVAL;
    a.src = src;
    a.dst = dst;
    a.tokens = tokens;
    a.count = count;
    a.pairs = max_pairs;
    return done(launch_pages_copy(a, cache->head_dim, cache->elem_bytes, (hipStream_t)stream));
}

}  // extern "C"
