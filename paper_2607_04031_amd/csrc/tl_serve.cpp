// C ABI of the serving-step operators: argument validation, the attention
// plan, dispatch.  Nothing is enqueued unless every check passes.
#include <algorithm>
#include <cmath>

#include "tl_internal.h"
#include "tl_serve.h"
#include "tl_serve_check.h"

namespace tl {
namespace {

constexpr int64_t kMaxStride = int64_t(1) << 30;
constexpr int kMaxNodes = 4096;
constexpr float kLog2e = 1.44269504088896340736f;

// Bytes from the first row's start to the last row's end.
int64_t span(int64_t rows, int64_t ld, int64_t width, int64_t elem) { return rows > 0 ? ((rows - 1) * ld + width) * elem : 0; }

}  // namespace

// Rows per tile: the fewest of 16, 32, 64 and 128 that hold a sequence's rows
// of one key head.  Keys are split where the tiles are too few to keep the CUs
// evenly busy, but not (us split and not, ragged lengths up to the one named):
//   - where no sequence has more than 1024 keys (16 rows: 2048 of 8 bits, 1536 of
//     16), since joining the partial results costs a second launch: one token
//     over 2048 8-bit tokens 17.4 and 14.3 (over 3000 15.3 and 19.8), over 1500
//     16-bit ones 16.2 and 14.8 (2048: 13.1 and 20.2);
//   - where each of the slots for workgroups gets a tile of its own and none is
//     long: 64 tokens over 2048 or 4096 39.0 and 33.7, 62.0 and 57.8; at 128 rows
//     two tiles to a slot, which trees need (64 of 32 nodes over 2048 tokens 128
//     and 121, 16-bit 135 and 117), and prompts, whose tiles differ, do not (8 of
//     512 tokens 148 and 167);
//   - where each gets four tiles;
//   - prompts over a 4-bit cache with a tile for every slot: whole tiles, the
//     longest of all first, since a slot that is free takes the next one.  Three
//     prompts of 2048 over 4096 (1180 tiles) 172 and 146, two of 2048 (1392) 125
//     and 98, six of 1024 (764) 67 and 47, one of 2048 (512) 77 and 63; of equal
//     length, 544 over 1088 (544) 67 and 53, over 8192 319 and 380, which is why
//     fewer than two tiles a slot have to be short or of different lengths (1088
//     over 8192 533 and 581, 1024 500 and 473, 1280 622 and 594: just past a multiple
//     of the slots long tiles of nearly one length would be 9 % faster split, and the
//     rule does not look for that).  A wave knows 64 sequences; above that tiles keep
//     the line's order: 64 prompts of up to 1024 113, 65 125 (8 bits 131 and 132).
// All of it goes by max_len, the caller's bound: one far above the lengths splits
// what need not be.
int64_t plan_attn(AttnLaunch* a, int head_dim, int elem_bytes) {
    constexpr int64_t kSlots = 2 * 256;
    a->group = a->q_heads / a->c.heads;
    a->group_shift = ilog2(a->group);
    a->group_magic = uint32_t((uint64_t((int64_t(1) << a->group_shift) - a->group) << 32) / uint64_t(a->group) + 1);
    const int64_t group = a->group, most = a->max_q * group;
    a->log2_rows = most <= 16 ? 4 : most <= 32 ? 5 : most <= 64 ? 6 : 7;
    const int64_t rows = int64_t(1) << a->log2_rows;
    a->log2_keys = elem_bytes != 2 || rows == 128 ? 6 : 5;
    a->max_tiles = std::min(a->num_seqs * ((most + rows - 1) / rows), a->total_q * group / rows + a->num_seqs) * a->c.heads;
    const bool wide = rows == 128;
    const int64_t whole = rows > 16 ? 1024 : elem_bytes != 2 ? 2048 : 1536;
    const bool enough = wide ? a->mask && a->max_tiles >= 2 * kSlots && a->max_len <= 2048 : a->max_tiles >= kSlots && a->max_len <= 4096;
    a->split = a->max_len > whole && !enough && a->max_tiles < 4 * kSlots;
    a->sorted = elem_bytes == TL_KV_E2M1 && wide && !a->mask && a->num_seqs <= 64 && a->max_tiles >= kSlots &&
                (a->max_len <= 4096 || 2 * a->max_q >= a->max_len || a->max_tiles >= 2 * kSlots);
    if (a->sorted) a->split = false;
    a->groups = int(a->split ? kSlots : a->max_tiles);
    return a->split ? 2 * a->groups * rows * (head_dim + 2) + a->groups * 8 : 0;
}

}  // namespace tl

using namespace tl;

extern "C" {

int tl_kv_bytes(const tl_kv_cache* cache, int64_t* data, int64_t* exps) {
    if (!data || !exps) return TL_EINVAL;
    int64_t d, e;
    const int rc = check_sizes(cache, &d, &e);
    if (rc != TL_OK) return rc;
    *data = d;
    *exps = e;
    return TL_OK;
}

int tl_kv_append(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv, int32_t in_dtype,
                 int64_t n, int32_t q_heads, const int32_t* slots, const tl_rope* rope, void* Q_out,
                 const tl_kv_cache* cache, void* stream) {
    int64_t data, exps;
    KvAppendLaunch a{};
    const int rc = check_cache(cache, &data, &exps, &a.c);
    if (rc != TL_OK) return rc;
    if (n < 0 || q_heads < 0 || (in_dtype != TL_IN_F32 && in_dtype != TL_IN_BF16)) return TL_EINVAL;
    if (n == 0) return TL_OK;
    a.n = n;
    if ((K == nullptr) != (V == nullptr) || (Q == nullptr) != (q_heads == 0) || (Q == nullptr) != (Q_out == nullptr)) return TL_EINVAL;
    if (!Q && !K) return TL_EINVAL;
    if (q_heads > 4096) return TL_EUNSUPPORTED;
    const int D = cache->head_dim, in = in_dtype == TL_IN_F32 ? 4 : 2;
    const void* src[3] = {Q, K, V};
    const int64_t ld[3] = {ldq, ldk, ldv};
    const int heads[3] = {q_heads, K ? cache->kv_heads : 0, K ? cache->kv_heads : 0};
    for (int i = 0; i < 3; ++i) {
        a.src[i] = src[i];
        a.ld[i] = ld[i];
        a.heads[i] = heads[i];
        if (!src[i]) continue;
        if (!aligned(src[i], 16) || ld[i] < int64_t(heads[i]) * D || ld[i] * in % 16) return TL_EINVAL;
        if (ld[i] > kMaxStride) return TL_EUNSUPPORTED;
    }
    if (K && bad_pointer(slots, 4)) return TL_EINVAL;
    if (Q && !aligned(Q_out, 16)) return TL_EINVAL;
    a.slots = K ? slots : nullptr;
    if (rope) {
        if (rope->axes < 1 || rope->axes > 3 || rope->rot_dim < 16 || rope->rot_dim > D || rope->rot_dim % 16) return TL_EINVAL;
        if (bad_pointer(rope->positions, 4) || bad_pointer(rope->inv_freq, 4)) return TL_EINVAL;
        int64_t pairs = 0;
        for (int i = 0; i < rope->axes; ++i) {
            if (rope->sections[i] < 0) return TL_EINVAL;
            a.sections[i] = rope->sections[i];
            pairs += rope->sections[i];
        }
        if (pairs != rope->rot_dim / 2) return TL_EINVAL;
        a.positions = rope->positions;
        a.inv_freq = rope->inv_freq;
        a.rot_dim = rope->rot_dim;
        a.interleaved = rope->interleaved != 0;
    }
    if (n > kMaxInt || kv_append_workgroups(a, D) > most_workgroups(kKvThreads)) return TL_EUNSUPPORTED;
    // outputs: the queries and the cache's arrays (no part of this call without keys)
    const Range out = {Q_out, n * q_heads * D * 2}, arrays[4] = {{cache->k, data}, {cache->v, data}, {cache->k_exp, exps}, {cache->v_exp, exps}};
    auto hit = [&](const Range& r) { return overlap(out, r) || (K && hits_cache(cache, data, exps, r)); };
    for (int i = 0; i < 3; ++i)
        if (hit({src[i], span(n, ld[i], int64_t(heads[i]) * D, in)})) return TL_EINVAL;
    if (hit({a.slots, n * 4})) return TL_EINVAL;
    if (rope && (hit({rope->positions, n * rope->axes * 4}) || hit({rope->inv_freq, rope->rot_dim / 2 * 4}))) return TL_EINVAL;
    if (K && hits_cache(cache, data, exps, out)) return TL_EINVAL;
    for (int i = 0; K && i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(arrays[i], arrays[j])) return TL_EINVAL;
    a.src_f32 = in_dtype == TL_IN_F32;
    a.q_out = static_cast<uint16_t*>(Q_out);
    return done(launch_kv_append(a, D, cache->elem_bytes, (hipStream_t)stream));
}

int tl_kv_read(const tl_kv_cache* cache, const int32_t* slots, int64_t n, void* K_out, void* V_out, void* stream) {
    int64_t data, exps;
    KvView view;
    const int rc = check_cache(cache, &data, &exps, &view);
    if (rc != TL_OK) return rc;
    if (n < 0) return TL_EINVAL;
    if (n == 0) return TL_OK;
    if (bad_pointer(slots, 4) || (!K_out && !V_out) || !aligned(K_out, 16) || !aligned(V_out, 16)) return TL_EINVAL;
    const int64_t row = int64_t(cache->kv_heads) * cache->head_dim;
    if (n > kMaxInt || kv_read_workgroups(view, cache->head_dim, n) > most_workgroups(kKvThreads)) return TL_EUNSUPPORTED;
    const Range k = {K_out, n * row * 2}, v = {V_out, n * row * 2}, s = {slots, n * 4};
    if (overlap(k, v) || overlap(k, s) || overlap(v, s)) return TL_EINVAL;
    if (hits_cache(cache, data, exps, k) || hits_cache(cache, data, exps, v)) return TL_EINVAL;
    return done(launch_kv_read(view, cache->head_dim, cache->elem_bytes, slots, n, static_cast<uint16_t*>(K_out),
                               static_cast<uint16_t*>(V_out), (hipStream_t)stream));
}

int tl_kv_keep(const tl_kv_cache* cache, const int32_t* page_table, int64_t max_pages, const int32_t* starts,
               const int32_t* path, int64_t max_path, const int32_t* counts, int32_t num_seqs, void* stream) {
    int64_t data, exps;
    KvKeepLaunch a{};
    const int rc = check_cache(cache, &data, &exps, &a.c);
    if (rc != TL_OK) return rc;
    if (num_seqs < 0 || max_pages < 1 || max_path < 1) return TL_EINVAL;
    if (num_seqs == 0) return TL_OK;
    if (bad_pointer(page_table, 4) || bad_pointer(starts, 4) || bad_pointer(path, 4) || bad_pointer(counts, 4)) return TL_EINVAL;
    if (max_path > kMaxNodes || num_seqs > most_workgroups(kKvThreads) / cache->kv_heads) return TL_EUNSUPPORTED;
    a.page_table = page_table;
    a.max_pages = max_pages;
    a.starts = starts;
    a.path = path;
    a.counts = counts;
    a.num_seqs = num_seqs;
    a.max_path = int(max_path);
    return done(launch_kv_keep(a, cache->head_dim, cache->elem_bytes, (hipStream_t)stream));
}

int tl_attn(const void* Q, int64_t ldq, const tl_kv_cache* cache, const int32_t* page_table, int64_t max_pages,
            const int32_t* lens, const int32_t* q_offsets, const uint32_t* mask, int32_t mask_words, int32_t num_seqs,
            int64_t total_q, int64_t max_q, int64_t max_len, int32_t q_heads, float scale, void* O, void* stream) {
    int64_t data, exps;
    AttnLaunch a{};
    const int rc = check_cache(cache, &data, &exps, &a.c);
    if (rc != TL_OK) return rc;
    if (num_seqs < 0 || total_q < 0 || max_q < 0 || max_len < 0 || max_pages < 1) return TL_EINVAL;
    if (q_heads < 1 || q_heads % cache->kv_heads || !(scale > 0.f) || !std::isfinite(scale)) return TL_EINVAL;
    if (mask && (mask_words < 1 || !aligned(mask, 4))) return TL_EINVAL;
    const int D = cache->head_dim;
    const int64_t width = int64_t(q_heads) * D;
    if (total_q > 0 && num_seqs > 0) {
        if (bad_pointer(Q, 16) || bad_pointer(O, 16) || bad_pointer(page_table, 4) || bad_pointer(lens, 4) || bad_pointer(q_offsets, 4)) return TL_EINVAL;
        if (ldq < width || ldq % 8) return TL_EINVAL;
    }
    if (!std::isfinite(scale * kLog2e)) return TL_EUNSUPPORTED;
    if (ldq > kMaxStride || max_len > kMaxStride || q_heads > kMaxStride / std::max<int64_t>(total_q, 1) || (mask && mask_words > 65536)) return TL_EUNSUPPORTED;
    if (total_q == 0 || num_seqs == 0 || max_q == 0) return TL_OK;
    if (max_pages > kMaxInt) return TL_EUNSUPPORTED;
    const Range out = {O, total_q * width * 2};
    if (overlap(out, {Q, span(total_q, ldq, width, 2)}) || hits_cache(cache, data, exps, out) ||
        overlap(out, {mask, total_q * mask_words * 4}) || overlap(out, {page_table, num_seqs * max_pages * 4}) ||
        overlap(out, {lens, int64_t(num_seqs) * 4}) || overlap(out, {q_offsets, (int64_t(num_seqs) + 1) * 4})) return TL_EINVAL;
    a.q = static_cast<const uint16_t*>(Q);
    a.ldq = ldq;
    a.page_table = page_table;
    a.max_pages = max_pages;
    a.lens = lens;
    a.q_offsets = q_offsets;
    a.mask = mask;
    a.mask_words = mask_words;
    a.num_seqs = num_seqs;
    a.total_q = total_q;
    a.max_q = std::min(max_q, total_q);
    a.max_len = max_len;
    a.q_heads = q_heads;
    a.scale_log2 = scale * kLog2e;
    a.out = static_cast<uint16_t*>(O);
    const int64_t floats = plan_attn(&a, D, cache->elem_bytes);
    if (a.max_tiles > most_workgroups(kAttnThreads)) return TL_EUNSUPPORTED;
    StreamHold hold;
    if (floats > 0) {
        void* ws = nullptr;
        const int st = stream_workspace((hipStream_t)stream, size_t(floats) * 4, &hold, &ws);
        if (st != TL_OK) return st;
        a.ws = static_cast<float*>(ws);
    }
    return done(launch_attn(a, D, cache->elem_bytes, (hipStream_t)stream));
}

int tl_verify(const void* logits, int32_t logits_dtype, int64_t vocab, const int32_t* node_offsets, const int32_t* parents,
              const int32_t* tokens, int32_t num_seqs, int64_t total_nodes, int32_t max_nodes, const void* draft,
              int32_t draft_dtype, const float* temperature, const float* uniform, const float* noise, int32_t* path,
              int32_t* counts, int32_t* next, void* stream) {
    if (vocab < 1 || num_seqs < 0 || total_nodes < 0 || max_nodes < 1) return TL_EINVAL;
    if (logits_dtype != TL_OUT_F32 && logits_dtype != TL_OUT_BF16) return TL_EINVAL;
    if (draft && draft_dtype != TL_OUT_F32 && draft_dtype != TL_OUT_BF16) return TL_EINVAL;
    if (num_seqs == 0) return TL_OK;
    if (bad_pointer(node_offsets, 4) || bad_pointer(temperature, 4) || bad_pointer(path, 4) || bad_pointer(counts, 4) || bad_pointer(next, 4)) return TL_EINVAL;
    if (bad_pointer(noise, 16) || !aligned(draft, 16)) return TL_EINVAL;
    if (total_nodes > 0 && (bad_pointer(logits, 16) || bad_pointer(parents, 4) || bad_pointer(tokens, 4) || bad_pointer(uniform, 4))) return TL_EINVAL;
    if (vocab > (1 << 26) || total_nodes > kMostVerifyNodes || num_seqs > kMostVerifySeqs || max_nodes > kMaxNodes) return TL_EUNSUPPORTED;
    VerifyLaunch a{};
    a.logits = logits;
    a.logits_bf16 = logits_dtype == TL_OUT_BF16;
    a.vocab = vocab;
    a.offsets = node_offsets;
    a.parents = parents;
    a.tokens = tokens;
    a.num_seqs = num_seqs;
    a.total = total_nodes;
    a.max_nodes = max_nodes;
    a.draft = draft;
    a.draft_bf16 = draft && draft_dtype == TL_OUT_BF16;
    a.temperature = temperature;
    a.uniform = uniform;
    a.noise = noise;
    a.path = path;
    a.counts = counts;
    a.next = next;
    StreamHold hold;
    const int st = stream_workspace((hipStream_t)stream, size_t(verify_workspace_bytes(vocab, total_nodes, num_seqs, max_nodes)), &hold, &a.ws);
    if (st != TL_OK) return st;
    return done(launch_verify(a, (hipStream_t)stream));
}

}  // extern "C"
