// Internal declarations of the serving-step operators: the paged key/value
// cache (tl_kv.hip), its pages (tl_pages.hip), attention over it (tl_attn.hip)
// and the verification of drafted tokens (tl_verify.hip).  The entry points in tl_serve.cpp and tl_pages.cpp check all
// arguments; the launchers only enqueue.
#pragma once

#include <cstdint>
#include <type_traits>

#include <hip/hip_runtime.h>

#include "../../include/tl.h"

namespace tl {

// A cache as the kernels use it.  A page holds, for every key/value head, one
// block of keys and one of values of page_tokens tokens, in the order in which
// the attention kernel's matrix operands take them, so that each of its loads
// is 1 KB without gaps.  With c = 16 / elem_bytes elements to a 16-byte chunk:
//   keys    [page][head][t / 16][d / c][t % 16][d % c]
//   values  [page][head][t / 4c][d / 16][t % 16 / 4][d % 16][t % 4c / 16][t % 4]
// and, 8 bits, the biased exponents of the scales (one per token and head):
//   keys    [page][head][t / 64][t % 16][t % 64 / 16]
//   values  [page][head][t / 64][t % 16 / 4][t % 64 / 16][t % 4]
// 4 bits: bytes as of an 8-bit cache with half the head size, of which byte b
// holds two elements (keys 2 b and 2 b + 1, values 32 (b / 16) + b % 16 and 16
// on, the first one low), and of the exponents [B = head size / 32] blocks
// where 8 bits have one:
//   keys    [page][head][t / 64][B][t % 16][t % 64 / 16]
//   values  [page][head][t / 64][B][t % 16 / 4][t % 64 / 16][t % 4]
struct KvView {
    uint8_t* k;
    uint8_t* v;
    uint8_t* k_exp;
    uint8_t* v_exp;
    int64_t num_pages;
    int log2_page;      // page_tokens = 1 << log2_page >= 64
    int heads;
};

// Element offsets inside a (page, head) block of page_tokens * D elements.
template <int D, int ELEM>
__host__ __device__ inline int kv_key_at(int t, int d) {
    constexpr int c = 16 / ELEM;
    return ((t >> 4) * (D / c) + d / c) * (16 * c) + (t & 15) * c + d % c;
}
template <int D, int ELEM>
__host__ __device__ inline int kv_value_at(int t, int d) {
    constexpr int c = 16 / ELEM;
    return t / (4 * c) * (4 * c * D) + (d >> 4) * (64 * c) + ((t & 15) >> 2) * (16 * c) + (d & 15) * c +
           (t % (4 * c) >> 4) * 4 + (t & 3);
}
// Offsets of the exponent of block b of B.
__host__ __device__ inline int kv_key_exp_at(int t, int b = 0, int B = 1) { return (t & ~63) * B + b * 64 + (t & 15) * 4 + ((t & 63) >> 4); }
__host__ __device__ inline int kv_value_exp_at(int t, int b = 0, int B = 1) {
    return (t & ~63) * B + b * 64 + ((t & 15) >> 2) * 16 + ((t & 63) >> 4) * 4 + (t & 3);
}

// Of an element type (elem_bytes of the cache): the stored elements of a head
// and their bytes -- of 4 bits, two to a byte -- and the exponents of a token's
// head.
template <int ELEM>
constexpr bool kv_four() { return ELEM == TL_KV_E2M1; }
template <int D, int ELEM>
constexpr int kv_width() { return kv_four<ELEM>() ? D / 2 : D; }
template <int ELEM>
constexpr int kv_size() { return kv_four<ELEM>() ? 1 : ELEM; }
template <int D, int ELEM>
constexpr int kv_exps() { return kv_four<ELEM>() ? D / 32 : ELEM == 1 ? 1 : 0; }

// f(head size, element type) for those of a cache
template <typename F>
auto kv_as(int head_dim, int elem_bytes, F f) {
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    using E4 = std::integral_constant<int, TL_KV_E2M1>;
    using E8 = std::integral_constant<int, 1>;
    using E16 = std::integral_constant<int, 2>;
    if (head_dim == 64) return elem_bytes == 1 ? f(D64(), E8()) : elem_bytes == 2 ? f(D64(), E16()) : f(D64(), E4());
    return elem_bytes == 1 ? f(D128(), E8()) : elem_bytes == 2 ? f(D128(), E16()) : f(D128(), E4());
}

// Workgroups of a launch, at most: HIP takes fewer than 2^32 work-items in a
// dimension.  The entry points refuse a call with more in any of its launches.
constexpr int64_t most_workgroups(int threads) { return ((int64_t(1) << 32) - 1) / threads; }

struct KvAppendLaunch {
    KvView c;
    const void* src[3];       // queries, keys, values: rows of heads * D elements
    int64_t ld[3];            // elements between rows
    int heads[3];
    bool src_f32;
    int64_t n;
    const int32_t* slots;
    // rotary positions: rot_dim 0 for none
    const int32_t* positions; // [axes][n]
    const float* inv_freq;    // [rot_dim / 2]
    int rot_dim, sections[3];
    bool interleaved;
    uint16_t* q_out;          // bf16 [n][heads[0]][D]
};
constexpr int kKvThreads = 256;
int64_t kv_append_workgroups(const KvAppendLaunch& a, int head_dim);
hipError_t launch_kv_append(const KvAppendLaunch& a, int head_dim, int elem_bytes, hipStream_t stream);

int64_t kv_read_workgroups(const KvView& c, int head_dim, int64_t n);
hipError_t launch_kv_read(const KvView& c, int head_dim, int elem_bytes, const int32_t* slots, int64_t n, uint16_t* k_out,
                          uint16_t* v_out, hipStream_t stream);

struct KvKeepLaunch {
    KvView c;
    const int32_t* page_table;
    int64_t max_pages;
    const int32_t* starts;
    const int32_t* path;
    const int32_t* counts;
    int num_seqs, max_path;
};
hipError_t launch_kv_keep(const KvKeepLaunch& a, int head_dim, int elem_bytes, hipStream_t stream);

// A call on a pool of pages (tl_pages.hip).
constexpr int kPagesGrow = 0, kPagesFork = 1, kPagesCompact = 2;
constexpr int kPageThreads = 256;
constexpr int kPageBlock = 4096;    // pages whose bits a wave makes
constexpr int kMostPageRows = 65536;
constexpr int64_t kMostRowPages = int64_t(1) << 25, kMostEntries = int64_t(1) << 40;    // of a row, and of a table
struct PagesLaunch {
    int32_t* refs;
    int32_t* table;             // [num_rows][max_pages]
    int64_t num_pages, max_pages;
    int num_rows;
    int log2_page;
    int64_t n;                  // sequences (compact: moves at most)
    const int32_t* rows;        // the sequences' rows; fork: the children's
    const int32_t* parents;
    const int32_t* lens;
    int32_t* src;
    int32_t* dst;
    int32_t* tokens;
    int32_t* count;             // grow: missing
    // workspace: bits of the free pages, and their number before each word of a
    // block of pages and in the block; of each sequence the pages that it wants,
    // and the first entry without one
    int64_t blocks;
    unsigned long long* map;
    int32_t* before;
    int32_t* free;
    int32_t* want;
    int32_t* first;
    int64_t map_wave;           // the first wave of a launch that makes bits
};
hipError_t launch_pages_grow(const PagesLaunch& a, hipStream_t stream);
hipError_t launch_pages_free(const PagesLaunch& a, hipStream_t stream);
hipError_t launch_pages_fork(const PagesLaunch& a, hipStream_t stream);
hipError_t launch_pages_compact(const PagesLaunch& a, hipStream_t stream);

struct PagesCopyLaunch {
    KvView c;
    const int32_t* src;
    const int32_t* dst;
    const int32_t* tokens;      // nullptr: whole pages
    const int32_t* count;       // nullptr: all pairs
    int64_t pairs;
};
hipError_t launch_pages_copy(const PagesCopyLaunch& a, int head_dim, int elem_bytes, hipStream_t stream);

struct AttnLaunch {
    KvView c;
    const uint16_t* q;
    int64_t ldq;
    const int32_t* page_table;
    int64_t max_pages;
    const int32_t* lens;
    const int32_t* q_offsets;
    const uint32_t* mask;     // nullptr: causal
    int mask_words;
    int num_seqs;
    int64_t total_q, max_q, max_len;
    int q_heads;
    float scale_log2;         // scale * log2(e)
    uint16_t* out;
    // query heads of a key head, and the division by it of x < 2^31 as
    // (umulhi(x, magic) + x) >> shift (Granlund and Montgomery, "Division by
    // invariant integers using multiplication", 1994, Section 4)
    int group;
    uint32_t group_magic;
    int group_shift;
    // the plan: rows per tile, keys per chunk (powers of two), tiles of all
    // sequences and heads (an upper bound), whether keys are split over
    // workgroups, and how many of those
    int log2_rows, log2_keys;
    bool split;
    bool sorted;              // not split, at most 64 sequences: the longest tiles of all first
    int64_t max_tiles;
    int groups;
    float* ws;                // partial results: two per workgroup (split)
};
constexpr int kAttnThreads = 256;
// Fills the plan; returns the workspace it needs, in floats.
int64_t plan_attn(AttnLaunch* a, int head_dim, int elem_bytes);
hipError_t launch_attn(const AttnLaunch& a, int head_dim, int elem_bytes, hipStream_t stream);
// its first launch where tiles have 128 rows
hipError_t launch_attn_wide(const AttnLaunch& a, int head_dim, int elem_bytes, hipStream_t stream);

struct VerifyLaunch {
    const void* logits;
    bool logits_bf16;
    int64_t vocab;
    const int32_t* offsets;
    const int32_t* parents;
    const int32_t* tokens;
    int num_seqs;
    int64_t total;
    int max_nodes;
    const void* draft;        // nullptr: every drafted token was certain
    bool draft_bf16;
    const float* temperature;
    const float* uniform;
    const float* noise;
    int32_t* path;            // [num_seqs][max_nodes]
    int32_t* counts;
    int32_t* next;
    void* ws;
};
// rows with a workgroup of 256 threads or more each, sequences with one of 1024
constexpr int64_t kMostVerifyNodes = most_workgroups(256), kMostVerifySeqs = most_workgroups(1024);
int64_t verify_workspace_bytes(int64_t vocab, int64_t total, int num_seqs, int max_nodes);
hipError_t launch_verify(const VerifyLaunch& a, hipStream_t stream);

}  // namespace tl
