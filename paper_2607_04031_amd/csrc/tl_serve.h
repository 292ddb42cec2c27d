// Internal declarations of the serving-step operators: the paged key/value
// cache (tl_kv.hip), attention over it (tl_attn.hip) and the verification of
// drafted tokens (tl_verify.hip).  The entry points in tl_serve.cpp check all
// arguments; the launchers only enqueue.
#pragma once

#include <cstdint>

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
__host__ __device__ inline int kv_key_exp_at(int t) { return (t & ~63) + (t & 15) * 4 + ((t & 63) >> 4); }
__host__ __device__ inline int kv_value_exp_at(int t) { return (t & ~63) + ((t & 15) >> 2) * 16 + ((t & 63) >> 4) * 4 + (t & 3); }

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
