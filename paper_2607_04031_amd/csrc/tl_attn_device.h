// Shared by the attention kernels: how the work is laid out over workgroups,
// and the joining of partial results.
#pragma once

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {

__device__ inline f32x4v mfma_16x16x32(u32x4 a, u32x4 b, f32x4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, a), __builtin_bit_cast(bf16x8v, b), c, 0, 0, 0);
}

// The work is a line: sequence after sequence, in it head after head, in it
// tile after tile of rows, in it (split) chunk of keys after chunk.  Without a
// split a workgroup takes one tile of a head; with one, workgroup w of W takes
// the places [w T / W, (w + 1) T / W) of all T, so that all have the same to do
// whatever the lengths are, and writes what it has of a tile that it does not
// hold whole as a partial result: of the first tile in its slot 2 w, of the
// last in 2 w + 1.
struct Seq {
    int seq, first, n, len;     // first: row of the first new token; n: new tokens; len: keys
    int tiles, chunks;          // of rows; of keys (at least 1)
    int64_t before;             // places before the sequence
};

__device__ inline int attn_offset(const AttnLaunch& a, int i) { return max(0, min(a.q_offsets[i], int(a.total_q))); }

__device__ inline Seq attn_seq(const AttnLaunch& a, int b) {
    Seq s{b, 0, 0, 0, 0, 1, 0};
    if (b >= a.num_seqs) return s;
    s.first = attn_offset(a, b);
    s.n = max(0, attn_offset(a, b + 1) - s.first);
    s.len = int(max(int64_t(0), min(int64_t(a.lens[b]), min(a.max_pages << a.c.log2_page, a.max_len))));
    s.tiles = int((int64_t(s.n) * (a.q_heads / a.c.heads) + a.rows - 1) / a.rows);
    s.chunks = max(1, (s.len + (1 << a.log2_keys) - 1) >> a.log2_keys);
    return s;
}
__device__ inline int64_t attn_places(const AttnLaunch& a, const Seq& s) { return int64_t(s.tiles) * a.c.heads * (a.split ? s.chunks : 1); }

// a value that all lanes of the wave have, in a scalar register
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
    return int64_t(uint64_t(uint32_t(uniform(int(x >> 32)))) << 32 | uint32_t(uniform(int(x))));
}

// Memory that no kernel writes while this one runs: uniform reads of it are
// scalar loads, which vector loads in flight do not hold up.
typedef const __attribute__((address_space(4))) int32_t* ConstInts;

// The sequence that holds place p, and (total) the number of places; false past
// the end.  All lanes of a wave call it with the same p.
__device__ inline bool attn_find(const AttnLaunch& a, int64_t p, Seq* out, int64_t* total) {
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    bool found = false;
    for (int base = 0; base < a.num_seqs && (total || !found); base += 64) {
        Seq s = attn_seq(a, base + lane);
        const int64_t own = attn_places(a, s);
        int64_t upto = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int64_t x = __shfl_up((long long)upto, d);
            if (lane >= d) upto += x;
        }
        const unsigned long long past = __ballot(p < before + upto);
        if (past && !found) {
            const int who = __builtin_ctzll(past);
            out->seq = uniform(base + who);
            out->first = uniform(__shfl(s.first, who));
            out->n = uniform(__shfl(s.n, who));
            out->len = uniform(__shfl(s.len, who));
            out->tiles = uniform(__shfl(s.tiles, who));
            out->chunks = uniform(__shfl(s.chunks, who));
            out->before = before + uniform(int64_t(__shfl((long long)(upto - own), who)));
            found = true;
        }
        before += uniform(int64_t(__shfl((long long)upto, 63)));
    }
    if (total) *total = before;
    return found;
}

// Workgroups that share T places: at least kMinChunks chunks each.
constexpr int kMinChunks = 4;
__device__ inline int attn_groups(const AttnLaunch& a, int64_t total) {
    return int(max(int64_t(1), min(int64_t(a.groups), (total + kMinChunks - 1) / kMinChunks)));
}
__device__ inline int attn_group_of(int64_t p, int64_t total, int groups) { return int(((p + 1) * groups - 1) / total); }

// Neighbouring workgroups go to different XCDs in turn: give each XCD one run
// of the line, so that tiles over the same keys meet in one L2.
__device__ inline int attn_by_xcd(int block, int groups) {
    const int q = groups / 8, r = groups % 8, x = block % 8;
    return x * q + min(x, r) + block / 8;
}

// A partial result: rows x D weighted sums, then the rows' maxima, then their
// sums.  The workspace holds two per workgroup, then a note of each workgroup
// about the tile that begins in it and that the workgroups up to 'last' share.
template <int D>
__host__ __device__ constexpr int attn_partial_floats(int rows) { return rows * (D + 2); }
struct AttnShared {
    int first, n, head, tile, last, slot;   // last < 0: none
};
template <int D>
__host__ __device__ constexpr int64_t attn_shared_at(int groups, int rows) { return 2 * int64_t(groups) * attn_partial_floats<D>(rows); }

// Which of a lane's keys j0 + 16 mb + i (mb < MB, i < 4; counted from the first
// new token) the new token 'own' sees, bit 4 mb + i; those from j0 + left on do
// not exist.
template <int MB>
__device__ inline uint32_t attn_seen(const AttnLaunch& a, const Seq& s, int own, int j0, int left) {
    uint32_t seen = 0;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int j = j0 + 16 * mb;
        uint32_t bits = (1u << max(0, min(4, (a.mask ? -1 : own) + 1 - j))) - 1;     // up to itself; in a tree, before it
        if (a.mask) {
            const uint32_t* row = a.mask + int64_t(s.first + own) * a.mask_words;
            const int w = j >> 5;
            const uint64_t lo = w >= 0 && w < a.mask_words ? row[w] : 0u, hi = w + 1 >= 0 && w + 1 < a.mask_words ? row[w + 1] : 0u;
            bits |= uint32_t((hi << 32 | lo) >> (j & 31)) & 15u;
        }
        seen |= (bits & ((1u << max(0, min(4, left - 16 * mb))) - 1)) << (4 * mb);
    }
    return seen;
}

// the first n of a word's bytes, or 16-bit halves
__device__ inline uint32_t attn_first_bytes(int n) { return n <= 0 ? 0u : n >= 4 ? ~0u : (1u << (8 * n)) - 1; }
__device__ inline uint32_t attn_first_halves(int n) { return n <= 0 ? 0u : n >= 2 ? ~0u : 0xffffu; }

// all ones in those of a word's four E4M3 or two bf16 values that are no finite numbers
template <int ELEM>
__device__ inline uint32_t attn_odd(uint32_t w) {
    if (ELEM == 1) return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
    return ((((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
}

// bf16 1 if a bf16 is of a kind: infinity, -infinity, NaN
__device__ inline uint32_t attn_special(uint32_t x, int kind) {
    return (kind == 0 ? x == 0x7f80u : kind == 1 ? x == 0xff80u : (x & 0x7fffu) > 0x7f80u) ? 0x3f80u : 0u;
}

}  // namespace tl
