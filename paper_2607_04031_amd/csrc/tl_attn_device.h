// Shared by the attention kernels: how the work is laid out over workgroups,
// and the joining of partial results.
#pragma once

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {

__device__ inline f32x4v mfma_16x16x32(u32x4 a, u32x4 b, f32x4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, a), __builtin_bit_cast(bf16x8v, b), c, 0, 0, 0);
}

// Waits for the loads so far.  Before a loop that keeps loads in flight: where
// registers loaded ahead of it (the queries) are still on their way at its
// entry, the compiler has every pass through it wait for all loads instead.
__device__ inline void wait_for_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }    // vmcnt 0

// The same before reads of LDS that such loads write past the registers: the
// statement says that memory is another one, so that no read moves before the
// wait, whatever the builtin is taken to touch.
__device__ inline void wait_for_lds_loads() {
    wait_for_loads();
    asm volatile("" ::: "memory");
}

// The work is a line: sequence after sequence, in it head after head, in it
// tile after tile of rows.  Without a split a workgroup takes one tile of a
// head.  With one, a tile takes as many places as it costs, in sixteenths of a
// chunk of keys: its chunks and kTileCost for its start and end, a causal
// tile's chunks rising evenly from one tile to the next.  Workgroup w of W
// takes the places [w T / W, (w + 1) T / W) of all T and of each tile the
// chunks in proportion, so that all have the same to do whatever the lengths
// are; what it has of a tile that it does not hold whole it writes as a partial
// result: of the first tile in its slot 2 w, of the last in 2 w + 1.
constexpr int kTileCost = 96;
struct Seq {
    int seq, first, n, len;     // first: row of the first new token; n: new tokens; len: keys
    int rows;                   // new tokens that are computed: those within the caller's bound
    int tiles;                  // of rows
    int cost, rise;             // places of tile t: cost + (t + 1) rise
    int64_t before;             // places before the sequence
};

// the new token of a row: row / group
__device__ inline int attn_token(const AttnLaunch& a, int row) { return int((__umulhi(uint32_t(row), a.group_magic) + uint32_t(row)) >> a.group_shift); }

__device__ inline int attn_offset(const AttnLaunch& a, int i) { return max(0, min(a.q_offsets[i], int(a.total_q))); }

// a value that all lanes of the wave have, in a scalar register
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
    return int64_t(uint64_t(uint32_t(uniform(int(x >> 32)))) << 32 | uint32_t(uniform(int(x))));
}

// a / b of a >= 0, b > 0 below 2^53 by way of a double: a sixth of the
// instructions of a 64-bit integer division
__device__ inline int64_t quotient(int64_t a, int64_t b) {
    const int64_t q = int64_t(double(a) / double(b)), r = a - q * b;
    return q + (r >= b) - (r < 0);
}

// Memory that no kernel writes while this one runs: uniform reads of it are
// scalar loads, which vector loads in flight do not hold up.
typedef const __attribute__((address_space(4))) int32_t* ConstInts;

// What a workgroup knows of the line: up to 64 sequences are scanned once, and
// kept here; more are scanned again for every piece (a token each over up to
// 2048, 64 heads over 8: 64 sequences 34.4 us, 65 38.9, 256 124).
struct AttnLine {
    int first[64], n[64], len[64];
    int64_t upto[64];
};

__device__ inline void attn_sizes(const AttnLaunch& a, Seq* s) {
    s->rows = int(min(int64_t(s->n), a.max_q));      // the launch has workgroups for no more
    s->tiles = int((int64_t(s->rows) * a.group + (1 << a.log2_rows) - 1) >> a.log2_rows);
    const bool rises = !a.mask && s->tiles > 1;
    s->rise = rises ? attn_token(a, 16 << a.log2_rows) >> a.log2_keys : 0;
    s->cost = (((rises ? max(0, s->len - s->n) : s->len) + (1 << a.log2_keys) - 1) >> a.log2_keys) * 16 + kTileCost;
}
// places of the first t tiles of a head
__device__ inline int64_t attn_cost(const Seq& s, int t) { return int64_t(s.cost) * t + int64_t(s.rise) * t * (t + 1) / 2; }
// the tile at place y of a head
__device__ inline int attn_tile_at(const Seq& s, int64_t y) {
    if (!s.rise) return int(quotient(y, s.cost));
    const double b = s.cost + 0.5 * s.rise;
    int t = max(0, min(s.tiles - 1, int((sqrt(b * b + 2.0 * s.rise * double(y)) - b) / s.rise)));
    while (t > 0 && attn_cost(s, t) > y) --t;
    while (t < s.tiles - 1 && attn_cost(s, t + 1) <= y) ++t;
    return t;
}
__device__ inline int64_t attn_places(const AttnLaunch& a, const Seq& s) { return a.c.heads * (a.split ? attn_cost(s, s.tiles) : s.tiles); }

// Sequences base .. base + 63, one a lane: *upto gets the places up to each one's end.
__device__ inline Seq attn_scan(const AttnLaunch& a, int base, int64_t* upto) {
    Seq s{};
    const int lane = threadIdx.x & 63, b = base + lane;
    if (b < a.num_seqs) {
        const int to = attn_offset(a, b + 1), len = a.lens[b];
        s.first = attn_offset(a, b);
        s.n = max(0, to - s.first);
        s.len = int(max(int64_t(0), min(int64_t(len), min(a.max_pages << a.c.log2_page, a.max_len))));
        attn_sizes(a, &s);
    }
    *upto = b < a.num_seqs ? attn_places(a, s) : 0;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t x = __shfl_up((long long)*upto, d);
        if (lane >= d) *upto += x;
    }
    return s;
}

// The number of places; every wave calls it and keeps what it found in 'line'.
__device__ inline int64_t attn_total(const AttnLaunch& a, AttnLine* line) {
    int64_t before = 0, upto;
    for (int base = 0; base < a.num_seqs; base += 64) {
        const Seq s = attn_scan(a, base, &upto);
        if (a.num_seqs <= 64) {     // all waves write the same, and each reads what it wrote
            const int lane = threadIdx.x & 63;
            line->first[lane] = s.first;
            line->n[lane] = s.n;
            line->len[lane] = s.len;
            line->upto[lane] = upto;
        }
        before += uniform(int64_t(__shfl((long long)upto, 63)));
    }
    return before;
}

// The sequence that holds place p (below the total).
__device__ inline Seq attn_find(const AttnLaunch& a, const AttnLine* line, int64_t p) {
    const int lane = threadIdx.x & 63;
    Seq s{};
    int64_t before = 0;
    if (a.num_seqs <= 64) {
        const int who = uniform(__builtin_ctzll(__ballot(p < line->upto[lane]) | 1ull << 63));
        s.seq = who;
        s.first = uniform(line->first[who]);
        s.n = uniform(line->n[who]);
        s.len = uniform(line->len[who]);
        s.before = who ? uniform(line->upto[who - 1]) : 0;
    } else {
        for (int base = 0; base < a.num_seqs; base += 64) {
            int64_t upto;
            const Seq x = attn_scan(a, base, &upto);
            const unsigned long long past = __ballot(p < before + upto);
            if (past) {
                const int who = uniform(__builtin_ctzll(past));
                s.seq = base + who;
                s.first = uniform(__shfl(x.first, who));
                s.n = uniform(__shfl(x.n, who));
                s.len = uniform(__shfl(x.len, who));
                s.before = before + (who ? uniform(int64_t(__shfl((long long)upto, who - 1))) : 0);
                break;
            }
            before += uniform(int64_t(__shfl((long long)upto, 63)));
        }
    }
    attn_sizes(a, &s);
    return s;
}

// Workgroups that share T places: at least kMinCost of them each (one token of
// 64 heads over 8 and 8192 8-bit keys: 15.0 us; with 4 * 16 or 8 * 16 of chunks
// 15.9 and 16.8).  Where it takes away few of them, or of one sequence, a
// multiple of the tiles, so that tiles of one length end where workgroups do: a
// second piece costs a workgroup 4 us (three tokens over 1100: 16.9 and 22.5).
// Only one sequence's tiles are all of one length: of two to four ragged ones a
// multiple of the tiles ends nowhere in particular, and fewer workgroups are no
// faster (four tokens over 2500: one 19.1 and 24.5, four 23.7 and 23.2).
constexpr int kMinCost = 2 * 16 + kTileCost;
__device__ inline int attn_groups(const AttnLaunch& a, int64_t total) {
    const int most = int(max(int64_t(1), min(int64_t(a.groups), (total + kMinCost - 1) / kMinCost)));
    const int tiles = int(min(a.max_tiles, int64_t(most))), even = most / tiles * tiles;
    return even >= most - most / 8 || (a.num_seqs == 1 && most >= 2 * tiles) ? even : most;
}
__device__ inline int attn_group_of(int64_t p, int64_t total, int groups) { return int(quotient((p + 1) * groups - 1, total)); }

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
    int first, rows, head, tile, last, slot;    // last < 0: none
};
template <int D>
__host__ __device__ constexpr int64_t attn_shared_at(int groups, int rows) { return 2 * int64_t(groups) * attn_partial_floats<D>(rows); }

// A workgroup's run of the line, piece by piece.
struct AttnRun {
    int64_t place0, place, end, total;
    int groups, me;
};
template <int D>
__device__ inline AttnShared* attn_shared(const AttnLaunch& a) { return reinterpret_cast<AttnShared*>(a.ws + attn_shared_at<D>(a.groups, 1 << a.log2_rows)); }

// false: the workgroup has nothing to do
template <int D>
__device__ inline bool attn_begin(const AttnLaunch& a, AttnLine* line, AttnRun* r) {
    r->total = attn_total(a, line);
    r->groups = a.groups;
    r->me = blockIdx.x;
    if (a.split) {
        r->groups = attn_groups(a, r->total);
        const bool idle = r->me >= r->groups;
        if (!idle) r->me = attn_by_xcd(r->me, r->groups);
        if (threadIdx.x == 0) attn_shared<D>(a)[r->me].last = -1;
        if (idle) return false;
        r->place = uniform(quotient(r->me * r->total, r->groups));
        r->end = uniform(quotient((r->me + 1) * r->total, r->groups));
    } else {
        if (r->me >= r->total) return false;
        r->place = r->me = attn_by_xcd(r->me, int(r->total));
        r->end = r->place + 1;
    }
    r->place0 = r->place;
    return r->place < r->end;
}

// The piece that begins at r->place: chunks [chunk0, chunk1) of a tile of a head.
struct AttnPiece {
    Seq s;
    int head, tile, chunk0, chunk1;
    bool whole;
    int64_t slot;       // of its partial result, if it is not the whole tile
};
template <int D>
__device__ inline AttnPiece attn_piece(const AttnLaunch& a, const AttnLine* line, AttnRun* r) {
    AttnPiece p;
    p.s = attn_find(a, line, r->place);
    const int64_t in_seq = r->place - p.s.before;
    if (a.split) {
        const int64_t per_head = attn_cost(p.s, p.s.tiles);
        p.head = uniform(int(quotient(in_seq, per_head)));
        p.tile = uniform(attn_tile_at(p.s, in_seq - p.head * per_head));
    } else {
        p.head = uniform(int(quotient(in_seq, p.s.tiles)));
        p.tile = p.s.tiles - 1 - uniform(int(in_seq - int64_t(p.head) * p.s.tiles));    // the longest first
    }
    // chunks that some row of the tile sees
    const int last = min(p.s.rows - 1, attn_token(a, ((p.tile + 1) << a.log2_rows) - 1));
    const int end = a.mask ? p.s.len : max(0, min(p.s.len, p.s.len - p.s.n + last + 1));
    const int chunks = (end + (1 << a.log2_keys) - 1) >> a.log2_keys;
    p.chunk0 = 0;
    p.chunk1 = chunks;
    p.whole = true;
    p.slot = 0;
    if (!a.split) {
        ++r->place;
        return p;
    }
    const int64_t start = p.s.before + p.head * attn_cost(p.s, p.s.tiles) + attn_cost(p.s, p.tile), places = p.s.cost + int64_t(p.tile + 1) * p.s.rise;
    const int64_t to = min(places, r->end - start);
    p.chunk0 = r->place == start ? 0 : uniform(int(quotient(chunks * (r->place - start), places)));
    p.chunk1 = to == places ? chunks : uniform(int(quotient(chunks * to, places)));
    p.whole = r->place == start && to == places;
    p.slot = 2 * int64_t(r->me) + (start > r->place0 ? 1 : 0);
    r->place = start + to;
    if (start >= r->place0 && to < places && threadIdx.x == 0)      // others go on with it
        attn_shared<D>(a)[r->me] = AttnShared{p.s.first, p.s.rows, p.head, p.tile, attn_group_of(start + places - 1, r->total, r->groups), int(p.slot)};
    return p;
}

// The key that a chunk begins with in the pool, in tokens; negative: a page that is none.
struct AttnPages {
    ConstInts table;
    int num_pages, page_tokens, head_at, in_page, log2_chunks, keys;
    __device__ AttnPages(const AttnLaunch& a, int seq, int head)
        : table(ConstInts(a.page_table + int64_t(seq) * a.max_pages)), num_pages(int(a.c.num_pages)), page_tokens(a.c.heads << a.c.log2_page),
          head_at(head << a.c.log2_page), in_page((1 << (a.c.log2_page - a.log2_keys)) - 1), log2_chunks(a.c.log2_page - a.log2_keys), keys(1 << a.log2_keys) {}
    __device__ int page(int chunk, int before) const { return chunk < before ? table[chunk >> log2_chunks] : -1; }
    __device__ int64_t block(int chunk, int page) const {
        return page < 0 || page >= num_pages ? -1 : int64_t(page) * page_tokens + (head_at + (chunk & in_page) * keys);
    }
};

// Eight of a row's results, from d on: weighted sums o, their sum of weights l at the maximum m.
template <int D>
__device__ inline void attn_put(const AttnLaunch& a, const AttnPiece& p, int row, int d, const float (&o)[8], float m, float l) {
    const int rows = 1 << a.log2_rows, at = (p.tile << a.log2_rows) + row, i = attn_token(a, at);
    if (i >= p.s.rows) return;
    if (p.whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;    // a row that sees no key: zeros
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16(o[2 * j] * inv, o[2 * j + 1] * inv);
        *reinterpret_cast<u32x4*>(a.out + (int64_t(p.s.first + i) * a.q_heads + p.head * a.group + at - i * a.group) * D + d) = w;
    } else {
        float* part = a.ws + p.slot * attn_partial_floats<D>(rows);
#pragma unroll
        for (int j = 0; j < 8; j += 4) *reinterpret_cast<f32x4v*>(part + row * D + d + j) = f32x4v{o[j], o[j + 1], o[j + 2], o[j + 3]};
        if (d == 0) {
            part[rows * D + row] = m;
            part[rows * D + rows + row] = l;
        }
    }
}

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

// 1 in those of a word's bytes that are 0xff: less that, they are scales of
// 2^127 and not of infinity, of which 0 times is 0.  No entry that was written
// has such a scale; one that was not may have any, and rows need not see it.
__device__ inline uint32_t attn_full_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & w & 0x80808080u) >> 7; }

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

// Infinities and NaNs among the values of chunk c (at 'block' in the pool), for
// the row 'row' of the tile in each of a wave's 16 columns: one kind at a time,
// to the rows that see one.  odd: rows x D / 8 words, 4 bits an element
// (infinity, -infinity, NaN).
template <int D, int ELEM, int MB>
__device__ inline void attn_odd_chunk(const AttnLaunch& a, const AttnPiece& p, int c, int64_t block, int row, uint32_t* odd) {
    const int lane = threadIdx.x & 63, g = lane >> 4, i = attn_token(a, (p.tile << a.log2_rows) + row);
    const int key0 = c * (16 * MB) + 4 * g, left = p.s.len - key0;
    const uint32_t seen = i < p.s.rows ? attn_seen<MB>(a, p.s, i, key0 - (p.s.len - p.s.n), left) : 0u;
#pragma unroll 1
    for (int step = 0; step < 3 * (D / 16) * (MB / 2); ++step) {
        const int kind = step % 3, db = step / 3 % (D / 16), h = step / 3 / (D / 16);
        constexpr int per = 16 / ELEM * 4 / 32;     // 32-key steps of a load: 2 (8 bits) or 1
        u32x4 vf = reinterpret_cast<const u32x4*>(a.c.v + block * (D * ELEM))[(h / per * (D / 16) + db) * 64 + lane], is, ones;
        if (ELEM == 1) {
            const uint32_t lo = h ? vf[2] : vf[0], hi = h ? vf[3] : vf[1];
            vf = u32x4{fp8_to_bf16<false>(lo, 1.f), fp8_to_bf16<true>(lo, 1.f), fp8_to_bf16<false>(hi, 1.f), fp8_to_bf16<true>(hi, 1.f)};
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            vf[j] &= attn_first_halves(left - 32 * h - 16 * (j >> 1) - 2 * (j & 1));
            is[j] = attn_special(vf[j] & 0xffffu, kind) | attn_special(vf[j] >> 16, kind) << 16;
            const uint32_t two = seen >> (8 * h + 2 * j);
            ones[j] = (two & 1 ? 0x3f80u : 0u) | (two & 2 ? 0x3f800000u : 0u);
        }
        const f32x4v hits = mfma_16x16x32(is, ones, f32x4v{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int j = 0; j < 4; ++j)     // elements 16 db + 4 g + j of the row: 4 bits each
            if (hits[j] > 0.f) atomicOr(&odd[row * (D / 8) + db * 2 + (g >> 1)], 1u << (16 * (g & 1) + 4 * j + kind));
    }
}

__device__ inline void attn_add_odd(uint32_t odd, float (&o)[8]) {
    for (int j = 0; j < 8; ++j) {
        if (odd >> (4 * j) & 1) o[j] += INFINITY;
        if (odd >> (4 * j) & 2) o[j] -= INFINITY;
        if (odd >> (4 * j) & 4) o[j] = NAN;
    }
}

}  // namespace tl
