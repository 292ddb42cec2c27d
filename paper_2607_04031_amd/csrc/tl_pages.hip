// The pages of a key/value cache: handing them out, forking, giving back,
// compacting, and copying what they hold.
//
// Free pages go out in rising order, so that every call has one right answer:
// the pages that nobody refers to become a map of bits, 4096 pages a wave, with
// their number (page_map); the r-th free one is then found by a scan of the
// numbers and one of a block's bits.  What a call hands out it takes from that
// map, so that references may change meanwhile.  Tables and references change by
// exchanges and sums, in whose order nothing depends: every entry of a table
// holds one reference to its page before and after, also where rows are named
// twice.
//
// A call is a chain of phases, each of which needs the one before whole: as
// launches, or, where there is little to do, one after the other in one
// workgroup (a launch costs 2.6 us, a barrier nothing).  Chains of latencies bound
// them, not bytes: a phase is three to six loads or atomics that wait for one another
// (0.5 - 1 us each), and its instructions, which no cache holds yet.  On the GPU,
// us, by phase: fork to 3 children, 25 pages, 6.5; to 448, 15867 pages, 5.0 and 10.2;
// grow of 6 rows, 203 pages, 9.2, of 384 rows, 92670 pages, 5.8 and 7.3; free of 2
// rows 2.2, of 128 rows 3.6; compact of 76 pages 4.4, of 15485 pages, half of them
// in use, 5.1, 7.0 and 4.0.  Copies of that many are at the memory's rate: 64 MB read
// and written in 21.6 us; 4-bit pages have half the bytes of 8-bit ones (8000 of 64
// tokens of a head 19.6 us, 8 bits 34.2; 448 3.8 and 4.3).
// Every row of grow and fork sums what the rows before it want, so that many rows
// take the square of their number: grow and fork of 4096 rows 22 and 21 us, of
// 16384 79 and 112, of 65536 667 and 1149.  A row's pages are found by one wave, 64 at a
// time: those of a prompt of 8192 tokens (128) 15 us, of 32 such 26, of 131072 tokens
// (2048) 194.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {
namespace {

constexpr int kThreads = kPageThreads;
constexpr int kWide = 1024;             // threads of a call that is one workgroup: a wave for each of so many sequences
constexpr int kFewBlocks = 4, kFewRows = 16, kFewEntries = 64;     // blocks of pages; the table's entries, in waves' loads
constexpr int kBlock = kPageBlock;      // pages of a wave's bits: a word of 64 a lane
typedef unsigned long long u64;

// the waves of a phase, and the sums that they take over their lanes
struct Crew {
    int64_t wave, waves;
    int lane;
};
__device__ inline Crew crew() {
    return Crew{int64_t(blockIdx.x) * (blockDim.x / 64) + threadIdx.x / 64, int64_t(gridDim.x) * (blockDim.x / 64), int(threadIdx.x & 63)};
}
// Sum of a list's first n, its loads in flight together.
__device__ inline int64_t sum_of(const int32_t* list, int64_t n, int lane) {
    int64_t sum = 0;
    for (int64_t base = 0; base < n; base += 64 * 4) {
        int x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = base + 64 * j + lane < n ? list[base + 64 * j + lane] : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += x[j];
    }
    return over_lanes(sum);
}

// LDS that a wave's lanes write for one another
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Bits of the free pages, and their number before each word of a block and in
// it, block after block.
__device__ inline void page_map(const PagesLaunch& a, const Crew& w, int64_t first_wave) {
    for (int64_t b = w.wave - first_wave; b < a.blocks; b += w.waves) {
        if (b < 0) continue;
        const int64_t base = b * kBlock;
        u64 mine = 0;
        // sixteen words at a time, the next ones' loads under way; short code, which a call finds in no cache
        int refs[16], next[16];
        auto load = [&](int part, int (&to)[16]) {
#pragma unroll
            for (int j = 0; j < 16; ++j) to[j] = a.refs[min(base + (part * 16 + j) * 64 + w.lane, a.num_pages - 1)];
        };
        load(0, refs);
#pragma unroll 1
        for (int part = 0; part < 4 && base + part * 1024 < a.num_pages; ++part) {
            load(part + 1, next);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const u64 bits = __ballot(refs[j] == 0 && base + (part * 16 + j) * 64 + w.lane < a.num_pages);
                if (w.lane == part * 16 + j) mine = bits;
                refs[j] = next[j];
            }
        }
        const int n = __popcll(mine), upto = upto_lane(n);
        a.map[b * 64 + w.lane] = mine;
        a.before[b * 64 + w.lane] = upto - n;
        if (w.lane == 63) a.free[b] = upto;
    }
}

// Where the r-th free page is, for ever larger r: the block, and the free pages
// before it.
struct PageCursor {
    int64_t block;
    int64_t before;
};
// the first block with the r-th free page in it; a.blocks: there is none
__device__ inline void page_seek(const PagesLaunch& a, const Crew& w, int64_t r, PageCursor* c) {
    while (c->block < a.blocks) {
        const int n = c->block + w.lane < a.blocks ? a.free[c->block + w.lane] : 0;
        const int64_t upto = upto_lane(int64_t(n));
        const u64 past = __ballot(c->before + upto > r);
        if (past) {
            const int at = __builtin_ctzll(past);
            c->before += of_lane(upto - n, at);
            c->block += at;
            return;
        }
        c->before += of_lane(upto, 63);
        c->block += 64;
    }
    c->block = a.blocks;
}
// Free pages of rank [r, r + count), count <= 64, to 'to' in LDS; returns how many there are.
__device__ inline int page_take(const PagesLaunch& a, const Crew& w, int64_t r, int count, PageCursor* c, int32_t* to) {
    int got = 0;
    while (got < count) {
        page_seek(a, w, r + got, c);
        if (c->block >= a.blocks) break;
        u64 bits = a.map[c->block * 64 + w.lane];
        const int n = __popcll(bits);
        int64_t rank = c->before + a.before[c->block * 64 + w.lane];
        const int64_t end = r + count;
        if (rank < end && rank + n > r) {
            for (; bits; bits &= bits - 1, ++rank)
                if (rank >= r && rank < end) to[rank - r] = int32_t(c->block * kBlock + w.lane * 64 + __builtin_ctzll(bits));
        }
        got = int(min(end, c->before + a.free[c->block]) - r);
    }
    wave_sync();
    return got;
}

__device__ inline int pages_of(const PagesLaunch& a, int len) { return int(min(a.max_pages, (int64_t(max(len, 0)) + (1 << a.log2_page) - 1) >> a.log2_page)); }
__device__ inline int32_t* row_of(const PagesLaunch& a, int row) { return row >= 0 && row < a.num_rows ? a.table + row * a.max_pages : nullptr; }
__device__ inline bool is_page(const PagesLaunch& a, int page) { return page >= 0 && page < a.num_pages; }
// a table's entry lets go of a page
__device__ inline void let_go(const PagesLaunch& a, int page) {
    if (is_page(a, page)) atomicSub(&a.refs[page], 1);
}

// grow, first phase: how many entries of each row need a page, and the first of them
__device__ void grow_count(const PagesLaunch& a, const Crew& w) {
    for (int64_t i = w.wave; i < a.n; i += w.waves) {
        const int32_t* row = row_of(a, a.rows[i]);
        const int need = row ? pages_of(a, a.lens[i]) : 0;
        int count = 0, first = need;
        for (int base = 0; base < need; base += 64 * 4) {
            int page[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) page[j] = row[min(base + 64 * j + w.lane, need - 1)];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u64 none = __ballot(page[j] < 0 && base + 64 * j + w.lane < need);
                if (none && first == need) first = base + 64 * j + __builtin_ctzll(none);
                count += __popcll(none);
            }
        }
        if (w.lane == 0) a.want[i] = count, a.first[i] = first;
    }
}
// second phase: the pages
__device__ void grow_give(const PagesLaunch& a, const Crew& w, int32_t* pages) {
    for (int64_t i = w.wave; i < max(a.n, int64_t(1)); i += w.waves) {
        const int want = a.n ? a.want[i] : 0;
        if (want == 0 && i < a.n - 1) continue;
        // the first entries are on their way while the sums are made
        int32_t* row = want ? row_of(a, a.rows[i]) : nullptr;
        const int need = want ? pages_of(a, a.lens[i]) : 0, first = want ? a.first[i] : 0;
        int old = first + w.lane < need ? row[first + w.lane] : 0;
        int64_t rank = sum_of(a.want, i, w.lane);
        if (i >= a.n - 1) {                                 // the last one knows them all
            const int64_t missing = rank + want - sum_of(a.free, a.blocks, w.lane);
            if (w.lane == 0) *a.count = int32_t(min(max(int64_t(0), missing), int64_t(INT32_MAX)));
        }
        PageCursor c{0, 0};
        for (int base = first; base < need; base += 64) {
            if (base > first) old = base + w.lane < need ? row[base + w.lane] : 0;
            const u64 none = __ballot(old < 0);
            if (!none) continue;
            const int got = page_take(a, w, rank, __popcll(none), &c, pages);
            const int mine = __popcll(none & ((1ull << w.lane) - 1));
            // a row that is named twice: the one that comes second leaves its page free
            if (old < 0 && mine < got && atomicCAS(&row[base + w.lane], old, pages[mine]) == old) a.refs[pages[mine]] = 1;
            rank += __popcll(none);
            wave_sync();
            if (got < __popcll(none)) break;
        }
    }
}

// fork, first phase: which children need a page of their own; of the rows that are
// their own parents those whose page another entry names too
__device__ void fork_count(const PagesLaunch& a, const Crew& w) {
    for (int64_t i = w.wave * 64 + w.lane; i < a.n; i += w.waves * 64) {
        const int32_t *from = row_of(a, a.parents[i]), *to = row_of(a, a.rows[i]);
        const int64_t len = min(int64_t(max(a.lens[i], 0)), a.max_pages << a.log2_page), full = len >> a.log2_page;
        const int page = from && to && (len & ((1 << a.log2_page) - 1)) ? from[full] : -1;
        a.want[i] = is_page(a, page) && (from != to || a.refs[page] != 1) ? 1 : 0;
    }
}
// second phase: the children's rows, and the pairs to copy
__device__ void fork_give(const PagesLaunch& a, const Crew& w, int32_t* pages) {
    for (int64_t i = w.wave; i < max(a.n, int64_t(1)); i += w.waves) {
        const int want = a.n ? a.want[i] : 0;
        const int32_t* from = a.n ? row_of(a, a.parents[i]) : nullptr;
        int32_t* to = a.n ? row_of(a, a.rows[i]) : nullptr;
        const int64_t len = from ? min(int64_t(max(a.lens[i], 0)), a.max_pages << a.log2_page) : 0;
        const int full = int(len >> a.log2_page), part = int(len & ((1 << a.log2_page) - 1));
        const bool same = from && from == to;
        // the parent's entries are on their way while the child's own page is found
        int page[8], old = want ? from[full] : -1;
        auto load = [&](int64_t base) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t at = base + 64 * j + w.lane;
                page[j] = at < full + (same && part) ? from[at] : -1;
            }
        };
        load(0);
        const bool last = i >= a.n - 1;
        const int64_t rank = want || last ? sum_of(a.want, i, w.lane) : 0;
        if (last) {
            const int64_t all = rank + want, pairs = min(all, sum_of(a.free, a.blocks, w.lane));
            if (w.lane == 0) a.count[0] = int32_t(pairs), a.count[1] = int32_t(all - pairs);
            for (int64_t j = pairs + w.lane; j < a.n; j += 64) a.src[j] = a.dst[j] = a.tokens[j] = -1;
        }
        if (!to) continue;
        const int kept = full + (same && part && !want);    // entries that go on as they are
        int own = -1;
        if (want) {
            PageCursor c{0, 0};
            const bool found = page_take(a, w, rank, 1, &c, pages);
            if (found) own = pages[0];
            else if (same && is_page(a, old)) own = old;    // shared as before: nothing of the row is lost
            wave_sync();
            if (found && w.lane == 0) {
                a.src[rank] = old;
                a.dst[rank] = own;
                a.tokens[rank] = part;
            }
            if (own >= 0 && w.lane == 0) atomicAdd(&a.refs[own], 1);
        }
        for (int64_t base = 0; base < a.max_pages; base += 64 * 8) {
            if (base) load(base);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t at = base + 64 * j + w.lane;
                if (at >= a.max_pages) break;
                const bool shared = at < kept && is_page(a, page[j]);
                if (shared) atomicAdd(&a.refs[page[j]], 1);
                page[j] = atomicExch(&to[at], shared ? page[j] : at == full ? own : -1);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (base + 64 * j + w.lane < a.max_pages) let_go(a, page[j]);
        }
    }
}

// compact, second phase: of U pages in use, the M that lie behind the first U
// pages, from the last one on, go to the free ones among those, from the first
// one on.  With f(p) free pages before p, page p is the (U - 1 - (p - f(p)))-th
// in use from the end.  A wave takes a quarter of a block, a page a lane; what
// it leaves in 'before' counts from the first page on.
__device__ void compact_list(const PagesLaunch& a, const Crew& w) {
    const int64_t used = a.num_pages - sum_of(a.free, a.blocks, w.lane), at_used = used / kBlock;   // the block of page U
    const int64_t before_used = sum_of(a.free, min(at_used, a.blocks), w.lane);
    int rest = 0;
    if (at_used < a.blocks) {
        const int64_t left = used - at_used * kBlock - w.lane * 64;     // pages of this lane's word before page U
        rest = __popcll(a.map[at_used * 64 + w.lane] & (left <= 0 ? 0 : left >= 64 ? ~0ull : (1ull << left) - 1));
    }
    const int64_t moves = min(before_used + over_lanes(rest), a.n);
    if (w.wave == 0 && w.lane == 0) a.count[0] = int32_t(moves), a.count[1] = int32_t(used);
    for (int64_t k = moves + w.wave * 64 + w.lane; k < a.n; k += w.waves * 64) a.src[k] = a.dst[k] = -1;
    for (int64_t item = w.wave; item < a.blocks * 4; item += w.waves) {
        // a word a lane, the numbers before them counted from the first page on
        const int64_t mine = item * 16 + (w.lane & 15);
        const u64 word = a.map[mine];
        const int before = int(sum_of(a.free, item / 4, w.lane)) + a.before[mine];
        wave_sync();
        if (w.lane < 16) a.before[mine] = before;
#pragma unroll 1
        for (int j = 0; j < 16 && (item * 16 + j) * 64 < a.num_pages; ++j) {
            const u64 bits = u64(of_lane(int64_t(word), j));
            const int64_t page = (item * 16 + j) * 64 + w.lane, f = of_lane(before, j) + __popcll(bits & ((1ull << w.lane) - 1));
            const int64_t k = used - 1 - (page - f);
            if (bits >> w.lane & 1) {
                if (page < used && f < moves) a.dst[f] = int32_t(page);
            } else if (page >= used && page < a.num_pages && k < moves) {
                a.src[k] = int32_t(page);
            }
        }
    }
}
// third phase: references and tables follow
__device__ void compact_apply(const PagesLaunch& a, const Crew& w) {
    const int64_t moves = a.count[0], used = a.count[1], thread = w.wave * 64 + w.lane, threads = w.waves * 64;
#pragma unroll 1
    for (int64_t k = thread; k < moves; k += threads) {
        const int src = a.src[k], dst = a.dst[k];
        a.refs[dst] = a.refs[src];
        a.refs[src] = 0;
    }
    const int64_t entries = int64_t(a.num_rows) * a.max_pages;
#pragma unroll 1
    for (int64_t i = thread; i < entries; i += threads) {
        const int page = a.table[i];
        if (page < used || page >= a.num_pages) continue;
        const u64 bits = a.map[page / 64], bit = 1ull << (page % 64);
        const int64_t k = used - 1 - (page - (a.before[page / 64] + __popcll(bits & (bit - 1))));
        if (!(bits & bit) && k < moves) a.table[i] = a.dst[k];
    }
}

// what the phases before wrote is there for those after, in one workgroup
__device__ inline void next_phase() {
    __threadfence_block();
    __syncthreads();
}

template <int OP, int PHASE>       // PHASE 0: all of them, whose notes to one another stay in LDS
__global__ __launch_bounds__(PHASE ? kThreads : kWide) void pages_kernel(PagesLaunch a) {
    __shared__ int32_t pages_s[(PHASE ? kThreads : kWide) / 64][64];
    __shared__ u64 map_s[PHASE ? 1 : kFewBlocks * 64];
    __shared__ int32_t before_s[PHASE ? 1 : kFewBlocks * 64], free_s[PHASE ? 1 : kFewBlocks], want_s[PHASE ? 1 : kFewRows], first_s[PHASE ? 1 : kFewRows];
    const Crew w = crew();
    int32_t* pages = pages_s[threadIdx.x / 64];
    if (PHASE == 0) a.map = map_s, a.before = before_s, a.free = free_s, a.want = want_s, a.first = first_s;
    if (PHASE <= 1) {
        if (OP == kPagesGrow) grow_count(a, w);
        if (OP == kPagesFork) fork_count(a, w);
        page_map(a, w, PHASE == 1 ? a.map_wave : 0);
    }
    if (PHASE == 0) next_phase();
    if (PHASE == 0 || PHASE == 2) {
        if (OP == kPagesGrow) grow_give(a, w, pages);
        if (OP == kPagesFork) fork_give(a, w, pages);
        if (OP == kPagesCompact) compact_list(a, w);
    }
    if (PHASE == 0 && OP == kPagesCompact) next_phase();
    if ((PHASE == 0 || PHASE == 3) && OP == kPagesCompact) compact_apply(a, w);
}

// free: a row's entries from the len-th token's page on, 64 at a time
__global__ __launch_bounds__(kThreads) void pages_free_kernel(PagesLaunch a, int parts) {
    const Crew w = crew();
    const int64_t i = w.wave / parts;
    if (i >= a.n) return;
    int32_t* row = row_of(a, a.rows[i]);
    if (!row) return;
    const int64_t at = (a.lens ? pages_of(a, a.lens[i]) : 0) + (w.wave - i * parts) * 64 + w.lane;
    for (int64_t j = at; j < a.max_pages; j += int64_t(parts) * 64) let_go(a, atomicExch(&row[j], -1));
}

// ---------------------------------------------------------------------------
// copy: a workgroup takes 64 tokens of a head of a pair of pages, one run of
// bytes in each of the cache's arrays.
// ---------------------------------------------------------------------------
template <int BYTES, int EXPS>      // of a token's head: of keys (and of values), and their exponents
__global__ __launch_bounds__(kThreads) void pages_copy_kernel(PagesCopyLaunch a) {
    constexpr int kChunks = 64 * BYTES / 16, kLoads = (kChunks + kThreads - 1) / kThreads;
    const int log2_groups = a.c.log2_page - 6, per = a.c.heads << log2_groups;
    const int64_t count = a.count ? *a.count : a.pairs;
    for (int64_t u = blockIdx.x; u < a.pairs * per; u += gridDim.x) {
        const int64_t pair = quotient(u, per);
        const int rest = int(u - pair * per), group = rest & ((1 << log2_groups) - 1);
        // the pair is loaded while it is not known yet whether it is one
        const int64_t src = a.src[pair], dst = a.dst[pair];
        const int tokens = a.tokens ? a.tokens[pair] : 1 << a.c.log2_page;
        if (pair >= count) break;
        if (src < 0 || src >= a.c.num_pages || dst < 0 || dst >= a.c.num_pages || src == dst || group * 64 >= tokens) continue;
        const int64_t from = (src * per + rest) * 64, to = (dst * per + rest) * 64;        // tokens of one head
        const u32x4 *k0 = reinterpret_cast<const u32x4*>(a.c.k + from * BYTES), *v0 = reinterpret_cast<const u32x4*>(a.c.v + from * BYTES);
        u32x4 *k1 = reinterpret_cast<u32x4*>(a.c.k + to * BYTES), *v1 = reinterpret_cast<u32x4*>(a.c.v + to * BYTES);
        u32x4 k[kLoads], v[kLoads], e = {0, 0, 0, 0};
        // exponents: 4 EXPS chunks of the keys', then of the values'
        const int chunk = threadIdx.x % (EXPS ? 4 * EXPS : 1), which = threadIdx.x / (EXPS ? 4 * EXPS : 1);
        uint8_t* exps = which ? a.c.v_exp : a.c.k_exp;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = i * kThreads + threadIdx.x;
            if (kChunks % kThreads && x >= kChunks) break;
            k[i] = k0[x], v[i] = v0[x];
        }
        if (EXPS && which < 2) e = reinterpret_cast<const u32x4*>(exps + from * EXPS)[chunk];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = i * kThreads + threadIdx.x;
            if (kChunks % kThreads && x >= kChunks) break;
            k1[x] = k[i], v1[x] = v[i];
        }
        if (EXPS && which < 2) reinterpret_cast<u32x4*>(exps + to * EXPS)[chunk] = e;
    }
}

uint32_t groups_of(int64_t waves) { return uint32_t(std::max<int64_t>(1, (waves + kThreads / 64 - 1) / (kThreads / 64))); }

template <int OP>
hipError_t launch_phases(const PagesLaunch& given, int64_t first, int64_t second, int64_t third, hipStream_t stream) {
    PagesLaunch a = given;
    // One workgroup of sixteen waves where each has a block, a sequence and a few entries at most.  As one workgroup and as
    // launches, us: grow of 1000 pages, 16 rows 4.3 and 5.0, 64 rows 6.4 and 5.3; of 16000, 6.6 and 7.1, 8.6 and 7.5; of
    // 60000, 16 rows, 11.4 and 7.3.  fork of 1000 pages, 4 rows 7.6 and 8.6, 64 rows 34 and 11.8; of 16000, 16 rows 12.7 and
    // 12.5; of 60000 17.3 and 12.5.  compact of 1000 pages, 4096 entries 11.2 and 13.9, 8192 entries 12.4 and 14.0, 16384 15.3
    // and 14.0; of 16000 pages 18.4 and 18.7, 22.2 and 18.4, 24.7 and 18.6; of 60000, 512 entries, 30 and 17.
    if (a.blocks <= kFewBlocks && second <= kFewRows && third <= kFewEntries) {
        hipLaunchKernelGGL((pages_kernel<OP, 0>), dim3(1), dim3(kWide), 0, stream, a);
        return hipGetLastError();
    }
    a.map_wave = first;
    hipLaunchKernelGGL((pages_kernel<OP, 1>), dim3(groups_of(first + a.blocks)), dim3(kThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((pages_kernel<OP, 2>), dim3(groups_of(second)), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess || !third) return e;
    hipLaunchKernelGGL((pages_kernel<OP, 3>), dim3(groups_of(std::min<int64_t>(third, 4096))), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_grow(const PagesLaunch& a, hipStream_t stream) { return launch_phases<kPagesGrow>(a, a.n, a.n, 0, stream); }
hipError_t launch_pages_fork(const PagesLaunch& a, hipStream_t stream) { return launch_phases<kPagesFork>(a, (a.n + 63) / 64, a.n, 0, stream); }
hipError_t launch_pages_compact(const PagesLaunch& a, hipStream_t stream) {
    return launch_phases<kPagesCompact>(a, 0, a.blocks * 4, std::max((int64_t(a.num_rows) * a.max_pages + 63) / 64, (a.n + 63) / 64), stream);
}

hipError_t launch_pages_free(const PagesLaunch& a, hipStream_t stream) {
    // entries of a row for a wave: 64, and more than that only where the launch would be too large
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((a.max_pages + 63) / 64, (int64_t(1) << 22) / a.n));
    hipLaunchKernelGGL(pages_free_kernel, dim3(groups_of(a.n * parts)), dim3(kThreads), 0, stream, a, int(parts));
    return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyLaunch& a, int head_dim, int elem_bytes, hipStream_t stream) {
    const int64_t units = a.pairs * a.c.heads << (a.c.log2_page - 6);
    return kv_as(head_dim, elem_bytes, [&](auto d, auto e) {
        constexpr int D = d(), E = e();
        hipLaunchKernelGGL((pages_copy_kernel<kv_width<D, E>() * kv_size<E>(), kv_exps<D, E>()>), dim3(uint32_t(std::min<int64_t>(units, 2048))),
                           dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    });
}

}  // namespace tl
