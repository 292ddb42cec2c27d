// Verification of drafted tokens.  Three launches:
//   stats   every node's logits row, in ranges: maximum (and where it is first)
//           and sum of exponentials -- all the bytes there are to read, so this
//           is bound by HBM where the rows are many
//   walk    a workgroup per sequence goes from the root to an accepted child
//           while there is one.  Against a draft's distribution, each rejected
//           child but a node's last costs a pass over the vocabulary, which one
//           CU takes 13 us for at 131072 tokens (its vector units bound it), so
//           that further workgroups of the sequence take parts of it (8 trees
//           of 32 nodes, a call: 71.7 us with 4 of them, 59.3 with 8, 54.1 with 16)
//   sample  the last node's distribution less what its rejected children took,
//           in ranges: the token with the largest ratio of weight to noise (an
//           exponential race: P(token wins) is proportional to its weight)
// Row ranges are joined in their order, and the race's winner does not depend
// on it, so results are the same from call to call.
//
// 32 trees of up to 24 nodes over 131072 tokens, bf16 logits, fp32 draft: 29 us
// (4.3 TB/s), 30 and 16; a chain of five over 50257: 4, 5 and 9, latencies.
#include <hip/hip_runtime.h>

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {
namespace {

constexpr int kThreads = 256;
constexpr int kWalkThreads = 1024;
constexpr int kAtOnce = 8;                          // elements of a lane's load
constexpr int kMinRange = kThreads * kAtOnce;       // one load of each lane
constexpr int kMaxRanges = 64;                      // one lane joins each
constexpr int kMaxParts = 64;                       // of a pass over the vocabulary in the walk; one lane joins each
constexpr int kWalkers = 16;                        // workgroups of a sequence in the walk, at most
constexpr int kMaxPolls = 1 << 16;                  // of a helper that waits for work
constexpr float kLog2e = 1.44269504088896340736f;

struct RowStat {
    float top, sum;     // maximum; sum of 2^((z - top) c)
    int first;          // the first index of the maximum
    int pad;
};
struct Last {           // what walk leaves for sample
    int row;            // node's row, -1: a sequence without nodes
    int tried;          // children that were tried and rejected
    float top, sum;
    int first;
    unsigned arrived;
};
// What a walk's workgroups share.  The first one leads: it writes down a pass and opens its parts by 'claim'; whoever
// adds to that takes a part, the leader too, and leaves its sum.  The leader waits for parts that were taken only, and a
// helper for the leader no longer than kMaxPolls looks, so that no wait depends on which workgroups run at once.
struct Pass {
    int row, tried;     // a node's row; rejected children so far
    float top, sum;
    int first;
    unsigned claim;     // pass << 8 | next part; kNoPart: none yet; kOver: the walk has ended
    unsigned taken;     // parts done, of all passes
    int pad;
};
constexpr unsigned kNoPart = 0x80, kOver = 0xffffff80u;   // their parts: past the last by far, and far from the byte's end
static_assert(kMaxParts + 2 * kWalkers < 0x80, "a pass that everybody adds to once too often");
struct Best {           // largest weight / noise of what is left, and of the whole distribution
    float rest;
    int rest_at;
    float all;
    int all_at;
};
typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));

struct Params {
    VerifyLaunch a;
    int ranges, sample_ranges;      // of a row, in stats and in sample
    int64_t range, sample_range;    // their elements, multiples of kMinRange
    RowStat* stats;     // [total][ranges]
    int parts;          // of a pass over the vocabulary in the walk
    int64_t part;       // their elements, a multiple of kWalkThreads * kAtOnce
    int walkers;        // workgroups of a sequence in the walk
    Last* last;         // [num_seqs]
    Pass* pass;         // [num_seqs]
    float* sums;        // [num_seqs][kMaxParts]
    Best* best;         // [num_seqs][sample_ranges]
    float* mass;        // [num_seqs][max_nodes]: 1 / sum left before each tried child
    int32_t* tried;     // [num_seqs][max_nodes]: the tried children's tokens
};

template <typename T>
__device__ inline void put_through(T* to, T x) { __hip_atomic_store(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ inline T read_past(const T* from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// what was written through before is where others read it
__device__ inline void wait_for_stores() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ inline int offset_of(const VerifyLaunch& a, int i) { return max(0, min(a.offsets[i], int(a.total))); }

// 2^((z - top) c) is the softmax's numerator
__device__ inline float rate_of(float temperature) { return temperature > 0.f ? fminf(1.f / temperature, 1e38f) * kLog2e : 0.f; }

template <bool BF16>
__device__ inline float load_one(const void* p, int64_t at) {
    if (BF16) return __uint_as_float(uint32_t(static_cast<const uint16_t*>(p)[at]) << 16);
    return static_cast<const float*>(p)[at];
}

// eight elements from any element's address
template <bool BF16>
__device__ inline void load_eight(const void* p, int64_t at, float (&x)[8]) {
    if (BF16) {
        u32x4 w;
        __builtin_memcpy(&w, static_cast<const uint16_t*>(p) + at, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[2 * j] = bf16_lo(w[j]), x[2 * j + 1] = bf16_hi(w[j]);
    } else {
        __builtin_memcpy(x, static_cast<const float*>(p) + at, 32);
    }
}
template <bool BF16>
__device__ inline void load_some(const void* p, int64_t at, int some, float fill, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < some ? load_one<BF16>(p, at + j) : fill;
}

__device__ inline void take(float& v, int& at, float w, int j) {
    if (w > v || (w == v && j < at)) v = w, at = j;
}

__device__ inline RowStat join(const RowStat& x, const RowStat& y, float c) {
    RowStat r;
    r.top = fmaxf(x.top, y.top);
    r.first = x.top > y.top ? x.first : y.top > x.top ? y.first : min(x.first, y.first);
    const float base = r.top == -INFINITY ? 0.f : r.top;
    r.sum = (x.sum != 0.f ? x.sum * __builtin_amdgcn_exp2f((x.top - base) * c) : 0.f) +
            (y.sum != 0.f ? y.sum * __builtin_amdgcn_exp2f((y.top - base) * c) : 0.f);
    r.pad = 0;
    return r;
}

__device__ inline RowStat shuffled(const RowStat& x, int m) {
    return RowStat{__shfl_xor(x.top, m), __shfl_xor(x.sum, m), __shfl_xor(x.first, m), 0};
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(Params p) {
    __shared__ RowStat part[kThreads / 64];
    if (p.walkers > 1) {
        for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < p.a.num_seqs; i += int64_t(gridDim.x) * kThreads) {
            p.pass[i].claim = kNoPart;
            p.pass[i].taken = 0;
        }
    }
    const int64_t row = blockIdx.x / p.ranges;
    const int range = blockIdx.x - int(row * p.ranges);
    const int64_t V = p.a.vocab, from = range * p.range, to = min(V, from + p.range);
    constexpr int kAhead = 4;                       // loads in flight, the first of them before the temperature is known
    const int64_t base = row * V, last = to - (kAhead - 1) * kMinRange - kAtOnce;
    int64_t v = from + threadIdx.x * kAtOnce;
    float x[kAhead][8];
    auto load = [&](int64_t v) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) load_eight<BF16>(p.a.logits, base + v + u * kMinRange, x[u]);
    };
    if (v <= last) load(v);
    // the row's sequence: how many sequences begin at or before it
    int seq = -1;
    for (int b = 0; b < p.a.num_seqs; b += 64) {
        const int i = b + (threadIdx.x & 63);
        seq += __popcll(__ballot(i < p.a.num_seqs && offset_of(p.a, i) <= row));
    }
    const float c = rate_of(p.a.temperature[max(seq, 0)]);
    RowStat s{-INFINITY, 0.f, int(from), 0};
    auto add = [&](const float (&x)[8], int64_t v) {
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        if (top > s.top) {
            s.sum *= s.top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s.top - top) * c);
            s.top = top;
#pragma unroll
            for (int j = 7; j >= 0; --j)
                if (x[j] == top) s.first = int(v) + j;
        }
        const float b = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
        for (int j = 0; j < 8; ++j) s.sum += __builtin_amdgcn_exp2f((x[j] - b) * c);
    };
    while (v <= last) {
        float y[kAhead][8];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[u][j] = x[u][j];
        const int64_t next = v + kAhead * kMinRange;
        if (next <= last) load(next);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) add(y[u], v + u * kMinRange);
        v = next;
    }
    for (; v < to; v += kMinRange) {
        float y[8];
        if (v + kAtOnce <= to) load_eight<BF16>(p.a.logits, base + v, y);
        else load_some<BF16>(p.a.logits, base + v, int(to - v), -INFINITY, y);
        add(y, v);
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) s = join(s, shuffled(s, m), c);
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 64; ++w) s = join(s, part[w], c);
        p.stats[row * p.ranges + range] = s;
    }
}

// What is left of a node's distribution at token v after 'tried' rejected
// children: max(rest / mass - draft, 0) for each, or 0 for a tried token of a
// certain draft.
template <bool Z16, bool Q16>
struct Rest {
    const Params& p;
    int64_t base;               // the node's first logit
    float c, top, inv;
    int first;
    bool greedy;
    const float* inv_mass;      // 1 / sum left before each tried child, in LDS

    __device__ float whole(float z, int64_t v) const {
        return greedy ? (v == first ? 1.f : 0.f) : __builtin_amdgcn_exp2f((z - top) * c) * inv;
    }
    __device__ float less(float r, float q, int tried) const {
        for (int t = 0; t < tried; ++t) r = fmaxf(r * inv_mass[t] - q, 0.f);
        return r;
    }
};

// A thread's share of what is left of part 'part' of a node's distribution after 'tried' >= 1 rejected children.
template <bool Z16, bool Q16>
__device__ inline float left_of(const Params& p, const Rest<Z16, Q16>& rest, int tried, int part) {
    const VerifyLaunch& a = p.a;
    const int64_t to = min(a.vocab, (part + 1) * p.part);
    const float scale = rest.inv_mass[0];
    float sum = 0.f;
    for (int64_t v = part * p.part + threadIdx.x * kAtOnce; v < to; v += kWalkThreads * kAtOnce) {
        float z[8], d[8];
        if (v + kAtOnce <= to) {
            load_eight<Z16>(a.logits, rest.base + v, z);
            load_eight<Q16>(a.draft, rest.base + v, d);
        } else {
            load_some<Z16>(a.logits, rest.base + v, int(to - v), -INFINITY, z);     // a weight of 0
            load_some<Q16>(a.draft, rest.base + v, int(to - v), 0.f, d);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float r = fmaxf(rest.whole(z[j], v + j) * scale - d[j], 0.f);
            for (int t = 1; t < tried; ++t) r = fmaxf(r * rest.inv_mass[t] - d[j], 0.f);
            sum += r;
        }
    }
    return sum;
}

// The sum over a workgroup, for its first wave.
__device__ inline float sum_of(float x, float* waves) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x / 64] = x;
    __syncthreads();
    x = (threadIdx.x & 63) < kWalkThreads / 64 ? waves[threadIdx.x & 63] : 0.f;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
    return x;
}

// The walk's node and what was rejected of it: what a pass over the vocabulary has to know.
struct Node {
    int row, tried;
    float top, sum;
    int first;
};

template <bool Z16, bool Q16>
__global__ __launch_bounds__(kWalkThreads) void verify_walk_kernel(Params p) {
    extern __shared__ int lds[];                // [3][max_nodes]
    constexpr int kHeld = 256;                  // nodes whose numbers are fetched ahead of the walk, all at once
    __shared__ int token_s[kHeld];
    __shared__ float uniform_s[kHeld], z_s[kHeld], q_s[kHeld];      // z, q: the token's, at its parent
    __shared__ Node node_s;
    __shared__ float waves[kWalkThreads / 64], sums_s[kMaxParts], left_s;
    __shared__ int part_s, pass_s;
    const VerifyLaunch& a = p.a;
    int* parents = lds;
    int* tokens = lds + a.max_nodes;            // tried children's tokens
    float* inv_mass = reinterpret_cast<float*>(lds + 2 * a.max_nodes);
    const int seq = blockIdx.x % a.num_seqs, lane = threadIdx.x & 63;
    const bool leads = int(blockIdx.x) < a.num_seqs;    // the first workgroups of the launch, which start first
    const float temperature = a.temperature[seq], c = rate_of(temperature);
    Pass* shared = p.pass + seq;
    float* mass = p.mass + int64_t(seq) * a.max_nodes;
    float* sums = p.sums + int64_t(seq) * kMaxParts;
    auto rest_of = [&](const Node& x) {
        return Rest<Z16, Q16>{p, x.row * a.vocab, c, x.top, 1.f / x.sum, x.first, !(temperature > 0.f), inv_mass};
    };
    // Takes parts of passes while some are open; a helper reads what they are about.  Thread 0 alone looks at what the
    // workgroups share.
    auto take_parts = [&](int known) {
        for (;;) {
            __syncthreads();
            if (threadIdx.x == 0) {
                const unsigned x = __hip_atomic_fetch_add(&shared->claim, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                part_s = (x & 0xff) < unsigned(p.parts) ? int(x & 0xff) : -1;
                pass_s = int(x >> 8);
            }
            __syncthreads();
            const int part = part_s;
            if (part < 0) return known;
            if (pass_s != known) {              // it stays as it is until this part is done
                known = pass_s;
                if (threadIdx.x == 0)
                    node_s = Node{read_past(&shared->row), read_past(&shared->tried), read_past(&shared->top), read_past(&shared->sum), read_past(&shared->first)};
                __syncthreads();
                for (int i = threadIdx.x; i < node_s.tried; i += kWalkThreads) inv_mass[i] = read_past(mass + i);
                __syncthreads();
            }
            const Node node = node_s;
            const float sum = sum_of(left_of(p, rest_of(node), node.tried, part), waves);
            if (threadIdx.x == 0) {
                put_through(sums + part, sum);
                wait_for_stores();
                __hip_atomic_fetch_add(&shared->taken, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
    };
    if (!leads) {
        for (int known = 0;;) {
            __syncthreads();                    // everybody has read part_s
            if (threadIdx.x == 0) {
                unsigned x = kNoPart;
                for (int polls = 0; polls < kMaxPolls; ++polls) {
                    x = read_past(&shared->claim);
                    if (x >> 8 == kOver >> 8 || (x & 0xff) < unsigned(p.parts)) break;
                    __builtin_amdgcn_s_sleep(4);
                }
                part_s = x >> 8 != kOver >> 8 && (x & 0xff) < unsigned(p.parts);
            }
            __syncthreads();
            if (!part_s) return;
            known = take_parts(known);
        }
    }
    const int first = offset_of(a, seq), n = min(max(0, offset_of(a, seq + 1) - first), a.max_nodes);
    int32_t* path = a.path + int64_t(seq) * a.max_nodes;
    auto z_and_q = [&](int parent, int token, float* z, float* q) {
        const int64_t at = (first + parent) * a.vocab + token;
        *z = load_one<Z16>(a.logits, at);
        *q = a.draft ? load_one<Q16>(a.draft, at) : 1.f;
    };
    for (int i = threadIdx.x; i < a.max_nodes; i += kWalkThreads) {
        if (i < n) {
            const int parent = a.parents[first + i], token = a.tokens[first + i];
            const float uniform = a.uniform[first + i];
            parents[i] = parent;
            if (i < kHeld) {
                token_s[i] = token;
                uniform_s[i] = uniform;
                if (parent >= 0 && parent < i && token >= 0 && token < a.vocab) z_and_q(parent, token, z_s + i, q_s + i);
            }
        }
        path[i] = -1;
    }
    int at = 0, depth = 0, tried = 0, passes = 0;
    __syncthreads();
    while (n > 0) {
        if (threadIdx.x == 0) path[depth] = at;
        ++depth;
        const int row = first + at;
        if (threadIdx.x < 64) {                 // join the row's ranges
            RowStat s{-INFINITY, 0.f, 0x7fffffff, 0};
            if (lane < p.ranges) s = p.stats[int64_t(row) * p.ranges + lane];
#pragma unroll
            for (int m = 1; m < 64; m *= 2) s = join(s, shuffled(s, m), c);
            if (lane == 0) node_s = Node{row, 0, s.top, s.sum, s.first};
        }
        __syncthreads();
        const Node node = node_s;
        const Rest<Z16, Q16> rest = rest_of(node);
        tried = 0;
        int accepted = -1, child = at;
        float left = 1.f;                       // sum of what is left
        auto next_child = [&](int after) {      // of 'at', -1: none
            for (int b = (after + 1) & ~63; b < n; b += 64) {
                const int i = b + lane;
                const unsigned long long hit = __ballot(i > after && i < n && parents[i] == at);
                if (hit) return b + __builtin_ctzll(hit);
            }
            return -1;
        };
        for (child = next_child(child); child >= 0;) {
            const bool held = child < kHeld;
            const int x = held ? token_s[child] : a.tokens[first + child];
            const int following = next_child(child);
            if (x >= 0 && x < a.vocab) {
                float z, q;
                if (held) z = z_s[child], q = q_s[child];
                else z_and_q(at, x, &z, &q);
                float r = rest.whole(z, x);
                if (a.draft) {
                    r = rest.less(r, q, tried);
                } else {
                    for (int t = 0; t < tried; ++t)
                        if (tokens[t] == x) r = 0.f;
                }
                if ((held ? uniform_s[child] : a.uniform[first + child]) * q * left < r) {
                    accepted = child;
                    break;
                }
                __syncthreads();                // everybody has read the lists
                if (threadIdx.x == 0) {
                    inv_mass[tried] = 1.f / fmaxf(left, 1e-30f);
                    tokens[tried] = x;
                    node_s.tried = tried + 1;
                    if (p.walkers > 1) put_through(mass + tried, inv_mass[tried]);
                }
                ++tried;
                __syncthreads();
                if (!a.draft) {
                    left -= r;
                } else if (following >= 0) {    // the next child is measured against the sum of what is left
                    if (p.walkers > 1) {
                        ++passes;
                        if (threadIdx.x == 0) {
                            put_through(&shared->row, node.row);
                            put_through(&shared->tried, tried);
                            put_through(&shared->top, node.top);
                            put_through(&shared->sum, node.sum);
                            put_through(&shared->first, node.first);
                            wait_for_stores();
                            put_through(&shared->claim, unsigned(passes) << 8);
                            wait_for_stores();
                        }
                        take_parts(passes);
                        if (threadIdx.x == 0) {
                            while (read_past(&shared->taken) < unsigned(passes * p.parts)) __builtin_amdgcn_s_sleep(1);
                            asm volatile("" ::: "memory");
                        }
                        __syncthreads();
                        if (lane < p.parts && threadIdx.x < 64) sums_s[lane] = read_past(sums + lane);
                    } else {
                        for (int part = 0; part < p.parts; ++part) {
                            const float sum = sum_of(left_of(p, rest, tried, part), waves);
                            if (threadIdx.x == 0) sums_s[part] = sum;
                            __syncthreads();
                        }
                    }
                    if (threadIdx.x < 64) {     // of all parts, in one order whoever took them
                        float sum = lane < p.parts ? sums_s[lane] : 0.f;
#pragma unroll
                        for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
                        if (lane == 0) left_s = sum;
                    }
                    __syncthreads();
                    left = left_s;
                }
            }
            child = following;
        }
        __syncthreads();
        if (accepted < 0) break;
        at = accepted;
    }
    if (p.walkers > 1 && threadIdx.x == 0) put_through(&shared->claim, kOver);
    for (int i = threadIdx.x; i < tried; i += kWalkThreads) {
        mass[i] = inv_mass[i];
        p.tried[int64_t(seq) * a.max_nodes + i] = tokens[i];
    }
    if (threadIdx.x == 0) {
        a.counts[seq] = depth;
        p.last[seq] = Last{n > 0 ? first + at : -1, tried, node_s.top, node_s.sum, node_s.first, 0u};
        if (n == 0) a.next[seq] = -1;
    }
}

template <bool Z16, bool Q16>
__global__ __launch_bounds__(kThreads) void verify_sample_kernel(Params p) {
    extern __shared__ int lds[];                // [2][max_nodes]
    __shared__ Best part[kThreads / 64];
    const VerifyLaunch& a = p.a;
    const int seq = blockIdx.x / p.sample_ranges, range = blockIdx.x - seq * p.sample_ranges;
    const Last last = p.last[seq];
    if (last.row < 0) return;
    float* inv_mass = reinterpret_cast<float*>(lds);
    int* tokens = lds + a.max_nodes;
    if (last.tried) {
        for (int i = threadIdx.x; i < last.tried; i += kThreads) {
            inv_mass[i] = p.mass[int64_t(seq) * a.max_nodes + i];
            tokens[i] = p.tried[int64_t(seq) * a.max_nodes + i];
        }
        __syncthreads();
    }
    const float temperature = a.temperature[seq];
    const Rest<Z16, Q16> rest{p, int64_t(last.row) * a.vocab, rate_of(temperature), last.top, 1.f / last.sum, last.first, !(temperature > 0.f), inv_mass};
    const float* noise = a.noise + int64_t(seq) * a.vocab;
    const bool drafted = a.draft && last.tried;
    const int64_t from = range * p.sample_range, to = min(a.vocab, from + p.sample_range);
    Best b{0.f, 0x7fffffff, 0.f, 0x7fffffff};
    for (int64_t v = from + threadIdx.x * kAtOnce; v < to; v += kMinRange) {
        float z[8], q[8], e[8];
        if (v + kAtOnce <= to) {
            load_eight<Z16>(a.logits, rest.base + v, z);
            load_eight<false>(noise, v, e);
            if (drafted) load_eight<Q16>(a.draft, rest.base + v, q);
        } else {
            const int some = int(to - v);
            load_some<Z16>(a.logits, rest.base + v, some, -INFINITY, z);
            load_some<false>(noise, v, some, 1.f, e);
            if (drafted) load_some<Q16>(a.draft, rest.base + v, some, 0.f, q);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t x = v + j;
            const float w = rest.whole(z[j], x);
            float r = drafted ? rest.less(w, q[j], last.tried) : w;
            const float near = __builtin_amdgcn_rcpf(e[j]) * 1.00001f;      // the quotient itself where it may be the largest
            if (w * near > b.all) take(b.all, b.all_at, w / e[j], int(x));
            if (r * near > b.rest) {
                if (!a.draft)                   // a certain draft: nothing is left of a token that was tried
                    for (int t = 0; t < last.tried; ++t) r = tokens[t] == x ? 0.f : r;
                if (r > 0.f) take(b.rest, b.rest_at, r / e[j], int(x));
            }
        }
    }
    auto best_of_wave = [&]() {
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            take(b.rest, b.rest_at, __shfl_xor(b.rest, m), __shfl_xor(b.rest_at, m));
            take(b.all, b.all_at, __shfl_xor(b.all, m), __shfl_xor(b.all_at, m));
        }
    };
    best_of_wave();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = b;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    // The last range to arrive finishes the sequence (walk left the count at 0).  Ranges run on different XCDs: their
    // results are written through and read past the L2s, which a fence would write back whole.
    unsigned long long* mine = reinterpret_cast<unsigned long long*>(p.best + int64_t(seq) * p.sample_ranges);
    unsigned arrived = 0;
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 64; ++w) {
            take(b.rest, b.rest_at, part[w].rest, part[w].rest_at);
            take(b.all, b.all_at, part[w].all, part[w].all_at);
        }
        const u64x2 x = __builtin_bit_cast(u64x2, b);
        put_through(mine + 2 * range, x[0]);
        put_through(mine + 2 * range + 1, x[1]);
        wait_for_stores();
        arrived = __hip_atomic_fetch_add(&p.last[seq].arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (__shfl(arrived, 0) != unsigned(p.sample_ranges) - 1) return;
    b = Best{0.f, 0x7fffffff, 0.f, 0x7fffffff};
    if (threadIdx.x < unsigned(p.sample_ranges))
        b = __builtin_bit_cast(Best, u64x2{read_past(mine + 2 * threadIdx.x), read_past(mine + 2 * threadIdx.x + 1)});
    best_of_wave();
    // nothing left (every probability went to the draft): the distribution itself; no finite logit: token 0
    if (threadIdx.x == 0) a.next[seq] = b.rest > 0.f ? b.rest_at : b.all > 0.f ? b.all_at : 0;
}

// Ranges of a row: as many as give a few thousand workgroups, of at least one
// load for every lane, and one lane to join each.
int ranges_of(int64_t vocab, int64_t rows) {
    const int64_t most = (vocab + kMinRange - 1) / kMinRange;
    return int(std::max<int64_t>(1, std::min<int64_t>({most, kMaxRanges, (2048 + rows - 1) / std::max<int64_t>(rows, 1)})));
}
int64_t range_of(int64_t vocab, int ranges) { return ((vocab + ranges - 1) / ranges + kMinRange - 1) / kMinRange * kMinRange; }

int64_t round16(int64_t x) { return (x + 15) & ~int64_t(15); }

template <bool Z16, bool Q16>
hipError_t verify_as(const Params& p, hipStream_t stream) {
    const VerifyLaunch& a = p.a;
    if (a.total > 0) {
        hipLaunchKernelGGL((verify_stats_kernel<Z16>), dim3(uint32_t(a.total * p.ranges)), dim3(kThreads), 0, stream, p);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((verify_walk_kernel<Z16, Q16>), dim3(uint32_t(a.num_seqs) * p.walkers), dim3(kWalkThreads), 3 * a.max_nodes * sizeof(int), stream, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_sample_kernel<Z16, Q16>), dim3(uint32_t(a.num_seqs) * p.sample_ranges), dim3(kThreads), 2 * a.max_nodes * sizeof(int), stream, p);
    return hipGetLastError();
}

}  // namespace

int64_t verify_workspace_bytes(int64_t vocab, int64_t total, int num_seqs, int max_nodes) {
    return total * ranges_of(vocab, total) * sizeof(RowStat) +
           num_seqs * (ranges_of(vocab, num_seqs) * sizeof(Best) + sizeof(Last) + sizeof(Pass) + kMaxParts * sizeof(float) + 2 * round16(max_nodes * 4));
}

hipError_t launch_verify(const VerifyLaunch& a, hipStream_t stream) {
    constexpr int64_t kLoad = kWalkThreads * kAtOnce, kAtMost = 256;
    Params p{};
    p.a = a;
    p.ranges = ranges_of(a.vocab, a.total);
    p.range = range_of(a.vocab, p.ranges);
    p.sample_ranges = ranges_of(a.vocab, a.num_seqs);
    p.sample_range = range_of(a.vocab, p.sample_ranges);
    // a part: one load for every lane; several workgroups to a sequence where it can reject two children against a draft,
    // and no more than the CUs take at once
    p.parts = int(std::min<int64_t>(kMaxParts, (a.vocab + kLoad - 1) / kLoad));
    p.part = ((a.vocab + p.parts - 1) / p.parts + kLoad - 1) / kLoad * kLoad;
    p.walkers = a.draft && a.max_nodes > 2 && a.total > 0 ? int(std::max<int64_t>(1, std::min<int64_t>({kWalkers, p.parts, kAtMost / a.num_seqs}))) : 1;
    uint8_t* at = static_cast<uint8_t*>(a.ws);
    auto take = [&](int64_t bytes) {
        uint8_t* from = at;
        at += bytes;
        return from;
    };
    p.stats = reinterpret_cast<RowStat*>(take(a.total * p.ranges * sizeof(RowStat)));
    p.best = reinterpret_cast<Best*>(take(int64_t(a.num_seqs) * p.sample_ranges * sizeof(Best)));
    p.pass = reinterpret_cast<Pass*>(take(a.num_seqs * sizeof(Pass)));
    p.sums = reinterpret_cast<float*>(take(a.num_seqs * kMaxParts * sizeof(float)));
    p.mass = reinterpret_cast<float*>(take(a.num_seqs * round16(a.max_nodes * 4)));
    p.tried = reinterpret_cast<int32_t*>(take(a.num_seqs * round16(a.max_nodes * 4)));
    p.last = reinterpret_cast<Last*>(take(a.num_seqs * sizeof(Last)));
    if (a.logits_bf16) return a.draft_bf16 ? verify_as<true, true>(p, stream) : verify_as<true, false>(p, stream);
    return a.draft_bf16 ? verify_as<false, true>(p, stream) : verify_as<false, false>(p, stream);
}

}  // namespace tl
