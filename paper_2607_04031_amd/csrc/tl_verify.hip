// Verification of drafted tokens.  Three launches:
//   stats   every node's logits row, in ranges: maximum (and where it is first)
//           and sum of exponentials -- all the bytes there are to read, so this
//           is bound by HBM where the rows are many
//   walk    a workgroup per sequence goes from the root to an accepted child
//           while there is one
//   sample  the last node's distribution less what its rejected children took,
//           in ranges: the token with the largest ratio of weight to noise (an
//           exponential race: P(token wins) is proportional to its weight)
// Row ranges are joined in their order, and the race's winner does not depend
// on it, so results are the same from call to call.
#include <hip/hip_runtime.h>

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {
namespace {

constexpr int kThreads = 256;
constexpr int kWalkThreads = 1024;
constexpr int kMaxRanges = 32;
constexpr int kMinRange = 4096;
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
struct Best {
    float rest, all;    // largest weight / noise of what is left, and of the whole distribution
    int rest_at, all_at;
};

struct Params {
    VerifyLaunch a;
    int ranges;         // of a row, in stats and in sample
    int64_t range;      // elements, a multiple of 8
    RowStat* stats;     // [total][ranges]
    Last* last;         // [num_seqs]
    Best* best;         // [num_seqs][ranges]
    float* mass;        // [num_seqs][max_nodes]: sum left before each tried child
    int32_t* tried;     // [num_seqs][max_nodes]: the tried children's tokens
};

__device__ inline int offset_of(const VerifyLaunch& a, int i) { return max(0, min(a.offsets[i], int(a.total))); }

// 2^((z - top) c) is the softmax's numerator
__device__ inline float rate_of(float temperature) { return temperature > 0.f ? fminf(1.f / temperature, 1e38f) * kLog2e : 0.f; }

template <bool BF16>
__device__ inline float load_one(const void* p, int64_t at) {
    if (BF16) return __uint_as_float(uint32_t(static_cast<const uint16_t*>(p)[at]) << 16);
    return static_cast<const float*>(p)[at];
}

// four elements from any element's address
template <bool BF16>
__device__ inline void load_four(const void* p, int64_t at, float (&x)[4]) {
    if (BF16) {
        u32x2 w;
        __builtin_memcpy(&w, static_cast<const uint16_t*>(p) + at, 8);
        x[0] = bf16_lo(w[0]), x[1] = bf16_hi(w[0]), x[2] = bf16_lo(w[1]), x[3] = bf16_hi(w[1]);
    } else {
        __builtin_memcpy(x, static_cast<const float*>(p) + at, 16);
    }
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
    const int64_t row = blockIdx.x / p.ranges;
    const int range = blockIdx.x - int(row * p.ranges);
    const int64_t V = p.a.vocab, from = range * p.range, to = min(V, from + p.range);
    // the row's sequence: how many sequences begin at or before it
    __shared__ int seq_s;
    if (threadIdx.x < 64) {
        int seq = -1;
        for (int b = 0; b < p.a.num_seqs; b += 64) {
            const int i = b + threadIdx.x;
            seq += __popcll(__ballot(i < p.a.num_seqs && offset_of(p.a, i) <= row));
        }
        if (threadIdx.x == 0) seq_s = max(seq, 0);
    }
    __syncthreads();
    const float c = rate_of(p.a.temperature[seq_s]);
    RowStat s{-INFINITY, 0.f, int(from), 0};
    const int64_t base = row * V;
    for (int64_t v = from + threadIdx.x * 4; v < to; v += kThreads * 4) {
        float x[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (v + 4 <= to) {
            load_four<BF16>(p.a.logits, base + v, x);
        } else {
            for (int j = 0; j < int(to - v); ++j) x[j] = load_one<BF16>(p.a.logits, base + v + j);
        }
        const float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        if (top > s.top) {
            s.sum *= s.top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s.top - top) * c);
            s.top = top;
#pragma unroll
            for (int j = 3; j >= 0; --j)
                if (x[j] == top) s.first = int(v) + j;
        }
        const float b = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
        for (int j = 0; j < 4; ++j) s.sum += __builtin_amdgcn_exp2f((x[j] - b) * c);
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
    const float* mass;
    const int32_t* tokens;

    __device__ float whole(float z, int64_t v) const {
        return greedy ? (v == first ? 1.f : 0.f) : __builtin_amdgcn_exp2f((z - top) * c) * inv;
    }
    __device__ float less(float r, float q, int tried) const {
        for (int t = 0; t < tried; ++t) r = fmaxf(r / fmaxf(mass[t], 1e-30f) - q, 0.f);
        return r;
    }
};

template <bool Z16, bool Q16>
__global__ __launch_bounds__(kWalkThreads) void verify_walk_kernel(Params p) {
    extern __shared__ int parents[];            // [max_nodes]
    __shared__ RowStat stat_s;
    __shared__ float sums[kWalkThreads / 64];
    const VerifyLaunch& a = p.a;
    const int seq = blockIdx.x, lane = threadIdx.x & 63;
    const int first = offset_of(a, seq), n = min(max(0, offset_of(a, seq + 1) - first), a.max_nodes);
    int32_t* path = a.path + int64_t(seq) * a.max_nodes;
    for (int i = threadIdx.x; i < a.max_nodes; i += kWalkThreads) {
        if (i < n) parents[i] = a.parents[first + i];
        path[i] = -1;
    }
    const float temperature = a.temperature[seq], c = rate_of(temperature);
    float* mass = p.mass + int64_t(seq) * a.max_nodes;
    int32_t* tokens = p.tried + int64_t(seq) * a.max_nodes;
    int at = 0, depth = 0, tried = 0;
    __syncthreads();
    while (n > 0) {
        if (threadIdx.x == 0) path[depth] = at;
        ++depth;
        const int64_t row = first + at;
        if (threadIdx.x < 64) {                 // join the row's ranges
            RowStat s{-INFINITY, 0.f, 0, 0};
            if (lane < p.ranges) s = p.stats[row * p.ranges + lane];
            else s.first = 0x7fffffff;
#pragma unroll
            for (int m = 1; m < 64; m *= 2) s = join(s, shuffled(s, m), c);
            if (lane == 0) stat_s = s;
        }
        __syncthreads();
        const RowStat stat = stat_s;
        Rest<Z16, Q16> rest{p, row * a.vocab, c, stat.top, 1.f / stat.sum, stat.first, !(temperature > 0.f), mass, tokens};
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
            const int64_t x = a.tokens[first + child];
            const int following = next_child(child);
            if (x >= 0 && x < a.vocab) {
                float r = rest.whole(load_one<Z16>(a.logits, rest.base + x), x);
                float q = 1.f;
                if (a.draft) {
                    q = load_one<Q16>(a.draft, rest.base + x);
                    r = rest.less(r, q, tried);
                } else {
                    for (int t = 0; t < tried; ++t)
                        if (tokens[t] == x) r = 0.f;
                }
                if (a.uniform[first + child] * q * left < r) {
                    accepted = child;
                    break;
                }
                __syncthreads();                // everybody has read the lists
                if (threadIdx.x == 0) {
                    mass[tried] = left;
                    tokens[tried] = int(x);
                }
                ++tried;
                __syncthreads();
                if (!a.draft) {
                    left -= r;
                } else if (following >= 0) {    // the next child is measured against the sum of what is left
                    float sum = 0.f;
                    for (int64_t v = threadIdx.x; v < a.vocab; v += kWalkThreads)
                        sum += rest.less(rest.whole(load_one<Z16>(a.logits, rest.base + v), v), load_one<Q16>(a.draft, rest.base + v), tried);
#pragma unroll
                    for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
                    if (lane == 0) sums[threadIdx.x / 64] = sum;
                    __syncthreads();
                    left = 0.f;
                    for (int w = 0; w < kWalkThreads / 64; ++w) left += sums[w];
                }
            }
            child = following;
        }
        __syncthreads();
        if (accepted < 0) break;
        at = accepted;
    }
    if (threadIdx.x == 0) {
        a.counts[seq] = depth;
        p.last[seq] = Last{n > 0 ? first + at : -1, tried, stat_s.top, stat_s.sum, stat_s.first, 0u};
        if (n == 0) a.next[seq] = -1;
    }
}

template <bool Z16, bool Q16>
__global__ __launch_bounds__(kThreads) void verify_sample_kernel(Params p) {
    __shared__ Best part[kThreads / 64];
    __shared__ unsigned arrived;
    const VerifyLaunch& a = p.a;
    const int seq = blockIdx.x / p.ranges, range = blockIdx.x - seq * p.ranges;
    const Last last = p.last[seq];
    if (last.row < 0) return;
    const float temperature = a.temperature[seq];
    const float* mass = p.mass + int64_t(seq) * a.max_nodes;
    const int32_t* tokens = p.tried + int64_t(seq) * a.max_nodes;
    const Rest<Z16, Q16> rest{p, int64_t(last.row) * a.vocab, rate_of(temperature), last.top, 1.f / last.sum, last.first, !(temperature > 0.f), mass, tokens};
    const float* noise = a.noise + int64_t(seq) * a.vocab;
    const int64_t from = range * p.range, to = min(a.vocab, from + p.range);
    Best b{0.f, 0.f, 0x7fffffff, 0x7fffffff};
    for (int64_t v = from + threadIdx.x * 4; v < to; v += kThreads * 4) {
        float z[4], q[4] = {0.f, 0.f, 0.f, 0.f}, e[4];
        const int some = int(min(int64_t(4), to - v));
        if (some == 4) {
            load_four<Z16>(a.logits, rest.base + v, z);
            load_four<false>(noise, v, e);
            if (a.draft && last.tried) load_four<Q16>(a.draft, rest.base + v, q);
        } else {
            for (int j = 0; j < some; ++j) {
                z[j] = load_one<Z16>(a.logits, rest.base + v + j);
                e[j] = noise[v + j];
                if (a.draft && last.tried) q[j] = load_one<Q16>(a.draft, rest.base + v + j);
            }
        }
        for (int j = 0; j < some; ++j) {
            const int64_t x = v + j;
            const float w = rest.whole(z[j], x);
            if (w / e[j] > b.all) b.all = w / e[j], b.all_at = int(x);
            float r = w;
            if (a.draft) r = rest.less(w, q[j], last.tried);
            if (r / e[j] > b.rest) {
                if (!a.draft)
                    for (int t = 0; t < last.tried; ++t)
                        if (tokens[t] == x) r = 0.f;
                if (r / e[j] > b.rest) b.rest = r / e[j], b.rest_at = int(x);
            }
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        take(b.rest, b.rest_at, __shfl_xor(b.rest, m), __shfl_xor(b.rest_at, m));
        take(b.all, b.all_at, __shfl_xor(b.all, m), __shfl_xor(b.all_at, m));
    }
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = b;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 64; ++w) {
            take(b.rest, b.rest_at, part[w].rest, part[w].rest_at);
            take(b.all, b.all_at, part[w].all, part[w].all_at);
        }
        Best* mine = p.best + int64_t(seq) * p.ranges;
        mine[range] = b;
        // the last range to arrive finishes the sequence (walk left the count at 0)
        __threadfence();
        arrived = __hip_atomic_fetch_add(&p.last[seq].arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        if (arrived == unsigned(p.ranges) - 1) {
            __threadfence();
            for (int i = 0; i < p.ranges; ++i) {
                take(b.rest, b.rest_at, mine[i].rest, mine[i].rest_at);
                take(b.all, b.all_at, mine[i].all, mine[i].all_at);
            }
            // nothing left (every probability went to the draft): the distribution itself; no finite logit: token 0
            a.next[seq] = b.rest > 0.f ? b.rest_at : b.all > 0.f ? b.all_at : 0;
        }
    }
}

int ranges_of(int64_t vocab, int64_t rows) {
    const int64_t most = (vocab + kMinRange - 1) / kMinRange;
    return int(std::max<int64_t>(1, std::min<int64_t>({most, kMaxRanges, (2048 + rows - 1) / std::max<int64_t>(rows, 1)})));
}

int64_t round16(int64_t x) { return (x + 15) & ~int64_t(15); }

template <bool Z16, bool Q16>
hipError_t verify_as(const Params& p, hipStream_t stream) {
    const VerifyLaunch& a = p.a;
    if (a.total > 0) {
        hipLaunchKernelGGL((verify_stats_kernel<Z16>), dim3(uint32_t(a.total * p.ranges)), dim3(kThreads), 0, stream, p);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((verify_walk_kernel<Z16, Q16>), dim3(a.num_seqs), dim3(kWalkThreads), a.max_nodes * sizeof(int), stream, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_sample_kernel<Z16, Q16>), dim3(uint32_t(a.num_seqs) * p.ranges), dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

int64_t verify_workspace_bytes(int64_t vocab, int64_t total, int num_seqs, int max_nodes) {
    const int64_t r = ranges_of(vocab, total);
    return total * r * sizeof(RowStat) + num_seqs * (r * sizeof(Best) + round16(sizeof(Last)) + 2 * round16(max_nodes * 4));
}

hipError_t launch_verify(const VerifyLaunch& a, hipStream_t stream) {
    Params p{};
    p.a = a;
    p.ranges = ranges_of(a.vocab, a.total);
    p.range = ((a.vocab + p.ranges - 1) / p.ranges + 7) / 8 * 8;
    uint8_t* at = static_cast<uint8_t*>(a.ws);
    p.stats = reinterpret_cast<RowStat*>(at);
    at += a.total * p.ranges * sizeof(RowStat);
    p.best = reinterpret_cast<Best*>(at);
    at += int64_t(a.num_seqs) * p.ranges * sizeof(Best);
    p.last = reinterpret_cast<Last*>(at);
    at += a.num_seqs * round16(sizeof(Last));
    p.mass = reinterpret_cast<float*>(at);
    at += a.num_seqs * round16(a.max_nodes * 4);
    p.tried = reinterpret_cast<int32_t*>(at);
    if (a.logits_bf16) return a.draft_bf16 ? verify_as<true, true>(p, stream) : verify_as<true, false>(p, stream);
    return a.draft_bf16 ? verify_as<false, true>(p, stream) : verify_as<false, false>(p, stream);
}

}  // namespace tl
