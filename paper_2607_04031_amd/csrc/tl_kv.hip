// The paged key/value cache: rotary positions and quantisation on the way in,
// reading entries back, and moving the entries of an accepted path.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {
namespace {

constexpr int kThreads = kKvThreads;

// Where a token's entries lie: its page (valid, or negative) and place in it.
__device__ inline int64_t page_of(const KvView& c, int slot, int* t) {
    const int64_t page = slot >> c.log2_page;
    *t = slot & ((1 << c.log2_page) - 1);
    return slot >= 0 && page < c.num_pages ? page : -1;
}

// Byte offset of a (page, head) block, and of its exponents.
template <int D, int ELEM>
__device__ inline int64_t block_at(const KvView& c, int64_t page, int head) {
    return ((page * c.heads + head) << c.log2_page) * (D * ELEM);
}
__device__ inline int64_t exps_at(const KvView& c, int64_t page, int head) { return (page * c.heads + head) << c.log2_page; }

// ---------------------------------------------------------------------------
// append: x -> rotated x (queries and keys) -> bf16, or E4M3 with the scale
// 2^e, e the smallest with max |x| <= 448 * 2^e over the head, so that scaling
// is exact and each element is rounded once.  A lane holds 8 elements of one
// head.  The angle position * inv_freq is reduced to a fraction of a turn in 64
// bits (at position 10^5 its 32-bit product would be off by 0.005), once per
// pair and token of a workgroup, through LDS.
//
// Few tokens: a workgroup takes one token and a part of its heads, and its
// values go out byte by byte to their places in the transposed blocks; the
// launch bounds it.  Many tokens (windows): queries a token per workgroup, keys
// 16 tokens and values 64 tokens of a head, so that whole cache lines are
// written where the slots follow one another; HBM bounds it (8192 rows of 64
// heads over 8: 70 us, 4.8 TB/s; a single row: 3.5 us).
// ---------------------------------------------------------------------------
constexpr int kKeyWindow = 16, kValueWindow = 64;

// Window w of a list of slots: the tokens up to 64 whose slots share a group of
// 64 of a page if the list goes on from its first slot (pages may come in any
// order).  run: they do, one after another, all in the cache.
struct Window {
    int64_t first, page;    // first token; its page
    int count, start, place;    // tokens; the group's first token in the page; the first token's place in the group
    bool run;
};
__device__ inline bool find_window(const KvView& c, const int32_t* slots, int64_t n, int64_t w, Window* out) {
    const int64_t from = w * kValueWindow - (slots[0] & (kValueWindow - 1));
    out->first = max(from, int64_t(0));
    out->count = int(min(from + kValueWindow, n) - out->first);
    if (out->count <= 0) return false;
    const int slot = slots[out->first];
    const bool next = threadIdx.x >= unsigned(out->count) || unsigned(slots[out->first + threadIdx.x]) == unsigned(slot) + threadIdx.x;
    int t;
    out->page = page_of(c, slot, &t);
    out->start = t & ~(kValueWindow - 1);
    out->place = t & (kValueWindow - 1);
    out->run = __syncthreads_and(next) && out->page >= 0 && out->place + out->count <= kValueWindow;
    return true;
}

// A group's values in LDS: the 64 tokens of an element in the order of its
// chunks.  The byte of token t, the token of place x, and the element and first
// byte of the group's 16-byte chunk u.
template <int ELEM>
__device__ inline int value_byte(int t) {
    constexpr int c = 16 / ELEM;
    return ((t / (4 * c) * 4 + ((t & 15) >> 2)) * c + (t % (4 * c) >> 4) * 4 + (t & 3)) * ELEM;
}
template <int ELEM>
__device__ inline int value_token(int x) {
    constexpr int c = 16 / ELEM;
    return x / (4 * c) * (4 * c) + x % c / 4 * 16 + x / c % 4 * 4 + (x & 3);
}
template <int D, int ELEM>
__device__ inline void value_chunk(int u, int* d, int* at) {
    constexpr int per = D * 4;          // chunks of 4 c tokens
    const int x = u % per;
    *d = x / 64 * 16 + (x & 15);
    *at = (u / per * 4 + (x >> 4 & 3)) * 16;
}

template <bool F32>
__device__ inline void load_row8(const void* src, int64_t at, float (&x)[8]) {
    if (F32) {
        const f32x4v* p = reinterpret_cast<const f32x4v*>(static_cast<const float*>(src) + at);
        const f32x4v u = p[0], v = p[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = u[i], x[4 + i] = v[i];
    } else {
        const u32x4 u = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(src) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(u[i]), x[2 * i + 1] = bf16_hi(u[i]);
    }
}

__device__ inline void angle_of(const KvAppendLaunch& a, int64_t token, int pair, float* cos_to, float* sin_to) {
    const int axis = pair < a.sections[0] ? 0 : pair < a.sections[0] + a.sections[1] ? 1 : 2;
    const double turns = double(a.positions[axis * a.n + token]) * double(a.inv_freq[pair]) * 0.15915494309189533577;
    const float frac = float(turns - rint(turns));
    sincospif(2.f * frac, sin_to, cos_to);
}

// x of a lane (elements d0 .. d0 + 7 of a head), turned; the head's lanes call it together
__device__ inline void turn(const KvAppendLaunch& a, const float* cos_s, const float* sin_s, int lane, int d0, float (&x)[8]) {
    const int half = a.rot_dim / 2;
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const bool in = d0 + i < a.rot_dim;
            const float c = in ? cos_s[(d0 + i) / 2] : 1.f, s = in ? sin_s[(d0 + i) / 2] : 0.f;
            const float u = x[i] * c - x[i + 1] * s, v = x[i + 1] * c + x[i] * s;
            x[i] = u;
            x[i + 1] = v;
        }
    } else {
        const bool in = d0 < a.rot_dim, low = d0 < half;   // half is a multiple of 8
        const int partner = in ? (low ? d0 + half : d0 - half) / 8 : lane;
        const int from = (threadIdx.x & 63) - lane + partner;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl(x[i], from);
            const int pair = low ? d0 + i : d0 - half + i;
            const float c = in ? cos_s[pair] : 1.f, s = in ? sin_s[pair] : 0.f;
            x[i] = low ? x[i] * c - other * s : x[i] * c + other * s;
        }
    }
}

__device__ inline u32x4 to_bf16(const float (&x)[8]) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    return o;
}

// E4M3 of a head's elements over LANES lanes, and the exponent of its scale
template <int LANES>
__device__ inline u32x2 to_fp8(const float (&x)[8], int* exponent) {
    float amax = 0.f;   // NaN elements take no part
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
    for (int m = 1; m < LANES; m *= 2) amax = fmaxf(amax, __shfl_xor(amax, m));
    // amax = f * 2^(b - 127), 1 <= f < 2: 448 * 2^e = 1.75 * 2^(8 + e) fits it from e = b - 135 on, one more where f > 1.75
    const uint32_t bits = min(__float_as_uint(amax), 0x7f7fffffu);   // an infinity counts as the largest finite value
    int e = int(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u);
    e = amax > 0.f ? max(e, -126) : 0;
    const float inv = exp_scale(127 - e);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = x[i] * inv;
        y[i] = s > 448.f ? 448.f : s < -448.f ? -448.f : s;   // infinities saturate, a NaN stays one
    }
    u32x2 o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        o[i] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true));
    }
    *exponent = e;
    return o;
}

// keys of a lane into the cache
template <int D, int ELEM>
__device__ inline void put_key(const KvView& c, int slot, int head, int lane, const float (&x)[8]) {
    int t, e = 0;
    const u32x2 o8 = ELEM == 1 ? to_fp8<D / 8>(x, &e) : u32x2{0, 0};
    const int64_t page = page_of(c, slot, &t);
    if (page < 0) return;
    uint8_t* to = c.k + block_at<D, ELEM>(c, page, head) + kv_key_at<D, ELEM>(t, lane * 8) * ELEM;
    if (ELEM == 2) {
        *reinterpret_cast<u32x4*>(to) = to_bf16(x);
    } else {
        *reinterpret_cast<u32x2*>(to) = o8;
        if (lane == 0) c.k_exp[exps_at(c, page, head) + kv_key_exp_at(t)] = uint8_t(e + 127);
    }
}

// values of a lane (as stored: 4 bf16 pairs, or two words of E4M3 and the exponent), element by element
template <int D, int ELEM>
__device__ inline void put_value(const KvView& c, int slot, int head, int lane, u32x4 o, int e) {
    int t;
    const int64_t page = page_of(c, slot, &t);
    if (page < 0) return;
    const int64_t block = block_at<D, ELEM>(c, page, head);
    if (ELEM == 2) {
        uint16_t* v = reinterpret_cast<uint16_t*>(c.v + block);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[kv_value_at<D, 2>(t, lane * 8 + i)] = uint16_t(o[i / 2] >> (i % 2 * 16));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) c.v[block + kv_value_at<D, 1>(t, lane * 8 + i)] = uint8_t(o[i / 4] >> (i % 4 * 8));
        if (lane == 0) c.v_exp[exps_at(c, page, head) + kv_value_exp_at(t)] = uint8_t(e + 127);
    }
}

template <int D, int ELEM>
__device__ inline u32x4 stored(const float (&x)[8], int* e) {
    if (ELEM == 2) return to_bf16(x);
    const u32x2 o = to_fp8<D / 8>(x, e);
    return u32x4{o[0], o[1], 0, 0};
}

// heads [first, last) of one token, 256 / (D / 8) at a time; heads count through queries, keys and values
template <int D, int ELEM, bool F32>
__device__ void append_token(const KvAppendLaunch& a, int64_t token, int first, int last, float* cos_s, float* sin_s) {
    constexpr int kLanes = D / 8, kHeads = kThreads / kLanes;
    const int lane = threadIdx.x % kLanes, d0 = lane * 8;
    auto find = [&](int head, int* in) {       // 0 queries, 1 keys, 2 values, 3 none
        int which = 0;
        *in = head;
        while (which < 3 && *in >= a.heads[which]) *in -= a.heads[which++];
        return head < last ? which : 3;
    };
    int head, which = find(first + threadIdx.x / kLanes, &head);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (which < 3) load_row8<F32>(a.src[which], token * a.ld[which] + int64_t(head) * D + d0, x);
    const int slot = a.slots ? a.slots[token] : -1;
    if (a.rot_dim) {
        if (threadIdx.x < unsigned(a.rot_dim / 2)) angle_of(a, token, threadIdx.x, cos_s + threadIdx.x, sin_s + threadIdx.x);
        __syncthreads();
    }
    for (int base = first; base < last; base += kHeads) {
        int next_head;
        const int next_which = find(base + kHeads + threadIdx.x / kLanes, &next_head);
        float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (next_which < 3) load_row8<F32>(a.src[next_which], token * a.ld[next_which] + int64_t(next_head) * D + d0, y);
        if (a.rot_dim && which < 2) turn(a, cos_s, sin_s, lane, d0, x);   // heads lie in whole groups of lanes
        if (which == 0) *reinterpret_cast<u32x4*>(a.q_out + (token * a.heads[0] + head) * D + d0) = to_bf16(x);
        if (which == 1) put_key<D, ELEM>(a.c, slot, head, lane, x);
        if (which == 2) {
            int e = 0;
            const u32x4 o = stored<D, ELEM>(x, &e);
            put_value<D, ELEM>(a.c, slot, head, lane, o, e);
        }
        which = next_which;
        head = next_head;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = y[i];
    }
}

template <int D, int ELEM, bool F32>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvAppendLaunch a, int head_blocks) {
    __shared__ float cos_s[D / 2], sin_s[D / 2];
    const int64_t token = blockIdx.x / head_blocks;
    const int per = kThreads / (D / 8), block = int(blockIdx.x - token * head_blocks);
    append_token<D, ELEM, F32>(a, token, block * per, min((block + 1) * per, a.heads[0] + a.heads[1] + a.heads[2]), cos_s, sin_s);
}

struct AppendBlocks {
    int keys, values;               // workgroups; the others take queries
    int key_heads, query_heads;     // of a workgroup
};

template <int D, int ELEM, bool F32>
__global__ __launch_bounds__(kThreads) void kv_append_window_kernel(KvAppendLaunch a, AppendBlocks b) {
    constexpr int kLanes = D / 8, kTokens = kThreads / kLanes;
    constexpr int kStride = kValueWindow * ELEM + 4;           // bytes of an element's tokens in LDS: an odd number of words
    __shared__ __attribute__((aligned(16))) uint8_t lds[D * kStride > kKeyWindow * D * 4 ? D * kStride : kKeyWindow * D * 4];
    const int lane = threadIdx.x % kLanes, d0 = lane * 8, mine = threadIdx.x / kLanes;
    if (int(blockIdx.x) < b.keys) {                            // 16 tokens' keys of some heads
        float* cos_s = reinterpret_cast<float*>(lds);
        float* sin_s = cos_s + kKeyWindow * D / 2;
        const int parts = (a.heads[1] + b.key_heads - 1) / b.key_heads, window = blockIdx.x / parts;
        const int head0 = (blockIdx.x - window * parts) * b.key_heads, head1 = min(head0 + b.key_heads, a.heads[1]);
        const int64_t first = int64_t(window) * kKeyWindow - (a.slots[0] & (kKeyWindow - 1));
        const int half = a.rot_dim / 2;
        for (int i = threadIdx.x; i < kKeyWindow * half; i += kThreads) {
            const int j = i / half, pair = i - j * half;
            if (first + j >= 0 && first + j < a.n) angle_of(a, first + j, pair, cos_s + j * (D / 2) + pair, sin_s + j * (D / 2) + pair);
        }
        __syncthreads();
        constexpr int kGroups = kThreads / (kKeyWindow * kLanes);      // heads at a time
        const int j = mine % kKeyWindow;
        const int64_t token = first + j;
        if (token < 0 || token >= a.n) return;
        const int slot = a.slots[token];
        int head = head0 + mine / kKeyWindow;
        float x[8];
        if (head < head1) load_row8<F32>(a.src[1], token * a.ld[1] + int64_t(head) * D + d0, x);
        for (; head < head1; head += kGroups) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i];
            if (head + kGroups < head1) load_row8<F32>(a.src[1], token * a.ld[1] + int64_t(head + kGroups) * D + d0, x);
            if (a.rot_dim) turn(a, cos_s + j * (D / 2), sin_s + j * (D / 2), lane, d0, y);
            put_key<D, ELEM>(a.c, slot, head, lane, y);
        }
        return;
    }
    if (int(blockIdx.x) < b.keys + b.values) {                 // 64 tokens' values of a head
        const int block = blockIdx.x - b.keys, head = block % a.heads[2];
        Window w;
        if (!find_window(a.c, a.slots, a.n, block / a.heads[2], &w)) return;
        for (int j = mine; j < w.count; j += kTokens) {
            float x[8];
            load_row8<F32>(a.src[2], (w.first + j) * a.ld[2] + int64_t(head) * D + d0, x);
            int e = 0;
            const u32x4 o = stored<D, ELEM>(x, &e);
            if (!w.run) {
                put_value<D, ELEM>(a.c, a.slots[w.first + j], head, lane, o, e);
                continue;
            }
            const int t = w.place + j;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint8_t* to = lds + (d0 + i) * kStride + value_byte<ELEM>(t);
                if (ELEM == 1) *to = uint8_t(o[i / 4] >> (i % 4 * 8));
                else *reinterpret_cast<uint16_t*>(to) = uint16_t(o[i / 2] >> (i % 2 * 16));
            }
            if (ELEM == 1 && lane == 0) a.c.v_exp[exps_at(a.c, w.page, head) + w.start + kv_value_exp_at(t)] = uint8_t(e + 127);
        }
        if (!w.run) return;
        __syncthreads();
        uint8_t* group = a.c.v + block_at<D, ELEM>(a.c, w.page, head) + w.start * (D * ELEM);
        for (int u = threadIdx.x; u < D * ELEM * 4; u += kThreads) {    // 16-byte chunks: their element and bytes
            int d, at;
            value_chunk<D, ELEM>(u, &d, &at);
            const uint8_t* from = lds + d * kStride + at;
            if (w.count == kValueWindow) {
                u32x4 x;
                __builtin_memcpy(&x, __builtin_assume_aligned(from, 4), 16);
                reinterpret_cast<u32x4*>(group)[u] = x;
            } else {
                for (int i = 0; i < 16 / ELEM; ++i) {
                    const int j = value_token<ELEM>(at / ELEM + i) - w.place;
                    if (j < 0 || j >= w.count) continue;
                    if (ELEM == 1) group[u * 16 + i] = from[i];
                    else reinterpret_cast<uint16_t*>(group)[u * 8 + i] = reinterpret_cast<const uint16_t*>(from)[i];
                }
            }
        }
        return;
    }
    float* cos_s = reinterpret_cast<float*>(lds);
    const int parts = (a.heads[0] + b.query_heads - 1) / b.query_heads;
    const int64_t block = blockIdx.x - b.keys - b.values, token = block / parts;
    const int head0 = int(block - token * parts) * b.query_heads;
    append_token<D, ELEM, F32>(a, token, head0, min(head0 + b.query_heads, a.heads[0]), cos_s, cos_s + D / 2);
}

// ---------------------------------------------------------------------------
// read: entries back to dense bf16 rows; a slot outside the cache reads zeros.
// A lane takes 8 elements of one token and head.  Many tokens: a workgroup takes
// 64 of a head, and where their slots fill a group it loads that whole, without
// gaps, and turns it into rows in LDS (8192 tokens of 8 heads in 8 bits: 11.1
// us, 4.6 TB/s; one token 2.3).
// ---------------------------------------------------------------------------
template <int D, int ELEM>
__device__ inline u32x4 read_key(const KvView& c, int64_t page, int head, int t, int d0) {
    const uint8_t* from = c.k + block_at<D, ELEM>(c, page, head) + kv_key_at<D, ELEM>(t, d0) * ELEM;
    if (ELEM == 2) return *reinterpret_cast<const u32x4*>(from);
    const float s = exp_scale(c.k_exp[exps_at(c, page, head) + kv_key_exp_at(t)]);
    const u32x2 w = *reinterpret_cast<const u32x2*>(from);
    return u32x4{fp8_to_bf16<false>(w[0], s), fp8_to_bf16<true>(w[0], s), fp8_to_bf16<false>(w[1], s), fp8_to_bf16<true>(w[1], s)};
}

template <int D, int ELEM>
__device__ inline u32x4 read_value(const KvView& c, int64_t page, int head, int t, int d0) {
    const int64_t block = block_at<D, ELEM>(c, page, head);
    if (ELEM == 2) {
        const uint16_t* v = reinterpret_cast<const uint16_t*>(c.v + block);
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            o[j] = uint32_t(v[kv_value_at<D, 2>(t, d0 + 2 * j)]) | uint32_t(v[kv_value_at<D, 2>(t, d0 + 2 * j + 1)]) << 16;
        return o;
    }
    const float s = exp_scale(c.v_exp[exps_at(c, page, head) + kv_value_exp_at(t)]);
    u32x2 w = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j / 4] |= uint32_t(c.v[block + kv_value_at<D, 1>(t, d0 + j)]) << (j % 4 * 8);
    return u32x4{fp8_to_bf16<false>(w[0], s), fp8_to_bf16<true>(w[0], s), fp8_to_bf16<false>(w[1], s), fp8_to_bf16<true>(w[1], s)};
}

template <int D, int ELEM>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvView c, const int32_t* slots, int64_t n, uint16_t* k_out, uint16_t* v_out) {
    const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int per = c.heads * (D / 8);
    const int64_t token = i / per;
    if (token >= n) return;
    const int rest = int(i - token * per), head = rest / (D / 8), d0 = rest % (D / 8) * 8;
    int t;
    const int64_t page = page_of(c, slots[token], &t);
    const u32x4 zero = {0, 0, 0, 0};
    const int64_t at = (token * c.heads + head) * D + d0;
    if (k_out) *reinterpret_cast<u32x4*>(k_out + at) = page >= 0 ? read_key<D, ELEM>(c, page, head, t, d0) : zero;
    if (v_out) *reinterpret_cast<u32x4*>(v_out + at) = page >= 0 ? read_value<D, ELEM>(c, page, head, t, d0) : zero;
}

template <int D, int ELEM>
__global__ __launch_bounds__(kThreads) void kv_read_window_kernel(KvView c, const int32_t* slots, int64_t n, uint16_t* k_out, uint16_t* v_out) {
    constexpr int kLanes = D / 8, kTokens = kThreads / kLanes, kChunk = 16 / ELEM;
    constexpr int kRow = D * ELEM + 16;                        // bytes of a token's keys in LDS
    constexpr int kStride = kValueWindow * ELEM + 4;           // bytes of an element's tokens in LDS
    __shared__ __attribute__((aligned(16))) uint8_t k_s[kValueWindow * kRow];
    __shared__ __attribute__((aligned(16))) uint8_t v_s[D * kStride];
    const int lane = threadIdx.x % kLanes, d0 = lane * 8, mine = threadIdx.x / kLanes;
    const int head = blockIdx.x % c.heads;
    Window w;
    if (!find_window(c, slots, n, blockIdx.x / c.heads, &w)) return;
    const u32x4 zero = {0, 0, 0, 0};
    if (!w.run) {
        for (int j = mine; j < w.count; j += kTokens) {
            int t;
            const int64_t page = page_of(c, slots[w.first + j], &t), at = ((w.first + j) * c.heads + head) * D + d0;
            if (k_out) *reinterpret_cast<u32x4*>(k_out + at) = page >= 0 ? read_key<D, ELEM>(c, page, head, t, d0) : zero;
            if (v_out) *reinterpret_cast<u32x4*>(v_out + at) = page >= 0 ? read_value<D, ELEM>(c, page, head, t, d0) : zero;
        }
        return;
    }
    // the whole group, 16 bytes a lane without gaps, turned into rows in LDS
    const int64_t block = block_at<D, ELEM>(c, w.page, head) + w.start * (D * ELEM);
    constexpr int kChunks = D * ELEM * 4 / kThreads;
    u32x4 k[kChunks], v[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        k[i] = reinterpret_cast<const u32x4*>(c.k + block)[i * kThreads + threadIdx.x];
        v[i] = reinterpret_cast<const u32x4*>(c.v + block)[i * kThreads + threadIdx.x];
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int u = i * kThreads + threadIdx.x, t = u / (16 * (D / kChunk)) * 16 + (u & 15), j = u / 16 % (D / kChunk);
        *reinterpret_cast<u32x4*>(k_s + t * kRow + j * 16) = k[i];
        int d, at;
        value_chunk<D, ELEM>(u, &d, &at);
#pragma unroll
        for (int x = 0; x < 4; ++x) *reinterpret_cast<uint32_t*>(v_s + d * kStride + at + 4 * x) = v[i][x];
    }
    __syncthreads();
    for (int j = mine; j < w.count; j += kTokens) {
        const int t = w.place + j;
        const int64_t at = ((w.first + j) * c.heads + head) * D + d0, exps = exps_at(c, w.page, head) + w.start;
        u32x4 x;
        const uint8_t* from = v_s + d0 * kStride + value_byte<ELEM>(t);
        if (ELEM == 2) {
            x = *reinterpret_cast<const u32x4*>(k_s + t * kRow + d0 * 2);
            if (k_out) *reinterpret_cast<u32x4*>(k_out + at) = x;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = uint32_t(*reinterpret_cast<const uint16_t*>(from + 2 * i * kStride)) |
                       uint32_t(*reinterpret_cast<const uint16_t*>(from + (2 * i + 1) * kStride)) << 16;
        } else {
            u32x2 y = *reinterpret_cast<const u32x2*>(k_s + t * kRow + d0);
            float s = exp_scale(c.k_exp[exps + kv_key_exp_at(t)]);
            x = u32x4{fp8_to_bf16<false>(y[0], s), fp8_to_bf16<true>(y[0], s), fp8_to_bf16<false>(y[1], s), fp8_to_bf16<true>(y[1], s)};
            if (k_out) *reinterpret_cast<u32x4*>(k_out + at) = x;
            y = u32x2{0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i / 4] |= uint32_t(from[i * kStride]) << (i % 4 * 8);
            s = exp_scale(c.v_exp[exps + kv_value_exp_at(t)]);
            x = u32x4{fp8_to_bf16<false>(y[0], s), fp8_to_bf16<true>(y[0], s), fp8_to_bf16<false>(y[1], s), fp8_to_bf16<true>(y[1], s)};
        }
        if (v_out) *reinterpret_cast<u32x4*>(v_out + at) = x;
    }
}

// ---------------------------------------------------------------------------
// keep: entry starts + i <- entry starts + path[i].  A workgroup takes one
// sequence and head; path rises and path[i] >= i, so a batch of entries whose
// sources are all in registers before the first of them is written (a barrier
// between) cannot overwrite a source of a later batch.  A launch and a chain of
// loads bound it: 64 sequences of up to 64 tokens 5.8 us.
// ---------------------------------------------------------------------------
template <int D, int ELEM>
__global__ __launch_bounds__(kThreads) void kv_keep_kernel(KvKeepLaunch a) {
    constexpr int kBatch = kThreads * 16 / (D * ELEM);      // entries whose keys are one 16-byte chunk per thread
    constexpr int kElems = kBatch * D / kThreads;           // elements of their values per thread
    constexpr int kChunks = D * ELEM / 16;
    using E = typename std::conditional<ELEM == 1, uint8_t, uint16_t>::type;
    __shared__ int page_s[2][kBatch], place_s[2][kBatch];   // of an entry's source and destination; page -1: it stays
    const int seq = blockIdx.x / a.c.heads, head = blockIdx.x - seq * a.c.heads;
    const int32_t* table = a.page_table + int64_t(seq) * a.max_pages;
    const int32_t* path = a.path + int64_t(seq) * a.max_path;
    const int64_t start = a.starts[seq];
    const int count = min(a.counts[seq], a.max_path);
    auto find = [&](int64_t token, int* t) {                // a token's page, -1: none
        const int64_t p = token >> a.c.log2_page;
        *t = int(token & ((int64_t(1) << a.c.log2_page) - 1));
        if (token < 0 || p >= a.max_pages) return -1;
        const int page = table[p];
        return page >= 0 && page < a.c.num_pages ? page : -1;
    };
    for (int base = 0; base < count; base += kBatch) {
        const int some = min(count - base, kBatch);
        if (int(threadIdx.x) < some) {
            const int i = base + threadIdx.x, from = path[i];
            int page0 = -1, page1 = -1, t0 = 0, t1 = 0;
            if (from > i) {
                page0 = find(start + from, &t0);
                page1 = find(start + i, &t1);
            }
            page_s[0][threadIdx.x] = page1 >= 0 ? page0 : -1;
            page_s[1][threadIdx.x] = page1;
            place_s[0][threadIdx.x] = t0;
            place_s[1][threadIdx.x] = t1;
        }
        __syncthreads();
        auto key = [&](int end) {                           // of this thread: 0 the source's chunk, 1 the destination's
            const int i = threadIdx.x / kChunks, d = threadIdx.x % kChunks * (16 / ELEM);
            return reinterpret_cast<u32x4*>(a.c.k + block_at<D, ELEM>(a.c, page_s[end][i], head) + kv_key_at<D, ELEM>(place_s[end][i], d) * ELEM);
        };
        auto value = [&](int end, int u) {
            return reinterpret_cast<E*>(a.c.v + block_at<D, ELEM>(a.c, page_s[end][u / D], head)) + kv_value_at<D, ELEM>(place_s[end][u / D], u % D);
        };
        const bool has_key = int(threadIdx.x / kChunks) < some && page_s[0][threadIdx.x / kChunks] >= 0;
        const bool has_exp = ELEM == 1 && int(threadIdx.x) < some && page_s[0][threadIdx.x] >= 0;
        u32x4 k;
        E v[kElems];
        uint8_t exps[2];
        if (has_key) k = *key(0);
#pragma unroll
        for (int j = 0; j < kElems; ++j) {
            const int u = j * kThreads + threadIdx.x;
            if (u / D < some && page_s[0][u / D] >= 0) v[j] = *value(0, u);
        }
        if (has_exp) {
            const int64_t at = exps_at(a.c, page_s[0][threadIdx.x], head);
            exps[0] = a.c.k_exp[at + kv_key_exp_at(place_s[0][threadIdx.x])];
            exps[1] = a.c.v_exp[at + kv_value_exp_at(place_s[0][threadIdx.x])];
        }
        __syncthreads();
        if (has_key) *key(1) = k;
#pragma unroll
        for (int j = 0; j < kElems; ++j) {
            const int u = j * kThreads + threadIdx.x;
            if (u / D < some && page_s[0][u / D] >= 0) *value(1, u) = v[j];
        }
        if (has_exp) {
            const int64_t at = exps_at(a.c, page_s[1][threadIdx.x], head);
            a.c.k_exp[at + kv_key_exp_at(place_s[1][threadIdx.x])] = exps[0];
            a.c.v_exp[at + kv_value_exp_at(place_s[1][threadIdx.x])] = exps[1];
        }
        __syncthreads();
    }
}

// Rows from which windows are taken: us at 64 heads over 8, per token and in windows, 256 rows 6.0 and 7.3 (append),
// 512 10.4 and 8.5, 8192 119 and 72; read, 512 3.4 and 4.0, 1024 4.5 and 4.2, 8192 22.8 and 10.7.
constexpr int64_t kAppendWindowRows = 512, kReadWindowRows = 1024;

// All workgroups; *b: in windows.
int64_t append_blocks(const KvAppendLaunch& a, int D, AppendBlocks* b) {
    const int per = kThreads / (D / 8);
    if (a.n < kAppendWindowRows) return a.n * ((a.heads[0] + a.heads[1] + a.heads[2] + per - 1) / per);
    // one window more than the rows need: the first one may begin inside.  A workgroup takes all heads (their angles
    // once) where the rows alone are enough for the CUs, otherwise as few as it can
    const bool many = a.n >= 2048;
    b->key_heads = many ? std::max(1, a.heads[1]) : std::max(1, per / kKeyWindow);
    b->query_heads = many ? std::max(1, a.heads[0]) : per;
    const int64_t keys = ((a.n + kKeyWindow - 1) / kKeyWindow + 1) * ((a.heads[1] + b->key_heads - 1) / b->key_heads);
    const int64_t values = a.heads[2] * ((a.n + kValueWindow - 1) / kValueWindow + 1);
    b->keys = int(keys);
    b->values = int(values);
    return keys + values + a.n * ((a.heads[0] + b->query_heads - 1) / b->query_heads);
}

template <int D, int ELEM, bool F32>
hipError_t append_from(const KvAppendLaunch& a, hipStream_t stream) {
    AppendBlocks b{};
    const uint32_t blocks = uint32_t(append_blocks(a, D, &b));
    if (a.n >= kAppendWindowRows) hipLaunchKernelGGL((kv_append_window_kernel<D, ELEM, F32>), dim3(blocks), dim3(kThreads), 0, stream, a, b);
    else hipLaunchKernelGGL((kv_append_kernel<D, ELEM, F32>), dim3(blocks), dim3(kThreads), 0, stream, a, int(blocks / a.n));
    return hipGetLastError();
}

template <int D, int ELEM>
hipError_t append_as(const KvAppendLaunch& a, hipStream_t stream) {
    return a.src_f32 ? append_from<D, ELEM, true>(a, stream) : append_from<D, ELEM, false>(a, stream);
}

template <int D, int ELEM>
hipError_t read_as(const KvView& c, const int32_t* slots, int64_t n, uint16_t* k_out, uint16_t* v_out, hipStream_t stream) {
    const uint32_t blocks = uint32_t(kv_read_workgroups(c, D, n));
    if (n >= kReadWindowRows) hipLaunchKernelGGL((kv_read_window_kernel<D, ELEM>), dim3(blocks), dim3(kThreads), 0, stream, c, slots, n, k_out, v_out);
    else hipLaunchKernelGGL((kv_read_kernel<D, ELEM>), dim3(blocks), dim3(kThreads), 0, stream, c, slots, n, k_out, v_out);
    return hipGetLastError();
}

template <int D, int ELEM>
hipError_t keep_as(const KvKeepLaunch& a, hipStream_t stream) {
    hipLaunchKernelGGL((kv_keep_kernel<D, ELEM>), dim3(uint32_t(a.num_seqs) * a.c.heads), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

int64_t kv_append_workgroups(const KvAppendLaunch& a, int head_dim) {
    AppendBlocks b{};
    return append_blocks(a, head_dim, &b);
}

int64_t kv_read_workgroups(const KvView& c, int head_dim, int64_t n) {
    return n >= kReadWindowRows ? ((n + kValueWindow - 1) / kValueWindow + 1) * c.heads : (n * c.heads * (head_dim / 8) + kThreads - 1) / kThreads;
}

hipError_t launch_kv_append(const KvAppendLaunch& a, int head_dim, int elem_bytes, hipStream_t stream) {
    if (head_dim == 64) return elem_bytes == 1 ? append_as<64, 1>(a, stream) : append_as<64, 2>(a, stream);
    return elem_bytes == 1 ? append_as<128, 1>(a, stream) : append_as<128, 2>(a, stream);
}

hipError_t launch_kv_read(const KvView& c, int head_dim, int elem_bytes, const int32_t* slots, int64_t n, uint16_t* k_out, uint16_t* v_out, hipStream_t stream) {
    if (head_dim == 64) return elem_bytes == 1 ? read_as<64, 1>(c, slots, n, k_out, v_out, stream) : read_as<64, 2>(c, slots, n, k_out, v_out, stream);
    return elem_bytes == 1 ? read_as<128, 1>(c, slots, n, k_out, v_out, stream) : read_as<128, 2>(c, slots, n, k_out, v_out, stream);
}

hipError_t launch_kv_keep(const KvKeepLaunch& a, int head_dim, int elem_bytes, hipStream_t stream) {
    if (head_dim == 64) return elem_bytes == 1 ? keep_as<64, 1>(a, stream) : keep_as<64, 2>(a, stream);
    return elem_bytes == 1 ? keep_as<128, 1>(a, stream) : keep_as<128, 2>(a, stream);
}

}  // namespace tl
