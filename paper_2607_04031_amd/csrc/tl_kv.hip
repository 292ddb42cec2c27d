// The paged key/value cache: rotary positions and quantisation on the way in,
// reading entries back, and moving the entries of an accepted path.
#include <hip/hip_runtime.h>

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {
namespace {

constexpr int kThreads = 256;

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
// is exact and each element is rounded once.  A workgroup takes one token and
// kThreads / (D / 8) of its heads; a lane holds 8 elements of one head.  The
// angle position * inv_freq is reduced to a fraction of a turn in 64 bits (at
// position 10^5 its 32-bit product would be off by 0.005) once per pair and
// token, through LDS.  Bound by HBM for prompts (every row once in, queries and
// entries once out) and by the launch for a few tokens.
// ---------------------------------------------------------------------------
template <int D, int ELEM, bool SRC_F32>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvAppendLaunch a, int head_blocks) {
    constexpr int kLanes = D / 8, kHeads = kThreads / kLanes;
    __shared__ float cos_s[D / 2], sin_s[D / 2];
    const int64_t token = blockIdx.x / head_blocks;
    const int lane = threadIdx.x % kLanes, d0 = lane * 8;
    int head = (blockIdx.x - token * head_blocks) * kHeads + threadIdx.x / kLanes;
    int which = 0;
    if (head >= a.heads[0]) {
        head -= a.heads[0];
        which = 1;
        if (head >= a.heads[1]) {
            head -= a.heads[1];
            which = head < a.heads[2] ? 2 : 3;
        }
    }
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    if (which < 3) {
        const int64_t at = token * a.ld[which] + int64_t(head) * D + d0;
        if (SRC_F32) {
            const f32x4v* p = reinterpret_cast<const f32x4v*>(static_cast<const float*>(a.src[which]) + at);
            const f32x4v u = p[0], v = p[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = u[i], x[4 + i] = v[i];
        } else {
            const u32x4 u = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.src[which]) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(u[i]), x[2 * i + 1] = bf16_hi(u[i]);
        }
    }
    const int slot = a.slots ? a.slots[token] : -1;
    const int half = a.rot_dim / 2;
    if (a.rot_dim) {
        const int pair = threadIdx.x;
        if (pair < half) {
            const int axis = pair < a.sections[0] ? 0 : pair < a.sections[0] + a.sections[1] ? 1 : 2;
            const double turns = double(a.positions[axis * a.n + token]) * double(a.inv_freq[pair]) * 0.15915494309189533577;
            const float frac = float(turns - rint(turns));
            sincospif(2.f * frac, &sin_s[pair], &cos_s[pair]);
        }
        __syncthreads();
        if (which < 2) {   // heads lie in whole groups of lanes: the partner lanes are in this branch too
            float y[8];
            if (a.interleaved) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const bool in = d0 + i < a.rot_dim;
                    const float c = in ? cos_s[(d0 + i) / 2] : 1.f, s = in ? sin_s[(d0 + i) / 2] : 0.f;
                    y[i] = x[i] * c - x[i + 1] * s;
                    y[i + 1] = x[i + 1] * c + x[i] * s;
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
                    y[i] = low ? x[i] * c - other * s : x[i] * c + other * s;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = y[i];
        }
    }
    if (which == 0) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        *reinterpret_cast<u32x4*>(a.q_out + (token * a.heads[0] + head) * D + d0) = o;
        return;
    }
    int t = 0;
    const int64_t page = page_of(a.c, slot, &t);
    if (which > 2 || page < 0) return;
    const int64_t block = block_at<D, ELEM>(a.c, page, head);
    if (ELEM == 2) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        if (which == 1) {
            *reinterpret_cast<u32x4*>(a.c.k + block + kv_key_at<D, 2>(t, d0) * 2) = o;
        } else {
            uint16_t* v = reinterpret_cast<uint16_t*>(a.c.v + block);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[kv_value_at<D, 2>(t, d0 + i)] = uint16_t(o[i / 2] >> (i % 2 * 16));
        }
        return;
    }
    float amax = 0.f;   // NaN elements take no part
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) amax = fmaxf(amax, __shfl_xor(amax, m));
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
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        o[i] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true));
    }
    const int64_t exps = exps_at(a.c, page, head);
    if (which == 1) {
        *reinterpret_cast<u32x2*>(a.c.k + block + kv_key_at<D, 1>(t, d0)) = o;
        if (lane == 0) a.c.k_exp[exps + kv_key_exp_at(t)] = uint8_t(e + 127);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) a.c.v[block + kv_value_at<D, 1>(t, d0 + i)] = uint8_t(o[i / 4] >> (i % 4 * 8));
        if (lane == 0) a.c.v_exp[exps + kv_value_exp_at(t)] = uint8_t(e + 127);
    }
}

// ---------------------------------------------------------------------------
// read: entries back to dense bf16 rows; a slot outside the cache reads zeros.
// A lane takes 8 elements of one token and head.
// ---------------------------------------------------------------------------
template <int D, int ELEM>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvView c, const int32_t* slots, int64_t n, uint16_t* k_out, uint16_t* v_out) {
    const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int per = c.heads * (D / 8);
    const int64_t token = i / per;
    if (token >= n) return;
    const int rest = int(i - token * per), head = rest / (D / 8), d0 = rest % (D / 8) * 8;
    int t;
    const int64_t page = page_of(c, slots[token], &t);
    u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (page >= 0) {
        const int64_t block = block_at<D, ELEM>(c, page, head);
        if (ELEM == 2) {
            k = *reinterpret_cast<const u32x4*>(c.k + block + kv_key_at<D, 2>(t, d0) * 2);
            const uint16_t* vp = reinterpret_cast<const uint16_t*>(c.v + block);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = uint32_t(vp[kv_value_at<D, 2>(t, d0 + 2 * j)]) | uint32_t(vp[kv_value_at<D, 2>(t, d0 + 2 * j + 1)]) << 16;
        } else {
            const int64_t exps = exps_at(c, page, head);
            const float ks = exp_scale(c.k_exp[exps + kv_key_exp_at(t)]), vs = exp_scale(c.v_exp[exps + kv_value_exp_at(t)]);
            const u32x2 w = *reinterpret_cast<const u32x2*>(c.k + block + kv_key_at<D, 1>(t, d0));
            u32x2 x = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j / 4] |= uint32_t(c.v[block + kv_value_at<D, 1>(t, d0 + j)]) << (j % 4 * 8);
            k = u32x4{fp8_to_bf16<false>(w[0], ks), fp8_to_bf16<true>(w[0], ks), fp8_to_bf16<false>(w[1], ks), fp8_to_bf16<true>(w[1], ks)};
            v = u32x4{fp8_to_bf16<false>(x[0], vs), fp8_to_bf16<true>(x[0], vs), fp8_to_bf16<false>(x[1], vs), fp8_to_bf16<true>(x[1], vs)};
        }
    }
    const int64_t at = (token * c.heads + head) * D + d0;
    if (k_out) *reinterpret_cast<u32x4*>(k_out + at) = k;
    if (v_out) *reinterpret_cast<u32x4*>(v_out + at) = v;
}

// ---------------------------------------------------------------------------
// keep: entry starts + i <- entry starts + path[i].  A workgroup takes one
// sequence and head; path rises and path[i] >= i, so a batch of entries whose
// sources are all in registers before the first of them is written (a barrier
// between) cannot overwrite a source of a later batch.
// ---------------------------------------------------------------------------
template <int D, int ELEM>
__global__ __launch_bounds__(kThreads) void kv_keep_kernel(KvKeepLaunch a) {
    constexpr int kBatch = kThreads * 16 / (D * ELEM);      // entries whose keys are one 16-byte chunk per thread
    constexpr int kElems = kBatch * D / kThreads;           // elements of their values per thread
    constexpr int kChunks = D * ELEM / 16;
    using E = typename std::conditional<ELEM == 1, uint8_t, uint16_t>::type;
    const int seq = blockIdx.x / a.c.heads, head = blockIdx.x - seq * a.c.heads;
    const int32_t* table = a.page_table + int64_t(seq) * a.max_pages;
    const int32_t* path = a.path + int64_t(seq) * a.max_path;
    const int64_t start = a.starts[seq];
    const int count = min(a.counts[seq], a.max_path);
    // page (or -1) and place of a sequence's token
    auto find = [&](int64_t token, int* t) -> int64_t {
        const int64_t p = token >> a.c.log2_page;
        *t = int(token & ((int64_t(1) << a.c.log2_page) - 1));
        if (token < 0 || p >= a.max_pages) return -1;
        const int64_t page = table[p];
        return page >= 0 && page < a.c.num_pages ? page : -1;
    };
    auto moves = [&](int i) { return i < count && path[i] > i; };
    for (int base = 0; base < count; base += kBatch) {
        u32x4 key;
        E value[kElems];
        uint8_t exps[2];
        bool has_key = false, has_exp = false;
        uint32_t has_value = 0;
        int t;
        {
            const int i = base + threadIdx.x / kChunks, d = threadIdx.x % kChunks * (16 / ELEM);
            int64_t page = moves(i) ? find(start + path[i], &t) : -1;
            if (page >= 0) {
                has_key = true;
                key = *reinterpret_cast<const u32x4*>(a.c.k + block_at<D, ELEM>(a.c, page, head) + kv_key_at<D, ELEM>(t, d) * ELEM);
            }
        }
#pragma unroll
        for (int j = 0; j < kElems; ++j) {
            const int u = j * kThreads + threadIdx.x, i = base + u / D, d = u % D;
            const int64_t page = moves(i) ? find(start + path[i], &t) : -1;
            if (page >= 0) {
                has_value |= 1u << j;
                value[j] = reinterpret_cast<const E*>(a.c.v + block_at<D, ELEM>(a.c, page, head))[kv_value_at<D, ELEM>(t, d)];
            }
        }
        if (ELEM == 1 && threadIdx.x < kBatch) {
            const int i = base + threadIdx.x;
            const int64_t page = moves(i) ? find(start + path[i], &t) : -1;
            if (page >= 0) {
                has_exp = true;
                exps[0] = a.c.k_exp[exps_at(a.c, page, head) + kv_key_exp_at(t)];
                exps[1] = a.c.v_exp[exps_at(a.c, page, head) + kv_value_exp_at(t)];
            }
        }
        __syncthreads();
        if (has_key) {
            const int i = base + threadIdx.x / kChunks, d = threadIdx.x % kChunks * (16 / ELEM);
            const int64_t page = find(start + i, &t);
            if (page >= 0) *reinterpret_cast<u32x4*>(a.c.k + block_at<D, ELEM>(a.c, page, head) + kv_key_at<D, ELEM>(t, d) * ELEM) = key;
        }
#pragma unroll
        for (int j = 0; j < kElems; ++j) {
            const int u = j * kThreads + threadIdx.x, i = base + u / D, d = u % D;
            if (has_value >> j & 1) {
                const int64_t page = find(start + i, &t);
                if (page >= 0) reinterpret_cast<E*>(a.c.v + block_at<D, ELEM>(a.c, page, head))[kv_value_at<D, ELEM>(t, d)] = value[j];
            }
        }
        if (has_exp) {
            const int64_t page = find(start + base + threadIdx.x, &t);
            if (page >= 0) {
                a.c.k_exp[exps_at(a.c, page, head) + kv_key_exp_at(t)] = exps[0];
                a.c.v_exp[exps_at(a.c, page, head) + kv_value_exp_at(t)] = exps[1];
            }
        }
        __syncthreads();
    }
}

template <int D, int ELEM>
hipError_t append_as(const KvAppendLaunch& a, hipStream_t stream) {
    const int per = kThreads / (D / 8);
    const int blocks = (a.heads[0] + a.heads[1] + a.heads[2] + per - 1) / per;
    const dim3 grid(uint32_t(a.n * blocks));
    if (a.src_f32) hipLaunchKernelGGL((kv_append_kernel<D, ELEM, true>), grid, dim3(kThreads), 0, stream, a, blocks);
    else hipLaunchKernelGGL((kv_append_kernel<D, ELEM, false>), grid, dim3(kThreads), 0, stream, a, blocks);
    return hipGetLastError();
}

template <int D, int ELEM>
hipError_t read_as(const KvView& c, const int32_t* slots, int64_t n, uint16_t* k_out, uint16_t* v_out, hipStream_t stream) {
    const int64_t lanes = n * c.heads * (D / 8);
    hipLaunchKernelGGL((kv_read_kernel<D, ELEM>), dim3(uint32_t((lanes + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, c, slots, n, k_out, v_out);
    return hipGetLastError();
}

template <int D, int ELEM>
hipError_t keep_as(const KvKeepLaunch& a, hipStream_t stream) {
    hipLaunchKernelGGL((kv_keep_kernel<D, ELEM>), dim3(uint32_t(a.num_seqs) * a.c.heads), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

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
