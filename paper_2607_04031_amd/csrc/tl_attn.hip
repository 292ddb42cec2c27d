// Attention of the new tokens of every sequence over a paged cache.
//
// One workgroup takes a tile of rows -- the (new token, query head) pairs that
// share a sequence and a key head, 16 NT of them -- and a range of the keys in
// chunks of 64; its four waves take the chunks in turn, each with a running
// maximum m and sum l per row:
//     s = q k^T scale,  m' = max(m, max s),  l = l 2^(m - m') + sum 2^(s - m'),
//     O = O 2^(m - m') + 2^(s - m') V        (s and m in units of log2 e)
// and are joined in LDS.  Keys are the rows of the first product, S^T = K Q^T
// (MFMA 16x16x32), and the values' transposes of the second, O^T = V^T P^T: a
// lane's four sums of two 16-key blocks of S^T are its eight operand elements
// of P^T, so the probabilities go from one product to the next without leaving
// the lane, and the page layout has both operands lie as 16-byte chunks in
// lane order.  8-bit entries become bf16 in registers: keys with their scale
// (a power of two: exact), values without it, the probabilities times the
// values' scale being rounded to bf16 in any case.
#include <hip/hip_runtime.h>

#include "tl_serve.h"
#include "tl_serve_device.h"

namespace tl {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// Sequence of a flat tile index and the tile's place in it: tiles go sequence
// by sequence.  Every lane of every wave calls it; false past the last tile.
struct TileAt {
    int seq, tile, first, n;   // first: row of the sequence's first new token; n: its new tokens
};
__device__ inline int offset_of(const AttnLaunch& a, int i) { return max(0, min(a.q_offsets[i], int(a.total_q))); }
__device__ bool find_tile(const AttnLaunch& a, int group, int rows, int flat, TileAt* at) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < a.num_seqs; base += 64) {
        const int b = base + lane;
        const int first = b < a.num_seqs ? offset_of(a, b) : 0;
        const int n = b < a.num_seqs ? max(0, offset_of(a, b + 1) - first) : 0;
        int upto = int((int64_t(n) * group + rows - 1) / rows);
        const int own = upto;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(upto, d);
            if (lane >= d) upto += x;
        }
        const unsigned long long past = __ballot(flat < before + upto);
        if (past) {
            const int who = __builtin_ctzll(past);
            at->seq = base + who;
            at->tile = flat - before - __shfl(upto - own, who);
            at->first = __shfl(first, who);
            at->n = __shfl(n, who);
            return true;
        }
        before += __shfl(upto, 63);
    }
    return false;
}

// What a tile's rows may see, and in how many units of work.
struct Reach {
    int len, start;     // keys of the sequence; key of its first new token
    int end;            // keys that any row of the tile may see
    int units;
};
__device__ inline Reach reach_of(const AttnLaunch& a, const TileAt& at, int group, int rows) {
    Reach r;
    const int64_t room = min(a.max_pages << a.c.log2_page, a.max_len);
    r.len = int(max(int64_t(0), min(int64_t(a.lens[at.seq]), room)));
    r.start = r.len - at.n;
    const int last = min(at.n - 1, (at.tile * rows + rows - 1) / group);
    r.end = a.mask ? r.len : max(0, min(r.len, r.start + last + 1));
    const int chunks = (r.end + 63) / 64;
    r.units = max(1, (chunks + a.chunks_per_unit - 1) / a.chunks_per_unit);
    return r;
}

template <int D, int NT>
struct PartialSize {
    static constexpr int kRows = 16 * NT, kFloats = kRows * (D + 2);
};

template <int D, int ELEM, int NT>
__global__ __launch_bounds__(kThreads) void attn_kernel(AttnLaunch a) {
    constexpr int kRows = 16 * NT;
    constexpr int kLoads = D * ELEM / 16;          // 1 KB loads of a chunk's keys, and of its values
    constexpr int kSteps = D / 32;                 // MFMA steps along the head
    constexpr int kPad = D + 4;
    __shared__ float o_s[kRows * kPad];
    __shared__ float m_s[kWaves][kRows], l_s[kWaves][kRows];
    const int heads = a.c.heads, group = a.q_heads / heads;
    const int head = blockIdx.x % heads, rest = blockIdx.x / heads;
    const int unit = rest % a.max_units, flat = rest / a.max_units;
    TileAt at;
    if (!find_tile(a, group, kRows, flat, &at)) return;
    const Reach r = reach_of(a, at, group, kRows);
    if (unit >= r.units) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;

    // this lane's rows: queries as the second operand of K Q^T, in the order of the keys' chunks
    s16x8 q[NT][kSteps];
    int sees[NT];                  // causal: keys below this one; tree: the row's mask words start here
    bool valid[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = at.tile * kRows + nt * 16 + col;
        const int i = row / group;
        valid[nt] = i < at.n;
        sees[nt] = a.mask ? i : r.start + i + 1;
        const uint16_t* qp = a.q + int64_t(at.first + (valid[nt] ? i : 0)) * a.ldq + int64_t(head * group + (valid[nt] ? row % group : 0)) * D;
#pragma unroll
        for (int f = 0; f < kSteps; ++f) {
            const int d = ELEM == 1 ? (4 * (f / 2) + g) * 16 + f % 2 * 8 : (4 * f + g) * 8;
            q[nt][f] = valid[nt] ? *reinterpret_cast<const s16x8*>(qp + d) : s16x8{0, 0, 0, 0, 0, 0, 0, 0};
        }
    }
    // chunks below this one are seen whole by every row
    const int whole = a.mask ? max(0, r.start) / 64 : max(0, min(r.len, r.start + at.tile * kRows / group + 1)) / 64;

    f32x4v o[NT][D / 16];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = -INFINITY;
        l[nt] = 0.f;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) o[nt][db] = f32x4v{0.f, 0.f, 0.f, 0.f};
    }
    const int chunk_end = min((unit + 1) * a.chunks_per_unit, (r.end + 63) / 64);
    const int32_t* table = a.page_table + int64_t(at.seq) * a.max_pages;
    const int log2_chunks = a.c.log2_page - 6;     // chunks of a page
    for (int chunk = unit * a.chunks_per_unit + wave; chunk < chunk_end; chunk += kWaves) {
        const int64_t page = table[chunk >> log2_chunks];
        if (page < 0 || page >= a.c.num_pages) continue;       // a page that is none: keys that nobody sees
        const int in_page = chunk & ((1 << log2_chunks) - 1);
        const int64_t block = ((page * heads + head) << a.c.log2_page) + in_page * 64;   // first key, in tokens
        const u32x4* kp = reinterpret_cast<const u32x4*>(a.c.k + block * (D * ELEM)) + lane;
        const u32x4* vp = reinterpret_cast<const u32x4*>(a.c.v + block * (D * ELEM)) + lane;
        u32x4 kw[kLoads], vw[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) kw[i] = kp[i * 64];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) vw[i] = vp[i * 64];
        uint32_t k_exp = 0;
        u32x4 v_exp = {0, 0, 0, 0};
        if (ELEM == 1) {
            k_exp = *reinterpret_cast<const uint32_t*>(a.c.k_exp + block + col * 4);
            v_exp = *reinterpret_cast<const u32x4*>(a.c.v_exp + block + g * 16);
        }
        // S^T: keys 16 mb + 4 g + i of the chunk, row col
        f32x4v s[NT][4];
#pragma unroll
        for (int mb = 0; mb < 4; ++mb) {
            s16x8 kf[kSteps];
            if (ELEM == 1) {
                const float scale = exp_scale(k_exp >> (8 * mb) & 0xff);
#pragma unroll
                for (int f = 0; f < kSteps; ++f) {
                    const u32x4 w = kw[mb * (kLoads / 4) + f / 2];
                    const uint32_t lo = w[f % 2 * 2], hi = w[f % 2 * 2 + 1];
                    kf[f] = __builtin_bit_cast(s16x8, u32x4{fp8_to_bf16<false>(lo, scale), fp8_to_bf16<true>(lo, scale),
                                                            fp8_to_bf16<false>(hi, scale), fp8_to_bf16<true>(hi, scale)});
                }
            } else {
#pragma unroll
                for (int f = 0; f < kSteps; ++f) kf[f] = __builtin_bit_cast(s16x8, kw[mb * (kLoads / 4) + f]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                s[nt][mb] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int f = 0; f < kSteps; ++f)
                    s[nt][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, kf[f]),
                                                                       __builtin_bit_cast(bf16x8v, q[nt][f]), s[nt][mb], 0, 0, 0);
            }
        }
        const bool masked = chunk >= whole;
        uint32_t seen[NT];         // bit 4 mb + i
        if (masked) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                seen[nt] = 0;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = chunk * 64 + (e >> 2) * 16 + 4 * g + (e & 3);
                    bool ok = valid[nt] && key < r.len;
                    if (a.mask) {
                        const int j = key - r.start;
                        if (j >= 0) {
                            ok = ok && (j >> 5) < a.mask_words;
                            if (ok) ok = a.mask[int64_t(at.first + sees[nt]) * a.mask_words + (j >> 5)] >> (j & 31) & 1;
                        }
                    } else {
                        ok = ok && key < sees[nt];
                    }
                    seen[nt] |= uint32_t(ok) << e;
                    if (!ok) s[nt][e >> 2][e & 3] = -INFINITY;
                }
            }
        }
        // running maximum and sum; P^T as bf16 operands of two 32-key steps
        s16x8 p[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[nt][e >> 2][e & 3]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float next = fmaxf(m[nt], top * a.scale_log2);
            const float base = next == -INFINITY ? 0.f : next;
            const float shrink = __builtin_amdgcn_exp2f(m[nt] - base);
            m[nt] = next;
            float sum = 0.f, w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nt][e >> 2][e & 3], a.scale_log2, -base));
                sum += x;
                w[e] = x;
                if (ELEM == 1) w[e] = x * exp_scale(v_exp[e >> 2] >> (8 * (e & 3)) & 0xff);
            }
            if (masked) {
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = seen[nt] >> e & 1 ? w[e] : 0.f;    // a scale past the end may be anything
            }
            l[nt] = l[nt] * shrink + sum;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) o[nt][db] *= shrink;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                p[nt][h] = __builtin_bit_cast(s16x8, u32x4{pack_bf16(w[8 * h], w[8 * h + 1]), pack_bf16(w[8 * h + 2], w[8 * h + 3]),
                                                           pack_bf16(w[8 * h + 4], w[8 * h + 5]), pack_bf16(w[8 * h + 6], w[8 * h + 7])});
        }
        // O^T: elements 16 db + 4 g + i of the head, row col
        const int left = r.len - chunk * 64 - 4 * g;       // this lane's key 16 mb + i exists where that is below left
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 vf;
                if (ELEM == 1) {
                    const u32x4 w = vw[db];
                    vf = u32x4{fp8_to_bf16<false>(w[2 * h], 1.f), fp8_to_bf16<true>(w[2 * h], 1.f),
                               fp8_to_bf16<false>(w[2 * h + 1], 1.f), fp8_to_bf16<true>(w[2 * h + 1], 1.f)};
                } else {
                    vf = vw[h * (D / 16) + db];
                }
                u32x4 special = {0, 0, 0, 0};              // bf16 elements that are no finite numbers
                if (masked) {
                    bool any = false;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int k0 = (2 * h + (x >> 1)) * 16 + (x & 1) * 2;
                        vf[x] &= (k0 < left ? 0xffffu : 0u) | (k0 + 1 < left ? 0xffff0000u : 0u);
                        const uint32_t hit = ((vf[x] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((vf[x] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                        special[x] = vf[x] & hit;
                        vf[x] &= ~hit;
                        any |= hit != 0;
                    }
                    if (__ballot(any)) {
                        // 0 * NaN would reach rows that do not see the key: infinities and NaNs
                        // go in one kind at a time, to the rows that see one
#pragma unroll 1
                        for (int kind = 0; kind < 3; ++kind) {
                            u32x4 is;
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                const uint32_t lo = special[x] & 0xffffu, hi = special[x] >> 16;
                                const bool a0 = kind == 0 ? lo == 0x7f80u : kind == 1 ? lo == 0xff80u : (lo & 0x7fu) != 0;
                                const bool a1 = kind == 0 ? hi == 0x7f80u : kind == 1 ? hi == 0xff80u : (hi & 0x7fu) != 0;
                                is[x] = (a0 ? 0x3f80u : 0u) | (a1 ? 0x3f800000u : 0u);
                            }
                            const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                u32x4 ones;
#pragma unroll
                                for (int x = 0; x < 4; ++x) {
                                    const uint32_t two = seen[nt] >> (8 * h + 2 * x) & 3;
                                    ones[x] = (two & 1 ? 0x3f80u : 0u) | (two & 2 ? 0x3f800000u : 0u);
                                }
                                const f32x4v hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, is),
                                                                                           __builtin_bit_cast(bf16x8v, ones), f32x4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    if (hits[i] > 0.f) o[nt][db][i] += add;
                            }
                        }
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    o[nt][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, vf),
                                                                       __builtin_bit_cast(bf16x8v, p[nt][h]), o[nt][db], 0, 0, 0);
            }
        }
    }

    // join the waves
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        l[nt] += __shfl_xor(l[nt], 16);
        l[nt] += __shfl_xor(l[nt], 32);
        if (g == 0) {
            m_s[wave][nt * 16 + col] = m[nt];
            l_s[wave][nt * 16 + col] = l[nt];
        }
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        if (wave == w) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int row = nt * 16 + col;
                float top = m_s[0][row];
#pragma unroll
                for (int x = 1; x < kWaves; ++x) top = fmaxf(top, m_s[x][row]);
                const float f = __builtin_amdgcn_exp2f(m[nt] - (top == -INFINITY ? 0.f : top));
#pragma unroll
                for (int db = 0; db < D / 16; ++db) {
                    f32x4v* to = reinterpret_cast<f32x4v*>(o_s + row * kPad + db * 16 + 4 * g);
                    // a wave without keys adds nothing (its m is -infinity: f and o are 0)
                    *to = w ? *to + o[nt][db] * f : o[nt][db] * f;
                }
            }
        }
        __syncthreads();
    }
    for (int u = threadIdx.x; u < kRows * (D / 8); u += kThreads) {
        const int row = u / (D / 8), d = u % (D / 8) * 8;
        const int all = at.tile * kRows + row, i = all / group;
        if (i >= at.n) continue;
        float top = m_s[0][row], sum = 0.f;
#pragma unroll
        for (int x = 1; x < kWaves; ++x) top = fmaxf(top, m_s[x][row]);
#pragma unroll
        for (int x = 0; x < kWaves; ++x) sum += l_s[x][row] * __builtin_amdgcn_exp2f(m_s[x][row] - (top == -INFINITY ? 0.f : top));
        const float* from = o_s + row * kPad + d;
        if (r.units == 1) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;    // a row that sees no key: zeros
            u32x4 w;
#pragma unroll
            for (int x = 0; x < 4; ++x) w[x] = pack_bf16(from[2 * x] * inv, from[2 * x + 1] * inv);
            *reinterpret_cast<u32x4*>(a.out + (int64_t(at.first + i) * a.q_heads + head * group + all % group) * D + d) = w;
        } else {
            float* part = a.ws + ((int64_t(flat) * heads + head) * a.max_units + unit) * PartialSize<D, NT>::kFloats;
#pragma unroll
            for (int x = 0; x < 8; x += 4)
                *reinterpret_cast<f32x4v*>(part + row * D + d + x) = *reinterpret_cast<const f32x4v*>(from + x);
            if (d == 0) {
                part[kRows * D + row] = top;
                part[kRows * D + kRows + row] = sum;
            }
        }
    }
}

// Joins the units of tiles that have several, in their order.
template <int D, int NT>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnLaunch a) {
    constexpr int kRows = 16 * NT, kFloats = PartialSize<D, NT>::kFloats;
    const int heads = a.c.heads, group = a.q_heads / heads;
    const int head = blockIdx.x % heads, flat = blockIdx.x / heads;
    TileAt at;
    if (!find_tile(a, group, kRows, flat, &at)) return;
    const Reach r = reach_of(a, at, group, kRows);
    if (r.units == 1) return;
    const float* parts = a.ws + (int64_t(flat) * heads + head) * a.max_units * kFloats;
    for (int u = threadIdx.x; u < kRows * (D / 8); u += kThreads) {
        const int row = u / (D / 8), d = u % (D / 8) * 8;
        const int all = at.tile * kRows + row, i = all / group;
        if (i >= at.n) continue;
        float top = -INFINITY, sum = 0.f, o[8];
        for (int x = 0; x < r.units; ++x) top = fmaxf(top, parts[int64_t(x) * kFloats + kRows * D + row]);
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = 0.f;
        for (int x = 0; x < r.units; ++x) {
            const float* part = parts + int64_t(x) * kFloats;
            const float f = __builtin_amdgcn_exp2f(part[kRows * D + row] - base);
            sum += f * part[kRows * D + kRows + row];
            const f32x4v lo = *reinterpret_cast<const f32x4v*>(part + row * D + d), hi = *reinterpret_cast<const f32x4v*>(part + row * D + d + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += f * lo[j], o[4 + j] += f * hi[j];
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        u32x4 w;
#pragma unroll
        for (int x = 0; x < 4; ++x) w[x] = pack_bf16(o[2 * x] * inv, o[2 * x + 1] * inv);
        *reinterpret_cast<u32x4*>(a.out + (int64_t(at.first + i) * a.q_heads + head * group + all % group) * D + d) = w;
    }
}

template <int D, int ELEM, int NT>
hipError_t attn_as(const AttnLaunch& a, hipStream_t stream) {
    const uint32_t tiles = uint32_t(a.max_tiles) * a.c.heads;
    hipLaunchKernelGGL((attn_kernel<D, ELEM, NT>), dim3(tiles * a.max_units), dim3(kThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.max_units > 1) {
        hipLaunchKernelGGL((attn_join_kernel<D, NT>), dim3(tiles), dim3(kThreads), 0, stream, a);
        e = hipGetLastError();
    }
    return e;
}

template <int D, int ELEM>
hipError_t attn_rows(const AttnLaunch& a, hipStream_t stream) {
    return a.rows == 16 ? attn_as<D, ELEM, 1>(a, stream) : a.rows == 32 ? attn_as<D, ELEM, 2>(a, stream) : attn_as<D, ELEM, 4>(a, stream);
}

}  // namespace

hipError_t launch_attn(const AttnLaunch& a, int head_dim, int elem_bytes, hipStream_t stream) {
    if (head_dim == 64) return elem_bytes == 1 ? attn_rows<64, 1>(a, stream) : attn_rows<64, 2>(a, stream);
    return elem_bytes == 1 ? attn_rows<128, 1>(a, stream) : attn_rows<128, 2>(a, stream);
}

}  // namespace tl
