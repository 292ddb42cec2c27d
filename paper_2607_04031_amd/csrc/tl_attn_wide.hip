// Attention for many rows per sequence and key head (prompts, large trees): the
// products of attn_kernel (tl_attn.hip) for 128 rows, 32 a wave, whose four
// waves share every chunk of 64 keys.  A chunk is loaded once per workgroup, as
// it lies in the pages, a chunk ahead; on its way into LDS 4- and 8-bit entries become
// bf16 operands, once instead of once per wave.  Two chunks' buffers: one is
// filled while the other is read, one barrier a chunk.  Operands of one
// instruction are 1 KB without gaps in LDS, so reads have no bank conflicts.
//
// Bound by the matrix and vector work of its waves, which hide one another's
// only in part (MFMA busy for 36 % of the cycles, 8 bits 32 %, 4 bits 38 %, at 2.12 -
// 2.15 GHz), and by the starts and ends of pieces of tiles.  Three prompts, 135
// GFLOP, bf16: 153 - 155 us, the join of partial results 13.5; trees of 64
// tokens, 107 GFLOP over 8-bit entries, 151 - 160 us, the join 10.3.  Prompts over
// 4-bit entries, 135 GFLOP, 144 - 158 us without a join (whole tiles, the longest
// first), 172 and 13.4 in equal parts: of a chunk's 3.7 thousand cycles (clock reads
// in a copy of the kernel, which cost some themselves) a wave converts for 674,
// loads for 378, multiplies for 937 and 1131, takes 405 for the softmax and 199 at
// the barrier.  4 bits sum the weights, rounded as the products take
// them, by a product with ones (2 of 34 MFMA, for 32 additions a lane), and have
// both row tiles' softmax run side by side.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "tl_attn_device.h"

namespace tl {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
static_assert(kThreads == kAttnThreads, "the limit of a launch's workgroups");
constexpr int kRowTiles = 2;            // of 16 rows, a wave's
constexpr int kRows = 16 * kRowTiles * kWaves;
constexpr int kKeys = 64;
constexpr float kSlack = 8.f;

// 16 bytes a lane from global memory (base + voff) to LDS, at the wave's base in the order of the lanes, past the
// registers.  In assembly, since the compiler has every later read of LDS wait for such loads, also one of another buffer;
// wait_for_lds_loads(), and a barrier for other waves, stand before the reads that they are for.  Nothing else in the
// kernels uses M0.
__device__ inline void load_to_lds(const uint8_t* base, uint32_t voff, u32x4* lds) {
    const uint32_t la = uint32_t(uintptr_t((__attribute__((address_space(3))) void*)lds));
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(la) : "memory", "m0");
#pragma clang diagnostic pop
}

template <int D, int ELEM>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void attn_wide_kernel(AttnLaunch a) {
    constexpr int kSteps = D / 32;                 // MFMA steps along the head
    constexpr int kOperands = D / 8;               // of a chunk's keys, and of its values: 1 KB each
    constexpr bool kFour = kv_four<ELEM>();
    constexpr int kLoads = kFour ? 1 : D * ELEM / 64;  // 16-byte loads of a thread for a chunk's keys, and for its values (4 bits: D / 8 bytes)
    constexpr int kTokenBytes = kv_width<D, ELEM>() * kv_size<ELEM>();
    constexpr int kPad = D + 4;
    __shared__ u32x4 kv_s[2][2][kOperands * 64];   // [buffer][keys, values]; at the end the waves' results
    __shared__ __attribute__((aligned(16))) float scale_s[2][kKeys];    // of the values
    __shared__ uint32_t odd_s[kRows * (D / 8)];
    __shared__ int odd_any;
    __shared__ AttnLine line;
    static_assert(kWaves * 16 * kPad * 4 <= sizeof kv_s, "results of a row tile in the buffers");
    AttnRun run;
    if (!attn_begin<D>(a, &line, &run)) return;
    const int wave = uniform(int(threadIdx.x >> 6)), row0 = wave * (16 * kRowTiles);
    for (int i = threadIdx.x; i < kRows * (D / 8); i += kThreads) odd_s[i] = 0;
    if (threadIdx.x == 0) odd_any = 0;
    __syncthreads();
    while (run.place < run.end) {
        const AttnPiece piece = attn_piece<D, kFour>(a, &line, &run);
        const Seq& s = piece.s;
        const int thread = hidden(int(threadIdx.x)), lane = thread & 63, g = lane >> 4, col = lane & 15;
        // keys below 'all' are seen by every row, keys from 'end' on by none: of the workgroup's, and of the wave's
        const int start = s.len - s.n;
        auto all_of = [&](int first) { return max(0, min(s.len, a.mask ? start : start + attn_token(a, first) + 1)); };
        auto end_of = [&](int first, int count) {
            return attn_token(a, first) >= s.rows ? 0 : max(0, min(s.len, a.mask ? s.len : start + min(s.rows - 1, attn_token(a, first + count - 1)) + 1));
        };
        const int first_row = piece.tile * kRows + row0;
        const int all_here = uniform(all_of(piece.tile * kRows)), all = uniform(all_of(first_row));
        const int chunk_end = uniform(min(piece.chunk1, (end_of(piece.tile * kRows, kRows) + kKeys - 1) / kKeys));
        const int wave_end = uniform(min(chunk_end, (end_of(first_row, 16 * kRowTiles) + kKeys - 1) / kKeys));

        // this lane's rows: queries as the second operand of K Q^T, in the order of the keys' chunks
        u32x4 q[kRowTiles][kSteps];
        int own[kRowTiles];
#pragma unroll
        for (int nt = 0; nt < kRowTiles; ++nt) {
            const int row = first_row + nt * 16 + col;
            own[nt] = attn_token(a, row);
            const bool valid = own[nt] < s.rows;
            const uint16_t* qp = a.q + int64_t(s.first + (valid ? own[nt] : 0)) * a.ldq + int64_t(piece.head * a.group + (valid ? row - own[nt] * a.group : 0)) * D;
            if (!valid) own[nt] = -1;
#pragma unroll
            for (int f = 0; f < kSteps; ++f) {
                const int d = kFour ? D / 4 * g + 8 * f : ELEM == 1 ? (4 * (f / 2) + g) * 16 + f % 2 * 8 : (4 * f + g) * 8;
                q[nt][f] = *reinterpret_cast<const u32x4*>(qp + d);        // rows past the end: the first one's, not stored
            }
        }
        f32x4v o[kRowTiles][D / 16];
        float m[kRowTiles], l[kRowTiles];
        f32x4v ones_sum[kRowTiles];     // 4 bits: the rounded weights' sums, by a product with ones (any element)
#pragma unroll
        for (int nt = 0; nt < kRowTiles; ++nt) {
            m[nt] = -INFINITY;
            l[nt] = 0.f;
            ones_sum[nt] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int db = 0; db < D / 16; ++db) o[nt][db] = f32x4v{0.f, 0.f, 0.f, 0.f};
        }

        const AttnPages pages(a, s.seq, piece.head);
        u32x4 kw[ELEM == 1 ? kLoads : 1], vw[kLoads];
        uint32_t k_exp = 0, v_exp = 0, odd = 0;
        // 4 bits: a block of 16 keys, and of the values 32 of the head's elements (head size 64: half of the keys) for each wave
        constexpr int kHalves = D / 64;
        AttnKey4<D> kw4;
        uint32_t vw4[2 * kHalves], v_exp4[2 * kHalves];
        const int value_block = kHalves == 2 ? wave : wave / 2, value_half = kHalves == 2 ? 0 : wave % 2;
        // the operand that load i of this wave's values is: (16 of the head's elements, 32 keys)
        auto value_at = [&](int i) {
            const int at = i * kWaves + wave;
            return at % (D / 16) * 2 + at / (D / 16);
        };
        // A chunk from the pages (for a page that is none: from a block that exists): 16-bit entries straight into LDS, 8-bit
        // ones into registers.
        auto fetch = [&](int64_t block, int buffer) {
            const int64_t from = max(block, int64_t(0));
            const uint8_t* kb = a.c.k + from * kTokenBytes;
            const uint8_t* vb = a.c.v + from * kTokenBytes;
            if (kFour) {
                kw4 = attn_key4<D, false>(kb + wave * 16 * kTokenBytes, lane);
                k_exp = *reinterpret_cast<const uint32_t*>(a.c.k_exp + from * kv_exps<D, ELEM>() + attn_key4_exp<D>(lane));
                const uint32_t* v = reinterpret_cast<const uint32_t*>(vb + value_block * 1024 + lane * 16) + 2 * value_half;
                const uint32_t* e = reinterpret_cast<const uint32_t*>(a.c.v_exp + from * kv_exps<D, ELEM>() + value_block * 64 + g * 16) + 2 * value_half;
                if (kHalves == 2) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(v), y = *reinterpret_cast<const u32x4*>(e);
#pragma unroll
                    for (int m = 0; m < 2 * kHalves; ++m) vw4[m] = x[m], v_exp4[m] = y[m];
                } else {
                    const u32x2 x = *reinterpret_cast<const u32x2*>(v), y = *reinterpret_cast<const u32x2*>(e);
#pragma unroll
                    for (int m = 0; m < 2 * kHalves; ++m) vw4[m] = x[m & 1], v_exp4[m] = y[m & 1];
                }
                return;
            }
            if (ELEM == 2) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int at = i * kWaves + wave;
                    load_to_lds(kb + at * 1024, lane * 16, kv_s[buffer][0] + at * 64);
                    load_to_lds(vb + at * 1024, lane * 16, kv_s[buffer][1] + value_at(i) * 64);
                }
                return;
            }
            const u32x4* kp = reinterpret_cast<const u32x4*>(kb) + thread;
            const u32x4* vp = reinterpret_cast<const u32x4*>(vb) + thread;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) kw[i] = kp[i * kThreads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) vw[i] = vp[i * kThreads];
            k_exp = *reinterpret_cast<const uint32_t*>(a.c.k_exp + from + col * 4);
            if (thread < kKeys) v_exp = a.c.v_exp[from + kv_value_exp_at(thread)];
        };
        // What is left to do to a chunk that was fetched: 8-bit entries become operands in LDS.  Where some row does not see
        // all of it, entries past the end may be anything, and their scales and values count as 0; so do infinities and NaNs
        // among the others for now: 0 * NaN would reach rows that do not see the key.
        auto put = [&](auto may_mask, int buffer, int chunk) {
            u32x4* ks = kv_s[buffer][0] + lane;
            u32x4* vs = kv_s[buffer][1] + lane;
            const bool masked = decltype(may_mask)::value && chunk * kKeys + kKeys > all_here;
            if (kFour) {
                const float scale = attn_exp4(k_exp >> (8 * wave), 0);
#pragma unroll
                for (int f = 0; f < kSteps; ++f) ks[(wave * kSteps + f) * 64] = fp4_to_bf16x8(kw4.step[f], scale);
                uint32_t some = 0;
                if (masked) {           // any code is a finite number, under a finite scale
#pragma unroll
                    for (int m = 0; m < 2 * kHalves; ++m) {
                        v_exp4[m] &= attn_first_bytes(s.len - chunk * kKeys - 4 * g - 16 * (2 * value_half + m));
                        some |= attn_odd_exps(v_exp4[m]);
                    }
                }
                const bool odd_exps = masked && __ballot(some);
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    u32x4 vf[2];
                    attn_values4(vw4[2 * h], vw4[2 * h + 1], v_exp4[2 * h], v_exp4[2 * h + 1], &vf[0], &vf[1]);
                    if (odd_exps) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const uint32_t bad = attn_odd<2>(vf[j / 4][j % 4]);
                            vf[j / 4][j % 4] &= ~bad;
                            odd |= bad;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) vs[((2 * value_block + j) * 2 + value_half + h) * 64] = vf[j];
                }
                return;
            }
            if (masked) {
                const int left = s.len - chunk * kKeys;             // keys of the chunk that exist
                if (thread >= left) v_exp = 0;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    if (ELEM == 2) vw[i] = vs[value_at(i) * 64];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int first = ELEM == 1 ? 16 * j : (i * kWaves + wave) / (D / 16) * 32 + 16 * (j >> 1) + 2 * (j & 1);
                        vw[i][j] &= ELEM == 1 ? attn_first_bytes(left - 4 * g - first) : attn_first_halves(left - 4 * g - first);
                        const uint32_t bad = attn_odd<ELEM>(vw[i][j]);
                        vw[i][j] &= ~bad;
                        odd |= bad;
                    }
                    if (ELEM == 2) vs[value_at(i) * 64] = vw[i];
                }
            }
            if (ELEM == 2) return;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int at = i * kWaves + wave;
                constexpr int kPer = D / 64;            // loads of a 16-key block
                const float scale = exp_scale(k_exp >> (8 * (at / kPer)) & 0xff);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t k0 = kw[ELEM == 1 ? i : 0][2 * h], k1 = kw[ELEM == 1 ? i : 0][2 * h + 1], v0 = vw[i][2 * h], v1 = vw[i][2 * h + 1];
                    ks[(2 * at + h) * 64] = u32x4{fp8_to_bf16<false>(k0, scale), fp8_to_bf16<true>(k0, scale), fp8_to_bf16<false>(k1, scale), fp8_to_bf16<true>(k1, scale)};
                    vs[(2 * at + h) * 64] = u32x4{fp8_to_bf16<false>(v0, 1.f), fp8_to_bf16<true>(v0, 1.f), fp8_to_bf16<false>(v1, 1.f), fp8_to_bf16<true>(v1, 1.f)};
                }
            }
            if (thread < kKeys) scale_s[buffer][thread] = exp_scale(min(v_exp, 0xfeu));    // as attn_full_bytes
        };
        // Operands are read from LDS four ahead of the products that take them: left to itself, the compiler reads one
        // and waits for it, twenty times a chunk.  A wave in its products goes before the other one of its SIMD (8 bits: 1 - 2 %
        // less time, 16 bits the same).
        auto compute = [&](auto may_mask, int buffer, int chunk) {
            const u32x4* ks = kv_s[buffer][0] + lane;
            const u32x4* vs = kv_s[buffer][1] + lane;
            // what the rows see, before the products need the registers
            const bool masked = decltype(may_mask)::value && chunk * kKeys + kKeys > all;
            uint32_t seen[kRowTiles];
            if (masked) {
                const int key0 = chunk * kKeys + 4 * g, left = s.len - key0;
#pragma unroll
                for (int nt = 0; nt < kRowTiles; ++nt) seen[nt] = own[nt] >= 0 ? attn_seen<4>(a, s, own[nt], key0 - start, left) : 0u;
            }
            // S^T: keys 16 mb + 4 g + i of the chunk, row col
            f32x4v x[kRowTiles][4];
            u32x4 kf[2][4], vf[2][4];
#pragma unroll
            for (int nt = 0; nt < kRowTiles; ++nt)
#pragma unroll
                for (int mb = 0; mb < 4; ++mb) x[nt][mb] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int mb = 0; mb < 4; ++mb) kf[0][mb] = ks[mb * kSteps * 64];
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int f = 0; f < kSteps; ++f) {
                __builtin_amdgcn_sched_barrier(0);
                if (f + 1 < kSteps) {
#pragma unroll
                    for (int mb = 0; mb < 4; ++mb) kf[(f + 1) & 1][mb] = ks[(mb * kSteps + f + 1) * 64];
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) vf[0][i] = vs[i * 64];
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int mb = 0; mb < 4; ++mb)
#pragma unroll
                    for (int nt = 0; nt < kRowTiles; ++nt) x[nt][mb] = mfma_16x16x32(kf[f & 1][mb], q[nt][f], x[nt][mb]);
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            if (masked) {
#pragma unroll
                for (int nt = 0; nt < kRowTiles; ++nt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[nt][e >> 2][e & 3] = seen[nt] >> e & 1 ? x[nt][e >> 2][e & 3] : -INFINITY;
            }
            // running maximum and sum, as in attn_kernel
            u32x4 p[kRowTiles][2];
            if (kFour) {
                // both row tiles together: the one's instructions run while the other's results are on their way
                float top[kRowTiles];
                bool grows = false;
#pragma unroll
                for (int nt = 0; nt < kRowTiles; ++nt) {
                    top[nt] = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 16; ++e) top[nt] = fmaxf(top[nt], x[nt][e >> 2][e & 3]);
                    grows |= top[nt] * a.scale_log2 > m[nt] + kSlack;
                }
                if (__ballot(grows)) {
#pragma unroll
                    for (int nt = 0; nt < kRowTiles; ++nt) {
                        top[nt] = fmaxf(top[nt], __shfl_xor(top[nt], 16));
                        top[nt] = fmaxf(top[nt], __shfl_xor(top[nt], 32));
                        const float grown = fmaxf(m[nt], top[nt] * a.scale_log2);
                        const float shrink = __builtin_amdgcn_exp2f(m[nt] - (grown == -INFINITY ? 0.f : grown));
                        m[nt] = grown;
                        ones_sum[nt] *= shrink;
#pragma unroll
                        for (int db = 0; db < D / 16; ++db) o[nt][db] *= shrink;
                    }
                }
                float base[kRowTiles];
#pragma unroll
                for (int nt = 0; nt < kRowTiles; ++nt) base[nt] = m[nt] == -INFINITY ? 0.f : m[nt];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
#pragma unroll
                        for (int nt = 0; nt < kRowTiles; ++nt) {
                            const f32x4v& z = x[nt][2 * h + (e >> 2)];
                            p[nt][h][e / 2] = pack_bf16(__builtin_amdgcn_exp2f(__builtin_fmaf(z[e & 3], a.scale_log2, -base[nt])),
                                                        __builtin_amdgcn_exp2f(__builtin_fmaf(z[(e & 3) + 1], a.scale_log2, -base[nt])));
                        }
            }
#pragma unroll
            for (int nt = 0; nt < (kFour ? 0 : kRowTiles); ++nt) {
                float top = -INFINITY;
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, x[nt][e >> 2][e & 3]);
                if (__ballot(top * a.scale_log2 > m[nt] + kSlack)) {
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float want = top * a.scale_log2;
                    const float grown = fmaxf(m[nt], want);
                    const float shrink = __builtin_amdgcn_exp2f(m[nt] - (grown == -INFINITY ? 0.f : grown));
                    m[nt] = grown;
                    l[nt] *= shrink;
#pragma unroll
                    for (int db = 0; db < D / 16; ++db) o[nt][db] *= shrink;
                }
                const float base = m[nt] == -INFINITY ? 0.f : m[nt];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float w[8];
                    f32x4v scale[2];
                    if (ELEM == 1) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) scale[b] = *reinterpret_cast<const f32x4v*>(&scale_s[buffer][16 * (2 * h + b) + 4 * g]);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[nt][2 * h + (e >> 2)][e & 3], a.scale_log2, -base));
                        l[nt] += y;
                        w[e] = ELEM == 1 ? y * scale[e >> 2][e & 3] : y;
                    }
                    p[nt][h] = u32x4{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])};
                }
            }
            // O^T: elements 16 db + 4 g + i of the head, row col
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int t = 0; t < D / 32; ++t) {
                __builtin_amdgcn_sched_barrier(0);
                if (t + 1 < D / 32) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) vf[(t + 1) & 1][i] = vs[(4 * (t + 1) + i) * 64];
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int nt = 0; nt < kRowTiles; ++nt) o[nt][2 * t + i / 2] = mfma_16x16x32(vf[t & 1][i], p[nt][i & 1], o[nt][2 * t + i / 2]);
                if (kFour && t < 2) {
#pragma unroll
                    for (int nt = 0; nt < kRowTiles; ++nt) ones_sum[nt] = mfma_16x16x32(u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}, p[nt][t & 1], ones_sum[nt]);
                }
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        };

        // 4- and 8-bit chunks go from the pages to registers during the chunk but one before theirs, and on into LDS at the start of
        // the one before; 16-bit ones into LDS during the one before.
        constexpr bool kInRegisters = ELEM != 2;
        constexpr int kAhead = kInRegisters ? 2 : 1;
        int64_t block = pages.block(piece.chunk0, pages.page(piece.chunk0, chunk_end));
        int64_t next = pages.block(piece.chunk0 + 1, pages.page(piece.chunk0 + 1, chunk_end));
        int next_page = pages.page(piece.chunk0 + 2, chunk_end);
        if (piece.chunk0 < chunk_end) {
            fetch(block, 0);
            if (ELEM == 2) wait_for_lds_loads();
            put(std::true_type(), 0, piece.chunk0);
            if (kInRegisters) fetch(next, 0);
        }
        wait_for_lds_loads();
        __syncthreads();
        // chunks that all rows see whole, and the next one too; then the others
        int chunk = piece.chunk0;
        auto go = [&](auto may_mask, int before) {
            constexpr bool kMasked = decltype(may_mask)::value;
            for (; chunk < before; ++chunk) {
                const int buffer = (chunk - piece.chunk0) & 1;
                const bool more = !kMasked || chunk + 1 < chunk_end;
                if (kInRegisters && more) put(may_mask, buffer ^ 1, chunk + 1);
                const int64_t after = pages.block(chunk + 2, next_page);
                next_page = pages.page(chunk + 3, chunk_end);
                if (kInRegisters || more) fetch(kAhead == 2 ? after : next, buffer ^ 1);
                if (block >= 0 && (!kMasked || chunk < wave_end)) compute(may_mask, buffer, chunk);
                if (ELEM == 2) {
                    wait_for_lds_loads();
                    if (kMasked && more) put(may_mask, buffer ^ 1, chunk + 1);
                }
                block = next;
                next = after;
                __syncthreads();
            }
        };
        go(std::false_type(), min(chunk_end, all_here / kKeys) - 1);
        go(std::true_type(), chunk_end);

        if (__ballot(odd)) odd_any = 1;
        __syncthreads();
        if (odd_any) {
            for (int c = piece.chunk0; c < wave_end; ++c) {
                const int64_t at = pages.block(c, pages.page(c, chunk_end));
                if (c * kKeys + kKeys <= all_here || at < 0) continue;
#pragma unroll 1
                for (int nt = 0; nt < kRowTiles; ++nt) attn_odd_chunk<D, ELEM, 4>(a, piece, c, at, row0 + nt * 16 + col, odd_s);
            }
        }
        const int lane2 = hidden(int(threadIdx.x & 63)), g2 = lane2 >> 4, col2 = lane2 & 15;
        // a wave's results, a row tile at a time, through LDS of its own
        float* mine = reinterpret_cast<float*>(kv_s) + wave * 16 * kPad;
#pragma unroll
        for (int nt = 0; nt < kRowTiles; ++nt) {
            l[nt] += __shfl_xor(l[nt], 16);
            l[nt] += __shfl_xor(l[nt], 32);
            if (kFour) l[nt] = ones_sum[nt][0];
#pragma unroll
            for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4v*>(mine + col2 * kPad + db * 16 + 4 * g2) = o[nt][db];
            __builtin_amdgcn_wave_barrier();
            for (int u = lane2; u < 16 * (D / 8); u += 64) {
                const int r = u / (D / 8), row = row0 + nt * 16 + r, d = u % (D / 8) * 8;
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = mine[r * kPad + d + j];
                if (odd_any) attn_add_odd(odd_s[row * (D / 8) + d / 8], x);
                attn_put<D>(a, piece, row, d, x, __shfl(m[nt], r), __shfl(l[nt], r));
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        if (odd_any) {          // uniform
            for (int i = threadIdx.x; i < kRows * (D / 8); i += kThreads) odd_s[i] = 0;
            __syncthreads();
            if (threadIdx.x == 0) odd_any = 0;
            __syncthreads();
        }
    }
}

}  // namespace

hipError_t launch_attn_wide(const AttnLaunch& a, int head_dim, int elem_bytes, hipStream_t stream) {
    return kv_as(head_dim, elem_bytes, [&](auto d, auto e) {
        hipLaunchKernelGGL((attn_wide_kernel<d(), e()>), dim3(a.groups), dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    });
}

}  // namespace tl
