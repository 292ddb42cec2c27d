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
// values' scale being rounded to bf16 in any case: the operand holds no more.
// The sum l is of the unrounded ones.  Against 64 bits the error is 2.2e-3 of
// the result, of which the output's own rounding is 1.7e-3.
//
// 4-bit entries become bf16 with their scales, keys and values (exact: two
// significant bits times a power of two), as fast as an fma per pair; a byte of
// the values holds elements d and d + 16, so that two of a lane's pairs, sorted by
// v_perm, are the operands of two blocks of the head.  Any code is finite, so that
// infinities and NaNs are looked for among the scales, 64 tokens at a time, and
// among the values only where a scale can make them.  The scaled MFMA, which
// takes E2M1 as it lies, is not used: its sum was off by 8.5e-5 of sum |ab|.
//
// Single tokens are bound by HBM: 32 sequences of up to 8192 tokens, 64 heads
// over 8, 8 bits: 59 us, 5.7 TB/s, and 4.8 us for the join; 4 bits: 36 us, 4.9
// TB/s (6.3 in the middle; a workgroup's start takes over 3 us), and 4.7.  Few chunks per
// workgroup are bound by its start and end: three chains of five tokens over
// 131072, 8 heads over one, 30 us (2.5 TB/s) and 7 us, 4 bits 25 (conversions, made
// by both waves that share the keys) and 7.6; one token over 517, 6.7 us, 4 bits 7.5.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "tl_attn_device.h"

namespace tl {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
static_assert(kThreads == kAttnThreads, "the limit of a launch's workgroups");
constexpr float kSlack = 8.f;

template <int D, int ELEM, int NT, int RG>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void attn_kernel(AttnLaunch a) {
    constexpr int kRows = 16 * NT * RG;            // of the tile; a wave has 16 NT of them
    constexpr int kKeyWaves = kWaves / RG;         // waves that share rows split the chunks
    constexpr bool kFour = kv_four<ELEM>();
    constexpr int kBlocks = kFour ? 4 : 4 / ELEM;  // 16-key blocks of a chunk
    constexpr int kKeys = 16 * kBlocks;
    constexpr int kParts = NT == 2 && kBlocks == 4 ? 2 : 1;    // of a chunk, one after the other, for registers
    constexpr int kLoads = kFour ? D / 32 : D / 16;    // 1 KB loads of a chunk's keys, and of its values
    constexpr int kPer = kFour ? 1 : kLoads / kBlocks; // of a block's keys
    constexpr int kTokenBytes = kv_width<D, ELEM>() * kv_size<ELEM>();
    constexpr int kSteps = D / 32;                 // MFMA steps along the head
    constexpr int kPad = D + 4;
    // 32 rows over 4- and 8-bit keys: the queries stay in LDS (which holds the results later), for registers
    constexpr bool kQueriesInLds = NT == 2 && ELEM != 2 && D == 128;
    __shared__ __attribute__((aligned(16))) float o_s[kWaves * 16 * NT * kPad];
    __shared__ float m_s[kKeyWaves][kRows], l_s[kKeyWaves][kRows];
    // rows' elements that an infinity (bit 0), -infinity (1) or NaN (2) among the values reaches: 4 bits each
    __shared__ uint32_t odd_s[kRows * (D / 8)];
    __shared__ int odd_any;
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wave = uniform(int(threadIdx.x >> 6)), key_wave = wave % kKeyWaves, row0 = wave / kKeyWaves * (16 * NT);
    __shared__ AttnLine line;
    AttnRun run;
    if (!attn_begin<D>(a, &line, &run)) return;
    for (int i = threadIdx.x; i < kRows * (D / 8); i += kThreads) odd_s[i] = 0;
    if (threadIdx.x == 0) odd_any = 0;
    __syncthreads();
    while (run.place < run.end) {
        const AttnPiece piece = attn_piece<D, false>(a, &line, &run);
        const Seq& s = piece.s;
        const int head = piece.head, tile = piece.tile;
        // keys below 'all' are seen by every row of the wave, keys from 'end' on by none
        const int start = s.len - s.n, first_row = tile * kRows + row0;
        const int all = uniform(max(0, min(s.len, a.mask ? start : start + attn_token(a, first_row) + 1)));
        const int end = uniform(max(0, min(s.len, a.mask ? s.len : start + min(s.rows - 1, attn_token(a, first_row + 16 * NT - 1)) + 1)));
        const int chunk_end = attn_token(a, first_row) >= s.rows ? 0 : min(piece.chunk1, (end + kKeys - 1) / kKeys);

        // this lane's rows: queries as the second operand of K Q^T, in the order of the keys' chunks
        u32x4 q[kQueriesInLds ? 1 : NT][kQueriesInLds ? 1 : kSteps];
        u32x4* q_s = reinterpret_cast<u32x4*>(o_s) + row0 / 16 * kSteps * 64 + lane;
        int own[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = first_row + nt * 16 + col;
            own[nt] = attn_token(a, row);
            const bool valid = own[nt] < s.rows;
            const uint16_t* qp = a.q + int64_t(s.first + (valid ? own[nt] : 0)) * a.ldq + int64_t(head * a.group + (valid ? row - own[nt] * a.group : 0)) * D;
            if (!valid) own[nt] = -1;
#pragma unroll
            for (int f = 0; f < kSteps; ++f) {
                const int d = kFour ? D / 4 * g + 8 * f : ELEM == 1 ? (4 * (f / 2) + g) * 16 + f % 2 * 8 : (4 * f + g) * 8;
                const u32x4 x = *reinterpret_cast<const u32x4*>(qp + d);       // rows past the end: the first one's, not stored
                if (kQueriesInLds) q_s[(nt * kSteps + f) * 64] = x;            // waves that share rows write the same
                else q[nt][f] = x;
            }
        }
        f32x4v o[NT][D / 16];
        float m[NT], l[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt] = -INFINITY;
            l[nt] = 0.f;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) o[nt][db] = f32x4v{0.f, 0.f, 0.f, 0.f};
        }
        const AttnPages pages(a, s.seq, head);
        // Keys of the next chunk are loaded under this one's softmax and second product, its values under the next one's
        // first, page numbers a chunk earlier.  Past the end (and for pages that are none) a block that exists is loaded.
        u32x4 kw[kBlocks][kPer], vw[kLoads], v_exp = {0, 0, 0, 0};
        AttnKey4<D> kw4[kFour ? kBlocks : 1];
        u32x4 v_exp4[kFour ? kLoads : 1];
        uint32_t k_exp = 0;
        auto load_keys = [&](int64_t block) {
            if (kFour) {
#pragma unroll
                for (int mb = 0; mb < kBlocks; ++mb)
                    kw4[kFour ? mb : 0] = attn_key4<D, RG == 1>(a.c.k + (max(block, int64_t(0)) + 16 * mb) * kTokenBytes, lane);
                k_exp = *reinterpret_cast<const uint32_t*>(a.c.k_exp + max(block, int64_t(0)) * kv_exps<D, ELEM>() + attn_key4_exp<D>(lane));
                return;
            }
            const u32x4* p = reinterpret_cast<const u32x4*>(a.c.k + max(block, int64_t(0)) * kTokenBytes) + lane;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) kw[i / kPer][i % kPer] = RG == 1 ? __builtin_nontemporal_load(p + i * 64) : p[i * 64];
            if (ELEM == 1) k_exp = *reinterpret_cast<const uint32_t*>(a.c.k_exp + max(block, int64_t(0)) + col * 4);
        };
        auto load_values = [&](int64_t block) {
            const u32x4* p = reinterpret_cast<const u32x4*>(a.c.v + max(block, int64_t(0)) * kTokenBytes) + lane;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) vw[i] = RG == 1 ? __builtin_nontemporal_load(p + i * 64) : p[i * 64];
            if (ELEM == 1) v_exp = *reinterpret_cast<const u32x4*>(a.c.v_exp + max(block, int64_t(0)) + g * 16);
            if (kFour) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    v_exp4[kFour ? i : 0] = *reinterpret_cast<const u32x4*>(a.c.v_exp + max(block, int64_t(0)) * kv_exps<D, ELEM>() + i * 64 + g * 16);
            }
        };
        // a 32-key operand of O^T = V^T P^T: half h of an 8-bit load's 16 keys, or a whole 16-bit load
        auto value_of = [&](int db, int h) {
            const u32x4 w = vw[db];
            if (ELEM == 2) return w;
            return u32x4{fp8_to_bf16<false>(w[2 * h], 1.f), fp8_to_bf16<true>(w[2 * h], 1.f),
                         fp8_to_bf16<false>(w[2 * h + 1], 1.f), fp8_to_bf16<true>(w[2 * h + 1], 1.f)};
        };
        int chunk = piece.chunk0 + key_wave;
        int64_t block = pages.block(chunk, pages.page(chunk, chunk_end)), next = -1;
        int next_page = pages.page(chunk + kKeyWaves, chunk_end);
        uint32_t odd = 0;
        if (chunk < chunk_end) {
            load_keys(block);
            load_values(block);
        }
        wait_for_loads();
        auto step = [&](auto is_masked) {
            constexpr bool masked = decltype(is_masked)::value;
            const int left = block < 0 ? 0 : s.len - chunk * kKeys - 4 * g;        // this lane's key 16 mb + i exists below that
            bool odd_exps = false;      // 4 bits: some value of the wave's may be infinite or NaN
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
                // S^T: keys 16 mb + 4 g + i of the chunk, row col
                constexpr int kB = kBlocks / kParts;
                const int mb0 = part * kB;
                f32x4v x[NT][kB];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int mb = 0; mb < kB; ++mb) x[nt][mb] = f32x4v{0.f, 0.f, 0.f, 0.f};
                if (kQueriesInLds) asm volatile("" ::: "memory");              // read them again for every part
#pragma unroll
                for (int f = 0; f < kSteps; ++f) {
                    u32x4 qf[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) qf[nt] = kQueriesInLds ? q_s[(nt * kSteps + f) * 64] : q[kQueriesInLds ? 0 : nt][kQueriesInLds ? 0 : f];
#pragma unroll
                    for (int mb = 0; mb < kB; ++mb) {
                        u32x4 kf;
                        if (kFour) {
                            kf = fp4_to_bf16x8(kw4[kFour ? mb0 + mb : 0].step[f], attn_exp4(k_exp, mb0 + mb));
                        } else if (ELEM == 1) {
                            const float scale = exp_scale(k_exp >> (8 * (mb0 + mb)) & 0xff);
                            const uint32_t lo = kw[mb0 + mb][f / 2][f % 2 * 2], hi = kw[mb0 + mb][f / 2][f % 2 * 2 + 1];
                            kf = u32x4{fp8_to_bf16<false>(lo, scale), fp8_to_bf16<true>(lo, scale), fp8_to_bf16<false>(hi, scale), fp8_to_bf16<true>(hi, scale)};
                        } else {
                            kf = kw[mb0 + mb][f];
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) x[nt][mb] = mfma_16x16x32(kf, qf[nt], x[nt][mb]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (!masked && part == kParts - 1) load_keys(next);
                if (masked) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint32_t seen = own[nt] >= 0 ? attn_seen<kB>(a, s, own[nt], chunk * kKeys + 16 * mb0 + 4 * g - start, left - 16 * mb0) : 0u;
#pragma unroll
                        for (int e = 0; e < 4 * kB; ++e) x[nt][e >> 2][e & 3] = seen >> e & 1 ? x[nt][e >> 2][e & 3] : -INFINITY;
                    }
                    // entries past the end may be anything: their scales and values count as 0.  So do infinities and NaNs
                    // among the others for now: 0 * NaN would reach rows that do not see the key
                    if (part == 0 && kFour) {       // any code is a finite number, under a finite scale
#pragma unroll
                        for (int i = 0; i < kLoads; ++i)
#pragma unroll
                            for (int mb = 0; mb < kBlocks; ++mb) v_exp4[kFour ? i : 0][mb] &= attn_first_bytes(left - 16 * mb);
                        uint32_t some = 0;
#pragma unroll
                        for (int i = 0; i < kLoads; ++i)
#pragma unroll
                            for (int mb = 0; mb < kBlocks; ++mb) some |= attn_odd_exps(v_exp4[kFour ? i : 0][mb]);
                        odd_exps = __ballot(some) != 0;
                    }
                    if (part == 0 && !kFour) {
#pragma unroll
                        for (int mb = 0; mb < kBlocks; ++mb) {
                            v_exp[mb] &= attn_first_bytes(left - 16 * mb);
                            v_exp[mb] -= attn_full_bytes(v_exp[mb]);
                        }
#pragma unroll
                        for (int i = 0; i < kLoads; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                vw[i][j] &= ELEM == 1 ? attn_first_bytes(left - 16 * j) : attn_first_halves(left - 16 * (j >> 1) - 2 * (j & 1));
                                const uint32_t bad = attn_odd<ELEM>(vw[i][j]);
                                vw[i][j] &= ~bad;
                                odd |= bad;
                            }
                    }
                }
                if (!masked && block < 0) continue;        // a page that is none: keys that nobody sees
                // running maximum and sum, P^T (times the values' scales) as operands of 32-key steps.  The sums are
                // relative to an m up to kSlack below the maximum (a factor of at most 2^kSlack), so that they need
                // rescaling only when the maximum has grown by that
                u32x4 p[NT][kB / 2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 4 * kB; ++e) top = fmaxf(top, x[nt][e >> 2][e & 3]);
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
                    for (int h = 0; h < kB / 2; ++h) {
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[nt][2 * h + (e >> 2)][e & 3], a.scale_log2, -base));
                            l[nt] += y;
                            w[e] = ELEM == 1 ? y * exp_scale(v_exp[mb0 + 2 * h + (e >> 2)] >> (8 * (e & 3)) & 0xff) : y;
                        }
                        p[nt][h] = u32x4{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])};
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                // O^T: elements 16 db + 4 g + i of the head, row col
                if (kFour) {
#pragma unroll
                    for (int i = 0; i < kLoads; ++i)
#pragma unroll
                        for (int h = 0; h < kB / 2; ++h) {
                            const int m = mb0 + 2 * h;
                            const u32x4 e = v_exp4[kFour ? i : 0];
                            u32x4 vf[2];
                            attn_values4(vw[i][m & 3], vw[i][(m + 1) & 3], e[m & 3], e[(m + 1) & 3], &vf[0], &vf[1]);
                            if (masked && odd_exps) {
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    const uint32_t bad = attn_odd<2>(vf[j / 4][j % 4]);
                                    vf[j / 4][j % 4] &= ~bad;
                                    odd |= bad;
                                }
                            }
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) o[nt][2 * i + j] = mfma_16x16x32(vf[j], p[nt][h], o[nt][2 * i + j]);
                        }
                }
#pragma unroll
                for (int db = 0; db < (kFour ? 0 : D / 16); ++db)
#pragma unroll
                    for (int h = 0; h < kB / 2; ++h) {
                        const u32x4 vf = value_of(db, mb0 / 2 + h);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) o[nt][db] = mfma_16x16x32(vf, p[nt][h], o[nt][db]);
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (masked) load_keys(next);
            load_values(next);
        };
        // chunks that the wave's rows see whole, then the others
        auto go = [&](auto is_masked, int before) {
            for (; chunk < before; chunk += kKeyWaves) {
                next = pages.block(chunk + kKeyWaves, next_page);
                next_page = pages.page(chunk + 2 * kKeyWaves, chunk_end);
                step(is_masked);
                block = next;
            }
        };
        go(std::false_type(), min(chunk_end, all / kKeys));
        go(std::true_type(), chunk_end);

        // join the waves that share rows
        if (__ballot(odd) && lane == 0) odd_any = 1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            l[nt] += __shfl_xor(l[nt], 16);
            l[nt] += __shfl_xor(l[nt], 32);
            if (g == 0) {
                m_s[key_wave][row0 + nt * 16 + col] = m[nt];
                l_s[key_wave][row0 + nt * 16 + col] = l[nt];
            }
        }
        if (kQueriesInLds) __syncthreads();     // all have read their queries
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
                *reinterpret_cast<f32x4v*>(o_s + ((wave * NT + nt) * 16 + col) * kPad + db * 16 + 4 * g) = o[nt][db];
        __syncthreads();
        const bool odd_here = odd_any;      // of all waves; read before a faster one may set it for its next piece
        if (odd_here) {
            for (int c = piece.chunk0 + key_wave; c < chunk_end; c += kKeyWaves) {
                const int64_t at = pages.block(c, pages.page(c, chunk_end));
                if (c * kKeys + kKeys <= all || at < 0) continue;
#pragma unroll 1
                for (int nt = 0; nt < NT; ++nt) attn_odd_chunk<D, ELEM, kBlocks>(a, piece, c, at, row0 + nt * 16 + col, odd_s);
            }
            __syncthreads();
        }
        for (int u = threadIdx.x; u < kRows * (D / 8); u += kThreads) {
            const int row = u / (D / 8), d = u % (D / 8) * 8;
            // the waves that have the row, and its place with them
            const int first = row / (16 * NT) * kKeyWaves, at = row % (16 * NT);
            float top = m_s[0][row], sum = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 1; w < kKeyWaves; ++w) top = fmaxf(top, m_s[w][row]);
#pragma unroll
            for (int w = 0; w < kKeyWaves; ++w) {
                // a wave without keys adds nothing: its m is -infinity, its sums are 0
                const float f = __builtin_amdgcn_exp2f(m_s[w][row] - (top == -INFINITY ? 0.f : top));
                const float* from = o_s + ((first + w) * 16 * NT + at) * kPad + d;
                sum += l_s[w][row] * f;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] += from[j] * f;
            }
            if (odd_here) attn_add_odd(odd_s[row * (D / 8) + d / 8], x);
            attn_put<D>(a, piece, row, d, x, top, sum);
        }
        __syncthreads();
        if (odd_here) {         // uniform
            for (int i = threadIdx.x; i < kRows * (D / 8); i += kThreads) odd_s[i] = 0;
            __syncthreads();
            if (threadIdx.x == 0) odd_any = 0;
            __syncthreads();
        }
    }
}

// The workgroup of the first launch with the which-th of the tiles that it and
// later ones share; -1: there are fewer.  Every wave finds it for itself.
__device__ inline int attn_shared_tile(const AttnShared* notes, int groups, int which) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < groups; base += 64 * 8) {
        bool is[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int w = base + 64 * i + lane;
            is[i] = notes[min(w, groups - 1)].last >= 0 && w < groups;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned long long some = __ballot(is[i]);
            const unsigned long long it = __ballot(is[i] && __popcll(some & ((1ull << lane) - 1)) == which);
            if (it) return base + 64 * i + __builtin_ctzll(it);
            which -= __popcll(some);
        }
    }
    return -1;
}

// Joins the partial results of a tile that begins in one workgroup of the first
// launch and ends in a later one, in their order: ROWS rows of it, a thread for
// eight elements, the parts dealt to groups of threads.  FEW tiles: the
// blockIdx.x-th one that is shared; else the one of workgroup blockIdx.x.
template <int D, int ROWS, bool FEW>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnLaunch a) {
    constexpr int kCols = D / 8, kParts = kThreads / (ROWS * kCols);
    __shared__ float o_s[kParts][ROWS][D];
    __shared__ float m_s[kParts][ROWS], l_s[kParts][ROWS];
    const int begin = FEW ? uniform(attn_shared_tile(attn_shared<D>(a), a.groups, blockIdx.x)) : int(blockIdx.x);
    if (begin < 0) return;
    const AttnShared t = attn_shared<D>(a)[begin];
    const int rows = 1 << a.log2_rows, floats = attn_partial_floats<D>(rows);
    const int c = threadIdx.x % kCols * 8, j = threadIdx.x / kCols % ROWS, part = threadIdx.x / (kCols * ROWS);
    const int row = blockIdx.y * ROWS + j, all_row = t.tile * rows + row, own = attn_token(a, all_row);
    if (t.last < 0 || attn_token(a, t.tile * rows + int(blockIdx.y) * ROWS) >= t.rows) return;
    float top = -INFINITY, sum = 0.f, o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.f;
    if (own < t.rows) {
#pragma unroll 4
        for (int w = begin + part; w <= t.last; w += kParts) {
            const float* p = a.ws + (w == begin ? t.slot : 2 * int64_t(w)) * floats;
            const float m = p[rows * D + row], l = p[rows * D + rows + row];
            const f32x4v lo = *reinterpret_cast<const f32x4v*>(p + row * D + c), hi = *reinterpret_cast<const f32x4v*>(p + row * D + c + 4);
            const float next = fmaxf(top, m), base = next == -INFINITY ? 0.f : next;
            const float f = __builtin_amdgcn_exp2f(top - base), h = __builtin_amdgcn_exp2f(m - base);
            top = next;
            sum = sum * f + l * h;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = o[i] * f + lo[i] * h, o[4 + i] = o[4 + i] * f + hi[i] * h;
        }
    }
    if (kParts > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o_s[part][j][c + i] = o[i];
        if (c == 0) {
            m_s[part][j] = top;
            l_s[part][j] = sum;
        }
        __syncthreads();
        if (part != 0) return;
        for (int x = 1; x < kParts; ++x) {
            const float next = fmaxf(top, m_s[x][j]), base = next == -INFINITY ? 0.f : next;
            const float f = __builtin_amdgcn_exp2f(top - base), h = __builtin_amdgcn_exp2f(m_s[x][j] - base);
            top = next;
            sum = sum * f + l_s[x][j] * h;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = o[i] * f + o_s[x][j][c + i] * h;
        }
    }
    if (own >= t.rows) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(o[2 * i] * inv, o[2 * i + 1] * inv);
    *reinterpret_cast<u32x4*>(a.out + (int64_t(t.first + own) * a.q_heads + t.head * a.group + all_row - own * a.group) * D + c) = w;
}

template <int D, int ELEM, int NT, int RG>
hipError_t attn_as(const AttnLaunch& a, hipStream_t stream) {
    hipLaunchKernelGGL((attn_kernel<D, ELEM, NT, RG>), dim3(a.groups), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <int D, int ELEM>
hipError_t attn_rows(const AttnLaunch& a, hipStream_t stream) {
    hipError_t e = a.log2_rows == 4   ? attn_as<D, ELEM, 1, 1>(a, stream)
                   : a.log2_rows == 5 ? attn_as<D, ELEM, 2, 1>(a, stream)
                   : a.log2_rows == 6 ? attn_as<D, ELEM, 2, 2>(a, stream)
                                      : launch_attn_wide(a, D, ELEM, stream);
    if (e != hipSuccess || !a.split) return e;
    // the more parts a tile has, the more threads share a row's: with 170 parts (3 tiles of 64 rows) a row each is
    // 8 us faster than four, with 64 parts (8 tiles of 32) 3 us, with 42 (12 tiles of 16) 2.5 us slower
    const int rows = 1 << a.log2_rows;
    if (a.groups >= 64 * a.max_tiles && rows <= 64) hipLaunchKernelGGL((attn_join_kernel<D, 1, true>), dim3(a.max_tiles, rows), dim3(kThreads), 0, stream, a);
    else if (rows <= 64) hipLaunchKernelGGL((attn_join_kernel<D, 4, false>), dim3(a.groups, rows / 4), dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((attn_join_kernel<D, 16, false>), dim3(a.groups, rows / 16), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn(const AttnLaunch& a, int head_dim, int elem_bytes, hipStream_t stream) {
    return kv_as(head_dim, elem_bytes, [&](auto d, auto e) { return attn_rows<d(), e()>(a, stream); });
}

}  // namespace tl
