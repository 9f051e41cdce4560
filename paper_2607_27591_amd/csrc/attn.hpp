// Attention of new tokens over the 4-bit paged cache: the kernels, and their variant by shape.
// Compiled once per dtype (attn_f16.hip, attn_bf16.hip).
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace prox {

constexpr int kAttnWaves = 4;
constexpr int kAttnWhole = 16;         // ... that are never split
constexpr float kAttnNone = -3.0e38f;  // running maximum before the first score (finite: no inf - inf)
// The running maximum m of a row's scores (log2) is raised only when a score exceeds it by more
// than this: weights stay below 2^8, and sums and outputs are rescaled a few times in all.
constexpr float kAttnSlack = 8.0f;

// Waves per SIMD that a variant is compiled for: as many as leave none of its registers in scratch memory, or up to
// 3 of them (head_dim 128 with 4 groups, 256 with 2 or 4, and two tiles of 128 in fp16; 8 or 16 bytes a lane).
constexpr int attn_waves(int D, int NG, int QT, int E) {
    if (E < 4) return D == 64 ? (NG == 1 ? 6 : 5) : D == 128 ? 4 : NG < 8 ? 3 : 2;
    if (QT == 1) return D == 64 ? 5 : D == 128 ? (NG == 4 ? 3 : 4) : (NG == 2 ? 3 : 2);
    return D == 64 ? (NG == 1 ? 3 : 2) : D == 128 ? (NG == 1 ? 3 : 2) : 1;
}

// A lane's W words of a half block of keys or a block of values (kv_k_word, kv_v_word).
template <int W>
__device__ __forceinline__ void load_words(uint32_t (&out)[W], const uint8_t *p, int lane) {
    if constexpr (W == 2) {
        const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(p) + lane);
        out[0] = v[0];
        out[1] = v[1];
    } else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p) + 64 * i + lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[4 * i + e] = v[e];
        }
    }
}

// Scales of a lane's E tokens of each half block (kv_slot): word e holds token e of both.
template <int E>
using Scales = uint32_t __attribute__((ext_vector_type(E)));
template <int E>
__device__ __forceinline__ Scales<E> load_scales(const uint8_t *row, int token0) {
    return *reinterpret_cast<const Scales<E> *>(row + 4 * token0);
}
__device__ __forceinline__ float slot_scale(uint32_t w, int j) { return f16_bits_to_float(j ? w >> 16 : w & 0xFFFFu); }

// Lanes of a row of 16 that are 4 K apart.
template <int K>
__device__ __forceinline__ uint32_t from_bank(uint32_t v) {   // lane i gets that of lane (i + 4 K) % 16
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + 16 - 4 * K, 0xF, 0xF, false);
}
template <int K, int BANKS>   // ... in the banks of a mask, old elsewhere
__device__ __forceinline__ uint32_t take_bank(uint32_t old, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, K == 0 ? 0xE4 : 0x120 + 16 - 4 * K, 0xF, BANKS, false);
}
template <int K>
__device__ __forceinline__ float from_bank(float v) { return __uint_as_float(from_bank<K>(__float_as_uint(v))); }
// Value e of the E that a lane takes of v: lanes 4 E i .. 4 E i + 4 E - 1 of a row of 16 take
// v[E i ..].
template <int E>
__device__ __forceinline__ float own_of(const v4f &v, int e) {
    int r = __float_as_int(v[e]);
    if constexpr (E == 1) r = __builtin_amdgcn_update_dpp(r, __float_as_int(v[1]), 0xE4, 0xF, 0x2, false);
    if constexpr (E < 4) r = __builtin_amdgcn_update_dpp(r, __float_as_int(v[2 + e]), 0xE4, 0xF, E == 1 ? 0x4 : 0xC, false);
    if constexpr (E == 1) r = __builtin_amdgcn_update_dpp(r, __float_as_int(v[3]), 0xE4, 0xF, 0x8, false);
    return __int_as_float(r);
}

// a * s with s an fp16 scale in place: as a fused add of 0 it is one v_fma_mix_f32, without a
// conversion (a and s nonnegative, or the result added up: the sign of a zero is no matter).
__device__ __forceinline__ float times(float a, float s) { return fmaf(a, s, 0.0f); }

typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {   // rounded to nearest even
    const bf16v2 v = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, v);
}
// a - lo(w) and a - hi(w), what a rounding to bf16 left over (exact): one dot product each,
// with (-1, 0) and (0, -1).  The constants stay in registers: as literals of the
// instruction their products came out as 0.
struct Bf16Left {
    uint32_t lo = 0x0000BF80u, hi = 0xBF800000u;
    __device__ __forceinline__ Bf16Left() { asm("" : "+v"(lo), "+v"(hi)); }
    __device__ __forceinline__ float minus_lo(float a, uint32_t w) const { return dot2<kBF16>(w, lo, a); }
    __device__ __forceinline__ float minus_hi(float a, uint32_t w) const { return dot2<kBF16>(w, hi, a); }
};

__device__ __forceinline__ float max_swap16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_swap32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// First row of the partial results of a tile: head_dim sums a row, then (maximum, sum of
// weights) of all rows.
__device__ __forceinline__ size_t attn_part_row(const AttnArgs &A, int split, int s, int head, int tile) {
    return ((((size_t)split * A.s.n_seq + s) * A.c.heads + head) * A.tiles + tile) * A.part_rows;
}

// What a wave keeps of QT tiles of 16 query rows (row l % 16 in lane l) during its pass:
// the unnormalised output and the offset's part of it, maximum m of scale times the score,
// the lane's part of the sum of weights l; a score above top raises m.
// E < 4: up to 4 E rows, standing 4 / E times side by side (row l % (4 E) in lane l), so that a lane
// has E of its four tokens of a half block to weigh.  In the second product lanes 0 .. 4 E - 1 of
// 16 hold the weights' first terms, the next 4 E the second (one product for both), the others
// nothing that counts.
// The arithmetic of a softmax on 16 rows would bound a few rows: 16 x 8192 tokens, head_dim 128,
// 4 rows 38.3 to 31.1 us, 8 rows 39.3 to 34.2; 131072 tokens, 4 rows 38.8 to 32.8 (group 64).
template <int D, int NG, int QT, int E>
struct AttnRows {
    static_assert(E == 4 || QT == 1, "one tile");
    static constexpr int VT = D / 16, VPG = VT / NG;
    static __device__ __forceinline__ int row_of(int lane) { return lane % (4 * E); }
    static __device__ __forceinline__ int token0(int lane) { return lane / 16 * 4 + lane % 16 / (4 * E) * E; }
    v4f acc[QT][VT], off[QT][NG];
    float m[QT], l[QT], top[QT];
    int lo[QT], hi[QT];                    // positions that the row sees
    int hi_min, hi_max, lo_min, lo_max;    // over the tiles' rows

    // Rows r0 .. r1 of the sequence and kv head (the last one again past them).
    __device__ __forceinline__ void start(const AttnArgs &A, const SeqTokens &sq, int r0, int r1) {
        const int i0 = r0 / A.ratio, i1 = r1 / A.ratio, row = row_of(lane_id());
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            hi[u] = sq.pos0 + min(r0 + 16 * u + row, r1) / A.ratio;
            lo[u] = attn_first(hi[u], A.window);
            m[u] = top[u] = kAttnNone;
            l[u] = 0.0f;
#pragma unroll
            for (int i = 0; i < VT; ++i) acc[u][i] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int g = 0; g < NG; ++g) off[u][g] = v4f{0, 0, 0, 0};
        }
        hi_min = sq.pos0 + i0;
        hi_max = sq.pos0 + i1;
        lo_min = attn_first(hi_min, A.window);
        lo_max = attn_first(hi_max, A.window);
    }
    // Whether some row does not see all of the block at p0.
    __device__ __forceinline__ bool edge(int p0) const { return p0 + kKvBlock - 1 > hi_min || p0 < lo_max; }

    // Scores of the block at p0 to weights, the sums raised to a new maximum where it takes one.
    __device__ __forceinline__ void weigh(float (&sc)[QT][2][E], int p0, bool edge, float scale, float slack) {
        const int t0 = token0(lane_id());
        uint32_t seen[QT];   // bit 4 j + e: the row sees the token
        bool up = false;
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            float mx = kAttnNone;
            if (edge) {
                seen[u] = 0;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int p = p0 + 16 * j + t0 + e;
                        const bool ok = p <= hi[u] && p >= lo[u];
                        seen[u] |= (uint32_t)ok << (4 * j + e);
                        sc[u][j][e] = ok ? sc[u][j][e] : kAttnNone;   // whatever stands there
                    }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) mx = fmaxf(mx, sc[u][j][e]);
            up |= mx > top[u];
        }
        if (__any(up)) {
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                float mx = kAttnNone;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < E; ++e) mx = fmaxf(mx, sc[u][j][e]);
                mx = max_swap32(max_swap16(mx));
                if constexpr (E == 1) mx = fmaxf(mx, from_bank<1>(mx));
                if constexpr (E < 4) mx = fmaxf(mx, from_bank<2>(mx));
                const float m2 = fmaxf(m[u], mx * scale), f = __builtin_amdgcn_exp2f(m[u] - m2);
                top[u] = fmaxf(top[u], mx + slack);
                m[u] = m2;
                l[u] *= f;
#pragma unroll
                for (int i = 0; i < VT; ++i) acc[u][i] *= f;
#pragma unroll
                for (int g = 0; g < NG; ++g) off[u][g] *= f;
            }
        }
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float p = __builtin_amdgcn_exp2f(fmaf(sc[u][j][e], scale, -m[u]));
                    if (edge) p = (seen[u] >> (4 * j + e)) & 1 ? p : 0.0f;
                    sc[u][j][e] = p;
                    l[u] += p;
                }
    }

    // Weights times values: value(i) is the operand of channels 16 i .. 16 i + 15, vs their scales.
    template <typename Value>
    __device__ __forceinline__ void add(const float (&p)[QT][2][E], const Scales<E> (&vs)[NG], int p0, bool edge,
                                        const Bf16Left &left, Value value) {
        const int t0 = token0(lane_id());
        const uint4 minus = Int4Oct<kBF16>::minus();
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            uint4 ph[QT], pl[QT];
            float f[2][E];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    f[j][e] = slot_scale(vs[g][e], j);
                    if (edge) {   // tokens that no row sees may hold anything
                        const int q = p0 + 16 * j + t0 + e;
                        f[j][e] = q <= hi_max && q >= lo_min ? f[j][e] : 0.0f;
                    }
                }
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                uint32_t wh[4], wl[4];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float a = times(p[u][0][e], f[0][e]), c = times(p[u][1][e], f[1][e]);
                    wh[e] = pack_bf16(a, c);
                    wl[e] = pack_bf16(left.minus_lo(a, wh[e]), left.minus_hi(c, wh[e]));
                }
                if constexpr (E == 1) {   // lanes 0 .. 3 the first terms of all four tokens, 4 .. 7 the second
                    const uint32_t a = wh[0], c = wl[0];
                    wh[0] = take_bank<3, 0x2>(a, c);
                    wh[1] = take_bank<0, 0x2>(from_bank<1>(a), c);
                    wh[2] = take_bank<1, 0x2>(from_bank<2>(a), c);
                    wh[3] = take_bank<2, 0x2>(from_bank<3>(a), c);
                } else if constexpr (E == 2) {   // lanes 0 .. 7, 8 .. 15
                    const uint32_t a0 = wh[0], a1 = wh[1], c0 = wl[0], c1 = wl[1];
                    wh[0] = take_bank<2, 0xC>(a0, c0);
                    wh[1] = take_bank<2, 0xC>(a1, c1);
                    wh[2] = take_bank<0, 0xC>(from_bank<2>(a0), c0);
                    wh[3] = take_bank<0, 0xC>(from_bank<2>(a1), c1);
                }
                ph[u] = make_uint4(wh[0], wh[1], wh[2], wh[3]);
                if constexpr (E == 4) pl[u] = make_uint4(wl[0], wl[1], wl[2], wl[3]);
                off[u][g] = mfma32<kBF16>(minus, ph[u], off[u][g]);
                if constexpr (E == 4) off[u][g] = mfma32<kBF16>(minus, pl[u], off[u][g]);
            }
#pragma unroll
            for (int i = g * VPG; i < (g + 1) * VPG; ++i) {
                const uint4 a = value(i);
#pragma unroll
                for (int u = 0; u < QT; ++u) acc[u][i] = mfma32<kBF16>(a, ph[u], acc[u][i]);
#pragma unroll
                for (int u = 0; u < QT; ++u)
                    if constexpr (E == 4) acc[u][i] = mfma32<kBF16>(a, pl[u], acc[u][i]);
            }
        }
    }

    // The offset's part comes off, before it can outgrow the sums.
    __device__ __forceinline__ void flush() {
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
#pragma unroll
                for (int i = g * VPG; i < (g + 1) * VPG; ++i) acc[u][i] += off[u][g];
                off[u][g] = v4f{0, 0, 0, 0};
            }
    }
};

// Scores of two half blocks of 16 tokens: sums of a group, base its start (the offset's part), its scales applied.
template <int NG, int QT, int E>
__device__ __forceinline__ void add_scores(float (&sc)[QT][2][E], const v4f (&d)[QT][2], const Scales<E> &ks, int g) {
#pragma unroll
    for (int u = 0; u < QT; ++u)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float f = slot_scale(ks[e], j), s = own_of<E>(d[u][j], e);
                sc[u][j][e] = g == 0 ? times(s, f) : fmaf(s, f, sc[u][j][e]);
            }
}

// Query row r of a sequence and kv head as an operand: word w of the lane.
template <int D>
__device__ __forceinline__ uint4 query_word(const AttnArgs &A, const SeqTokens &sq, int head, int r, int w) {
    const int i = r / A.ratio;
    const uint16_t *p = A.q + (size_t)(sq.t0 + i) * A.ldq + (size_t)(head * A.ratio + r - i * A.ratio) * D + 8 * (lane_id() / 16);
    const uint4 v = *reinterpret_cast<const uint4 *>(p + 32 * w);
    return make_uint4(v.x ^ A.q_sign, v.y ^ A.q_sign, v.z ^ A.q_sign, v.w ^ A.q_sign);
}

// Blocks of a sequence and kv head in the cache.
template <int D, int NG>
struct AttnBlocks {
    const int32_t *table;
    int per, last;   // blocks of a page, the last block
    __device__ __forceinline__ AttnBlocks(const AttnArgs &A, int s, int end)
        : table(A.s.table + (size_t)s * A.s.max_pages), per(A.c.page_size / kKvBlock), last(end - 1) {}
    __device__ __forceinline__ int page_of(const AttnArgs &A, int b) const { return A.page_shift >= 0 ? b >> A.page_shift : b / per; }
    __device__ __forceinline__ int page_id(const AttnArgs &A, int b) const { return table[page_of(A, min(b, last))]; }
    // Record of block b on page id; where the page lies outside the cache, or past the end, ok is
    // false and the cache's first record stands in (loaded, not used).
    __device__ __forceinline__ const uint8_t *record(const AttnArgs &A, int head, int b, int end, int id, bool &ok) const {
        const int pid = __builtin_amdgcn_readfirstlane(id);
        ok = b < end && pid >= 0 && pid < A.c.n_pages;
        const size_t at = (size_t)pid * A.c.page_bytes + ((size_t)head * per + (b - page_of(A, b) * per)) * KvLayout(D, D / NG).record;
        return A.c.blob + (ok ? at : 0);
    }
};

// One pass over the cache with the running maximum and sum of the softmax.  A wave takes
// blocks of 32 tokens; with K the codes of 16 tokens and Q 16 query rows of one kv head,
//   S^T = K Q^T             codes exact with an offset (base starts each group's sum), scales
//                           on the fp32 sums: lane l gets tokens 4 (l / 16) + e of row l % 16
//   P   = 2^(c S - m)       fp32; l += P
//   O^T += V^T (P sv)^T     P times the values' scale, rounded to two bf16 terms (2^-17), is
//                           the second product's operand as it stands, no lane exchange; the
//                           codes' offset comes off with a product of its own (off), every 8
//                           blocks.
// Two terms, as one bf16 term would add as much error as the rounding of a bf16 output, and
// eight times that of an fp16 one; bf16 and not fp16, as P sv spans any range.
// Bound by HBM for single tokens (a record is read once and contiguous; the next one's loads
// are in flight): 131072 tokens of 8 kv heads, 32 query heads, 33.4 us with the join (143 MB, 4.3
// TB/s), the VALU busy for 70 % of this kernel's cycles.  By VALU issue for many rows, for which QT
// tiles of 16 rows share the codes: 2 x 512 queries over 4096 tokens, 32 heads, 134 us in a stream of
// calls (480 TFLOP/s), 153 by itself at a lower clock; VALU 75 % and MFMA 34 % of the cycles.
// The four waves' results are joined through LDS, those of several workgroups of a long
// cache by attn_join_kernel.
template <int DT, int D, int NG, int QT, int E>
__global__ __launch_bounds__(64 * kAttnWaves, attn_waves(D, NG, QT, E)) void attn_kernel(AttnArgs A) {
    constexpr int R = 16 * QT, KW = D / 32, VT = D / 16, SPG = KW / NG;
    constexpr int TC = VT < 8 ? VT : 8;   // channel tiles joined at a time
    constexpr KvLayout L(D, D / NG);
    // Queries and base as operands during the pass (read again for each block, which leaves
    // their registers to more waves), the waves' results afterwards.
    constexpr int QB = QT * (KW + NG), OB = kAttnWaves * TC;
    __shared__ v4f smem[QB > OB ? QB : OB][kWave];
    v4f (&o_sh)[QB > OB ? QB : OB][kWave] = smem;
    __shared__ float m_sh[kAttnWaves][16], l_sh[kAttnWaves][16];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int lane = lane_id(), h = lane / 16, col = lane % 16;
    int id = blockIdx.x;
    const int split = id % A.splits;
    id /= A.splits;
    const int tile = id % A.tiles;
    id /= A.tiles;
    const int head = id % A.c.heads, s = id / A.c.heads;
    const SeqTokens sq = seq_tokens(A.s, s);
    const int rows = sq.n * A.ratio, r0 = tile * R;
    if (r0 >= rows) return;
    const AttnSpan sp = attn_span(sq, A.ratio, A.window, A.splits, r0, min(r0 + R, rows) - 1);
    if (split > 0 && split >= sp.eff) return;
    const int b_end = min(sp.b0 + (split + 1) * sp.per, sp.b1);

    uint32_t xk[2][KW], xv[VT];
    using Rows = AttnRows<D, NG, QT, E>;
    Scales<E> xks[NG], xvs[NG];
    const int t0 = Rows::token0(lane);
    const AttnBlocks<D, NG> blocks(A, s, sp.b1);
    auto load_k = [&](const uint8_t *rec) {
        load_words(xk[0], rec, lane);
        load_words(xk[1], rec + 64 * KW * 4, lane);
#pragma unroll
        for (int g = 0; g < NG; ++g) xks[g] = load_scales<E>(rec + L.k_scales + g * 64, t0);
    };
    auto load_v = [&](const uint8_t *rec) {
        load_words(xv, rec + L.v_codes, lane);
#pragma unroll
        for (int g = 0; g < NG; ++g) xvs[g] = load_scales<E>(rec + L.v_scales + g * 64, t0);
    };
    // Keys of the next block are asked for once this block's are used, values likewise; the
    // page of the one after it.
    const int first = sp.b0 + split * sp.per + wave;
    int next_id = 0;
    bool next_ok = false;
    const uint8_t *next = A.c.blob;
    if (first < b_end) {
        next = blocks.record(A, head, first, b_end, blocks.page_id(A, first), next_ok);
        next_id = blocks.page_id(A, first + kAttnWaves);
        load_k(next);
        load_v(next);
    }
    const int r_last = min(r0 + R, rows) - 1;
    const Int4Oct<DT> kop;
    const Int4Oct<kBF16> vop;
    const Bf16Left left;
#pragma unroll
    for (int u = 0; u < QT; ++u)
        for (int w = wave; w < KW; w += kAttnWaves)
            smem[u * KW + w][lane] = __builtin_bit_cast(v4f, query_word<D>(A, sq, head, min(r0 + 16 * u + Rows::row_of(lane), r_last), w));
    __syncthreads();
    for (int ug = wave; ug < QT * NG; ug += kAttnWaves) {
        v4f d{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < SPG; ++w)
            d = mfma32<DT>(Int4Oct<DT>::minus(), __builtin_bit_cast(uint4, smem[ug / NG * KW + ug % NG * SPG + w][lane]), d);
        smem[QT * KW + ug][lane] = d;
    }
    __syncthreads();
    Rows X;
    X.start(A, sq, r0, r_last);
    const float slack = kAttnSlack / A.scale;
    int done = 0;
    for (int b = first; b < b_end; b += kAttnWaves) {
        const bool ok = next_ok;
        next = blocks.record(A, head, b + kAttnWaves, b_end, next_id, next_ok);
        next_id = blocks.page_id(A, b + 2 * kAttnWaves);
        float sc[QT][2][E];
        if (ok) {
            asm volatile("" ::: "memory");   // the queries stay in LDS
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                v4f d[QT][2];
#pragma unroll
                for (int u = 0; u < QT; ++u) d[u][0] = d[u][1] = smem[QT * KW + u * NG + g][lane];
#pragma unroll
                for (int w = g * SPG; w < (g + 1) * SPG; ++w) {
                    uint4 q[QT];
#pragma unroll
                    for (int u = 0; u < QT; ++u) q[u] = __builtin_bit_cast(uint4, smem[u * KW + w][lane]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint4 a = kop(xk[j][w]);
#pragma unroll
                        for (int u = 0; u < QT; ++u) d[u][j] = mfma32<DT>(a, q[u], d[u][j]);
                    }
                }
                add_scores<NG>(sc, d, xks[g], g);
            }
        }
        load_k(next);
        if (ok) {
            const bool edge = X.edge(b * kKvBlock);
            X.weigh(sc, b * kKvBlock, edge, A.scale, slack);
            X.add(sc, xvs, b * kKvBlock, edge, left, [&](int i) { return vop(xv[i]); });
            if ((++done & 7) == 0) X.flush();
        }
        load_v(next);
    }
    X.flush();

    // The waves' results: o = sum_w 2^(m_w - m) o_w, l alike, in a fixed order.
    float *part_o = reinterpret_cast<float *>(A.ws);
    float2 *part_ml = reinterpret_cast<float2 *>(part_o + (size_t)kAttnPartRows * D);
    const size_t prow = attn_part_row(A, split, s, head, tile);
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        float lw = add_swap32(add_swap16(X.l[u]));
        if constexpr (E == 1) lw += from_bank<1>(lw);
        if constexpr (E < 4) lw += from_bank<2>(lw);
        if (u > 0) __syncthreads();
        if (h == 0) {
            m_sh[wave][col] = X.m[u];
            l_sh[wave][col] = lw;
        }
        __syncthreads();
        float mm = m_sh[0][col], ll = 0.0f;
#pragma unroll
        for (int w = 1; w < kAttnWaves; ++w) mm = fmaxf(mm, m_sh[w][col]);
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) ll = fmaf(l_sh[w][col], __builtin_amdgcn_exp2f(m_sh[w][col] - mm), ll);
        const float f = __builtin_amdgcn_exp2f(X.m[u] - mm);
        const int r = r0 + 16 * u + col, i = r / A.ratio;
        uint16_t *dst = A.out + (size_t)(sq.t0 + i) * A.ldo + (size_t)(head * A.ratio + r - i * A.ratio) * D + 4 * h;
        const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
        if (sp.eff > 1 && wave == 0 && h == 0 && r < rows) part_ml[prow + 16 * u + col] = make_float2(mm, ll);
#pragma unroll
        for (int c = 0; c < VT; c += TC) {
            if (c > 0) __syncthreads();
#pragma unroll
            for (int i2 = 0; i2 < TC; ++i2) o_sh[wave * TC + i2][lane] = X.acc[u][c + i2] * f;
            __syncthreads();
            for (int i2 = wave; i2 < TC; i2 += kAttnWaves) {
                v4f o = o_sh[i2][lane];
#pragma unroll
                for (int w = 1; w < kAttnWaves; ++w) o += o_sh[w * TC + i2][lane];
                if constexpr (E < 4) {   // the two terms' products
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] += from_bank<E>(o[e]);
                }
                if (r >= rows) continue;
                if (sp.eff > 1) {
                    *reinterpret_cast<v4f *>(part_o + (prow + 16 * u + col) * D + 16 * (c + i2) + 4 * h) = o;
                } else {
                    const uint32_t w0 = float_to_half<DT>(o[0] * inv) | (uint32_t)float_to_half<DT>(o[1] * inv) << 16;
                    const uint32_t w1 = float_to_half<DT>(o[2] * inv) | (uint32_t)float_to_half<DT>(o[3] * inv) << 16;
                    *reinterpret_cast<uint2 *>(dst + 16 * (c + i2)) = make_uint2(w0, w1);
                }
            }
        }
    }
}

// The splits' results of one query row per workgroup, in a fixed order: D / 4 threads hold the
// channels, the groups of them take the splits in turn.  Bound by its launch and a chain of loads
// (length, maxima and sums): 3.4 us for 32 rows of 16 splits, 5.2 for 32 rows of 128.
constexpr int kAttnMaxSplits = 1024;
template <int DT, int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs A, int R) {
    constexpr int CT = D / 4, P = 256 / CT, PER = kAttnMaxSplits / 256;
    __shared__ float w_sh[kAttnMaxSplits], red[8];
    __shared__ v4f o_sh[P][CT];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
    const int row = blockIdx.x;   // (sequence, new token, query head)
    const int hq = row % A.q_heads, s = row / A.q_heads / A.s.max_new, i = row / A.q_heads % A.s.max_new;
    const SeqTokens sq = seq_tokens(A.s, s);
    if (i >= sq.n) return;
    const int head = hq / A.ratio, r = i * A.ratio + hq % A.ratio, tile = r / R;
    const AttnSpan sp = attn_span(sq, A.ratio, A.window, A.splits, tile * R, min((tile + 1) * R, sq.n * A.ratio) - 1);
    if (sp.eff <= 1) return;
    const float *part_o = reinterpret_cast<const float *>(A.ws);
    const float2 *part_ml = reinterpret_cast<const float2 *>(part_o + (size_t)kAttnPartRows * D);
    const size_t stride = attn_part_row(A, 1, 0, 0, 0), at = attn_part_row(A, 0, s, head, tile) + r % R;
    const int p = tid / CT, c = tid % CT;
    const float *src = part_o + at * D + 4 * c;
    constexpr int U = 4;   // 2 or 8: 8192 tokens 11.7 or 11.4 us in all, instead of 11.2
    v4f first[U];          // asked for together with the maxima
#pragma unroll
    for (int j = 0; j < U; ++j) first[j] = *reinterpret_cast<const v4f *>(src + (size_t)min(p + P * j, sp.eff - 1) * stride * D);
    float2 ml[PER];
    float mm = kAttnNone;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int k = tid + 256 * j;
        ml[j] = k < sp.eff ? part_ml[at + k * stride] : make_float2(kAttnNone, 0.0f);
        mm = fmaxf(mm, ml[j].x);
    }
    for (int x = 1; x < kWave; x <<= 1) mm = fmaxf(mm, __shfl_xor(mm, x));
    if (lane == 0) red[wave] = mm;
    __syncthreads();
    mm = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float ll = 0.0f;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const float f = __builtin_amdgcn_exp2f(ml[j].x - mm);
        if (tid + 256 * j < sp.eff) w_sh[tid + 256 * j] = f;
        ll = fmaf(ml[j].y, f, ll);
    }
    ll = wave_sum(ll);
    if (lane == 0) red[4 + wave] = ll;
    __syncthreads();
    ll = (red[4] + red[5]) + (red[6] + red[7]);
    v4f o{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < U; ++j)
        if (p + P * j < sp.eff) o += w_sh[p + P * j] * first[j];
#pragma unroll 4
    for (int k = p + P * U; k < sp.eff; k += P) o += w_sh[k] * *reinterpret_cast<const v4f *>(src + k * stride * D);
    o_sh[p][c] = o;
    __syncthreads();
    if (p > 0) return;
#pragma unroll
    for (int j = 1; j < P; ++j) o += o_sh[j][c];
    const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
    const uint32_t w0 = float_to_half<DT>(o[0] * inv) | (uint32_t)float_to_half<DT>(o[1] * inv) << 16;
    const uint32_t w1 = float_to_half<DT>(o[2] * inv) | (uint32_t)float_to_half<DT>(o[3] * inv) << 16;
    *reinterpret_cast<uint2 *>(A.out + (size_t)(sq.t0 + i) * A.ldo + (size_t)hq * D + 4 * c) = make_uint2(w0, w1);
}

// Blocks that a tile of R rows sees at most.
inline int attn_blocks(const AttnArgs &a, int R) {
    const int all = (a.s.max_kv + kKvBlock - 1) / kKvBlock;
    if (a.window == 0) return all;
    const long long seen = ((long long)a.window + R / a.ratio + 2 * kKvBlock) / kKvBlock;
    return seen < all ? (int)seen : all;
}

template <int DT, int D, int NG, int QT, int E>
hipError_t run_attn(AttnArgs &a, hipStream_t s) {
    constexpr int R = 16 * QT;
    a.tiles = (int)(((long long)a.s.max_new * a.ratio + R - 1) / R);
    // Splits: at most as many workgroups as the chip holds at a time, one wave of each on a SIMD, no
    // shorter than kAttnMinBlocks, as far as the partial results fit their area.  All W workgroups
    // that a CU holds pay where each has 4 W blocks (its start and its join take that long), two
    // where a CU has 15 blocks or more, else one (three is never taken, nor measured); in us, four a CU and what is taken:
    //   8192 tokens 11.5, 11.0;  16384 15.2, 13.2;  32768 17.8, 16.3;  8 x 2000 (15 blocks) 13.9, 12.7
    // and with one, two, four, eight a CU:  32 x 8192, ragged 70, 45.7, 36.0, 39.5;  131072 tokens
    // 43.7, 33.3, 33.7, 39.3.  Up to kAttnWhole blocks are left whole: joining takes longer than the
    // blocks (one launch more).
    const long long base = (long long)a.s.n_seq * a.c.heads * a.tiles;
    const int blocks = attn_blocks(a, R);
    const long long work = blocks * base / 256;   // blocks per CU
    constexpr int W = attn_waves(D, NG, QT, E);
    const int per_cu = work >= 4 * W * W ? W : work >= 15 && W > 2 ? 2 : 1;
    long long n = blocks > kAttnWhole ? 256 * per_cu / base : 1;
    if (n > kAttnMaxSplits) n = kAttnMaxSplits;
    a.part_rows = (int)((long long)a.s.max_new * a.ratio < R ? a.s.max_new * a.ratio : R);
    if (n > kAttnPartRows / a.part_rows / base) n = kAttnPartRows / a.part_rows / base;
    if (n > (blocks + kAttnMinBlocks - 1) / kAttnMinBlocks) n = (blocks + kAttnMinBlocks - 1) / kAttnMinBlocks;
    a.splits = n < 1 ? 1 : (int)n;
    attn_kernel<DT, D, NG, QT, E><<<(unsigned)(base * a.splits), 64 * kAttnWaves, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const long long rows = (long long)a.s.n_seq * a.s.max_new * a.q_heads;
    attn_join_kernel<DT, D><<<(unsigned)rows, 256, 0, s>>>(a, R);
    return hipGetLastError();
}

// Up to 4 and up to 8 rows of a sequence and kv head share the softmax's lanes (AttnRows).  Up to
// 16 rows one tile; more, two tiles a workgroup share the codes (2 x 512 queries over 4096 tokens,
// group 128: 135 us against 160), but at head_dim 256, where their sums leave one wave a SIMD (118
// us against 180), and not four (193 us).  One tile too where a CU has up to 32 of a tile's blocks,
// as more workgroups are ready sooner than fewer that do less in all; in us, one and two:
//   32 heads, 64 queries, 500 tokens 9.9, 13.8;  5 queries, 2000 10.4, 11.7;  32768 24.0, 23.3
//   64 queries, 2000 20.1, 20.9;  8192 37.9, 35.4;  256 queries, 2000 49.3, 47.0
template <int DT, int D, int NG>
hipError_t launch_attn_rows(AttnArgs &a, hipStream_t s) {
    const long long rows = (long long)a.s.max_new * a.ratio;
    if constexpr (D < 256) {
        const long long work = a.s.n_seq * ((rows + 15) / 16) * a.c.heads * attn_blocks(a, 16) / 256;   // blocks per CU
        if (rows > 16 && work > 32) return run_attn<DT, D, NG, 2, 4>(a, s);
    }
    if (rows <= 4) return run_attn<DT, D, NG, 1, 1>(a, s);
    if (rows <= 8) return run_attn<DT, D, NG, 1, 2>(a, s);
    return run_attn<DT, D, NG, 1, 4>(a, s);
}

template <int DT>
hipError_t launch_attn_dt(AttnArgs &a, hipStream_t s) {
    const int ng = a.c.dim / a.c.group;
    if (a.c.dim == 64) return ng == 1 ? launch_attn_rows<DT, 64, 1>(a, s) : launch_attn_rows<DT, 64, 2>(a, s);
    if (a.c.dim == 128)
        return ng == 1 ? launch_attn_rows<DT, 128, 1>(a, s)
               : ng == 2 ? launch_attn_rows<DT, 128, 2>(a, s) : launch_attn_rows<DT, 128, 4>(a, s);
    return ng == 2 ? launch_attn_rows<DT, 256, 2>(a, s)
           : ng == 4 ? launch_attn_rows<DT, 256, 4>(a, s) : launch_attn_rows<DT, 256, 8>(a, s);
}

}  // namespace prox
