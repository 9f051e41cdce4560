// Projections on INT4 weights with group scales, y = x W^T (+ bias) for up to 64 rows: the
// kernel, and its variant by shape.  Compiled once per dtype (linear_f16.hip,
// linear_bf16.hip).
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace prox {

// y^T = W x^T as MFMAs: 16 outputs by 16 batch rows by 32 inputs each.  The codes enter as
// exact 16-bit values with an offset, the offset's part (Int4Oct::minus times x, one more
// product per 32 inputs for all NT tiles) starts each group's sum, and the scale is applied
// to the group's fp32 sum: nothing but fp32 sums is rounded before y.  The codes are read once: bound by
// HBM for few rows (28672 x 8192, one row 24.6 us, 4.9 TB/s; 8192 x 8192, 16 rows 12.1 us, 2.9 TB/s
// beside x and unpacking), by VALU, LDS and MFMA issue for many (28672 x 8192, 64 rows 51 us in a
// stream of calls, 590 TFLOP/s, 56 by itself at a lower clock; each of them a third of the cycles).  A
// workgroup takes WN * NT tiles of 16 outputs over all inputs, so that no partial sums leave it; its 8 waves take NT tiles each of 8 / WN blocks of 128 inputs at a time.
// They are added in a fixed order through LDS.
// x goes through LDS from whole rows of 256 bytes to operand order (a load of operands
// straight from the rows touches 64 lines at a time and takes four times as long), where the
// WN waves of a block share it: x is read from the L2 once per workgroup, for which WN * NT
// grows with the batch.
// GPB: groups per block of 128 (4, 2, or 1 for groups of 128 and more).
constexpr int kLinearWaves = 8;

// Four waves of a block that stage a row tile each work out its offset's part for all of them
// (28672 x 8192, 64 rows: 55.0 to 51.0 us; two waves with two tiles each: 14336 x 4096, 20.9 to
// 21.3).
template <int RG, int WN>
constexpr bool kLinearShare = WN == 4 && RG / WN % 4 == 0;

template <int NT, int RG, int WN, int GPB>
constexpr size_t linear_lds() {
    constexpr int MT = (RG + 3) / 4, WK = kLinearWaves / WN, TILES = NT * MT, RT = TILES < 8 ? TILES : 8;
    constexpr size_t base = kLinearShare<RG, WN> ? GPB * 256 : 0;
    constexpr size_t stage = (WN == 1 ? 1 : 2) * (size_t)WK * MT * (4096 + base), red = (size_t)kLinearWaves * RT * 1024;
    return stage > red ? stage : red;
}

// RG: groups of four batch rows.
template <int DT, int NT, int RG, int WN, int GPB, bool TAIL>
__global__ __launch_bounds__(64 * kLinearWaves) void linear_kernel(LinearArgs A) {
    constexpr int MT = (RG + 3) / 4, WK = kLinearWaves / WN, TILES = NT * MT, RT = TILES < 8 ? TILES : 8;
    static_assert(RG % WN == 0, "the waves of a block load the same number of rows");
    // Steps that loads run ahead (4: 28672 x 8192, one row 24.6 to 30.4 us).
    constexpr int DEPTH = 2;
    constexpr int XL = RG / WN;                     // loads of 4 rows of a block by each of its waves
    // Operands of x read one product ahead (8192 x 8192, 64 rows: 22.0 to 21.0 us; 28672 x 8192
    // 51.0 to 50.4), but with 8 loads of x in flight, which leave it no registers (14336 x 4096,
    // 64 rows: 21.2 to 23.5).
    constexpr int XB = WN > 1 && XL <= 4 ? 2 : 1;
    constexpr int STAGE = WK * MT * 256;            // 16-byte chunks of x: [slot][row tile][chunk of the row][row ^ chunk]
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr bool SHARE = kLinearShare<RG, WN>;
    u32x4 *xs = reinterpret_cast<u32x4 *>(smem);
    v4f *bs = reinterpret_cast<v4f *>(smem + 2 * (size_t)STAGE * 16);   // SHARE: [buffer][slot][row tile][group][row]
    const LinearLayout L(A.n, A.k, A.group);
    const int n = A.n, k = A.k, row0 = blockIdx.y * 4 * RG, batch = min(A.batch - row0, 4 * RG);   // rows of this workgroup
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int lane = lane_id(), h = lane / 16, col = lane % 16;
    const int slot = wave / WN, nw = wave % WN;
    const int tile0 = (blockIdx.x * WN + nw) * NT;
    const Int4Oct<DT> oct;
    const uint4 minus = Int4Oct<DT>::minus();
    // Load l of this wave: rows 4 (nw XL + l) + h, chunk col of 8 inputs; past the batch its
    // last row again (their columns are not stored).
    const uint16_t *xr[XL];
#pragma unroll
    for (int l = 0; l < XL; ++l) xr[l] = A.x + (size_t)(row0 + min(4 * (nw * XL + l) + h, batch - 1)) * A.ldx + 8 * col;
    const uint8_t *codes[NT];
    const uint16_t *scales[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {   // past the last tile: the last again, not stored
        const int tile = min(tile0 + t, L.tiles - 1);
        codes[t] = A.blob + (size_t)tile * L.blocks * 1024 + lane * 16;
        scales[t] = reinterpret_cast<const uint16_t *>(A.blob + L.scales) + tile * L.tile_scales() + 4 * GPB * h;
    }
    v4f acc[NT][MT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = v4f{0, 0, 0, 0};
    u32x4 c[DEPTH][NT], xv[DEPTH][XL];   // of step j in set j % DEPTH, DEPTH steps ahead
    u32x2 sc[DEPTH][NT][GPB];
    auto load_codes = [&](int b, u32x4 (&cv)[NT], u32x2 (&sv)[NT][GPB]) {
        if (b >= L.blocks) return;
#pragma unroll
        for (int t = 0; t < NT; ++t) cv[t] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes[t] + (size_t)b * 1024));
        const uint32_t unit = GPB == 1 ? (uint32_t)b * A.per_group >> 20 : (uint32_t)b;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint16_t *p = scales[t] + (size_t)unit * GPB * kLinearRows;
            if constexpr (GPB == 1) {
                sv[t][0] = *reinterpret_cast<const u32x2 *>(p);
            } else {
#pragma unroll
                for (int g = 0; g < GPB; g += 2) {
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(p + 4 * g);
                    sv[t][g] = u32x2{v[0], v[1]};
                    sv[t][g + 1] = u32x2{v[2], v[3]};
                }
            }
        }
    };
    auto load_x = [&](int b, u32x4 (&v)[XL]) {
        if (b >= L.blocks) return;
        const int k0 = b * kLinearBlock;
        const bool in = !TAIL || k0 + 8 * col < k;
#pragma unroll
        for (int l = 0; l < XL; ++l) {
            v[l] = *reinterpret_cast<const u32x4 *>(xr[l] + (TAIL && !in ? -8 * col : k0));
            if (TAIL && !in) v[l] = u32x4{0, 0, 0, 0};
        }
    };
    auto stage = [&](int buf, const u32x4 (&v)[XL]) {
#pragma unroll
        for (int l = 0; l < XL; ++l) {
            const int row = 4 * (nw * XL + l) + h;
            xs[buf * STAGE + (slot * MT + row / 16) * 256 + col * 16 + ((row % 16) ^ col)] = v[l];
        }
    };
    // The offset's part of the row tiles that this wave has staged.
    auto stage_base = [&](int buf) {
#pragma unroll
        for (int q = 0; q < XL / 4; ++q) {
            const int m = nw * (XL / 4) + q;
            const u32x4 *xb = xs + buf * STAGE + (slot * MT + m) * 256;
#pragma unroll
            for (int g = 0; g < GPB; ++g) {
                v4f d{0, 0, 0, 0};
#pragma unroll
                for (int i = g * 4 / GPB; i < (g + 1) * 4 / GPB; ++i)
                    d = mfma32<DT>(minus, __builtin_bit_cast(uint4, xb[(4 * i + h) * 16 + (col ^ (4 * i + h))]), d);
                if (h == 0) bs[(((buf * WK + slot) * MT + m) * GPB + g) * 16 + col] = d;
            }
        }
    };
    // Step j (blocks j WK + slot) computes from its LDS buffer, asks for the codes of step
    // j + DEPTH, stages the x of step j + 1 and asks for that of step j + 1 + DEPTH.
    auto step = [&](int b, int par) {
        const int buf = WN == 1 ? 0 : par % 2, next = (par + 1) % DEPTH;
        u32x4 cc[NT];
        u32x2 cs[NT][GPB];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            cc[t] = c[par][t];
#pragma unroll
            for (int g = 0; g < GPB; ++g) cs[t][g] = sc[par][t][g];
        }
        load_codes(b + DEPTH * WK, c[par], sc[par]);
        if (b < L.blocks) {
            const u32x4 *xb = xs + buf * STAGE + slot * MT * 256;
            uint4 xf[XB][MT];
            auto load_xf = [&](int i) {
#pragma unroll
                for (int m = 0; m < MT; ++m) xf[i % XB][m] = __builtin_bit_cast(uint4, xb[m * 256 + (4 * i + h) * 16 + (col ^ (4 * i + h))]);
            };
#pragma unroll
            for (int i = 0; i < XB - 1; ++i) load_xf(i);
#pragma unroll
            for (int g = 0; g < GPB; ++g) {
                v4f s[NT][MT], base[MT];
                if constexpr (SHARE) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) base[m] = bs[(((buf * WK + slot) * MT + m) * GPB + g) * 16 + col];
                }
#pragma unroll
                for (int i = g * 4 / GPB; i < (g + 1) * 4 / GPB; ++i) {
                    const bool first = i == g * 4 / GPB;
                    if (i + XB - 1 < 4) load_xf(i + XB - 1);
                    if constexpr (XB > 1) __builtin_amdgcn_sched_barrier(0);
                    if constexpr (!SHARE) {
#pragma unroll
                        for (int m = 0; m < MT; ++m) base[m] = mfma32<DT>(minus, xf[i % XB][m], first ? v4f{0, 0, 0, 0} : base[m]);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint4 a = oct(cc[t][i]);
#pragma unroll
                        for (int m = 0; m < MT; ++m) s[t][m] = mfma32<DT>(a, xf[i % XB][m], first ? (SHARE ? base[m] : v4f{0, 0, 0, 0}) : s[t][m]);
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float f[4] = {f16_bits_to_float(cs[t][g][0] & 0xFFFFu), f16_bits_to_float(cs[t][g][0] >> 16),
                                        f16_bits_to_float(cs[t][g][1] & 0xFFFFu), f16_bits_to_float(cs[t][g][1] >> 16)};
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t][m][e] = fmaf(f[e], SHARE ? s[t][m][e] : s[t][m][e] + base[m][e], acc[t][m][e]);
                }
            }
        }
        if constexpr (WN == 1) wave_lds_fence();   // x is this wave's own: LDS serves it in order
        if (b + WK < L.blocks) stage(buf ^ (WN == 1 ? 0 : 1), xv[next]);
        if constexpr (SHARE) {
            wave_lds_fence();
            if (b + WK < L.blocks) stage_base(buf ^ 1);
        }
        load_x(b + (DEPTH + 1) * WK, xv[next]);
        if constexpr (WN == 1) wave_lds_fence();
        else __syncthreads();
    };
#pragma unroll
    for (int p = 0; p < DEPTH; ++p) {
        load_x(slot + p * WK, xv[p]);
        load_codes(slot + p * WK, c[p], sc[p]);
    }
    if (slot < L.blocks) stage(0, xv[0]);
    if constexpr (SHARE) {
        wave_lds_fence();
        if (slot < L.blocks) stage_base(0);
    }
    load_x(slot + DEPTH * WK, xv[0]);
    if constexpr (WN == 1) wave_lds_fence();
    else __syncthreads();
    for (int b0 = 0; b0 < L.blocks; b0 += DEPTH * WK) {
#pragma unroll
        for (int p = 0; p < DEPTH; ++p)
            if (b0 + p * WK < L.blocks) step(b0 + p * WK + slot, p);
    }
    __syncthreads();
    // The slots' sums, RT tiles at a time, over the staging area.
    v4f *red = reinterpret_cast<v4f *>(smem);   // [wave][RT][lane]
#pragma unroll
    for (int r = 0; r < TILES; r += RT) {
        if (r > 0) __syncthreads();
#pragma unroll
        for (int u = 0; u < RT; ++u) red[(wave * RT + u) * kWave + lane] = acc[(r + u) / MT][(r + u) % MT];
        __syncthreads();
        for (int u = slot; u < RT; u += WK) {
            v4f s = red[(nw * RT + u) * kWave + lane];
#pragma unroll
            for (int w = 1; w < WK; ++w) s += red[((w * WN + nw) * RT + u) * kWave + lane];
            const int t = (r + u) / MT, b = 16 * ((r + u) % MT) + col;
            const int j = (tile0 + t) * kLinearRows + 4 * h;
            if (b < batch) {
                uint16_t *dst = A.y + (size_t)(row0 + b) * A.ldy;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < n) dst[j + e] = float_to_half<DT>(s[e] + (A.bias ? half_to_float<DT>(A.bias[j + e]) : 0.0f));
            }
        }
    }
}

template <int DT, int NT, int RG, int WN, int GPB, bool TAIL>
static hipError_t run_linear(const LinearArgs &a, hipStream_t s) {
    constexpr int R = kLinearRows * NT * WN;
    constexpr size_t lds = linear_lds<NT, RG, WN, GPB>();
    auto *kernel = linear_kernel<DT, NT, RG, WN, GPB, TAIL>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)((a.n + R - 1) / R), (unsigned)((a.batch + 4 * RG - 1) / (4 * RG)));
    kernel<<<grid, 64 * kLinearWaves, lds, s>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_linear_dt(const LinearArgs &a, hipStream_t s) {
    const int gpb = a.group == 32 ? 4 : a.group == 64 ? 2 : 1;   // a block past k has groups of 32 or 64 only
    const bool tail = a.k % kLinearBlock != 0;
    const int n = a.n, batch = a.batch;
#define LINEAR(NT_, RG_, WN_)                                                                                  \
    return (gpb == 4 ? (tail ? run_linear<DT, NT_, RG_, WN_, 4, true>(a, s) : run_linear<DT, NT_, RG_, WN_, 4, false>(a, s))                      \
     : gpb == 2 ? (tail ? run_linear<DT, NT_, RG_, WN_, 2, true>(a, s) : run_linear<DT, NT_, RG_, WN_, 2, false>(a, s))                    \
                : run_linear<DT, NT_, RG_, WN_, 1, false>(a, s))
    // Outputs (16 NT WN) and rows (4 RG) per workgroup: the variant that reads least (codes once
    // per row tile, x once per group of outputs) among those with at most one workgroup per CU, as
    // a second one on some CUs leaves the others idle.  In us, by outputs x rows:
    //   7 rows    9973 x 3456   32: 10.3, 48: 7.6, 64: 8.5
    //   32 rows   1024 x 4096   16 x 16: 5.0, 16 x 32: 6.9      4096 x 4096  32 x 16: 7.4, 16 x 32: 8.8
    //             8192 x 8192   32 x 32: 16.1, 64 x 32: 21.9    14336 x 4096 64 x 32: 13.4, 128 x 32: 20.8
    //             28672 x 8192  32 x 32: 55, 64 x 32: 43, 128 x 32: 39
    //   64 rows   1024 x 4096   16 x 16: 6.0, 32 x 16: 7.1, 32 x 64: 15.4
    //             4096 x 4096   64 x 16: 9.8, 32 x 32: 10.1, 32 x 64: 15.6
    //             8192 x 8192   64 x 32: 21.0, 32 x 64: 25.8    14336 x 4096 64 x 64: 20.9, 64 x 32: 25.8
    //             28672 x 8192  64 x 64: 78, 128 x 64: 51
    // Up to 8 rows read little of x, and 32 outputs serve every n above (28672 x 8192, one row,
    // with 16 / 32 / 64: 26.4 / 24.6 / 27.0).  48 outputs are for n from 8193 to 12288 only; what
    // n past a larger multiple of 4096 leaves idle is not taken up.
    // The table is of groups of 128.  Groups of 64 and 32 hold two and four times the scales, and 64
    // rows x 64 outputs keep 8 to 34 registers a lane in scratch memory then, 64 x 128 and 16 x 64 up to 5.  In us, groups
    // 128, 64, 32, 64 rows:  14336 x 4096 20.6, 25.2, 34.1;  28672 x 8192 50.4, 55.0, 69.9;  8192 x 8192
    // 21.0, 23.0, 27.9;  4096 x 4096 9.6, 9.8, 11.6;  16 rows, 28672 x 8192 32.2, 33.0, 38.7.
    const int cus = 256;
    auto fits = [&](int outputs, int rows) { return (n + outputs - 1) / outputs * ((batch + rows - 1) / rows) <= cus; };
    if (batch <= 4) {
        if (fits(16, 4)) LINEAR(1, 1, 1);
        if (!fits(32, 4) && fits(48, 4)) LINEAR(3, 1, 1);
        LINEAR(2, 1, 1);
    }
    if (batch <= 8) {
        if (fits(16, 8)) LINEAR(1, 2, 1);
        if (!fits(32, 8) && fits(48, 8)) LINEAR(3, 2, 1);
        LINEAR(2, 2, 1);
    }
    if (fits(16, 16)) LINEAR(1, 4, 1);
    if (fits(32, 16)) LINEAR(2, 4, 1);
    if (batch <= 16) {
        if (fits(48, 16)) LINEAR(3, 4, 1);
        LINEAR(4, 4, 1);
    }
    if (batch <= 32) {
        if (fits(32, 32)) LINEAR(2, 8, 1);
        if (fits(64, 32)) LINEAR(2, 8, 2);
        LINEAR(2, 8, 4);
    }
    if (fits(64, 16)) LINEAR(4, 4, 1);
    if (fits(64, 32)) LINEAR(2, 8, 2);
    if (fits(64, 64)) LINEAR(2, 16, 2);
    LINEAR(2, 16, 4);
#undef LINEAR
}

}  // namespace prox
