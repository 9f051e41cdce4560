// Projections on 8-bit integers, y = (c_x c_w^T) sigma_x sigma_w (+ bias): weights packed and unpacked, and
// the product: y^T = W x^T as 16 x 16 x 64 MFMAs, exact in 32 bits.  The weights go from the caches to registers as
// operands (every wave's outputs are its own, and their layout is the operands'), x through LDS, where the waves share it;
// the sums are scaled and rounded once.  Few rows are bound by the weights' bytes (28672 x 8192, 16 rows 40.1 us,
// 5.9 TB/s), many by power: at 4096 rows the clock falls to 1.85 GHz (693 to 731 us by the card, 2630 to 2780 TOP/s).  What saves power there:
// 16 x 16 x 64 products rather than 32 x 32 x 32 (random operands, nothing else: 3695 and 3160 TOP/s), one operand
// kept from product to product (4075 TOP/s).
#include "linear_w8.hpp"

namespace prox {

namespace {

// Packing: a workgroup takes the 16 outputs of a tile, 16 lanes each, 16 inputs a lane and step, and reads them twice
// (the second time from the L2), so that it writes whole runs of 1024 bytes.  28672 x 8192 270 us (705 MB, 2.6 TB/s).
// A code is the exact quotient's, as rows in 8 bits have it: where 32 bits leave it near the middle of two, 64 decide.
template <int DT>
__global__ __launch_bounds__(256) void pack_w8_kernel(const uint16_t *__restrict__ w, int n, int k, uint8_t *__restrict__ blob) {
    const Linear8Layout L(n, k);
    const int nb = blockIdx.x / 4, tile = blockIdx.x % 4, l = threadIdx.x % 16, r = threadIdx.x / 16;
    const int j = nb * kLinear8N + w8_output(tile, r);
    const uint16_t *src = w + (size_t)j * k;
    const int kk = j < n ? k : 0;
    auto load16 = [&](int i, uint32_t (&v)[8]) {   // past k: 0
        if (i + 16 <= kk) {
            __builtin_memcpy(v, __builtin_assume_aligned(src + i, 2), 32);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t lo = i + 2 * e < kk ? src[i + 2 * e] : 0u, hi = i + 2 * e + 1 < kk ? src[i + 2 * e + 1] : 0u;
                v[e] = lo | hi << 16;
            }
        }
    };
    uint32_t top = 0;   // bits of sizes, which order like them, NaN above all
    for (int i = 16 * l; i < kk; i += 256) {
        uint32_t v[8];
        load16(i, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, max(v[e] & 0x7FFFu, v[e] >> 16 & 0x7FFFu));
    }
    for (int m = 1; m < 16; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    const float most = half_to_float<DT>((uint16_t)top);
    const bool finite = most < INFINITY, plain = finite && most >= 0x1p-100f;   // 127 / most is a finite number
    if (l == 0) reinterpret_cast<float *>(blob + L.scales)[j] = finite ? (float)((double)most * (1.0 / 127.0)) : __uint_as_float(0x7FC00000u);
    const float s = plain ? 127.0f / most : 0.0f;
    for (int c = l; c < 4 * L.kblocks; c += 16) {   // chunks of 16 inputs
        uint32_t v[8], word[4];
        load16(16 * c, v);
        float far = plain ? 0.0f : 1.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float p = e % 2 ? hi_to_float<DT>(v[e / 2]) : lo_to_float<DT>(v[e / 2]);
            const float m = fmaf(p, s, 12582912.0f);   // 1.5 * 2^23: rounds to whole numbers, half to even
            far = fmaxf(far, fabsf(fmaf(p, s, 12582912.0f - m)));
            const uint32_t code = __float_as_uint(m) & 0xFFu;
            word[e / 4] = e % 4 ? word[e / 4] | code << (8 * (e % 4)) : code;
        }
        if (far > 0.49997f) {   // off by 127 * 3 * 2^-24 at most
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = e % 2 ? hi_to_float<DT>(v[e / 2]) : lo_to_float<DT>(v[e / 2]);
                const uint32_t code = finite && most > 0.0f ? (uint32_t)(int)rint((double)p * 127.0 / (double)most) & 0xFFu : 0u;
                word[e / 4] = e % 4 ? word[e / 4] | code << (8 * (e % 4)) : code;
            }
        }
        const size_t at = (((size_t)nb * L.kblocks + c / 4) * 4 + tile) * 1024 + (size_t)((c % 4) * 16 + r) * 16;
        *reinterpret_cast<uint4 *>(blob + at) = make_uint4(word[0], word[1], word[2], word[3]);
    }
}

// Inverse view: a thread takes (output, input) items, a grid apart.
__global__ __launch_bounds__(256) void unpack_w8_kernel(const uint8_t *__restrict__ blob, int n, int k, int8_t *__restrict__ codes,
                                                        float *__restrict__ scales) {
    const Linear8Layout L(n, k);
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < (long long)n * k; id += (long long)gridDim.x * 256) {
        const int j = (int)(id / k), i = (int)(id % k), o = j % kLinear8N;
        const int tile = o / 4 % 4, r = 4 * (o / 16) + o % 4;
        const size_t at = (((size_t)(j / kLinear8N) * L.kblocks + i / 64) * 4 + tile) * 1024 + (size_t)(i % 64 / 16 * 16 + r) * 16 + i % 16;
        codes[id] = (int8_t)blob[at];
        if (i == 0) scales[j] = reinterpret_cast<const float *>(blob + L.scales)[j];
    }
}

// Weights that are read once by a call (ONCE) are loaded as a stream: 28672 x 8192, 16 rows 40.1 us, without 44.6.
template <bool ONCE>
__device__ __forceinline__ u32x4 load_weights(const uint8_t *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
    else return *reinterpret_cast<const u32x4 *>(p);
}

// Four outputs from j of a row: scales, bias and rounding.
template <int DT>
__device__ __forceinline__ uint2 finish4(const Linear8Args &A, const float *ws, int j, float sx, v4i acc) {
    const v4f sw = *reinterpret_cast<const v4f *>(ws + j);   // padded to 64 outputs
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf((float)acc[e] * sw[e], sx, A.bias ? half_to_float<DT>(A.bias[min(j + e, A.n - 1)]) : 0.0f);
    return make_uint2(round_pair<DT>(v[0], v[1]), round_pair<DT>(v[2], v[3]));
}

// W8Shape: a wave takes 16 NT outputs by 16 MT rows; a workgroup WN x WM waves, WK times: its WK parts take a step of
// 128 inputs in turn.  S: halves of a step whose weights are in registers or on the way; XD: steps of x alike.
template <int NT_, int MT_, int WM_, int WN_, int WK_, int S_, int XD_>
struct W8Shape {
    static constexpr int NT = NT_, MT = MT_, WM = WM_, WN = WN_, WK = WK_, S = S_, XD = XD_;
    static constexpr int OUTS = 16 * NT * WN, ROWS = 16 * MT * WM, PART = 64 * WM * WN, THREADS = PART * WK;
    static constexpr int XL = ROWS * 8 / PART;                     // loads of x of a step by each of its threads
    static constexpr int PM = MT < 4 ? MT : 4, PH = MT / PM;       // row fragments of a phase, phases of a half
    static constexpr int U = S % 2 ? S : S / 2 > XD ? S / 2 : XD;  // steps until the sets of registers stand as before
    static constexpr int WAVES = THREADS / 64;
    static constexpr int MC = WAVES * NT * MT <= 128 ? MT : 128 / (WAVES * NT);   // row fragments whose parts are added at a time
    static constexpr bool TILE = NT == 4 && (WK == 1 || MC % WK == 0);   // whole rows of 64 outputs are written through LDS
    static constexpr int MINE = WK == 1 ? (MT < 4 ? MT : 4) : MC / WK;   // row fragments of a part at a time, then
    static constexpr size_t stage = (size_t)2 * WK * ROWS * 128;
    static constexpr size_t last = WK == 1 ? (size_t)WAVES * MINE * 2048 : (size_t)WAVES * NT * MC * 1024;
    static constexpr size_t lds = stage > last ? stage : last;
    static_assert(XL * PART == ROWS * 8 && PM * PH == MT && (2 * U) % S == 0 && U % XD == 0, "whole loads, phases and turns");
    static_assert(lds <= 163840 && MT % MC == 0 && (TILE || MC == MT), "LDS");
};

// ONCE: no two workgroups read the same weights.
template <int DT, class C, bool ONCE>
__global__ __launch_bounds__(C::THREADS, (C::THREADS + 511) / 512 * 2) void linear_w8_kernel(Linear8Args A, int mtiles, int ntiles) {
    constexpr int NT = C::NT, MT = C::MT, WM = C::WM, WN = C::WN, WK = C::WK, S = C::S, XD = C::XD, ROWS = C::ROWS, XL = C::XL;
    constexpr int PM = C::PM, PH = C::PH, U = C::U, H = 2 * U;
    extern __shared__ __align__(16) unsigned char smem[];
    const int nblocks = (A.n + kLinear8N - 1) / kLinear8N;
    // Workgroups go round the 8 XCDs: each takes a run of tiles, 4 row tiles deep.
    const int total = mtiles * ntiles, id = (int)blockIdx.x, q = total / 8, rem = total % 8;
    const int xcd = id % 8, at = xcd * q + min(xcd, rem) + id / 8;
    const int group = at / (4 * ntiles), depth = min(4, mtiles - 4 * group), in = at - group * 4 * ntiles;
    const int row0 = (4 * group + in % depth) * ROWS, ntile = in / depth;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = lane_id();
    const int part = wave / (WM * WN), wm = wave % WM, wn = wave / WM % WN, h = lane / 16, col = lane % 16;
    const int pt = (int)threadIdx.x % C::PART;
    const int tile0 = (ntile * WN + wn) * NT;   // of 16 outputs
    const uint8_t *w = A.codes + (size_t)min(tile0 / 4, nblocks - 1) * A.kblocks * 4096 + tile0 % 4 * 1024;
    v4i *xs = reinterpret_cast<v4i *>(smem) + part * 2 * ROWS * 8;   // [buffer][row][chunk of 16 inputs ^ row % 8]
    // Rows past the last: the last again (not stored).  Inputs past k: any, they meet codes 0.
    const int8_t *x = A.x + (size_t)row0 * A.ldx;
    const int chunk = pt % 8, kend = (A.k - 1) / 16 * 16;
    int xrow[XL];
#pragma unroll
    for (int l = 0; l < XL; ++l) xrow[l] = min(l * (C::PART / 8) + pt / 8, A.rows - 1 - row0) * (int)A.ldx;
    const int xst = (pt / 8) * 8 + (chunk ^ (pt / 8 % 8));
    const int ksteps = A.kblocks / 2, steps = (ksteps + WK - 1) / WK;   // step i of this part: inputs from 128 (i WK + part)
    v4i acc[NT][MT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = v4i{0, 0, 0, 0};
    v4i xv[XD][XL], wv[S][NT], b[2][PM];
    auto load_x = [&](int set, int l, int i) {
        xv[set][l] = *reinterpret_cast<const v4i *>(x + (uint32_t)(xrow[l] + min((min(i, steps - 1) * WK + part) * 128 + chunk * 16, kend)));
    };
    auto store_x = [&](int set, int l, int i) {
        v4i v = xv[set][l];
        if (WK > 1 && i * WK + part >= ksteps) v = v4i{0, 0, 0, 0};   // past the last step of all: weights of another meet zeros
        xs[(i % 2) * ROWS * 8 + l * C::PART + xst] = v;
    };
    auto load_w = [&](int set, int t, int i) {   // half i
        const int k = min(2 * (min(i / 2, steps - 1) * WK + part) + i % 2, A.kblocks - 1);
        wv[set][t] = __builtin_bit_cast(v4i, load_weights<ONCE>(w + (size_t)k * 4096 + (uint32_t)(lane * 16 + t * 1024)));
    };
    auto read_b = [&](int p, int m, int buf) {
        const int row = (wm * MT + p % PH * PM + m) * 16 + col;
        b[p % 2][m] = xs[buf * ROWS * 8 + row * 8 + ((4 * (p / PH) + h) ^ (col % 8))];
    };
    auto part_sync = [&] {
        if constexpr (WM * WN == 1) wave_lds_fence();   // x is this wave's own: LDS serves it in order
        else __syncthreads();
    };
    // Loads are counted in order: those in flight before the first step stand as they do before every other.
#pragma unroll
    for (int l = 0; l < XL; ++l) load_x(0, l, 0);
#pragma unroll
    for (int l = 0; l < XL; ++l) store_x(0, l, 0);
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
#pragma unroll
        for (int d = 1; d <= XD; ++d)
            if (i == (S - 2 - 2 * (XD - d) > 0 ? S - 2 - 2 * (XD - d) : 0)) {
#pragma unroll
                for (int l = 0; l < XL; ++l) load_x(d % XD, l, d);
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < NT; ++t) load_w(i, t, i);
        __builtin_amdgcn_sched_barrier(0);
    }
    part_sync();
#pragma unroll
    for (int m = 0; m < PM; ++m) read_b(0, m, 0);
    for (int i0 = 0; i0 < steps; i0 += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u, buf = i % 2;
            if (i >= steps) break;
#pragma unroll
            for (int p = 0; p < 2 * PH; ++p) {
                // The operands of the next phase; those of the next step are there behind the barrier.
                if (p == 2 * PH - 1) part_sync();
                const int half = 2 * u + p / PH;
#pragma unroll
                for (int m = 0; m < PM; ++m) {
                    // Reads, loads and stores between the products, which leave 12 of 16 cycles to them.  Past the last
                    // step: the last again, unused (no branches, which would cost the count of loads in flight).
                    read_b((p + 1) % (2 * PH), m, p == 2 * PH - 1 ? buf ^ 1 : buf);
                    if (p % PH == 0) {   // into the set of the half before, of which no product is left
#pragma unroll
                        for (int t = m * NT / PM; t < (m + 1) * NT / PM; ++t) load_w((half + H - 1) % S, t, 2 * i + p / PH + S - 1);
                    }
                    if (p == (PH > 1)) {
#pragma unroll
                        for (int l = m * XL / PM; l < (m + 1) * XL / PM; ++l) {
                            store_x((u + 1) % XD, l, i + 1);
                            load_x((u + 1) % XD, l, i + 1 + XD);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int e = 0; e < NT; ++e) {   // one operand of two stays from product to product: less power, a higher clock
                        const int t = m % 2 ? NT - 1 - e : e;
                        acc[t][p % PH * PM + m] = mfma16_i8(wv[half % S][t], b[p % 2][m], acc[t][p % PH * PM + m]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }
    const float *ws = A.sw;
    v4i *red = reinterpret_cast<v4i *>(smem);   // [wave][row fragment][tile][lane]
    // The parts' sums of row fragments m0 .. m0 + MC - 1, to LDS (but those that the part itself adds up, if it takes
    // whole fragments); and of tile (t, m0 + m) of this wave's outputs and rows.
    auto share = [&](int m0) {
        __syncthreads();
#pragma unroll
        for (int m = 0; m < C::MC; ++m) {
            if (C::TILE && m / C::MINE == part) continue;
#pragma unroll
            for (int t = 0; t < NT; ++t) red[((wave * C::MC + m) * NT + t) * kWave + lane] = acc[t][m0 + m];
        }
        __syncthreads();
    };
    auto sum = [&](int t, int m) {
        v4i s{0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < WK; ++g) s += red[(((g * WM * WN + wave % (WM * WN)) * C::MC + m) * NT + t) * kWave + lane];
        return s;
    };
    const int row1 = row0 + wm * MT * 16;
    if constexpr (C::TILE) {   // this part's row fragments, MINE at a time
        constexpr int MINE = C::MINE, EACH = MINE * WK;
        const int j0 = tile0 * 16;
        const bool whole = j0 + 64 <= A.n;
        v4i *out = reinterpret_cast<v4i *>(smem) + wave * MINE * 128;
#pragma unroll
        for (int m0 = 0; m0 < MT; m0 += EACH) {
            v4i v[4][MINE];
            if constexpr (WK > 1) share(m0);
#pragma unroll
            for (int f = 0; f < MINE; ++f)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if constexpr (WK == 1) {
                        v[t][f] = acc[t][m0 + f];
                    } else {
                        v[t][f] = v4i{0, 0, 0, 0};
#pragma unroll
                        for (int g = 0; g < WK; ++g)
                            v[t][f] += g == part ? acc[t][m0 + g * MINE + f]
                                                 : red[(((g * WM * WN + wave % (WM * WN)) * C::MC + part * MINE + f) * NT + t) * kWave + lane];
                    }
                }
            if constexpr (WK > 1) __syncthreads();
            else wave_lds_fence();
            if (j0 >= A.n) continue;
            const int first = row1 + (m0 + part * MINE) * 16;
#pragma unroll
            for (int f = 0; f < MINE; ++f) {
                const float sx = A.scales[min(first + 16 * f + col, A.rows - 1)];
#pragma unroll
                for (int c = 0; c < 2; ++c) {   // outputs 16 h + 8 c .. + 7
                    const uint2 lo = finish4<DT>(A, ws, j0 + 16 * h + 8 * c, sx, v[2 * c][f]);
                    const uint2 hi = finish4<DT>(A, ws, j0 + 16 * h + 8 * c + 4, sx, v[2 * c + 1][f]);
                    out[f * 128 + col * 8 + ((2 * h + c) ^ (col % 8))] = v4i{(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
                }
            }
            wave_lds_fence();
#pragma unroll
            for (int l = 0; l < 2 * MINE; ++l) {   // 8 lanes write the 128 bytes of a row
                const int r = 8 * l + lane / 8, c = lane % 8;
                if (first + r >= A.rows) continue;
                const v4i o = out[r * 8 + (c ^ (r % 8))];
                uint16_t *dst = A.y + (size_t)(first + r) * A.ldy + j0 + 8 * c;
                if (whole) {
                    __builtin_memcpy(__builtin_assume_aligned(dst, 2), &o, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (j0 + 8 * c + e < A.n) dst[e] = (uint16_t)((uint32_t)o[e / 2] >> (16 * (e % 2)));
                }
            }
        }
    } else {   // tiles in turn among the parts
        share(0);
        for (int v = part; v < NT * MT; v += WK) {
            const int t = v % NT, m = v / NT, row = row1 + 16 * m + col;
            const int j = (tile0 + t) / 4 * kLinear8N + w8_output((tile0 + t) % 4, 4 * h);
            if (row >= A.rows || j >= A.n) continue;
            const uint2 o = finish4<DT>(A, ws, j, A.scales[row], sum(t, m));
            uint16_t *dst = A.y + (size_t)row * A.ldy + j;
            if (j + 4 <= A.n) {
                __builtin_memcpy(__builtin_assume_aligned(dst, 2), &o, 8);
            } else {
                dst[0] = (uint16_t)o.x;
                if (j + 1 < A.n) dst[1] = (uint16_t)(o.x >> 16);
                if (j + 2 < A.n) dst[2] = (uint16_t)o.y;
            }
        }
    }
}

template <int DT, class C, bool ONCE>
hipError_t run_once(const Linear8Args &a, hipStream_t s) {
    auto *kernel = linear_w8_kernel<DT, C, ONCE>;
    if constexpr (C::lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::lds);
        if (e != hipSuccess) return e;
    }
    // The outputs of a block of 64 are spread over its four tiles: all of them are needed.
    const int mtiles = (a.rows + C::ROWS - 1) / C::ROWS, ntiles = ((a.n + 63) / 64 * 64 + C::OUTS - 1) / C::OUTS;
    kernel<<<(unsigned)(mtiles * ntiles), C::THREADS, C::lds, s>>>(a, mtiles, ntiles);
    return hipGetLastError();
}

template <int DT, class C>
hipError_t run(const Linear8Args &a, hipStream_t s) {
    if constexpr (C::ROWS <= 64) {
        if (a.rows <= C::ROWS) return run_once<DT, C, true>(a, s);
    }
    return run_once<DT, C, false>(a, s);
}

}  // namespace

hipError_t launch_pack_linear_w8(int dtype, const void *w, int n, int k, void *blob, hipStream_t s) {
    const Linear8Layout L(n, k);
    auto *wp = static_cast<const uint16_t *>(w);
    auto *b = static_cast<uint8_t *>(blob);
    if (dtype == kBF16) pack_w8_kernel<kBF16><<<4 * L.nblocks, 256, 0, s>>>(wp, n, k, b);
    else pack_w8_kernel<kF16><<<4 * L.nblocks, 256, 0, s>>>(wp, n, k, b);
    return hipGetLastError();
}

hipError_t launch_unpack_linear_w8(const void *blob, int n, int k, int8_t *codes, float *scales, hipStream_t s) {
    const long long blocks = ((long long)n * k + 255) / 256;
    unpack_w8_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(static_cast<const uint8_t *>(blob), n, k, codes, scales);
    return hipGetLastError();
}

// The variant by shape: the one that takes least by a model of its rounds of 256 workgroups, one a CU: each its start
// and last step, and a time per 1024 inputs that grows with the workgroups under way, as they share the L2s and the power.
// The weights' bytes from HBM, which all variants read alike for few rows, are left out: it ranks, and is no estimate there.
// Larger tiles read less for each product, which bounds all but the largest; smaller ones fill the CUs.  In us at
// k = 4096 (bf16, streams of calls), for 1 round and for 4:
//   256 x 256  59.8, 227    128 x 256  34.2, 142    128 x 128  22.0, 84    64 x 256  21.7, 96    64 x 128  14.2, 53
//   32 x 128   11.3, 41     64 x 64    11.2, 39     32 x 64    8.3, 28     32 x 32   7.1, 17     16 x 64   7.1, 20.5
//   16 x 32    7.1, 13      16 x 16    7.1, 9.6
// 512 rows, 6144 x 4096: 128 x 128 19.1, 64 x 128 25.5, 128 x 256 25.4, 256 x 256 40.8.  128 rows, 4096 x 4096: 32 x 64
// 8.3, 32 x 32 10.0, 64 x 64 11, 128 x 128 17.6.  64 rows, 28672 x 8192: 64 x 128 41.6, 32 x 128 58.6, 64 x 64 55.
struct W8Cost {
    int rows, outs;
    float start, few, all;   // us; per 1024 inputs with one workgroup under way, and 256
};
constexpr int kW8Variants = 12;
constexpr long long kW8MaxGrid = 1 << 23;
constexpr W8Cost kW8Cost[kW8Variants] = {{256, 256, 5.0f, 8.4f, 12.6f}, {128, 256, 4.0f, 4.7f, 7.0f}, {128, 128, 4.0f, 2.7f, 4.2f},
                                         {64, 256, 3.5f, 3.0f, 5.0f},   {64, 128, 3.0f, 1.6f, 2.6f},  {32, 128, 2.5f, 1.2f, 1.8f},
                                         {64, 64, 3.0f, 1.1f, 1.6f},    {32, 64, 2.4f, 0.7f, 1.05f},  {32, 32, 1.8f, 0.35f, 0.5f},
                                         {16, 64, 1.5f, 0.6f, 0.85f},   {16, 32, 1.3f, 0.3f, 0.45f},  {16, 16, 1.0f, 0.25f, 0.35f}};
constexpr float kW8Launch = 2.0f;

// Workgroups of 512 threads, within the 32 bits of a grid.
inline bool w8_fits(const W8Cost &c, int rows, int n) {
    return ((long long)rows + c.rows - 1) / c.rows * ((n + c.outs - 1) / c.outs) < kW8MaxGrid;
}

inline float w8_time(const W8Cost &c, int rows, int n, float k1024) {
    const long long tiles = ((long long)rows + c.rows - 1) / c.rows * ((n + c.outs - 1) / c.outs), full = tiles / 256;
    const float rest = (float)(tiles % 256) / 256.0f;
    float t = (float)full * (c.start + k1024 * c.all);
    if (rest > 0.0f) t += c.start + k1024 * (c.few + (c.all - c.few) * rest);
    return t;
}

inline int w8_variant(int rows, int n, float k1024, float *least) {   // the largest tiles fit (linear_w8_fits)
    int best = 0;
    *least = w8_time(kW8Cost[0], rows, n, k1024);
    for (int v = 1; v < kW8Variants; ++v) {
        const float t = w8_time(kW8Cost[v], rows, n, k1024);
        if (t < *least && w8_fits(kW8Cost[v], rows, n)) best = v, *least = t;
    }
    return best;
}

template <int DT>
hipError_t run_variant(int v, const Linear8Args &a, hipStream_t s) {
    switch (v) {
    case 0: return run<DT, W8Shape<4, 8, 2, 4, 1, 3, 1>>(a, s);
    case 1: return run<DT, W8Shape<4, 8, 1, 4, 2, 3, 1>>(a, s);
    case 2: return run<DT, W8Shape<4, 4, 2, 2, 2, 4, 2>>(a, s);
    case 3: return run<DT, W8Shape<4, 4, 1, 4, 2, 4, 2>>(a, s);
    case 4: return run<DT, W8Shape<4, 4, 1, 2, 4, 4, 2>>(a, s);
    case 5: return run<DT, W8Shape<4, 2, 1, 2, 4, 4, 2>>(a, s);
    case 6: return run<DT, W8Shape<4, 4, 1, 1, 8, 4, 1>>(a, s);
    case 7: return run<DT, W8Shape<4, 2, 1, 1, 8, 4, 2>>(a, s);
    case 8: return run<DT, W8Shape<2, 2, 1, 1, 8, 4, 2>>(a, s);
    case 9: return run<DT, W8Shape<4, 1, 1, 1, 8, 4, 2>>(a, s);
    case 10: return run<DT, W8Shape<2, 1, 1, 1, 8, 4, 2>>(a, s);
    default: return run<DT, W8Shape<1, 1, 1, 1, 8, 4, 2>>(a, s);
    }
}

// A call whose last round would leave many CUs idle is cut in two launches: outputs that make whole rounds of large
// tiles, and the rest in tiles of their own (2048 rows, 10240 x 8192: 256 x 256 180 us, 128 x 256 172, 8192 outputs of the
// one and 2048 in 128 x 128 148).
template <int DT>
hipError_t launch_dt(const Linear8Args &a, hipStream_t s) {
    const float k1024 = (float)a.k / 1024.0f;
    float least = 0.0f;
    int best = w8_variant(a.rows, a.n, k1024, &least), rest = -1, cut = 0;
    for (int v = 0; v < 2; ++v) {
        const W8Cost &c = kW8Cost[v];
        const long long mtiles = ((long long)a.rows + c.rows - 1) / c.rows, ntiles = (a.n + c.outs - 1) / c.outs;
        const long long whole = mtiles * ntiles / 256 * 256 / mtiles;   // columns of tiles of the whole rounds
        if (whole < 1 || whole >= ntiles || !w8_fits(c, a.rows, a.n)) continue;
        const int n0 = (int)whole * c.outs;
        float t;
        const int u = w8_variant(a.rows, a.n - n0, k1024, &t);
        t += w8_time(c, a.rows, n0, k1024) + kW8Launch;
        if (t < least) best = v, rest = u, cut = n0, least = t;
    }
    if (rest < 0) return run_variant<DT>(best, a, s);
    Linear8Args b = a;
    b.n = cut;
    const hipError_t e = run_variant<DT>(best, b, s);
    if (e != hipSuccess) return e;
    b.n = a.n - cut;
    b.codes += (size_t)(cut / kLinear8N) * a.kblocks * (kLinear8N * kLinear8K);
    b.sw += cut;
    b.y += cut;
    if (b.bias) b.bias += cut;
    return run_variant<DT>(rest, b, s);
}

bool linear_w8_fits(int rows, int n) { return w8_fits(kW8Cost[0], rows, n); }

hipError_t launch_linear_w8(int dtype, const Linear8Args &a, hipStream_t s) {
    return dtype == kBF16 ? launch_dt<kBF16>(a, s) : launch_dt<kF16>(a, s);
}

}  // namespace prox
