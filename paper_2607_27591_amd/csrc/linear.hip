// Projections on INT4 weights with group scales: packing, its inverse view, and
// y = x W^T (+ bias) for up to 64 rows.
#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace prox {

// Packing: a workgroup takes the 16 rows of a tile over one unit of inputs (a group,
// at least 128), 16 lanes a row, so that it writes whole blocks of 1024 bytes.  A unit of
// 128 is read once, a longer group twice.  Bound by HBM (weights read once).
template <int DT>
__global__ __launch_bounds__(256) void pack_linear_kernel(const uint16_t *__restrict__ w, int n, int k,
                                                          int group, uint8_t *__restrict__ blob) {
    const LinearLayout L(n, k, group);
    const int tile = blockIdx.x, l = threadIdx.x % 16, r = threadIdx.x / 16;
    const int unit = group > kLinearBlock ? group : kLinearBlock;
    const int first = (int)blockIdx.y * unit;
    const int j = tile * kLinearRows + r;
    const uint16_t *src = w + (size_t)j * k;
    uint16_t *scales = reinterpret_cast<uint16_t *>(blob + L.scales) + (size_t)tile * L.groups * kLinearRows + r;
    auto load = [&](int i) {   // past the matrix: zeros
        return j < n && i < k ? *reinterpret_cast<const uint4 *>(src + i) : make_uint4(0, 0, 0, 0);
    };
    const int span = group < kLinearBlock ? group / 8 : 16;   // lanes of a group
    uint4 v = load(first + 8 * l);
    uint32_t a = abs_max8<DT>(v);
    for (int i = kLinearBlock; i < unit; i += kLinearBlock) a = max(a, abs_max8<DT>(load(first + i + 8 * l)));
    for (int m = 1; m < span; m <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, m));
    const GroupScale s = group_scale<DT>(a, 7);
    const int g = (first + 8 * l) / group;
    if (l % span == 0 && g < L.groups) scales[(size_t)g * kLinearRows] = s.bits;
    for (int i = 0; i < unit; i += kLinearBlock) {
        if (i > 0) v = load(first + i + 8 * l);
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            int q = quantise<DT>(half_of(v, e), s.sigma, s.inv, 7.0f);
            if (s.sigma == 0.0f) q = 0;   // a NaN weight too
            word |= (uint32_t)(q + 8) << (4 * nibble_of(e));
        }
        const size_t blk = (size_t)tile * L.blocks + (first + i) / kLinearBlock;
        *reinterpret_cast<uint32_t *>(blob + blk * 1024 + (size_t)((l % 4) * 16 + r) * 16 + (l / 4) * 4) = word;
    }
}

// Inverse view: one thread per (row, 8 inputs).
__global__ __launch_bounds__(256) void unpack_linear_kernel(const uint8_t *__restrict__ blob, int n, int k,
                                                            int group, int8_t *__restrict__ codes,
                                                            uint16_t *__restrict__ scales) {
    const LinearLayout L(n, k, group);
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int per = k / 8;
    if (id >= (long long)n * per) return;
    const int j = (int)(id / per), ch = (int)(id % per);
    const int c = ch % 16;   // chunk of the block
    const size_t blk = (size_t)(j / kLinearRows) * L.blocks + ch / 16;
    const uint32_t word = *reinterpret_cast<const uint32_t *>(
        blob + blk * 1024 + (size_t)((c % 4) * 16 + j % kLinearRows) * 16 + (c / 4) * 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) codes[id * 8 + e] = (int8_t)((int)((word >> (4 * nibble_of(e))) & 15) - 8);
    const int g = ch * 8 / group;
    if (ch * 8 % group == 0)
        scales[(size_t)j * L.groups + g] = reinterpret_cast<const uint16_t *>(
            blob + L.scales)[((size_t)(j / kLinearRows) * L.groups + g) * kLinearRows + j % kLinearRows];
}

// y^T = W x^T as MFMAs: 16 outputs by 16 batch rows by 32 inputs each.  The codes enter as
// exact 16-bit values with an offset, the offset's part (bias times the sum of x, one more
// product per 32 inputs for all NT tiles) starts each group's sum, and the scale is applied
// to the group's fp32 sum, so that nothing is rounded before y.  Bound by HBM: the codes are read
// once.  A workgroup takes NT tiles of 16 outputs over all inputs, its 8 waves blocks of
// 128 inputs in turn, so that 8 KB of each tile stream together and no partial sums leave
// the workgroup; they are added in a fixed order through LDS.  x is read from the L2, once
// per workgroup, for which NT grows with the batch.
// GPB: groups per block of 128 (4, 2, or 1 for groups of 128 and more).
constexpr int kLinearWaves = 8;
constexpr int kLinearRedTiles = 8;   // 16 x 16 tiles added at a time: 64 KB of LDS

template <int DT, int NT, int MT, int GPB>
__global__ __launch_bounds__(64 * kLinearWaves) void linear_kernel(
    const uint8_t *__restrict__ blob, int n, int k, int group, const uint16_t *__restrict__ x, int64_t ldx, int batch,
    const uint16_t *__restrict__ bias, uint16_t *__restrict__ y, int64_t ldy) {
    constexpr int TILES = NT * MT, RT = TILES < kLinearRedTiles ? TILES : kLinearRedTiles;
    __shared__ v4f red[kLinearWaves][RT][kWave];
    const LinearLayout L(n, k, group);
    const int lane = lane_id(), wave = threadIdx.x / kWave, h = lane / 16;
    const int tile0 = blockIdx.x * NT;
    const Int4Oct<DT> oct;
    const uint4 minus = Int4Oct<DT>::minus();
    const uint16_t *xr[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) xr[m] = x + (size_t)min(16 * m + lane % 16, batch - 1) * ldx + 8 * h;
    const uint8_t *codes[NT];
    const uint16_t *scales[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {   // past the last tile: the last again, not stored
        const int tile = min(tile0 + t, L.tiles - 1);
        codes[t] = blob + (size_t)tile * L.blocks * 1024 + lane * 16;
        scales[t] = reinterpret_cast<const uint16_t *>(blob + L.scales) + (size_t)tile * L.groups * kLinearRows + 4 * h;
    }
    v4f acc[NT][MT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = v4f{0, 0, 0, 0};
    uint4 c[NT];
    auto load_codes = [&](int b, uint4 (&v)[NT]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) v[t] = load_stream16(codes[t] + (size_t)b * 1024);
    };
    if (wave < L.blocks) load_codes(wave, c);
    for (int b = wave; b < L.blocks; b += kLinearWaves) {
        uint4 xv[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k0 = b * kLinearBlock + 32 * i;   // k is a multiple of 32
                xv[m][i] = k0 < k ? *reinterpret_cast<const uint4 *>(xr[m] + k0) : make_uint4(0, 0, 0, 0);
            }
        uint2 sc[NT][GPB];
        const int g0 = GPB == 1 ? b * kLinearBlock / group : b * GPB;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int g = 0; g < GPB; ++g)
                sc[t][g] = *reinterpret_cast<const uint2 *>(scales[t] + (size_t)min(g0 + g, L.groups - 1) * kLinearRows);
        uint4 cn[NT];
        if (b + kLinearWaves < L.blocks) load_codes(b + kLinearWaves, cn);
#pragma unroll
        for (int g = 0; g < GPB; ++g) {
            v4f base[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                base[m] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int i = g * 4 / GPB; i < (g + 1) * 4 / GPB; ++i) base[m] = mfma32<DT>(minus, xv[m][i], base[m]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                v4f s[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) s[m] = base[m];
                const uint32_t w[4] = {c[t].x, c[t].y, c[t].z, c[t].w};
#pragma unroll
                for (int i = g * 4 / GPB; i < (g + 1) * 4 / GPB; ++i) {
                    const uint4 a = oct(w[i]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) s[m] = mfma32<DT>(a, xv[m][i], s[m]);
                }
                const float f[4] = {f16_bits_to_float(sc[t][g].x & 0xFFFFu), f16_bits_to_float(sc[t][g].x >> 16),
                                    f16_bits_to_float(sc[t][g].y & 0xFFFFu), f16_bits_to_float(sc[t][g].y >> 16)};
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][m][e] = fmaf(f[e], s[m][e], acc[t][m][e]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) c[t] = cn[t];
    }
    // The waves' sums: RT tiles at a time, wave w adds tile w of them.
#pragma unroll
    for (int r = 0; r < TILES; r += RT) {
        if (r > 0) __syncthreads();
#pragma unroll
        for (int u = 0; u < RT; ++u) red[wave][u][lane] = acc[(r + u) / MT][(r + u) % MT];
        __syncthreads();
        if (wave < RT) {
            v4f s = red[0][wave][lane];
#pragma unroll
            for (int w = 1; w < kLinearWaves; ++w) s += red[w][wave][lane];
            const int t = (r + wave) / MT, b = 16 * ((r + wave) % MT) + lane % 16;
            const int j = (tile0 + t) * kLinearRows + 4 * h;
            if (b < batch) {
                uint16_t *dst = y + (size_t)b * ldy;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < n) dst[j + e] = float_to_half<DT>(s[e] + (bias ? half_to_float<DT>(bias[j + e]) : 0.0f));
            }
        }
    }
}

hipError_t launch_pack_linear(int dtype, const void *w, int n, int k, int group, void *blob, hipStream_t s) {
    const LinearLayout L(n, k, group);
    const int unit = group > kLinearBlock ? group : kLinearBlock;
    const dim3 grid((unsigned)L.tiles, (unsigned)((k + unit - 1) / unit));
    auto *wp = static_cast<const uint16_t *>(w);
    auto *b = static_cast<uint8_t *>(blob);
    if (dtype == kBF16) pack_linear_kernel<kBF16><<<grid, 256, 0, s>>>(wp, n, k, group, b);
    else pack_linear_kernel<kF16><<<grid, 256, 0, s>>>(wp, n, k, group, b);
    return hipGetLastError();
}

hipError_t launch_unpack_linear(const void *blob, int n, int k, int group, int8_t *codes, uint16_t *scales,
                                hipStream_t s) {
    const long long blocks = ((long long)n * (k / 8) + 255) / 256;
    unpack_linear_kernel<<<(unsigned)blocks, 256, 0, s>>>(static_cast<const uint8_t *>(blob), n, k, group, codes, scales);
    return hipGetLastError();
}

template <int DT, int NT, int MT>
static void launch_linear_t(const uint8_t *blob, int n, int k, int group, const uint16_t *x, int64_t ldx, int batch,
                            const uint16_t *bias, uint16_t *y, int64_t ldy, hipStream_t s) {
    const unsigned grid = (unsigned)((n + kLinearRows * NT - 1) / (kLinearRows * NT));
    const int threads = 64 * kLinearWaves;
    if (group == 32) linear_kernel<DT, NT, MT, 4><<<grid, threads, 0, s>>>(blob, n, k, group, x, ldx, batch, bias, y, ldy);
    else if (group == 64) linear_kernel<DT, NT, MT, 2><<<grid, threads, 0, s>>>(blob, n, k, group, x, ldx, batch, bias, y, ldy);
    else linear_kernel<DT, NT, MT, 1><<<grid, threads, 0, s>>>(blob, n, k, group, x, ldx, batch, bias, y, ldy);
}

hipError_t launch_linear(int dtype, const void *blob, int n, int k, int group, const void *x, int64_t ldx, int batch,
                         const void *bias, void *y, int64_t ldy, hipStream_t s) {
    auto *bl = static_cast<const uint8_t *>(blob);
    auto *xp = static_cast<const uint16_t *>(x);
    auto *bp = static_cast<const uint16_t *>(bias);
    auto *yp = static_cast<uint16_t *>(y);
#define LINEAR(NT_, MT_)                                                                                     \
    do {                                                                                                     \
        if (dtype == kBF16) launch_linear_t<kBF16, NT_, MT_>(bl, n, k, group, xp, ldx, batch, bp, yp, ldy, s); \
        else launch_linear_t<kF16, NT_, MT_>(bl, n, k, group, xp, ldx, batch, bp, yp, ldy, s);               \
    } while (0)
    if (batch <= 16) LINEAR(1, 1);
    else if (batch <= 32) LINEAR(2, 2);
    else LINEAR(2, 4);
#undef LINEAR
    return hipGetLastError();
}

}  // namespace prox
