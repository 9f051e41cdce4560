// INT4 weights of projections: packing and its inverse view, and the entry of linear.hpp.
#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace prox {

// Packing: a workgroup takes the 16 rows of a tile over one unit of inputs (a group,
// at least 128), 16 lanes a row, so that it writes whole blocks of 1024 bytes.  A unit of
// 128 is read once, a longer group twice.  Bound by HBM (weights read once):
// 28672 x 8192, group 128, 246 us (590 MB, 2.4 TB/s).
template <int DT>
__global__ __launch_bounds__(256) void pack_linear_kernel(const uint16_t *__restrict__ w, int n, int k,
                                                          int group, uint8_t *__restrict__ blob) {
    const LinearLayout L(n, k, group);
    const int tile = blockIdx.x, l = threadIdx.x % 16, r = threadIdx.x / 16;
    const int unit = group > kLinearBlock ? group : kLinearBlock;
    const int first = (int)blockIdx.y * unit;
    const int j = tile * kLinearRows + r;
    const uint16_t *src = w + (size_t)j * k;
    uint16_t *scales = reinterpret_cast<uint16_t *>(blob + L.scales);
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
    if (l % span == 0) scales[L.scale_at(tile, g, r)] = s.bits;   // of zeros past n and k: 0
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

// Inverse view: a thread takes (row, 8 inputs) items, a grid apart.
__global__ __launch_bounds__(256) void unpack_linear_kernel(const uint8_t *__restrict__ blob, int n, int k,
                                                            int group, int8_t *__restrict__ codes,
                                                            uint16_t *__restrict__ scales) {
    const LinearLayout L(n, k, group);
    const int per = k / 8;
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < (long long)n * per;
         id += (long long)gridDim.x * 256) {
        const int j = (int)(id / per), ch = (int)(id % per);
        const int c = ch % 16;   // chunk of the block
        const size_t blk = (size_t)(j / kLinearRows) * L.blocks + ch / 16;
        const uint32_t word = *reinterpret_cast<const uint32_t *>(
            blob + blk * 1024 + (size_t)((c % 4) * 16 + j % kLinearRows) * 16 + (c / 4) * 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) codes[id * 8 + e] = (int8_t)((int)((word >> (4 * nibble_of(e))) & 15) - 8);
        const int g = ch * 8 / group;
        if (ch * 8 % group == 0)
            scales[(size_t)j * L.groups + g] =
                reinterpret_cast<const uint16_t *>(blob + L.scales)[L.scale_at(j / kLinearRows, g, j % kLinearRows)];
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
    unpack_linear_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(
        static_cast<const uint8_t *>(blob), n, k, group, codes, scales);
    return hipGetLastError();
}


hipError_t launch_linear(int dtype, const void *blob, int n, int k, int group, const void *x, int64_t ldx, int batch,
                         const void *bias, void *y, int64_t ldy, hipStream_t s) {
    const uint32_t per = (uint32_t)(group < kLinearBlock ? 1 : group / kLinearBlock);   // blocks of a group
    const LinearArgs a{static_cast<const uint8_t *>(blob), n, k, group, static_cast<const uint16_t *>(x), ldx, batch,
                       static_cast<const uint16_t *>(bias), static_cast<uint16_t *>(y), ldy, ((1u << 20) + per - 1) / per};
    return dtype == kBF16 ? launch_linear_bf16(a, s) : launch_linear_f16(a, s);
}

}  // namespace prox
