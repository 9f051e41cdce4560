// Projections on 8-bit integers, y = (c_x c_w^T) sigma_x sigma_w (+ bias): weights packed and unpacked, and
// the product.
#include "linear_w8.hpp"

namespace prox {

namespace {

template <int DT>
__device__ __forceinline__ uint16_t to_half(float v) {   // NaN stays NaN
    if constexpr (DT == kBF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return float_to_f16_rne(v);
}

// Packing: a workgroup takes the 16 outputs of a tile, 16 lanes each, and reads them twice (the second time
// from the L2), so that it writes whole runs of 1024 bytes.
template <int DT>
__global__ __launch_bounds__(256) void pack_w8_kernel(const uint16_t *__restrict__ w, int n, int k, uint8_t *__restrict__ blob) {
    const Linear8Layout L(n, k);
    const int nb = blockIdx.x / 4, tile = blockIdx.x % 4, l = threadIdx.x % 16, r = threadIdx.x / 16;
    const int j = nb * kLinear8N + w8_output(tile, r);
    const uint16_t *src = w + (size_t)j * k;
    const int kk = j < n ? k : 0;
    double most = 0.0;
    int bad = 0;
    for (int i = l; i < kk; i += 16) {
        const float v = fabsf(half_to_float<DT>(src[i]));
        if (!(v < INFINITY)) bad = 1;
        most = fmax(most, (double)v);
    }
    for (int m = 1; m < 16; m <<= 1) {
        most = fmax(most, __shfl_xor(most, m));
        bad |= __shfl_xor(bad, m);
    }
    if (l == 0)
        reinterpret_cast<float *>(blob + L.scales)[j] = bad ? __uint_as_float(0x7FC00000u) : (float)(most / 127.0);
    const bool zero = bad || most == 0.0;
    for (int c = l; c < 4 * L.kblocks; c += 16) {   // chunks of 16 inputs
        uint32_t word[4] = {0, 0, 0, 0};
        for (int e = 0; e < 16; ++e) {
            const int i = 16 * c + e;
            const int code = i < kk && !zero ? (int)rint((double)half_to_float<DT>(src[i]) * 127.0 / most) : 0;
            word[e / 4] |= (uint32_t)(code & 0xFF) << (8 * (e % 4));
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

// A wave takes 64 outputs of 16 rows over all inputs.
template <int DT>
__global__ __launch_bounds__(256) void linear_w8_kernel(Linear8Args A) {
    const Linear8Layout L(A.n, A.k);
    const int wave = threadIdx.x / kWave, lane = lane_id(), h = lane / 16, col = lane % 16;
    const int groups = (L.nblocks + 3) / 4;
    const int nb = (int)(blockIdx.x % groups) * 4 + wave, row = (int)(blockIdx.x / groups) * 16 + col;
    if (nb >= L.nblocks) return;
    const int8_t *x = A.x + (size_t)min(row, A.rows - 1) * A.ldx;
    const uint8_t *w = A.blob + (size_t)nb * L.kblocks * 4096 + lane * 16;
    v4i acc[4] = {};
    for (int b = 0; b < L.kblocks; ++b) {
        const int i = 64 * b + 16 * h;
        v4i xv = {0, 0, 0, 0};
        if (i < A.k) xv = *reinterpret_cast<const v4i *>(x + i);   // up to 15 bytes past k, times codes 0
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = mfma16_i8(*reinterpret_cast<const v4i *>(w + (size_t)b * 4096 + t * 1024), xv, acc[t]);
    }
    if (row >= A.rows) return;
    const float *ws = reinterpret_cast<const float *>(A.blob + L.scales);
    const float xs = A.scales[row];
    for (int t = 0; t < 4; ++t)
        for (int e = 0; e < 4; ++e) {
            const int j = nb * kLinear8N + w8_output(t, 4 * h + e);
            if (j < A.n)
                A.y[(size_t)row * A.ldy + j] = to_half<DT>(fmaf((float)acc[t][e] * ws[j], xs, A.bias ? half_to_float<DT>(A.bias[j]) : 0.0f));
        }
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

hipError_t launch_linear_w8(int dtype, const Linear8Args &a, hipStream_t s) {
    const Linear8Layout L(a.n, a.k);
    const unsigned grid = (unsigned)((L.nblocks + 3) / 4) * (unsigned)((a.rows + 15) / 16);
    if (dtype == kBF16) linear_w8_kernel<kBF16><<<grid, 256, 0, s>>>(a);
    else linear_w8_kernel<kF16><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace prox
