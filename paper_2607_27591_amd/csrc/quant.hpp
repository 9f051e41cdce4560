// The symmetric quantiser of proxies, INT4 weights and the 4-bit key/value cache
// (Sec. 4.3): one fp16 scale per group, codes rounded half to even.
#pragma once

#include "common.hpp"

namespace prox {

// IEEE binary16 round-to-nearest-even of a binary64 value, from the bit
// fields of the double.
__device__ inline uint16_t f64_to_f16_rne(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint16_t sign = (uint16_t)((u >> 48) & 0x8000u);
    const uint64_t a = u & 0x7FFFFFFFFFFFFFFFull;
    if (a >= 0x7FF0000000000000ull) return sign | (a > 0x7FF0000000000000ull ? 0x7E00 : 0x7C00);
    if (a < 0x0010000000000000ull) return sign;   // below 2^-1022: rounds to zero
    const int e = (int)(a >> 52) - 1023;
    if (e > 15) return sign | 0x7C00;
    const uint64_t m = (a & 0x000FFFFFFFFFFFFFull) | 0x0010000000000000ull;  // 53 bits
    // Normal results keep 11 significant bits; subnormal ones count 2^-24 units.
    const int shift = e >= -14 ? 42 : 28 - e;
    if (shift > 62) return sign;
    uint64_t keep = m >> shift;
    const uint64_t rem = m & ((1ull << shift) - 1);
    const uint64_t half = 1ull << (shift - 1);
    if (rem > half || (rem == half && (keep & 1))) ++keep;
    if (e >= -14) {
        int E = e;
        if (keep == 2048) { keep = 1024; ++E; }
        if (E > 15) return sign | 0x7C00;
        return sign | (uint16_t)((E + 15) << 10) | (uint16_t)(keep - 1024);
    }
    return sign | (uint16_t)keep;   // 1024 encodes the smallest normal
}

template <int DT>
__device__ __forceinline__ double w_to_f64(uint16_t h) { return (double)half_to_float<DT>(h); }

// Symmetric quantisation of one group: sigma = fp16_rne(amax / qmax) from the
// largest magnitude pattern (15 bits, ordered like the magnitudes).
struct GroupScale {
    float sigma, inv;   // sigma and 1 / sigma (0 when sigma is 0)
    uint16_t bits;
};
template <int DT>
__device__ __forceinline__ GroupScale group_scale(uint32_t amax_bits, int qmax) {
    GroupScale s;
    s.bits = f64_to_f16_rne(w_to_f64<DT>((uint16_t)amax_bits) / (double)qmax);
    s.sigma = f16_bits_to_float(s.bits);
    s.inv = s.sigma != 0.0f ? 1.0f / s.sigma : 0.0f;
    return s;
}

// clamp(round_half_even(w / sigma), -qmax, qmax), exactly as the fp64 quotient
// rounds.  w inv is within 2^-22 |w / sigma| of it, under 1e-4 for every
// quotient that occurs (at most 1.5 * 127, where sigma is subnormal), so the two
// round alike unless w inv lies within 1e-4 of a half: those (about 1 in 5000)
// take the fp64 division.
template <int DT>
__device__ __forceinline__ int quantise(uint32_t wbits, float sigma, float inv, float qmax) {
    const float w = half_to_float<DT>((uint16_t)wbits);
    const float r = w * inv;
    float n = rintf(r);
    if (fabsf(r - n) > 0.4999f) n = (float)rint((double)w / (double)sigma);
    return (int)fminf(fmaxf(n, -qmax), qmax);
}

// The largest finite-ordered magnitude pattern of 8 packed 16-bit floats (NaN
// patterns count as 0).
template <int DT>
__device__ __forceinline__ uint32_t abs_max8(const uint4 &v) {
    constexpr uint32_t inf = DT == kBF16 ? 0x7F80u : 0x7C00u;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t lo = w[q] & 0x7FFFu, hi = (w[q] >> 16) & 0x7FFFu;
        m = max(m, lo <= inf ? lo : 0u);
        m = max(m, hi <= inf ? hi : 0u);
    }
    return m;
}

// Maximum over each 16-lane row, in every lane of the row.
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor1, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor2, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppRor4, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppRor8, 0xF, 0xF, false));
    return v;
}

__device__ __forceinline__ uint32_t half_of(const uint4 &v, int e) {   // e a constant
    const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
    return (e & 1) ? w >> 16 : w & 0xFFFFu;
}

}  // namespace prox
