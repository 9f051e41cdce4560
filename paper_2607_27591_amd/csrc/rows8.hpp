// Arguments of the kernels on rows in 8 bits.
#pragma once

#include <type_traits>

#include "common.hpp"

namespace prox {

enum { kActSilu = 0, kActGelu = 1 };

struct NormArgs {
    const uint16_t *x, *y, *gain;   // y, gain may be NULL
    uint16_t *r, *out;              // may be NULL
    int8_t *codes;                  // NULL: no codes, no scales
    float *scales;
    int64_t ldx, ldy, ldr, ldo, ldc;
    int rows, d;
    float eps;
    double inv_d;   // 1 / d
};
struct QuantArgs {
    const uint16_t *x, *up;   // up NULL: codes of x
    int8_t *codes;
    float *scales;
    int64_t ldx, ldu, ldc;
    int rows, d, act;
};
hipError_t launch_rmsnorm_q8(int dtype, const NormArgs &a, hipStream_t s);
hipError_t launch_quant_q8(int dtype, const QuantArgs &a, hipStream_t s);
hipError_t launch_read_q8(const int8_t *codes, int64_t ldc, const float *scales, int rows, int d, float *out, hipStream_t s);

}  // namespace prox
