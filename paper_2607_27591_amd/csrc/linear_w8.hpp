// Arguments of the projection on 8-bit integers.
#pragma once

#include "common.hpp"

namespace prox {

struct Linear8Args {
    const uint8_t *codes;   // of the weights (Linear8Layout), and their scales
    const float *sw;
    int n, k, kblocks;
    const int8_t *x;        // [rows][ldx]
    const float *scales;    // [rows]
    int64_t ldx;
    int rows;
    const uint16_t *bias;   // or NULL
    uint16_t *y;
    int64_t ldy;
};
hipError_t launch_pack_linear_w8(int dtype, const void *w, int n, int k, void *blob, hipStream_t s);
hipError_t launch_unpack_linear_w8(const void *blob, int n, int k, int8_t *codes, float *scales, hipStream_t s);
bool linear_w8_fits(int rows, int n);   // its tiles, the largest at the least, in one grid
hipError_t launch_linear_w8(int dtype, const Linear8Args &a, hipStream_t s);

}  // namespace prox
