// Rows in 8 bits: the norm and the activation that make them, and their inverse view.
//
// A row p is held as codes c_i = rne(127 p_i / A), A = max|p|, and a scale sigma = fp32(factor A / 127), and
// stands for sigma c.  The quotient decides, not its rounding: a code is the same in every run, and the one that
// 64 bits give.  In 32 bits 127 / A and its product with p are off by less than 127 * 3 * 2^-24, so only quotients
// that near to the middle of two codes (1 in 20000) are divided again in 64 bits, where p (24 bits at most) times
// 127 is exact and a true tie comes out as one.
//
// Each row is read once into registers, 8 elements (a chunk) a thread and step; one reduction over its threads
// gives all that the codes need, since the norm's 1 / rms cancels from 127 p / A.
#include "rows8.hpp"

namespace prox {

namespace {

constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23: adding it rounds to whole numbers, half to even
constexpr uint32_t kInf = 0x7F800000u;

// 8 elements of a row that may start at any element; past its end 0 (n: elements left, at least 1).
__device__ __forceinline__ uint4 load8(const uint16_t *p, int n) {
    uint4 v{0, 0, 0, 0};
    if (n >= 8) {
        __builtin_memcpy(&v, __builtin_assume_aligned(p, 2), 16);
    } else {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) w[e / 2] |= (uint32_t)p[e] << (16 * (e % 2));
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}
__device__ __forceinline__ void store8(uint16_t *p, int n, const uint32_t (&w)[4]) {
    if (n >= 8) {
        __builtin_memcpy(__builtin_assume_aligned(p, 2), w, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
    }
}
// Codes are the low bytes of t; rows of codes start on 16 bytes.
__device__ __forceinline__ void store_codes(int8_t *p, int n, const uint32_t (&t)[8]) {
    uint2 v;
    v.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[3], t[2], 0x0c0c0400u), __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u), 0x05040100u);
    v.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[7], t[6], 0x0c0c0400u), __builtin_amdgcn_perm(t[5], t[4], 0x0c0c0400u), 0x05040100u);
    if (n >= 8) {
        *reinterpret_cast<uint2 *>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = (int8_t)((e < 4 ? v.x : v.y) >> (8 * (e % 4)));
    }
}

template <int DT>
__device__ __forceinline__ float elem(const uint4 &v, int e) {   // e a constant
    const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
    return (e & 1) ? hi_to_float<DT>(w) : lo_to_float<DT>(w);
}
// Element e of a chunk, e not a constant.
template <int DT>
__device__ __forceinline__ float elem_at(const uint4 &v, int e) {
    const uint32_t a = e & 2 ? v.y : v.x, b = e & 2 ? v.w : v.z, w = e & 4 ? b : a;
    return half_to_float<DT>((uint16_t)(e & 1 ? w >> 16 : w));
}

// Two values rounded to the dtype (NaN stays NaN).
template <int DT>
__device__ __forceinline__ uint32_t round_pair(float a, float b) {
    if constexpr (DT == kBF16) {
        const bf16x2 v{(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        const f16x2 v{(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
}

__device__ __forceinline__ double dpp_swap(double v, int step) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const int lo = __shfl_xor((int)(uint32_t)u, step), hi = __shfl_xor((int)(uint32_t)(u >> 32), step);
    return __longlong_as_double((long long)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo));
}

// Reductions over the T threads of a row, the same bits in each of them.  T = 64: a wave by itself.
template <int T>
struct RowReduce {
    struct Part {
        double sum;
        uint32_t top;
    };
    __device__ __forceinline__ void operator()(double &sum, uint32_t &top, Part *lds) const {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            sum += dpp_swap(sum, m);
            top = max(top, (uint32_t)__shfl_xor((int)top, m));
        }
        if constexpr (T > 64) {
            __syncthreads();   // an earlier use of lds is over
            if (lane_id() == 0) lds[threadIdx.x / kWave] = Part{sum, top};
            __syncthreads();
            sum = 0.0, top = 0;
#pragma unroll
            for (int w = 0; w < T / 64; ++w) {
                sum += lds[w].sum;
                top = max(top, lds[w].top);
            }
        }
    }
    // The largest of non-negative doubles (bits order like the values).
    __device__ __forceinline__ double largest(double v, Part *lds) const {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) v = fmax(v, dpp_swap(v, m));
        if constexpr (T > 64) {
            __syncthreads();
            if (lane_id() == 0) lds[threadIdx.x / kWave].sum = v;
            __syncthreads();
            v = 0.0;
#pragma unroll
            for (int w = 0; w < T / 64; ++w) v = fmax(v, lds[w].sum);
        }
        return v;
    }
};

// rne(127 p / top) in 64 bits.
__device__ __forceinline__ uint32_t exact_code(double p, double top) { return (uint32_t)(int)rint(p * 127.0 / top); }

__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7FC00000u); }

// T threads a row, CH chunks a thread.
template <int DT, int T, int CH>
__global__ __launch_bounds__(T == 64 ? 256 : T) void rmsnorm_kernel(NormArgs A) {
    using Reduce = RowReduce<T>;
    __shared__ typename Reduce::Part lds[T / 64];
    const Reduce reduce;
    const int row = T == 64 ? (int)blockIdx.x * 4 + (int)threadIdx.x / 64 : (int)blockIdx.x;
    const int t = T == 64 ? lane_id() : (int)threadIdx.x;
    if (T == 64 && row >= A.rows) return;   // whole waves, which share nothing
    const int d = A.d;
    uint4 r[CH], g[CH];
    uint32_t top = 0;
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = (c * T + t) * 8, n = d - i;
        r[c] = g[c] = make_uint4(0, 0, 0, 0);
        if (n > 0) {
            r[c] = load8(A.x + (size_t)row * A.ldx + i, n);
            if (A.gain) g[c] = load8(A.gain + i, n);
        }
    }
    if (A.y) {   // the sum is rounded to the dtype: the norm is of the residual as it is kept
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int i = (c * T + t) * 8, n = d - i;
            if (n <= 0) continue;
            const uint4 y = load8(A.y + (size_t)row * A.ldy + i, n);
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = round_pair<DT>(elem<DT>(r[c], 2 * q) + elem<DT>(y, 2 * q), elem<DT>(r[c], 2 * q + 1) + elem<DT>(y, 2 * q + 1));
            r[c] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = (c * T + t) * 8, n = d - i;
        if (n <= 0) continue;
        if (A.r) store8(A.r + (size_t)row * A.ldr + i, n, {r[c].x, r[c].y, r[c].z, r[c].w});
        if (!A.gain) {
            const uint32_t one = DT == kBF16 ? 0x3F803F80u : 0x3C003C00u;
            g[c] = make_uint4(one, one, one, one);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = elem<DT>(r[c], e);
            sum = fma((double)v, (double)v, sum);   // bf16 squares leave 32 bits
            top = max(top, __float_as_uint(v * elem<DT>(g[c], e)) & 0x7FFFFFFFu);   // NaN above all
        }
    }
    reduce(sum, top, lds);
    const double mean = sum / (double)d + (double)A.eps;
    const double inv = mean > 0.0 ? 1.0 / sqrt(mean) : 0.0;   // a row of zeros and eps 0: zeros
    const float topf = __uint_as_float(top), invf = (float)inv;
    // Products and 1 / rms well inside 32 bits, everything finite.
    const bool plain = topf >= 0x1p-60f && topf <= 0x1p100f && invf >= 0x1p-100f && invf <= 0x1p60f && sum < 1e300;
    if (plain) {
        const float s = 127.0f / topf;
        if (t == 0 && A.codes) A.scales[row] = (float)((double)topf * inv / 127.0);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int i = (c * T + t) * 8, n = d - i;
            if (n <= 0) continue;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = elem<DT>(r[c], e) * elem<DT>(g[c], e);   // exact
            if (A.out) {
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] = round_pair<DT>(p[2 * q] * invf, p[2 * q + 1] * invf);
                store8(A.out + (size_t)row * A.ldo + i, n, w);
            }
            if (A.codes) {
                uint32_t code[8];
                float far = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float m = fmaf(p[e], s, kMagic);
                    far = fmaxf(far, fabsf(fmaf(p[e], s, kMagic - m)));
                    code[e] = __float_as_uint(m);
                }
                if (far > 0.49997f) {   // 127 * 3 * 2^-24 from the middle
#pragma unroll 1
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t k = exact_code((double)(elem_at<DT>(r[c], e) * elem_at<DT>(g[c], e)), (double)topf);
#pragma unroll
                        for (int f = 0; f < 8; ++f) code[f] = f == e ? k : code[f];
                    }
                }
                store_codes(A.codes + (size_t)row * A.ldc + i, n, code);
            }
        }
        return;
    }
    // Rows at the ends of the range or not finite, in 64 bits.
    double most = 0.0, bad = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if ((c * T + t) * 8 >= d) continue;
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const double p = (double)elem_at<DT>(r[c], e) * (double)elem_at<DT>(g[c], e);
            if (!(fabs(p) < INFINITY)) bad = 1.0;
            most = fmax(most, fabs(p));
        }
    }
    most = reduce.largest(most, lds);
    bad = reduce.largest(bad, lds);
    const bool finite = bad == 0.0 && sum < INFINITY;
    if (t == 0 && A.codes) A.scales[row] = finite ? (float)(most * inv / 127.0) : quiet_nan();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = (c * T + t) * 8, n = d - i;
        if (n <= 0) continue;
        uint32_t code[8];
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double p = (double)elem<DT>(r[c], e) * (double)elem<DT>(g[c], e);
            o[e] = (float)(p * inv);
            code[e] = finite && most > 0.0 ? exact_code(p, most) : 0u;
        }
        if (A.out) {
            const uint32_t w[4] = {round_pair<DT>(o[0], o[1]), round_pair<DT>(o[2], o[3]), round_pair<DT>(o[4], o[5]), round_pair<DT>(o[6], o[7])};
            store8(A.out + (size_t)row * A.ldo + i, n, w);
        }
        if (A.codes) store_codes(A.codes + (size_t)row * A.ldc + i, n, code);
    }
}

// What is quantised, in 64 bits and rounded to 32.
template <int ACT>
__device__ __forceinline__ float exact_act(float g, float u) {
    const double z = g;
    if constexpr (ACT == kActSilu) return (float)((double)u * (z / (1.0 + exp(-z))));
    else if constexpr (ACT == kActGelu) return (float)((double)u * (0.5 * z * erfc(z * -0.70710678118654752440)));
    else return g;
}

template <int DT, int T, int CH, int ACT>
__global__ __launch_bounds__(T == 64 ? 256 : T) void quant_kernel(QuantArgs A) {
    using Reduce = RowReduce<T>;
    __shared__ typename Reduce::Part lds[T / 64];
    const Reduce reduce;
    const int row = T == 64 ? (int)blockIdx.x * 4 + (int)threadIdx.x / 64 : (int)blockIdx.x;
    const int t = T == 64 ? lane_id() : (int)threadIdx.x;
    if (T == 64 && row >= A.rows) return;
    const int d = A.d;
    double most = 0.0, bad = 0.0;
    auto value = [&](int c, float (&v)[8]) {
        const int i = (c * T + t) * 8, n = d - i;
        const uint4 g = load8(A.x + (size_t)row * A.ldx + i, n);
        uint4 u = g;
        if constexpr (ACT != kActNone) u = load8(A.up + (size_t)row * A.ldu + i, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = exact_act<ACT>(elem<DT>(g, e), elem<DT>(u, e));
    };
    for (int c = 0; c < CH; ++c) {
        if ((c * T + t) * 8 >= d) continue;
        float v[8];
        value(c, v);
        for (int e = 0; e < 8; ++e) {
            if (!(fabsf(v[e]) < INFINITY)) bad = 1.0;
            most = fmax(most, (double)fabsf(v[e]));
        }
    }
    most = reduce.largest(most, lds);
    bad = reduce.largest(bad, lds);
    if (t == 0) A.scales[row] = bad == 0.0 ? (float)(most / 127.0) : quiet_nan();
    for (int c = 0; c < CH; ++c) {
        const int i = (c * T + t) * 8, n = d - i;
        if (n <= 0) continue;
        float v[8];
        value(c, v);
        uint32_t code[8];
        for (int e = 0; e < 8; ++e) code[e] = bad == 0.0 && most > 0.0 ? exact_code((double)v[e], most) : 0u;
        store_codes(A.codes + (size_t)row * A.ldc + i, n, code);
    }
}

// sigma c of four codes a thread.
__global__ __launch_bounds__(256) void read_q8_kernel(const int8_t *__restrict__ codes, int64_t ldc, const float *__restrict__ scales,
                                                      int rows, int d, float *__restrict__ out) {
    const int per = (d + 3) / 4;
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < (long long)rows * per; id += (long long)gridDim.x * 256) {
        const int row = (int)(id / per), i = (int)(id % per) * 4;
        const float s = scales[row];
        for (int e = i; e < min(i + 4, d); ++e) out[(size_t)row * d + e] = s * (float)codes[(size_t)row * ldc + e];
    }
}

// Threads a row and chunks a thread.
template <typename F>
hipError_t by_width(int d, F f) {
    const int chunks = (d + 7) / 8;
    if (chunks <= 64) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (chunks <= 256) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (chunks <= 1024) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
    if (chunks <= 4096) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 8>{});
}

template <int DT, int ACT>
hipError_t quant_act(const QuantArgs &a, hipStream_t s) {
    return by_width(a.d, [&](auto t, auto ch) {
        constexpr int T = decltype(t)::value, CH = decltype(ch)::value;
        quant_kernel<DT, T, CH, ACT><<<T == 64 ? (a.rows + 3) / 4 : a.rows, T == 64 ? 256 : T, 0, s>>>(a);
        return hipGetLastError();
    });
}

template <int DT>
hipError_t quant_dt(const QuantArgs &a, hipStream_t s) {
    if (!a.up) return quant_act<DT, kActNone>(a, s);
    return a.act == 0 ? quant_act<DT, kActSilu>(a, s) : quant_act<DT, kActGelu>(a, s);
}

template <int DT>
hipError_t norm_dt(const NormArgs &a, hipStream_t s) {
    return by_width(a.d, [&](auto t, auto ch) {
        constexpr int T = decltype(t)::value, CH = decltype(ch)::value;
        rmsnorm_kernel<DT, T, CH><<<T == 64 ? (a.rows + 3) / 4 : a.rows, T == 64 ? 256 : T, 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_rmsnorm_q8(int dtype, const NormArgs &a, hipStream_t s) {
    return dtype == kBF16 ? norm_dt<kBF16>(a, s) : norm_dt<kF16>(a, s);
}

hipError_t launch_quant_q8(int dtype, const QuantArgs &a, hipStream_t s) {
    return dtype == kBF16 ? quant_dt<kBF16>(a, s) : quant_dt<kF16>(a, s);
}

hipError_t launch_read_q8(const int8_t *codes, int64_t ldc, const float *scales, int rows, int d, float *out, hipStream_t s) {
    const long long blocks = ((long long)rows * ((d + 3) / 4) + 255) / 256;
    read_q8_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(codes, ldc, scales, rows, d, out);
    return hipGetLastError();
}

}  // namespace prox
