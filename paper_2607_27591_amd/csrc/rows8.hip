// Rows in 8 bits: the norm and the activation that make them, and their inverse view.
//
// A row p is held as codes c_i = rne(127 p_i / A), A = max|p|, and a scale sigma = fp32(factor A / 127), and
// stands for sigma c.  The quotient decides, not its rounding: a code is the same in every run, and the one that
// 64 bits give.  In 32 bits 127 / A and its product with p are off by less than 127 * 3 * 2^-24, so only quotients
// that near to the middle of two codes (1 in 20000) are divided again in 64 bits, where p (24 bits at most) times
// 127 is exact and a true tie comes out as one.
//
// Each row is read once into registers, 8 elements (a chunk) a thread and step; one reduction over its threads
// gives all that the codes need, since the norm's 1 / rms cancels from 127 p / A.  Bound by HBM.  (The norm of more than
// 32768 values a row keeps 17 to 63 registers a lane in scratch.)
#include "rows8.hpp"

namespace prox {

namespace {

constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23: adding it rounds to whole numbers, half to even

// f(0), .. f(N - 1), each with a constant of its own.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// 8 elements of a row that may start at any element; n of them (at least 1) where the row ends there (TAIL), else 0.
template <bool TAIL>
__device__ __forceinline__ uint4 load8(const uint16_t *p, int n) {
    uint4 v{0, 0, 0, 0};
    if (!TAIL || n >= 8) {
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
// STREAM: past the caches' usual order, for what the next kernel does not read (the residual: norm of 2048 x 8192
// 20.9 us, else 26.8; codes so would cost the projection behind them more than the norm gains).
template <bool TAIL, bool STREAM>
__device__ __forceinline__ void store8(uint16_t *p, int n, const uint4 &v) {
    if (!TAIL || n >= 8) {
        const u32x4_any w{v.x, v.y, v.z, v.w};
        if constexpr (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_any *>(p));
        else *reinterpret_cast<u32x4_any *>(p) = w;
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
    }
}
// Rows of codes start on 16 bytes.
template <bool TAIL>
__device__ __forceinline__ void store_codes(int8_t *p, int n, const uint2 &v) {
    if (!TAIL || n >= 8) {
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
__device__ __forceinline__ void set_code(uint2 &v, int e, uint32_t code) {
    const int s = 8 * (e & 3);
    const uint32_t m = 0xFFu << s, k = (code & 0xFFu) << s;
    if (e < 4) v.x = (v.x & ~m) | k;
    else v.y = (v.y & ~m) | k;
}

// Moves on the VALU, lane ^ 1, 2 and, among 16 and 64 lanes, rotations that pair the halves.
template <int STEP>
__device__ __forceinline__ uint32_t peer(uint32_t v) {
    if constexpr (STEP == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor1, 0xF, 0xF, false);
    else if constexpr (STEP == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor2, 0xF, 0xF, false);
    else if constexpr (STEP == 4) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppRor4, 0xF, 0xF, false);
    else return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppRor8, 0xF, 0xF, false);
}
template <int STEP>
__device__ __forceinline__ double peer(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = peer<STEP>((uint32_t)u), hi = peer<STEP>((uint32_t)(u >> 32));
    return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
// Both halves of a pair of lanes 16 or 32 apart.
template <int STEP>
__device__ __forceinline__ void both(uint32_t v, uint32_t &a, uint32_t &b) {
    if constexpr (STEP == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        a = r[0], b = r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        a = r[0], b = r[1];
    }
}
template <int STEP>
__device__ __forceinline__ void both(double v, double &a, double &b) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    uint32_t l0, l1, h0, h1;
    both<STEP>((uint32_t)u, l0, l1);
    both<STEP>((uint32_t)(u >> 32), h0, h1);
    a = __longlong_as_double((long long)(((uint64_t)h0 << 32) | l0));
    b = __longlong_as_double((long long)(((uint64_t)h1 << 32) | l1));
}
// f symmetric: the same bits in every lane, since every step joins pairs of lanes that see each other.  A rotation by 4
// of 16 lanes does so once lanes 8 apart agree, so after that by 8 (before it, sums in 64 bits differ between quads).
template <typename V, typename F>
__device__ __forceinline__ V wave_join(V v, F f) {
    v = f(v, peer<1>(v));
    v = f(v, peer<2>(v));
    v = f(v, peer<8>(v));
    v = f(v, peer<4>(v));
    V a, b;
    both<16>(v, a, b);
    v = f(a, b);
    both<32>(v, a, b);
    return f(a, b);
}

// A value joined over the T threads of a row, the same in each of them.  T = 64: a wave by itself.  AGAIN: lds has
// been used before.
template <int T, bool AGAIN, typename V, typename F>
__device__ __forceinline__ V row_join(V v, V *lds, F f) {
    v = wave_join(v, f);
    if constexpr (T > 64) {
        if constexpr (AGAIN) __syncthreads();
        if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < T / 64; ++w) v = f(v, lds[w]);
    }
    return v;
}
// Two of them behind one barrier.
template <int T, typename V, typename F, typename W, typename G>
__device__ __forceinline__ void row_join2(V &v, V *lds, F f, W &u, W *lds2, G g) {
    v = wave_join(v, f);
    u = wave_join(u, g);
    if constexpr (T > 64) {
        if (lane_id() == 0) lds[threadIdx.x / kWave] = v, lds2[threadIdx.x / kWave] = u;
        __syncthreads();
        v = lds[0], u = lds2[0];
#pragma unroll
        for (int w = 1; w < T / 64; ++w) v = f(v, lds[w]), u = g(u, lds2[w]);
    }
}
struct Add {
    __device__ __forceinline__ double operator()(double a, double b) const { return a + b; }
};
struct Most {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); }
    __device__ __forceinline__ double operator()(double a, double b) const { return fmax(a, b); }
};

// rne(127 p / top) in 64 bits.
__device__ __forceinline__ uint32_t exact_code(double p, double top) { return (uint32_t)(int)rint(p * 127.0 / top); }

// The codes of 8 values, s = 127 / A, and which of them are too near to the middle of two codes to be told in
// 32 bits: off by at most |c| rel + 3e-5.
__device__ __forceinline__ uint2 fast_codes(const float (&p)[8], float s, uint32_t &near, float rel) {
    uint32_t c[8];
    float far[8], most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float m = fmaf(p[e], s, kMagic), whole = m - kMagic;
        far[e] = fmaf(fabsf(whole), rel, fabsf(fmaf(p[e], s, -whole)));
        most = fmaxf(most, far[e]);
        c[e] = __float_as_uint(m);
    }
    near = 0;
    if (most > 0.49997f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) near |= far[e] > 0.49997f ? 1u << e : 0u;
    }
    auto four = [&](int e) {
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[e + 3], c[e + 2], 0x0c0c0400u), __builtin_amdgcn_perm(c[e + 1], c[e], 0x0c0c0400u), 0x05040100u);
    };
    return make_uint2(four(0), four(4));
}

__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7FC00000u); }

// How rows are cut: T threads a row, CH chunks a thread.  64 threads: a row a wave, 4 a workgroup.
template <int T_, int CH_>
struct Cut {
    static constexpr int T = T_, CH = CH_, threads = T == 64 ? 256 : T;
    static constexpr bool wave = T == 64;
};

// TAIL: d is no multiple of 8.
template <int DT, class C, bool TAIL>
__global__ __launch_bounds__(C::threads) void rmsnorm_kernel(NormArgs A) {
    constexpr bool WAVE = C::wave;
    constexpr int T = C::T, CH = C::CH;
    __shared__ double sums[T / 64];
    __shared__ uint32_t tops[T / 64];
    const int row = WAVE ? (int)blockIdx.x * 4 + (int)threadIdx.x / 64 : (int)blockIdx.x;
    const int t = WAVE ? lane_id() : (int)threadIdx.x;
    if (WAVE && row >= A.rows) return;   // whole waves, which share nothing
    const int d = A.d;
    const uint16_t *x = A.x + (size_t)row * A.ldx, *y = A.y + (size_t)row * A.ldy;
    uint4 r[CH], g[CH];
    uint32_t top = 0;
    double sum = 0.0;
    each<CH>([&](auto c) {
        const int i = (c * T + t) * 8, n = d - i;
        r[c] = g[c] = make_uint4(0, 0, 0, 0);
        if (n > 0) {
            r[c] = load8<TAIL>(x + i, n);
            if (A.gain) g[c] = load8<TAIL>(A.gain + i, n);
        }
    });
    if (A.y) {   // the sum is rounded to the dtype: the norm is of the residual as it is kept
        uint4 v[CH];
        each<CH>([&](auto c) {
            const int i = (c * T + t) * 8, n = d - i;
            v[c] = make_uint4(0, 0, 0, 0);
            if (n > 0) v[c] = load8<TAIL>(y + i, n);
        });
        each<CH>([&](auto c) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = round_pair<DT>(elem<DT>(r[c], 2 * q) + elem<DT>(v[c], 2 * q), elem<DT>(r[c], 2 * q + 1) + elem<DT>(v[c], 2 * q + 1));
            r[c] = make_uint4(w[0], w[1], w[2], w[3]);
        });
    }
    if (A.r) {
        each<CH>([&](auto c) {
            const int i = (c * T + t) * 8, n = d - i;
            if (n > 0) store8<TAIL, true>(A.r + (size_t)row * A.ldr + i, n, r[c]);
        });
    }
    each<CH>([&](auto c) {
        if (!A.gain) {
            const uint32_t one = DT == kBF16 ? 0x3F803F80u : 0x3C003C00u;
            g[c] = make_uint4(one, one, one, one);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = elem<DT>(r[c], e);
            sum = fma((double)v, (double)v, sum);   // in 64 bits: squares of bf16 leave 32
            top = max(top, __float_as_uint(v * elem<DT>(g[c], e)) & 0x7FFFFFFFu);   // NaN above all
        }
    });
    row_join2<T>(sum, sums, Add(), top, tops, Most());
    const double mean = fma(sum, A.inv_d, (double)A.eps);
    const float topf = __uint_as_float(top);
    // Products and 1 / rms well inside 32 bits, everything finite.  Products below 2^-126 lose bits: 2^-150, which a 1 / rms of
    // 2^12 at most (any with eps from 6e-8) leaves far below the smallest step of the dtype.
    // Rows of a smaller rms go the 64-bit way (2048 x 8192 of rms 1e-5, eps 0: 47 us, else 21); a power of 2 of 1 / rms multiplied in
    // first keeps them here, but takes 1 to 3% of every call with a 16-bit output.
    if (topf >= 0x1p-60f && topf <= 0x1p100f && mean >= 0x1p-24 && mean <= 0x1p110) {
        // 1 / sqrt(mean) to about 2^-50: 32 bits, and two terms of the series of what is left.
        const double y0 = (double)__builtin_amdgcn_rsqf((float)mean), left = fma(-mean * y0, y0, 1.0);
        const double inv = fma(y0 * left, fma(left, 0.375, 0.5), y0);
        const float s = 127.0f / topf, invf = (float)inv;
        if (t == 0 && A.codes) A.scales[row] = (float)((double)topf * inv * (1.0 / 127.0));
        each<CH>([&](auto c) {
            const int i = (c * T + t) * 8, n = d - i;
            if (n <= 0) return;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = elem<DT>(r[c], e) * elem<DT>(g[c], e);   // 22 bits at most: exact from 2^-126 on
            if (A.out) {
                const uint4 w = make_uint4(round_pair<DT>(p[0] * invf, p[1] * invf), round_pair<DT>(p[2] * invf, p[3] * invf),
                                           round_pair<DT>(p[4] * invf, p[5] * invf), round_pair<DT>(p[6] * invf, p[7] * invf));
                store8<TAIL, false>(A.out + (size_t)row * A.ldo + i, n, w);
            }
            if (A.codes) {
                uint32_t near;
                uint2 code = fast_codes(p, s, near, 0.0f);
                for (; near; near &= near - 1) {
                    const int e = __builtin_ctz(near);
                    set_code(code, e, exact_code((double)(elem_at<DT>(r[c], e) * elem_at<DT>(g[c], e)), (double)topf));
                }
                store_codes<TAIL>(A.codes + (size_t)row * A.ldc + i, n, code);
            }
        });
        return;
    }
    // Rows at the ends of the range or not finite, in 64 bits.
    const double inv = mean == 0.0 ? 0.0 : 1.0 / sqrt(mean);   // a row of zeros and eps 0: zeros; a NaN spoils its row
    double most = 0.0, bad = 0.0;
    each<CH>([&](auto c) {
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const double p = (double)elem_at<DT>(r[c], e) * (double)elem_at<DT>(g[c], e);
            if (!(fabs(p) < INFINITY)) bad = 1.0;
            most = fmax(most, fabs(p));
        }
    });
    most = row_join<T, true>(most, sums, Most());
    bad = row_join<T, true>(bad, sums, Most());
    const bool finite = bad == 0.0 && sum < INFINITY;
    if (t == 0 && A.codes) A.scales[row] = finite ? (float)(most * inv / 127.0) : quiet_nan();
    each<CH>([&](auto c) {
        const int i = (c * T + t) * 8, n = d - i;
        if (n <= 0) return;
        uint2 code = make_uint2(0, 0);
        uint4 o = make_uint4(0, 0, 0, 0);
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const double p = (double)elem_at<DT>(r[c], e) * (double)elem_at<DT>(g[c], e);
            const uint32_t h = (round_pair<DT>((float)(p * inv), 0.0f) & 0xFFFFu) << (16 * (e & 1));
            if (e < 2) o.x |= h;
            else if (e < 4) o.y |= h;
            else if (e < 6) o.z |= h;
            else o.w |= h;
            if (finite && most > 0.0) set_code(code, e, exact_code(p, most));
        }
        if (A.out) store8<TAIL, false>(A.out + (size_t)row * A.ldo + i, n, o);
        if (A.codes) store_codes<TAIL>(A.codes + (size_t)row * A.ldc + i, n, code);
    });
}

// What is quantised, in 64 bits and rounded to 32.
template <int ACT>
__device__ __forceinline__ float exact_act(float g, float u) {
    const double z = g;
    if constexpr (ACT == kActSilu) return (float)((double)u * (z / (1.0 + exp(-z))));
    else return (float)((double)u * (0.5 * z * erfc(z * -0.70710678118654752440)));
}
// The same in 32 bits, for gates from kFarGate on; off by rel_act(g) of its size at most, g the least of some gates and 0:
//   SiLU: the exponent's product rounds (1.5 |g| 2^-24 of the exponential, which matters where g < 0), exp2 and 1 / x are
//   good to 2^-23, three more roundings: (1.5 |g| + 8) 2^-24;
//   GELU: z Phi(z) = max(z, 0) - |z| Phi(-|z|), Phi(-z) = exp(-z^2 / 2) t Q(t), t = 1 / (1 + 0.305 z), with a
//   polynomial of degree 7 fitted to exp(z^2 / 2) Phi(-z) over [0, 13] (off by 9.6e-8 of it); the exponent rounds like
//   z^2: (1.5 g^2 + 16) 2^-24.
template <int ACT>
constexpr float kFarGate = ACT == kActSilu ? -80.0f : -12.0f;
template <int ACT>
__device__ __forceinline__ float fast_act(float g, float u) {
    if constexpr (ACT == kActSilu) {
        return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f)) * u;
    } else {
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.305f, 1.0f));
        float q = 0.036698908f;
        q = fmaf(q, t, -0.15298693f);
        q = fmaf(q, t, 0.18571411f);
        q = fmaf(q, t, -0.03797383f);
        q = fmaf(q, t, 0.12101983f);
        q = fmaf(q, t, 0.10342152f);
        q = fmaf(q, t, 0.1224667f);
        q = fmaf(q, t, 0.12163974f);
        const float h = q * t * __builtin_amdgcn_exp2f(g * g * -0.72134752f);   // Phi(-|g|)
        return fmaf(-fabsf(g), h, fmaxf(g, 0.0f)) * u;
    }
}
template <int ACT>
__device__ __forceinline__ float rel_act(float g) {
    if constexpr (ACT == kActSilu) return fmaf(g, -0x1p-23f, 0x1p-20f);
    else return fmaf(g * g, 0x1p-23f, 0x1p-19f);
}

template <int DT, class C, bool TAIL>
__global__ __launch_bounds__(C::threads) void quant_kernel(QuantArgs A) {
    constexpr bool WAVE = C::wave;
    constexpr int T = C::T, CH = C::CH;
    __shared__ uint32_t tops[T / 64];
    const int row = WAVE ? (int)blockIdx.x * 4 + (int)threadIdx.x / 64 : (int)blockIdx.x;
    const int t = WAVE ? lane_id() : (int)threadIdx.x;
    if (WAVE && row >= A.rows) return;
    const int d = A.d;
    const uint16_t *x = A.x + (size_t)row * A.ldx;
    uint4 v[CH];
    uint32_t top = 0;
    each<CH>([&](auto c) {
        const int i = (c * T + t) * 8, n = d - i;
        v[c] = n > 0 ? load8<TAIL>(x + i, n) : make_uint4(0, 0, 0, 0);
    });
    each<CH>([&](auto c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(elem<DT>(v[c], e)) & 0x7FFFFFFFu);   // NaN above all
    });
    top = row_join<T, false>(top, tops, Most());
    const float topf = __uint_as_float(top), s = 127.0f / topf;
    const bool finite = top < 0x7F800000u, plain = topf >= 0x1p-100f;   // s is a finite number
    if (t == 0) A.scales[row] = finite ? (float)((double)topf * (1.0 / 127.0)) : quiet_nan();
    int8_t *codes = A.codes + (size_t)row * A.ldc;
    each<CH>([&](auto c) {
        const int i = (c * T + t) * 8, n = d - i;
        if (n <= 0) return;
        uint32_t near = 0xFFu;
        uint2 code = make_uint2(0, 0);
        if (plain) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = elem<DT>(v[c], e);
            code = fast_codes(p, s, near, 0.0f);
        }
        if (!finite || top == 0) near = 0, code = make_uint2(0, 0);
#pragma unroll 1
        for (; near; near &= near - 1) {
            const int e = __builtin_ctz(near);
            set_code(code, e, exact_code((double)elem_at<DT>(v[c], e), (double)topf));
        }
        store_codes<TAIL>(codes + i, n, code);
    });
}

// The codes go by the exact activations (exact_act), which are worked out for few of them only: those that may be the
// row's largest and those that stand near the middle of two codes by their values in 32 bits.  They are listed, and
// worked out when the row's registers are free, from the inputs again.
constexpr int kListed = 256;
struct GatedRow {
    uint32_t n_top, n_near;
    uint16_t may_top[kListed], near[kListed];   // elements of the row
};

template <int DT, class C, bool TAIL, int ACT>
__global__ __launch_bounds__(C::threads) void gated_kernel(QuantArgs A) {
    constexpr bool WAVE = C::wave;
    constexpr int T = C::T, CH = C::CH;
    __shared__ uint32_t parts[T / 64], parts2[T / 64];
    __shared__ GatedRow lists[WAVE ? 4 : 1];
    const int row = WAVE ? (int)blockIdx.x * 4 + (int)threadIdx.x / 64 : (int)blockIdx.x;
    const int t = WAVE ? lane_id() : (int)threadIdx.x;
    if (WAVE && row >= A.rows) return;
    GatedRow &L = lists[WAVE ? threadIdx.x / 64 : 0];
    auto sync = [] {
        if constexpr (WAVE) wave_lds_fence();
        else __syncthreads();
    };
    if (t == 0) L.n_top = L.n_near = 0;
    const int d = A.d;
    const uint16_t *x = A.x + (size_t)row * A.ldx, *u = A.up + (size_t)row * A.ldu;
    int8_t *codes = A.codes + (size_t)row * A.ldc;
    float v[CH][8], least[CH], low = 0.0f;
    uint32_t top = 0;
    {
        uint4 gv[CH], uv[CH];
        each<CH>([&](auto c) {
            const int i = (c * T + t) * 8, n = d - i;
            gv[c] = n > 0 ? load8<TAIL>(x + i, n) : make_uint4(0, 0, 0, 0);
            uv[c] = n > 0 ? load8<TAIL>(u + i, n) : make_uint4(0, 0, 0, 0);
        });
        each<CH>([&](auto c) {
            least[c] = 0.0f;
            if (c > 0 && c * T * 8 >= d) {   // no thread has any
#pragma unroll
                for (int e = 0; e < 8; ++e) v[c][e] = 0.0f;
                return;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = elem<DT>(gv[c], e);
                least[c] = fminf(least[c], g);
                v[c][e] = fast_act<ACT>(g, elem<DT>(uv[c], e));
                top = max(top, __float_as_uint(v[c][e]) & 0x7FFFFFFFu);   // NaN above all
            }
            low = fminf(low, least[c]);
        });
    }
    const float mine = __uint_as_float(top);
    uint32_t lows = __float_as_uint(low) & 0x7FFFFFFFu;   // of gates below 0, bits order like sizes
    row_join2<T>(top, parts, Most(), lows, parts2, Most());
    low = __uint_as_float(lows | 0x80000000u);
    const float topf = __uint_as_float(top);
    bool slow = !(topf >= 0x1p-60f && topf <= 0x1p100f);   // ends of the range, not finite
    const float rel_top = rel_act<ACT>(fmaxf(low, kFarGate<ACT>));   // topf is off by this much, unless a far gate makes the largest
    if (!slow) {
        const float s = 127.0f / topf, from = topf * (1.0f - 0x1p-14f);
        each<CH>([&](auto c) {
            const int i = (c * T + t) * 8, n = d - i;
            if (n <= 0) return;
            uint32_t near, may = 0;
            const uint2 code = fast_codes(v[c], s, near, rel_act<ACT>(least[c]) + rel_top);
            if (mine >= from) {
#pragma unroll
                for (int e = 0; e < 8; ++e) may |= fabsf(v[c][e]) >= from ? 1u << e : 0u;
            }
            if (least[c] < kFarGate<ACT>) near = may = n >= 8 ? 0xFFu : (1u << n) - 1;
#pragma unroll 1
            for (; near; near &= near - 1) {
                const uint32_t at = atomicAdd(&L.n_near, 1u);
                if (at < kListed) L.near[at] = (uint16_t)(i + __builtin_ctz(near));
            }
#pragma unroll 1
            for (; may; may &= may - 1) {
                const uint32_t at = atomicAdd(&L.n_top, 1u);
                if (at < kListed) L.may_top[at] = (uint16_t)(i + __builtin_ctz(may));
            }
            store_codes<TAIL>(codes + i, n, code);
        });
        sync();
        slow = L.n_top > kListed || L.n_near > kListed;
    }
    auto exact = [&](int i) { return exact_act<ACT>(half_to_float<DT>(x[i]), half_to_float<DT>(u[i])); };
    auto largest = [&] {   // slow: of every element
        const int n = slow ? d : (int)L.n_top;
        uint32_t most = 0;
#pragma unroll 1
        for (int i = t; i < n; i += T) most = max(most, __float_as_uint(exact(slow ? i : (int)L.may_top[i])) & 0x7FFFFFFFu);
        return row_join<T, true>(most, parts, Most());
    };
    uint32_t most = largest();
    if (!slow && fabsf(__uint_as_float(most) - topf) > rel_top * topf) {   // a far gate makes it: the codes may be off by more
        slow = true;
        most = largest();
    }
    const int n_near = slow ? d : (int)L.n_near;
    const bool finite = most < 0x7F800000u;
    const double mostd = (double)__uint_as_float(most);
    if (t == 0) A.scales[row] = finite ? (float)(mostd * (1.0 / 127.0)) : quiet_nan();
#pragma unroll 1
    for (int i = t; i < n_near; i += T) {
        const int e = slow ? i : (int)L.near[i];
        codes[e] = finite && most > 0 ? (int8_t)exact_code((double)exact(e), mostd) : (int8_t)0;
    }
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// sigma c: a workgroup takes 1024 chunks of 4 codes, of one row or several (a row of d has ceil(d / 4)).
__global__ __launch_bounds__(256) void read_q8_kernel(const int8_t *__restrict__ codes, int64_t ldc, const float *__restrict__ scales,
                                                      int rows, int d, float *__restrict__ out) {
    const int per = (d + 3) / 4;
    const long long start = (long long)blockIdx.x * 1024;
    const int row0 = (int)(start / per), off0 = (int)(start - (long long)row0 * per);
    const float inv = 1.0f / (float)per;
#pragma unroll
    for (int l = 0; l < 4; ++l) {
        const int at = off0 + l * 256 + (int)threadIdx.x;   // below 2^15
        int q = (int)((float)at * inv), i = at - q * per;   // the quotient, or one off
        if (i < 0) --q, i += per;
        else if (i >= per) ++q, i -= per;
        const int row = row0 + q, n = d - 4 * i;
        if (row >= rows) break;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + (size_t)row * ldc + 4 * i);
        const float s = scales[row];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = s * (float)(int8_t)(w >> (8 * e));
        float *dst = out + (size_t)row * d + 4 * i;
        if (n >= 4) {
            // Not read here again (as a stream: 2048 x 28672 42.6 us, else 76).
            __builtin_nontemporal_store(f32x4_any{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_any *>(dst));
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) dst[e] = v[e];
        }
    }
}

// Few rows take a thread for every chunk or two; many rows more chunks a thread, whose loads are on the way together, and
// fewer threads, so that a CU has several rows in different stages.  Whole multiples of 4 waves: 7 waves of 8 chunks
// a thread, SwiGLU of 2048 x 28672, took 68 us, 8 waves 60, 14 of 4 chunks 80.  Norm of 8192 x 2048, 1 chunk a
// thread and 4: 24.6 and 29.8; 2048 x 8192, 2 and 4: 26.9, 28.7, SwiGLU 19.1, 17.5; norm of 2048 x 16384, 2 and 4: 59.2, 52.6.
template <typename F>
hipError_t by_width(int rows, int d, bool gated, F f) {
    const int chunks = (d + 7) / 8;
    const bool many = rows >= 1024;   // 4 a CU
    if (chunks <= 64) return f(Cut<64, 1>{});
    if (chunks <= 256) return f(Cut<256, 1>{});
    if (chunks <= 512) return f(Cut<256, 2>{});
    if (chunks <= 1024) return many && gated ? f(Cut<256, 4>{}) : f(Cut<512, 2>{});
    if (chunks <= 2048) return many ? f(Cut<512, 4>{}) : f(Cut<1024, 2>{});
    if (chunks <= 4096) return many ? f(Cut<512, 8>{}) : f(Cut<1024, 4>{});
    return f(Cut<1024, 8>{});
}

template <int DT>
hipError_t quant_dt(const QuantArgs &a, hipStream_t s) {
    return by_width(a.rows, a.d, a.up != nullptr, [&](auto cut) {
        using C = decltype(cut);
        constexpr unsigned threads = C::threads;
        const unsigned grid = C::wave ? (a.rows + 3) / 4 : a.rows;
        const bool tail = a.d % 8 != 0;
        if (!a.up) {
            if (tail) quant_kernel<DT, C, true><<<grid, threads, 0, s>>>(a);
            else quant_kernel<DT, C, false><<<grid, threads, 0, s>>>(a);
        } else if (a.act == kActSilu) {
            if (tail) gated_kernel<DT, C, true, kActSilu><<<grid, threads, 0, s>>>(a);
            else gated_kernel<DT, C, false, kActSilu><<<grid, threads, 0, s>>>(a);
        } else {
            if (tail) gated_kernel<DT, C, true, kActGelu><<<grid, threads, 0, s>>>(a);
            else gated_kernel<DT, C, false, kActGelu><<<grid, threads, 0, s>>>(a);
        }
        return hipGetLastError();
    });
}

template <int DT>
hipError_t norm_dt(const NormArgs &a, hipStream_t s) {
    return by_width(a.rows, a.d, false, [&](auto cut) {
        using C = decltype(cut);
        constexpr unsigned threads = C::threads;
        const unsigned grid = C::wave ? (a.rows + 3) / 4 : a.rows;
        if (a.d % 8) rmsnorm_kernel<DT, C, true><<<grid, threads, 0, s>>>(a);
        else rmsnorm_kernel<DT, C, false><<<grid, threads, 0, s>>>(a);
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
    const long long blocks = ((long long)rows * ((d + 3) / 4) + 1023) / 1024;   // 2^26 at most
    read_q8_kernel<<<(unsigned)blocks, 256, 0, s>>>(codes, ldc, scales, rows, d, out);
    return hipGetLastError();
}

}  // namespace prox
