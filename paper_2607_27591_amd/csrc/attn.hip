// Attention of new tokens over the 4-bit paged cache.
#include "common.hpp"
#include "kernels.hpp"

namespace prox {

struct AttnArgs {
    KvCache c;
    KvSeqs s;
    const uint16_t *q;
    uint16_t *out;
    int64_t ldq, ldo;
    int q_heads, window;
    float scale;
};

// One workgroup per (sequence, new token, query head); its four waves take the blocks of
// 32 tokens in turn, each with its own running maximum m and sum l of the softmax,
//   m' = max(m, max s_p),  l' = l e^(m - m') + sum e^(s_p - m'),  o likewise,
// joined at the end.
template <int DT, int D>
__global__ __launch_bounds__(256) void attn_kernel(AttnArgs A) {
    constexpr int W = 4, CH = D / kWave;
    __shared__ float q[D], p_sh[W][kKvBlock], o_sh[W][D], m_sh[W], l_sh[W];
    const KvLayout L(D, A.c.group);
    const int h = blockIdx.x % A.q_heads;
    const int row = blockIdx.x / A.q_heads, s = row / A.s.max_new, i = row % A.s.max_new;
    const SeqTokens sq = seq_tokens(A.s, s);
    if (i >= sq.n) return;
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
    const int pos = sq.pos0 + i, head = h / (A.q_heads / A.c.heads);
    const int from = A.window > 0 ? max(pos - A.window + 1, 0) : 0;
    if (tid < D) q[tid] = half_to_float<DT>(A.q[(size_t)(sq.t0 + i) * A.ldq + (size_t)h * D + tid]) * A.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.0f, o[CH] = {};
    const int end = pos + 1;   // <= len <= max_kv
    for (int b = from / kKvBlock + wave; b * kKvBlock < end; b += W) {
        const uint8_t *rec = kv_record(A.c, A.s, L.record, s, head, b);
        if (!rec) continue;
        const int t = lane % 32, half = lane / 32;   // token, half of the words
        float sum = 0.0f;
        for (int w = half * (D / 16); w < (half + 1) * (D / 16); ++w) {   // chunk of 8 channels
            const uint32_t word = *reinterpret_cast<const uint32_t *>(
                rec + (size_t)(((t / 16) * 64 + (w % 4) * 16 + t % 16) * (D / 32) + w / 4) * 4);
            const float sc = f16_bits_to_float(*reinterpret_cast<const uint16_t *>(
                rec + L.k_scales + (8 * w / A.c.group) * 64 + kv_slot(t) * 2));
            float d = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) d = fmaf((float)((int)((word >> (4 * nibble_of(e))) & 15) - 8), q[8 * w + e], d);
            sum = fmaf(d, sc, sum);
        }
        sum = add_swap32(sum);
        const int p0 = b * kKvBlock + t;
        if (p0 < from || p0 >= end) sum = -INFINITY;   // whatever stands there
        float mx = sum;
        for (int x = 1; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
        const float m2 = fmaxf(m, mx), alpha = m == -INFINITY ? 0.0f : __expf(m - m2);
        const float pr = sum == -INFINITY ? 0.0f : __expf(sum - m2);
        float ps = pr;
        for (int x = 1; x < 32; x <<= 1) ps += __shfl_xor(ps, x);
        l = fmaf(l, alpha, ps);
        m = m2;
        if (lane < 32) p_sh[wave][t] = pr;
        wave_lds_fence();
#pragma unroll
        for (int u = 0; u < CH; ++u) {
            const int c = lane + kWave * u;
            float acc = o[u] * alpha;
            for (int hh = 0; hh < 4; ++hh) {
                const uint32_t word = *reinterpret_cast<const uint32_t *>(
                    rec + L.v_codes + (size_t)((hh * 16 + c % 16) * (D / 16) + c / 16) * 4);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int tt = j < 4 ? 4 * hh + j : 12 + 4 * hh + j;
                    const float pv = p_sh[wave][tt];
                    const float sc = f16_bits_to_float(*reinterpret_cast<const uint16_t *>(
                        rec + L.v_scales + (c / A.c.group) * 64 + kv_slot(tt) * 2));
                    if (pv != 0.0f) acc = fmaf(pv * sc, (float)((int)((word >> (4 * j)) & 15) - 8), acc);
                }
            }
            o[u] = acc;
        }
        wave_lds_fence();
    }
#pragma unroll
    for (int u = 0; u < CH; ++u) o_sh[wave][lane + kWave * u] = o[u];
    if (lane == 0) { m_sh[wave] = m; l_sh[wave] = l; }
    __syncthreads();
    if (tid < D) {
        float mm = -INFINITY, ll = 0.0f, oo = 0.0f;
        for (int w = 0; w < W; ++w) mm = fmaxf(mm, m_sh[w]);
        for (int w = 0; w < W; ++w)
            if (m_sh[w] != -INFINITY) {
                const float a = __expf(m_sh[w] - mm);
                ll = fmaf(l_sh[w], a, ll);
                oo = fmaf(o_sh[w][tid], a, oo);
            }
        A.out[(size_t)(sq.t0 + i) * A.ldo + (size_t)h * D + tid] = float_to_half<DT>(ll > 0.0f ? oo / ll : 0.0f);
    }
}

hipError_t launch_attn(int dtype, const KvCache &c, const KvSeqs &s, const void *q, int q_heads, int64_t ldq,
                       float scale, int window, void *out, int64_t ldo, void *ws, hipStream_t stream) {
    (void)ws;
    const AttnArgs A{c, s, static_cast<const uint16_t *>(q), static_cast<uint16_t *>(out), ldq, ldo, q_heads, window, scale};
    const unsigned grid = (unsigned)((long long)s.n_seq * s.max_new * q_heads);
#define ATTN(DT_)                                                                    \
    do {                                                                             \
        if (c.dim == 64) attn_kernel<DT_, 64><<<grid, 256, 0, stream>>>(A);          \
        else if (c.dim == 128) attn_kernel<DT_, 128><<<grid, 256, 0, stream>>>(A);   \
        else attn_kernel<DT_, 256><<<grid, 256, 0, stream>>>(A);                     \
    } while (0)
    if (dtype == kBF16) ATTN(kBF16);
    else ATTN(kF16);
#undef ATTN
    return hipGetLastError();
}

}  // namespace prox
