// The 4-bit paged key/value cache: rotation and append, and the inverse view.
#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace prox {

// Rotation (a cos - b sin, a sin + b cos) in 64 bits: products of a 16-bit value and an
// fp32 cosine are exact there, so each result is rounded three times (64, 32, 16 bits)
// whatever the order, and no code next to a border depends on how it was summed.  The
// 64-bit arithmetic hides behind the loads.
template <int DT>
__device__ __forceinline__ uint32_t rounded(double v) {
    float r = (float)v;
    asm("" : "+v"(r));   // else the compiler rounds to fp16 in one step, and to bf16 in two
    return float_to_half<DT>(r);
}
template <int DT>
__device__ __forceinline__ uint32_t rotated_a(float a, float b, float cos, float sin) {
    return rounded<DT>(fma((double)a, (double)cos, -((double)b * (double)sin)));
}
template <int DT>
__device__ __forceinline__ uint32_t rotated_b(float a, float b, float cos, float sin) {
    return rounded<DT>(fma((double)a, (double)sin, (double)b * (double)cos));
}
template <int DT>
__device__ __forceinline__ float elem(const uint4 &v, int e) { return half_to_float<DT>((uint16_t)half_of(v, e)); }
__device__ __forceinline__ uint4 packed8(const uint32_t (&h)[8]) {
    return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
}
template <int N>
__device__ __forceinline__ void load_floats(float (&out)[N], const float *p) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const float4 v = *reinterpret_cast<const float4 *>(p + 4 * i);
        out[4 * i] = v.x;
        out[4 * i + 1] = v.y;
        out[4 * i + 2] = v.z;
        out[4 * i + 3] = v.w;
    }
}

// Chunks (channels c0 .. c0 + 7, dim / 2 + c0 ..) that turn together.
template <int DT>
__device__ __forceinline__ void rotate_halves(uint4 &a, uint4 &b, const float (&cos)[8], const float (&sin)[8]) {
    uint32_t x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = rotated_a<DT>(elem<DT>(a, e), elem<DT>(b, e), cos[e], sin[e]);
        y[e] = rotated_b<DT>(elem<DT>(a, e), elem<DT>(b, e), cos[e], sin[e]);
    }
    a = packed8(x);
    b = packed8(y);
}
// A chunk of four pairs (2 i, 2 i + 1).
template <int DT>
__device__ __forceinline__ uint4 rotate_pairs(const uint4 &v, const float (&cos)[4], const float (&sin)[4]) {
    uint32_t x[8];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        x[2 * p] = rotated_a<DT>(elem<DT>(v, 2 * p), elem<DT>(v, 2 * p + 1), cos[p], sin[p]);
        x[2 * p + 1] = rotated_b<DT>(elem<DT>(v, 2 * p), elem<DT>(v, 2 * p + 1), cos[p], sin[p]);
    }
    return packed8(x);
}

// Scale of a group from its largest magnitude pattern, finite (a bf16 group past 7 * 65504
// is clamped by its codes).
template <int DT>
__device__ __forceinline__ GroupScale kv_scale(uint32_t amax_bits) {
    GroupScale s = group_scale<DT>(amax_bits, 7);
    if (s.bits > 0x7BFFu) {
        s.bits = 0x7BFFu;
        s.sigma = 65504.0f;
        s.inv = 1.0f / 65504.0f;
    }
    return s;
}

// Code word of a chunk, element e at nibble place(e).
template <int DT, typename Place>
__device__ __forceinline__ uint32_t code_word(const uint4 &v, const GroupScale &s, Place place) {
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        int q = quantise<DT>(half_of(v, e), s.sigma, s.inv, 7.0f);
        if (s.sigma == 0.0f) q = 0;
        word |= (uint32_t)(q + 8) << (4 * place(e));
    }
    return word;
}

struct AppendArgs {
    KvCache c;
    KvSeqs s;
    const uint16_t *k, *v, *q;
    uint16_t *q_out;
    int64_t ldk, ldv, ldq, ldq_out;
    int q_heads;
    Rope rope;
    int blocks;       // blocks of 32 tokens that the new tokens of a sequence may touch
    int kv_items;
};

// Bound for prompts by HBM (q, k, v and the table's rows read, q and the cache written) and a busy VALU
// (59 % of the cycles), by a chain of loads (length, page, data) for single tokens: 4.8 us for 16
// of them, 24.1 us for 4 x 1024 with 32 query and 8 kv heads of 128 (90 MB, 3.7 TB/s).
// A workgroup takes the new tokens of one (sequence, block of 32 tokens, kv head), so that
// each word of V codes, which holds 8 tokens of a channel, has one writer: waves 0, 1 keys,
// waves 2, 3 values, D / 8 lanes a token.  Words that keep older tokens are read and
// merged.  The workgroups after those rotate the queries.
constexpr int kHeads = 4;   // query heads that share a thread's cosines and sines
template <int DT, int D>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs A) {
    constexpr int LT = D / 8;         // lanes of a token: chunks of 8 channels
    constexpr int TP = 128 / LT;      // tokens per pass of a half workgroup
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= A.kv_items) {   // queries: kHeads heads of one (token, unit) a thread
        const int half = A.rope.dim / 2;
        const bool pairs = A.rope.table && !A.rope.interleaved;   // units of two chunks that turn together
        const uint32_t turn = pairs ? half / 8 : 0, units = turn + (D - 16 * turn) / 8;
        const uint32_t sets = (A.q_heads + kHeads - 1) / kHeads;
        const uint32_t id = (blockIdx.x - (uint32_t)A.kv_items) * 256u + tid;   // [row][set][unit]
        const uint32_t u = id % units, rest = id / units, set = rest % sets, row = rest / sets;
        const uint32_t s = row / A.s.max_new, i = row % A.s.max_new;
        if (s >= (uint32_t)A.s.n_seq) return;
        const SeqTokens sq = seq_tokens(A.s, s);
        const int pos = sq.pos0 + (int)i;
        if ((int)i >= sq.n || pos < 0) return;
        const int h0 = set * kHeads, n = min(A.q_heads - h0, kHeads);
        const uint16_t *src = A.q + (size_t)(sq.t0 + i) * A.ldq + (size_t)h0 * D;
        uint16_t *dst = A.q_out + (size_t)(sq.t0 + i) * A.ldq_out + (size_t)h0 * D;
        const float *trow = A.rope.table ? A.rope.table + (size_t)pos * A.rope.dim : nullptr;
        if (u < turn) {   // both halves read before either is written: q_out may be q
            float cos[8], sin[8];
            load_floats(cos, trow + 8 * u);
            load_floats(sin, trow + half + 8 * u);
            uint4 a[kHeads], b[kHeads];
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
                const uint16_t *p = src + min(h, n - 1) * D + 8 * u;
                a[h] = *reinterpret_cast<const uint4 *>(p);
                b[h] = *reinterpret_cast<const uint4 *>(p + half);
            }
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
                if (h >= n) break;
                rotate_halves<DT>(a[h], b[h], cos, sin);
                *reinterpret_cast<uint4 *>(dst + h * D + 8 * u) = a[h];
                *reinterpret_cast<uint4 *>(dst + h * D + half + 8 * u) = b[h];
            }
        } else {
            const int c0 = 16 * turn + 8 * (u - turn);
            const bool turns = trow && A.rope.interleaved && c0 < A.rope.dim;
            float cos[4] = {}, sin[4] = {};
            if (turns) {
                load_floats(cos, trow + c0 / 2);
                load_floats(sin, trow + half + c0 / 2);
            }
            uint4 a[kHeads];
#pragma unroll
            for (int h = 0; h < kHeads; ++h) a[h] = *reinterpret_cast<const uint4 *>(src + min(h, n - 1) * D + c0);
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
                if (h >= n) break;
                *reinterpret_cast<uint4 *>(dst + h * D + c0) = turns ? rotate_pairs<DT>(a[h], cos, sin) : a[h];
            }
        }
        return;
    }
    __shared__ uint32_t vcodes[kKvBlock][LT];   // [token][chunk], channel e at nibble e
    const KvLayout L(D, A.c.group);
    const uint32_t sb = blockIdx.x / (uint32_t)A.c.heads;
    const int head = (int)(blockIdx.x - sb * A.c.heads), s = (int)(sb / (uint32_t)A.blocks);
    const SeqTokens sq = seq_tokens(A.s, s);
    const int first = max(sq.pos0, 0), end = sq.pos0 + sq.n;   // positions to write
    const int b = first / kKvBlock + (int)(sb % (uint32_t)A.blocks);
    if (first >= end || b * kKvBlock >= end) return;
    uint8_t *rec = kv_record(A.c, A.s, L.record, s, head, b);
    if (!rec) return;
    const int lo = max(first - b * kKvBlock, 0), hi = min(end - b * kKvBlock, kKvBlock);   // new tokens [lo, hi)
    // Words of V codes that keep older tokens are asked for first.
    constexpr int NW = 4 * D / 256;
    uint32_t *words = reinterpret_cast<uint32_t *>(rec + L.v_codes);
    uint32_t mask[NW], old[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const int w = tid + 256 * i, h = w / 4 % 64 / 16;
        mask[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = j < 4 ? 4 * h + j : 12 + 4 * h + j;
            mask[i] |= t >= lo && t < hi ? 15u << (4 * j) : 0u;
        }
        old[i] = mask[i] != 0 && mask[i] != 0xFFFFFFFFu ? words[w] : 0u;
    }
    const bool keys = tid < 128;
    const int ch = tid % LT, span = A.c.group / 8;   // lanes of a group
    const int t0 = lo + (tid % 128) / LT;
    const int64_t ld = keys ? A.ldk : A.ldv;
    const uint16_t *src = (keys ? A.k : A.v) + (size_t)head * D;
    constexpr int NP = 2;   // passes whose loads go out together (4: 148 registers, 29.4 us)
    const int half = A.rope.dim / 2, c0 = 8 * ch;
    const bool turns = keys && A.rope.table && c0 < A.rope.dim, second = turns && !A.rope.interleaved && c0 >= half;
    const int i0 = A.rope.interleaved ? c0 / 2 : second ? c0 - half : c0;   // first frequency
    const int partner = A.rope.interleaved || !turns ? c0 : second ? c0 - half : c0 + half;
    for (int tb = t0; tb < hi; tb += NP * TP) {
        uint4 own[NP], other[NP];
        float cos[NP][8], sin[NP][8];
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int t = min(tb + j * TP, hi - 1), pos = b * kKvBlock + t;
            const uint16_t *row = src + (size_t)(sq.t0 + pos - sq.pos0) * ld;
            own[j] = *reinterpret_cast<const uint4 *>(row + c0);
            if (turns) {
                const float *trow = A.rope.table + (size_t)pos * A.rope.dim + i0;
                if (A.rope.interleaved) {
                    float c4[4], s4[4];
                    load_floats(c4, trow);
                    load_floats(s4, trow + half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        cos[j][e] = c4[e];
                        sin[j][e] = s4[e];
                    }
                } else {
                    other[j] = *reinterpret_cast<const uint4 *>(row + partner);
                    load_floats(cos[j], trow);
                    load_floats(sin[j], trow + half);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int t = tb + j * TP;
            if (t >= hi) break;   // whole tokens: the shuffles below stay inside one
            uint4 v = own[j];
            if (turns) {
                uint32_t x[8];
                if (A.rope.interleaved) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[2 * e] = rotated_a<DT>(elem<DT>(v, 2 * e), elem<DT>(v, 2 * e + 1), cos[j][e], sin[j][e]);
                        x[2 * e + 1] = rotated_b<DT>(elem<DT>(v, 2 * e), elem<DT>(v, 2 * e + 1), cos[j][e], sin[j][e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)   // the second of a pair is b cos + a sin: the first one's with -sin
                        x[e] = rotated_a<DT>(elem<DT>(v, e), elem<DT>(other[j], e), cos[j][e], second ? -sin[j][e] : sin[j][e]);
                }
                v = packed8(x);
            }
            uint32_t a = abs_max8<DT>(v);
            for (int m = 1; m < span; m <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, m));
            const GroupScale sc = kv_scale<DT>(a);
            if (ch % span == 0)
                *reinterpret_cast<uint16_t *>(rec + (keys ? L.k_scales : L.v_scales) + (ch / span) * 64 + kv_slot(t) * 2) = sc.bits;
            if (keys)
                *reinterpret_cast<uint32_t *>(rec + kv_k_word(D, t, ch) * 4) = code_word<DT>(v, sc, [](int e) { return nibble_of(e); });
            else
                vcodes[t][ch] = code_word<DT>(v, sc, [](int e) { return e; });
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        if (!mask[i]) continue;
        const int w = tid + 256 * i, lane = w / 4 % 64, c = (w / 256 * 4 + w % 4) * 16 + lane % 16, h = lane / 16;   // kv_v_word(lane, c / 16) == w
        uint32_t codes = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = j < 4 ? 4 * h + j : 12 + 4 * h + j;
            codes |= ((vcodes[t][c / 8] >> (4 * (c % 8))) & 15u) << (4 * j);   // unwritten rows: masked
        }
        words[w] = (old[i] & ~mask[i]) | (codes & mask[i]);
    }
}

// One thread per (row, head, 8 channels).  Bound by its writes, 8 bytes a channel: 6 x up to 700 tokens
// of 4 heads of 128 in 6.8 us.
__global__ __launch_bounds__(256) void kv_read_kernel(KvCache c, KvSeqs q, float *__restrict__ k, float *__restrict__ v) {
    const KvLayout L(c.dim, c.group);
    const int LT = c.dim / 8, per = c.heads * LT;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row = id / per;
    if (row >= (long long)q.n_seq * q.max_new) return;
    const int s = (int)(row / q.max_new), i = (int)(row % q.max_new);
    const SeqTokens sq = seq_tokens(q, s);
    const int pos = sq.pos0 + i;
    if (i >= sq.n || pos < 0) return;
    const int head = (int)(id % per) / LT, ch = (int)(id % per) % LT;
    const uint8_t *rec = kv_record(c, q, L.record, s, head, pos / kKvBlock);
    float kv[8] = {}, vv[8] = {};
    if (rec) {
        const int t = pos % kKvBlock, g = 8 * ch / c.group;
        const float ks = f16_bits_to_float(*reinterpret_cast<const uint16_t *>(rec + L.k_scales + g * 64 + kv_slot(t) * 2));
        const float vs = f16_bits_to_float(*reinterpret_cast<const uint16_t *>(rec + L.v_scales + g * 64 + kv_slot(t) * 2));
        const uint32_t kw = *reinterpret_cast<const uint32_t *>(
            rec + kv_k_word(c.dim, t, ch) * 4);
        const int lane0 = ((t % 16) / 4) * 16, nib = t % 4 + 4 * (t / 16);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int cc = 8 * ch + e;
            const uint32_t vw = *reinterpret_cast<const uint32_t *>(
                rec + L.v_codes + kv_v_word(lane0 + cc % 16, cc / 16) * 4);
            kv[e] = ks * (float)((int)((kw >> (4 * nibble_of(e))) & 15) - 8);
            vv[e] = vs * (float)((int)((vw >> (4 * nib)) & 15) - 8);
        }
    }
    const size_t o = ((size_t)(sq.t0 + i) * c.heads + head) * c.dim + 8 * ch;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        *reinterpret_cast<float4 *>(k + o + 4 * p) = make_float4(kv[4 * p], kv[4 * p + 1], kv[4 * p + 2], kv[4 * p + 3]);
        *reinterpret_cast<float4 *>(v + o + 4 * p) = make_float4(vv[4 * p], vv[4 * p + 1], vv[4 * p + 2], vv[4 * p + 3]);
    }
}

hipError_t launch_kv_append(int dtype, const KvCache &c, const KvSeqs &s, const void *k, int64_t ldk, const void *v,
                            int64_t ldv, const void *q, int q_heads, int64_t ldq, void *q_out, int64_t ldq_out,
                            const Rope &rope, hipStream_t stream) {
    AppendArgs A{c, s, static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v),
                 static_cast<const uint16_t *>(q), static_cast<uint16_t *>(q_out), ldk, ldv, ldq, ldq_out, q_heads,
                 rope, (s.max_new + 2 * kKvBlock - 2) / kKvBlock, 0};
    A.kv_items = s.n_seq * A.blocks * c.heads;   // at most 2^23 workgroups in all (checked)
    long long q_wgs = 0;
    if (q) {
        const int turn = rope.table && !rope.interleaved ? rope.dim / 16 : 0;
        const long long units = (long long)((q_heads + kHeads - 1) / kHeads) * (turn + (c.dim - 16 * turn) / 8);
        q_wgs = ((long long)s.n_seq * s.max_new * units + 255) / 256;
    }
    const unsigned grid = (unsigned)A.kv_items + (unsigned)q_wgs;
#define APPEND(DT_)                                                                       \
    do {                                                                                  \
        if (c.dim == 64) kv_append_kernel<DT_, 64><<<grid, 256, 0, stream>>>(A);          \
        else if (c.dim == 128) kv_append_kernel<DT_, 128><<<grid, 256, 0, stream>>>(A);   \
        else kv_append_kernel<DT_, 256><<<grid, 256, 0, stream>>>(A);                     \
    } while (0)
    if (dtype == kBF16) APPEND(kBF16);
    else APPEND(kF16);
#undef APPEND
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvCache &c, const KvSeqs &s, float *k, float *v, hipStream_t stream) {
    const long long n = (long long)s.n_seq * s.max_new * c.heads * (c.dim / 8);
    kv_read_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(c, s, k, v);
    return hipGetLastError();
}

}  // namespace prox
