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
__device__ __forceinline__ uint32_t rotated(float a, float b, float sign, float cos, float sin) {
    // own a cos + sign * other sin
    float r = (float)fma((double)a, (double)cos, (double)(sign * b) * (double)sin);
    asm("" : "+v"(r));   // else the compiler rounds to fp16 in one step, and to bf16 in two
    return float_to_half<DT>(r);
}

// Chunk of 8 channels from c0 (c0 % 8 == 0) of one head of one token, rotated.
// row: the head's first channel; trow: the position's row of the table.
template <int DT>
__device__ __forceinline__ uint4 rotated_chunk(const uint16_t *row, int c0, const float *trow, const Rope &rope) {
    const uint4 own = *reinterpret_cast<const uint4 *>(row + c0);
    if (!trow || c0 >= rope.dim) return own;
    const int half = rope.dim / 2;
    uint32_t h[8];
    if (rope.interleaved) {
        const float4 c = *reinterpret_cast<const float4 *>(trow + c0 / 2);
        const float4 s = *reinterpret_cast<const float4 *>(trow + half + c0 / 2);
        const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const float a = half_to_float<DT>((uint16_t)half_of(own, 2 * p));
            const float b = half_to_float<DT>((uint16_t)half_of(own, 2 * p + 1));
            h[2 * p] = rotated<DT>(a, b, -1.0f, cs[p], sn[p]);
            h[2 * p + 1] = rotated<DT>(b, a, 1.0f, cs[p], sn[p]);
        }
    } else {
        const bool lo = c0 < half;
        const int i = lo ? c0 : c0 - half;
        const uint4 other = *reinterpret_cast<const uint4 *>(row + (lo ? c0 + half : i));
        const float sign = lo ? -1.0f : 1.0f;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float4 c = *reinterpret_cast<const float4 *>(trow + i + 4 * q);
            const float4 s = *reinterpret_cast<const float4 *>(trow + half + i + 4 * q);
            const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int p = 0; p < 4; ++p)
                h[4 * q + p] = rotated<DT>(half_to_float<DT>((uint16_t)half_of(own, 4 * q + p)),
                                           half_to_float<DT>((uint16_t)half_of(other, 4 * q + p)), sign, cs[p], sn[p]);
        }
    }
    return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
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
    long long kv_items;
};

// A workgroup takes the new tokens of one (sequence, block of 32 tokens, kv head), so that
// each word of V codes, which holds 8 tokens of a channel, has one writer: waves 0, 1 keys,
// waves 2, 3 values, D / 8 lanes a token.  Words that keep older tokens are read and
// merged.  The workgroups after those rotate the queries.
template <int DT, int D>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs A) {
    constexpr int LT = D / 8;         // lanes of a token: chunks of 8 channels
    constexpr int TP = 128 / LT;      // tokens per pass of a half workgroup
    const int tid = threadIdx.x;
    if ((long long)blockIdx.x >= A.kv_items) {   // queries
        const int half = A.rope.dim / 2;
        const bool pairs = A.rope.table && !A.rope.interleaved;   // two chunks turn together
        const int turn = pairs ? half / 8 : 0;
        const int units = turn + (D - 16 * turn) / 8;
        const long long per = (long long)A.q_heads * units;
        const long long id = ((long long)blockIdx.x - A.kv_items) * 256 + tid;
        const long long row = id / per;
        if (row >= (long long)A.s.n_seq * A.s.max_new) return;
        const int s = (int)(row / A.s.max_new), i = (int)(row % A.s.max_new);
        const SeqTokens sq = seq_tokens(A.s, s);
        const int pos = sq.pos0 + i;
        if (i >= sq.n || pos < 0) return;
        const int h = (int)(id % per) / units, u = (int)(id % per) % units;
        const uint16_t *src = A.q + (size_t)(sq.t0 + i) * A.ldq + (size_t)h * D;
        uint16_t *dst = A.q_out + (size_t)(sq.t0 + i) * A.ldq_out + (size_t)h * D;
        const float *trow = A.rope.table ? A.rope.table + (size_t)pos * A.rope.dim : nullptr;
        if (u < turn) {   // both halves read before either is written: q_out may be q
            const uint4 a = rotated_chunk<DT>(src, 8 * u, trow, A.rope);
            const uint4 b = rotated_chunk<DT>(src, half + 8 * u, trow, A.rope);
            *reinterpret_cast<uint4 *>(dst + 8 * u) = a;
            *reinterpret_cast<uint4 *>(dst + half + 8 * u) = b;
        } else {
            const int c0 = 16 * turn + 8 * (u - turn);
            *reinterpret_cast<uint4 *>(dst + c0) = rotated_chunk<DT>(src, c0, trow, A.rope);
        }
        return;
    }
    __shared__ uint32_t vcodes[kKvBlock][LT];   // [token][chunk], channel e at nibble e
    const KvLayout L(D, A.c.group);
    const int head = (int)(blockIdx.x % A.c.heads);
    const long long sb = blockIdx.x / A.c.heads;
    const int s = (int)(sb / A.blocks);
    const SeqTokens sq = seq_tokens(A.s, s);
    const int first = max(sq.pos0, 0), end = sq.pos0 + sq.n;   // positions to write
    const int b = first / kKvBlock + (int)(sb % A.blocks);
    if (first >= end || b * kKvBlock >= end) return;
    uint8_t *rec = kv_record(A.c, A.s, L.record, s, head, b);
    if (!rec) return;
    const int lo = max(first - b * kKvBlock, 0), hi = min(end - b * kKvBlock, kKvBlock);   // new tokens [lo, hi)
    const bool keys = tid < 128;
    const int ch = tid % LT, span = A.c.group / 8;   // lanes of a group
    for (int t = lo + (tid % 128) / LT; t < hi; t += TP) {
        const int pos = b * kKvBlock + t;
        const size_t row = (size_t)(sq.t0 + pos - sq.pos0);
        uint4 v;
        if (keys)
            v = rotated_chunk<DT>(A.k + row * A.ldk + (size_t)head * D, 8 * ch,
                                  A.rope.table ? A.rope.table + (size_t)pos * A.rope.dim : nullptr, A.rope);
        else
            v = *reinterpret_cast<const uint4 *>(A.v + row * A.ldv + (size_t)head * D + 8 * ch);
        uint32_t a = abs_max8<DT>(v);
        for (int m = 1; m < span; m <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, m));   // lanes of one token
        const GroupScale sc = kv_scale<DT>(a);
        if (ch % span == 0)
            *reinterpret_cast<uint16_t *>(rec + (keys ? L.k_scales : L.v_scales) + (ch / span) * 64 + kv_slot(t) * 2) = sc.bits;
        if (keys)
            *reinterpret_cast<uint32_t *>(rec + kv_k_word(D, t, ch) * 4) =
                code_word<DT>(v, sc, [](int e) { return nibble_of(e); });
        else
            vcodes[t][ch] = code_word<DT>(v, sc, [](int e) { return e; });
    }
    __syncthreads();
    uint32_t *words = reinterpret_cast<uint32_t *>(rec + L.v_codes);
    for (int w = tid; w < 4 * D; w += 256) {
        const int lane = w / 4 % 64, c = (w / 256 * 4 + w % 4) * 16 + lane % 16, h = lane / 16;   // kv_v_word(lane, c / 16) == w
        uint32_t mask = 0, codes = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = j < 4 ? 4 * h + j : 12 + 4 * h + j;
            if (t >= lo && t < hi) {
                mask |= 15u << (4 * j);
                codes |= ((vcodes[t][c / 8] >> (4 * (c % 8))) & 15u) << (4 * j);
            }
        }
        if (mask) words[w] = mask == 0xFFFFFFFFu ? codes : (words[w] & ~mask) | codes;
    }
}

// One thread per (row, head, 8 channels).
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
    A.kv_items = (long long)s.n_seq * A.blocks * c.heads;
    long long q_wgs = 0;
    if (q) {
        const int turn = rope.table && !rope.interleaved ? rope.dim / 16 : 0;
        const long long units = (long long)q_heads * (turn + (c.dim - 16 * turn) / 8);
        q_wgs = ((long long)s.n_seq * s.max_new * units + 255) / 256;
    }
    const unsigned grid = (unsigned)(A.kv_items + q_wgs);
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
