// C-ABI of the attention half of a decoder layer (declared in include/prox.h): argument
// validation on the host, then one launch each.
#include <prox.h>

#include <cfloat>
#include <cmath>

#include "kernels.hpp"

using namespace prox;

namespace {

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool dtype_ok(int dt) { return dt == PROX_F16 || dt == PROX_BF16; }
prox_status hip_status(hipError_t e) { return e == hipSuccess ? PROX_OK : PROX_ERR_HIP; }

// Workgroups of one launch at most: 256 threads each, within the 32 bits of a grid.
constexpr long long kMaxGrid = 1 << 23;

bool linear_shape_ok(int n, int k, int group) {
    return n >= 1 && n <= PROX_MAX_LINEAR_N && k >= 1 && k <= PROX_MAX_LINEAR_K &&
           (group == 32 || group == 64 || (group >= 128 && group % 128 == 0)) && k % group == 0;
}

prox_status check_linear(const prox_w4_linear *q) {
    if (!q || !q->blob || !aligned(q->blob, 256) || !dtype_ok(q->dtype)) return PROX_ERR_INVALID;
    if (q->n < 1 || q->k < 1) return PROX_ERR_INVALID;
    if (!linear_shape_ok(q->n, q->k, q->group)) return PROX_ERR_UNSUPPORTED;
    if (q->bytes < LinearLayout(q->n, q->k, q->group).total) return PROX_ERR_WORKSPACE;
    return PROX_OK;
}

bool kv_shape_ok(int heads, int dim, int group, int page_size, int n_pages) {
    return heads >= 1 && heads <= 256 && (dim == 64 || dim == 128 || dim == 256) &&
           (group == 32 || group == 64 || group == 128) && group <= dim && page_size >= kKvBlock &&
           page_size % kKvBlock == 0 && page_size <= 32768 && n_pages >= 1 && n_pages <= 1 << 24;
}

size_t kv_page_bytes(int heads, int dim, int group, int page_size) {
    return (size_t)heads * (page_size / kKvBlock) * KvLayout(dim, group).record;
}

prox_status check_cache(const prox_kv_cache *c, KvCache *out) {
    if (!c || !c->blob || !aligned(c->blob, 256) || !dtype_ok(c->dtype)) return PROX_ERR_INVALID;
    if (!kv_shape_ok(c->kv_heads, c->head_dim, c->group, c->page_size, c->n_pages)) return PROX_ERR_UNSUPPORTED;
    const size_t page = kv_page_bytes(c->kv_heads, c->head_dim, c->group, c->page_size);
    if (c->bytes < page * (size_t)c->n_pages) return PROX_ERR_WORKSPACE;
    *out = KvCache{static_cast<uint8_t *>(c->blob), c->kv_heads, c->head_dim, c->group, c->page_size, c->n_pages, page};
    return PROX_OK;
}

prox_status check_seqs(const prox_kv_seqs *s, const prox_kv_cache *c, KvSeqs *out) {
    if (!s || !s->kv_len || !s->page_table) return PROX_ERR_INVALID;
    if (!aligned(s->kv_len, 4) || !aligned(s->page_table, 4) || !aligned(s->cu_new, 4)) return PROX_ERR_INVALID;
    if (s->n_seq < 1 || s->max_new < 1 || s->n_tokens < 0 || s->max_pages < 1 || s->max_kv < 0) return PROX_ERR_INVALID;
    if (!s->cu_new && (long long)s->n_seq * s->max_new != s->n_tokens) return PROX_ERR_INVALID;
    const long long room = (long long)s->max_pages * c->page_size;
    if (s->max_kv > room) return PROX_ERR_INVALID;
    const long long max_kv = s->max_kv ? s->max_kv : room;
    if (s->n_seq > 65536 || max_kv > 1 << 30 || s->max_new > 1 << 30) return PROX_ERR_UNSUPPORTED;
    *out = KvSeqs{s->cu_new, s->kv_len, s->page_table, s->n_seq, s->max_new, s->n_tokens, (int)max_kv, s->max_pages};
    return PROX_OK;
}

// Rows of heads * dim values with a stride of ld elements.
bool rows_ok(const void *p, int64_t ld, int heads, int dim) {
    return p && aligned(p, 16) && ld >= (int64_t)heads * dim && ld % 8 == 0;
}

}  // namespace

extern "C" {

size_t prox_linear_w4_bytes(int n, int k, int group) {
    return linear_shape_ok(n, k, group) ? LinearLayout(n, k, group).total : 0;
}

prox_status prox_pack_linear_w4(const void *w, const prox_w4_linear *q, hipStream_t stream) {
    const prox_status st = check_linear(q);
    if (st != PROX_OK) return st;
    if (!w || !aligned(w, 16)) return PROX_ERR_INVALID;
    return hip_status(launch_pack_linear(q->dtype, w, q->n, q->k, q->group, q->blob, stream));
}

prox_status prox_unpack_linear_w4(const prox_w4_linear *q, int8_t *codes, uint16_t *scales, hipStream_t stream) {
    const prox_status st = check_linear(q);
    if (st != PROX_OK) return st;
    if (!codes || !scales || !aligned(scales, 2)) return PROX_ERR_INVALID;
    return hip_status(launch_unpack_linear(q->blob, q->n, q->k, q->group, codes, scales, stream));
}

prox_status prox_linear_w4(const prox_w4_linear *q, const void *x, int64_t ldx, int batch, const void *bias, void *y,
                           int64_t ldy, hipStream_t stream) {
    const prox_status st = check_linear(q);
    if (st != PROX_OK) return st;
    if (!x || !y || !aligned(x, 16) || !aligned(y, 2) || !aligned(bias, 2)) return PROX_ERR_INVALID;
    if (batch < 1 || batch > PROX_MAX_BATCH) return PROX_ERR_INVALID;
    if (batch > 1 && (ldx < q->k || ldx % 8 != 0 || ldy < q->n)) return PROX_ERR_INVALID;
    return hip_status(launch_linear(q->dtype, q->blob, q->n, q->k, q->group, x, ldx, batch, bias, y, ldy, stream));
}

size_t prox_kv_bytes(int kv_heads, int head_dim, int group, int page_size, int n_pages) {
    if (!kv_shape_ok(kv_heads, head_dim, group, page_size, n_pages)) return 0;
    return kv_page_bytes(kv_heads, head_dim, group, page_size) * (size_t)n_pages;
}

prox_status prox_kv_append(const prox_kv_cache *c, const prox_kv_seqs *s, const void *k, int64_t ldk, const void *v,
                           int64_t ldv, const void *q, int q_heads, int64_t ldq, void *q_out, int64_t ldq_out,
                           const prox_rope *rope, hipStream_t stream) {
    KvCache kc;
    KvSeqs ks;
    prox_status st = check_cache(c, &kc);
    if (st != PROX_OK) return st;
    st = check_seqs(s, c, &ks);
    if (st != PROX_OK) return st;
    if (!q != !q_out) return PROX_ERR_INVALID;
    if (q && (q_heads < 1 || q_heads > 4096)) return PROX_ERR_INVALID;
    Rope r{nullptr, 0, 0};
    if (rope) {
        if (!rope->table || !aligned(rope->table, 16) || rope->dim < 16 || rope->n_pos < ks.max_kv) return PROX_ERR_INVALID;
        if (rope->dim % 16 != 0 || rope->dim > kc.dim) return PROX_ERR_UNSUPPORTED;
        r = Rope{rope->table, rope->dim, rope->interleaved};
    }
    if (ks.n_tokens == 0) return PROX_OK;
    if (!rows_ok(k, ldk, kc.heads, kc.dim) || !rows_ok(v, ldv, kc.heads, kc.dim)) return PROX_ERR_INVALID;
    if (q && (!rows_ok(q, ldq, q_heads, kc.dim) || !rows_ok(q_out, ldq_out, q_heads, kc.dim) ||
              (q == q_out && ldq != ldq_out)))
        return PROX_ERR_INVALID;
    const long long items = ((long long)ks.max_new + 2 * kKvBlock - 2) / kKvBlock * ks.n_seq * kc.heads;
    if (items > kMaxGrid) return PROX_ERR_UNSUPPORTED;   // n_seq * max_new is at most 2^28 past here
    if (q && items + (long long)ks.n_seq * ks.max_new * q_heads * (kc.dim / 8) / 256 + 1 > kMaxGrid) return PROX_ERR_UNSUPPORTED;
    return hip_status(launch_kv_append(c->dtype, kc, ks, k, ldk, v, ldv, q, q_heads, ldq, q_out, ldq_out, r, stream));
}

prox_status prox_kv_read(const prox_kv_cache *c, const prox_kv_seqs *s, float *k, float *v, hipStream_t stream) {
    KvCache kc;
    KvSeqs ks;
    prox_status st = check_cache(c, &kc);
    if (st != PROX_OK) return st;
    st = check_seqs(s, c, &ks);
    if (st != PROX_OK) return st;
    if (ks.n_tokens == 0) return PROX_OK;
    if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return PROX_ERR_INVALID;
    if ((long long)ks.n_seq * ks.max_new * kc.heads * (kc.dim / 8) / 256 > kMaxGrid) return PROX_ERR_UNSUPPORTED;
    return hip_status(launch_kv_read(kc, ks, k, v, stream));
}

size_t prox_kv_attn_workspace_bytes(int head_dim) {
    return head_dim == 64 || head_dim == 128 || head_dim == 256 ? attn_workspace_bytes(head_dim) : 0;
}

prox_status prox_kv_attn(const prox_kv_cache *c, const prox_kv_seqs *s, const void *q, int q_heads, int64_t ldq,
                         float scale, int window, void *out, int64_t ldo, void *ws, size_t ws_bytes,
                         hipStream_t stream) {
    KvCache kc;
    KvSeqs ks;
    prox_status st = check_cache(c, &kc);
    if (st != PROX_OK) return st;
    st = check_seqs(s, c, &ks);
    if (st != PROX_OK) return st;
    if (q_heads < 1 || q_heads > 4096 || q_heads % kc.heads != 0 || window < 0) return PROX_ERR_INVALID;
    const double scale2 = std::fabs((double)scale) * 1.4426950408889634;   // of powers of 2
    if (!(scale2 <= FLT_MAX)) return PROX_ERR_INVALID;
    if (!ws || !aligned(ws, 256)) return PROX_ERR_INVALID;
    if (ws_bytes < attn_workspace_bytes(kc.dim)) return PROX_ERR_WORKSPACE;
    if (ks.n_tokens == 0) return PROX_OK;
    if (!rows_ok(q, ldq, q_heads, kc.dim) || !rows_ok(out, ldo, q_heads, kc.dim) || (q == out && ldq != ldo))
        return PROX_ERR_INVALID;
    if (window >= ks.max_kv) window = 0;    // no row stands at max_kv or past it
    const int ratio = q_heads / kc.heads;   // at least 16 rows a workgroup (a split grid is small)
    if (ks.n_seq * (((long long)ks.max_new * ratio + 15) / 16) * kc.heads > kMaxGrid) return PROX_ERR_UNSUPPORTED;
    const int per = kc.page_size / kKvBlock;
    AttnArgs a{kc, ks, static_cast<const uint16_t *>(q), static_cast<uint16_t *>(out), ldq, ldo, q_heads,
               ratio, window, (float)scale2, scale < 0 ? 0x80008000u : 0u, -1, ws, 0, 0, 0};
    for (int i = 0; i < 16; ++i)
        if (per == 1 << i) a.page_shift = i;
    return hip_status(c->dtype == PROX_BF16 ? launch_attn_bf16(a, stream) : launch_attn_f16(a, stream));
}

}  // extern "C"
