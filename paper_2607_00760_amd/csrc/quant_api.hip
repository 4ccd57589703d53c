// quant_api.hip -- C ABI of the operators around the 8-bit KV cache and of
// the norm-and-rotation pass (see include/mosaic.h): argument validation,
// workspace layout, launches.  No C++ exception crosses the ABI.
#include <cstdarg>
#include <cstdio>

#include "../../include/mosaic.h"
#include "norm_rope.h"
#include "quant.h"

using namespace mosaic;

namespace {

mosaic_status fail(mosaic_status st, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return st;
}

mosaic_status done(hipError_t e, const char *what) {
    if (e != hipSuccess) return fail(MOSAIC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    set_last_error("");
    return MOSAIC_OK;
}

constexpr int MAX_THREADS = 0x7fffffff;                    // of a launch along its first dimension

bool off16(const void *p) { return (uintptr_t)p % 16 != 0; }
uint64_t align256(uint64_t x) { return (x + 255) & ~uint64_t(255); }

mosaic_status quant_shape(const mosaic_quant_cache *c) {
    if (!c) return fail(MOSAIC_ERR_INVALID, "NULL cache");
    if (c->head_dim != D) return fail(MOSAIC_ERR_UNSUPPORTED, "head_dim %d", c->head_dim);
    if (c->block_len != 32 && c->block_len != 64) return fail(MOSAIC_ERR_UNSUPPORTED, "block_len %d: 32 or 64", c->block_len);
    if (c->dtype != MOSAIC_FP16 && c->dtype != MOSAIC_BF16) return fail(MOSAIC_ERR_INVALID, "dtype %d", c->dtype);
    if (c->format != MOSAIC_E4M3 && c->format != MOSAIC_INT8) return fail(MOSAIC_ERR_INVALID, "format %d", c->format);
    if (c->num_seqs < 1 || c->num_kv_heads < 1 || c->group_size < 1 || c->group_size > 8 || c->max_blocks < 1)
        return fail(MOSAIC_ERR_INVALID, "num_seqs %d, num_kv_heads %d, group_size %d, max_blocks %d", c->num_seqs, c->num_kv_heads,
                    c->group_size, c->max_blocks);
    const long long pairs = (long long)c->num_seqs * c->num_kv_heads;
    if (pairs > Q_PAIRS) return fail(MOSAIC_ERR_UNSUPPORTED, "%lld (sequence, kv head) pairs: at most %d", pairs, Q_PAIRS);
    if ((long long)c->max_blocks * c->block_len > 0x3fffffff || pairs * c->max_blocks > 0x3fffffff)
        return fail(MOSAIC_ERR_UNSUPPORTED, "%d blocks of %d tokens for %lld pairs", c->max_blocks, c->block_len, pairs);
    return MOSAIC_OK;
}

mosaic_status quant_arrays(const mosaic_quant_cache *c, QCache &q) {
    const mosaic_status st = quant_shape(c);
    if (st != MOSAIC_OK) return st;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->bound_scale || !c->bounds || !c->k_tail || !c->v_tail || !c->lens ||
        !c->arrivals || !c->refused)
        return fail(MOSAIC_ERR_INVALID, "NULL array in the cache");
    if (off16(c->k) || off16(c->v) || off16(c->bounds) || off16(c->k_tail) || off16(c->v_tail))
        return fail(MOSAIC_ERR_INVALID, "codes, bounds and tails must be 16-byte aligned");
    if (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale | (uintptr_t)c->bound_scale | (uintptr_t)c->lens | (uintptr_t)c->arrivals |
         (uintptr_t)c->refused) % 4)
        return fail(MOSAIC_ERR_INVALID, "scales and lengths must be 4-byte aligned");
    q = QCache{c->num_seqs, c->num_kv_heads, c->group_size, c->max_blocks, c->max_blocks * c->block_len, (uint8_t *)c->k, (uint8_t *)c->v, c->k_scale, c->v_scale,
               c->bound_scale, c->bounds, (uint16_t *)c->k_tail, (uint16_t *)c->v_tail, c->lens, c->arrivals, c->refused};
    return MOSAIC_OK;
}

struct QuantWs { uint64_t scores, list, total; };          // the attention's part first
QuantWs quant_ws(const mosaic_quant_cache *c) {
    const uint64_t pairs = (uint64_t)c->num_seqs * c->num_kv_heads;
    QuantWs w;
    w.scores = align256(quant_attn_ws_bytes((int)pairs));
    w.list = w.scores + align256(pairs * q_score_stride(c->max_blocks) * 4);
    w.total = w.list + align256(pairs * c->max_blocks * 4);
    return w;
}

mosaic_status attend_args(const mosaic_quant_cache *c, const void *q, const float *out, const void *ws, size_t ws_bytes, QCache &qc) {
    const mosaic_status st = quant_arrays(c, qc);
    if (st != MOSAIC_OK) return st;
    if (!q || !out || !ws) return fail(MOSAIC_ERR_INVALID, "NULL argument");
    if (off16(q) || off16(out) || (uintptr_t)ws % 256)
        return fail(MOSAIC_ERR_INVALID, "q and out must be 16-byte, the workspace 256-byte aligned");
    const uint64_t need = quant_ws(c).total;
    if (ws_bytes < need) return fail(MOSAIC_ERR_INVALID, "workspace %zu < %llu", ws_bytes, (unsigned long long)need);
    return MOSAIC_OK;
}

hipError_t attend(const mosaic_quant_cache *c, const QCache &qc, const void *q, float *out, float scale, const QSel &sel, void *ws,
                  void *stream) {
    const auto f = c->format == MOSAIC_INT8 ? launch_quant_attn_int8 : launch_quant_attn_e4m3;
    return f(qc, c->block_len, c->dtype, (const uint16_t *)q, scale, sel, ws, out, (hipStream_t)stream);
}

// strides of a tensor of n0 x n1 x n2 rows that leave some row misaligned (the
// stride of a dimension of one row may be anything)
bool bad_strides(const int64_t *s, int n0, int n1, int n2) {
    return ((n0 > 1 ? s[0] : 0) | (n1 > 1 ? s[1] : 0) | (n2 > 1 ? s[2] : 0)) % 8 != 0;
}

// rows of an output that share memory, along one of its dimensions
bool rows_overlap(const int64_t *s, int n0, int n1, int n2) {
    const int n[3] = {n0, n1, n2};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && s[i] > -D && s[i] < D) return true;
    return false;
}

}  // namespace

extern "C" {

mosaic_status mosaic_quant_append(const mosaic_quant_cache *c, const void *k, const void *v, const int64_t *k_strides,
                                  const int64_t *v_strides, const int32_t *new_lens, int32_t max_new, void *stream) {
    QCache q;
    const mosaic_status st = quant_arrays(c, q);
    if (st != MOSAIC_OK) return st;
    if (!k || !v || !k_strides || !v_strides) return fail(MOSAIC_ERR_INVALID, "NULL argument");
    if (max_new < 0) return fail(MOSAIC_ERR_INVALID, "max_new %d", max_new);
    const int S = c->num_seqs, H = c->num_kv_heads;
    if (off16(k) || off16(v) || bad_strides(k_strides, S, H, max_new) || bad_strides(v_strides, S, H, max_new))
        return fail(MOSAIC_ERR_INVALID, "k/v must be 16-byte aligned, their strides multiples of 8 elements");
    if ((uintptr_t)new_lens % 4) return fail(MOSAIC_ERR_INVALID, "new_lens must be 4-byte aligned");
    const long long room = (long long)c->max_blocks * c->block_len;
    if (!new_lens && max_new > room) return fail(MOSAIC_ERR_CAPACITY, "%d tokens for a cache of %lld", max_new, room);
    if (max_new == 0) return done(hipSuccess, "");
    if (max_new > MAX_THREADS / 8) return fail(MOSAIC_ERR_UNSUPPORTED, "max_new %d: at most %d", max_new, MAX_THREADS / 8);
    const QNew n{(const uint16_t *)k, (const uint16_t *)v, k_strides[0], k_strides[1], k_strides[2], v_strides[0], v_strides[1],
                 v_strides[2], new_lens, max_new};
    return done(launch_quant_append(q, c->format, c->block_len, c->dtype, n, (hipStream_t)stream), "append launch");
}

mosaic_status mosaic_quant_workspace_bytes(const mosaic_quant_cache *c, size_t *bytes) {
    if (!bytes) return fail(MOSAIC_ERR_INVALID, "NULL argument");
    const mosaic_status st = quant_shape(c);
    if (st != MOSAIC_OK) return st;
    *bytes = quant_ws(c).total;
    return done(hipSuccess, "");
}

mosaic_status mosaic_quant_decode_attention(const mosaic_quant_cache *c, const void *q, float *out, float sm_scale, void *ws,
                                            size_t ws_bytes, void *stream) {
    QCache qc;
    const mosaic_status st = attend_args(c, q, out, ws, ws_bytes, qc);
    if (st != MOSAIC_OK) return st;
    return done(attend(c, qc, q, out, sm_scale, QSel{1, 1, nullptr}, ws, stream), "attention launch");
}

mosaic_status mosaic_quant_select_attention(const mosaic_quant_cache *c, const void *q, float *out, float sm_scale,
                                            int32_t select_num, int32_t select_den, int32_t *blocks, void *ws, size_t ws_bytes,
                                            void *stream) {
    QCache qc;
    const mosaic_status st = attend_args(c, q, out, ws, ws_bytes, qc);
    if (st != MOSAIC_OK) return st;
    if (select_num < 1 || select_den < select_num) return fail(MOSAIC_ERR_INVALID, "select %d / %d", select_num, select_den);
    if ((uintptr_t)blocks % 4) return fail(MOSAIC_ERR_INVALID, "blocks must be 4-byte aligned");
    const QuantWs w = quant_ws(c);
    int32_t *list = blocks ? blocks : (int32_t *)((uint8_t *)ws + w.list);
    const hipError_t e = launch_quant_select(qc, c->block_len, c->dtype, (const uint16_t *)q, select_num, select_den,
                                             (float *)((uint8_t *)ws + w.scores), list, (hipStream_t)stream);
    if (e != hipSuccess) return done(e, "selection launch");
    return done(attend(c, qc, q, out, sm_scale, QSel{select_num, select_den, list}, ws, stream), "attention launch");
}

mosaic_status mosaic_qk_norm_rope(const mosaic_rows *q, const mosaic_rows *k, const mosaic_rows *v, int32_t num_seqs,
                                  int32_t num_tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t dtype,
                                  const void *q_weight, const void *k_weight, float eps, const void *positions,
                                  int32_t pos_bytes, const int64_t *pos_strides, const float *inv_freq, int32_t rot_dim,
                                  int32_t interleaved, void *stream) {
    if (!q || !k || !positions || !pos_strides || !inv_freq) return fail(MOSAIC_ERR_INVALID, "NULL argument");
    if (head_dim != D) return fail(MOSAIC_ERR_UNSUPPORTED, "head_dim %d", head_dim);
    if (dtype != MOSAIC_FP16 && dtype != MOSAIC_BF16) return fail(MOSAIC_ERR_INVALID, "dtype %d", dtype);
    if (num_seqs < 0 || num_tokens < 0 || q_heads < 1 || kv_heads < 1 || q_heads > 1 << 20 || kv_heads > 1 << 20)
        return fail(MOSAIC_ERR_INVALID, "num_seqs %d, num_tokens %d, q_heads %d, kv_heads %d", num_seqs, num_tokens, q_heads, kv_heads);
    if (rot_dim < 16 || rot_dim > D || rot_dim % 16) return fail(MOSAIC_ERR_UNSUPPORTED, "rot_dim %d: a multiple of 16 up to %d", rot_dim, D);
    if (pos_bytes != 4 && pos_bytes != 8) return fail(MOSAIC_ERR_INVALID, "pos_bytes %d", pos_bytes);
    if (!q_weight != !k_weight) return fail(MOSAIC_ERR_INVALID, "weights of both queries and keys, or of neither");
    if (!(eps >= 0.0f)) return fail(MOSAIC_ERR_INVALID, "eps %g", (double)eps);
    if ((long long)num_seqs * num_tokens > MAX_THREADS / 256)
        return fail(MOSAIC_ERR_UNSUPPORTED, "%d x %d tokens: at most %d", num_seqs, num_tokens, MAX_THREADS / 256);
    if ((uintptr_t)positions % pos_bytes || (uintptr_t)inv_freq % 4 || off16(q_weight) || off16(k_weight))
        return fail(MOSAIC_ERR_INVALID, "misaligned positions, inv_freq or weights");
    const mosaic_rows *rows[3] = {q, k, v};
    NormRope a{};
    for (int i = 0; i < 3; ++i) {
        const mosaic_rows *r = rows[i];
        if (!r) continue;
        if (!r->in || !r->out) return fail(MOSAIC_ERR_INVALID, "NULL rows");
        const int heads = i == 0 ? q_heads : kv_heads;
        if (off16(r->in) || off16(r->out) || bad_strides(r->in_strides, num_seqs, num_tokens, heads) ||
            bad_strides(r->out_strides, num_seqs, num_tokens, heads))
            return fail(MOSAIC_ERR_INVALID, "rows must be 16-byte aligned, their strides multiples of 8 elements");
        if (rows_overlap(r->out_strides, num_seqs, num_tokens, heads))
            return fail(MOSAIC_ERR_INVALID, "rows of an output overlap");
        (i == 0 ? a.q : (i == 1 ? a.k : a.vp)) = NormRope::Part{(const uint16_t *)r->in, (uint16_t *)r->out, r->in_strides[0], r->in_strides[1],
                                                               r->in_strides[2], r->out_strides[0], r->out_strides[1], r->out_strides[2]};
    }
    if (num_seqs == 0 || num_tokens == 0) return done(hipSuccess, "");
    a.qw = (const uint16_t *)q_weight;
    a.kw = (const uint16_t *)k_weight;
    a.inv_freq = inv_freq;
    a.pos = positions;
    a.pos_seq = pos_strides[0];
    a.pos_tok = pos_strides[1];
    a.seqs = num_seqs;
    a.n = num_tokens;
    a.hq = q_heads;
    a.hkv = kv_heads;
    a.half = rot_dim / 2;
    a.pos64 = pos_bytes == 8;
    a.v = v != nullptr;
    a.eps = eps;
    return done(launch_norm_rope(a, dtype, interleaved, (hipStream_t)stream), "norm and rotation launch");
}

}  // extern "C"
