// Host side of the operators around the step: rotation, attention, the paged 8-bit cache.  Argument checks, workspace, dispatch.
#include <math.h>
#include <string.h>

#include "attend.cuh"

using namespace finch;

namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
finch_status cuda_status(cudaError_t e) {
    if (e == cudaSuccess) return FINCH_OK;
    (void)cudaGetLastError();
    return FINCH_ERR_CUDA;
}

// Kernels run on the device that is current: it has to be the context's, whose memory they write.
finch_status check_device(const finch_ctx *ctx) {
    if (ctx->dry) return FINCH_ERR_UNSUPPORTED;
    return ctx->on_own_device() ? FINCH_OK : FINCH_ERR_INVALID_ARG;
}

finch_status check_rope(const finch_ctx *ctx, const finch_rope *rope) {
    if (!rope) return FINCH_OK;
    if (rope->rotary_dim <= 0 || rope->rotary_dim > ctx->model.d || (rope->pairing != 0 && rope->pairing != 1)) return FINCH_ERR_INVALID_ARG;
    if (rope->rotary_dim % 16) return FINCH_ERR_UNSUPPORTED;
    return isfinite(rope->magnitude) ? FINCH_OK : FINCH_ERR_INVALID_ARG;
}

// The same rows in place, or no byte in common.
bool same_view(const finch_tensor *a, const finch_tensor *b) {
    return a->ptr == b->ptr && a->stride_layer == b->stride_layer && a->stride_head == b->stride_head && a->stride_tok == b->stride_tok;
}

struct AttendWs {
    size_t rows, ml_off, total;
};
AttendWs attend_ws(const ModelView &mv, int64_t total_q, int sms, int rows_per_cta) {
    AttendWs w;
    w.rows = attend_partial_rows(mv, total_q, sms, rows_per_cta);
    w.ml_off = align_up(w.rows * mv.d * sizeof(float));
    w.total = w.ml_off + align_up(w.rows * sizeof(float2));
    if (w.total == 0) w.total = kAlign;
    return w;
}
int sm_count(const finch_ctx *ctx) { return ctx->sm_count > 0 ? ctx->sm_count : 148; }
// rows of the CTAs that there can be splits of: the larger of the two paths' (a batch's tensors may keep it off the tensor cores)
AttendWs attend_ws(const finch_ctx *ctx, int64_t total_q) { return attend_ws(ctx->model, total_q, sm_count(ctx), kAttendTcRows); }
// pieces of units of the paged cache's attention
AttendWs pages_ws(const finch_ctx *ctx) {
    AttendWs w;
    w.rows = (size_t)pages_ctas(sm_count(ctx)) * 2 * kPagesRows;
    w.ml_off = align_up(w.rows * ctx->model.d * sizeof(float));
    w.total = w.ml_off + align_up(w.rows * sizeof(float2));
    return w;
}

AttendOut attend_out(const finch_tensor *out, float *row_lse, void *ws, const AttendWs &w) {
    AttendOut o = {(char *)out->ptr, out->stride_layer, out->stride_head, out->stride_tok, row_lse, (float *)ws, (float2 *)((char *)ws + w.ml_off), 1};
    return o;
}

finch_status check_paged(const finch_ctx *ctx, const finch_pages *pg, const finch_paged_batch *b, bool append) {
    if (!ctx || !pg || !b) return FINCH_ERR_INVALID_ARG;
    if (b->batch < 0 || b->batch > ctx->cfg.max_batch || b->max_len < 0) return FINCH_ERR_INVALID_ARG;
    const int32_t total = append ? b->total_new : b->total_q, most = append ? b->max_new : b->max_q;
    if (total < 0 || most < 0 || most > total) return FINCH_ERR_INVALID_ARG;
    if (!append && most > ctx->cfg.max_prompt) return FINCH_ERR_INVALID_ARG;
    const int64_t tokens = (int64_t)b->max_len + (append ? most : 0);
    if (tokens > ctx->cfg.max_candidates) return FINCH_ERR_INVALID_ARG;
    if (b->batch == 0) return FINCH_OK;
    if (!b->len || !(append ? b->new_off : b->q_off)) return FINCH_ERR_INVALID_ARG;
    if (pg->n_open <= 0 || !pg->open_k || !pg->open_v) return FINCH_ERR_INVALID_ARG;
    if (!pg->open_slot && pg->n_open < b->batch) return FINCH_ERR_INVALID_ARG;
    if (pg->n_pages < 0 || pg->table_width < 0) return FINCH_ERR_INVALID_ARG;
    const int64_t pages = tokens / FINCH_PAGE_TOKENS;  // full ones, of the longest request
    if (pages > 0 && (pages > pg->table_width || pg->n_pages <= 0 || !pg->k || !pg->v || !pg->k_scale || !pg->v_scale || !pg->table))
        return FINCH_ERR_INVALID_ARG;
    if (!aligned16(pg->k) || !aligned16(pg->v) || !aligned16(pg->open_k) || !aligned16(pg->open_v)) return FINCH_ERR_BAD_LAYOUT;
    return FINCH_OK;
}

}  // namespace

extern "C" {

finch_status finch_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor, double original, double low,
                                    double high, double *inv_freq) {
    if (!inv_freq || rotary_dim <= 0 || rotary_dim % 2 || rotary_dim > 256) return FINCH_ERR_INVALID_ARG;
    if (!(theta >= 1.0) || isinf(theta) || scaling < FINCH_ROPE_PLAIN || scaling > FINCH_ROPE_PARTS) return FINCH_ERR_INVALID_ARG;
    if (scaling != FINCH_ROPE_PLAIN && (!(factor >= 1.0) || isinf(factor))) return FINCH_ERR_INVALID_ARG;
    if (scaling == FINCH_ROPE_PARTS && (!(original > 0.0) || isinf(original) || !(low >= 0.0) || !(high > low) || isinf(high)))
        return FINCH_ERR_INVALID_ARG;
    if (scaling == FINCH_ROPE_BASE && rotary_dim == 2) return FINCH_ERR_INVALID_ARG;
    if (scaling == FINCH_ROPE_BASE) theta *= pow(factor, rotary_dim / (rotary_dim - 2.0));
    const double two_pi = 6.283185307179586476925;
    for (int t = 0; t < rotary_dim / 2; ++t) {
        double f = pow(theta, -2.0 * t / rotary_dim);
        if (scaling == FINCH_ROPE_LINEAR) f /= factor;
        if (scaling == FINCH_ROPE_PARTS) {
            double keep = (original * f / two_pi - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
            f = keep * f + (1.0 - keep) * f / factor;
        }
        inv_freq[t] = f;
    }
    return FINCH_OK;
}

finch_status finch_rope_init(finch_rope *out, int32_t rotary_dim, int32_t pairing, float magnitude, const double *inv_freq) {
    if (!out || !inv_freq || rotary_dim <= 0 || rotary_dim > 256) return FINCH_ERR_INVALID_ARG;
    if (pairing != 0 && pairing != 1) return FINCH_ERR_INVALID_ARG;
    if (!isfinite(magnitude)) return FINCH_ERR_INVALID_ARG;
    if (rotary_dim % 16) return FINCH_ERR_UNSUPPORTED;
    for (int t = 0; t < rotary_dim / 2; ++t)
        if (!(fabs(inv_freq[t]) <= 2.0)) return FINCH_ERR_INVALID_ARG;  // angles of any position stay below 2^32
    memset(out, 0, sizeof(*out));
    out->rotary_dim = rotary_dim;
    out->pairing = pairing;
    out->magnitude = magnitude;
    memcpy(out->inv_freq, inv_freq, sizeof(double) * (rotary_dim / 2));
    return FINCH_OK;
}

finch_status finch_rotate(finch_ctx *ctx, const finch_tensor *q, const finch_tensor *k, int32_t tokens, const int32_t *pos,
                          const finch_rope *rope, const void *q_weight, const void *k_weight, float eps, const finch_tensor *out_q,
                          const finch_tensor *out_k, void *cuda_stream) {
    if (!ctx || tokens < 0 || !q || !k || !out_q || !out_k) return FINCH_ERR_INVALID_ARG;
    finch_status s;
    const bool none = tokens == 0;
    const finch_tensor *in[2] = {q, k}, *out[2] = {out_q, out_k};
    const int heads[2] = {ctx->model.Hq, ctx->model.Hkv};
    for (int i = 0; i < 2; ++i) {
        if ((s = check_tensor(ctx, in[i], true))) return s;
        if ((s = check_tensor(ctx, out[i], true))) return s;
        if ((in[i]->ptr == nullptr) != (out[i]->ptr == nullptr)) return FINCH_ERR_INVALID_ARG;
    }
    if (!none && !q->ptr && !k->ptr) return FINCH_ERR_INVALID_ARG;
    if ((s = check_rope(ctx, rope))) return s;
    if (rope && !pos && !none) return FINCH_ERR_INVALID_ARG;
    if (!rope && !q_weight && !k_weight) return FINCH_ERR_INVALID_ARG;  // nothing to do
    if ((q_weight || k_weight) && (!(eps >= 0.f) || isinf(eps))) return FINCH_ERR_INVALID_ARG;
    if (!aligned16(q_weight) || !aligned16(k_weight)) return FINCH_ERR_BAD_LAYOUT;
    // rows are independent and each is read before it is written: in place, or apart
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            if (!(i == j && same_view(out[i], in[j])) && views_overlap(ctx, out[i], tokens, heads[i], in[j], tokens, heads[j]))
                return FINCH_ERR_INVALID_ARG;
        }
    if (views_overlap(ctx, out_q, tokens, heads[0], out_k, tokens, heads[1])) return FINCH_ERR_INVALID_ARG;
    if ((s = check_device(ctx))) return s;
    return cuda_status(launch_rotate(*ctx, view_of(q), view_of(k), view_of(out_q), view_of(out_k), tokens, pos, rope, q_weight, k_weight,
                                     eps, (cudaStream_t)cuda_stream));
}

finch_status finch_attend_workspace_bytes(const finch_ctx *ctx, const finch_batch *batch, size_t *out) {
    if (!out) return FINCH_ERR_INVALID_ARG;
    finch_status s = check_batch(ctx, batch);
    if (s) return s;
    *out = attend_ws(ctx, batch->total_q).total;
    return FINCH_OK;
}

finch_status finch_attend_plan(const finch_ctx *ctx, const finch_batch *batch, int32_t *path, int32_t *cluster, int32_t *splits) {
    if (!path) return FINCH_ERR_INVALID_ARG;
    finch_status s = check_batch(ctx, batch);
    if (s) return s;
    const size_t rows = attend_ws(ctx, batch->total_q).rows;
    int c = 1, n = 1;
    *path = FINCH_ATTEND_MULTIPLY_ADD;
    if (attend_tc_supported(*ctx))
        attend_tc_plan(*ctx, view_of(batch), rows, *path, c, n);
    else
        n = attend_simt_splits(*ctx, view_of(batch), rows);
    if (cluster) *cluster = c;
    if (splits) *splits = n;
    return FINCH_OK;
}

finch_status finch_attend(finch_ctx *ctx, const finch_tensor *q, const finch_tensor *cache_k, const finch_tensor *cache_v,
                          const finch_tensor *chunk_k, const finch_tensor *chunk_v, const finch_batch *batch, int32_t causal,
                          const finch_tensor *out, float *row_lse, void *ws, size_t ws_bytes, void *cuda_stream) {
    finch_status s = check_batch(ctx, batch);
    if (s) return s;
    const bool no_q = batch->total_q == 0, no_cache = batch->total_cache == 0, no_chunk = batch->total_chunk == 0;
    if ((s = check_tensor(ctx, q, no_q))) return s;
    if ((s = check_tensor(ctx, cache_k, no_cache))) return s;
    if ((s = check_tensor(ctx, cache_v, no_cache))) return s;
    if ((s = check_tensor(ctx, chunk_k, no_chunk))) return s;
    if ((s = check_tensor(ctx, chunk_v, no_chunk))) return s;
    if ((s = check_tensor(ctx, out, no_q))) return s;
    if (causal != 0 && causal != 1) return FINCH_ERR_INVALID_ARG;
    if (batch->row_norm) return FINCH_ERR_INVALID_ARG;  // a weighting of scores; attention rows sum to one
    const finch_tensor *ins[4] = {cache_k, cache_v, chunk_k, chunk_v};
    for (int i = 0; i < 4; ++i)
        if (views_overlap(ctx, out, batch->total_q, ctx->model.Hq, ins[i], i < 2 ? batch->total_cache : batch->total_chunk, ctx->model.Hkv))
            return FINCH_ERR_INVALID_ARG;
    if (views_overlap(ctx, out, batch->total_q, ctx->model.Hq, q, batch->total_q, ctx->model.Hq)) return FINCH_ERR_INVALID_ARG;
    // the CTAs (and warps) that share a row read its extra term, and one of them writes its row_lse
    if (row_lse && batch->prompt_self_lse) {
        const uintptr_t a = (uintptr_t)row_lse, n = (uintptr_t)batch->prompt_self_lse;
        const uintptr_t bytes = (uintptr_t)ctx->model.L * ctx->model.Hq * batch->total_q * sizeof(float);
        if (a < n + bytes && n < a + bytes) return FINCH_ERR_INVALID_ARG;
    }
    if (!ws) return FINCH_ERR_INVALID_ARG;
    if (!aligned16(ws)) return FINCH_ERR_BAD_LAYOUT;
    const AttendWs w = attend_ws(ctx, batch->total_q);
    if (ws_bytes < w.total) return FINCH_ERR_WORKSPACE_TOO_SMALL;
    if ((s = check_device(ctx))) return s;
    const AttendOut o = attend_out(out, row_lse, ws, w);
    const TensorView qv = view_of(q), ck = view_of(cache_k), cv = view_of(cache_v), hk = view_of(chunk_k), hv = view_of(chunk_v);
    const BatchView bv = view_of(batch);
    cudaError_t e = cudaErrorNotSupported;
    if (attend_tc_supported(*ctx))
        e = launch_attend_tc(*ctx, qv, ck, cv, hk, hv, bv, causal, o, w.rows, (cudaStream_t)cuda_stream);
    if (e == cudaErrorNotSupported)
        e = launch_attend_simt(*ctx, qv, ck, cv, hk, hv, bv, causal, o, w.rows, (cudaStream_t)cuda_stream);
    return cuda_status(e);
}

finch_status finch_pages_append(finch_ctx *ctx, const finch_pages *pages, const finch_paged_batch *batch, const finch_tensor *new_k,
                                const finch_tensor *new_v, const finch_rope *rope, const int32_t *pos, int32_t *out_len,
                                void *cuda_stream) {
    finch_status s = check_paged(ctx, pages, batch, true);
    if (s) return s;
    const bool none = batch->total_new == 0;
    if ((s = check_tensor(ctx, new_k, none))) return s;
    if ((s = check_tensor(ctx, new_v, none))) return s;
    if ((s = check_rope(ctx, rope))) return s;
    // every CTA of a request reads its length: the new one may not take its place under them
    if (out_len && batch->batch > 0) {
        const uintptr_t a = (uintptr_t)out_len, n = (uintptr_t)batch->len, bytes = (uintptr_t)batch->batch * sizeof(int32_t);
        if (a < n + bytes && n < a + bytes) return FINCH_ERR_INVALID_ARG;
    }
    if ((s = check_device(ctx))) return s;
    return cuda_status(launch_pages_append(*ctx, view_of(pages), view_of(batch), view_of(new_k), view_of(new_v), pos, rope, out_len,
                                           (cudaStream_t)cuda_stream));
}

finch_status finch_pages_workspace_bytes(const finch_ctx *ctx, const finch_paged_batch *batch, size_t *out) {
    if (!ctx || !batch || !out || batch->batch < 0 || batch->batch > ctx->cfg.max_batch) return FINCH_ERR_INVALID_ARG;
    *out = pages_ws(ctx).total;
    return FINCH_OK;
}

finch_status finch_pages_attend(finch_ctx *ctx, const finch_pages *pages, const finch_paged_batch *batch, const finch_tensor *q,
                                const finch_tensor *out, float *row_lse, void *ws, size_t ws_bytes, void *cuda_stream) {
    finch_status s = check_paged(ctx, pages, batch, false);
    if (s) return s;
    const bool none = batch->total_q == 0;
    if ((s = check_tensor(ctx, q, none))) return s;
    if ((s = check_tensor(ctx, out, none))) return s;
    if (views_overlap(ctx, out, batch->total_q, ctx->model.Hq, q, batch->total_q, ctx->model.Hq)) return FINCH_ERR_INVALID_ARG;
    if (!ws) return FINCH_ERR_INVALID_ARG;
    if (!aligned16(ws)) return FINCH_ERR_BAD_LAYOUT;
    const AttendWs w = pages_ws(ctx);
    if (ws_bytes < w.total) return FINCH_ERR_WORKSPACE_TOO_SMALL;
    if ((s = check_device(ctx))) return s;
    return cuda_status(launch_pages_attend(*ctx, view_of(pages), view_of(batch), view_of(q), attend_out(out, row_lse, ws, w),
                                           (cudaStream_t)cuda_stream));
}

}  // extern "C"
