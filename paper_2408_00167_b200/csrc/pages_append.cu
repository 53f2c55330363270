// Append of K and V rows to the paged 8-bit cache (pages.cuh), K rotated to its position on the way.
//
//   scale = max |x| / 448 over the finite elements of a page's 64 rows of one head, code = e4m3(x / scale), round to nearest,
//   ties to even, beyond the range to the largest
//
// Bandwidth: rows of 2 or 4 bytes an element in, a byte an element out.  A CTA takes one page of K or V of some KV heads: 8 threads for each
// eight of a row's elements hold the page in registers (eight rows each), so that its rows are read once, the largest
// element is found by shuffles and one exchange through shared memory, and codes leave as 64-bit stores.  The heads of a CTA
// share the page's cosines and sines.  Rows behind the last full page go to the open rows.  The request's open rows are read by the
// CTA of its first page and written by the CTA of its last: both are the same CTA, page after page, reads before writes.
#include "pages.cuh"
#include "rotate.cuh"
#include "score_tc_common.cuh"

namespace finch {
namespace {

constexpr int kHeadsPlain = 4;              // heads of a CTA where nothing turns
constexpr int kPasses = 8;                  // rows that a thread holds
constexpr int kRowsPass = kPage / kPasses;  // rows of the CTA and pass

constexpr uint64_t kMinusZero2 = 0x8000000080000000ull;  // fma2 with it is a multiplication

struct AppendArgs {
    ModelView mv;
    PagesView pg;
    PagedView bv;
    TensorView k, v;
    const int *pos;
    int *out_len;
    int *status;
    int heads_per_cta;
};

__device__ __forceinline__ uint2 to_e4m3(const float (&x)[kRotVec]) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i], x[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2], x[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
        w[i] = (uint32_t)lo | (uint32_t)hi << 16;
    }
    return make_uint2(w[0], w[1]);
}

// ROPE: K turns.  The registers of the turn would cost the plain kernel half of the pages that an SM has in flight.
template <typename T, int LPR, bool ROPE>
__global__ void __launch_bounds__(kRowsPass * LPR, (sizeof(T) == 2 && !ROPE ? 768 : 512) / (kRowsPass * LPR)) append_kernel(AppendArgs p, const __grid_constant__ finch_rope rope) {
    constexpr int kThreads = kRowsPass * LPR, kWarps = kThreads / 32;
    extern __shared__ float2 table[];  // [kPage][rotary_dim / 2]
    __shared__ double freq[128];
    __shared__ float warp_max[2][kWarps];
    dependency_wait();
    const ModelView &mv = p.mv;
    const int b = blockIdx.y, groups = (mv.Hkv + p.heads_per_cta - 1) / p.heads_per_cta;
    const int l = blockIdx.z / groups, h0 = blockIdx.z % groups * p.heads_per_cta, page0 = blockIdx.x / 2;
    const bool is_k = blockIdx.x % 2 == 0;
    const PagedInfo u = paged_info(p.pg, p.bv, b, true);
    const bool speaks = blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0;
    const bool fits = u.ok && (u.len + u.n) / kPage <= p.pg.table_width;
    if (!fits) {
        if (speaks) {
            atomicOr(p.status, FINCH_DEV_BAD_BATCH);
            if (p.out_len) p.out_len[b] = p.bv.len[b];
        }
        return;
    }
    if (speaks && p.out_len) p.out_len[b] = u.len + u.n;
    if (u.n == 0) return;
    const int waiting = u.len % kPage;                    // open rows in front of the new ones
    const int full = (waiting + u.n) / kPage;             // pages that are full now
    const bool turns = ROPE && is_k;
    const int half = turns ? rope.rotary_dim / 2 : 0;
    if (turns) {
        for (int i = threadIdx.x; i < half; i += kThreads) freq[i] = rope.inv_freq[i];
    }
    const int at = threadIdx.x % LPR, row_of = threadIdx.x / LPR;
    const bool live = at * kRotVec < mv.d;
    int turn = 0;  // buffer of warp_max
    // The CTA of page 0 also takes the rows that stay open.
    const TensorView &in = is_k ? p.k : p.v;
    for (int page = page0; page <= full; page = page0 == 0 && page < full ? full : full + 1) {
        if (page == full && page0 != 0) return;
        const int first = page * kPage - waiting;          // new row in the page's first slot (negative: an open row)
        const int from = max(0, -first), to = min(kPage, u.n - first);   // slots with new rows
        if (from >= to) continue;                          // nothing stays open
        int number = 0;
        if (page < full) {
            number = p.pg.table[(int64_t)b * p.pg.table_width + u.len / kPage + page];
            if (number < 0 || number >= p.pg.n_pages) {
                if (threadIdx.x == 0) atomicOr(p.status, FINCH_DEV_BAD_INDEX);
                continue;
            }
        }
        for (int i = 0; i < p.heads_per_cta; ++i) {
            const int h = h0 + i;
            if (h >= mv.Hkv) break;
            const T *src = (const T *)in.ptr + l * in.stride_layer + h * in.stride_head + (int64_t)(u.row0 + first) * in.stride_tok;
            T *open = (T *)(is_k ? p.pg.open_k : p.pg.open_v) + p.pg.open_row(mv, l, u.slot, h) * mv.d;
            Eight<T> x[kPasses];
#pragma unroll
            for (int a = 0; a < kPasses; ++a) {
                const int slot = a * kRowsPass + row_of;
                x[a].zero();
                if (live && slot < to) {
                    if (slot >= from)
                        x[a].load(src + slot * in.stride_tok + at * kRotVec);
                    else if (page < full)
                        x[a].load(open + slot * mv.d + at * kRotVec);
                }
            }
            if (turns) {
                if (i == 0) {  // the page's cosines and sines, under the loads of the first head
                    __syncthreads();
                    rotary_table(table + from * half, rope, freq, to - from,
                                 [&](int r) { return p.pos ? p.pos[u.row0 + first + from + r] : u.len + first + from + r; });
                    __syncthreads();
                }
#pragma unroll
                for (int a = 0; a < kPasses; ++a) {
                    const int slot = a * kRowsPass + row_of;
                    const bool fresh = slot >= from && slot < to;
                    if (!__any_sync(0xffffffffu, fresh)) continue;
                    float y[kRotVec];
                    x[a].get(y);
                    rotate8<LPR>(y, table + (fresh ? slot : from) * half, at, rope.rotary_dim, rope.pairing);
                    if (fresh) x[a].set(y);  // a row waits, and is quantised, in the model's type
                }
            }
            if (page == full) {  // new rows of the page that stays open
#pragma unroll
                for (int a = 0; a < kPasses; ++a) {
                    const int slot = a * kRowsPass + row_of;
                    if (live && slot >= from && slot < to) x[a].store(open + slot * mv.d + at * kRotVec);
                }
                continue;
            }
            uint32_t bits = 0;
#pragma unroll
            for (int a = 0; a < kPasses; ++a) x[a].fold_magnitude(bits);
            float top = __uint_as_float(Eight<T>::magnitude(bits));
            const bool finite = !__any_sync(0xffffffffu, !(top < INFINITY));  // of this warp's elements
            if (!finite) {
                top = 0.f;
#pragma unroll
                for (int a = 0; a < kPasses; ++a) {
                    float y[kRotVec];
                    x[a].get(y);
#pragma unroll
                    for (int e = 0; e < kRotVec; ++e) top = fmaxf(top, fabsf(y[e]) < INFINITY ? fabsf(y[e]) : 0.f);
                }
            }
#pragma unroll
            for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
            turn ^= 1;  // a warp that is here has passed the barrier behind the other buffer's last readers
            if (threadIdx.x % 32 == 0) warp_max[turn][threadIdx.x / 32] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, warp_max[turn][w]);
            const float scale = __fdiv_rn(top, kE4m3Max);
            const int64_t ph = p.pg.page_head(mv, l, number, h);
            uint8_t *dst = (is_k ? p.pg.k : p.pg.v) + ph * kPage * mv.d + row_of * mv.d + at * kRotVec;
            // a scale near an end of fp32's range, and what it divides, move towards the middle first
            const float lift = scale < 0x1p-64f ? 0x1p64f : (scale > 0x1p64f ? 0x1p-64f : 1.f);
            const float by = scale > 0.f ? scale * lift : 1.f, inv = __frcp_rn(by);
            const uint64_t by2 = tc::pack2(by, by), inv2 = tc::pack2(-inv, -inv);
#pragma unroll
            for (int a = 0; a < kPasses; ++a) {
                float y[kRotVec];
                x[a].get_negated(y);
                if (lift != 1.f) {
#pragma unroll
                    for (int e = 0; e < kRotVec; ++e) y[e] *= lift;
                }
                // The correctly rounded quotient: q = x * inv, corrected once by its exact remainder (Markstein's theorem).  With -x
                // in y the remainder is q * by + y, and the signs of zeros come out as a division's.
#pragma unroll
                for (int e = 0; e < kRotVec; e += 2) {
                    const uint64_t y2 = tc::pack2(y[e], y[e + 1]), q = tc::fma2(y2, inv2, kMinusZero2);
                    float c0, c1;
                    tc::unpack2(tc::fma2(tc::fma2(q, by2, y2), inv2, q), c0, c1);
                    if (!finite) {  // an infinity has no remainder
                        c0 = fabsf(y[e]) < INFINITY ? c0 : -y[e];
                        c1 = fabsf(y[e + 1]) < INFINITY ? c1 : -y[e + 1];
                    }
                    y[e] = c0, y[e + 1] = c1;
                }
                if (live) *(uint2 *)(dst + a * kRowsPass * mv.d) = to_e4m3(y);
            }
            if (threadIdx.x == 0) (is_k ? p.pg.k_scale : p.pg.v_scale)[ph] = scale;
        }
    }
}

template <typename T, int LPR, bool ROPE>
cudaError_t launch(const Ctx &ctx, AppendArgs p, const finch_rope &rope, cudaStream_t stream) {
    const int pages = (kPage - 1 + p.bv.max_new + kPage - 1) / kPage;  // a request can touch
    // Heads that share a page's cosines and sines, fewer where that leaves SMs without work.
    int per = ROPE ? p.mv.Hkv : kHeadsPlain;
    while (per > 1 && 2 * (int64_t)pages * p.bv.batch * p.mv.L * ((p.mv.Hkv + per - 1) / per) < 8 * ctx.sm_count) per = (per + 1) / 2;
    p.heads_per_cta = per;
    const size_t smem = ROPE ? (size_t)kPage * (rope.rotary_dim / 2) * sizeof(float2) : 0;
    if (smem > 48 * 1024 - 4096) {
        const int bit = kSmemAppend + (sizeof(T) == 4);
        if (!ctx.smem_ready(bit)) {
            cudaError_t e = cudaFuncSetAttribute(append_kernel<T, LPR, ROPE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPage * 128 * sizeof(float2));
            if (e != cudaSuccess) return e;
            ctx.smem_set(bit);
        }
    }
    ctx.launches += 1;
    return launch_chained(append_kernel<T, LPR, ROPE>, dim3(2 * pages, p.bv.batch, p.mv.L * ((p.mv.Hkv + per - 1) / per)),
                          dim3(kRowsPass * LPR), smem, stream, p, rope);
}

template <typename T, bool ROPE>
cudaError_t launch_d(const Ctx &ctx, const AppendArgs &p, const finch_rope &rope, cudaStream_t stream) {
    if (p.mv.d <= 32) return launch<T, 4, ROPE>(ctx, p, rope, stream);
    if (p.mv.d <= 64) return launch<T, 8, ROPE>(ctx, p, rope, stream);
    if (p.mv.d <= 128) return launch<T, 16, ROPE>(ctx, p, rope, stream);
    return launch<T, 32, ROPE>(ctx, p, rope, stream);
}

}  // namespace

cudaError_t launch_pages_append(const Ctx &ctx, const PagesView &pg, const PagedView &bv, const TensorView &k, const TensorView &v,
                                const int *pos, const finch_rope *rope, int *out_len, cudaStream_t stream) {
    if (bv.batch == 0) return cudaSuccess;
    const AppendArgs p = {ctx.model, pg, bv, k, v, pos, out_len, ctx.d_status, 1};
    static const finch_rope none = {};
    if (ctx.model.elem_bytes == 4)
        return rope ? launch_d<float, true>(ctx, p, *rope, stream) : launch_d<float, false>(ctx, p, none, stream);
    return rope ? launch_d<__nv_bfloat16, true>(ctx, p, *rope, stream) : launch_d<__nv_bfloat16, false>(ctx, p, none, stream);
}

}  // namespace finch
