// RMS norm of every query and key head and the rotary embedding, in one pass over q and k.
//
//   y = x * rsqrt(mean(x^2) + eps) * w      (a head's row, fp32; with weights only)
//   pairs of y turn by position * inv_freq  (rotate.cuh; with a rope only)
//
// Pure bandwidth: every element is read and written once.  A CTA takes up to 8 tokens and all their heads (or some of them, where
// there are too few tokens to fill the SMs): a token's cosines and sines are formed once, in shared memory, and stay in the
// registers of the warps that walk its heads.  A row is LPR lanes with eight elements each, several rows to a warp, and a warp has
// the loads of kAhead rounds in flight.
#include "rotate.cuh"
#include "score_tc_common.cuh"

namespace finch {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotWarps = kRotThreads / 32;
constexpr uint64_t kMinusZero2 = 0x8000000080000000ull;  // fma2 with it is a multiplication

struct RotateArgs {
    TensorView q, k, out_q, out_k;
    const void *q_weight, *k_weight;
    const int *pos;
    int Hq, Hkv, d, tokens;
    int tok_per_cta, heads_per_cta;
    float eps;
};

// ROPE: nothing turns, halves, neighbours (a variant each: together they would spill)
enum { kNone = 0, kHalves = 1, kNeighbours = 2 };
template <typename T, int LPR, int ROPE>
__global__ void __launch_bounds__(kRotThreads, 4) rotate_kernel(RotateArgs p, const __grid_constant__ finch_rope rope) {
    extern __shared__ float2 table[];  // [tok_per_cta][rotary_dim / 2]
    __shared__ double freq[ROPE != kNone ? 128 : 1];
    constexpr int kRows = 32 / LPR;    // rows of a warp and round
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;
    const float inv_d = 1.f / (float)p.d;
    dependency_wait();
    const int l = blockIdx.z, tok0 = blockIdx.x * p.tok_per_cta, h_first = blockIdx.y * p.heads_per_cta;
    const int n_tok = min(p.tok_per_cta, p.tokens - tok0), h_end = min(h_first + p.heads_per_cta, p.Hq + p.Hkv);
    const int half = ROPE != kNone ? rope.rotary_dim / 2 : 0;
    if (ROPE != kNone) {
        for (int i = threadIdx.x; i < half; i += kRotThreads) freq[i] = rope.inv_freq[i];
        __syncthreads();
        rotary_table(table, rope, freq, n_tok, [&](int row) { return p.pos[tok0 + row]; });
        __syncthreads();
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, at = lane % LPR, e0 = at * kRotVec;
    const bool live = e0 < p.d;
    // the warps of the CTA share out its tokens, those of a token its heads
    const int token = warp % p.tok_per_cta, step = kRotWarps / p.tok_per_cta * kRows;
    if (token >= n_tok) return;
    // This lane's part of the turn, y' = y co + partner si: the partner is the pair's other element, in this lane or in lane `other`.
    const bool turns = ROPE != kNone && e0 < rope.rotary_dim, low = e0 < half;
    constexpr bool beside = ROPE == kNeighbours;
    const int other = turns && !beside ? lane - at + (low ? at + half / kRotVec : at - half / kRotVec) : lane;
    const int64_t tok = tok0 + token;
    // The heads [h0, h1) of q or k among those of the CTA; `shift` heads lie in front of the tensor's.
    auto walk = [&](const TensorView &in, const TensorView &out, const void *weights, int shift, int h0, int h1) {
        // co, si times the norm's weights: a row is then (x co + partner si) times its root
        uint64_t co[kRotVec / 2], si[kRotVec / 2];
        {
            Eight<T> w;
            float g[kRotVec], c[kRotVec], n[kRotVec];
            w.zero();
            if (weights && live) w.load((const T *)weights + (int64_t)l * p.d + e0);
            w.get(g);
            if (!weights) {
#pragma unroll
                for (int i = 0; i < kRotVec; ++i) g[i] = 1.f;
            }
            const float2 *cs = table + token * half;
#pragma unroll
            for (int i = 0; i < kRotVec; ++i) {
                const float of_partner = beside ? g[i ^ 1] : __shfl_sync(0xffffffffu, g[i], other);
                c[i] = g[i], n[i] = 0.f;
                if (turns) {
                    const float2 t = cs[beside ? (e0 + i) / 2 : (low ? e0 + i : e0 + i - half)];
                    c[i] *= t.x;
                    n[i] = ((beside ? i % 2 == 0 : low) ? -t.y : t.y) * of_partner;
                }
            }
#pragma unroll
            for (int i = 0; i < kRotVec / 2; ++i) co[i] = tc::pack2(c[2 * i], c[2 * i + 1]), si[i] = tc::pack2(n[2 * i], n[2 * i + 1]);
        }
        int first = max(h0, h_first) + warp / p.tok_per_cta * kRows;  // the warp's first row; this lane's is `row` behind it
        const int row = lane / LPR;
        const int h_last = min(h1, h_end);
        const T *src = (const T *)in.ptr + l * in.stride_layer + tok * in.stride_tok + (first + row - shift) * in.stride_head + e0;
        T *dst = (T *)out.ptr + l * out.stride_layer + tok * out.stride_tok + (first + row - shift) * out.stride_head + e0;
        const int64_t src_step = step * in.stride_head, dst_step = step * out.stride_head;
        Eight<T> x[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) x[a].zero();
        for (; first < h_last; first += kAhead * step) {
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                if (first + row + a * step < h_last && live) x[a].load(src);
                src += src_step;
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                if (first + a * step >= h_last) break;  // the whole warp
                float y[kRotVec];
                x[a].get(y);
                uint64_t y2[kRotVec / 2];
#pragma unroll
                for (int i = 0; i < kRotVec / 2; ++i) y2[i] = tc::fma2(tc::pack2(y[2 * i], y[2 * i + 1]), co[i], kMinusZero2);
                if (ROPE != kNone) {
                    uint64_t z2[kRotVec / 2];
                    if (beside) {
#pragma unroll
                        for (int i = 0; i < kRotVec / 2; ++i) z2[i] = tc::pack2(y[2 * i + 1], y[2 * i]);
                    } else {
                        Eight<T> o = x[a];
                        float z[kRotVec];
                        o.from_lane(other);
                        o.get(z);
#pragma unroll
                        for (int i = 0; i < kRotVec / 2; ++i) z2[i] = tc::pack2(z[2 * i], z[2 * i + 1]);
                    }
                    if (turns) {
#pragma unroll
                        for (int i = 0; i < kRotVec / 2; ++i) y2[i] = tc::fma2(z2[i], si[i], y2[i]);
                    }
                }
                if (weights) {
                    uint64_t sum2 = 0;
#pragma unroll
                    for (int i = 0; i < kRotVec / 2; ++i) {
                        const uint64_t v = tc::pack2(y[2 * i], y[2 * i + 1]);
                        sum2 = tc::fma2(v, v, sum2);
                    }
                    float sum, odd;
                    tc::unpack2(sum2, sum, odd);
                    sum = live ? sum + odd : 0.f;  // a lane behind the row's end adds nothing, whatever a row that was not finite left in it
#pragma unroll
                    for (int m = 1; m < LPR; m <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
                    const float r = rsqrtf(fmaf(sum, inv_d, p.eps));
                    const uint64_t r2 = tc::pack2(r, r);
#pragma unroll
                    for (int i = 0; i < kRotVec / 2; ++i) y2[i] = tc::fma2(y2[i], r2, kMinusZero2);
                }
#pragma unroll
                for (int i = 0; i < kRotVec / 2; ++i) tc::unpack2(y2[i], y[2 * i], y[2 * i + 1]);
                x[a].set(y);
                if (first + row + a * step < h_last && live) x[a].store(dst);
                dst += dst_step;
            }
        }
    };
    if (p.Hq > h_first) walk(p.q, p.out_q, p.q_weight, 0, 0, p.Hq);
    if (p.Hq + p.Hkv > h_first && h_end > p.Hq) walk(p.k, p.out_k, p.k_weight, p.Hq, p.Hq, p.Hq + p.Hkv);
}

template <typename T, int LPR, int ROPE>
cudaError_t launch(const Ctx &ctx, RotateArgs p, const finch_rope &rope, cudaStream_t stream) {
    const int sms = ctx.sm_count, heads = p.Hq + p.Hkv, L = ctx.model.L;
    // Tokens of a CTA: up to 8, fewer where that leaves SMs without a CTA; then fewer heads.
    int tok = 8;
    while (tok > 1 && (int64_t)L * ((p.tokens + tok - 1) / tok) < 2 * sms) tok /= 2;
    int per = heads;
    const int least = kRotWarps / tok * (32 / LPR);  // a round of a CTA
    while (per > least && (int64_t)L * ((p.tokens + tok - 1) / tok) * ((heads + per - 1) / per) < sms) per = (per + 1) / 2;
    p.tok_per_cta = tok;
    p.heads_per_cta = per;
    const size_t smem = ROPE != kNone ? (size_t)tok * (rope.rotary_dim / 2) * sizeof(float2) : 0;
    ctx.launches += 1;
    return launch_chained(rotate_kernel<T, LPR, ROPE>, dim3((p.tokens + tok - 1) / tok, (heads + per - 1) / per, L), dim3(kRotThreads), smem,
                          stream, p, rope);
}

template <typename T, int ROPE>
cudaError_t launch_d(const Ctx &ctx, const RotateArgs &p, const finch_rope &rope, cudaStream_t stream) {
    if (p.d <= 32) return launch<T, 4, ROPE>(ctx, p, rope, stream);
    if (p.d <= 64) return launch<T, 8, ROPE>(ctx, p, rope, stream);
    if (p.d <= 128) return launch<T, 16, ROPE>(ctx, p, rope, stream);
    return launch<T, 32, ROPE>(ctx, p, rope, stream);
}

template <typename T>
cudaError_t launch_t(const Ctx &ctx, const RotateArgs &p, const finch_rope *rope, cudaStream_t stream) {
    static const finch_rope none = {};
    if (!rope) return launch_d<T, kNone>(ctx, p, none, stream);
    return rope->pairing ? launch_d<T, kNeighbours>(ctx, p, *rope, stream) : launch_d<T, kHalves>(ctx, p, *rope, stream);
}

}  // namespace

cudaError_t launch_rotate(const Ctx &ctx, const TensorView &q, const TensorView &k, const TensorView &out_q, const TensorView &out_k,
                          int tokens, const int *pos, const finch_rope *rope, const void *q_weight, const void *k_weight, float eps,
                          cudaStream_t stream) {
    const ModelView &mv = ctx.model;
    const RotateArgs p = {q, k, out_q, out_k, q_weight, k_weight, pos, q.ptr ? mv.Hq : 0, k.ptr ? mv.Hkv : 0, mv.d, tokens, 0, 0, eps};
    if (tokens == 0 || p.Hq + p.Hkv == 0) return cudaSuccess;
    return mv.elem_bytes == 4 ? launch_t<float>(ctx, p, rope, stream) : launch_t<__nv_bfloat16>(ctx, p, rope, stream);
}

}  // namespace finch
