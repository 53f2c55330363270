// RMS norm of every query and key head and the rotary embedding, in one pass over q and k.
//
//   y = x * rsqrt(mean(x^2) + eps) * w      (a head's row, fp32; with weights only)
//   pairs of y turn by position * inv_freq  (rotate.cuh; with a rope only)
//
// Pure bandwidth: every element is read and written once.  A CTA takes a few tokens and all their heads (or some of them, where
// there are too few tokens to fill the SMs), so that a token's cosines and sines are formed once; a row is LPR lanes with
// eight elements each, several rows to a warp, and a warp has the loads of kAhead rounds in flight.
#include "rotate.cuh"

namespace finch {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotWarps = kRotThreads / 32;
constexpr int kAhead = 4;

struct RotateArgs {
    TensorView q, k, out_q, out_k;
    const void *q_weight, *k_weight;
    const int *pos;
    int Hq, Hkv, d, tokens;
    int tok_per_cta, heads_per_cta;
    float eps;
    int has_rope;
};

template <typename T, int LPR>
__global__ void __launch_bounds__(kRotThreads) rotate_kernel(RotateArgs p, const __grid_constant__ finch_rope rope) {
    extern __shared__ float2 table[];  // [tok_per_cta][rotary_dim / 2]
    __shared__ double freq[128];
    constexpr int kRows = 32 / LPR;    // rows of a warp and round
    dependency_wait();
    const int l = blockIdx.z, tok0 = blockIdx.x * p.tok_per_cta, h0 = blockIdx.y * p.heads_per_cta;
    const int n_tok = min(p.tok_per_cta, p.tokens - tok0), n_heads = min(p.heads_per_cta, p.Hq + p.Hkv - h0);
    const int half = p.has_rope ? rope.rotary_dim / 2 : 0;
    if (p.has_rope) {
        for (int i = threadIdx.x; i < half; i += kRotThreads) freq[i] = rope.inv_freq[i];
        __syncthreads();
        rotary_table(table, rope, freq, n_tok, [&](int row) { return p.pos[tok0 + row]; });
        __syncthreads();
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, at = lane % LPR;
    const bool live = at * kRotVec < p.d;
    // rows (token, head), heads innermost: kRows of them to a warp and round
    const int rows = n_tok * n_heads;
    for (int r0 = warp * kRows; r0 < rows; r0 += kRotWarps * kRows * kAhead) {
        Eight<T> x[kAhead];
        const T *src[kAhead];
        T *dst[kAhead];
        int tok[kAhead];
        bool is_q[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int r = r0 + a * kRotWarps * kRows + lane / LPR;
            src[a] = nullptr;
            tok[a] = 0;
            is_q[a] = true;
            dst[a] = nullptr;
            if (r < rows) {
                tok[a] = r / n_heads;
                const int h = h0 + r - tok[a] * n_heads;
                is_q[a] = h < p.Hq;
                const TensorView &in = is_q[a] ? p.q : p.k, &out = is_q[a] ? p.out_q : p.out_k;
                const int hh = is_q[a] ? h : h - p.Hq;
                src[a] = (const T *)in.ptr + l * in.stride_layer + hh * in.stride_head + (int64_t)(tok0 + tok[a]) * in.stride_tok;
                dst[a] = (T *)out.ptr + l * out.stride_layer + hh * out.stride_head + (int64_t)(tok0 + tok[a]) * out.stride_tok;
            }
            x[a].zero();
            if (src[a] && live) x[a].load(src[a] + at * kRotVec);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const T *w = (const T *)(is_q[a] ? p.q_weight : p.k_weight);
            float y[kRotVec];
            x[a].get(y);
            if (__any_sync(0xffffffffu, src[a] && w)) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < kRotVec; ++i) sum = fmaf(y[i], y[i], sum);
#pragma unroll
                for (int m = 1; m < LPR; m <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
                if (w) {
                    const float r = rsqrtf(sum / (float)p.d + p.eps);
                    if (live) {
                        Eight<T> g8;
                        float g[kRotVec];
                        g8.load(w + (int64_t)l * p.d + at * kRotVec);
                        g8.get(g);
#pragma unroll
                        for (int i = 0; i < kRotVec; ++i) y[i] = y[i] * r * g[i];
                    }
                }
            }
            if (p.has_rope) rotate8<LPR, false>(y, table + tok[a] * half, at, rope.rotary_dim, rope.pairing);
            x[a].set(y);
            if (src[a] && live) x[a].store(dst[a] + at * kRotVec);
        }
    }
}

template <typename T, int LPR>
cudaError_t launch(const Ctx &ctx, RotateArgs p, const finch_rope &rope, cudaStream_t stream) {
    const int sms = ctx.sm_count, heads = p.Hq + p.Hkv, L = ctx.model.L;
    // Tokens of a CTA: up to 8, fewer where that leaves SMs without a CTA; then fewer heads.
    int tok = 8;
    while (tok > 1 && (int64_t)L * ((p.tokens + tok - 1) / tok) < 2 * sms) tok /= 2;
    int per = heads;
    const int least = kRotWarps * (32 / LPR);  // a round of a CTA
    while (per > least && (int64_t)L * ((p.tokens + tok - 1) / tok) * ((heads + per - 1) / per) < sms) per = (per + 1) / 2;
    p.tok_per_cta = tok;
    p.heads_per_cta = per;
    const size_t smem = p.has_rope ? (size_t)tok * (rope.rotary_dim / 2) * sizeof(float2) : 0;
    ctx.launches += 1;
    return launch_chained(rotate_kernel<T, LPR>, dim3((p.tokens + tok - 1) / tok, (heads + per - 1) / per, L), dim3(kRotThreads), smem,
                          stream, p, rope);
}

template <typename T>
cudaError_t launch_t(const Ctx &ctx, const RotateArgs &p, const finch_rope &rope, cudaStream_t stream) {
    if (p.d <= 32) return launch<T, 4>(ctx, p, rope, stream);
    if (p.d <= 64) return launch<T, 8>(ctx, p, rope, stream);
    if (p.d <= 128) return launch<T, 16>(ctx, p, rope, stream);
    return launch<T, 32>(ctx, p, rope, stream);
}

}  // namespace

cudaError_t launch_rotate(const Ctx &ctx, const TensorView &q, const TensorView &k, const TensorView &out_q, const TensorView &out_k,
                          int tokens, const int *pos, const finch_rope *rope, const void *q_weight, const void *k_weight, float eps,
                          cudaStream_t stream) {
    const ModelView &mv = ctx.model;
    RotateArgs p = {q, k, out_q, out_k, q_weight, k_weight, pos, q.ptr ? mv.Hq : 0, k.ptr ? mv.Hkv : 0, mv.d, tokens, 0, 0, eps, rope != nullptr};
    if (tokens == 0 || p.Hq + p.Hkv == 0) return cudaSuccess;
    static const finch_rope none = {};
    const finch_rope &r = rope ? *rope : none;
    return mv.elem_bytes == 4 ? launch_t<float>(ctx, p, r, stream) : launch_t<__nv_bfloat16>(ctx, p, r, stream);
}

}  // namespace finch
