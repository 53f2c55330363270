// Attention of packed query rows over [cache ; chunk] with fp32 multiply-adds: fp32 inputs, head dimensions above 128, and
// tensors that the TMA unit cannot describe.
//
// A CTA takes 64 rows of one KV head (its query heads times some tokens: they share every key) and a split of its keys, 64 at a
// time, staged as fp32.  A thread owns 4 x 4 logits, then 4 rows x D / 16 outputs; the rows' running maximum and sum are kept by the 16 threads of a
// row group alike.  Bound by shared-memory reads (8 128-bit reads to 64 multiply-adds).
#include "attend.cuh"

namespace finch {
namespace {

using tc::fma2;
using tc::pack2;
using tc::unpack2;

constexpr int kR = kAttendSimtRows, kK = 64, kThreads = 256;

struct SimtArgs {
    ModelView mv;
    BatchView bv;
    TensorView q, ck, cv, hk, hv;
    AttendOut out;
    int *status;
    int causal, heads, tok, chunks, row_tiles;  // query heads and tokens of a row tile, tiles of heads per KV head, of tokens
    float scale2;
};

__device__ __forceinline__ float4 load4f(const float *p) { return *(const float4 *)p; }
__device__ __forceinline__ float4 load4f(const __nv_bfloat16 *p) {
    const uint2 v = *(const uint2 *)p;
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xffff0000u));
}

template <int D>
struct Smem {
    static constexpr int kPitch = D + 4;
    float q[kR * kPitch], k[kK * kPitch], v[kK * D], p[kR * (kK + 4)];
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) attend_simt_kernel(SimtArgs p) {
    extern __shared__ __align__(16) char raw[];
    Smem<D> &sm = *(Smem<D> *)raw;
    constexpr int kPitch = Smem<D>::kPitch, kCols = D / 64;
    dependency_wait();
    const ModelView &mv = p.mv;
    const int b = blockIdx.y, d = mv.d;
    int x = blockIdx.x;
    const int split = x % p.out.splits;
    x /= p.out.splits;
    const int hc = x % p.chunks;
    x /= p.chunks;
    const int kvh = x % mv.Hkv, l = x / mv.Hkv % mv.L, tile = p.row_tiles - 1 - x / mv.Hkv / mv.L;  // long causal rows first
    UnitInfo u = unit_info(mv, p.bv, 0, b);
    if (!u.ok) {
        if (threadIdx.x == 0) atomicOr(p.status, FINCH_DEV_BAD_BATCH);
        return;
    }
    const int t0 = tile * p.tok;
    if (t0 >= u.n_q) return;
    const int h0 = hc * p.heads, n_heads = min(p.heads, mv.g - h0);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;

    // row r of the tile: token t0 + r % tok of query head kvh * g + h0 + r / tok
    auto row_live = [&](int r) { return r / p.tok < n_heads && t0 + r % p.tok < u.n_q; };
    for (int i = threadIdx.x; i < kR * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < d && row_live(r))
            v = load4f((const T *)p.q.ptr + l * p.q.stride_layer + (int64_t)(kvh * mv.g + h0 + r / p.tok) * p.q.stride_head +
                       (int64_t)(u.q0 + t0 + r % p.tok) * p.q.stride_tok + c);
        *(float4 *)(sm.q + r * kPitch + c) = v;
    }
    int limit[4], most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = ty * 4 + i;
        limit[i] = row_live(r) ? attend_limit(p.bv, u, t0 + r % p.tok, p.causal) : 0;
        most = max(most, limit[i]);
    }
    __shared__ int most_s;
    if (threadIdx.x == 0) most_s = 0;
    __syncthreads();
    if (tx == 0 && most > 0) atomicMax(&most_s, most);
    __syncthreads();
    most = most_s;
    const int tiles = (most + kK - 1) / kK;
    const int tile0 = (int)((int64_t)tiles * split / p.out.splits), tile1 = (int)((int64_t)tiles * (split + 1) / p.out.splits);

    float m[4], sum[4];
    uint64_t o[4][kCols][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY, sum[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[i][c][0] = o[i][c][1] = 0;
    }
    for (int kt = tile0; kt < tile1; ++kt) {
        const int j0 = kt * kK;
        __syncthreads();  // everyone is through with the previous tile
        for (int i = threadIdx.x; i < kK * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4) * 4, j = j0 + r;
            float4 k4 = make_float4(0.f, 0.f, 0.f, 0.f), v4 = k4;
            if (c < d && j < u.N) {
                const bool cached = j < u.c;
                const TensorView &kt = cached ? p.ck : p.hk, &vt = cached ? p.cv : p.hv;
                const int64_t row = cached ? u.cache0 + j : u.chunk0 + j - u.c;
                k4 = load4f((const T *)kt.ptr + l * kt.stride_layer + kvh * kt.stride_head + row * kt.stride_tok + c);
                v4 = load4f((const T *)vt.ptr + l * vt.stride_layer + kvh * vt.stride_head + row * vt.stride_tok + c);
            }
            *(float4 *)(sm.k + r * kPitch + c) = k4;
            *(float4 *)(sm.v + r * D + c) = v4;
        }
        __syncthreads();
        uint64_t acc[4][4] = {};
#pragma unroll 4
        for (int c = 0; c < d; c += 4) {
            ulonglong2 kk[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) kk[j] = *(const ulonglong2 *)(sm.k + (tx + 16 * j) * kPitch + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const ulonglong2 qq = *(const ulonglong2 *)(sm.q + (ty * 4 + i) * kPitch + c);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fma2(qq.y, kk[j].y, fma2(qq.x, kk[j].x, acc[i][j]));
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float s[4], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float lo, hi;
                unpack2(acc[i][j], lo, hi);
                s[j] = j0 + tx + 16 * j < limit[i] ? (lo + hi) * p.scale2 : -INFINITY;
                top = fmaxf(top, s[j]);
            }
#pragma unroll
            for (int w = 1; w < 16; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float now = fmaxf(m[i], top), ref = now == -INFINITY ? 0.f : now;
            const float f = exp2f(m[i] - ref);
            float add = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = exp2f(s[j] - ref);
                add += s[j];
                sm.p[(ty * 4 + i) * (kK + 4) + tx + 16 * j] = s[j];
            }
#pragma unroll
            for (int w = 1; w < 16; w <<= 1) add += __shfl_xor_sync(0xffffffffu, add, w);
            sum[i] = sum[i] * f + add;
            m[i] = now;
            const uint64_t f2 = pack2(f, f);
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[i][c][0] = fma2(o[i][c][0], f2, 0), o[i][c][1] = fma2(o[i][c][1], f2, 0);
        }
        __syncwarp();  // a row's weights are written and read by the same half-warp
        const int keys = min(kK, most - j0);
        // A key that a row does not see has weight zero there, and zero times an infinity is none: keys that are not finite
        // everywhere are added for the rows that see them only.
        for (int j = 0; j < keys; ++j) {
            ulonglong2 vv[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) vv[c] = *(const ulonglong2 *)(sm.v + j * D + tx * 4 + 64 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = sm.p[(ty * 4 + i) * (kK + 4) + j];
                if (j0 + j < limit[i]) {
                    const uint64_t w2 = pack2(w, w);
#pragma unroll
                    for (int c = 0; c < kCols; ++c) o[i][c][0] = fma2(w2, vv[c].x, o[i][c][0]), o[i][c][1] = fma2(w2, vv[c].y, o[i][c][1]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = ty * 4 + i;
        if (!row_live(r)) continue;
        const int h = kvh * mv.g + h0 + r / p.tok, t = u.q0 + t0 + r % p.tok;
        const int64_t row = attend_row(mv, p.bv.total_q, l, h, t);
        float lse, inv = 1.f;
        if (p.out.splits == 1) inv = attend_finish(m[i], sum[i], p.bv.self_lse, row, lse);
        const int64_t slot = split * ((int64_t)mv.L * mv.Hq * p.bv.total_q) + row;
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            float4 v;
            unpack2(o[i][c][0], v.x, v.y);
            unpack2(o[i][c][1], v.z, v.w);
            const int at = tx * 4 + 64 * c;
            if (at >= d) continue;
            if (p.out.splits == 1) {
                v = sum[i] == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
                store4<T>((T *)p.out.ptr + l * p.out.stride_layer + h * p.out.stride_head + (int64_t)t * p.out.stride_tok + at, v);
            } else {
                *(float4 *)(p.out.part_o + slot * d + at) = v;
            }
        }
        if (tx == 0) {
            if (p.out.splits > 1)
                p.out.part_ml[slot] = make_float2(m[i], sum[i]);
            else if (p.out.row_lse)
                p.out.row_lse[row] = lse;
        }
    }
}

template <typename T, int D>
cudaError_t launch(const Ctx &ctx, const SimtArgs &p, dim3 grid, cudaStream_t stream) {
    const int bit = kSmemAttendSimt + (sizeof(T) == 4) + 2 * (D == 128) + 4 * (D == 256);
    if (!ctx.smem_ready(bit)) {
        cudaError_t e = cudaFuncSetAttribute(attend_simt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Smem<D>));
        if (e != cudaSuccess) return e;
        ctx.smem_set(bit);
    }
    ctx.launches += 1;
    return launch_chained(attend_simt_kernel<T, D>, grid, dim3(kThreads), sizeof(Smem<D>), stream, p);
}
template <typename T>
cudaError_t launch_t(const Ctx &ctx, const SimtArgs &p, dim3 grid, cudaStream_t stream) {
    if (p.mv.d <= 64) return launch<T, 64>(ctx, p, grid, stream);
    if (p.mv.d <= 128) return launch<T, 128>(ctx, p, grid, stream);
    return launch<T, 256>(ctx, p, grid, stream);
}

}  // namespace

cudaError_t launch_attend_simt(const Ctx &ctx, const TensorView &q, const TensorView &ck, const TensorView &cv, const TensorView &hk,
                               const TensorView &hv, const BatchView &bv, int causal, AttendOut out, size_t partial_rows,
                               cudaStream_t stream) {
    if (bv.batch == 0 || bv.max_q == 0) return cudaSuccess;
    const ModelView &mv = ctx.model;
    SimtArgs p = {mv, bv, q, ck, cv, hk, hv, out, ctx.d_status, causal, 0, 0, 0, 0, mv.scale * kLog2e};
    // As many heads as share their keys, at least one token
    p.heads = mv.g < kR ? mv.g : kR;
    p.tok = kR / p.heads;
    p.chunks = (mv.g + p.heads - 1) / p.heads;
    const int tiles = (bv.max_q + p.tok - 1) / p.tok;
    const int64_t units = (int64_t)mv.L * mv.Hkv * p.chunks;
    const size_t rows = (size_t)mv.L * mv.Hq * bv.total_q;
    int splits = attend_splits(units * tiles * bv.batch, 2 * ctx.sm_count, (bv.max_cache + bv.max_chunk + kK - 1) / kK, 2);
    while (splits > 1 && splits * rows > partial_rows) --splits;
    p.out.splits = splits;
    p.row_tiles = tiles;
    const int64_t ctas = units * splits * tiles;
    if (ctas > INT_MAX) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)ctas, bv.batch);
    cudaError_t e = mv.elem_bytes == 4 ? launch_t<float>(ctx, p, grid, stream) : launch_t<__nv_bfloat16>(ctx, p, grid, stream);
    if (e == cudaSuccess && splits > 1) e = launch_merge_splits(ctx, bv, p.out, stream);
    return e;
}

}  // namespace finch
