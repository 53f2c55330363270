// Attention of packed query rows over [cache ; chunk] with fp32 multiply-adds: fp32 inputs, head dimensions above 128, and
// tensors that the TMA unit cannot describe.
//
// A CTA takes 64 rows of one KV head (its query heads times some tokens: they share every key), or 32 or 16 where few rows leave SMs
// without work, and a split of its keys, 64 at a time, staged as fp32; fp32 tiles of up to 128 dimensions come by cp.async while the tile
// before is worked on.  A thread owns 4 (2, 1) rows of 4 logits, then of D / 16 outputs, four keys at a time; the rows' running maximum and
// sum are kept by the 16 threads of a row group alike.  Bound by shared-memory reads (8 128-bit reads to 64 multiply-adds).
#include "attend.cuh"

namespace finch {
namespace {

using tc::fma2;
using tc::pack2;
using tc::unpack2;

constexpr int kK = 64;

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

template <bool B>
struct Flag {
    static constexpr bool value = B;
};

template <typename T, int D, int R>
struct Tiles {
    static constexpr bool kAhead = sizeof(T) == 4 && D <= 128;   // the next tile is on its way
    static constexpr int kPitch = D + 4, kBufs = kAhead ? 2 : 1, kThreads = 256, kRows = R / 16;
    float q[R * kPitch], k[kBufs][kK * kPitch], v[kBufs][kK * D], p[R * (kK + 4)];
};

template <typename T, int D, int R>
__global__ void __launch_bounds__(256) attend_simt_kernel(SimtArgs p) {
    extern __shared__ __align__(16) char raw[];
    using Mem = Tiles<T, D, R>;
    Mem &sm = *(Mem *)raw;
    constexpr int kPitch = Mem::kPitch, kCols = D / 64, kThreads = Mem::kThreads, kR = R, kRM = Mem::kRows;  // rows of a thread
    constexpr bool kAhead = Mem::kAhead;
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
    int limit[kRM], most = 0;
#pragma unroll
    for (int i = 0; i < kRM; ++i) {
        const int r = ty * kRM + i;
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

    float m[kRM], sum[kRM];
    uint64_t o[kRM][kCols][2];
#pragma unroll
    for (int i = 0; i < kRM; ++i) {
        m[i] = -INFINITY, sum[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[i][c][0] = o[i][c][1] = 0;
    }
    // K and V rows of one tile; rows behind the last candidate and dimensions behind the head's are zeros
    auto fetch = [&](int kt) {
        float *ks = sm.k[kt % Mem::kBufs], *vs = sm.v[kt % Mem::kBufs];
        for (int i = threadIdx.x; i < kK * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4) * 4, j = kt * kK + r;
            const bool there = c < d && j < u.N, cached = j < u.c;
            const TensorView &k = cached ? p.ck : p.hk, &v = cached ? p.cv : p.hv;
            const int64_t row = there ? (cached ? u.cache0 + j : u.chunk0 + j - u.c) : 0;
            const T *from_k = (const T *)k.ptr + l * k.stride_layer + kvh * k.stride_head + row * k.stride_tok + c;
            const T *from_v = (const T *)v.ptr + l * v.stride_layer + kvh * v.stride_head + row * v.stride_tok + c;
            if constexpr (kAhead) {
                if (there) {
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(ks + r * kPitch + c)), "l"(from_k) : "memory");
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(vs + r * D + c)), "l"(from_v) : "memory");
                    continue;
                }
            }
            const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
            *(float4 *)(ks + r * kPitch + c) = there ? load4f(from_k) : zero;
            *(float4 *)(vs + r * D + c) = there ? load4f(from_v) : zero;
        }
        if constexpr (kAhead) asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (kAhead && tile0 < tile1) fetch(tile0);
    for (int kt = tile0; kt < tile1; ++kt) {
        const int j0 = kt * kK;
        __syncthreads();  // everyone is through with the previous tile
        if constexpr (kAhead) {
            if (kt + 1 < tile1) fetch(kt + 1);
            if (kt + 1 < tile1)
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            else
                asm volatile("cp.async.wait_group 0;" ::: "memory");
        } else {
            fetch(kt);
        }
        __syncthreads();
        const float *ks = sm.k[kt % Mem::kBufs], *vs = sm.v[kt % Mem::kBufs];
        uint64_t acc[kRM][4] = {};
#pragma unroll 4
        for (int c = 0; c < d; c += 4) {
            ulonglong2 kk[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) kk[j] = *(const ulonglong2 *)(ks + (tx + 16 * j) * kPitch + c);
#pragma unroll
            for (int i = 0; i < kRM; ++i) {
                const ulonglong2 qq = *(const ulonglong2 *)(sm.q + (ty * kRM + i) * kPitch + c);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fma2(qq.y, kk[j].y, fma2(qq.x, kk[j].x, acc[i][j]));
            }
        }
#pragma unroll
        for (int i = 0; i < kRM; ++i) {
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
                sm.p[(ty * kRM + i) * (kK + 4) + tx + 16 * j] = s[j];
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
        // A key that a row does not see has weight zero there, and zero times an infinity is none: where some row does not see a key, keys
        // are added for the rows that do only.
        int seen = limit[0];
#pragma unroll
        for (int i = 1; i < kRM; ++i) seen = min(seen, limit[i]);
        seen -= j0;
        const int keys = min(kK, most - j0), common = max(0, min(keys, seen)) & ~3;
        auto add = [&](int i, float w, const ulonglong2 (&vv)[kCols]) {
            const uint64_t w2 = pack2(w, w);
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[i][c][0] = fma2(w2, vv[c].x, o[i][c][0]), o[i][c][1] = fma2(w2, vv[c].y, o[i][c][1]);
        };
        auto four = [&](int j, auto masked) {
            float4 w[kRM];
#pragma unroll
            for (int i = 0; i < kRM; ++i) w[i] = *(const float4 *)(sm.p + (ty * kRM + i) * (kK + 4) + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ulonglong2 vv[kCols];
#pragma unroll
                for (int c = 0; c < kCols; ++c) vv[c] = *(const ulonglong2 *)(vs + (j + e) * D + tx * 4 + 64 * c);
#pragma unroll
                for (int i = 0; i < kRM; ++i)
                    if (!decltype(masked)::value || j0 + j + e < limit[i]) add(i, e == 0 ? w[i].x : (e == 1 ? w[i].y : (e == 2 ? w[i].z : w[i].w)), vv);
            }
        };
        int j = 0;
#pragma unroll 2
        for (; j < common; j += 4) four(j, Flag<false>{});
#pragma unroll 1
        for (; j < keys; j += 4) four(j, Flag<true>{});
    }
#pragma unroll
    for (int i = 0; i < kRM; ++i) {
        const int r = ty * kRM + i;
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

template <typename T, int D, int R>
cudaError_t launch(const Ctx &ctx, const SimtArgs &p, dim3 grid, cudaStream_t stream) {
    const int bit = kSmemAttendSimt + (R == 64) + 2 * (R == 32);  // a context has one type and head dimension
    if (!ctx.smem_ready(bit)) {
        cudaError_t e = cudaFuncSetAttribute(attend_simt_kernel<T, D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Tiles<T, D, R>));
        if (e != cudaSuccess) return e;
        ctx.smem_set(bit);
    }
    ctx.launches += 1;
    return launch_chained(attend_simt_kernel<T, D, R>, grid, dim3(256), sizeof(Tiles<T, D, R>), stream, p);
}
template <typename T, int R>
cudaError_t launch_d(const Ctx &ctx, const SimtArgs &p, dim3 grid, cudaStream_t stream) {
    if (p.mv.d <= 64) return launch<T, 64, R>(ctx, p, grid, stream);
    if (p.mv.d <= 128) return launch<T, 128, R>(ctx, p, grid, stream);
    return launch<T, 256, R>(ctx, p, grid, stream);
}
template <typename T>
cudaError_t launch_t(const Ctx &ctx, const SimtArgs &p, int rows, dim3 grid, cudaStream_t stream) {
    if (rows == 16) return launch_d<T, 16>(ctx, p, grid, stream);
    return rows == 32 ? launch_d<T, 32>(ctx, p, grid, stream) : launch_d<T, 64>(ctx, p, grid, stream);
}

struct Plan {
    int per_cta, heads, tok, chunks, row_tiles, splits;
};

// Host arithmetic on the batch's bounds; partial_rows: rows of partial results that there is place for.
Plan make_plan(const Ctx &ctx, const BatchView &bv, size_t partial_rows) {
    const ModelView &mv = ctx.model;
    const int sms = ctx.sm_count > 0 ? ctx.sm_count : 148;   // a validation-only context has none
    Plan n;
    // 64 rows to a CTA, fewer where there are no more, or where that leaves most SMs without one and the keys are few (8 heads of 64: 16 rows
    // over 16 8.9 us with 64, 5.4 with 16; 256 over 256 19.0, 14.7 with 32, 16.8 with 16; 512 over 512 29, 35, 38; 100 over 2148 35, 43, 65)
    const int key_tiles = (bv.max_cache + kK - 1) / kK + (bv.max_chunk + kK - 1) / kK;
    int64_t units = 0, tiles = 0;
    for (n.per_cta = kAttendSimtRows;; n.per_cta /= 2) {
        // as many heads as share their keys, at least one token
        n.heads = mv.g < n.per_cta ? mv.g : n.per_cta;
        n.tok = n.per_cta / n.heads;
        n.chunks = (mv.g + n.heads - 1) / n.heads;
        tiles = (bv.max_q + n.tok - 1) / n.tok;
        units = (int64_t)mv.L * mv.Hkv * n.chunks;
        const bool fits = (int64_t)bv.max_q * mv.g * 2 <= n.per_cta, idle = key_tiles <= 4 && units * tiles * bv.batch < sms / 4;
        if (n.per_cta == 16 || !(fits || idle)) break;
    }
    n.row_tiles = (int)tiles;
    const size_t rows = (size_t)mv.L * mv.Hq * bv.total_q;
    n.splits = attend_splits(units * tiles * bv.batch, sms, key_tiles, 2);
    while (n.splits > 1 && n.splits * rows > partial_rows) --n.splits;
    return n;
}

}  // namespace

int attend_simt_splits(const Ctx &ctx, const BatchView &bv, size_t partial_rows) { return make_plan(ctx, bv, partial_rows).splits; }

cudaError_t launch_attend_simt(const Ctx &ctx, const TensorView &q, const TensorView &ck, const TensorView &cv, const TensorView &hk,
                               const TensorView &hv, const BatchView &bv, int causal, AttendOut out, size_t partial_rows,
                               cudaStream_t stream) {
    if (bv.batch == 0 || bv.max_q == 0) return cudaSuccess;
    const ModelView &mv = ctx.model;
    const Plan n = make_plan(ctx, bv, partial_rows);
    SimtArgs p = {mv, bv, q, ck, cv, hk, hv, out, ctx.d_status, causal, n.heads, n.tok, n.chunks, n.row_tiles, mv.scale * kLog2e};
    p.out.splits = n.splits;
    const int64_t ctas = (int64_t)mv.L * mv.Hkv * n.chunks * n.splits * n.row_tiles;
    if (ctas > INT_MAX) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)ctas, bv.batch);
    cudaError_t e = mv.elem_bytes == 4 ? launch_t<float>(ctx, p, n.per_cta, grid, stream) : launch_t<__nv_bfloat16>(ctx, p, n.per_cta, grid, stream);
    if (e == cudaSuccess && n.splits > 1) e = launch_merge_splits(ctx, bv, p.out, stream);
    return e;
}

}  // namespace finch
