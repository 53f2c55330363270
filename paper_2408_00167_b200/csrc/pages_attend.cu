// Attention of a request's newest tokens over its paged 8-bit cache (pages.cuh).
//
// Bound by the bytes of the cache: a page and KV head are 2 x 64 x d bytes that 8 query rows share.  A warp takes whole pages straight
// from global memory into the registers of mma.sync fragments, 16 bytes a lane and load: which dimension is which k index is free as
// long as both operands agree, and so is the order of the keys and, for the output, of the columns.  Codes turn into f16 exactly
// (two at a time); of V, whose pairs along k are two keys, bytes of two rows are interleaved first.
//
//   S = Q K^T   m = 16: rows 0-7 are the f16 heads of 8 query rows, rows 8-15 what the first rounding cut off, so that
//               q enters with 22 bits; a row is scaled by a power of two first, whatever its range.  Page and row scales
//               multiply the logits.
//   O += P V    the same for P = 2^(s - m) in [0, 1]; a page's product is folded into O (fp32) with its V scale.
//
// (tcgen05 wants 128 rows and its operands in shared memory: 8 rows would waste 15/16 of it and every code would make a second trip
// through shared memory.)  Keys that not all rows see and the open rows are taken one at a time with fp32 multiply-adds, dealt
// out over all warps of the unit.  Splits of a unit are merged by merge_splits.
#include "attend.cuh"

namespace finch {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kRows = kPagesRows;

struct DecodeArgs {
    ModelView mv;
    PagesView pg;
    PagedView bv;
    TensorView q;
    AttendOut out;
    int *status;
    int row_groups;
    float scale2;
};

__device__ __forceinline__ uint32_t half2_of(__half a, __half b) {
    const __half2 v = __halves2half2(a, b);
    return *(const uint32_t *)&v;
}
// codes in the low / high 16 bits of w -> two f16
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x, y -> their f16 heads and what is left of them, also in f16
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo) {
    const __half hx = __float2half_rn(x), hy = __float2half_rn(y);
    hi = half2_of(hx, hy);
    lo = half2_of(__float2half_rn(x - __half2float(hx)), __float2half_rn(y - __half2float(hy)));
}
// W consecutive words, aligned to their largest power of two
template <int W>
__device__ __forceinline__ void load_words(uint32_t *r, const uint8_t *p) {
    if constexpr (W % 4 == 0) {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const uint4 v = __ldg((const uint4 *)p + i / 4);
            r[i] = v.x, r[i + 1] = v.y, r[i + 2] = v.z, r[i + 3] = v.w;
        }
    } else if constexpr (W % 2 == 0) {
#pragma unroll
        for (int i = 0; i < W; i += 2) {
            const uint2 v = __ldg((const uint2 *)p + i / 2);
            r[i] = v.x, r[i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) r[i] = __ldg((const uint32_t *)p + i);
    }
}

template <int D>
struct Geometry {
    static constexpr int kKeys = D <= 128 ? 64 : 16;       // keys of a page that a warp holds at a time
    static constexpr int kVec = D % 64 == 0 ? 16 : 8;      // bytes of a K row that a lane loads at a time
    static constexpr int kChunks = D / (4 * kVec);
    static constexpr int kSteps = D / 16;                  // k steps of S
    static constexpr int kTiles = kKeys / 8;               // key tiles of S
    static constexpr int kWords = D / 32;                  // words of a V row that a lane loads
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) decode_kernel(DecodeArgs p) {
    using Geo = Geometry<D>;
    __shared__ __align__(16) float qs[kRows][D];
    __shared__ __align__(16) float part[kWarps][kRows][D];
    __shared__ float2 part_ml[kWarps][kRows];
    dependency_wait();
    const ModelView &mv = p.mv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tid = lane & 3;
    const int b = blockIdx.y, l = blockIdx.z;
    int x = blockIdx.x;
    const int split = x % p.out.splits;
    x /= p.out.splits;
    const int kvh = x % mv.Hkv, rg = x / mv.Hkv;
    const PagedInfo u = paged_info(p.pg, p.bv, b, false);
    if (!u.ok || u.len / kPage > p.pg.table_width) {
        if (threadIdx.x == 0) atomicOr(p.status, FINCH_DEV_BAD_BATCH);
        return;
    }
    const int rows = min(kRows, u.n * mv.g - rg * kRows);  // row r of the group: token (rg * 8 + r) / g, query head (..) % g of the KV head
    if (rows <= 0) return;
    auto token = [&](int r) { return (rg * kRows + r) / mv.g; };
    auto limit = [&](int r) { return max(0, u.len - u.n + token(r) + 1); };
    const int least = limit(0), most = limit(rows - 1);
    const int full = min(u.len, least) / kPage;            // pages that every row sees whole

    for (int i = threadIdx.x; i < kRows * D; i += kThreads) {
        const int r = i / D, c = i % D;
        float v = 0.f;
        if (r < rows)
            v = (float)((const T *)p.q.ptr)[l * p.q.stride_layer + (int64_t)(kvh * mv.g + (rg * kRows + r) % mv.g) * p.q.stride_head +
                                            (int64_t)(u.row0 + token(r)) * p.q.stride_tok + c];
        qs[r][c] = v * p.scale2;
    }
    __syncthreads();

    const int *table = p.pg.table + (int64_t)b * p.pg.table_width;
    const int page0 = (int)((int64_t)full * split / p.out.splits), page1 = (int)((int64_t)full * (split + 1) / p.out.splits);
    {
        // This lane's part of Q: row gid, dimensions chunk * 4 kVec + tid * kVec + 4 j of step (chunk, j), scaled to [1, 2).
        uint32_t qa[Geo::kSteps][4];
        float top = 0.f;
        for (int c = tid; c < D; c += 4) top = fmaxf(top, fabsf(qs[gid][c]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int ex = max(-126, min(126, (top > 0.f && top < INFINITY) ? ilogbf(top) : 0));
        const float down = exp2f((float)-ex), up = exp2f((float)ex);
#pragma unroll
        for (int s = 0; s < Geo::kSteps; ++s) {
            const int e = s * 4 / Geo::kVec * 4 * Geo::kVec + tid * Geo::kVec + s * 4 % Geo::kVec;
            const float4 v = *(const float4 *)&qs[gid][e];
            split2(v.x * down, v.y * down, qa[s][0], qa[s][1]);
            split2(v.z * down, v.w * down, qa[s][2], qa[s][3]);
        }
        float m = -INFINITY, sum = 0.f;
        float o[D / 8][2];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = 0.f;

        uint32_t kw[Geo::kTiles][D / 16], vw[Geo::kKeys / 16][4][Geo::kWords];
        float k_scale = 0.f, v_scale = 0.f;
        constexpr int kParts = kPage / Geo::kKeys;
        const int begin = page0 * kParts, end = page1 * kParts;  // parts of pages
        int number = 0;
        bool bad = false;
        auto load_k = [&](int it) {
            number = __ldg(table + it / kParts);
            bad = number < 0 || number >= p.pg.n_pages;
            if (bad) number = 0;                            // a page that exists: what is read of it does not count
            const int64_t ph = p.pg.page_head(mv, l, number, kvh);
            const uint8_t *k = p.pg.k + ph * (kPage * D) + it % kParts * Geo::kKeys * D;
            k_scale = __ldg(p.pg.k_scale + ph);
#pragma unroll
            for (int j = 0; j < Geo::kTiles; ++j)
#pragma unroll
                for (int c = 0; c < Geo::kChunks; ++c)
                    load_words<Geo::kVec / 4>(&kw[j][c * (Geo::kVec / 4)], k + (8 * j + gid) * D + c * 4 * Geo::kVec + tid * Geo::kVec);
        };
        auto load_v = [&](int it) {
            const int64_t ph = p.pg.page_head(mv, l, number, kvh);
            const uint8_t *v = p.pg.v + ph * (kPage * D) + it % kParts * Geo::kKeys * D;
            v_scale = __ldg(p.pg.v_scale + ph);
#pragma unroll
            for (int kk = 0; kk < Geo::kKeys / 16; ++kk)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    load_words<Geo::kWords>(vw[kk][i], v + (16 * kk + i / 2 * 8 + tid * 2 + i % 2) * D + gid * (D / 8));
        };
        // parts of a page go to one warp, pages around the warps
        auto next = [&](int it) { return (it + 1) % kParts ? it + 1 : it + 1 + (kWarps - 1) * kParts; };
        int it = begin + warp * kParts;
        if (it < end) {
            load_k(it);
            load_v(it);
        }
        for (; it < end; it = next(it)) {
            float s[Geo::kTiles][2];
            const float f = up * k_scale, vs = v_scale;
            const bool skip = bad;
            if (skip && lane == 0) atomicOr(p.status, FINCH_DEV_BAD_INDEX);
#pragma unroll
            for (int j = 0; j < Geo::kTiles; ++j) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < Geo::kSteps; ++t) mma16816(c, qa[t], codes_lo(kw[j][t]), codes_hi(kw[j][t]));
                s[j][0] = (c[0] + c[2]) * f;
                s[j][1] = (c[1] + c[3]) * f;
            }
            const int ahead = next(it);
            if (ahead < end) load_k(ahead);
            float now = m;
#pragma unroll
            for (int j = 0; j < Geo::kTiles; ++j) {
                if (skip) s[j][0] = s[j][1] = -INFINITY;
                now = fmaxf(now, fmaxf(s[j][0], s[j][1]));
            }
            now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 1));
            now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 2));
            const float ref = now == -INFINITY ? 0.f : now, corr = tc::ex2(m - ref);
            m = now;
            sum *= corr;
            uint32_t pa[Geo::kTiles / 2][4];
#pragma unroll
            for (int j = 0; j < Geo::kTiles; ++j) {
                const float p0 = tc::ex2(s[j][0] - ref), p1 = tc::ex2(s[j][1] - ref);
                sum += p0 + p1;
                split2(p0, p1, pa[j / 2][j % 2 * 2], pa[j / 2][j % 2 * 2 + 1]);
            }
#pragma unroll
            for (int w = 0; w < Geo::kWords; ++w) {
                float c[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0.f;
#pragma unroll
                for (int kk = 0; kk < Geo::kKeys / 16; ++kk) {
                    const uint32_t a0 = __byte_perm(vw[kk][0][w], vw[kk][1][w], 0x5140), a1 = __byte_perm(vw[kk][0][w], vw[kk][1][w], 0x7362);
                    const uint32_t b0 = __byte_perm(vw[kk][2][w], vw[kk][3][w], 0x5140), b1 = __byte_perm(vw[kk][2][w], vw[kk][3][w], 0x7362);
                    mma16816(c[0], pa[kk], codes_lo(a0), codes_lo(b0));
                    mma16816(c[1], pa[kk], codes_hi(a0), codes_hi(b0));
                    mma16816(c[2], pa[kk], codes_lo(a1), codes_lo(b1));
                    mma16816(c[3], pa[kk], codes_hi(a1), codes_hi(b1));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    o[4 * w + i][0] = fmaf(vs, skip ? 0.f : c[i][0] + c[i][2], o[4 * w + i][0] * corr);
                    o[4 * w + i][1] = fmaf(vs, skip ? 0.f : c[i][1] + c[i][3], o[4 * w + i][1] * corr);
                }
            }
            if (ahead < end) load_v(ahead);
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (tid == 0) part_ml[warp][gid] = make_float2(m, sum);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < D / 8; ++i) part[warp][gid][(tid * 2 + c) * (D / 8) + i] = o[i][c];
    }
    __syncwarp();

    // The rest, a key at a time: a lane has D / 32 neighbouring dimensions of each row.
    constexpr int kPer = D / 32;
    const int rest0 = full * kPage + split * kWarps + warp, step = p.out.splits * kWarps;
    if (rest0 < most) {
        float m[kRows], sum[kRows], o[kRows][kPer];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            m[r] = part_ml[warp][r].x, sum[r] = part_ml[warp][r].y;
#pragma unroll
            for (int i = 0; i < kPer; ++i) o[r][i] = part[warp][r][lane * kPer + i];
        }
        __syncwarp();
        for (int j = rest0; j < most; j += step) {
            float kx[kPer], vx[kPer];
            const int page = j / kPage;
            if (page < u.len / kPage) {
                const int number = __ldg(table + page);
                if (number < 0 || number >= p.pg.n_pages) {
                    if (lane == 0) atomicOr(p.status, FINCH_DEV_BAD_INDEX);
                    continue;
                }
                const int64_t ph = p.pg.page_head(mv, l, number, kvh), at = (ph * kPage + j % kPage) * D + lane * kPer;
                const float ks = __ldg(p.pg.k_scale + ph), vs = __ldg(p.pg.v_scale + ph);
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    kx[i] = (float)((const __nv_fp8_e4m3 *)p.pg.k)[at + i] * ks;
                    vx[i] = (float)((const __nv_fp8_e4m3 *)p.pg.v)[at + i] * vs;
                }
            } else {
                const int64_t at = (p.pg.open_row(mv, l, u.slot, kvh) + j % kPage) * D + lane * kPer;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    kx[i] = (float)((const T *)p.pg.open_k)[at + i];
                    vx[i] = (float)((const T *)p.pg.open_v)[at + i];
                }
            }
            float s[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                s[r] = 0.f;
#pragma unroll
                for (int i = 0; i < kPer; ++i) s[r] = fmaf(qs[r][lane * kPer + i], kx[i], s[r]);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int w = 16; w; w >>= 1) s[r] += __shfl_xor_sync(0xffffffffu, s[r], w);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                if (r >= rows || j >= limit(r)) continue;
                if (s[r] > m[r]) {
                    const float corr = tc::ex2(m[r] - s[r]);
                    sum[r] *= corr;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) o[r][i] *= corr;
                    m[r] = s[r];
                }
                const float w = tc::ex2(s[r] - (m[r] == -INFINITY ? 0.f : m[r]));
                sum[r] += w;
#pragma unroll
                for (int i = 0; i < kPer; ++i) o[r][i] = fmaf(w, vx[i], o[r][i]);
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (lane == 0) part_ml[warp][r] = make_float2(m[r], sum[r]);
#pragma unroll
            for (int i = 0; i < kPer; ++i) part[warp][r][lane * kPer + i] = o[r][i];
        }
    }
    __syncthreads();

    // The warps of the CTA in their order; a thread has four dimensions of a row.
    for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            if (part_ml[w][r].y != 0.f) m = fmaxf(m, part_ml[w][r].x);
        const float ref = m == -INFINITY ? 0.f : m;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 ml = part_ml[w][r];
            if (ml.y == 0.f) continue;
            const float f = exp2f(ml.x - ref);
            sum = fmaf(ml.y, f, sum);
            const float4 y = *(const float4 *)&part[w][r][c];
            v.x = fmaf(y.x, f, v.x), v.y = fmaf(y.y, f, v.y), v.z = fmaf(y.z, f, v.z), v.w = fmaf(y.w, f, v.w);
        }
        const int h = kvh * mv.g + (rg * kRows + r) % mv.g, t = u.row0 + token(r);
        const int64_t row = attend_row(mv, p.bv.total_q, l, h, t);
        if (p.out.splits > 1) {
            const int64_t slot = split * ((int64_t)mv.L * mv.Hq * p.bv.total_q) + row;
            *(float4 *)(p.out.part_o + slot * D + c) = v;
            if (c == 0) p.out.part_ml[slot] = make_float2(m, sum);
            continue;
        }
        float lse;
        const float inv = attend_finish(m, sum, nullptr, row, lse);
        if (sum == 0.f) v = make_float4(0.f, 0.f, 0.f, 0.f);
        else v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        store4<T>((T *)p.out.ptr + l * p.out.stride_layer + h * p.out.stride_head + (int64_t)t * p.out.stride_tok + c, v);
        if (p.out.row_lse && c == 0) p.out.row_lse[row] = lse;
    }
}

template <typename T>
cudaError_t launch_t(const Ctx &ctx, const DecodeArgs &p, dim3 grid, cudaStream_t stream) {
    ctx.launches += 1;
    switch (p.mv.d) {
        case 32: return launch_chained(decode_kernel<T, 32>, grid, dim3(kThreads), 0, stream, p);
        case 64: return launch_chained(decode_kernel<T, 64>, grid, dim3(kThreads), 0, stream, p);
        case 96: return launch_chained(decode_kernel<T, 96>, grid, dim3(kThreads), 0, stream, p);
        case 128: return launch_chained(decode_kernel<T, 128>, grid, dim3(kThreads), 0, stream, p);
        case 160: return launch_chained(decode_kernel<T, 160>, grid, dim3(kThreads), 0, stream, p);
        case 192: return launch_chained(decode_kernel<T, 192>, grid, dim3(kThreads), 0, stream, p);
        case 224: return launch_chained(decode_kernel<T, 224>, grid, dim3(kThreads), 0, stream, p);
        case 256: return launch_chained(decode_kernel<T, 256>, grid, dim3(kThreads), 0, stream, p);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_pages_attend(const Ctx &ctx, const PagesView &pg, const PagedView &bv, const TensorView &q, AttendOut out,
                                size_t partial_rows, cudaStream_t stream) {
    if (bv.batch == 0 || bv.max_q == 0) return cudaSuccess;
    const ModelView &mv = ctx.model;
    DecodeArgs p = {mv, pg, bv, q, out, ctx.d_status, (bv.max_q * mv.g + kRows - 1) / kRows, mv.scale * kLog2e};
    const int64_t units = (int64_t)mv.L * mv.Hkv * p.row_groups * bv.batch;
    const size_t rows = (size_t)mv.L * mv.Hq * bv.total_q;
    int splits = attend_splits(units, 2 * ctx.sm_count, bv.max_len / kPage, kWarps);
    while (splits > 1 && splits * rows > partial_rows) --splits;
    p.out.splits = splits;
    cudaError_t e;
    const int64_t ctas = (int64_t)splits * mv.Hkv * p.row_groups;
    if (ctas > INT_MAX) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)ctas, bv.batch, mv.L);
    e = mv.elem_bytes == 4 ? launch_t<float>(ctx, p, grid, stream) : launch_t<__nv_bfloat16>(ctx, p, grid, stream);
    if (e == cudaSuccess && splits > 1) e = launch_merge_splits_paged(ctx, pg, bv, p.out, stream);
    return e;
}

}  // namespace finch
