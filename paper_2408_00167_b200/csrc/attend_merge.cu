// Adds the key splits of a row: O = sum_s 2^(m_s - m) O_s, l likewise, in the order of the splits; out = O / l.
// A warp takes a row; bound by the partial results, which an L2 holds.
#include "attend.cuh"

namespace finch {
namespace {

struct MergeArgs {
    ModelView mv;
    BatchView bv;
    AttendOut out;
};

template <typename T>
__global__ void __launch_bounds__(128) merge_kernel(MergeArgs p) {
    dependency_wait();
    const ModelView &mv = p.mv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, b = blockIdx.y;
    const UnitInfo u = unit_info(mv, p.bv, 0, b);
    if (!u.ok) return;
    const int64_t id = (int64_t)blockIdx.x * 4 + warp;
    if (id >= (int64_t)p.bv.max_q * mv.L * mv.Hq) return;
    const int i = (int)(id % p.bv.max_q), lh = (int)(id / p.bv.max_q), l = lh / mv.Hq, h = lh - l * mv.Hq;
    if (i >= u.n_q) return;
    const int64_t rows = (int64_t)mv.L * mv.Hq * p.bv.total_q, row = attend_row(mv, p.bv.total_q, l, h, u.q0 + i);
    const float2 ml = lane < p.out.splits ? p.out.part_ml[lane * rows + row] : make_float2(-INFINITY, 0.f);
    float m = ml.y == 0.f ? -INFINITY : ml.x;
#pragma unroll
    for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    const float ref = m == -INFINITY ? 0.f : m;
    const float f = ml.y == 0.f ? 0.f : exp2f(ml.x - ref);
    float l_sum = 0.f;
    float4 o[2] = {};
    for (int s = 0; s < p.out.splits; ++s) {
        const float fs = __shfl_sync(0xffffffffu, f, s), ls = __shfl_sync(0xffffffffu, ml.y, s);
        if (ls == 0.f) continue;  // saw none of the row's keys; its O was not written
        l_sum = fmaf(ls, fs, l_sum);
        const float *src = p.out.part_o + (s * rows + row) * mv.d;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int d = c * 128 + lane * 4;
            if (d < mv.d) {
                const float4 v = *(const float4 *)(src + d);
                o[c].x = fmaf(v.x, fs, o[c].x), o[c].y = fmaf(v.y, fs, o[c].y);
                o[c].z = fmaf(v.z, fs, o[c].z), o[c].w = fmaf(v.w, fs, o[c].w);
            }
        }
    }
    float lse;
    const float inv = attend_finish(m, l_sum, p.bv.self_lse, row, lse);
    T *dst = (T *)p.out.ptr + l * p.out.stride_layer + h * p.out.stride_head + (int64_t)(u.q0 + i) * p.out.stride_tok;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int d = c * 128 + lane * 4;
        if (d < mv.d)
            store4<T>(dst + d, l_sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[c].x * inv, o[c].y * inv, o[c].z * inv, o[c].w * inv));
    }
    if (p.out.row_lse && lane == 0) p.out.row_lse[row] = lse;
}

}  // namespace

cudaError_t launch_merge_splits(const Ctx &ctx, const BatchView &bv, const AttendOut &out, cudaStream_t stream) {
    const MergeArgs p = {ctx.model, bv, out};
    const int64_t rows = (int64_t)bv.max_q * p.mv.L * p.mv.Hq;
    ctx.launches += 1;
    const dim3 grid((unsigned)((rows + 3) / 4), bv.batch);
    return ctx.model.elem_bytes == 4 ? launch_chained(merge_kernel<float>, grid, dim3(128), 0, stream, p)
                                     : launch_chained(merge_kernel<__nv_bfloat16>, grid, dim3(128), 0, stream, p);
}

}  // namespace finch
