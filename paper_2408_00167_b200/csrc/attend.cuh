// Shared by the attention kernels: where rows' results go, partial results of key splits, and their merge.
//
// A kernel that works on one of several key splits of a row leaves the row's unnormalised output O = sum_j 2^(s_j - m) v_j, fp32,
// with (m, l): the base-2 reference and l = sum_j 2^(s_j - m).  merge_splits adds the splits of a row in their order.
#pragma once

#include "pages.cuh"
#include "score_tc_common.cuh"

namespace finch {

constexpr int kAttendMaxSplits = 32;

struct AttendOut {
    char *ptr;
    int64_t stride_layer, stride_head, stride_tok;  // elements
    float *row_lse;                                 // [L][Hq][total_q] or null
    float *part_o;                                  // [splits][L * Hq * total_q][d]
    float2 *part_ml;                                // [splits][L * Hq * total_q]
    int splits;                                     // 1: kernels write out / row_lse themselves
};

// One row's place in the arrays of partial results.
__device__ __forceinline__ int64_t attend_row(const ModelView &mv, int total_q, int l, int h, int row) {
    return ((int64_t)l * mv.Hq + h) * total_q + row;
}

// How many candidates query row i of a request sees.
__device__ __forceinline__ int attend_limit(const BatchView &bv, const UnitInfo &u, int i, int causal) {
    const int lim = bv.row_limit ? bv.row_limit[u.q0 + i] : (causal ? u.N - u.n_q + i + 1 : u.N);
    return max(0, min(u.N, lim));
}

// (m, l) of a row -> log-sum-exp, and the factor of O; an extra term of the denominator (natural log) counts once.
__device__ __forceinline__ float attend_finish(float m, float l, const float *self_lse, int64_t row, float &lse) {
    if (self_lse) {
        const float x = self_lse[row] * kLog2e;
        if (l == 0.f) m = x;
        if (x > -INFINITY) {
            const float top = fmaxf(m, x), f = exp2f(m - top);
            // a sum against a reference far below the extra term is brought to it before the two are added
            const float total = l * f + exp2f(x - top);
            lse = (top + log2f(total)) * kLn2;
            return l == 0.f ? 0.f : f / total;
        }
    }
    lse = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    return l == 0.f ? 0.f : 1.f / l;
}

template <typename T>
__device__ __forceinline__ void store4(T *p, float4 x);
template <>
__device__ __forceinline__ void store4<float>(float *p, float4 x) { *(float4 *)p = x; }
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *p, float4 x) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    *(uint2 *)p = make_uint2(*(const uint32_t *)&a, *(const uint32_t *)&b);
}

// Key splits of a call: rows of `units` CTAs over `sms` SMs, at least `least` key tiles to a split.
inline int attend_splits(int64_t units, int sms, int key_tiles, int least) {
    int64_t s = units > 0 ? sms / units : 1;
    if (s > key_tiles / least) s = key_tiles / least;
    if (s > kAttendMaxSplits) s = kAttendMaxSplits;
    return s < 1 ? 1 : (int)s;
}

// Partial results: at most kAttendMaxSplits for a row, and no more than `sms` CTAs' rows in all (there are splits only where
// the CTAs are fewer than the SMs).
inline size_t attend_partial_rows(const ModelView &mv, int64_t total_q, int sms, int rows_per_cta) {
    const size_t rows = (size_t)mv.L * mv.Hq * total_q;
    const size_t a = rows * kAttendMaxSplits, b = (size_t)sms * rows_per_cta;
    return a < b ? a : b;
}

// The splits of every row of a call.
cudaError_t launch_merge_splits(const Ctx &ctx, const BatchView &bv, const AttendOut &out, cudaStream_t stream);

constexpr int kAttendTcRows = 256;    // rows of a CTA, tensor-core path
constexpr int kAttendSimtRows = 64;   // .. of the warp-level path
constexpr int kPagesRows = 8;         // .. of the paged path

bool attend_tc_supported(const Ctx &ctx);
// what the launches below make of a batch's bounds (FINCH_ATTEND_..)
void attend_tc_plan(const Ctx &ctx, const BatchView &bv, size_t partial_rows, int &path, int &cluster, int &clusters);
int attend_simt_splits(const Ctx &ctx, const BatchView &bv, size_t partial_rows);
cudaError_t launch_attend_tc(const Ctx &ctx, const TensorView &q, const TensorView &ck, const TensorView &cv, const TensorView &hk,
                             const TensorView &hv, const BatchView &bv, int causal, AttendOut out, size_t partial_rows, cudaStream_t stream);
cudaError_t launch_attend_simt(const Ctx &ctx, const TensorView &q, const TensorView &ck, const TensorView &cv, const TensorView &hk,
                               const TensorView &hv, const BatchView &bv, int causal, AttendOut out, size_t partial_rows,
                               cudaStream_t stream);
cudaError_t launch_pages_append(const Ctx &ctx, const PagesView &pg, const PagedView &bv, const TensorView &k, const TensorView &v,
                                const int *pos, const finch_rope *rope, int *out_len, cudaStream_t stream);
cudaError_t launch_pages_attend(const Ctx &ctx, const PagesView &pg, const PagedView &bv, const TensorView &q, AttendOut out,
                                cudaStream_t stream);
cudaError_t launch_rotate(const Ctx &ctx, const TensorView &q, const TensorView &k, const TensorView &out_q, const TensorView &out_k,
                          int tokens, const int *pos, const finch_rope *rope, const void *q_weight, const void *k_weight, float eps,
                          cudaStream_t stream);

}  // namespace finch
