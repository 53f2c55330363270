// Rotary positions, shared by the rotation of queries and keys and by the append to the paged cache.
//
// Pair t of a row at position p turns by the angle p * inv_freq[t]: (a, b) -> (a c - b s, a s + b c), c and s its cosine and
// sine times `magnitude`.  A position of a long context times a frequency needs more bits than fp32 has (2^-24 of 10^6 is 0.06
// radians), so the angle and its cosine and sine are formed in 64 bits and rounded to 32 once, a few hundred operations for a
// pair of a token that all its heads share.
#pragma once

#include "finch_internal.cuh"

namespace finch {

constexpr int kRotVec = 8;  // elements of a row that a lane holds

// (cos, sin) of pairs 0 .. half - 1 of `rows` positions into table[row * half + t]; pos(row) gives a row's position.
template <typename Pos>
__device__ __forceinline__ void rotary_table(float2 *table, const finch_rope &rope, const double *freq, int rows, Pos pos) {
    const int half = rope.rotary_dim / 2;
    for (int i = threadIdx.x; i < rows * half; i += blockDim.x) {
        const int row = i / half;
        double s, c;
        sincos((double)pos(row) * freq[i - row * half], &s, &c);
        table[i] = make_float2((float)(c * rope.magnitude), (float)(s * rope.magnitude));
    }
}

// Eight elements of a row, as fp32.
__device__ __forceinline__ void load8(const float *p, float (&x)[kRotVec]) {
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&x)[kRotVec]) {
    const uint4 v = *(const uint4 *)p;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store8(float *p, const float (&x)[kRotVec]) {
    *(float4 *)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4 *)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&x)[kRotVec]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *(const uint32_t *)&v;
    }
    *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
}

// a c - b s (SUB) or a c + b s, rounded to fp32 once: both products and their sum with the parts that fp32 cuts off (exact
// products by fused multiply-add, the two-sum of Knuth).
template <bool SUB>
__device__ __forceinline__ float turn_exact(float a, float c, float b, float s) {
    const float p = __fmul_rn(a, c), pe = __fmaf_rn(a, c, -p);
    float q = __fmul_rn(b, s), qe = __fmaf_rn(b, s, -q);
    if (SUB) q = -q, qe = -qe;
    const float sum = __fadd_rn(p, q), v = __fsub_rn(sum, p);
    const float e = __fadd_rn(__fsub_rn(p, __fsub_rn(sum, v)), __fsub_rn(q, v));
    const float out = __fadd_rn(sum, __fadd_rn(e, __fadd_rn(pe, qe)));
    return isfinite(out) ? out : sum;  // an infinity's cut-off part is not a number
}

// Turns the 8 elements that lane `at` of a row's LPR lanes holds; cs is the row's part of the table.  Every lane of the
// warp takes part.  rotary_dim is a multiple of 16, so that an element's partner half the rotary dimensions on has the same
// place in another lane's eight.  EXACT: the sum of the two products is rounded once.
template <int LPR, bool EXACT>
__device__ __forceinline__ void rotate8(float (&x)[kRotVec], const float2 *cs, int at, int rotary_dim, int pairing) {
    const int e0 = at * kRotVec, half = rotary_dim / 2;
    if (pairing) {
        if (e0 >= rotary_dim) return;
#pragma unroll
        for (int i = 0; i < kRotVec; i += 2) {
            const float2 t = cs[(e0 + i) / 2];
            const float a = x[i], b = x[i + 1];
            x[i] = EXACT ? turn_exact<true>(a, t.x, b, t.y) : a * t.x - b * t.y;
            x[i + 1] = EXACT ? turn_exact<false>(a, t.y, b, t.x) : a * t.y + b * t.x;
        }
    } else {
        const int lane = threadIdx.x & 31, first = lane - at, step = half / kRotVec;
        const bool low = e0 < half, turns = e0 < rotary_dim;
        const int partner = turns ? first + (low ? at + step : at - step) : lane;
#pragma unroll
        for (int i = 0; i < kRotVec; ++i) {
            const float other = __shfl_sync(0xffffffffu, x[i], partner);
            if (turns) {
                const float2 t = cs[low ? e0 + i : e0 + i - half];
                if (low)
                    x[i] = EXACT ? turn_exact<true>(x[i], t.x, other, t.y) : x[i] * t.x - other * t.y;
                else
                    x[i] = EXACT ? turn_exact<false>(other, t.y, x[i], t.x) : other * t.y + x[i] * t.x;
            }
        }
    }
}

}  // namespace finch
