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

// Sine and cosine of x, |x| < 2^32 radians: x minus the nearest multiple of pi/2 (Cody and Waite's reduction, pi/2 in two parts;
// the multiple times the first part cancels exactly in the fused multiply-add), then the Taylor polynomials on [-pi/4, pi/4],
// whose next terms are below 2^-57.  (The library's sincos also reduces arguments of any size and takes twice as long here.)
__device__ __forceinline__ void sincos_angle(double x, double &s, double &c) {
    const double two_over_pi = 0.63661977236758134308, half_pi = 1.5707963267948965580, half_pi_rest = 6.1232339957367660359e-17;
    const double round_to_int = 6755399441055744.0;  // 1.5 * 2^52: adding it leaves an integer in the low bits
    const double shifted = fma(x, two_over_pi, round_to_int), n = shifted - round_to_int;
    const int quadrant = __double2loint(shifted);
    const double r = fma(-n, half_pi_rest, fma(-n, half_pi, x)), r2 = r * r;
    // 1/k! for k = 17, 15, .. 3 and 16, 14, .. 2
    double ps = 2.8114572543455206e-15, pc = 4.7794773323873853e-14;
    ps = fma(ps, r2, -7.6471637318198164e-13), pc = fma(pc, r2, -1.1470745597729725e-11);
    ps = fma(ps, r2, 1.6059043836821613e-10), pc = fma(pc, r2, 2.0876756987868099e-9);
    ps = fma(ps, r2, -2.5052108385441720e-8), pc = fma(pc, r2, -2.7557319223985893e-7);
    ps = fma(ps, r2, 2.7557319223985893e-6), pc = fma(pc, r2, 2.4801587301587302e-5);
    ps = fma(ps, r2, -1.9841269841269841e-4), pc = fma(pc, r2, -1.3888888888888889e-3);
    ps = fma(ps, r2, 8.3333333333333333e-3), pc = fma(pc, r2, 4.1666666666666667e-2);
    ps = fma(ps, r2, -0.16666666666666667), pc = fma(pc, r2, -0.5);
    const double sr = fma(ps * r2, r, r), cr = fma(pc, r2, 1.0);
    const double a = quadrant & 1 ? cr : sr, b = quadrant & 1 ? sr : cr;
    s = quadrant & 2 ? -a : a;
    c = (quadrant + 1) & 2 ? -b : b;
}

// (cos, sin) of pairs 0 .. half - 1 of `rows` positions into table[row * half + t]; pos(row) gives a row's position.
template <typename Pos>
__device__ __forceinline__ void rotary_table(float2 *table, const finch_rope &rope, const double *freq, int rows, Pos pos) {
    const int half = rope.rotary_dim / 2;
    for (int i = threadIdx.x; i < rows * half; i += blockDim.x) {
        const int row = i / half;
        double s, c;
        sincos_angle((double)pos(row) * freq[i - row * half], s, c);
        table[i] = make_float2((float)(c * rope.magnitude), (float)(s * rope.magnitude));
    }
}

// Eight elements of a row, as they lie in memory and as fp32.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float *p) { a = *(const float4 *)p, b = *(const float4 *)(p + 4); }
    __device__ __forceinline__ void store(float *p) const { *(float4 *)p = a, *(float4 *)(p + 4) = b; }
    __device__ __forceinline__ void get(float (&x)[kRotVec]) const {
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
    __device__ __forceinline__ void from_lane(int lane) {
        a.x = __shfl_sync(0xffffffffu, a.x, lane), a.y = __shfl_sync(0xffffffffu, a.y, lane);
        a.z = __shfl_sync(0xffffffffu, a.z, lane), a.w = __shfl_sync(0xffffffffu, a.w, lane);
        b.x = __shfl_sync(0xffffffffu, b.x, lane), b.y = __shfl_sync(0xffffffffu, b.y, lane);
        b.z = __shfl_sync(0xffffffffu, b.z, lane), b.w = __shfl_sync(0xffffffffu, b.w, lane);
    }
    // The bits of the largest magnitude so far (as unsigned numbers magnitudes are in order, infinities and NaN behind all others).
    __device__ __forceinline__ void fold_magnitude(uint32_t &top) const {
        float x[kRotVec];
        get(x);
#pragma unroll
        for (int i = 0; i < kRotVec; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    }
    __device__ __forceinline__ static uint32_t magnitude(uint32_t top) { return top; }
    __device__ __forceinline__ void get_negated(float (&x)[kRotVec]) const {
        get(x);
#pragma unroll
        for (int i = 0; i < kRotVec; ++i) x[i] = -x[i];
    }
    __device__ __forceinline__ void set(const float (&x)[kRotVec]) {
        a = make_float4(x[0], x[1], x[2], x[3]), b = make_float4(x[4], x[5], x[6], x[7]);
    }
};
template <>
struct Eight<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *(const uint4 *)p; }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *(uint4 *)p = v; }
    __device__ __forceinline__ void get(float (&x)[kRotVec]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void from_lane(int lane) {
        v.x = __shfl_sync(0xffffffffu, v.x, lane), v.y = __shfl_sync(0xffffffffu, v.y, lane);
        v.z = __shfl_sync(0xffffffffu, v.z, lane), v.w = __shfl_sync(0xffffffffu, v.w, lane);
    }
    // two 16-bit lanes of magnitudes; `magnitude` gives the larger one as the bits of an fp32 number
    __device__ __forceinline__ void fold_magnitude(uint32_t &top) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
    }
    __device__ __forceinline__ static uint32_t magnitude(uint32_t top) { return max(top & 0xffff0000u, top << 16); }
    __device__ __forceinline__ void get_negated(float (&x)[kRotVec]) const {
        Eight<__nv_bfloat16> n;
        n.v = make_uint4(v.x ^ 0x80008000u, v.y ^ 0x80008000u, v.z ^ 0x80008000u, v.w ^ 0x80008000u);
        n.get(x);
    }
    __device__ __forceinline__ void set(const float (&x)[kRotVec]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 y = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *(const uint32_t *)&y;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

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
// place in another lane's eight.  The sum of the two products is rounded once.
template <int LPR>
__device__ __forceinline__ void rotate8(float (&x)[kRotVec], const float2 *cs, int at, int rotary_dim, int pairing) {
    const int e0 = at * kRotVec, half = rotary_dim / 2;
    if (pairing) {
        if (e0 >= rotary_dim) return;
#pragma unroll
        for (int i = 0; i < kRotVec; i += 2) {
            const float2 t = cs[(e0 + i) / 2];
            const float a = x[i], b = x[i + 1];
            x[i] = turn_exact<true>(a, t.x, b, t.y);
            x[i + 1] = turn_exact<false>(a, t.y, b, t.x);
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
                    x[i] = turn_exact<true>(x[i], t.x, other, t.y);
                else
                    x[i] = turn_exact<false>(other, t.y, x[i], t.x);
            }
        }
    }
}

}  // namespace finch
