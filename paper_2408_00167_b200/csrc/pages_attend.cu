// Attention of a request's newest tokens over its paged 8-bit cache (pages.cuh).
//
// Bound by the bytes of the cache: a page and KV head are 2 x 64 x d bytes that 8 query rows share.  A warp copies whole pages
// into three slots of shared memory of its own (two on their way while one is read) and reads them as mma.sync fragments, 16 bytes a
// lane: which dimension is which k index is free as long as both operands agree, and so is the order of the keys and, for the output,
// of the rows.  Codes turn into f16 exactly (two
// at a time); of V, whose pairs along k are two keys, bytes of two rows are interleaved first.
//
//   S^T = K Q^T   16 keys x 8 query rows.  Rows of Q are f16 after a power of two took their range: exact for bf16 elements down to
//                 2^-30 of the row's largest; fp32 inputs enter as two f16 parts, 22 bits down to 2^-16 of it, 2^-38 of it at the least.
//                 Page and row scales multiply the logits.
//   O^T += V^T P^T  16 dimensions x 8 rows.  P = 2^(s - m) in [0, 1] enters, lifted, as two f16 parts, turned from the layout of S^T
//                 by movmatrix; a page's product is folded into O (fp32) with its V scale.
//
// (tcgen05 wants 128 rows and its operands in shared memory: 8 rows would waste 15/16 of it and every code would go through shared
// memory once more, as f16.)  The open rows go the same way, 16 to a warp, in bf16: bf16 as they are, fp32 as three parts.
//
// The work is a list of items: for every request, layer, KV head and group of 8 rows (a unit) its full pages, then one for the open
// rows.  A CTA takes an equal share of consecutive items: all CTAs have the same number of pages, whatever the lengths.  A unit within
// one CTA is finished there; pieces of others go to the CTA's two slots of the workspace (its first piece, its last), and the CTA that
// delivers the last piece of a unit adds them in their order.
#include "attend.cuh"

namespace finch {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kRows = kPagesRows;
constexpr int kCtasPerSm = 2;
// P in [0, 1] is lifted by 2^15 where it becomes f16: weights down to 2^-18 of the largest keep 22 bits, smaller ones are off by at
// most 2^-40 of it, so that a long cache's many small weights add up.  Q's elements, scaled into [1, 2) by the row's largest, are
// lifted by 2^13 likewise.
constexpr float kLift = 32768.f, kDrop = 1.f / kLift, kLiftLog2 = 15.f, kQueryLift = 8192.f;
constexpr int kScan = 4;   // requests of a lane and step of the search for a CTA's items

struct DecodeArgs {
    ModelView mv;
    PagesView pg;
    PagedView bv;
    TensorView q;
    AttendOut out;      // part_o [2 C][8][d], part_ml [2 C][8]
    int *pieces;        // [C] pieces delivered of the unit that begins in a CTA and ends in another; zero before and after a call
    int *status;
    float scale2;
};

struct Request {
    PagedInfo u;
    int pages;   // items of a unit: full pages, one more for open rows (or for nothing at all)
    int groups;  // of rows
    int units;   // at most INT_MAX / 8, which the host checks of the bounds
    __device__ __forceinline__ int items() const { return pages + (u.len % kPage > 0 || pages == 0); }
    __device__ __forceinline__ int64_t all_items() const { return (int64_t)units * items(); }
};
__device__ __forceinline__ Request request_of(const DecodeArgs &p, int b) {
    Request r;
    r.u = paged_info(p.pg, p.bv, b, false);
    r.u.ok = r.u.ok && r.u.len / kPage <= p.pg.table_width;
    r.pages = r.u.ok ? r.u.len / kPage : 0;
    r.groups = r.u.ok ? (r.u.n * p.mv.g + kRows - 1) / kRows : 0;
    r.units = r.groups * p.mv.Hkv * p.mv.L;
    return r;
}

// A quotient that fits an int, in 32 bits where its operands do.
__device__ __forceinline__ int quotient(int64_t a, int64_t b) {
    return a <= INT_MAX && b <= INT_MAX ? (int)a / (int)b : (int)(a / b);
}
// Equal shares: `more` CTAs have one item above `each`.  With `groups` equal groups of items and of CTAs (the units of a single
// request) every group is shared by itself, so that no CTA has pieces of two units.
struct Shares {
    int64_t each, of_group;
    int more, ctas;
    __device__ __forceinline__ Shares(int64_t items, int all_ctas, int groups) {
        of_group = groups > 1 ? quotient(items, groups) : items;
        ctas = all_ctas / groups;
        each = of_group <= INT_MAX ? (int)of_group / ctas : of_group / ctas;
        more = (int)(of_group - each * ctas);
    }
    __device__ __forceinline__ int64_t begin(int c) const {
        const int g = c / ctas, r = c - g * ctas;
        return of_group * g + each * r + min(r, more);
    }
    __device__ __forceinline__ int of(int64_t item) const {
        const int g = item < of_group ? 0 : quotient(item, of_group);
        item -= of_group * g;
        const int64_t big = (each + 1) * more;
        return g * ctas + (item < big ? quotient(item, each + 1) : more + quotient(item - big, each));
    }
};

// Where a CTA's items begin: request, and the items in front of it.  Every warp searches by itself, kScan requests to a lane.
struct Place {
    int b, groups;  // groups: of Shares
    int64_t in_front, total;
    Request r;
};
__device__ __forceinline__ Place find_items(const DecodeArgs &p) {
    const int lane = threadIdx.x & 31, batch = p.bv.batch;
    Place place;
    place.b = 0, place.groups = 1, place.in_front = place.total = 0;
    if (batch == 1) {
        const Request r = place.r = request_of(p, 0);
        if (!r.u.ok && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.status, FINCH_DEV_BAD_BATCH);
        place.total = r.all_items();
        if (r.units > 0 && gridDim.x % r.units == 0) place.groups = r.units;
        return place;
    }
    const bool one_step = batch <= 32 * kScan;
    for (int pass = one_step ? 1 : 0; pass < 2; ++pass) {
        int64_t before = 0;
        for (int base = 0; base < batch; base += 32 * kScan) {
            int64_t n[kScan], mine = 0;
#pragma unroll
            for (int i = 0; i < kScan; ++i) {
                const int b = base + lane * kScan + i;
                n[i] = 0;
                if (b < batch) {
                    const Request r = request_of(p, b);
                    n[i] = r.all_items();
                    if (!r.u.ok && blockIdx.x == 0 && threadIdx.x < 32) atomicOr(p.status, FINCH_DEV_BAD_BATCH);
                }
                mine += n[i];
            }
            int64_t incl = mine;
#pragma unroll
            for (int x = 1; x < 32; x <<= 1) {
                const int64_t up = __shfl_up_sync(0xffffffffu, incl, x);
                if (lane >= x) incl += up;
            }
            int64_t at = before + incl - mine;
            before += __shfl_sync(0xffffffffu, incl, 31);
            if (one_step) place.total = before;
            if (pass == 1) {
                const int64_t begin = Shares(place.total, gridDim.x, 1).begin(blockIdx.x);
                int hit = -1;
                int64_t hit_at = 0;
#pragma unroll
                for (int i = 0; i < kScan; ++i) {
                    if (at <= begin && begin < at + n[i]) hit = base + lane * kScan + i, hit_at = at;
                    at += n[i];
                }
                const unsigned who = __ballot_sync(0xffffffffu, hit >= 0);
                if (who) {
                    place.b = __shfl_sync(0xffffffffu, hit, __ffs(who) - 1);
                    place.in_front = __shfl_sync(0xffffffffu, hit_at, __ffs(who) - 1);
                    place.r = request_of(p, place.b);
                    return place;
                }
            }
        }
        place.total = before;
    }
    place.r.units = 0;
    return place;  // no items at all
}

__device__ __forceinline__ uint32_t half2_of(float x, float y) {
    const __half2 v = __floats2half2_rn(x, y);
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
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {  // an 8 x 8 matrix of f16, two of a row to a lane
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// x, y -> their f16 heads and what is left of them, also in f16
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo) {
    hi = half2_of(x, y);
    const float2 h = __half22float2(*(const __half2 *)&hi);
    lo = half2_of(x - h.x, y - h.y);
}
// The power of two at or below a magnitude's, and its inverse, where both are normal numbers, also after the lift.
__device__ __forceinline__ void power_of_two(float top, float &up, float &down) {
    int ex = (int)(__float_as_uint(top) >> 23) - 127;
    ex = top > 0.f ? max(-110, min(126, ex)) : 0;
    up = __uint_as_float((uint32_t)(127 + ex) << 23);
    down = __uint_as_float((uint32_t)(127 - ex) << 23);
}
// W consecutive words, aligned to their largest power of two
template <int W>
__device__ __forceinline__ void load_words(uint32_t *r, const void *p) {
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
template <typename T>
__device__ __forceinline__ void two_of(const uint32_t *w, int i, float &x, float &y) {  // elements 2i and 2i + 1 of packed words
    if constexpr (sizeof(T) == 4)
        x = __uint_as_float(w[2 * i]), y = __uint_as_float(w[2 * i + 1]);
    else
        x = __uint_as_float(w[i] << 16), y = __uint_as_float(w[i] & 0xffff0000u);
}

template <int D>
struct Geometry {
    static constexpr int kVec = D % 64 == 0 ? 16 : 8;      // neighbouring dimensions of a K or Q row in a lane
    static constexpr int kChunks = D / (4 * kVec);         // .. and how many such runs
    static constexpr int kSteps = D / 16;                  // k steps of S^T: four dimensions of a lane each
    static constexpr int kTiles = kPage / 16;              // key tiles
    static constexpr int kWords = D / 32;                  // words of a V row's codes in a lane
    static constexpr int kSlot = kPage * D;                // bytes of a page's K or V of one head
    static constexpr int kSlots = 3;                       // of a warp
    static constexpr int kSmem = kWarps * kSlots * kSlot;
    static_assert(kRows * (D + 4) * 4 <= kSlots * kSlot, "a warp's result takes the place of its pages");
    // Where byte `x` of row `row` lies in a slot.  A quarter of a warp reads two rows' halves (K) or four rows' neighbouring
    // 16 bytes (V): of rows of 128 bytes or a multiple the 16-byte pieces change places so that these are in different banks.
    __device__ __forceinline__ static int place(int row, int x) {
        if constexpr (D % 128 == 0) return row * D + (x ^ ((((row >> 2) ^ row) & 1) << 6 | ((row >> 1) & 1) << 5));
        return row * D + x;
    }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int W>
__device__ __forceinline__ void read_words(uint32_t *r, uint32_t addr) {
    if constexpr (W % 4 == 0) {
#pragma unroll
        for (int i = 0; i < W; i += 4)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]) : "r"(addr + i * 4));
    } else if constexpr (W % 2 == 0) {
#pragma unroll
        for (int i = 0; i < W; i += 2) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r[i]), "=r"(r[i + 1]) : "r"(addr + i * 4));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r[i]) : "r"(addr + i * 4));
    }
}

// A warp's running result for 8 rows: lane (gid, tid) has rows 2 tid and 2 tid + 1, and of them dimensions gid D/8 .. + D/8 - 1.
template <int D>
struct Running {
    float m[2], sum[2], o[D / 8][2];
    __device__ __forceinline__ void clear() {
        m[0] = m[1] = -INFINITY, sum[0] = sum[1] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = 0.f;
    }
    // Softmax step over NT tiles of 16 keys: s[t] = logits of (key gid, rows 2 tid, 2 tid + 1), (key gid + 8, ..) become P; corr: the
    // factors of what was before.  P and sum are lifted, o is not.
    template <int NT>
    __device__ __forceinline__ void weights(float (&s)[NT][4], float (&corr)[2]) {
        float now[2] = {m[0], m[1]}, ref[2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) now[i % 2] = fmaxf(now[i % 2], s[t][i]);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) now[r] = fmaxf(now[r], __shfl_xor_sync(0xffffffffu, now[r], x));
            ref[r] = now[r] == -INFINITY ? 0.f : now[r];
            corr[r] = tc::ex2(m[r] - ref[r]);
            ref[r] -= kLiftLog2;
            m[r] = now[r];
            sum[r] *= corr[r];  // a lane's own keys only: the lanes' sums are added at the end
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = tc::ex2(s[t][i] - ref[i % 2]);
                sum[i % 2] += s[t][i];
            }
        }
    }
    // P as B fragments of two f16 parts
    template <int NT>
    __device__ __forceinline__ static void parts(const float (&s)[NT][4], uint32_t (&ph)[NT][2], uint32_t (&pl)[NT][2]) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t hi, lo;
                split2(s[t][2 * h], s[t][2 * h + 1], hi, lo);
                ph[t][h] = transposed(hi), pl[t][h] = transposed(lo);
            }
    }
    __device__ __forceinline__ void fold(int i, const float (&c)[4], float scale, const float (&corr)[2]) {
        o[i][0] = fmaf(scale, c[0], o[i][0] * corr[0]), o[i][1] = fmaf(scale, c[1], o[i][1] * corr[1]);
        o[i + 1][0] = fmaf(scale, c[2], o[i + 1][0] * corr[0]), o[i + 1][1] = fmaf(scale, c[3], o[i + 1][1] * corr[1]);
    }
};

__device__ __forceinline__ void mma16816_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// x, y -> N parts of bf16, 8 bits each with the range of fp32; an infinity is its first part.
template <int N>
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t (&w)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        w[n] = *(const uint32_t *)&h;
        const float hx = __uint_as_float(w[n] << 16), hy = __uint_as_float(w[n] & 0xffff0000u);
        x = fabsf(hx) == INFINITY ? 0.f : x - hx, y = fabsf(hy) == INFINITY ? 0.f : y - hy;
    }
}
// Four neighbouring elements as pairs of parts: one part of bf16, three of fp32 (24 bits, no common power of two: rows that differ
// by any order, or that a query row does not see, leave one another alone).
__device__ __forceinline__ void load_parts(const __nv_bfloat16 *p, bool there, uint32_t (&w)[2][1]) {
    const uint2 x = there ? __ldg((const uint2 *)p) : make_uint2(0, 0);
    w[0][0] = x.x, w[1][0] = x.y;
}
__device__ __forceinline__ void load_parts(const float *p, bool there, uint32_t (&w)[2][3]) {
    const float4 x = there ? __ldg((const float4 *)p) : make_float4(0.f, 0.f, 0.f, 0.f);
    split_bf16(x.x, x.y, w[0]);
    split_bf16(x.z, x.w, w[1]);
}

// 16 open rows: bf16 enters as it is, fp32 and P as three bf16 parts (products of parts below 2^-24 are left out).  Keys key0 + gid
// (+ 8) of the slot, `rest` of which hold tokens; j0 the token of key0 + gid.
template <typename T, int D>
__device__ __forceinline__ void open_rows(Running<D> &run, const T *q, bool live, const T *k, const T *v, int key0, int rest, int j0,
                                          const int (&lim)[2], float scale2) {
    constexpr int N = sizeof(T) == 4 ? 3 : 1;
    const int lane = threadIdx.x & 31, gid = lane >> 2, tid = lane & 3;
    const int ka = key0 + gid, kb = ka + 8;
    float s[1][4] = {{0.f, 0.f, 0.f, 0.f}}, corr[2];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {  // four dimensions of the lane: 16 i + 4 tid
        const int e = 16 * i + 4 * tid;
        uint32_t x[2][N], y[2][N], z[2][N];
        load_parts(k + ka * D + e, ka < rest, x);
        load_parts(k + kb * D + e, kb < rest, y);
        load_parts(q + e, live, z);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int m = 0; m + n < N; ++m) mma16816_bf16(s[0], x[0][n], y[0][n], x[1][n], y[1][n], z[0][m], z[1][m]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[0][i] = j0 + i / 2 * 8 < lim[i % 2] ? s[0][i] * scale2 : -INFINITY;
    run.weights(s, corr);
    uint32_t pf[2][3];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        split_bf16(s[0][2 * h], s[0][2 * h + 1], pf[h]);
#pragma unroll
        for (int n = 0; n < 3; ++n) pf[h][n] = transposed(pf[h][n]);
    }
#pragma unroll
    for (int e = 0; e < D / 8; e += 4) {
        uint32_t w[4][2][N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = key0 + tid * 2 + i / 2 * 8 + i % 2;
            load_parts(v + key * D + gid * (D / 8) + e, key < rest, w[i]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t a0 = __byte_perm(w[0][j][n], w[1][j][n], 0x5410), a1 = __byte_perm(w[0][j][n], w[1][j][n], 0x7632);
                const uint32_t a2 = __byte_perm(w[2][j][n], w[3][j][n], 0x5410), a3 = __byte_perm(w[2][j][n], w[3][j][n], 0x7632);
#pragma unroll
                for (int m = 0; m + n < 3; ++m) mma16816_bf16(c, a0, a1, a2, a3, pf[0][m], pf[1][m]);
            }
            run.fold(e + 2 * j, c, kDrop, corr);
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) decode_kernel(DecodeArgs p) {
    using Geo = Geometry<D>;
    constexpr bool kTwoParts = sizeof(T) == 4;   // of a query row, of open rows
    constexpr int kWordsT = sizeof(T) == 4 ? 1 : 2;  // elements to a word
    extern __shared__ __align__(128) uint8_t ring[];  // [warp][slot] pages; a warp's result [row][D + 4] in place of its pages
    __shared__ float2 part_ml[kWarps][kRows];
    __shared__ int last_s;
    dependency_wait();
    const ModelView &mv = p.mv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tid = lane & 3;
    uint8_t *mine = ring + warp * Geo::kSlots * Geo::kSlot;
    auto part = [&](int w, int r) { return (float *)(ring + w * Geo::kSlots * Geo::kSlot) + r * (D + 4); };
    const Place place = find_items(p);
    const Shares shares(place.total, gridDim.x, place.groups);
    int64_t at = shares.begin(blockIdx.x);
    const int64_t end = shares.begin(blockIdx.x + 1);
    if (at >= end) return;
    int b = place.b;
    int64_t in_front = place.in_front;
    Request req = place.r;

    for (int piece = 0; at < end; ++piece) {
        while (at >= in_front + req.all_items()) {  // the next request that has work
            in_front += req.all_items();
            req = request_of(p, ++b);
        }
        const PagedInfo &u = req.u;
        const int items = req.items(), unit = quotient(at - in_front, items);
        const int64_t unit_at = in_front + (int64_t)unit * items;
        const int item0 = (int)(at - unit_at), item1 = (int)min((int64_t)items, item0 + (end - at));
        const bool whole = item0 == 0 && item1 == items;
        at += item1 - item0;
        const int rg = unit % req.groups, kvh = unit / req.groups % mv.Hkv, l = unit / req.groups / mv.Hkv;
        // row r of the group: token (rg * 8 + r) / g, query head (rg * 8 + r) % g of the KV head
        const int rows = min(kRows, u.n * mv.g - rg * kRows);
        auto token = [&](int r) { return (rg * kRows + r) / mv.g; };
        auto limit = [&](int r) { return r < rows ? max(0, u.len - u.n + token(r) + 1) : 0; };
        const int least = limit(0), lim[2] = {limit(2 * tid), limit(2 * tid + 1)};

        if (piece > 0) __syncthreads();  // the last piece's results are read: pages may take their place

        // ---- full pages: a page to a warp.  Its three slots take K and V of its pages in turn: one is read, two are on their way.
        const int *table = p.pg.table + (int64_t)b * p.pg.table_width;
        const int page1 = min(item1, req.pages), n_mine = max(0, (page1 - (item0 + warp) + kWarps - 1) / kWarps);
        const uint32_t mine_u = ptx::smem_u32(mine);
        auto number_of = [&](int n) { return n < n_mine ? __ldg(table + item0 + warp + n * kWarps) : 0; };
        auto good = [&](int number) { return number >= 0 && number < p.pg.n_pages; };
        auto place_of = [&](int number) { return p.pg.page_head(mv, l, good(number) ? number : 0, kvh); };  // of a bad one nothing enters the result
        auto fetch = [&](int n, int number, bool is_v) {   // K or V of this warp's n-th page
            if (n < n_mine) {
                const uint8_t *src = (is_v ? p.pg.v : p.pg.k) + place_of(number) * Geo::kSlot;
                const uint32_t slot = mine_u + (2 * n + is_v) % Geo::kSlots * Geo::kSlot;
#pragma unroll
                for (int i = 0; i < Geo::kSlot / 512; ++i) {
                    const int x = (i * 32 + lane) * 16;
                    copy16(slot + Geo::place(x / D, x % D), src + x);
                }
            }
            copies_commit();
        };
        int n0 = number_of(0), n1 = number_of(1), n2 = number_of(2);
        float k_scale = 0.f, v_scale = 0.f;
        if (n_mine > 0) k_scale = __ldg(p.pg.k_scale + place_of(n0)), v_scale = __ldg(p.pg.v_scale + place_of(n0));
        fetch(0, n0, false);
        fetch(0, n0, true);
        fetch(1, n1, false);

        // ---- Q: row gid's dimensions of this lane, scaled into [1, 2); up[r]: what logits of rows 2 tid + r are multiplied by
        uint32_t qh[Geo::kSteps][2], ql[kTwoParts ? Geo::kSteps : 1][2];
        float up[2];
        {
            uint32_t w[D / 4 / kWordsT];
            const T *src = (const T *)p.q.ptr + l * p.q.stride_layer + (int64_t)(kvh * mv.g + (rg * kRows + gid) % mv.g) * p.q.stride_head +
                           (int64_t)(u.row0 + token(gid)) * p.q.stride_tok;
#pragma unroll
            for (int i = 0; i < D / 4 / kWordsT; ++i) w[i] = 0;
            if (gid < rows) {
#pragma unroll
                for (int c = 0; c < Geo::kChunks; ++c)
                    load_words<Geo::kVec / kWordsT>(&w[c * Geo::kVec / kWordsT], src + c * 4 * Geo::kVec + tid * Geo::kVec);
            }
            float top = 0.f, x, y;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                two_of<T>(w, i, x, y);
                top = fmaxf(top, fmaxf(fabsf(x), fabsf(y)));
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            float big, down;
            power_of_two(top, big, down);
            down *= kQueryLift, big *= p.scale2 / kQueryLift;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                two_of<T>(w, i, x, y);
                if constexpr (kTwoParts)
                    split2(x * down, y * down, qh[i / 2][i % 2], ql[i / 2][i % 2]);
                else
                    qh[i / 2][i % 2] = half2_of(x * down, y * down);
            }
            up[0] = __shfl_sync(0xffffffffu, big, 8 * tid);
            up[1] = __shfl_sync(0xffffffffu, big, 8 * tid + 4);
        }
        Running<D> run;
        run.clear();

        {
#pragma unroll 1
            for (int n = 0; n < n_mine; ++n) {
                const float f[2] = {up[0] * k_scale, up[1] * k_scale};
                const bool skip = !good(n0);
                const float vs = v_scale * kDrop;
                if (skip && lane == 0) atomicOr(p.status, FINCH_DEV_BAD_INDEX);
                if (n + 1 < n_mine) k_scale = __ldg(p.pg.k_scale + place_of(n1)), v_scale = __ldg(p.pg.v_scale + place_of(n1));
                copies_wait<2>();
                __syncwarp();
                float s[Geo::kTiles][4];
#pragma unroll
                for (int t = 0; t < Geo::kTiles; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
                {
                    const uint32_t slot = mine_u + 2 * n % Geo::kSlots * Geo::kSlot;
                    constexpr int kW = Geo::kVec / 4;
#pragma unroll
                    for (int c = 0; c < Geo::kChunks; ++c) {
                        uint32_t kw[Geo::kTiles][2][kW];
#pragma unroll
                        for (int t = 0; t < Geo::kTiles; ++t)
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                read_words<kW>(kw[t][h], slot + Geo::place(16 * t + 8 * h + gid, c * 4 * Geo::kVec + tid * Geo::kVec));
                        // a product waits for the one before it on the same accumulator: the tiles take turns
#pragma unroll
                        for (int j = 0; j < kW; ++j)
#pragma unroll
                            for (int t = 0; t < Geo::kTiles; ++t) {
                                const int i = c * kW + j;
                                const uint32_t a0 = codes_lo(kw[t][0][j]), a1 = codes_lo(kw[t][1][j]), a2 = codes_hi(kw[t][0][j]), a3 = codes_hi(kw[t][1][j]);
                                mma16816(s[t], a0, a1, a2, a3, qh[i][0], qh[i][1]);
                                if constexpr (kTwoParts) mma16816(s[t], a0, a1, a2, a3, ql[i][0], ql[i][1]);
                            }
                    }
                }
                __syncwarp();
                fetch(n + 1, n1, true);
                const int j0 = (item0 + warp + n * kWarps) * kPage + gid;
#pragma unroll
                for (int t = 0; t < Geo::kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[t][i] *= f[i % 2];
                if (skip || j0 - gid + kPage > least) {
#pragma unroll
                    for (int t = 0; t < Geo::kTiles; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (skip || j0 + 16 * t + i / 2 * 8 >= lim[i % 2]) s[t][i] = -INFINITY;
                }
                uint32_t hi[Geo::kTiles][2], lo[Geo::kTiles][2];
                float corr[2];
                run.weights(s, corr);
                run.parts(s, hi, lo);
                copies_wait<2>();
                __syncwarp();
                if (!skip) {  // weights of zero take no NaN out: a refused page leaves the result (of which corr is 1, or which is 0) as it is
                    const uint32_t slot = mine_u + (2 * n + 1) % Geo::kSlots * Geo::kSlot;
                    constexpr int kW = Geo::kWords, kHalf = kW > 4 ? kW / 2 : kW;   // words at a time (accumulators: 8 registers a word)
                    static_assert(kW % kHalf == 0 || kW == 5 || kW == 7, "");
                    constexpr int kStep = kW == 5 || kW == 7 ? kW : kHalf;
#pragma unroll
                    for (int w0 = 0; w0 < kW; w0 += kStep) {
                        float c[2 * kStep][4];
#pragma unroll
                        for (int i = 0; i < 2 * kStep; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0.f;
#pragma unroll
                        for (int t = 0; t < Geo::kTiles; ++t) {
                            uint32_t vw[4][kStep];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                read_words<kStep>(vw[i], slot + Geo::place(16 * t + i / 2 * 8 + tid * 2 + i % 2, gid * (D / 8) + w0 * 4));
#pragma unroll
                            for (int w = 0; w < kStep; ++w) {
                                const uint32_t x0 = __byte_perm(vw[0][w], vw[1][w], 0x5140), x1 = __byte_perm(vw[0][w], vw[1][w], 0x7362);
                                const uint32_t y0 = __byte_perm(vw[2][w], vw[3][w], 0x5140), y1 = __byte_perm(vw[2][w], vw[3][w], 0x7362);
                                const uint32_t a0 = codes_lo(x0), a1 = codes_hi(x0), a2 = codes_lo(y0), a3 = codes_hi(y0);
                                const uint32_t e0 = codes_lo(x1), e1 = codes_hi(x1), e2 = codes_lo(y1), e3 = codes_hi(y1);
                                mma16816(c[2 * w], a0, a1, a2, a3, hi[t][0], hi[t][1]);
                                mma16816(c[2 * w + 1], e0, e1, e2, e3, hi[t][0], hi[t][1]);
                                mma16816(c[2 * w], a0, a1, a2, a3, lo[t][0], lo[t][1]);
                                mma16816(c[2 * w + 1], e0, e1, e2, e3, lo[t][0], lo[t][1]);
                            }
                        }
#pragma unroll
                        for (int w = 0; w < kStep; ++w) {
                            run.fold(4 * (w0 + w), c[2 * w], vs, corr);
                            run.fold(4 * (w0 + w) + 2, c[2 * w + 1], vs, corr);
                        }
                    }
                }
                __syncwarp();
                n0 = n1, n1 = n2, n2 = number_of(n + 3);
                fetch(n + 2, n1, false);
            }
            copies_wait<0>();  // empty groups
            __syncwarp();
        }

        // ---- open rows: 16 keys to a warp
        const int rest = item1 == items ? u.len % kPage : 0, key0 = warp * 16;
        if (key0 < rest) {
            const int64_t open = p.pg.open_row(mv, l, u.slot, kvh) * D;
            const int j0 = u.len - rest + key0 + gid;
            open_rows<T, D>(run, (const T *)p.q.ptr + l * p.q.stride_layer + (int64_t)(kvh * mv.g + (rg * kRows + gid) % mv.g) * p.q.stride_head +
                                     (int64_t)(u.row0 + token(gid)) * p.q.stride_tok,
                            gid < rows, (const T *)p.pg.open_k + open, (const T *)p.pg.open_v + open, key0, rest, j0, lim, p.scale2);
        }

        // ---- the warps of the CTA in their order; a thread has four dimensions of a row
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) run.sum[r] += __shfl_xor_sync(0xffffffffu, run.sum[r], x);
            if (gid == 0) part_ml[warp][2 * tid + r] = make_float2(run.m[r], run.sum[r] * kDrop);
#pragma unroll
            for (int i = 0; i < D / 8; i += 4)
                *(float4 *)(part(warp, 2 * tid + r) + gid * (D / 8) + i) = make_float4(run.o[i][r], run.o[i + 1][r], run.o[i + 2][r], run.o[i + 3][r]);
        }
        __syncthreads();
        auto finish = [&](int r, int c, float m, float sum, float4 v) {
            const int h = kvh * mv.g + (rg * kRows + r) % mv.g, t = u.row0 + token(r);
            const int64_t row = attend_row(mv, p.bv.total_q, l, h, t);
            float lse;
            const float inv = attend_finish(m, sum, nullptr, row, lse);
            v = sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
            store4<T>((T *)p.out.ptr + l * p.out.stride_layer + h * p.out.stride_head + (int64_t)t * p.out.stride_tok + c, v);
            if (p.out.row_lse && c == 0) p.out.row_lse[row] = lse;
        };
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
                const float f = ml.y == 0.f ? 0.f : tc::ex2(ml.x - ref);
                sum = fmaf(ml.y, f, sum);
                const float4 y = *(const float4 *)(part(w, r) + c);
                v.x = fmaf(y.x, f, v.x), v.y = fmaf(y.y, f, v.y), v.z = fmaf(y.z, f, v.z), v.w = fmaf(y.w, f, v.w);
            }
            if (whole) {
                finish(r, c, m, sum, v);
            } else {
                const int64_t slot = (2 * (int64_t)blockIdx.x + (piece > 0)) * kRows + r;
                __stcg((float4 *)(p.out.part_o + slot * D + c), v);
                if (c == 0) __stcg(p.out.part_ml + slot, make_float2(m, sum));
            }
        }
        if (whole) continue;
        // ---- the CTA that delivers a unit's last piece adds them
        const int c0 = shares.of(unit_at), c1 = shares.of(unit_at + items - 1);
        __syncthreads();
        if (threadIdx.x == 0) {
            // releases the CTA's pieces, which the barrier has put in front of it, and acquires those of the CTAs before
            int n;
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(n) : "l"(p.pieces + c0) : "memory");
            last_s = n == c1 - c0;
            if (last_s) p.pieces[c0] = 0;  // nobody else comes
        }
        __syncthreads();
        if (!last_s) continue;
        for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4) * 4;
            auto slot_of = [&](int cta) { return (2 * (int64_t)cta + (shares.begin(cta) < unit_at)) * kRows + r; };
            float m = -INFINITY, sum = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            constexpr int kBatch = 8;   // pieces in flight
            for (int base = c0; base <= c1; base += kBatch) {
                float2 ml[kBatch];
                float4 y[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int64_t slot = slot_of(min(base + k, c1));
                    ml[k] = __ldcg(p.out.part_ml + slot);
                    y[k] = __ldcg((const float4 *)(p.out.part_o + slot * D + c));
                    if (base + k > c1) ml[k].y = 0.f;
                }
                float now = m;
#pragma unroll
                for (int k = 0; k < kBatch; ++k)
                    if (ml[k].y != 0.f) now = fmaxf(now, ml[k].x);
                const float ref = now == -INFINITY ? 0.f : now, corr = tc::ex2(m - ref);
                m = now;
                sum *= corr, v.x *= corr, v.y *= corr, v.z *= corr, v.w *= corr;
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    if (ml[k].y == 0.f) continue;  // saw none of the row's keys
                    const float f = tc::ex2(ml[k].x - ref);
                    sum = fmaf(ml[k].y, f, sum);
                    v.x = fmaf(y[k].x, f, v.x), v.y = fmaf(y[k].y, f, v.y), v.z = fmaf(y[k].z, f, v.z), v.w = fmaf(y[k].w, f, v.w);
                }
            }
            finish(r, c, m, sum, v);
        }
    }
}

template <typename T, int D>
cudaError_t launch(const Ctx &ctx, const DecodeArgs &p, dim3 grid, cudaStream_t stream) {
    const int bit = kSmemDecode + (sizeof(T) == 4);  // a context has one head dimension
    if (!ctx.smem_ready(bit)) {
        cudaError_t e = cudaFuncSetAttribute(decode_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geometry<D>::kSmem);
        if (e != cudaSuccess) return e;
        ctx.smem_set(bit);
    }
    ctx.launches += 1;
    return launch_chained(decode_kernel<T, D>, grid, dim3(kThreads), Geometry<D>::kSmem, stream, p);
}
template <typename T>
cudaError_t launch_t(const Ctx &ctx, const DecodeArgs &p, dim3 grid, cudaStream_t stream) {
    switch (p.mv.d) {
        case 32: return launch<T, 32>(ctx, p, grid, stream);
        case 64: return launch<T, 64>(ctx, p, grid, stream);
        case 96: return launch<T, 96>(ctx, p, grid, stream);
        case 128: return launch<T, 128>(ctx, p, grid, stream);
        case 160: return launch<T, 160>(ctx, p, grid, stream);
        case 192: return launch<T, 192>(ctx, p, grid, stream);
        case 224: return launch<T, 224>(ctx, p, grid, stream);
        case 256: return launch<T, 256>(ctx, p, grid, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

int pages_ctas(int sms) { return kCtasPerSm * sms; }

cudaError_t launch_pages_attend(const Ctx &ctx, const PagesView &pg, const PagedView &bv, const TensorView &q, AttendOut out,
                                cudaStream_t stream) {
    if (bv.batch == 0 || bv.max_q == 0) return cudaSuccess;
    const ModelView &mv = ctx.model;
    const DecodeArgs p = {mv, pg, bv, q, out, ctx.pieces, ctx.d_status, mv.scale * kLog2e};
    const int64_t max_units = (int64_t)mv.L * mv.Hkv * ((bv.max_q * (int64_t)mv.g + kRows - 1) / kRows);
    if (max_units * kRows > INT_MAX) return cudaErrorInvalidConfiguration;
    // Every warp of a CTA a page where there are few; for a single request whole numbers of CTAs to a unit, where that takes no more
    // than a tenth of them away.
    const int64_t pages = (bv.max_len + kPage - 1) / kPage > 0 ? (bv.max_len + kPage - 1) / kPage : 1;
    const int most = pages_ctas(ctx.sm_count);
    int64_t per_unit = (pages + kWarps - 1) / kWarps;
    if (per_unit * max_units * bv.batch > most) per_unit = most / max_units;
    const int64_t aligned = per_unit * max_units, shared = max_units * bv.batch * ((pages + kWarps - 1) / kWarps);
    int ctas = (int)(shared < most ? shared : most);
    if (bv.batch == 1 && 10 * aligned >= 9 * (int64_t)ctas) ctas = (int)aligned;
    return mv.elem_bytes == 4 ? launch_t<float>(ctx, p, dim3(ctas), stream) : launch_t<__nv_bfloat16>(ctx, p, dim3(ctas), stream);
}

}  // namespace finch
