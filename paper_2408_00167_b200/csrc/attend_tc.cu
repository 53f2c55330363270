// Attention of packed query rows over [cache ; chunk] on the tensor cores (bf16, head dimensions up to 128).
//
//   S = Q K^T, O = softmax(S) V, a row's softmax over its first `limit` candidates, by the online recurrence over key tiles:
//   m' = max(m, max S), O = O 2^(m - m') + P V with P = 2^(S - m'), l = l 2^(m - m') + sum P.
//
// Rows.  A tile is 128 rows of one KV head: all its query heads (they share every key) times as many tokens as fit, row =
// head * tok + token, which is how one TMA box lays them out.  Keys come in tiles of 128 that do not straddle the cache / chunk seam.
//
// Streams.  A CTA works on two streams at a time, a softmax warpgroup each, so that the tensor core multiplies for one while the other
// exponentiates: two row tiles against the same keys, or, for requests of a single row tile, one row tile against the even and
// the odd key tiles (whose results are added through shared memory at the end).  Or two CTAs with one stream each share an SM.
//
// Tensor memory (512 columns): S of each stream (128), over whose first half P is written as bf16, and O of each stream.  P never leaves
// tensor memory: it is the A operand of P V.  V tiles are B operands with their rows along K.
// Order.  One thread issues S(s, i+1) behind P V (s, i): the completion of S then says that O is at rest, and the softmax warps
// may scale it.  They do so only when a row's maximum has grown by more than 2^8: until then P is taken against the old reference.
//
// A masked key has P = 0, but zero times a NaN or infinity is none: rows of V behind the last candidate, and behind the last that a
// row of the CTA sees where there are row limits, are cleared before they are multiplied.
#include "attend.cuh"

namespace finch {
namespace {

using namespace ptx;
using namespace tc;

constexpr float kGrowth = 8.f;       // binary orders that a row's maximum may grow before O is scaled
constexpr int kTileRows = 128;
constexpr int kFewTiles = 5, kManyTiles = 32;  // key tiles of one-stream CTAs: always, where every SM has work
constexpr int kMaxCluster = 4;
constexpr int kMaxParts = 2 * kMaxCluster;  // results of a row that meet in a cluster: its CTAs', of both streams where they share a row tile

struct TcArgs {
    ModelView mv;
    BatchView bv;
    AttendOut out;
    int *status;
    int causal, heads, tok, chunks, row_tiles;  // query heads and tokens of a row tile; tiles of heads per KV head; CTAs along the tokens
    int two_tiles;                               // streams are two row tiles (else: one tile's even and odd key tiles)
    int cluster;                                 // consecutive splits whose CTAs are a cluster and add their results there
    float scale2;
};

struct Maps {
    CUtensorMap q, ck, cv, hk, hv;
};

template <int S>
struct Stream {
    static constexpr int value = S;
};

// STREAMS = 2: one CTA to an SM.  STREAMS = 1: a CTA works on one row tile, two of them share an SM (and its tensor memory), and each is
// loaded, set up and written out under the other's work: for many short requests, where these take longer than the products.
template <int DP, int STREAMS>
struct Layout {
    static constexpr int kSlabs = DP / 64;
    static constexpr int kTile = kSlabs * kSlabBytes;
    static constexpr int kStages = STREAMS == 2 ? (DP == 128 ? 5 : 8) : (DP == 128 ? 2 : 5);
    static constexpr int kBytes = (STREAMS + kStages) * kTile + 1024;
    static constexpr int kThreads = 128 + STREAMS * 128;   // 4 control warps, 4 softmax warps to a stream
    static constexpr int kColumns = STREAMS * 256;         // of tensor memory
};

struct Barriers {
    uint64_t q_full[2], full[8], empty[8], s_full[2], p_full[2], o_full[2];
    uint64_t ragged[2], clean[2];  // the cache's, the chunk's last V tile: on its way, cleared behind its rows
};

// Where four columns of a row lie in a box: of 128 rows one behind the other, so that a warp's rows are read as one run.
__device__ __forceinline__ int piece_at(int row, int piece) { return (piece * 128 + row) * 16; }

// Where one row's result goes: the output and its log-sum-exp, or (unnormalised) the partial results of a split.
struct Row {
    const TcArgs &p;
    int64_t row, slot;
    __nv_bfloat16 *dst;
    bool writes, partial;
    float inv;
    __device__ __forceinline__ Row(const TcArgs &args, const UnitInfo &u, int l, int h, int t, bool w, int split) : p(args), writes(w), inv(1.f) {
        partial = p.out.splits > p.cluster;
        row = w ? attend_row(p.mv, p.bv.total_q, l, h, u.q0 + t) : 0;
        slot = split * ((int64_t)p.mv.L * p.mv.Hq * p.bv.total_q) + row;
        dst = (__nv_bfloat16 *)p.out.ptr + (int64_t)l * p.out.stride_layer + (int64_t)h * p.out.stride_head + (int64_t)(u.q0 + t) * p.out.stride_tok;
    }
    __device__ __forceinline__ void finish(float m, float l, bool notes = true) {
        if (!writes) return;
        if (partial) {
            if (notes) p.out.part_ml[slot] = make_float2(m, l);
            return;
        }
        float lse;
        inv = attend_finish(m, l, p.bv.self_lse, row, lse);   // 0 for a row without keys
        if (notes && p.out.row_lse) p.out.row_lse[row] = lse;
    }
    __device__ __forceinline__ void put(int c, const float *y) {  // eight columns
        if (!writes) return;
        if (partial) {
            float *po = p.out.part_o + slot * p.mv.d + c;
            *(float4 *)po = make_float4(y[0], y[1], y[2], y[3]);
            *(float4 *)(po + 4) = make_float4(y[4], y[5], y[6], y[7]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(y[2 * k + 1] * inv), "f"(y[2 * k] * inv));
            *(uint4 *)(dst + c) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

template <int DP, int STREAMS>
__global__ void __launch_bounds__(Layout<DP, STREAMS>::kThreads, 3 - STREAMS)
attend_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ TcArgs p) {
    using Lay = Layout<DP, STREAMS>;
    extern __shared__ uint8_t raw[];
    __shared__ Barriers bar;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    __shared__ int limit_s[2];
    uint8_t *smem = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    uint8_t *q_smem = smem, *ring = smem + STREAMS * Lay::kTile;
    // a stream's result in the ring's place: O of 128 rows, then (m, l) of each
    auto box = [&](int s) { return ring + s * (DP * 512 + 1024); };
    static_assert(STREAMS == 1 || 2 * (DP * 512 + 1024) <= Lay::kStages * Lay::kTile, "results take the ring's place");
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    dependency_wait();
    const ModelView &mv = p.mv;
    const int b = blockIdx.y;
    int x = blockIdx.x;
    const int split = x % p.out.splits;
    x /= p.out.splits;
    const int hc = x % p.chunks;
    x /= p.chunks;
    const int kvh = x % mv.Hkv, l = x / mv.Hkv % mv.L, tile = p.row_tiles - 1 - x / mv.Hkv / mv.L;  // long causal rows first
    const UnitInfo u = unit_info(mv, p.bv, 0, b);
    if (!u.ok) {
        if (threadIdx.x == 0) atomicOr(p.status, FINCH_DEV_BAD_BATCH);
        return;
    }
    const bool two_tiles = STREAMS == 2 && p.two_tiles;
    const int t0 = tile * (two_tiles ? 2 : 1) * p.tok;
    if (t0 >= u.n_q) return;
    const int h0 = kvh * mv.g + hc * p.heads, n_heads = min(p.heads, mv.g - hc * p.heads);

    // ---- set-up; how many candidates the rows of each stream see at most
    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&maps.q), prefetch_tensormap(&maps.ck), prefetch_tensormap(&maps.cv), prefetch_tensormap(&maps.hk), prefetch_tensormap(&maps.hv);
            for (int i = 0; i < Lay::kStages; ++i) mbar_init(&bar.full[i], 1), mbar_init(&bar.empty[i], 1);
            for (int i = 0; i < 2; ++i)
                mbar_init(&bar.q_full[i], 1), mbar_init(&bar.s_full[i], 1), mbar_init(&bar.p_full[i], 4), mbar_init(&bar.o_full[i], 1), mbar_init(&bar.ragged[i], 1), mbar_init(&bar.clean[i], 1);
            abort_flag = 0;
            fence_barrier_init();
        }
    } else if (warp == 1) {
        tmem_alloc(&tmem_slot, Lay::kColumns);
        tmem_relinquish();
    } else {
        const int s = warp - 2;
        if (s < STREAMS) {
            int most = 0;
            const int ts = t0 + (two_tiles ? s * p.tok : 0);
            for (int i = lane; i < p.tok; i += 32)
                if (ts + i < u.n_q) most = max(most, attend_limit(p.bv, u, ts + i, p.causal));
            most = __reduce_max_sync(0xffffffffu, most);
            if (lane == 0) limit_s[s] = most;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    // ---- key tiles of the CTA's split and of each stream
    const int cache_tiles = (u.c + kTileRows - 1) / kTileRows;
    auto tiles_for = [&](int limit) {
        return limit <= u.c ? (limit + kTileRows - 1) / kTileRows : cache_tiles + (limit - u.c + kTileRows - 1) / kTileRows;
    };
    const int all0 = tiles_for(limit_s[0]), all1 = STREAMS == 2 ? tiles_for(limit_s[1]) : 0, all = max(all0, all1);
    const int begin = (int)((int64_t)all * split / p.out.splits), end = (int)((int64_t)all * (split + 1) / p.out.splits);
    const int n_tiles = end - begin;                    // loaded
    // What a key tile holds for this CTA: with row limits, candidates behind the largest of its rows' may be memory that nobody has
    // written, like those behind the request's last.
    UnitInfo held = u;
    if (p.bv.row_limit) {
        const int most = STREAMS == 2 ? max(limit_s[0], limit_s[1]) : limit_s[0];
        held.c = min(u.c, most), held.m = max(0, most - u.c);
    }
    int count[2];                                        // of each stream
    if (STREAMS == 1) {
        count[0] = n_tiles, count[1] = 0;
    } else if (two_tiles) {
        count[0] = max(0, min(end, all0) - begin), count[1] = max(0, min(end, all1) - begin);
    } else {
        count[0] = (n_tiles + 1) / 2, count[1] = n_tiles / 2;
    }
    const bool gathers = STREAMS == 2 && (p.cluster > 1 || (!two_tiles && count[1] > 0));   // rows' results meet others in shared memory
    auto tile_of = [&](int s, int i) { return two_tiles || STREAMS == 1 ? i : 2 * i + s; };  // in the split
    // the last stream to use a tile frees it
    auto frees = [&](int s, int t) { return !two_tiles || s == 1 || t >= count[1]; };
    constexpr int kStages = Lay::kStages;

    if (warp < 4) regs_dec<STREAMS == 2 ? 104 : 72>();
    if (warp == 0) {
        // ---------------------------------------------------------------- producer
        if (lane == 0 && n_tiles > 0) {
            int item = 0, slot = 0;
            uint32_t ph = 1;   // of the slot's last reader: the first round waits for nobody
            bool ok = true;
            for (int t = 0; t < n_tiles && ok; ++t) {
                const KeyTile kt = key_tile(held, begin + t);
                for (int v = 0; v < 2; ++v, ++item, slot = slot + 1 == kStages ? (ph ^= 1, 0) : slot + 1) {
                    if (item >= kStages && !(ok = mbar_wait(&bar.empty[slot], ph, &abort_flag))) break;
                    mbar_expect_tx(&bar.full[slot], Lay::kTile);
                    const CUtensorMap *map = kt.is_chunk ? (v ? &maps.hv : &maps.hk) : (v ? &maps.cv : &maps.ck);
                    for (int c = 0; c < Lay::kSlabs; ++c)
                        tma_load_4d(ring + slot * Lay::kTile + c * kSlabBytes, map, &bar.full[slot], c * 64, kt.row0, kvh, l);
                    if (v && kt.valid < kTileRows) mbar_arrive(&bar.ragged[kt.is_chunk]);
                }
            }
            // no copy of this CTA is in flight when its shared memory goes to another
            for (int i = max(0, item - kStages); i < item; ++i) mbar_wait(&bar.full[i % kStages], (i / kStages) & 1, &abort_flag);
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issuer
        // The whole warp keeps the control flow, so that addresses and descriptors are warp-uniform; one lane issues.  This warp's
        // instructions are on the path of both streams: everything that is the same for every tile is formed in front of the loop.
        if (n_tiles > 0) {
            constexpr uint32_t idesc_s = idesc_bf16_f32(128, 128), idesc_o = idesc_bf16_f32(128, DP) | kIdescBMn;
            constexpr uint32_t kTile16 = Lay::kTile / 16;   // descriptors count 16 bytes
            auto agree = [](bool ok) { return __all_sync(0xffffffffu, ok) != 0; };
            bool ok = true;
            const uint32_t q_u = smem_u32(q_smem), ring_u = smem_u32(ring);
            const uint64_t qd0 = smem_desc_sw128(q_u), qd[2] = {qd0, two_tiles ? qd0 + kTile16 : qd0};
            const uint64_t kd = smem_desc_sw128(ring_u), vd = smem_desc_sw128_mn(ring_u, kSlabBytes);
            // the tiles whose V rows are cleared behind the last token: the cache's last, the chunk's last
            const int held_tiles = (held.c + kTileRows - 1) / kTileRows;
            const int ragged0 = held.c % kTileRows ? held_tiles - 1 - begin : -1;
            const int ragged1 = held.m % kTileRows ? held_tiles + (held.m + kTileRows - 1) / kTileRows - 1 - begin : -1;
            const int step = two_tiles || STREAMS == 1 ? 2 : 4;           // items from a stream's tile to its next
            // slot and phase of each stream's next K and V item
            int k_slot[2], v_slot[2], tile_k[2], tile_v[2];
            uint32_t k_ph[2] = {0, 0}, v_ph[2] = {0, 0}, p_ph[2] = {0, 0};
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                tile_k[s] = tile_v[s] = tile_of(s, 0);
                k_slot[s] = 2 * tile_k[s], v_slot[s] = k_slot[s] + 1;   // below kStages
            }
            auto issue_s = [&](auto stream) {
                constexpr int s = decltype(stream)::value;
                if (!agree(mbar_wait_now(&bar.full[k_slot[s]], k_ph[s], &abort_flag))) return false;
                tc_fence_after();
                const uint64_t b_desc = kd + k_slot[s] * kTile16;
                const bool last = frees(s, tile_k[s]);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k) {
                        const uint32_t at = ((k / 4) * kSlabBytes + (k % 4) * 32) / 16;
                        if (k == 0)
                            umma_bf16_first(tmem + s * 128, qd[s] + at, b_desc + at, idesc_s);
                        else
                            umma_bf16_acc(tmem + s * 128, qd[s] + at, b_desc + at, idesc_s);
                    }
                    umma_commit(&bar.s_full[s]);
                    if (last) umma_commit(&bar.empty[k_slot[s]]);
                }
                __syncwarp();
                tile_k[s] += step / 2;
                k_slot[s] += step;
                while (k_slot[s] >= kStages) k_slot[s] -= kStages, k_ph[s] ^= 1;
                return true;
            };
            auto issue_o = [&](auto stream, int i) {
                constexpr int s = decltype(stream)::value;
                const int t = tile_v[s];
                if (!agree(mbar_wait_now(&bar.full[v_slot[s]], v_ph[s], &abort_flag))) return false;
                if (t == ragged0 && !agree(mbar_wait_now(&bar.clean[0], 0, &abort_flag))) return false;
                if (t == ragged1 && !agree(mbar_wait_now(&bar.clean[1], 0, &abort_flag))) return false;
                if (!agree(mbar_wait_now(&bar.p_full[s], p_ph[s], &abort_flag))) return false;
                tc_fence_after();
                const uint64_t b_desc = vd + v_slot[s] * kTile16;
                const bool last = frees(s, t), end = i + 1 == count[s];
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kTileRows / 16; ++k)
                        umma_bf16_tmem(tmem + STREAMS * 128 + s * DP, tmem + s * 128 + k * 8, b_desc + k * (2048 / 16), idesc_o, i > 0 || k > 0);
                    if (last) umma_commit(&bar.empty[v_slot[s]]);
                    if (end) umma_commit(&bar.o_full[s]);
                }
                __syncwarp();
                p_ph[s] ^= 1;
                tile_v[s] += step / 2;
                v_slot[s] += step;
                while (v_slot[s] >= kStages) v_slot[s] -= kStages, v_ph[s] ^= 1;
                return true;
            };
            const Stream<0> s0;
            const Stream<1> s1;
            if (count[0] > 0) ok = agree(mbar_wait_now(&bar.q_full[0], 0, &abort_flag)) && issue_s(s0);
            if (STREAMS == 2 && ok && count[1] > 0) ok = agree(mbar_wait_now(&bar.q_full[two_tiles], 0, &abort_flag)) && issue_s(s1);
            const int most = max(count[0], count[1]);
            for (int i = 0; ok && i < most; ++i) {
                if (i < count[0]) ok = issue_o(s0, i);
                if (ok && i + 1 < count[0]) ok = issue_s(s0);
                if (STREAMS == 2 && ok && i < count[1]) ok = issue_o(s1, i);
                if (STREAMS == 2 && ok && i + 1 < count[1]) ok = issue_s(s1);
            }
        }
    } else if (warp == 3) {
        // ---------------------------------------------------------------- queries, beside the first keys
        if (lane == 0 && n_tiles > 0) {
            for (int s = 0; s < (two_tiles ? 2 : 1); ++s) {
                mbar_expect_tx(&bar.q_full[s], Lay::kSlabs * p.tok * p.heads * 128);
                for (int c = 0; c < Lay::kSlabs; ++c)
                    tma_load_4d(q_smem + s * Lay::kTile + c * kSlabBytes, &maps.q, &bar.q_full[s], c * 64, u.q0 + t0 + s * p.tok, h0, l);
            }
            for (int s = 0; s < (two_tiles ? 2 : 1); ++s) mbar_wait(&bar.q_full[s], 0, &abort_flag);
        }
    } else if (warp == 2) {
        // ---------------------------------------------------------------- V rows behind the last candidate that counts
        for (int t = 0; t < n_tiles; ++t) {
            const KeyTile kt = key_tile(held, begin + t);
            if (kt.valid == kTileRows) continue;
            const int item = 2 * t + 1, slot = item % kStages;
            // this warp has not seen the slot's earlier phases: it waits until the slot is this tile's, then for its bytes
            if (!__all_sync(0xffffffffu, mbar_wait_relaxed(&bar.ragged[kt.is_chunk], 0, &abort_flag, 200) &&
                                             mbar_wait(&bar.full[slot], (item / kStages) & 1, &abort_flag)))
                break;
            for (int i = lane; i < (kTileRows - kt.valid) * 8; i += 32)
#pragma unroll
                for (int c = 0; c < Lay::kSlabs; ++c)
                    *(uint4 *)(ring + slot * Lay::kTile + c * kSlabBytes + kt.valid * 128 + i * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.clean[kt.is_chunk]);
        }
    } else if (warp >= 4) {
        // ---------------------------------------------------------------- softmax
        regs_inc<STREAMS == 2 ? 200 : 184>();
        const int s = STREAMS == 2 ? (warp - 4) / 4 : 0, quarter = warp % 4, r = quarter * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t st = tmem + s * 128 + lane_base, ot = tmem + STREAMS * 128 + s * DP + lane_base;
        const int hr = r / p.tok, tr = t0 + (two_tiles ? s * p.tok : 0) + r % p.tok;
        const bool live = hr < n_heads && tr < u.n_q;
        const int limit = live ? attend_limit(p.bv, u, tr, p.causal) : u.N;
        // columns of tile t (of the request) that this row sees: one of these minus 128 t
        const int in_cache = min(limit, u.c), in_chunk = limit - u.c + cache_tiles * kTileRows;
        const float growth = kGrowth / p.scale2;
        float m = -INFINITY, sum = 0.f;
        bool ok = true;
        for (int i = 0; i < count[s]; ++i) {
            const int t = begin + tile_of(s, i), nv = (t < cache_tiles ? in_cache : in_chunk) - t * kTileRows;
            if (!(ok = __all_sync(0xffffffffu, mbar_wait_now(&bar.s_full[s], i & 1, &abort_flag)))) break;
            tc_fence_after();
            uint32_t v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_issue(st + c * 32, v[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_wait(v[c]);
            if (__any_sync(0xffffffffu, nv < kTileRows)) {
                keep_branch();
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c * 32 + e >= nv) v[c][e] = 0xff800000u;  // -inf
            }
            float top = fmaxf(fmaxf(chunk_max(v[0]), chunk_max(v[1])), fmaxf(chunk_max(v[2]), chunk_max(v[3])));
            if (__any_sync(0xffffffffu, live && top > m + growth)) {  // always at the first tile
                keep_branch();
                if (i > 0) {
                    const float now = top > m + growth ? top : m;
                    const float f = now == m ? 1.f : ex2((m - now) * p.scale2);
                    sum *= f;
                    m = now;
#pragma unroll 1
                    for (int c = 0; c < DP / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld_issue(ot + c * 32, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        tmem_st(ot + c * 32, o);
                    }
                    tmem_st_wait();
                } else {
                    m = top;
                }
            }
            const float negm = m == -INFINITY ? 0.f : -(m * p.scale2);
            const uint64_t s2 = pack2(p.scale2, p.scale2), n2 = pack2(negm, negm);
            uint64_t acc0 = 0, acc1 = 0;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t w[32];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const uint32_t *src = &v[2 * c + e / 16][e % 16 * 2];
                    const uint64_t a = exp2_pair(fma2(pack2(__uint_as_float(src[0]), __uint_as_float(src[1])), s2, n2));
                    const uint64_t d = exp2_pair(fma2(pack2(__uint_as_float(src[2]), __uint_as_float(src[3])), s2, n2));
                    acc0 = add2(acc0, a);
                    acc1 = add2(acc1, d);
                    float a0, a1, d0, d1;
                    unpack2(a, a0, a1);
                    unpack2(d, d0, d1);
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[e]) : "f"(a1), "f"(a0));
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[e + 1]) : "f"(d1), "f"(d0));
                }
                tmem_st(st + c * 32, w);
            }
            sum += sum_of(acc0, acc1);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.p_full[s]);
        }
        // ---- the row's result
        if (count[s] > 0 && ok) ok = __all_sync(0xffffffffu, mbar_wait_now(&bar.o_full[s], 0, &abort_flag));
        tc_fence_after();
        const float m2 = m * p.scale2;   // the reference in base-2 logits (-inf: none of the row's keys)
        if (!gathers) {
            Row row(p, u, l, h0 + hr, tr, live && (two_tiles || s == 0), split);
            row.finish(m2, sum);
#pragma unroll 1
            for (int c = 0; c < mv.d; c += 16) {
                uint32_t o[16];
                float y[16];
                if (count[s] > 0) {
                    tmem_ld_issue(ot + c, o);
                    tmem_ld_wait(o);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) y[e] = count[s] > 0 ? __uint_as_float(o[e]) : 0.f;
                row.put(c, y);
                row.put(c + 8, y + 8);
                __syncwarp();
            }
        } else if constexpr (STREAMS == 2) {
            // the pages' place is free when the other stream's MMAs are complete, too
            if (count[1 - s] > 0 && ok) ok = __all_sync(0xffffffffu, mbar_wait_now(&bar.o_full[1 - s], 0, &abort_flag));
            tc_fence_after();
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (count[s] > 0) {
#pragma unroll 1
                for (int c = 0; c < DP; c += 16) {
                    uint32_t o[16];
                    tmem_ld_issue(ot + c, o);
                    tmem_ld_wait(o);
#pragma unroll
                    for (int e = 0; e < 16; e += 4) *(uint4 *)(box(s) + piece_at(r, (c + e) / 4)) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                }
            }
            *(float2 *)(box(s) + DP * 512 + r * 8) = make_float2(m2, count[s] > 0 ? sum : 0.f);
        }
        tc_fence_before();
    }
    if constexpr (STREAMS == 2) if (gathers) {
        // ---- the streams and the CTAs that worked on the same rows: every CTA adds all of them for some columns
        __syncwarp();
        if (p.cluster > 1) {
            cluster_arrive();
            cluster_wait();
        } else if (warp >= 4) {
            asm volatile("bar.sync 1, 256;" ::: "memory");
        }
        if (warp >= 4) {
            const int rank = split % p.cluster, r = warp % 4 * 32 + lane;
            const int sets = two_tiles ? 2 : 1, parts = two_tiles ? p.cluster : 2 * p.cluster;
            const uint32_t box0 = smem_u32(box(0)), box1 = smem_u32(box(1));
            auto add = [&](auto remote) {
                constexpr bool kRemote = decltype(remote)::value == 1;
                for (int set = 0; set < sets; ++set) {
                    const int hr = r / p.tok, tr = t0 + set * p.tok + r % p.tok;
                    Row row(p, u, l, h0 + hr, tr, hr < n_heads && tr < u.n_q, split / p.cluster);
                    auto part_at = [&](int j) {
                        const uint32_t at = (two_tiles ? set : j % 2) ? box1 : box0;
                        return kRemote ? map_to_rank(at, two_tiles ? j : j / 2) : at;
                    };
                    float m[kMaxParts], f[kMaxParts], ref = -INFINITY, total = 0.f;
#pragma unroll
                    for (int j = 0; j < kMaxParts; ++j) {
                        m[j] = -INFINITY, f[j] = 0.f;
                        if (j < parts) {
                            const uint32_t at = part_at(j) + DP * 512 + r * 8;
                            const float2 ml = kRemote ? ld_remote(at) : lds64(at);
                            m[j] = ml.x, f[j] = ml.y;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < kMaxParts; ++j)
                        if (f[j] != 0.f) ref = fmaxf(ref, m[j]);
                    const float base = ref == -INFINITY ? 0.f : ref;
#pragma unroll
                    for (int j = 0; j < kMaxParts; ++j) {
                        const float g = f[j] == 0.f ? 0.f : ex2(m[j] - base);
                        total = fmaf(f[j], g, total);
                        f[j] = g;
                    }
                    row.finish(ref, total, rank == 0 && warp < 8);
#pragma unroll 1
                    for (int c = (rank + (warp - 4) / 4 * p.cluster) * 8; c < mv.d; c += 16 * p.cluster) {
                        float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j0 = 0; j0 < kMaxParts; j0 += 4) {
                            if (j0 >= parts) break;
                            float4 a[4][2];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (j0 + j < parts) {
                                    const uint32_t at = part_at(j0 + j) + piece_at(r, c / 4);
                                    a[j][0] = kRemote ? ld_remote_f32x4(at) : lds128(at);
                                    a[j][1] = kRemote ? ld_remote_f32x4(at + 2048) : lds128(at + 2048);
                                }
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (f[j0 + j] != 0.f) {  // .. and was written
                                    const float g = f[j0 + j];
                                    y[0] = fmaf(a[j][0].x, g, y[0]), y[1] = fmaf(a[j][0].y, g, y[1]), y[2] = fmaf(a[j][0].z, g, y[2]), y[3] = fmaf(a[j][0].w, g, y[3]);
                                    y[4] = fmaf(a[j][1].x, g, y[4]), y[5] = fmaf(a[j][1].y, g, y[5]), y[6] = fmaf(a[j][1].z, g, y[6]), y[7] = fmaf(a[j][1].w, g, y[7]);
                                }
                        }
                        row.put(c, y);
                    }
                }
            };
            if (p.cluster > 1) add(Stream<1>{}); else add(Stream<0>{});
        }
        if (p.cluster > 1) {
            __syncwarp();
            cluster_arrive();
            cluster_wait();   // nobody reads this CTA's shared memory any more
        }
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, Lay::kColumns);
    }
    if (threadIdx.x == 0 && abort_flag) atomicOr(p.status, FINCH_DEV_TIMEOUT);
}

template <int DP, int STREAMS>
cudaError_t launch(const Ctx &ctx, const Maps &maps, const TcArgs &p, dim3 grid, cudaStream_t stream) {
    using Lay = Layout<DP, STREAMS>;
    const int bit = kSmemAttendTc + (STREAMS == 2);   // a context has one head dimension
    if (!ctx.smem_ready(bit)) {
        cudaError_t e = cudaFuncSetAttribute(attend_tc_kernel<DP, STREAMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay::kBytes);
        if (e != cudaSuccess) return e;
        ctx.smem_set(bit);
    }
    ctx.launches += 1;
    return launch_chained_cluster(attend_tc_kernel<DP, STREAMS>, p.cluster, grid, dim3(Lay::kThreads), Lay::kBytes, stream, maps, p);
}

// A map of a row tile's queries: one box is `tok` tokens of `heads` heads.
bool make_q_map(CUtensorMap *map, const TensorView &t, int d, int64_t tokens, int heads, int layers, int tok, int box_heads) {
    EncodeTiledFn fn = encode_fn();
    if (!fn || !t.ptr || tokens <= 0) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)tokens, (cuuint64_t)heads, (cuuint64_t)layers};
    const cuuint64_t strides[3] = {(cuuint64_t)t.stride_tok * 2, (cuuint64_t)t.stride_head * 2, (cuuint64_t)t.stride_layer * 2};
    for (int i = 0; i < 3; ++i)
        if (strides[i] == 0 || strides[i] % 16 || strides[i] >= (1ull << 40)) return false;
    const cuuint32_t box[4] = {64, (cuuint32_t)tok, (cuuint32_t)box_heads, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<char *>(t.ptr), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Key splits of a call of `units` CTAs with `tiles` key tiles at most: first the CTAs of a cluster, then, for few rows and long
// contexts, several clusters whose results merge_splits adds.  In microseconds, measured with 512 rows a KV head on 8 of them: a key tile
// takes a CTA 1.8 (two row tiles) or 0.85 (two streams on one), the sum in a cluster of c CTAs about 8 or 1 + 0.8 c, a merge of
// clusters about 5 (128 prompt rows over 2176 keys: 26 without, 20 with clusters of two, 19 of four; 32 rows over 8224: 66, 41,
// 28, and 22 as four clusters of four).
void choose_splits(int sms, int64_t units, int tiles, int two_tiles, size_t room, int &cluster, int &splits) {
    cluster = splits = 1;
    const double tile_us = two_tiles ? 1.8 : 0.85;
    const int64_t slots = (int64_t)(sms / 18) * 16;   // SMs of GPCs of 16 to 18, in whole clusters
    auto waves = [&](int64_t ctas) { return (double)((ctas + sms - 1) / sms); };
    double best = waves(units) * tiles * tile_us;
    for (int c = 2; c <= kMaxCluster; c *= 2) {
        if (units * c > slots || tiles < 2 * c) break;
        const double t = (double)((tiles + c - 1) / c) * tile_us + (two_tiles ? 8.0 : 1.0 + 0.8 * c);
        if (t < best) best = t, cluster = splits = c;
    }
    if (cluster == kMaxCluster) {
        for (int g = 2; g <= kAttendMaxSplits && (size_t)g <= room; ++g) {
            const int c = cluster * g;
            if (units * c > slots || tiles < 2 * c) break;
            const double t = (double)((tiles + c - 1) / c) * tile_us + (two_tiles ? 8.0 : 1.0 + 0.8 * cluster) + 5.0;
            if (t < best) best = t, splits = c;
        }
    }
}

struct Plan {
    int heads, tok, chunks;   // query heads and tokens of a row tile, tiles of heads per KV head
    int two_tiles, row_tiles; // as in TcArgs
    bool one_stream;
    int cluster, splits;      // splits: all of a row's, cluster * clusters
};

// Host arithmetic on the batch's bounds.  room: partial results that there is place for, in sets of all rows.
Plan make_plan(const Ctx &ctx, const BatchView &bv, size_t room) {
    const ModelView &mv = ctx.model;
    const int sms = ctx.sm_count > 0 ? ctx.sm_count : 148;   // a validation-only context has none
    Plan n;
    n.heads = mv.g < kTileRows ? mv.g : kTileRows;
    n.tok = kTileRows / n.heads;
    n.chunks = (mv.g + n.heads - 1) / n.heads;
    // Two row tiles to a CTA, unless that leaves more than half of the SMs without one.
    const int64_t units = (int64_t)mv.L * mv.Hkv * n.chunks, one_tile = units * bv.batch * ((bv.max_q + n.tok - 1) / n.tok);
    n.two_tiles = bv.max_q > n.tok && 2 * one_tile > sms;
    const int key_tiles = (bv.max_cache + kTileRows - 1) / kTileRows + (bv.max_chunk + kTileRows - 1) / kTileRows;
    // One row tile to a CTA, two CTAs to an SM, where the keys are few, or not many and every SM has work (rows of 32 KV heads: 16 requests
    // of up to 512 66 us with two streams to a CTA, 51 with one; 64 of up to 64 97 and 48; 512 rows 15.9 and 14.3; but 64 rows of 4 requests
    // over 4160 keys 38 and 51, 1024 rows over 5120 87 and 90, 8192 rows of 8 KV heads 463 and 471)
    n.one_stream = key_tiles <= kFewTiles || (key_tiles <= kManyTiles && one_tile > sms);
    const int per_cta = n.two_tiles && !n.one_stream ? 2 * n.tok : n.tok;
    n.row_tiles = (bv.max_q + per_cta - 1) / per_cta;
    n.cluster = n.splits = 1;
    if (!n.one_stream) choose_splits(sms, units * n.row_tiles * bv.batch, key_tiles, n.two_tiles, room, n.cluster, n.splits);
    return n;
}

size_t room_for(const ModelView &mv, const BatchView &bv, size_t partial_rows) {
    const size_t rows = (size_t)mv.L * mv.Hq * bv.total_q;
    return partial_rows / (rows > 0 ? rows : 1);
}

}  // namespace

bool attend_tc_supported(const Ctx &ctx) { return ctx.cfg.dtype == FINCH_BF16 && ctx.model.d <= 128; }

void attend_tc_plan(const Ctx &ctx, const BatchView &bv, size_t partial_rows, int &path, int &cluster, int &clusters) {
    const Plan n = make_plan(ctx, bv, room_for(ctx.model, bv, partial_rows));
    path = n.one_stream ? FINCH_ATTEND_ONE_STREAM : (n.two_tiles ? FINCH_ATTEND_ROW_PAIRS : FINCH_ATTEND_KEY_PAIRS);
    cluster = n.cluster;
    clusters = n.splits / n.cluster;
}

cudaError_t launch_attend_tc(const Ctx &ctx, const TensorView &q, const TensorView &ck, const TensorView &cv, const TensorView &hk,
                             const TensorView &hv, const BatchView &bv, int causal, AttendOut out, size_t partial_rows, cudaStream_t stream) {
    if (bv.batch == 0 || bv.max_q == 0) return cudaSuccess;
    const ModelView &mv = ctx.model;
    const Plan n = make_plan(ctx, bv, room_for(mv, bv, partial_rows));
    TcArgs p = {mv, bv, out, ctx.d_status, causal, n.heads, n.tok, n.chunks, n.row_tiles, n.two_tiles, n.cluster, mv.scale * kLog2e};
    p.out.splits = n.splits;
    Maps maps;
    if (!make_q_map(&maps.q, q, mv.d, bv.total_q, mv.Hq, mv.L, p.tok, p.heads)) return cudaErrorNotSupported;
    // an absent tensor holds no tile; its map is never used
    const bool cache = bv.total_cache > 0 && ck.ptr && cv.ptr, chunk = bv.total_chunk > 0 && hk.ptr && hv.ptr;
    if (cache && (!make_map(&maps.ck, ck, mv.d, bv.total_cache, mv.Hkv, mv.L, kTileRows) ||
                  !make_map(&maps.cv, cv, mv.d, bv.total_cache, mv.Hkv, mv.L, kTileRows)))
        return cudaErrorNotSupported;
    if (chunk && (!make_map(&maps.hk, hk, mv.d, bv.total_chunk, mv.Hkv, mv.L, kTileRows) ||
                  !make_map(&maps.hv, hv, mv.d, bv.total_chunk, mv.Hkv, mv.L, kTileRows)))
        return cudaErrorNotSupported;
    if (!cache) maps.ck = maps.cv = maps.q;
    if (!chunk) maps.hk = maps.hv = maps.q;
    const int64_t ctas = (int64_t)mv.L * mv.Hkv * n.chunks * n.splits * n.row_tiles;
    if (ctas > INT_MAX) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)ctas, bv.batch);
    cudaError_t e;
    if (n.one_stream)
        e = mv.d <= 64 ? launch<64, 1>(ctx, maps, p, grid, stream) : launch<128, 1>(ctx, maps, p, grid, stream);
    else
        e = mv.d <= 64 ? launch<64, 2>(ctx, maps, p, grid, stream) : launch<128, 2>(ctx, maps, p, grid, stream);
    p.out.splits /= p.cluster;
    if (e == cudaSuccess && p.out.splits > 1) e = launch_merge_splits(ctx, bv, p.out, stream);
    return e;
}

}  // namespace finch
