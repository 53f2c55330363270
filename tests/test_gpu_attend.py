"""finch_attend and finch_rotate against plain implementations in 64 bits, at the sizes and masks where their tilings change."""
import math

import pytest

from paper_2408_00167_b200 import binding as fb
from paper_2408_00167_b200 import build as fbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    fbuild.build()
    fb.load()


GUARD = 300     # rows in front of and behind the packed rows of an output, which nothing may touch


class Attend:
    """One call: inputs, guarded outputs, context.  Everything that no request owns is NaN."""

    def __init__(self, L, Hq, Hkv, d, reqs, dtype="bf16", causal=True, limits=None, self_lse=False, token_major=False, slack=0, scale=0.0,
                 seed=0, spread=1.0):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.L, self.Hq, self.Hkv, self.d, self.reqs, self.causal = L, Hq, Hkv, d, reqs, causal
        off = lambda ns: [sum(ns[:i]) for i in range(len(ns) + 1)]
        self.q_off, self.chunk_off = off([r[0] for r in reqs]), off([r[2] for r in reqs])
        self.cache_off = off([r[1] + slack for r in reqs])

        def tensor(heads, rows, guard=0):
            shape = (L, rows + 2 * guard, heads, d) if token_major else (L, heads, rows + 2 * guard, d)
            t = torch.full(shape, math.nan, dtype=self.dtype, device="cuda")
            t = t.transpose(1, 2) if token_major else t
            return t[:, :, guard:guard + rows], t

        def fill(t, r0, n, factor=1.0):
            t[:, :, r0:r0 + n] = (factor * torch.randn((L, t.shape[1], n, d), generator=g, device="cuda")).to(self.dtype)

        self.q, _ = tensor(Hq, self.q_off[-1])
        self.ck, _ = tensor(Hkv, self.cache_off[-1])
        self.cv, _ = tensor(Hkv, self.cache_off[-1])
        self.hk, _ = tensor(Hkv, self.chunk_off[-1])
        self.hv, _ = tensor(Hkv, self.chunk_off[-1])
        for b, (n, c, m) in enumerate(reqs):
            fill(self.q, self.q_off[b], n, spread)
            for t in (self.ck, self.cv):
                fill(t, self.cache_off[b], c)
            for t in (self.hk, self.hv):
                fill(t, self.chunk_off[b], m)
        self.out, self.out_all = tensor(Hq, self.q_off[-1], GUARD)
        self.lse_all = torch.full((L, Hq, self.q_off[-1]), math.nan, device="cuda")
        self.self_lse = torch.randn((L, Hq, self.q_off[-1]), generator=g, device="cuda") * 2 + 3 if self_lse else None
        self.limit = None
        if limits is not None:
            self.limit = torch.tensor(limits, dtype=torch.int32, device="cuda")
        B = len(reqs)
        self.ctx = fb.finch_ctx_create(L, Hq, Hkv, d, fb.FINCH_BF16 if dtype == "bf16" else fb.FINCH_F32, scale=scale, max_batch=B,
                                       max_prompt=max(r[0] for r in reqs), max_candidates=max(max(r[1] for r in reqs) + max(r[2] for r in reqs), 1))
        self.scale = scale or 1 / math.sqrt(d)
        self.batch = fb.make_batch(self.q_off, self.chunk_off, self.cache_off, [r[1] for r in reqs], [r[1] for r in reqs],
                                   prompt_self_lse=self.self_lse, row_limit=self.limit)
        self.ws = torch.full((fb.finch_attend_workspace_bytes(self.ctx, self.batch),), 255, dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        fb.finch_attend(self.ctx, self.q, self.ck, self.cv, self.hk, self.hv, self.batch, self.out, self.lse_all, causal=self.causal,
                        ws=self.ws, stream=stream)

    def status(self):
        return fb.finch_device_status(self.ctx)

    def limits_of(self, b):
        n, c, m = self.reqs[b]
        if self.limit is not None:
            return [max(0, min(c + m, int(x))) for x in self.limit[self.q_off[b]:self.q_off[b + 1]]]
        return [max(0, c + m - n + i + 1) if self.causal else c + m for i in range(n)]

    def check(self, tensor_cores):
        import torch
        from attend_reference import attend_rows, check_rows
        assert self.status() == 0
        half = 2.0 ** -8 if tensor_cores else 0.0
        for b, (n, c, m) in enumerate(self.reqs):
            q0, c0, m0 = self.q_off[b], self.cache_off[b], self.chunk_off[b]
            for l in range(self.L):
                for h in range(self.Hq):
                    kv = h // (self.Hq // self.Hkv)
                    k = torch.cat([self.ck[l, kv, c0:c0 + c], self.hk[l, kv, m0:m0 + m]])
                    v = torch.cat([self.cv[l, kv, c0:c0 + c], self.hv[l, kv, m0:m0 + m]])
                    extra = None if self.self_lse is None else self.self_lse[l, h, q0:q0 + n]
                    want = attend_rows(self.q[l, h, q0:q0 + n], k, v, self.limits_of(b), self.scale, extra, half)
                    check_rows(self.out[l, h, q0:q0 + n], self.lse_all[l, h, q0:q0 + n], *want, what=f"request {b} layer {l} head {h}")
        # rows in front of and behind the packed ones are as they were
        for rows in (self.out_all[:, :, :GUARD], self.out_all[:, :, GUARD + self.q_off[-1]:]):
            assert torch.isnan(rows).all()

    def close(self):
        fb.finch_ctx_destroy(self.ctx)


def _check(*args, tensor_cores=True, **kw):
    a = Attend(*args, **kw)
    try:
        a.run()
        a.check(tensor_cores)
    finally:
        a.close()


@pytest.mark.parametrize("Hq,Hkv,d,reqs", [
    (2, 2, 128, [(1, 0, 1)]),                              # one token that sees itself
    (2, 1, 64, [(3, 0, 3)]),
    (2, 2, 128, [(128, 0, 128)]),                          # one whole tile, two streams over one key tile
    (2, 2, 128, [(129, 0, 129)]),                          # a second row tile of one row
    (1, 1, 128, [(300, 130, 300)]),                        # three row tiles, the seam inside a tile's width
    (4, 1, 128, [(65, 257, 65)]),                          # four heads to a tile of 32 tokens
    (8, 2, 64, [(37, 1, 37)]),
    (3, 1, 128, [(50, 64, 50)]),                           # 42 tokens to a tile: 126 rows
    (7, 1, 96, [(20, 100, 21)]),                           # 18 tokens, half of a slab of dimensions absent
    (16, 1, 32, [(11, 200, 11)]),
    (2, 1, 128, [(1, 2000, 1)]),                           # one token over many keys: key splits
    (2, 1, 128, [(5, 1111, 700)]),
    (2, 2, 64, [(200, 700, 200), (1, 5, 1), (64, 0, 64), (130, 129, 131)]),
    (4, 2, 128, [(33, 0, 33), (2, 127, 2), (260, 128, 260)]),
])
def test_causal_rows_at_the_tile_edges(Hq, Hkv, d, reqs):
    _check(1, Hq, Hkv, d, reqs, slack=70)


@pytest.mark.parametrize("reqs", [[(16, 500, 77)], [(128, 896, 128), (3, 1, 1)], [(257, 64, 30)]])
def test_rows_that_see_every_candidate(reqs):
    _check(2, 4, 2, 128, reqs, causal=False, slack=33)


def test_more_query_heads_than_a_tile_has_rows():
    _check(1, 130, 1, 32, [(2, 40, 3)])


def test_rows_beyond_the_keys_are_empty():
    """More rows than candidates: the first ones see nothing."""
    _check(1, 2, 1, 128, [(40, 3, 9), (5, 0, 1)])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_row_limits_in_any_order(dtype, d):
    n, c, m = 180, 200, 150
    limits = [(i * 37) % (c + m + 1) for i in range(n)]
    limits[:5] = [0, 1, c + m, c + m + 9, -4]
    limits[100:140] = [0] * 40
    _check(1, 2, 1, d, [(n, c, m)], dtype=dtype, limits=limits, tensor_cores=dtype == "bf16")


def test_a_tile_whose_rows_all_see_nothing():
    _check(1, 1, 1, 128, [(300, 100, 60)], limits=[0] * 256 + [160] * 44)


@pytest.mark.parametrize("reqs", [[(60, 100, 60)], [(3, 3000, 3)]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_extra_term_of_the_denominator(reqs, dtype):
    _check(1, 2, 1, 64, reqs, dtype=dtype, self_lse=True, tensor_cores=dtype == "bf16")


def test_an_empty_row_with_an_extra_term():
    _check(1, 2, 1, 64, [(9, 0, 4)], self_lse=True)


@pytest.mark.parametrize("dtype,Hq,Hkv,d,reqs", [
    ("f32", 2, 2, 64, [(1, 0, 1)]),
    ("f32", 2, 1, 64, [(65, 63, 65), (1, 64, 1)]),
    ("f32", 3, 1, 96, [(30, 65, 30)]),
    ("f32", 4, 2, 128, [(17, 900, 17)]),
    ("f32", 2, 1, 32, [(70, 10, 70)]),
    ("f32", 2, 1, 256, [(33, 70, 33)]),
    ("bf16", 2, 1, 160, [(33, 70, 33)]),
    ("bf16", 66, 1, 192, [(3, 130, 3)]),
    ("bf16", 2, 2, 256, [(20, 1000, 20)]),
])
def test_fp32_multiply_adds(dtype, Hq, Hkv, d, reqs):
    _check(1, Hq, Hkv, d, reqs, dtype=dtype, slack=5, tensor_cores=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_side_by_side_in_a_token(dtype):
    _check(2, 4, 2, 64, [(100, 50, 100), (7, 0, 7)], dtype=dtype, token_major=True, tensor_cores=dtype == "bf16")


@pytest.mark.parametrize("spread", [8.0, 60.0])
def test_logits_of_many_binary_orders(spread):
    """A row's maximum grows from tile to tile by more than the kernel lets pass without scaling its output."""
    _check(1, 2, 1, 128, [(40, 1500, 40)], spread=spread)


def test_many_layers_and_units():
    _check(3, 8, 4, 64, [(17, 150, 17)], slack=9)


def test_sequences_packed_behind_one_another_keep_apart():
    """What a request's rows see holds no other request's keys, whatever its neighbours' lengths are."""
    reqs = [(n, c, n) for n, c in ((1, 0), (2, 3), (31, 0), (32, 96), (33, 1), (127, 130), (5, 0), (128, 128))]
    _check(1, 4, 2, 64, reqs)


@pytest.mark.parametrize("reqs", [[(300, 200, 300)], [(2, 1500, 2)]])
def test_the_same_result_on_another_stream_in_a_graph_and_again(reqs):
    import torch
    a = Attend(1, 4, 2, 128, reqs)
    try:
        a.run()
        torch.cuda.synchronize()
        want, want_lse = a.out.clone(), a.lse_all.clone()
        side = torch.cuda.Stream()
        a.out.fill_(math.nan)
        torch.cuda.synchronize()
        a.run(stream=side)
        torch.cuda.synchronize()
        assert torch.equal(a.out, want) and torch.equal(a.lse_all, want_lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.run()
            a.run()
        for _ in range(3):
            a.out.fill_(math.nan)
            a.ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(a.out, want) and torch.equal(a.lse_all, want_lse)
        assert a.status() == 0
    finally:
        a.close()


def test_bad_metadata_is_reported_and_writes_nothing():
    import torch
    a = Attend(1, 2, 1, 64, [(20, 30, 20), (40, 10, 40)])
    try:
        a.batch.cache_len[1] = 31       # above the bound that the host gave
        a.run()
        assert a.status() == fb.FINCH_DEV_BAD_BATCH
        assert torch.isfinite(a.out[:, :, :20].float()).all() and torch.isnan(a.out[:, :, 20:].float()).all()
    finally:
        a.close()


def test_the_prompts_own_pass_gives_the_scores_their_extra_term():
    """row_lse of the prompt over its own keys, as prompt_self_lse of finch_score: the row's denominators then add up to those of
    one attention over candidates and prompt."""
    import torch
    L, Hq, Hkv, d, n, c, m = 1, 4, 2, 64, 24, 100, 60
    own = Attend(L, Hq, Hkv, d, [(n, 0, n)], seed=1)
    both = Attend(L, Hq, Hkv, d, [(n, c + m, n)], seed=2)
    try:
        for h in range(Hkv):
            both.hk[:, h], both.hv[:, h] = own.hk[:, h], own.hv[:, h]
        both.q.copy_(own.q)
        own.run()
        both.run()
        scores = torch.zeros((L, Hkv, c + m), device="cuda")
        lse = torch.zeros((L, Hq, n), device="cuda")
        ctx = fb.finch_ctx_create(L, Hq, Hkv, d, fb.FINCH_BF16, max_batch=1, max_prompt=n, max_candidates=c + m)
        batch = fb.make_batch([0, n], [0, m], [0, c], [c], [c], prompt_self_lse=own.lse_all)
        ws = torch.empty(fb.finch_workspace_bytes(ctx, batch), dtype=torch.uint8, device="cuda")
        fb.finch_score(ctx, own.q, both.ck[:, :, :c].contiguous(), both.ck[:, :, c:c + m].contiguous(), batch, scores, lse, ws)
        # two log-sum-exps of up to 184 fp32 logits below 2^5: sums and logits are each off by under 2^-15
        torch.testing.assert_close(lse, both.lse_all, rtol=0, atol=2 ** -14)
        fb.finch_ctx_destroy(ctx)
    finally:
        own.close()
        both.close()


# ---------------------------------------------------------------------------------------------- norms and positions

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,Hq,Hkv,d,tokens,rotary,pairing,norm", [
    (1, 2, 1, 128, 1, 128, 0, True),
    (1, 32, 8, 128, 1, 128, 1, False),
    (2, 3, 1, 64, 37, 32, 0, True),
    (1, 4, 2, 96, 9, 96, 0, True),
    (1, 4, 2, 96, 9, 16, 1, True),
    (1, 2, 2, 32, 300, 32, 1, False),
    (3, 2, 1, 256, 5, 192, 0, True),
    (1, 5, 1, 160, 17, 0, 0, True),          # norm alone
    (1, 8, 8, 128, 1300, 64, 0, True),
])
def test_rotate(dtype, L, Hq, Hkv, d, tokens, rotary, pairing, norm):
    import torch
    from attend_reference import HALF_STEP, turned
    tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(tokens)
    q, k = (torch.randn((L, tokens, h, d), generator=g, device="cuda").to(tdtype).transpose(1, 2) for h in (Hq, Hkv))
    w = [(1 + 0.2 * torch.randn((L, d), generator=g, device="cuda")).to(tdtype) if norm else None for _ in range(2)]
    pos = torch.randint(-5, 1000000, (tokens,), generator=g, device="cuda").to(torch.int32)
    freq = fb.finch_rope_frequencies(rotary, 500000.0) if rotary else []
    rope = fb.finch_rope_init(rotary, freq, pairing, magnitude=1.25) if rotary else None
    ctx = fb.finch_ctx_create(L, Hq, Hkv, d, fb.FINCH_BF16 if dtype == "bf16" else fb.FINCH_F32)
    out = [torch.full((L, h, tokens + 4, d), math.nan, dtype=tdtype, device="cuda") for h in (Hq, Hkv)]
    fb.finch_rotate(ctx, q, k, pos, *(o[:, :, 2:-2] for o in out), rope=rope, q_weight=w[0], k_weight=w[1], eps=1e-5)
    for x, o, weight in zip((q, k), out, w):
        y = x.double()
        if norm:
            y = y / (y.square().mean(-1, keepdim=True) + 1e-5).sqrt() * weight.double()[:, None, None]
        size = y.abs()
        if rotary:
            size = y.abs().clone()
            size[..., :rotary] = (y[..., :rotary].abs().amax(-1, keepdim=True)) * 2.5      # |a c| + |b s|, each at most 1.25 of the largest
            y = turned(y, pos, freq, rotary, pairing, 1.25)
        # fp32: a sum of d squares, its root, three products, two products and their sum, cosines rounded to fp32
        room = size * (d + 16) * 2.0 ** -24 + HALF_STEP[tdtype] * y.abs() * 1.001 + 1e-30
        got = o[:, :, 2:-2].double()
        assert float(((got - y).abs() / room).max()) <= 1.0
        assert torch.isnan(o[:, :, :2]).all() and torch.isnan(o[:, :, -2:]).all()
    # in place, and one tensor alone
    in_place = [q.clone(), k.clone()]
    fb.finch_rotate(ctx, *in_place, pos, *in_place, rope=rope, q_weight=w[0], k_weight=w[1], eps=1e-5)
    assert torch.equal(in_place[0], out[0][:, :, 2:-2]) and torch.equal(in_place[1], out[1][:, :, 2:-2])
    alone = torch.empty_like(k)
    if rotary or norm:
        fb.finch_rotate(ctx, None, k, pos, None, alone, rope=rope, k_weight=w[1], eps=1e-5)
        assert torch.equal(alone, out[1][:, :, 2:-2])
    assert fb.finch_device_status(ctx) == 0
    fb.finch_ctx_destroy(ctx)


def test_rotate_in_place_in_a_packed_projection():
    """q and k side by side in one buffer, as a fused projection leaves them."""
    import torch
    L, Hq, Hkv, d, T = 1, 4, 2, 64, 19
    buf = torch.randn((L, T, Hq + 2 * Hkv, d), device="cuda").to(torch.bfloat16)
    q, k = buf[:, :, :Hq].transpose(1, 2), buf[:, :, Hq:Hq + Hkv].transpose(1, 2)
    before = buf.clone()
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    rope = fb.finch_rope_init(d, fb.finch_rope_frequencies(d))
    ctx = fb.finch_ctx_create(L, Hq, Hkv, d, fb.FINCH_BF16)
    want = [torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())]
    fb.finch_rotate(ctx, q, k, pos, *want, rope=rope)
    fb.finch_rotate(ctx, q, k, pos, q, k, rope=rope)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(buf[:, :, Hq + Hkv:], before[:, :, Hq + Hkv:])
    fb.finch_ctx_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rotary,pairing", [(96, 0, 0), (96, 96, 0), (160, 64, 1), (192, 192, 0), (224, 224, 1)])
def test_a_head_that_is_not_finite_stays_alone(dtype, d, rotary, pairing):
    """A head of zeros with eps = 0, and one with a NaN, in head dimensions that leave lanes of a row unused; enough tokens that a warp
    walks a token's heads in several rounds.  Every other head is what it is without them, bit for bit."""
    import torch
    tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
    L, Hq, Hkv, tokens = 2, 24, 12, 1250
    g = torch.Generator(device="cuda").manual_seed(d)
    q, k = (torch.randn((L, h, tokens, d), generator=g, device="cuda").to(tdtype) for h in (Hq, Hkv))
    w = [(1 + 0.2 * torch.randn((L, d), generator=g, device="cuda")).to(tdtype) for _ in range(2)]
    pos = torch.randint(0, 100000, (tokens,), generator=g, device="cuda").to(torch.int32)
    rope = fb.finch_rope_init(rotary, fb.finch_rope_frequencies(rotary), pairing) if rotary else None
    ctx = fb.finch_ctx_create(L, Hq, Hkv, d, fb.FINCH_BF16 if dtype == "bf16" else fb.FINCH_F32)

    def run(q, k):
        out = [torch.full_like(x, math.nan) for x in (q, k)]
        fb.finch_rotate(ctx, q, k, pos, *out, rope=rope, q_weight=w[0], k_weight=w[1], eps=0.0)
        return out

    clean = run(q, k)
    for bad in (0.0, math.nan, math.inf):
        dirty = [q.clone(), k.clone()]
        for x in dirty:
            x[:, 1] = 0.0 if bad == 0.0 else x[:, 1]
            x[:, 1, ::3, 5] = bad
        for got, want in zip(run(*dirty), clean):
            others = [h for h in range(want.shape[1]) if h != 1]
            assert torch.isfinite(want.float()).all()
            assert torch.equal(got[:, others], want[:, others])
    fb.finch_ctx_destroy(ctx)
