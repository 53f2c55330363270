"""The paged 8-bit cache: append and attention against plain implementations in 64 bits."""
import math

import pytest

from paper_2408_00167_b200 import binding as fb
from paper_2408_00167_b200 import build as fbuild

pytestmark = pytest.mark.gpu
PAGE = fb.FINCH_PAGE_TOKENS


@pytest.fixture(scope="module", autouse=True)
def _built():
    fbuild.build()
    fb.load()


class Cache:
    """Pages in shuffled order, sentinels everywhere, and the rows that were appended (as the model has them) beside them."""

    def __init__(self, L, Hq, Hkv, d, batch, width, dtype="bf16", spare=3, slots=None, seed=0):
        import torch
        self.L, self.Hq, self.Hkv, self.d, self.B, self.width = L, Hq, Hkv, d, batch, width
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        n_pages = batch * width + spare
        self.k, self.v = (torch.full((L, n_pages, Hkv, PAGE, d), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2))  # NaN codes
        self.ks, self.vs = (torch.full((L, n_pages, Hkv), math.nan, device="cuda") for _ in range(2))
        n_open = batch if slots is None else max(slots) + 2
        self.ok, self.ov = (torch.full((L, n_open, Hkv, PAGE, d), math.nan, dtype=self.dtype, device="cuda") for _ in range(2))
        order = torch.randperm(n_pages, generator=self.g, device="cuda").to(torch.int32)
        self.table = order[:batch * width].reshape(batch, width).contiguous()
        self.slots = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
        self.pages = fb.make_pages(self.k, self.v, self.ks, self.vs, self.ok, self.ov, self.table, self.slots)
        self.lens = [0] * batch
        self.rows = [[torch.zeros((L, Hkv, 0, d), dtype=self.dtype, device="cuda") for _ in range(2)] for _ in range(batch)]
        self.ctx = fb.finch_ctx_create(L, Hq, Hkv, d, fb.FINCH_BF16 if dtype == "bf16" else fb.FINCH_F32, max_batch=batch, max_prompt=64,
                                       max_candidates=width * PAGE)

    def slot(self, b):
        return b if self.slots is None else int(self.slots[b])

    def append(self, counts, rope=None, pos=None, freq=None, factor=1.0):
        """counts[b] new rows; freq: (frequencies, rotary_dim, pairing) of `rope`, for the rows kept beside the cache."""
        import torch
        from attend_reference import turned
        off = [sum(counts[:i]) for i in range(self.B + 1)]
        new = [(factor * torch.randn((self.L, off[-1] + 2, self.Hkv, self.d), generator=self.g, device="cuda")).to(self.dtype).transpose(1, 2)[:, :, 1:-1]
               for _ in range(2)]
        batch = fb.make_paged_batch(self.lens, new_off=off)
        out_len = torch.full((self.B,), -7, dtype=torch.int32, device="cuda")
        fb.finch_pages_append(self.ctx, self.pages, batch, *new, out_len, rope=rope, pos=pos)
        for b in range(self.B):
            k, v = (x[:, :, off[b]:off[b + 1]] for x in new)
            if rope is not None:
                at = pos[off[b]:off[b + 1]] if pos is not None else self.lens[b] + torch.arange(counts[b], device="cuda")
                k = turned(k, at, *freq).float().to(self.dtype)
            self.rows[b] = [torch.cat([self.rows[b][0], k], 2), torch.cat([self.rows[b][1], v], 2)]
            self.lens[b] += counts[b]
        assert fb.finch_device_status(self.ctx) == 0
        assert out_len.tolist() == self.lens

    def check(self):
        """Pages and open rows hold what the definition says, and everything else its sentinel."""
        import torch
        from attend_reference import quantised
        k, v = torch.full_like(self.k, 0x7f), torch.full_like(self.v, 0x7f)
        ks, vs = torch.full_like(self.ks, math.nan), torch.full_like(self.vs, math.nan)
        for b in range(self.B):
            for w in range(self.lens[b] // PAGE):
                at = int(self.table[b, w])
                for pool, scales, x in ((k, ks, self.rows[b][0]), (v, vs, self.rows[b][1])):
                    pool[:, at], scales[:, at] = quantised(x[:, :, w * PAGE:(w + 1) * PAGE])
            rest = self.lens[b] % PAGE
            for open_rows, x in ((self.ok, self.rows[b][0]), (self.ov, self.rows[b][1])):
                assert torch.equal(open_rows[:, self.slot(b), :, :rest], x[:, :, self.lens[b] - rest:])
        for got, want in ((self.k, k), (self.v, v)):
            assert torch.equal(got, want)
        for got, want in ((self.ks, ks), (self.vs, vs)):
            assert torch.equal(got.nan_to_num(-1.0), want.nan_to_num(-1.0))

    def values(self, b):
        """The request's tokens as the cache holds them, fp64 [L][Hkv][len][d]."""
        import torch
        from attend_reference import dequantised
        out = []
        for pool, scales, rows in ((self.k, self.ks, self.ok), (self.v, self.vs, self.ov)):
            full, rest = self.lens[b] // PAGE, self.lens[b] % PAGE
            at = self.table[b, :full].long()
            x = dequantised(pool[:, at], scales[:, at]).transpose(1, 2).reshape(self.L, self.Hkv, full * PAGE, self.d)
            out.append(torch.cat([x, rows[:, self.slot(b), :, :rest].double()], 2))
        return out

    def attend(self, counts, spread=1.0):
        import torch
        from attend_reference import attend_rows, check_rows
        off = [sum(counts[:i]) for i in range(self.B + 1)]
        q = (spread * torch.randn((self.L, self.Hq, off[-1], self.d), generator=self.g, device="cuda")).to(self.dtype)
        out = torch.full((self.L, self.Hq, off[-1] + 8, self.d), math.nan, dtype=self.dtype, device="cuda")
        lse = torch.full((self.L, self.Hq, off[-1]), math.nan, device="cuda")
        batch = fb.make_paged_batch(self.lens, q_off=off)
        ws = torch.full((fb.finch_pages_workspace_bytes(self.ctx, batch),), 255, dtype=torch.uint8, device="cuda")
        fb.finch_pages_attend(self.ctx, self.pages, batch, q, out[:, :, 4:-4], lse, ws=ws)
        assert fb.finch_device_status(self.ctx) == 0
        assert torch.isnan(out[:, :, :4]).all() and torch.isnan(out[:, :, -4:]).all()
        for b in range(self.B):
            k, v = self.values(b)
            limits = [max(0, self.lens[b] - counts[b] + i + 1) for i in range(counts[b])]
            for l in range(self.L):
                for h in range(self.Hq):
                    rows = slice(off[b], off[b + 1])
                    kv = h // (self.Hq // self.Hkv)
                    # queries and weights enter the products with 22 bits: 2^-21 of a logit's sum of magnitudes, of a weight
                    want = list(attend_rows(q[l, h, rows], k[l, kv], v[l, kv], limits, 1 / math.sqrt(self.d), None, 2.0 ** -20))
                    if self.lens[b]:
                        big = q[l, h, rows].double().abs().amax(-1) * k[l, kv].abs().sum(-1).max() / math.sqrt(self.d) * 2.0 ** -21
                        want[3] = want[3] + big
                        want[2] = want[2] + 2 * big[:, None] * v[l, kv].abs().amax()
                    check_rows(out[l, h, 4 + off[b]:4 + off[b + 1]], lse[l, h, rows], *want, what=f"request {b} layer {l} head {h}")
        return out

    def close(self):
        fb.finch_ctx_destroy(self.ctx)


def _rope(d, rotary, pairing):
    freq = fb.finch_rope_frequencies(rotary, 10000.0)
    return fb.finch_rope_init(rotary, freq, pairing), (freq, rotary, pairing)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rotary,pairing", [(32, 32, 0), (64, 64, 1), (96, 32, 0), (128, 128, 0), (160, 160, 1), (256, 256, 0)])
def test_append_one_by_one_and_in_blocks(dtype, d, rotary, pairing):
    """Requests of different lengths, appends that fill a page exactly, end inside one, cross several, or add nothing."""
    c = Cache(2, 2, 2, d, 3, 5, dtype)
    rope, freq = _rope(d, rotary, pairing)
    try:
        for counts in ([1, 63, 64], [62, 1, 65], [1, 1, 0], [70, 129, 1], [0, 0, 62], [1, 1, 1]):
            c.append(counts, rope=rope, freq=freq)
            c.check()
    finally:
        c.close()


def test_append_without_rotation_in_slots_of_its_own():
    c = Cache(1, 4, 2, 128, 3, 4, slots=[4, 0, 2])
    try:
        c.append([100, 3, 64])
        c.append([28, 61, 1])
        c.check()
    finally:
        c.close()


def test_append_at_given_positions():
    import torch
    c = Cache(1, 4, 2, 64, 2, 3)
    rope, freq = _rope(64, 64, 0)
    try:
        pos = torch.tensor([900000 - 7 * i for i in range(90)], dtype=torch.int32, device="cuda")
        c.append([80, 10], rope=rope, freq=freq, pos=pos)
        c.check()
    finally:
        c.close()


def test_a_page_is_the_same_however_its_tokens_arrived():
    import torch
    whole, parts = Cache(1, 2, 1, 64, 1, 3), Cache(1, 2, 1, 64, 1, 3)
    rope, freq = _rope(64, 64, 0)
    try:
        k, v = (torch.randn((1, 1, 150, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
        for c, cuts in ((whole, [150]), (parts, [1, 62, 1, 64, 5, 17])):
            have = 0
            for n in cuts:
                batch = fb.make_paged_batch([have], new_off=[0, n])
                fb.finch_pages_append(c.ctx, c.pages, batch, k[:, :, have:have + n], v[:, :, have:have + n], rope=rope)
                have += n
            assert fb.finch_device_status(c.ctx) == 0
        for a, b in ((whole.k, parts.k), (whole.v, parts.v), (whole.ks.nan_to_num(), parts.ks.nan_to_num()), (whole.vs.nan_to_num(), parts.vs.nan_to_num()),
                     (whole.ok[:, :, :, :22], parts.ok[:, :, :, :22]), (whole.ov[:, :, :, :22], parts.ov[:, :, :, :22])):
            assert torch.equal(a, b)
    finally:
        whole.close()
        parts.close()


def test_values_at_the_ends_of_the_range():
    """Zeros, tiny and huge rows, infinities and NaN: a scale of zero for a page of zeros, what is not finite does not count for it."""
    import torch
    c = Cache(1, 1, 1, 32, 1, 5, dtype="f32")
    try:
        x = torch.randn((1, 1, 5 * PAGE, 32), generator=c.g, device="cuda")
        x[:, :, :PAGE] = 0
        x[:, :, PAGE:2 * PAGE] *= 1e-30
        x[:, :, 2 * PAGE:3 * PAGE] *= 1e30
        x[:, :, 3 * PAGE:4 * PAGE:7, 3] = math.inf
        x[:, :, 3 * PAGE + 1:4 * PAGE:7, 4] = -math.inf
        x[:, :, 4 * PAGE + 2, 5] = math.nan
        batch = fb.make_paged_batch([0], new_off=[0, 5 * PAGE])
        fb.finch_pages_append(c.ctx, c.pages, batch, x, x)
        from attend_reference import quantised
        for w in range(5):
            codes, scale = quantised(x[:, :, w * PAGE:(w + 1) * PAGE])
            at = int(c.table[0, w])
            got = c.k[:, at].view(torch.float8_e4m3fn).float()
            assert torch.equal(got.nan_to_num(999.0), codes.view(torch.float8_e4m3fn).float().nan_to_num(999.0))
            assert torch.equal(c.ks[:, at], scale) and torch.equal(c.v[:, at], c.k[:, at])
        assert float(c.ks[0, int(c.table[0, 0]), 0]) == 0.0
    finally:
        c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,lens,rows", [
    (2, 2, 128, [1, 0, 63, 64, 65], 1),              # nothing but open rows, an exact page, one row behind it
    (4, 1, 64, [640, 17, 129, 300, 256], 1),
    (8, 1, 128, [1500, 64, 128, 1, 700], 1),         # as many rows as a group holds
    (12, 1, 96, [333, 100, 64, 65, 0], 1),           # a second, partial group
    (3, 3, 32, [200, 5, 64, 128, 190], 2),           # two tokens: the last page is not whole for the first of them
    (4, 1, 128, [70, 64, 3, 130, 1000], 5),          # 20 rows, limits of their own
    (2, 1, 160, [100, 64, 1, 200, 130], 1),
    (2, 1, 192, [100, 64, 1, 200, 130], 1),
    (2, 1, 224, [100, 64, 1, 200, 130], 3),
    (8, 1, 256, [500, 64, 1, 63, 130], 1),
])
def test_attention_over_pages(dtype, Hq, Hkv, d, lens, rows):
    c = Cache(1, Hq, Hkv, d, len(lens), (max(lens) + PAGE - 1) // PAGE, dtype)
    try:
        c.append(lens)
        c.attend([rows] * len(lens))
        c.attend([i % (rows + 1) for i in range(len(lens))])      # also requests without a query
    finally:
        c.close()


@pytest.mark.parametrize("length", [5000, 20001])
def test_long_caches_are_split(length):
    c = Cache(1, 8, 2, 128, 1, (length + PAGE - 1) // PAGE)
    try:
        c.append([length])
        c.attend([1])
        c.attend([3], spread=20.0)
    finally:
        c.close()


def test_scales_of_pages_far_apart():
    """Pages whose scales differ by many orders, and a page of zeros."""
    c = Cache(1, 4, 1, 64, 1, 8)
    try:
        for factor in (1.0, 1e-6, 0.0, 30.0, 1e3, 1e-3):
            c.append([PAGE], factor=factor)
        c.append([9])
        c.check()
        c.attend([1])
    finally:
        c.close()


def test_layers_and_generation():
    """Append one token, attend, again and again over two pages' ends, three layers."""
    c = Cache(3, 4, 2, 64, 2, 4)
    rope, freq = _rope(64, 64, 0)
    try:
        c.append([60, 125], rope=rope, freq=freq)
        for _ in range(6):
            c.append([1, 1], rope=rope, freq=freq)
            c.attend([1, 1])
        c.check()
    finally:
        c.close()


def test_bad_page_numbers_are_reported_and_counted_as_absent():
    import torch
    from attend_reference import attend_rows, check_rows
    c = Cache(1, 2, 1, 64, 1, 4)
    try:
        c.append([200])
        before = c.k.clone()
        number = int(c.table[0, 1])
        for bad in (-1, c.k.shape[1], 2 ** 31 - 1):
            c.table[0, 1] = bad
            q = torch.randn((1, 2, 1, 64), device="cuda").to(torch.bfloat16)
            out, lse = torch.zeros_like(q), torch.zeros((1, 2, 1), device="cuda")
            batch = fb.make_paged_batch([200], q_off=[0, 1])
            ws = torch.empty(fb.finch_pages_workspace_bytes(c.ctx, batch), dtype=torch.uint8, device="cuda")
            fb.finch_pages_attend(c.ctx, c.pages, batch, q, out, lse, ws=ws)
            assert fb.finch_device_status(c.ctx) == fb.FINCH_DEV_BAD_INDEX
            c.table[0, 1] = number
            k, v = c.values(0)
            there = [i for i in range(200) if i // PAGE != 1]
            for h in range(2):
                want = attend_rows(q[0, h], k[0, 0, there], v[0, 0, there], [len(there)], 1 / 8, None, 2.0 ** -19)
                check_rows(out[0, h], None, *want)
            c.table[0, 1] = bad
            new = torch.randn((1, 1, 100, 64), device="cuda").to(torch.bfloat16)
            fb.finch_pages_append(c.ctx, c.pages, fb.make_paged_batch([40], new_off=[0, 100]), new, new)
            assert fb.finch_device_status(c.ctx) == fb.FINCH_DEV_BAD_INDEX
            c.table[0, 1] = number
            assert torch.equal(c.k[0, number], before[0, number])
            c.k.copy_(before)
            c.close()
            c = Cache(1, 2, 1, 64, 1, 4)
            c.append([200])
            before = c.k.clone()
            number = int(c.table[0, 1])
    finally:
        c.close()


def test_bad_lengths_and_slots_are_reported_and_write_nothing():
    import torch
    c = Cache(1, 2, 1, 64, 2, 3, slots=[0, 1])
    try:
        c.append([70, 70])
        q = torch.randn((1, 2, 2, 64), device="cuda").to(torch.bfloat16)
        for what, value in (("len", 71), ("len", -1), ("slot", 99), ("slot", -1)):
            batch = fb.make_paged_batch([70, 70], q_off=[0, 1, 2])
            if what == "len":
                batch.len[1] = value
            else:
                c.slots[1] = value
            out = torch.full_like(q, math.nan)
            ws = torch.empty(fb.finch_pages_workspace_bytes(c.ctx, batch), dtype=torch.uint8, device="cuda")
            fb.finch_pages_attend(c.ctx, c.pages, batch, q, out, ws=ws)
            assert fb.finch_device_status(c.ctx) == fb.FINCH_DEV_BAD_BATCH
            assert torch.isfinite(out[:, :, 0].float()).all() and torch.isnan(out[:, :, 1].float()).all()
            before = [t.clone() for t in (c.k, c.v, c.ok, c.ov)]
            add = fb.make_paged_batch([70, 70], new_off=[0, 0, 3])
            if what == "len":
                add.len[1] = value
            new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
            fb.finch_pages_append(c.ctx, c.pages, add, q[:, :1, :1].expand(1, 1, 3, 64).contiguous(), q[:, :1, :1].expand(1, 1, 3, 64).contiguous(), new_len)
            assert fb.finch_device_status(c.ctx) == fb.FINCH_DEV_BAD_BATCH
            assert new_len.tolist() == [70, value if what == "len" else 70]
            assert all(torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b)
                       for a, b in zip(before, (c.k, c.v, c.ok, c.ov)))
            c.slots[1] = 1
    finally:
        c.close()


def test_the_same_result_in_a_graph_with_lengths_that_grow_on_the_device():
    """One captured step, append then attention, replayed: the lengths that the append writes are the next replay's."""
    import torch
    c = Cache(1, 4, 2, 128, 2, 4)
    try:
        c.append([62, 130])
        lens = [torch.tensor(c.lens, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")]
        k, v, q = (torch.randn((1, h, 2, 128), device="cuda").to(torch.bfloat16) for h in (2, 2, 4))
        out = torch.zeros_like(q)
        add = fb.make_paged_batch(c.lens, new_off=[0, 1, 2], len_tensor=lens[0], max_len=4 * PAGE - 2)
        see = fb.make_paged_batch(c.lens, q_off=[0, 1, 2], len_tensor=lens[1], max_len=4 * PAGE - 1)
        ws = torch.empty(fb.finch_pages_workspace_bytes(c.ctx, see), dtype=torch.uint8, device="cuda")

        def step():
            fb.finch_pages_append(c.ctx, c.pages, add, k, v, lens[1])
            fb.finch_pages_attend(c.ctx, c.pages, see, q, out, ws=ws)
            lens[0].copy_(lens[1])

        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        torch.cuda.synchronize()
        for _ in range(4):
            for t in (k, v, q):
                t.normal_(generator=c.g)
            graph.replay()
            torch.cuda.synchronize()
            for b in range(2):
                c.rows[b] = [torch.cat([c.rows[b][0], k[:, :, b:b + 1]], 2), torch.cat([c.rows[b][1], v[:, :, b:b + 1]], 2)]
                c.lens[b] += 1
            c.check()
            got = out.clone()
            again = torch.zeros_like(out)
            fb.finch_pages_attend(c.ctx, c.pages, fb.make_paged_batch(c.lens, q_off=[0, 1, 2], max_len=4 * PAGE - 1), q, again, ws=ws)
            assert torch.equal(got, again)
        assert lens[0].tolist() == c.lens and fb.finch_device_status(c.ctx) == 0
    finally:
        c.close()


def _filled(k, v, dtype, Hq=1):
    """A cache of one request and layer that holds rows k and v, [Hkv][len][d]."""
    import torch
    Hkv, n, d = k.shape
    c = Cache(1, Hq, Hkv, d, 1, (n + PAGE - 1) // PAGE, dtype)
    rows = [x[None].to(c.dtype).contiguous() for x in (k, v)]
    fb.finch_pages_append(c.ctx, c.pages, fb.make_paged_batch([0], new_off=[0, n]), *rows)
    c.lens = [n]
    return c


def _attend_rows(c, q, see=None):
    """Rows q [Hq][n][d] over the cache of `_filled`: every weight counts by its own size, every logit by its own sum of magnitudes.
    see: the rows that are checked (all)."""
    import torch
    from attend_reference import attend_rows, check_rows
    n = q.shape[1]
    q = q[None].to(c.dtype).contiguous()
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:3], math.nan, device="cuda")
    batch = fb.make_paged_batch(c.lens, q_off=[0, n])
    ws = torch.empty(fb.finch_pages_workspace_bytes(c.ctx, batch), dtype=torch.uint8, device="cuda")
    fb.finch_pages_attend(c.ctx, c.pages, batch, q, out, lse, ws=ws)
    assert fb.finch_device_status(c.ctx) == 0
    k, v = c.values(0)
    see = range(n) if see is None else see
    for h in range(c.Hq):
        kv = h // (c.Hq // c.Hkv)
        for i in see:
            # a weight enters with 22 bits: 2^-21 of itself at most (2^-20 leaves room for its exponential), where that is above half a
            # step of the smallest f16 numbers, 2^-25, under a lift of 2^15: 2^-40 of the largest weight, itself at most 1
            want = list(attend_rows(q[0, h, i:i + 1], k[0, kv], v[0, kv], [c.lens[0] - n + i + 1], 1 / math.sqrt(c.d), None, 2.0 ** -20))
            want[2] = want[2] + 2.0 ** -40 * v[0, kv, :c.lens[0] - n + i + 1].abs().sum(0)
            check_rows(out[0, h, i:i + 1], lse[0, h, i:i + 1], *want, what=f"head {h} row {i}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 64, 150, 4000])
def test_many_small_weights_add_up(dtype, n):
    """One key in 64 takes nearly all the weight and has values of zero: what is left are weights of 2^-26 and below."""
    import torch
    k, v = torch.zeros((1, n, 64), device="cuda"), torch.ones((1, n, 64), device="cuda")
    k[:, 5::64, 0], v[:, 5::64] = 16.0, 0.0
    q = torch.zeros((1, 1, 64), device="cuda")
    for size in (9.0, 10.0, 11.0):       # weights of 2^-26, 2^-29 and 2^-32
        c = _filled(k, v, dtype)
        try:
            q[..., 0] = size
            _attend_rows(c, q)
        finally:
            c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 100])
def test_a_row_does_not_feel_the_size_of_keys_behind_it(dtype, n):
    """Open rows that the first query rows do not see: very large, or with keys that are not numbers."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((1, n, 64), generator=g, device="cuda") for _ in range(2))
    q = torch.randn((1, 5, 64), generator=g, device="cuda")
    k[:, -2], v[:, -2:] = 1e25, -1e25
    for last in (1e30, math.inf, math.nan):
        k[:, -1] = last
        c = _filled(k, v, dtype)
        try:
            _attend_rows(c, q, see=range(3))
        finally:
            c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 64, 150])
def test_rows_with_a_few_large_elements(dtype, n):
    """A query element thousands of times the others where keys are zero, and an open key and value likewise."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((2, n, 96), generator=g, device="cuda") for _ in range(2))
    q = torch.randn((4, 2, 96), generator=g, device="cuda")
    k[..., 7], q[..., 7] = 0.0, 20000.0
    if n % PAGE:
        k[:, -1, 11], q[..., 11] = 30000.0, 0.0
        v[:, -3, 13] = 20000.0
    c = _filled(k, v, dtype, Hq=4)
    try:
        _attend_rows(c, q)
    finally:
        c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,length,bad_pages,rows", [(64, 200, [1], 1), (96, 200, [0, 2], 3), (128, 64, [0], 1), (256, 700, [3, 9], 2), (128, 5000, [0, 7, 70], 4)])
def test_a_refused_page_is_not_there_whatever_page_0_holds(dtype, d, length, bad_pages, rows):
    """Page 0 is nobody's and holds NaN codes and scales; a unit with refused pages has the result of the pages that are left."""
    import torch
    from attend_reference import attend_rows, check_rows
    c = Cache(1, 4, 1, d, 1, (length + PAGE - 1) // PAGE, dtype)
    try:
        spare = next(n for n in range(1, c.k.shape[1]) if n not in set(c.table.flatten().tolist()))
        c.table[c.table == 0] = spare
        c.append([length])
        k, v = c.values(0)
        for i, w in enumerate(bad_pages):
            c.table[0, w] = (-1, c.k.shape[1], 2 ** 31 - 1)[i % 3]
        q = torch.randn((1, 4, rows, d), generator=c.g, device="cuda").to(c.dtype)
        out, lse = torch.full_like(q, math.nan), torch.full((1, 4, rows), math.nan, device="cuda")
        batch = fb.make_paged_batch([length], q_off=[0, rows])
        ws = torch.empty(fb.finch_pages_workspace_bytes(c.ctx, batch), dtype=torch.uint8, device="cuda")
        fb.finch_pages_attend(c.ctx, c.pages, batch, q, out, lse, ws=ws)
        assert fb.finch_device_status(c.ctx) == fb.FINCH_DEV_BAD_INDEX
        for h in range(4):
            for i in range(rows):
                there = [j for j in range(length - rows + i + 1) if j // PAGE not in bad_pages]
                # as in Cache.attend: queries and weights enter the products with 22 bits
                want = list(attend_rows(q[0, h, i:i + 1], k[0, 0, there], v[0, 0, there], [len(there)], 1 / math.sqrt(d), None, 2.0 ** -20))
                if there:
                    big = q[0, h, i:i + 1].double().abs().amax(-1) * k[0, 0].abs().sum(-1).max() / math.sqrt(d) * 2.0 ** -21
                    want[3], want[2] = want[3] + big, want[2] + 2 * big[:, None] * v[0, 0].abs().amax()
                check_rows(out[0, h, i:i + 1], lse[0, h, i:i + 1], *want, what=f"head {h} row {i}")
    finally:
        c.close()
