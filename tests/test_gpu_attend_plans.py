"""finch_attend and finch_pages_attend on every plan that their hosts make of a batch: pairs of row tiles, clusters, clusters whose results
a second launch adds, one-stream CTAs over many tiles, tensors that no tensor map describes, and batches above a warp's first search."""
import math

import pytest

from paper_2408_00167_b200 import binding as fb
from paper_2408_00167_b200 import build as fbuild
from test_gpu_attend import GUARD, Attend
from test_gpu_pages import Cache

pytestmark = pytest.mark.gpu
ONE, ROWS, KEYS = fb.FINCH_ATTEND_ONE_STREAM, fb.FINCH_ATTEND_ROW_PAIRS, fb.FINCH_ATTEND_KEY_PAIRS


@pytest.fixture(scope="module", autouse=True)
def _built():
    fbuild.build()
    fb.load()


def _some_rows(n, tok):
    """All of few rows; of many, those around the borders of row tiles of `tok` tokens, and one in 37."""
    if n <= 48:
        return list(range(n))
    near = {r + e for r in range(0, n + tok, tok) for e in (-2, -1, 0, 1)} | set(range(0, n, 37)) | {n - 1}
    return sorted(r for r in near if 0 <= r < n)


def _check(a, heads, plan=None, tensor_cores=True):
    """As Attend.check, for some heads and the rows of _some_rows; all other rows have to be finite."""
    import torch
    from attend_reference import attend_rows, check_rows
    try:
        if plan is not None:
            assert fb.finch_attend_plan(a.ctx, a.batch) == plan
        a.run()
        assert a.status() == 0
        g = a.Hq // a.Hkv
        tok = 128 // g
        for b, (n, c, m) in enumerate(a.reqs):
            q0, c0, m0 = a.q_off[b], a.cache_off[b], a.chunk_off[b]
            rows = _some_rows(n, tok)
            if not rows:
                continue
            at = torch.tensor(rows, device="cuda") + q0
            limits = [a.limits_of(b)[r] for r in rows]
            assert torch.isfinite(a.out[:, :, q0:q0 + n].float()).all()
            for l in range(a.L):
                for h in heads:
                    k = torch.cat([a.ck[l, h // g, c0:c0 + c], a.hk[l, h // g, m0:m0 + m]])
                    v = torch.cat([a.cv[l, h // g, c0:c0 + c], a.hv[l, h // g, m0:m0 + m]])
                    extra = None if a.self_lse is None else a.self_lse[l, h, at]
                    want = attend_rows(a.q[l, h, at], k, v, limits, a.scale, extra, 2.0 ** -8 if tensor_cores else 0.0)
                    check_rows(a.out[l, h, at], a.lse_all[l, h, at], *want, what=f"request {b} layer {l} head {h}")
        for rows in (a.out_all[:, :, :GUARD], a.out_all[:, :, GUARD + a.q_off[-1]:]):
            assert torch.isnan(rows).all()
    finally:
        a.close()


def _steps(n, *values):
    """Limits of n rows that change every 128 rows."""
    return [values[i // 128 % len(values)] for i in range(n)]


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("limits", [None, (800, 90), (90, 800), (0, 800, 130), (800, 0, 0)])
def test_pairs_of_row_tiles(d, limits):
    """Two row tiles against the same keys, causal or with more key tiles for the first, or for the second, or none for one."""
    n, c, m = 300, 500, 300
    a = Attend(1, 32, 32, d, [(n, c, m)], limits=limits and _steps(n, *limits), slack=40, self_lse=limits is not None)
    _check(a, [0, 31], (ROWS, 1, 1))


def test_pairs_of_row_tiles_of_grouped_heads_and_ragged_requests():
    """32 tokens of four heads to a row tile; requests of one row tile, of none, and of several."""
    a = Attend(1, 32, 8, 128, [(70, 300, 200), (32, 700, 32), (1, 0, 1), (128, 64, 128)], slack=11)
    _check(a, [0, 13, 31], (ROWS, 1, 1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("limits", [None, (1400, 90), (90, 1400), (0, 1400, 300)])
def test_pairs_of_row_tiles_in_a_cluster(d, limits):
    n, c, m = 300, 1100, 300
    a = Attend(1, 32, 32, d, [(n, c, m)], limits=limits and _steps(n, *limits), self_lse=limits is not None)
    _check(a, [0, 31], (ROWS, 2, 1))


@pytest.mark.parametrize("Hq,Hkv,reqs,plan", [
    (32, 32, [(20, 700, 20), (5, 900, 5), (1, 1, 1)], (KEYS, 1, 1)),                  # also a request of one key tile
    (32, 32, [(128, 1500, 128), (5, 300, 5)], (KEYS, 2, 1)),
    (32, 32, [(40, 4000, 40), (3, 4100, 3), (1, 0, 1), (9, 100, 9), (128, 2000, 128)], (KEYS, 1, 1)),   # more CTAs than SMs
])
def test_pairs_of_key_tiles(Hq, Hkv, reqs, plan):
    for d in (64, 128):
        _check(Attend(1, Hq, Hkv, d, reqs, slack=3), [0, 31], plan)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("reqs,limits,clusters", [
    ([(3, 8000, 3)], None, 8),
    ([(20, 7000, 300)], [0, 7300, 1, 128, 129, 3000] + [7000 - 300 * i for i in range(14)], 5),      # a row that sees nothing, rows of few splits
    ([(2, 8190, 2), (2, 100, 2), (0, 0, 0), (1, 4000, 1)], None, 6),                                  # requests with fewer key tiles than splits
])
def test_clusters_whose_results_a_second_launch_adds(d, reqs, limits, clusters):
    a = Attend(1, 4, 1, d, reqs, limits=limits, self_lse=limits is not None)
    _check(a, range(4), (KEYS, 4, clusters))


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("reqs", [[(600, 1000, 600)], [(33, 900, 33), (128, 800, 128), (1, 1000, 1), (64, 0, 64), (5, 770, 5)], [(130, 3700, 300), (129, 10, 200), (200, 64, 64)]])
def test_one_stream_over_many_key_tiles(d, reqs):
    _check(Attend(1, 32, 32, d, reqs, slack=5), [0, 31], (ONE, 1, 1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,req,plan,most", [
    (2, 1, (40, 130, 40), (ONE, 1, 1), [100, 128, 130, 131, 1, 0]),
    (32, 32, (300, 500, 300), (ROWS, 1, 1), [300, 500, 501, 690]),
    (32, 32, (300, 1100, 300), (ROWS, 2, 1), [1000, 1101]),
    (4, 1, (20, 900, 20), (KEYS, 4, 1), [70, 899, 910]),
    (4, 1, (3, 8000, 3), (KEYS, 4, 8), [7900, 64]),
    (32, 32, (600, 1000, 600), (ONE, 1, 1), [999, 1333]),
])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_candidates_that_no_row_sees_may_hold_anything(dtype, d, Hq, Hkv, req, plan, most):
    """Row limits that end in front of the last candidate: K and V behind the largest are NaN, as memory that nobody has written."""
    n, c, m = req
    for top in most:
        a = Attend(1, Hq, Hkv, d, [req], dtype=dtype, limits=[top if i % 5 == 3 else max(0, top - i % 67) for i in range(n)])
        a.ck[:, :, top:c] = a.cv[:, :, top:c] = math.nan
        a.hk[:, :, max(0, top - c):] = a.hv[:, :, max(0, top - c):] = math.nan
        _check(a, [0, Hq - 1], plan if dtype == "bf16" else None, dtype == "bf16")


def test_plans_of_few_keys():
    """Up to five key tiles a CTA has one stream; the tests of the tiles' edges take it."""
    a = Attend(1, 32, 32, 64, [(200, 300, 200)])
    _check(a, [0, 31], (ONE, 1, 1))


@pytest.mark.parametrize("d,reqs", [(128, [(70, 300, 70), (3, 1, 3)]), (64, [(5, 3000, 5)]), (96, [(33, 0, 33)])])
def test_tensors_that_no_tensor_map_describes(d, reqs):
    """A single layer with a layer stride of zero: bf16 rows in fp32 multiply-adds."""
    a = Attend(1, 4, 2, d, reqs, slack=7)
    for name in ("q", "hk", "ck"):
        t = getattr(a, name)
        s = t.stride()
        setattr(a, name, t.as_strided(t.shape, (0, *s[1:]), t.storage_offset()))
    _check(a, range(4), tensor_cores=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [127, 128, 129, 300])
def test_more_requests_than_a_warp_searches_at_once(batch, dtype):
    """The search for a CTA's items in one pass and in two; empty requests, requests without queries, and long ones between them."""
    import torch
    from attend_reference import attend_rows, check_rows
    Hq, Hkv, d = 4, 2, 64
    lens = [(0, 1, 64, 63, 130, 5, 65, 0, 17, 700)[i % 10] for i in range(batch)]
    counts = [(1, 1, 1, 0, 2, 1, 0, 1, 3, 1)[i % 10] for i in range(batch)]
    lens[-1], counts[-1] = 1000, 1
    c = Cache(1, Hq, Hkv, d, batch, 16, dtype)
    try:
        c.append(lens)
        off = [sum(counts[:i]) for i in range(batch + 1)]
        q = torch.randn((1, Hq, off[-1], d), generator=c.g, device="cuda").to(c.dtype)
        out, lse = torch.full_like(q, math.nan), torch.full((1, Hq, off[-1]), math.nan, device="cuda")
        meta = fb.make_paged_batch(lens, q_off=off)
        ws = torch.full((fb.finch_pages_workspace_bytes(c.ctx, meta),), 255, dtype=torch.uint8, device="cuda")
        fb.finch_pages_attend(c.ctx, c.pages, meta, q, out, lse, ws=ws)
        assert fb.finch_device_status(c.ctx) == 0
        assert torch.isfinite(out.float()).all()
        for b in sorted({0, 1, 2, 4, 8, 9, 123, 124, 126, batch - 3, batch - 2, batch - 1} & set(range(batch))):
            if not counts[b]:
                continue
            k, v = c.values(b)
            rows = slice(off[b], off[b + 1])
            for h in range(Hq):
                limits = [max(0, lens[b] - counts[b] + i + 1) for i in range(counts[b])]
                # as in Cache.attend: queries and weights enter the products with 22 bits
                want = list(attend_rows(q[0, h, rows], k[0, h // 2], v[0, h // 2], limits, 1 / 8, None, 2.0 ** -20))
                if lens[b]:
                    big = q[0, h, rows].double().abs().amax(-1) * k[0, h // 2].abs().sum(-1).max() / 8 * 2.0 ** -21
                    want[3], want[2] = want[3] + big, want[2] + 2 * big[:, None] * v[0, h // 2].abs().amax()
                check_rows(out[0, h, rows], lse[0, h, rows], *want, what=f"request {b} head {h}")
    finally:
        c.close()
