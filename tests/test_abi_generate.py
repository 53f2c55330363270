"""Refusals and host arithmetic of finch_rotate, finch_attend and the paged cache; no GPU (a validation-only context)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2408_00167_b200 import binding as fb
from paper_2408_00167_b200 import build as fbuild

OK, INVALID, UNSUPPORTED, LAYOUT, SMALL = (fb.FINCH_OK, fb.FINCH_ERR_INVALID_ARG, fb.FINCH_ERR_UNSUPPORTED, fb.FINCH_ERR_BAD_LAYOUT,
                                           fb.FINCH_ERR_WORKSPACE_TOO_SMALL)
BASE = 0x7000_0000_0000


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fb.load()


@pytest.fixture()
def ctx(lib):
    c = fb.finch_ctx_create(2, 8, 2, 64, fb.FINCH_BF16, max_batch=4, max_prompt=64, max_candidates=1024, device=-1)
    yield c
    fb.finch_ctx_destroy(c)


def tensor(slot, tokens, heads, d=64, shift=0, token_major=False, stride_tok=None):
    """Addresses only: validation never follows them."""
    at = BASE + 0x1000_0000 * (slot + 1) + shift
    if token_major:
        return fb.finch_tensor(at, tokens * heads * d, d, heads * d)
    st = d if stride_tok is None else stride_tok
    return fb.finch_tensor(at, heads * tokens * st, tokens * st, st)


NULL = fb.finch_tensor(None, 0, 0, 0)


def rope(rotary=64, pairing=0, magnitude=1.0):
    return fb.finch_rope_init(rotary, np.ones(rotary // 2), pairing, magnitude)


def test_frequencies_of_every_scaling(lib):
    """Against the formulas, and what they are for: the ends of the spectrum that a scaling keeps or divides."""
    plain = fb.finch_rope_frequencies(64, 10000.0)
    np.testing.assert_allclose(plain, 10000.0 ** (-2 * np.arange(32) / 64), rtol=1e-14)
    np.testing.assert_allclose(fb.finch_rope_frequencies(64, 10000.0, fb.FINCH_ROPE_LINEAR, 4.0), plain / 4, rtol=1e-14)
    base = fb.finch_rope_frequencies(64, 10000.0, fb.FINCH_ROPE_BASE, 4.0)
    assert base[0] == plain[0]
    np.testing.assert_allclose(base[-1], plain[-1] / 4, rtol=1e-12)      # the slowest pair is stretched by the whole factor
    parts = fb.finch_rope_frequencies(64, 10000.0, fb.FINCH_ROPE_PARTS, 4.0, original=4096, low=1, high=4)
    turns = 4096 * plain / (2 * math.pi)
    np.testing.assert_array_equal(parts[turns >= 4], plain[turns >= 4])
    np.testing.assert_allclose(parts[turns <= 1], plain[turns <= 1] / 4, rtol=1e-14)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.all(parts[mid] < plain[mid]) and np.all(parts[mid] > plain[mid] / 4)


@pytest.mark.parametrize("args", [(0, 1e4), (63, 1e4), (258, 1e4), (64, 0.5), (64, math.nan), (64, math.inf), (64, 1e4, 4), (64, 1e4, -1),
                                  (64, 1e4, 1, 0.5), (64, 1e4, 2, math.nan), (2, 1e4, 2, 2.0), (64, 1e4, 3, 2.0, 0.0),
                                  (64, 1e4, 3, 2.0, 8192.0, 4.0, 4.0), (64, 1e4, 3, 2.0, 8192.0, -1.0, 4.0)])
def test_frequencies_refuse(lib, args):
    with pytest.raises(fb.FinchError) as e:
        fb.finch_rope_frequencies(*args)
    assert e.value.status == INVALID


@pytest.mark.parametrize("rotary,freq,pairing,magnitude,status", [
    (64, np.ones(32), 2, 1.0, INVALID), (64, np.ones(32), 0, math.nan, INVALID), (64, np.full(32, math.nan), 0, 1.0, INVALID),
    (64, np.full(32, 2.5), 0, 1.0, INVALID), (24, np.ones(12), 0, 1.0, UNSUPPORTED)])
def test_rope_init_refuses(lib, rotary, freq, pairing, magnitude, status):
    with pytest.raises(fb.FinchError) as e:
        fb.finch_rope_init(rotary, freq, pairing, magnitude)
    assert e.value.status == status
    with pytest.raises(ValueError):
        fb.finch_rope_init(64, np.ones(31))


def test_rotate_refuses(lib, ctx):
    r = rope()

    def call(q=None, k=None, oq=None, ok=None, tokens=10, pos=BASE, rp=r, qw=None, kw=None, eps=1e-6):
        q, k = q or tensor(0, 10, 8), k or tensor(1, 10, 2)
        oq, ok = oq or tensor(2, 10, 8), ok or tensor(3, 10, 2)
        return lib.finch_rotate(ctx, C.addressof(q), C.addressof(k), tokens, pos, C.addressof(rp) if rp else None, qw, kw, eps,
                                C.addressof(oq), C.addressof(ok), None)
    assert call() == UNSUPPORTED                                  # valid: stops at the launch
    assert call(oq=tensor(0, 10, 8), ok=tensor(1, 10, 2)) == UNSUPPORTED      # in place
    assert call(k=NULL, ok=NULL) == UNSUPPORTED                   # queries alone
    assert call(rp=None, qw=BASE, pos=None) == UNSUPPORTED        # norm alone
    assert call(tokens=0, q=NULL, k=NULL, oq=NULL, ok=NULL) == UNSUPPORTED
    assert call(tokens=-1) == INVALID
    assert call(pos=None) == INVALID
    assert call(rp=None) == INVALID                               # nothing to do
    assert call(k=NULL) == INVALID                                # an output without its tensor
    assert call(q=NULL, k=NULL, oq=NULL, ok=NULL) == INVALID
    assert call(qw=BASE, eps=-1.0) == INVALID
    assert call(qw=BASE, eps=math.nan) == INVALID
    assert call(qw=BASE + 8) == LAYOUT
    assert call(q=tensor(0, 10, 8, shift=8)) == LAYOUT
    assert call(q=tensor(0, 10, 8, stride_tok=60)) == LAYOUT
    assert call(oq=tensor(0, 10, 8, shift=128)) == INVALID        # rows of the output over other rows of the input
    assert call(ok=tensor(0, 10, 2)) == INVALID
    assert call(oq=tensor(3, 10, 8)) == INVALID                   # the outputs over one another
    wide = rope(128)
    assert call(rp=wide) == INVALID                               # wider than a head
    bad = rope()
    bad.rotary_dim = 40
    assert call(rp=bad) == UNSUPPORTED
    # queries and keys side by side in one row of a fused projection, in place
    buf = lambda shift: fb.finch_tensor(BASE + shift * 2, 10 * 12 * 64, 64, 12 * 64)
    assert call(q=buf(0), k=buf(8 * 64), oq=buf(0), ok=buf(8 * 64)) == UNSUPPORTED
    assert call(q=buf(0), k=buf(7 * 64), oq=buf(0), ok=buf(7 * 64)) == INVALID
    assert lib.finch_rotate(None, None, None, 0, None, None, None, None, 0.0, None, None, None) == INVALID


def _batch(B=2, q=40, m=90, c=70, max_q=30, max_m=50, max_c=40, row_norm=0):
    return fb.finch_batch(B, BASE, BASE, BASE, BASE, BASE, q, m, c, max_q, max_c, max_m, 0, None, None, row_norm)


def test_attend_refuses(lib, ctx):
    def call(b=None, causal=1, out=None, ws=BASE, ws_bytes=1 << 40, **other):
        b = b or _batch()
        t = dict(q=tensor(0, b.total_q, 8), ck=tensor(1, b.total_cache, 2), cv=tensor(2, b.total_cache, 2), hk=tensor(3, b.total_chunk, 2),
                 hv=tensor(4, b.total_chunk, 2))
        t.update(other)
        out = out or tensor(5, b.total_q, 8)
        return lib.finch_attend(ctx, *(C.addressof(t[n]) for n in ("q", "ck", "cv", "hk", "hv")), C.addressof(b), causal, C.addressof(out), None,
                                ws, ws_bytes, None)
    assert call() == UNSUPPORTED
    assert call(_batch(c=0, max_c=0), ck=NULL, cv=NULL) == UNSUPPORTED            # no cache
    assert call(_batch(m=0, max_m=0), hk=NULL, hv=NULL) == UNSUPPORTED            # no chunk
    assert call(q=tensor(0, 40, 8, token_major=True), out=tensor(5, 40, 8, token_major=True)) == UNSUPPORTED
    assert call(causal=2) == INVALID
    assert call(_batch(row_norm=1)) == INVALID
    assert call(q=NULL) == INVALID
    assert call(cv=NULL) == INVALID
    assert call(_batch(max_q=65, q=100)) == INVALID                               # beyond the context's prompt
    assert call(_batch(max_c=1000, c=1000)) == INVALID
    assert call(_batch(B=5)) == INVALID
    assert call(hv=tensor(4, 90, 2, shift=4)) == LAYOUT
    assert call(out=tensor(0, 40, 8)) == INVALID                                  # over the queries
    assert call(out=tensor(4, 40, 8, shift=-64 * 2 * 5)) == INVALID               # over the chunk's values
    assert call(ws=None) == INVALID
    assert call(ws=BASE + 8) == LAYOUT
    need = C.c_size_t()
    b = _batch()
    assert lib.finch_attend_workspace_bytes(ctx, C.addressof(b), C.addressof(need)) == OK
    assert call(ws_bytes=need.value - 1) == SMALL and call(ws_bytes=need.value) == UNSUPPORTED
    assert lib.finch_attend_workspace_bytes(ctx, C.addressof(b), None) == INVALID
    assert lib.finch_attend_workspace_bytes(ctx, None, C.addressof(need)) == INVALID


def test_attend_workspace_of_the_most_rows_serves_every_call(lib):
    for L, Hq, Hkv, d in ((1, 32, 8, 128), (32, 32, 8, 128), (1, 64, 1, 256), (2, 3, 3, 32)):
        c = fb.finch_ctx_create(L, Hq, Hkv, d, fb.FINCH_BF16, max_batch=9, max_prompt=5000, max_candidates=100000, device=-1)
        room = 0
        for rows in (1, 2, 31, 32, 33, 100, 1000, 5000):
            b = _batch(B=1, q=rows, max_q=rows)
            need = C.c_size_t()
            assert lib.finch_attend_workspace_bytes(c, C.addressof(b), C.addressof(need)) == OK
            assert need.value >= room and need.value % 256 == 0
            room = need.value
        fb.finch_ctx_destroy(c)


def _pages(**kw):
    base = dict(k=BASE, v=BASE + (1 << 30), k_scale=BASE, v_scale=BASE, open_k=BASE, open_v=BASE, table=BASE, open_slot=None, n_pages=40,
                table_width=8, n_open=4)
    base.update(kw)
    return fb.finch_pages(*base.values())


def _paged(B=2, q=4, n=100, max_q=2, max_n=60, max_len=400, q_off=BASE, new_off=BASE, length=BASE):
    return fb.finch_paged_batch(B, q_off, new_off, length, q, n, max_q, max_n, max_len)


def _append(lib, ctx, pages=None, batch=None, k=None, v=None, r=None, out_len=BASE + 4096):
    pages, batch = pages or _pages(), batch or _paged()
    k, v = k or tensor(0, max(batch.total_new, 1), 2), v or tensor(1, max(batch.total_new, 1), 2)
    return lib.finch_pages_append(ctx, C.addressof(pages), C.addressof(batch), C.addressof(k), C.addressof(v), C.addressof(r) if r else None,
                                  None, out_len, None)


def _decode(lib, ctx, pages=None, batch=None, q=None, out=None, ws=BASE, ws_bytes=1 << 40):
    pages, batch = pages or _pages(), batch or _paged()
    q, out = q or tensor(0, max(batch.total_q, 1), 8), out or tensor(1, max(batch.total_q, 1), 8)
    return lib.finch_pages_attend(ctx, C.addressof(pages), C.addressof(batch), C.addressof(q), C.addressof(out), None, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_append, _decode])
def test_paged_calls_refuse(lib, ctx, call):
    assert call(lib, ctx) == UNSUPPORTED
    assert call(lib, ctx, batch=_paged(B=0, q=0, n=0, max_q=0, max_n=0)) == UNSUPPORTED
    assert call(lib, ctx, _pages(k=None, v=None, k_scale=None, v_scale=None, table=None, n_pages=0, table_width=0),
                _paged(max_len=3, max_n=60, n=60)) == UNSUPPORTED                 # no page is full: only open rows
    for bad in (dict(open_k=None), dict(open_v=None), dict(n_open=0), dict(n_open=1), dict(n_pages=0), dict(n_pages=-1), dict(table=None),
                dict(table_width=3), dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None)):
        assert call(lib, ctx, _pages(**bad)) == INVALID, bad
    assert call(lib, ctx, _pages(open_slot=BASE, n_open=1)) == UNSUPPORTED        # slots of their own
    for bad in (dict(k=BASE + 4), dict(v=BASE + 8), dict(open_k=BASE + 2), dict(open_v=BASE + 8)):
        assert call(lib, ctx, _pages(**bad)) == LAYOUT, bad
    for bad in (dict(B=-1), dict(B=5), dict(max_len=-1), dict(max_len=1025), dict(length=None)):
        assert call(lib, ctx, batch=_paged(**bad)) == INVALID, bad


def test_append_refuses(lib, ctx):
    assert _append(lib, ctx, batch=_paged(new_off=None)) == INVALID
    assert _append(lib, ctx, batch=_paged(q_off=None)) == UNSUPPORTED             # not read here
    assert _append(lib, ctx, batch=_paged(max_n=101)) == INVALID
    assert _append(lib, ctx, batch=_paged(n=-1)) == INVALID
    assert _append(lib, ctx, batch=_paged(max_len=1000)) == INVALID               # 1060 tokens of 1024
    assert _append(lib, ctx, k=NULL) == INVALID
    assert _append(lib, ctx, k=tensor(0, 100, 2, shift=8)) == LAYOUT
    assert _append(lib, ctx, r=rope(128)) == INVALID
    assert _append(lib, ctx, out_len=None) == UNSUPPORTED
    assert _append(lib, ctx, out_len=BASE) == INVALID                             # in place of the lengths
    assert _append(lib, ctx, out_len=BASE + 4) == INVALID
    assert _append(lib, ctx, out_len=BASE + 8) == UNSUPPORTED


def test_paged_attention_refuses(lib, ctx):
    assert _decode(lib, ctx, batch=_paged(q_off=None)) == INVALID
    assert _decode(lib, ctx, batch=_paged(new_off=None)) == UNSUPPORTED
    assert _decode(lib, ctx, batch=_paged(max_q=5)) == INVALID
    assert _decode(lib, ctx, batch=_paged(q=200, max_q=65)) == INVALID
    assert _decode(lib, ctx, q=NULL) == INVALID
    assert _decode(lib, ctx, out=tensor(0, 4, 8)) == INVALID
    assert _decode(lib, ctx, ws=None) == INVALID
    assert _decode(lib, ctx, ws=BASE + 4) == LAYOUT
    b, need = _paged(), C.c_size_t()
    assert lib.finch_pages_workspace_bytes(ctx, C.addressof(b), C.addressof(need)) == OK
    assert _decode(lib, ctx, ws_bytes=need.value - 1) == SMALL and _decode(lib, ctx, ws_bytes=need.value) == UNSUPPORTED
    assert lib.finch_pages_workspace_bytes(None, C.addressof(b), C.addressof(need)) == INVALID
    assert lib.finch_pages_workspace_bytes(ctx, C.addressof(b), None) == INVALID


def test_the_binding_refuses_other_types_shapes_and_devices(lib, ctx):
    """What the C call cannot see: a tensor of another dtype or shape.  Nothing is enqueued (the tensors are the CPU's)."""
    import torch
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    q, k = bf(2, 8, 5, 64), bf(2, 2, 5, 64)
    pos = torch.zeros(5, dtype=torch.int32)
    r = rope()
    for kw in (dict(k=k.float()), dict(k=bf(2, 2, 6, 64)), dict(out_q=bf(2, 8, 4, 64)), dict(pos=pos.long()), dict(pos=pos[:4]),
               dict(q_weight=bf(64)), dict(q_weight=torch.zeros(2, 64)), dict(out_k=None), dict(q=q.transpose(2, 3))):
        a = dict(q=q, k=k, pos=pos, out_q=torch.empty_like(q), out_k=torch.empty_like(k), rope=r)
        a.update(kw)
        with pytest.raises(ValueError):
            fb.finch_rotate(ctx, **a)
    batch = fb.make_batch([0, 5], [0, 5], [0, 0], [0], [0], device="cpu")
    e, lse, ws = bf(2, 2, 0, 64), torch.zeros((2, 8, 5)), torch.zeros(1 << 20, dtype=torch.uint8)
    for kw in (dict(chunk_v=k.float()), dict(out=bf(2, 8, 6, 64)), dict(row_lse=lse.double()), dict(row_lse=lse[:, :4])):
        a = dict(q=q, cache_k=e, cache_v=e, chunk_k=k, chunk_v=k, batch=batch, out=torch.empty_like(q), row_lse=lse, ws=ws)
        a.update(kw)
        with pytest.raises(ValueError):
            fb.finch_attend(ctx, **a)
    pool = lambda dtype=torch.uint8: torch.zeros((2, 3, 2, 64, 64), dtype=dtype)
    good = dict(k=pool(), v=pool(), k_scale=torch.zeros((2, 3, 2)), v_scale=torch.zeros((2, 3, 2)), open_k=bf(2, 1, 2, 64, 64), open_v=bf(2, 1, 2, 64, 64),
                table=torch.zeros((1, 3), dtype=torch.int32))
    for kw in (dict(v=pool(torch.int8)), dict(k_scale=torch.zeros((2, 2, 2))), dict(open_v=torch.zeros((2, 1, 2, 64, 64))),
               dict(table=torch.zeros((1, 3))), dict(open_slot=torch.zeros(2, dtype=torch.int32)), dict(k=pool()[:, :, :, :32])):
        with pytest.raises(ValueError):
            fb.make_pages(**{**good, **kw})
    pages, paged = fb.make_pages(**good), fb.make_paged_batch([10], q_off=[0, 5], new_off=[0, 5], device="cpu")
    with pytest.raises(ValueError):
        fb.finch_pages_append(ctx, pages, paged, k.float(), k)
    with pytest.raises(ValueError):
        fb.finch_pages_append(ctx, pages, paged, k, k, out_len=torch.zeros(1))
    with pytest.raises(ValueError):
        fb.finch_pages_attend(ctx, pages, paged, q, bf(2, 8, 4, 64), ws=ws)
    with pytest.raises(ValueError):
        fb.make_paged_batch([10], new_off=[0, 5], len_tensor=torch.zeros(1), device="cpu")


def test_a_cache_checks_the_document_that_fills_it(monkeypatch):
    """fill asks the compressor before it believes the lengths on the host, and moves nothing if that raises."""
    from paper_2408_00167_b200.generate import PagedCache
    moved = []
    monkeypatch.setattr(fb, "finch_pages_append", lambda *a, **k: moved.append(a))

    class Refused:
        L = Hkv = d = B = 1
        cache_len = np.array([3], dtype=np.int32)

        def verify(self):
            raise RuntimeError("status word")

    cache = PagedCache.__new__(PagedCache)
    cache.L = cache.Hkv = cache.d = cache.B = 1
    cache.max_tokens, cache.len = 64, np.zeros(1, dtype=np.int32)
    with pytest.raises(RuntimeError):
        cache.fill(Refused())
    assert not moved and cache.len.tolist() == [0]


def test_the_binding_refuses_tensors_that_do_not_hold_the_call(lib, ctx, monkeypatch):
    """A call takes addresses and strides; rows, heads and layers are the context's and the batch's.  A tensor that has fewer would be read
    and written behind its end, one of another type misread.  (The context has 2 layers, 8 and 2 heads of 64, bf16.)"""
    import torch
    monkeypatch.setattr(fb, "_stream", lambda stream: None)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)

    def refused(call, base, **changes):
        with pytest.raises(fb.FinchError) as e:          # as it is, a call stops at the launch
            call(ctx, **base)
        assert e.value.status == UNSUPPORTED
        for name, value in changes.items():
            for v in value:
                a = dict(base)
                for n, x in (v.items() if isinstance(v, dict) else [(name, v)]):
                    a[n] = x
                with pytest.raises(ValueError):
                    call(ctx, **a)

    q, k = bf(2, 8, 5, 64), bf(2, 2, 5, 64)
    refused(fb.finch_rotate, dict(q=q, k=k, pos=i32(1, 2, 3, 4, 5), out_q=bf(2, 8, 5, 64), out_k=bf(2, 2, 5, 64), rope=rope()),
            heads=[dict(q=bf(2, 4, 5, 64), out_q=bf(2, 4, 5, 64)), dict(k=bf(2, 1, 5, 64), out_k=bf(2, 1, 5, 64)),
                   dict(q=None, out_q=None, k=bf(2, 1, 5, 64), out_k=bf(2, 1, 5, 64))],
            layers=[dict(q=bf(1, 8, 5, 64), k=bf(1, 2, 5, 64), out_q=bf(1, 8, 5, 64), out_k=bf(1, 2, 5, 64))],
            dim=[dict(q=bf(2, 8, 5, 32), k=bf(2, 2, 5, 32), out_q=bf(2, 8, 5, 32), out_k=bf(2, 2, 5, 32))],
            dtype=[{n: x.float() for n, x in (("q", q), ("k", k), ("out_q", q), ("out_k", k))}],
            rank=[dict(q=bf(8), out_q=bf(8))])

    batch = fb.make_batch([0, 5], [0, 6], [0, 7], [7], [7], device="cpu")
    rows = fb.make_batch([0, 6], [0, 6], [0, 7], [7], [7], device="cpu")
    limited = lambda **kw: fb.make_batch([0, 5], [0, 6], [0, 7], [7], [7], device="cpu", **kw)
    space = torch.zeros(1 << 22, dtype=torch.uint8)
    attend = dict(q=q, cache_k=bf(2, 2, 7, 64), cache_v=bf(2, 2, 7, 64), chunk_k=bf(2, 2, 6, 64), chunk_v=bf(2, 2, 6, 64), batch=batch,
                  out=bf(2, 8, 5, 64), row_lse=torch.zeros(2, 8, 5), ws=space)
    refused(fb.finch_attend, attend, batch=[rows, limited(prompt_self_lse=torch.zeros(2, 8, 4)), limited(prompt_self_lse=torch.zeros(2, 8, 6)),
                                            limited(prompt_self_lse=torch.zeros(2, 8, 5).double()), limited(row_limit=i32(1, 2, 3, 4)),
                                            limited(row_limit=i32(1, 2, 3, 4, 5).long())],
            cache_k=[bf(2, 2, 6, 64), bf(2, 1, 7, 64), bf(1, 2, 7, 64)], cache_v=[bf(2, 2, 6, 64)], chunk_k=[bf(2, 2, 5, 64), bf(2, 2, 6, 32)],
            chunk_v=[bf(2, 2, 5, 64)], ws=[torch.zeros((1 << 22, 2), dtype=torch.uint8)[:, 0]],
            heads=[dict(q=bf(2, 4, 5, 64), out=bf(2, 4, 5, 64), row_lse=None)])
    # more rows than the batch's are a padded batch; row_lse then has the batch's
    padded = dict(attend, q=bf(2, 8, 9, 64), out=bf(2, 8, 9, 64), cache_k=bf(2, 2, 9, 64), chunk_v=bf(2, 2, 8, 64))
    refused(fb.finch_attend, padded, row_lse=[torch.zeros(2, 8, 9)])
    refused(fb.finch_attend, dict(attend, batch=limited(prompt_self_lse=torch.zeros(2, 8, 5), row_limit=i32(1, 2, 3, 4, 5, 6))))
    refused(fb.finch_attend, dict(attend, batch=limited(prompt_self_lse=torch.zeros(200))))         # one axis: a buffer that holds them

    def pages(L=2, Hkv=2, d=64, requests=2, dtype=torch.bfloat16):
        pool, scale = (lambda: torch.zeros((L, 3, Hkv, 64, d), dtype=torch.uint8)), (lambda: torch.zeros((L, 3, Hkv)))
        rows = lambda: torch.zeros((L, 2, Hkv, 64, d), dtype=dtype)
        return fb.make_pages(pool(), pool(), scale(), scale(), rows(), rows(), torch.zeros((requests, 3), dtype=torch.int32))

    two = fb.make_paged_batch([10, 3], q_off=[0, 2, 5], new_off=[0, 2, 5], device="cpu")
    six = fb.make_paged_batch([10, 3], q_off=[0, 2, 6], new_off=[0, 2, 6], device="cpu")
    other = [pages(L=1), pages(Hkv=1), pages(d=32), pages(requests=1), pages(dtype=torch.float32)]
    refused(fb.finch_pages_append, dict(pages=pages(), batch=two, new_k=k, new_v=k), pages=other, batch=[six],
            new_k=[bf(2, 2, 4, 64), bf(2, 1, 5, 64), bf(1, 2, 5, 64)], new_v=[bf(2, 2, 4, 64), bf(2, 2, 5, 32)])
    decode = dict(pages=pages(), batch=two, q=q, out=bf(2, 8, 5, 64), row_lse=torch.zeros(2, 8, 5), ws=space)
    refused(fb.finch_pages_attend, decode, pages=other, batch=[six], heads=[dict(q=bf(2, 4, 5, 64), out=bf(2, 4, 5, 64), row_lse=None)],
            ws=[torch.zeros((1 << 22, 2), dtype=torch.uint8)[:, 0]])
    refused(fb.finch_pages_attend, dict(decode, q=bf(2, 8, 7, 64), out=bf(2, 8, 7, 64)), row_lse=[torch.zeros(2, 8, 7)])
    with pytest.raises(ValueError):
        pages(dtype=torch.float16)
    # a handle from elsewhere: the tensors among themselves
    raw = C.c_void_p(ctx.value)
    with pytest.raises(ValueError):
        fb.finch_attend(raw, **dict(attend, cache_v=bf(2, 1, 7, 64)))
    with pytest.raises(ValueError):
        fb.finch_pages_append(raw, pages(Hkv=1), two, k, k)


def test_attend_refuses_log_sum_exps_over_the_extra_term(lib, ctx):
    """Several warps and CTAs read a row's extra term while one of them writes its log-sum-exp."""
    b, far = _batch(q=40), 0x2000_0000
    b.prompt_self_lse = BASE + far
    tensors = [tensor(0, 40, 8), tensor(1, 70, 2), tensor(2, 70, 2), tensor(3, 90, 2), tensor(4, 90, 2)]
    out, size = tensor(5, 40, 8), 2 * 8 * 40 * 4
    call = lambda lse: lib.finch_attend(ctx, *map(C.addressof, tensors), C.addressof(b), 1, C.addressof(out), lse, BASE, 1 << 40, None)
    for at in (0, 4, size - 4, 4 - size):
        assert call(BASE + far + at) == INVALID
    for at in (size, -size):
        assert call(BASE + far + at) == UNSUPPORTED               # valid: stops at the launch
    assert call(None) == UNSUPPORTED


def test_holders_stay_on_the_device_that_was_current(lib, monkeypatch):
    """device="cuda" is the device that is current when the object is made, for its contexts, its tensors and what later steps upload."""
    import torch
    from paper_2408_00167_b200.document import DocumentCompressor
    from paper_2408_00167_b200.generate import PagedCache
    current, seen, create = [3], [], fb.finch_ctx_create

    def on_cpu(name):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, device=None, **kw: (seen.append(device), real(*a, **kw))[1])

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(fb, "_stream", lambda stream: None)
    monkeypatch.setattr(fb, "finch_ctx_create", lambda *a, **kw: (seen.append(torch.device("cuda", kw["device"])), create(*a, **{**kw, "device": -1}))[1])
    for name in ("zeros", "full", "arange", "empty"):
        on_cpu(name)
    sizes = dict(n_layers=1, n_q_heads=2, n_kv_heads=1, head_dim=64, dtype=fb.FINCH_BF16)
    for make in (lambda **kw: PagedCache(batch=2, max_tokens=100, **sizes, **kw),
                 lambda **kw: DocumentCompressor(capacity=[8], max_prompt=4, max_chunk=4, **sizes, **kw)):
        for kw, want in ((dict(), "cuda:3"), (dict(device="cuda"), "cuda:3"), (dict(device="cuda:1"), "cuda:1"), (dict(device=torch.device("cuda", 0)), "cuda:0")):
            seen.clear()
            held = make(**kw)
            current[0] = 5
            assert seen and set(map(str, seen)) == {want} and str(held.device) == want
            current[0] = 3
            held.close()


def test_a_layer_gets_the_rows_of_every_step_once(lib, monkeypatch):
    """What append and attend of a PagedCache would get wrong: a layer twice in a step, attention before the step's rows are there, a
    layer that missed a step.  A layer that is never used does no harm."""
    import torch
    from paper_2408_00167_b200.generate import PagedCache
    create, calls = fb.finch_ctx_create, []
    monkeypatch.setattr(fb, "finch_ctx_create", lambda *a, **kw: create(*a, **{**kw, "device": -1}))
    monkeypatch.setattr(fb, "finch_pages_append", lambda *a, **kw: calls.append("append"))
    monkeypatch.setattr(fb, "finch_pages_attend", lambda *a, **kw: calls.append("attend"))
    cache = PagedCache(3, 2, 1, 64, fb.FINCH_F32, 2, max_tokens=70, max_step=2, device="cpu")
    k = lambda n: torch.zeros((1, 1, 2 * n, 64))
    q = lambda n: torch.zeros((1, 2, 2 * n, 64))

    def refused(call, *args):
        n = len(calls)
        with pytest.raises(ValueError):
            call(*args)
        assert len(calls) == n

    cache.step()
    refused(cache.attend, 0, q(1), q(1))
    cache.append(0, k(1), k(1))
    cache.attend(0, q(1), q(1))
    cache.attend(0, q(1), q(1))
    refused(cache.append, 0, k(1), k(1))
    refused(cache.attend, 1, q(1), q(1))
    cache.append(-2, k(1), k(1))                 # layer 1
    refused(cache.append, 1, k(1), k(1))
    cache.step(2)
    cache.append(0, k(2), k(2))
    refused(cache.attend, 1, q(2), q(2))
    refused(cache.append, 2, k(2), k(2))         # it has missed a step
    refused(cache.attend, 2, q(2), q(2))
    cache.append(1, k(2), k(2))
    cache.attend(1, q(2), q(2))
    refused(cache.append, 1, k(2), k(2))
    assert calls == ["append", "attend", "attend", "append", "append", "append", "attend"] and cache.len.tolist() == [3, 3]
    cache.close()


def test_a_cache_keeps_what_another_stream_reads(lib, monkeypatch):
    """A step's description made on one stream and read on another is held for that one (nothing is held where they are the same)."""
    import torch
    from paper_2408_00167_b200.generate import PagedCache
    create, now, held = fb.finch_ctx_create, ["a"], []
    monkeypatch.setattr(fb, "finch_ctx_create", lambda *a, **kw: create(*a, **{**kw, "device": -1}))
    for name in ("finch_pages_append", "finch_pages_attend"):
        monkeypatch.setattr(fb, name, lambda *a, **kw: None)
    monkeypatch.setattr(PagedCache, "_stream", lambda self: now[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: now[0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: held.append((self.data_ptr(), s)))
    cache = PagedCache(1, 2, 1, 64, fb.FINCH_F32, 2, max_tokens=70, device="cpu")
    k, q = torch.zeros((1, 1, 2, 64)), torch.zeros((1, 2, 2, 64))

    def both():
        held.clear()
        cache.append(0, k, k)
        cache.attend(0, q, q)
        return held

    cache.step()
    assert not both()
    lasting, seen = (cache._ws, cache.table, cache.slot, *cache._tensors), {"a"}
    for made, read in (("a", "b"), ("b", "a"), ("b", "b"), ("c", "c"), ("a", "c"), ("a", "a")):
        now[0] = made
        cache.step()
        now[0] = read
        want = [] if made == read else [cache._add.new_off, cache._add.len, cache._see.q_off, cache._see.len]
        want += [] if read in seen else lasting          # for good
        seen.add(read)
        assert sorted(both()) == sorted((t.data_ptr(), read) for t in want)
    cache.close()


def test_attend_plan(lib):
    """How a batch is shared out, on 148 SMs: the sizes at which the rule changes its mind, and its refusals."""
    ONE, ROWS, KEYS = fb.FINCH_ATTEND_ONE_STREAM, fb.FINCH_ATTEND_ROW_PAIRS, fb.FINCH_ATTEND_KEY_PAIRS

    def plan(Hq, Hkv, rows, cache, chunk, batch=1, d=128, dtype=fb.FINCH_BF16):
        c = fb.finch_ctx_create(1, Hq, Hkv, d, dtype, max_batch=batch, max_prompt=rows, max_candidates=cache + chunk, device=-1)
        try:
            off = lambda n: [n * i for i in range(batch + 1)]
            return fb.finch_attend_plan(c, fb.make_batch(off(rows), off(chunk), off(cache), [cache] * batch, [cache] * batch, device="cpu"))
        finally:
            fb.finch_ctx_destroy(c)

    assert plan(32, 32, 300, 340, 300) == (ROWS, 1, 1) and plan(32, 32, 300, 256, 300) == (ONE, 1, 1)      # six key tiles, five
    assert plan(32, 32, 300, 768, 300) == (ROWS, 1, 1) and plan(32, 32, 300, 896, 300) == (ROWS, 2, 1)     # nine, ten
    assert plan(32, 32, 600, 1024, 600) == (ONE, 1, 1)                                                     # 160 row tiles
    assert plan(32, 32, 600, 3456, 600) == (ONE, 1, 1) and plan(32, 32, 600, 3457, 600) == (ROWS, 1, 1)    # 32 key tiles, 33
    assert plan(32, 8, 128, 2048, 128) == (KEYS, 4, 1)
    assert plan(32, 8, 32, 8192, 32)[:2] == (KEYS, 4) and plan(32, 8, 32, 8192, 32)[2] > 1
    assert plan(8, 8, 8192, 0, 8192) == (ROWS, 1, 1)
    assert plan(32, 8, 128, 2048, 128, d=160)[:2] == (fb.FINCH_ATTEND_MULTIPLY_ADD, 1)
    assert plan(8, 8, 16, 0, 16, dtype=fb.FINCH_F32) == (fb.FINCH_ATTEND_MULTIPLY_ADD, 1, 1)
    assert plan(8, 8, 16, 500, 16, dtype=fb.FINCH_F32)[2] > 1
    c = fb.finch_ctx_create(1, 8, 8, 64, fb.FINCH_BF16, device=-1)
    b, out = _batch(B=1), C.c_int32()
    assert lib.finch_attend_plan(c, C.addressof(b), None, None, None) == INVALID
    assert lib.finch_attend_plan(c, None, C.addressof(out), None, None) == INVALID
    assert lib.finch_attend_plan(c, C.addressof(b), C.addressof(out), None, None) == OK
    assert lib.finch_attend_plan(c, C.addressof(_batch(B=0, q=0, m=0, c=0, max_q=0, max_m=0, max_c=0)), C.addressof(out), None, None) == OK
    fb.finch_ctx_destroy(c)
