"""The operators in a row, as a program that answers from a compressed document uses them: rotate and attend for the prompt's own
pass, its log-sum-exp into the scoring, the kept rows into pages, then tokens one by one."""
import math

import numpy as np
import pytest

from paper_2408_00167_b200 import binding as fb
from paper_2408_00167_b200 import build as fbuild
from paper_2408_00167_b200.document import DocumentCompressor
from paper_2408_00167_b200.generate import PagedCache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    fbuild.build()
    fb.load()


@pytest.mark.parametrize("dtype", [fb.FINCH_BF16, fb.FINCH_F32])
def test_a_document_is_compressed_and_answered_from(dtype):
    import torch
    from attend_reference import attend_rows, check_rows, dequantised, quantised, turned
    L, Hq, Hkv, d, B = 2, 8, 2, 64, 2
    prompt, chunk, keep, new_tokens = [9, 5], [150, 90], [130, 64], 67
    tdtype = torch.bfloat16 if dtype == fb.FINCH_BF16 else torch.float32
    g = torch.Generator(device="cuda").manual_seed(11)
    rows = lambda heads, n, layers=L: torch.randn((layers, heads, n, d), generator=g, device="cuda").to(tdtype)
    off = lambda ns: [0] + np.cumsum(ns).tolist()
    q_off, chunk_off = off(prompt), off(chunk)
    total = sum(prompt)
    freq = fb.finch_rope_frequencies(d, 10000.0)
    rope = fb.finch_rope_init(d, freq)

    # the prompt's pass over its own keys, all layers, queries and keys at their positions
    ctx = fb.finch_ctx_create(L, Hq, Hkv, d, dtype, max_batch=B, max_prompt=max(prompt), max_candidates=2 * max(prompt))
    q_raw, k_raw, v_own = rows(Hq, total), rows(Hkv, total), rows(Hkv, total)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in prompt]).cuda()
    q, k = torch.empty_like(q_raw), torch.empty_like(k_raw)
    fb.finch_rotate(ctx, q_raw, k_raw, pos, q, k, rope=rope)
    out, lse = torch.empty_like(q), torch.empty((L, Hq, total), device="cuda")
    batch = fb.make_batch(q_off, q_off, [0] * (B + 1), [0] * B, [0] * B)
    ws = torch.empty(fb.finch_attend_workspace_bytes(ctx, batch), dtype=torch.uint8, device="cuda")
    none = rows(Hkv, 0)
    fb.finch_attend(ctx, q, none, none, k, v_own, batch, out, lse, causal=True, ws=ws)
    assert fb.finch_device_status(ctx) == 0
    half = 2.0 ** -8 if dtype == fb.FINCH_BF16 else 0.0
    for b in range(B):
        r = slice(q_off[b], q_off[b + 1])
        for l in range(L):
            for h in range(Hq):
                want = attend_rows(q[l, h, r], k[l, h // 4, r], v_own[l, h // 4, r], range(1, prompt[b] + 1), 1 / 8, None, half)
                check_rows(out[l, h, r], lse[l, h, r], *want)
    fb.finch_ctx_destroy(ctx)

    # the document's chunk against the prompt, the prompt's own keys in the denominators
    doc = DocumentCompressor(L, Hq, Hkv, d, dtype, keep, max_prompt=max(prompt), max_chunk=max(chunk))
    chunk_k, chunk_v = rows(Hkv, sum(chunk)), rows(Hkv, sum(chunk))
    chunk_pos = torch.arange(sum(chunk), dtype=torch.int32, device="cuda")
    doc.step(q, q_off, chunk_k, chunk_v, chunk_pos, chunk_off, keep, prompt_self_lse=lse)
    doc.verify()

    # generation: a token a step, over the end of a page
    rope_new = fb.finch_rope_init(d, freq, pairing=1)
    cache = PagedCache(L, Hq, Hkv, d, dtype, B, max_tokens=max(keep) + new_tokens, rope=rope_new)
    cache.fill(doc)
    kept = [[t[:, :, int(doc.cache_off[b]):int(doc.cache_off[b]) + keep[b]].clone() for t in (doc.cache_k, doc.cache_v)] for b in range(B)]
    for step in range(new_tokens):
        new_k, new_v, new_q = rows(Hkv, B), rows(Hkv, B), rows(Hq, B)
        at = torch.tensor([t[0].shape[2] for t in kept], device="cuda")
        for b in range(B):
            turned_k = turned(new_k[:, :, b:b + 1], at[b:b + 1], freq, d, 1).float().to(tdtype)
            kept[b] = [torch.cat([kept[b][0], turned_k], 2), torch.cat([kept[b][1], new_v[:, :, b:b + 1]], 2)]
        cache.step()
        for l in range(L):
            got, got_lse = torch.empty_like(new_q[l:l + 1]), torch.empty((1, Hq, B), device="cuda")
            cache.append(l, new_k[l:l + 1], new_v[l:l + 1])
            cache.attend(l, new_q[l:l + 1], got, got_lse)
            if step % 11 and step != new_tokens - 1:
                continue
            for b in range(B):
                kv = []
                for x in kept[b]:
                    x = x[l]
                    full = x.shape[1] // 64 * 64
                    codes, scale = quantised(x[:, :full].reshape(Hkv, -1, 64, d))
                    kv.append(torch.cat([dequantised(codes, scale).reshape(Hkv, full, d), x[:, full:].double()], 1))
                for h in range(Hq):
                    qh = new_q[l, h, b:b + 1]
                    want = list(attend_rows(qh, kv[0][h // 4], kv[1][h // 4], [kv[0].shape[1]], 1 / 8, None, 2.0 ** -20))
                    big = qh.double().abs().amax(-1) * kv[0][h // 4].abs().sum(-1).max() / 8 * 2.0 ** -21   # queries enter with 22 bits
                    want[3], want[2] = want[3] + big, want[2] + 2 * big[:, None] * kv[1][h // 4].abs().amax()
                    check_rows(got[0, h, b:b + 1], got_lse[0, h, b:b + 1], *want, what=f"step {step} layer {l} request {b} head {h}")
    assert cache.status() == 0 and cache.len.tolist() == [n + new_tokens for n in keep]
    with pytest.raises(ValueError):
        cache.step(10)
    cache.close()
    doc.close()


def test_steps_of_several_tokens_and_a_batch_without_a_document():
    """Two tokens of every request a step (a draft that is verified): each sees the cache up to itself."""
    import torch
    from attend_reference import attend_rows, check_rows
    L, Hq, Hkv, d, B = 1, 4, 1, 128, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = PagedCache(L, Hq, Hkv, d, fb.FINCH_BF16, B, max_tokens=40, max_step=2)
    ks, vs = [], []
    for step in range(20):
        k, v, q = (torch.randn((1, h, 2 * B, d), generator=g, device="cuda").to(torch.bfloat16) for h in (Hkv, Hkv, Hq))
        ks.append(k), vs.append(v)
        cache.step(2)
        out = torch.empty_like(q)
        cache.append(0, k, v)
        cache.attend(0, q, out)
    for b in range(B):                     # fewer than 64 tokens: nothing has been quantised
        key, value = (torch.cat([x[0, 0, 2 * b:2 * b + 2] for x in xs]) for xs in (ks, vs))
        for h in range(Hq):
            want = attend_rows(q[0, h, 2 * b:2 * b + 2], key, value, [39, 40], 1 / math.sqrt(d), None, 2.0 ** -20)
            check_rows(out[0, h, 2 * b:2 * b + 2], None, *want)
    assert cache.status() == 0
    cache.close()


def test_calls_out_of_order():
    import torch
    x = torch.zeros((1, 2, 1, 64), device="cuda")
    cache = PagedCache(1, 2, 2, 64, fb.FINCH_F32, 1, max_tokens=4, max_step=2)
    try:
        for call in (lambda: cache.append(0, x, x), lambda: cache.attend(0, x, x.clone()), lambda: cache.step(3), lambda: cache.step(0)):
            with pytest.raises(ValueError):
                call()
        cache.step()
        cache.append(0, x, x)
        cache.attend(0, x, x.clone())
        two = torch.zeros((1, 2, 2, 64), device="cuda")
        for call in (lambda: cache.append(0, two, two), lambda: cache.append(0, x, x[:, :1]), lambda: cache.attend(0, two, two.clone())):
            with pytest.raises(ValueError):
                call()
        assert cache.status() == 0 and cache.len.tolist() == [1]
    finally:
        cache.close()


def test_a_document_whose_step_was_refused_does_not_become_a_cache():
    """The compressor's lengths on the host are a prediction; a step that the device refused has written no rows."""
    import torch
    L, Hq, Hkv, d = 1, 4, 2, 64
    doc = DocumentCompressor(L, Hq, Hkv, d, fb.FINCH_BF16, [32], max_prompt=8, max_chunk=100)
    cache = PagedCache(L, Hq, Hkv, d, fb.FINCH_BF16, 1, max_tokens=64)
    try:
        rows = lambda h, n: torch.randn((L, h, n, d), device="cuda").to(torch.bfloat16)
        doc._bufs[doc._cur]["len"].fill_(1)                  # the host's bound on the cache is 0
        doc.step(rows(Hq, 8), [0, 8], rows(Hkv, 100), rows(Hkv, 100), torch.arange(100, dtype=torch.int32, device="cuda"), [0, 100], [32])
        assert doc.cache_len.tolist() == [32]
        with pytest.raises(RuntimeError):
            cache.fill(doc)
        assert cache.len.tolist() == [0] and cache.status() == 0
        cache.fill(doc)                                      # again: there is nothing to move
        assert doc.cache_len.tolist() == [0] and cache.len.tolist() == [0]
    finally:
        cache.close()
        doc.close()


def test_steps_on_one_stream_and_calls_on_another():
    """Descriptions of steps are made on the current stream; a slow other stream still reads those of steps long past."""
    import torch
    Hq, Hkv, d, B, steps = 4, 2, 64, 3, 40
    g = torch.Generator(device="cuda").manual_seed(7)
    rows = [[torch.randn((1, h, B, d), generator=g, device="cuda") for h in (Hkv, Hkv, Hq)] for _ in range(steps)]
    side, results = torch.cuda.Stream(), []
    for other in (False, True):
        cache = PagedCache(1, Hq, Hkv, d, fb.FINCH_F32, B, max_tokens=steps)
        out = [torch.full_like(q, math.nan) for _, _, q in rows]
        torch.cuda.synchronize()
        stream = side if other else torch.cuda.current_stream()
        if other:
            with torch.cuda.stream(side):
                torch.cuda._sleep(200_000_000)      # some 0.1 s, in which all steps are made
        for (k, v, q), o in zip(rows, out):
            cache.step()
            with torch.cuda.stream(stream):
                cache.append(0, k, v)
                cache.attend(0, q, o)
            torch.full((B,), 1, dtype=torch.int32, device="cuda")     # takes memory of the sizes that a step's arrays have
        torch.cuda.synchronize()
        assert cache.status() == 0
        results.append(out)
        cache.close()
    assert all(torch.equal(a, b) for a, b in zip(*results)) and not any(torch.isnan(a).any() for a in results[0])
