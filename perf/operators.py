"""The operators around the compression step, as a program that encodes documents and generates from them calls them.

A case is a call of one of four operators:
  "rotate"  finch_rotate: RMS norm of every query and key head and the rotary embedding, in one pass;
  "attend"  finch_attend: softmax attention of packed query rows over [cache ; chunk], causal or not, with the rows' log-sum-exp;
  "append"  finch_pages_append: rows of K (rotated on the way) and V into a paged cache of 8-bit pages of 64 tokens, one scale
            for each page and head; rows of a page that is not full yet wait in the model's own type;
  "decode"  finch_pages_attend: attention of the newest tokens over that cache.

Inputs are seeded Gaussian draws made on the GPU.  With `own` false, `run` computes the operators with elementary torch
operations in 32 bits (angles, and what is rounded to 8 bits behind them, in 64); with `own` true it calls the library.
"""
import math
import random

import torch

own = False

PAGE = 64            # tokens of a page
E4M3_MAX = 448.0
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _model(layers=1, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16"):
    return dict(layers=layers, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype)


def _rotate(name=None, tokens=1, batch=1, norm=True, pairing=0, part=1, scaling="none", far=32768, **model):
    """`tokens` of each of `batch` sequences whose positions begin below `far`; 1/part of every head turns."""
    case = dict(op="rotate", tokens=tokens, batch=batch, norm=norm, pairing=pairing, part=part, scaling=scaling, far=far, **_model(**model))
    return dict(case, name=name) if name else case


def _attend(name=None, rows=128, cache=0, chunk=0, batch=1, mix=0, causal=True, limits=False, **model):
    """chunk = 0: the rows' own tokens are the chunk.  batch > 1: rows, cache and chunk are bounds of a ragged batch.
    limits: every row has a limit of its own, some of them zero."""
    case = dict(op="attend", rows=rows, cache=cache, chunk=chunk, batch=batch, mix=mix, causal=causal, limits=limits, **_model(**model))
    return dict(case, name=name) if name else case


def _append(name=None, tokens=1, length=0, batch=1, mix=0, rope=True, pairing=0, **model):
    """`tokens` rows to every request (batch > 1: at most) behind `length` (at most) that are there."""
    case = dict(op="append", tokens=tokens, length=length, batch=batch, mix=mix, rope=rope, pairing=pairing, **_model(**model))
    return dict(case, name=name) if name else case


def _decode(name=None, length=2048, rows=1, batch=1, mix=0, **model):
    case = dict(op="decode", length=length, rows=rows, batch=batch, mix=mix, **_model(**model))
    return dict(case, name=name) if name else case


def listed():
    return [
        # one generated token of one request: all latency
        _rotate("rotate_token"),
        # a chunk of 2048 tokens of four documents, interleaved pairs, half of each head, far out in a long context
        _rotate("rotate_chunk", tokens=2048, batch=4, pairing=1, part=2, scaling="parts", far=131072),
        # the prompt's pass over its own keys in a small fp32 model, the source of the step's prompt_self_lse
        _attend("attend_prompt_f32", rows=256, q_heads=8, kv_heads=8, head_dim=64, dtype="f32"),
        # a prompt of 128 tokens behind a full cache: few rows, many keys
        _attend("attend_prompt_cache", rows=128, cache=2048),
        # the chunk of a 32K-token document behind its compressed cache
        _attend("attend_chunk", rows=2048, cache=2048),
        # sixteen prompts of different lengths, packed, multi-head attention
        _attend("attend_packed", rows=512, batch=16, mix=4, kv_heads=32),
        # a text of 8192 tokens without compression
        _attend("attend_text", rows=8192),
        # a generated token of each of sixteen requests, one layer
        _append("append_token", tokens=1, length=4096, batch=16, mix=4),
        # a compressed cache of 2048 tokens moves into pages, all 32 layers
        _append("append_cache", tokens=2048, rope=False, layers=32),
        # generation from a cache of 2048 tokens, one request
        _decode("decode_one", length=2048),
        # sixteen requests with caches of up to 32K tokens
        _decode("decode_batch", length=32768, batch=16, mix=4),
        # a single request with a cache of 131K tokens
        _decode("decode_long", length=131072),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))

    q_heads, kv_heads, head_dim = rng.choice([(32, 8, 128), (32, 8, 128), (32, 32, 128), (8, 8, 64), (8, 2, 128), (16, 4, 64), (12, 4, 96)])
    model = dict(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype="f32" if rng.random() < 0.15 else "bf16")
    op, mix = rng.choice(["rotate", "attend", "attend", "append", "decode", "decode"]), rng.randint(0, 10**6)
    if op == "rotate":
        batch = log(1, 16)
        return _rotate(tokens=log(1, 8192 // batch), batch=batch, norm=rng.random() < 0.6, pairing=rng.randint(0, 1), part=rng.choice([1, 1, 2]),
                       scaling=rng.choice(["none", "linear", "base", "parts"]), far=log(1000, 1000000), **model)
    if op == "attend":
        batch = rng.choice([1, 1, log(2, 16)])
        if model["dtype"] == "f32":
            return _attend(rows=log(16, 1024 // batch), cache=rng.choice([0, log(64, 4096 // batch)]), batch=batch, mix=mix, **model)
        kind = rng.choice(["own", "own", "over", "limits"])
        rows = log(1, 4096 // batch)
        if kind == "own":
            return _attend(rows=rows, cache=rng.choice([0, log(64, 8192 // batch)]), batch=batch, mix=mix, **model)
        return _attend(rows=rows, cache=log(64, 6000 // batch), chunk=log(64, 2048 // batch), batch=batch, mix=mix, causal=False,
                       limits=kind == "limits", **model)
    if op == "append":
        if rng.random() < 0.5:
            return _append(tokens=1, length=log(1, 32768), batch=log(1, 64), mix=mix, pairing=rng.randint(0, 1), layers=log(1, 4), **model)
        return _append(tokens=log(16, 2048), batch=log(1, 4), mix=mix, rope=rng.random() < 0.5, pairing=rng.randint(0, 1),
                       layers=log(1, max(1, 64 // kv_heads)), **model)
    batch = rng.choice([1, log(1, 64)])
    return _decode(length=log(64, min(131072, 2**21 // kv_heads // batch)), rows=rng.choice([1, 1, 1, rng.randint(2, 8)]), batch=batch, mix=mix, **model)


# ---------------------------------------------------------------------------------------------- geometry

def _requests(case):
    """attend: (rows, cache, chunk); append: (tokens, length); decode: (rows, length) of every request."""
    r, B = random.Random(case["mix"]), case["batch"]

    def some(n, least):
        return n if B == 1 else r.randint(min(n, max(least, n // 16)), n)

    out = []
    for _ in range(B):
        if case["op"] == "attend":
            rows, cache = some(case["rows"], 1), some(case["cache"], 0)
            out.append((rows, cache, some(case["chunk"], 1) if case["chunk"] else rows))
        elif case["op"] == "append":
            out.append((some(case["tokens"], 1), some(case["length"], 1)))
        else:
            out.append((case["rows"], max(some(case["length"], 1), case["rows"])))
    return out


def _limits(case):
    """How many candidates each packed query row sees."""
    r, out = random.Random(case["mix"] + 1), []
    for n, c, m in _requests(case):
        for i in range(n):
            if case["limits"]:
                out.append(0 if r.random() < 0.05 else r.randint(0, c + m))
            else:
                out.append(max(0, c + m - n + i + 1) if case["causal"] else c + m)
    return out


def _pages_of(case):
    """Pages that each request of append or decode may touch."""
    extra = case["tokens"] if case["op"] == "append" else 0
    return -(-(case["length"] + extra) // PAGE)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    L, Hq, Hkv, d = case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "rotate":
        n = L * case["tokens"] * case["batch"] * (Hq + Hkv) * d
        return {"bytes": 2 * n * e, "flops": n * (7 if case["norm"] else 3)}
    reqs = _requests(case)
    if case["op"] == "attend":
        rows, keys = sum(n for n, _, _ in reqs), sum(c + m for _, c, m in reqs)
        return {"bytes": L * (e * d * (2 * Hq * rows + 2 * Hkv * keys) + 4 * Hq * rows), "flops": 4 * L * Hq * d * sum(_limits(case))}
    if case["op"] == "append":
        read = written = 0
        for n, have in reqs:
            full, rest = (have % PAGE + n) // PAGE, (have + n) % PAGE
            waiting = have % PAGE if full else 0              # rows of the open page that go into a page now
            read += (n + waiting) * e * d
            written += full * (PAGE * d + 4) + (rest if full else n) * e * d
        return {"bytes": 2 * L * Hkv * (read + written), "flops": 2 * L * Hkv * d * sum(n for n, _ in reqs) * 3}
    total = 0
    for n, have in reqs:
        total += L * (2 * Hkv * (have // PAGE * (PAGE * d + 4) + have % PAGE * d * e) + 2 * Hq * n * d * e)
    return {"bytes": total, "flops": sum(4 * L * Hq * d * (n * have - n * (n - 1) // 2) for n, have in reqs)}


# ---------------------------------------------------------------------------------------------- inputs

class _State:
    """A program's buffers, batch description and context; the context is freed with it."""
    ctx = None

    def __del__(self):
        if self.ctx:
            torch.cuda.synchronize()
            self.fb.finch_ctx_destroy(self.ctx)


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _frequencies(case, rotary_dim, theta=500000.0):
    """The angle per position of every pair, and the scalings for long contexts: "linear" divides the positions by 8, "base"
    raises the base, "parts" divides the slow pairs' frequencies only, by how often they turn within 8192 positions."""
    kind, factor = case.get("scaling", "none"), 8.0
    if kind == "base":
        theta = theta * factor ** (rotary_dim / (rotary_dim - 2.0))
    freq = [theta ** (-2.0 * t / rotary_dim) for t in range(rotary_dim // 2)]
    if kind == "linear":
        freq = [f / factor for f in freq]
    if kind == "parts":
        keep = [min(1.0, max(0.0, (8192.0 * f / (2.0 * math.pi) - 1.0) / (4.0 - 1.0))) for f in freq]
        freq = [w * f + (1.0 - w) * f / factor for w, f in zip(keep, freq)]
    return freq


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    s = _State()
    s.case = case
    dtype = DTYPES[case["dtype"]]
    L, Hq, Hkv, d = case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"]

    def rows(heads, tokens):
        return torch.randn((L, heads, tokens, d), generator=g, device="cuda").to(dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    if case["op"] == "rotate":
        T = case["tokens"] * case["batch"]
        # what a projection leaves: all heads of a token side by side
        s.q, s.k = (torch.randn((L, T, h, d), generator=g, device="cuda").to(dtype).transpose(1, 2) for h in (Hq, Hkv))
        s.out_q, s.out_k = (torch.zeros((L, h, T, d), dtype=dtype, device="cuda") for h in (Hq, Hkv))
        s.w_q, s.w_k = ((1 + 0.1 * torch.randn((L, d), generator=g, device="cuda")).to(dtype) for _ in range(2))
        first = torch.randint(0, case["far"], (case["batch"], 1), generator=g, device="cuda")
        s.pos = (first + torch.arange(case["tokens"], device="cuda")).reshape(-1).to(torch.int32)
        s.rotary_dim = d // case["part"]
        s.freq = torch.tensor(_frequencies(case, s.rotary_dim), dtype=torch.float64, device="cuda")
        bounds = (1, 1, 1)
    elif case["op"] == "attend":
        reqs = _requests(case)
        s.q_off, s.cache_off, s.chunk_off = (_offsets([r[i] for r in reqs]) for i in range(3))
        s.q = rows(Hq, s.q_off[-1])
        s.cache_k, s.cache_v, s.chunk_k, s.chunk_v = (rows(Hkv, n) for n in (s.cache_off[-1],) * 2 + (s.chunk_off[-1],) * 2)
        s.out = torch.zeros_like(s.q)
        s.lse = torch.zeros((L, Hq, s.q_off[-1]), device="cuda")
        s.limit = ints(_limits(case))
        s.row_of, s.cache_of, s.chunk_of = (ints(sum(([b] * r[i] for b, r in enumerate(reqs)), [])) for i in range(3))
        s.key_at = ints(sum((list(range(r[1])) for r in reqs), []) + sum((list(range(r[1], r[1] + r[2])) for r in reqs), []))
        bounds = (len(reqs), max(r[0] for r in reqs), max(r[1] for r in reqs) + max(r[2] for r in reqs))
    else:
        reqs = _requests(case)
        B, W = len(reqs), _pages_of(case)
        n_pages = B * W
        s.length = ints([r[1] for r in reqs])
        s.table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).reshape(B, W)
        shape = (L, n_pages, Hkv, PAGE, d)
        if case["op"] == "append":
            s.new_off = _offsets([r[0] for r in reqs])
            s.k, s.v = rows(Hkv, s.new_off[-1]), rows(Hkv, s.new_off[-1])
            s.request = ints(sum(([b] * r[0] for b, r in enumerate(reqs)), []))
            s.behind = ints(sum((list(range(r[0])) for r in reqs), []))
            s.freq = torch.tensor(_frequencies(case, d), dtype=torch.float64, device="cuda")
            s.page_k, s.page_v = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
            s.scale_k, s.scale_v = (torch.zeros(shape[:3], device="cuda") for _ in range(2))
            s.new_len = torch.zeros_like(s.length)
        else:
            s.q_off = _offsets([r[0] for r in reqs])
            s.q = rows(Hq, s.q_off[-1])
            s.page_k, s.scale_k, s.page_v, s.scale_v = (x for _ in range(2) for x in _filled(shape, g))
            s.out, s.lse = torch.zeros_like(s.q), torch.zeros((L, Hq, s.q_off[-1]), device="cuda")
        s.open_k, s.open_v = (torch.randn((L, B, Hkv, PAGE, d), generator=g, device="cuda").to(dtype) for _ in range(2))
        bounds = (B, case.get("rows", 1), case["length"] + case.get("tokens", 0))
    if own:
        _prepare_own(s, bounds)
    torch.cuda.synchronize()
    return s


def _filled(shape, g):
    """Pages as append leaves them: codes of Gaussian rows, the largest of a page and head at the end of the range."""
    pages, scales = torch.empty(shape, dtype=torch.uint8, device="cuda"), torch.empty(shape[:3], device="cuda")
    flat, flat_scale = pages.reshape(-1, *shape[2:]), scales.reshape(-1, shape[2])
    for at in range(0, flat.shape[0], 1024):
        x = torch.randn(flat[at:at + 1024].shape, generator=g, device="cuda")
        scale = x.abs().amax((-2, -1)) / E4M3_MAX
        flat[at:at + 1024] = (x / scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        flat_scale[at:at + 1024] = scale
    return pages, scales


def _prepare_own(s, bounds):
    """The handles that a program keeps: context, batch description, workspace."""
    from paper_2408_00167_b200 import binding as fb
    s.fb, case = fb, s.case
    s.ctx = fb.finch_ctx_create(case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"],
                                fb.FINCH_F32 if case["dtype"] == "f32" else fb.FINCH_BF16,
                                max_batch=bounds[0], max_prompt=bounds[1], max_candidates=bounds[2])
    if case["op"] == "rotate":
        s.rope = fb.finch_rope_init(s.rotary_dim, s.freq.tolist(), pairing=case["pairing"])
    elif case["op"] == "attend":
        reqs = _requests(case)
        s.batch = fb.make_batch(s.q_off, s.chunk_off, s.cache_off, [r[1] for r in reqs], [r[1] for r in reqs],
                                row_limit=s.limit if case["limits"] else None)
        s.ws = torch.empty(fb.finch_attend_workspace_bytes(s.ctx, s.batch), dtype=torch.uint8, device="cuda")
    else:
        s.pages = fb.make_pages(s.page_k, s.page_v, s.scale_k, s.scale_v, s.open_k, s.open_v, s.table)
        lengths = [r[1] for r in _requests(case)]
        if case["op"] == "append":
            s.rope = fb.finch_rope_init(case["head_dim"], s.freq.tolist(), pairing=case["pairing"]) if case["rope"] else None
            s.batch = fb.make_paged_batch(lengths, new_off=s.new_off)
        else:
            s.batch = fb.make_paged_batch(lengths, q_off=s.q_off)
            s.ws = torch.empty(fb.finch_pages_workspace_bytes(s.ctx, s.batch), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    return {"rotate": _run_rotate, "attend": _run_attend, "append": _run_append, "decode": _run_decode}[s.case["op"]](s)


def _turned(x, pos, freq, rotary_dim, pairing):
    """Rows x [..., tokens, d] turned by pos * freq: angles in 64 bits, their cosines and sines rounded to 32; in x's type."""
    angle = pos.double()[:, None] * freq
    c, sn = angle.cos().float().to(x.dtype), angle.sin().float().to(x.dtype)
    turn, rest = x[..., :rotary_dim], x[..., rotary_dim:]
    if pairing:
        a, b = turn[..., 0::2], turn[..., 1::2]
        out = torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2)
    else:
        a, b = turn.chunk(2, -1)
        out = torch.cat([a * c - b * sn, a * sn + b * c], -1)
    return torch.cat([out, rest], -1)


def _run_rotate(s):
    case = s.case
    if own:
        w_q, w_k = (s.w_q, s.w_k) if case["norm"] else (None, None)
        s.fb.finch_rotate(s.ctx, s.q, s.k, s.pos, s.out_q, s.out_k, rope=s.rope, q_weight=w_q, k_weight=w_k, eps=1e-6)
        return {"q": s.out_q, "k": s.out_k}

    def one(x, w):
        y = x.float()
        if case["norm"]:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w[:, None, None, :].float()
        return _turned(y, s.pos, s.freq, s.rotary_dim, case["pairing"]).to(x.dtype).contiguous()

    return {"q": one(s.q, s.w_q), "k": one(s.k, s.w_k)}


def _softmax(scores, v):
    """(softmax(scores) v, log-sum-exp) of scores [..., rows, keys], in place; a row of -inf gives zeros and -inf."""
    top = scores.amax(-1, keepdim=True)
    shift = torch.where(top == -math.inf, 0.0, top)
    weights = scores.sub_(shift).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights, v) / torch.where(total == 0, 1.0, total)
    return out, (shift + total.log()).squeeze(-1)


def _run_attend(s):
    case = s.case
    if own:
        s.fb.finch_attend(s.ctx, s.q, s.cache_k, s.cache_v, s.chunk_k, s.chunk_v, s.batch, s.out, s.lse, causal=case["causal"], ws=s.ws)
        return {"out": s.out, "lse": s.lse}
    L, Hq, Hkv, d = case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"]
    k, v = torch.cat([s.cache_k, s.chunk_k], 2).float(), torch.cat([s.cache_v, s.chunk_v], 2).float()
    key_of = torch.cat([s.cache_of, s.chunk_of])
    sees = (s.row_of[:, None] == key_of) & (s.key_at < s.limit[:, None])
    scores = torch.matmul(s.q.float().reshape(L, Hkv, -1, d), k.transpose(-1, -2)).mul_(1 / math.sqrt(d))
    scores = scores.reshape(L, Hq, s.q.shape[2], -1).masked_fill_(~sees, -math.inf)
    out, lse = _softmax(scores.reshape(L, Hkv, -1, scores.shape[-1]), v)
    return {"out": out.reshape(s.q.shape).to(s.q.dtype), "lse": lse.reshape(s.lse.shape)}


def _run_append(s):
    case = s.case
    pools = {"page_k": s.page_k.view(torch.float8_e4m3fn), "page_v": s.page_v.view(torch.float8_e4m3fn), "scale_k": s.scale_k,
             "scale_v": s.scale_v, "open_k": s.open_k, "open_v": s.open_v, "len": s.new_len}
    if own:
        s.fb.finch_pages_append(s.ctx, s.pages, s.batch, s.k, s.v, s.new_len, rope=s.rope)
        return pools
    L, B, Hkv, d = case["layers"], case["batch"], case["kv_heads"], case["head_dim"]
    added = torch.zeros_like(s.length).index_add_(0, s.request, torch.ones_like(s.request))
    s.new_len.copy_(s.length + added)
    waiting, first = s.length % PAGE, s.length // PAGE                   # rows of the open page, its number
    W = 1 + -(-case["tokens"] // PAGE)                                   # pages that a request can touch
    slot = (waiting[s.request] + s.behind).long()
    k = s.k
    if case["rope"]:   # in 64 bits: the next step's roundings to 8 bits have borders
        k = _turned(s.k.double(), s.length[s.request] + s.behind, s.freq, d, case["pairing"]).float().to(s.k.dtype)
    page = torch.arange(W, device="cuda")
    full = (page + 1) * PAGE <= (waiting + added)[:, None]                # [B][W]
    at = (first[:, None] + page).clamp(max=s.table.shape[1] - 1).long()
    number = torch.where(full, s.table.gather(1, at), s.page_k.shape[1])  # a page behind the last takes what is not full
    for x, page_x, scale_x, open_x in ((k, s.page_k, s.scale_k, s.open_k), (s.v, s.page_v, s.scale_v, s.open_v)):
        room = torch.zeros((L, B, W * PAGE, Hkv, d), dtype=x.dtype, device="cuda")
        room[:, :, :PAGE] = open_x.transpose(2, 3)
        room[:, s.request.long(), slot] = x.transpose(1, 2)
        rows = room.reshape(L, B, W, PAGE, Hkv, d).transpose(3, 4)        # [L][B][W][Hkv][PAGE][d]
        top = rows.float().abs().amax((-2, -1))
        scale = top / torch.full_like(top, E4M3_MAX)                       # a true quotient: a number as divisor is multiplied by its inverse
        code = (rows.float() / torch.where(scale == 0, 1.0, scale)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        for pool, new in ((page_x, code), (scale_x, scale)):
            wide = torch.cat([pool, pool[:, :1]], 1)
            wide[:, number.long()] = new
            pool.copy_(wide[:, :-1])
        last = ((waiting + added) // PAGE)[:, None]                       # the page that stays open
        tail = rows.gather(2, last.long().reshape(1, B, 1, 1, 1, 1).expand(L, B, 1, Hkv, PAGE, d)).squeeze(2)
        kept = torch.arange(PAGE, device="cuda") < ((waiting + added) % PAGE)[:, None]
        open_x.copy_(torch.where(kept[None, :, None, :, None], tail, open_x))
    return pools


def _run_decode(s):
    case = s.case
    if own:
        s.fb.finch_pages_attend(s.ctx, s.pages, s.batch, s.q, s.out, s.lse, ws=s.ws)
        return {"out": s.out, "lse": s.lse}
    L, B, Hq, Hkv, d, n = (case[x] for x in ("layers", "batch", "q_heads", "kv_heads", "head_dim", "rows"))
    W = s.table.shape[1]
    full = s.length // PAGE
    index = torch.arange(W * PAGE, device="cuda")
    there = index < s.length[:, None]                                     # [B][W * PAGE]
    is_open = (torch.arange(W, device="cuda") == full[:, None])[None, :, :, None, None, None]

    def values(pages, scales, open_rows):
        at = s.table.long()
        x = pages.view(torch.float8_e4m3fn)[:, at].float() * scales[:, at][..., None, None]    # [L][B][W][Hkv][PAGE][d]
        x = torch.where(is_open, open_rows[:, :, None].float(), x)
        return x.transpose(2, 3).reshape(L, B, Hkv, W * PAGE, d).masked_fill(~there[None, :, None, :, None], 0.0)

    k, v = values(s.page_k, s.scale_k, s.open_k), values(s.page_v, s.scale_v, s.open_v)
    q = s.q.float().reshape(L, Hkv, Hq // Hkv, B, n, d).permute(0, 3, 1, 2, 4, 5).reshape(L, B, Hkv, -1, d)
    sees = index < (s.length[:, None] - n + 1 + torch.arange(n, device="cuda"))[..., None]     # [B][n][W * PAGE]
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(1 / math.sqrt(d)).reshape(L, B, Hq, n, -1)
    scores = scores.masked_fill_(~sees[None, :, None], -math.inf).reshape(L, B, Hkv, -1, W * PAGE)
    out, lse = _softmax(scores, v)
    out = out.reshape(L, B, Hq, n, d).transpose(1, 2).reshape(L, Hq, B * n, d)
    return {"out": out.to(s.q.dtype), "lse": lse.reshape(L, B, Hq, n).transpose(1, 2).reshape(L, Hq, B * n)}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    """Row by row of the operators' definitions; None where a pass in 64 bits takes too long."""
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "attend": _exact_attend, "append": _exact_append, "decode": _exact_decode}[case["op"]](s, case)


def _pairs(case, rotary_dim):
    """The two coordinates of every pair that turns."""
    half = rotary_dim // 2
    return [(2 * t, 2 * t + 1) if case["pairing"] else (t, t + half) for t in range(half)]


def _exact_turn(y, pos, freq, pairs, rounded=False):
    """rounded: cosines and sines are of 32 bits, as the append defines them (what it rounds to 8 bits depends on it)."""
    z = y.clone()
    for t, (a, b) in enumerate(pairs):
        angle = pos.double() * freq[t]
        c, sn = angle.cos(), angle.sin()
        if rounded:
            c, sn = c.float().double(), sn.float().double()
        z[..., a], z[..., b] = y[..., a] * c - y[..., b] * sn, y[..., b] * c + y[..., a] * sn
    return z


def _exact_rotate(s, case):
    out = {}
    for name, x, w in (("q", s.q, s.w_q), ("k", s.k, s.w_k)):
        y = x.double()
        if case["norm"]:
            y = y / (y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + 1e-6).sqrt() * w.double()[:, None, None]
        out[name] = _exact_turn(y, s.pos, s.freq, _pairs(case, s.rotary_dim)).contiguous()
    return out


def _exact_rows(q, k, v, limits):
    """One head: every row's softmax over its first limits[i] keys."""
    logits = q @ k.T / math.sqrt(q.shape[-1])
    seen = torch.arange(k.shape[0], device="cuda")[None] < limits[:, None]
    logits = torch.where(seen, logits, torch.full_like(logits, -math.inf))
    lse = torch.logsumexp(logits, -1)
    weights = torch.where(seen, torch.exp(logits - lse[:, None]), torch.zeros_like(logits))
    return weights @ v, lse


def _exact_attend(s, case):
    out, lse = torch.zeros_like(s.q, dtype=torch.float64), torch.zeros_like(s.lse, dtype=torch.float64)
    group = case["q_heads"] // case["kv_heads"]
    for b, (n, c, m) in enumerate(_requests(case)):
        q0, c0, m0 = s.q_off[b], s.cache_off[b], s.chunk_off[b]
        limits = s.limit[q0:q0 + n]
        for l in range(case["layers"]):
            for h in range(case["q_heads"]):
                k = torch.cat([s.cache_k[l, h // group, c0:c0 + c], s.chunk_k[l, h // group, m0:m0 + m]]).double()
                v = torch.cat([s.cache_v[l, h // group, c0:c0 + c], s.chunk_v[l, h // group, m0:m0 + m]]).double()
                out[l, h, q0:q0 + n], lse[l, h, q0:q0 + n] = _exact_rows(s.q[l, h, q0:q0 + n].double(), k, v, limits)
    return {"out": out, "lse": lse}


def _exact_append(s, case):
    L, d, dtype = case["layers"], case["head_dim"], DTYPES[case["dtype"]]
    got = {"len": None}
    for name, new, pool, scales, waiting in (("k", s.k, s.page_k, s.scale_k, s.open_k), ("v", s.v, s.page_v, s.scale_v, s.open_v)):
        page, scale, open_rows = pool.view(torch.float8_e4m3fn).double(), scales.double(), waiting.double()
        for b, (n, have) in enumerate(_requests(case)):
            x = new[:, :, s.new_off[b]:s.new_off[b] + n].double()
            if name == "k" and case["rope"]:
                x = _exact_turn(x, have + torch.arange(n, device="cuda"), s.freq, _pairs(case, d), rounded=True)
                x = x.to(dtype).double()              # a row waits, and is quantised, in the model's own type
            x = torch.cat([open_rows[:, b, :, :have % PAGE], x], 2)
            whole = x.shape[2] // PAGE
            for w in range(whole):
                rows = x[:, :, w * PAGE:(w + 1) * PAGE]
                at = int(s.table[b, have // PAGE + w])
                scale[:, at] = (rows.abs().amax((-2, -1)) / E4M3_MAX).float().double()
                page[:, at] = (rows / scale[:, at][..., None, None]).float().to(torch.float8_e4m3fn).double()
            rest = x[:, :, whole * PAGE:]
            open_rows[:, b, :, :rest.shape[2]] = rest
        got["page_" + name], got["scale_" + name], got["open_" + name] = page, scale, open_rows
    return got


def _exact_decode(s, case):
    L, Hq, Hkv, n = case["layers"], case["q_heads"], case["kv_heads"], case["rows"]
    out, lse = torch.zeros_like(s.q, dtype=torch.float64), torch.zeros_like(s.lse, dtype=torch.float64)
    for b, (_, have) in enumerate(_requests(case)):
        at = s.table[b, :have // PAGE].long()
        limits = have - n + 1 + torch.arange(n, device="cuda")
        for l in range(L):
            for h in range(Hkv):
                k, v = (torch.cat([(pool[l, at, h].view(torch.float8_e4m3fn).double() * scale[l, at, h].double()[:, None, None]).reshape(-1, case["head_dim"]),
                                   rest[l, b, h, :have % PAGE].double()])
                        for pool, scale, rest in ((s.page_k, s.scale_k, s.open_k), (s.page_v, s.scale_v, s.open_v)))
                for i in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    rows = slice(s.q_off[b], s.q_off[b] + n)
                    out[l, i, rows], lse[l, i, rows] = _exact_rows(s.q[l, i, rows].double(), k, v, limits)
    return {"out": out, "lse": lse}
