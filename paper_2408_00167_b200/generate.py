"""Generation from compressed documents: a paged 8-bit cache that starts with a document's kept rows and grows token by token.

"Compression Output" of Finch (Section "Method") hands the compressed cache to the generation stage; this module is its
memory side.  It only orchestrates, as the chunk loop of document.py does: buffers, the page table, metadata and one library
call each for moving a compressed cache in, for a layer's new keys and values, and for a layer's attention.  The model's own
products stay with the caller:

    cache.fill(doc)                          # the kept rows of all layers, from a DocumentCompressor
    for token in ...:
        cache.step()                         # one more token for every request
        for layer in ...:
            finch_rotate(...)                # the layer's queries (and keys, if no rope was given to the cache)
            cache.append(layer, k, v)
            cache.attend(layer, q, out)

Kept keys are embedded at their slots when the compressor re-rotates them (its rope_theta), and `rope` embeds new keys at the
positions behind them.
"""
from __future__ import annotations

from typing import Optional

import numpy as np

from . import binding as fb
from .document import DocumentCompressor


class PagedCache:
    """The paged cache of a batch of requests with room for `max_tokens` tokens each.

    Every request owns as many pages as that takes; `len` is the host's count of its tokens, `pages` the library's
    description (its tensors are those that this object holds)."""

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: int, batch: int, max_tokens: int,
                 max_step: int = 1, scale: float = 0.0, rope: Optional[fb.finch_rope] = None, device="cuda"):
        import torch
        self.torch, self.device, self.rope = torch, fb.device_of(device), rope
        device = self.device
        self.L, self.Hq, self.Hkv, self.d, self.B = n_layers, n_q_heads, n_kv_heads, head_dim, batch
        self.max_tokens, self.max_step = max_tokens, max(max_step, 1)
        width = -(-max_tokens // fb.FINCH_PAGE_TOKENS)
        tdtype = torch.float32 if dtype == fb.FINCH_F32 else torch.bfloat16
        page = (fb.FINCH_PAGE_TOKENS, head_dim)
        codes = lambda: torch.zeros((n_layers, batch * width, n_kv_heads, *page), dtype=torch.uint8, device=device)
        scales = lambda: torch.zeros((n_layers, batch * width, n_kv_heads), dtype=torch.float32, device=device)
        rows = lambda: torch.zeros((n_layers, batch, n_kv_heads, *page), dtype=tdtype, device=device)
        self._tensors = [codes(), codes(), scales(), scales(), rows(), rows()]
        self.table = torch.arange(batch * width, dtype=torch.int32, device=device).reshape(batch, width)
        self.slot = torch.arange(batch, dtype=torch.int32, device=device)
        self.pages = fb.make_pages(*self._tensors, self.table, self.slot)
        # a layer's calls see that layer's part of every array
        self._of_layer = [fb.make_pages(*(t[l:l + 1] for t in self._tensors), self.table, self.slot) for l in range(n_layers)]
        bounds = dict(max_batch=max(batch, 1), max_prompt=self.max_step, max_candidates=max(max_tokens, 1), device=device.index or 0)
        self._ctx_all = fb.finch_ctx_create(n_layers, n_q_heads, n_kv_heads, head_dim, dtype, scale=scale, **bounds)
        self._ctx = fb.finch_ctx_create(1, n_q_heads, n_kv_heads, head_dim, dtype, scale=scale, **bounds)
        self.len = np.zeros(batch, dtype=np.int32)
        self._add = self._see = None
        self._ws = torch.empty(fb.finch_pages_workspace_bytes(self._ctx, fb.make_paged_batch(self.len, device="cpu")),
                               dtype=torch.uint8, device=device)
        self._made_on = self._step_on = self._stream()   # the streams that the arrays above and a step's description belong to
        self._readers = set()                            # other streams that have read the arrays above
        self._steps, self._has = 0, [0] * n_layers      # steps since the cache was filled, and those whose rows a layer has

    def close(self) -> None:
        for name in ("_ctx", "_ctx_all"):
            ctx = getattr(self, name, None)
            setattr(self, name, None)
            if ctx:
                fb.finch_ctx_destroy(ctx)

    def status(self) -> int:
        """Waits for the stream; the status words of both contexts, 0 = clean."""
        return fb.finch_device_status(self._ctx) | fb.finch_device_status(self._ctx_all)

    def fill(self, doc: DocumentCompressor) -> None:
        """The compressed caches of `doc` become the requests' first tokens, all layers, one call for each request (a request's
        kept rows need not fill its part of the compressor's buffers).  Nothing is rotated: kept keys stand at their slots.

        Waits for the compressor's steps: its lengths on the host are a prediction, and rows of a step that the device refused do
        not exist.  Raises RuntimeError then, as DocumentCompressor.verify does."""
        doc.verify()
        if (doc.L, doc.Hkv, doc.d, doc.B) != (self.L, self.Hkv, self.d, self.B):
            raise ValueError("PagedCache.fill: another model or batch")
        if int(doc.cache_len.max(initial=0)) > self.max_tokens:
            raise ValueError(f"PagedCache.fill: {int(doc.cache_len.max())} tokens, room for {self.max_tokens}")
        for b in range(self.B):
            n, at = int(doc.cache_len[b]), int(doc.cache_off[b])
            one = fb.make_pages(*self._tensors, self.table[b:b + 1], self.slot[b:b + 1])
            batch = fb.make_paged_batch([0], new_off=[0, n], device=self.device)
            self._read_here(batch, self._stream())
            fb.finch_pages_append(self._ctx_all, one, batch, doc.cache_k[:, :, at:at + n], doc.cache_v[:, :, at:at + n])
        self.len = doc.cache_len.astype(np.int32).copy()
        self._add = self._see = None
        self._steps, self._has = 0, [0] * self.L

    def step(self, tokens: int = 1) -> None:
        """`tokens` more of every request: appends and attention of all layers follow, then the next step."""
        if not 1 <= tokens <= self.max_step:
            raise ValueError(f"PagedCache.step: {tokens} tokens, 1 to {self.max_step} (max_step) can be one step")
        if int(self.len.max(initial=0)) + tokens > self.max_tokens:
            raise ValueError(f"PagedCache.step: room for {self.max_tokens} tokens")
        off = np.arange(self.B + 1, dtype=np.int32) * tokens
        self._step_on = self._stream()
        self._add = fb.make_paged_batch(self.len, new_off=off, device=self.device)
        self.len = self.len + np.int32(tokens)
        self._see = fb.make_paged_batch(self.len, q_off=off, device=self.device)
        self._steps += 1

    def _stream(self):
        return fb._stream(None) if self.device.type == "cuda" else None

    def _read_here(self, batch, made_on) -> None:
        """A step's description is replaced by the next one's, and everything goes when the cache does: memory that the current stream's
        kernels read, where it was allocated for another stream, waits for them before it serves another purpose."""
        now, held = self._stream(), ()
        if now != made_on:
            held = batch.q_off, batch.new_off, batch.len
        if now != self._made_on and now not in self._readers:      # once is for good
            self._readers.add(now)
            held += *self._tensors, self.table, self.slot, self._ws
        for t in held:
            if t is not None:
                t.record_stream(self.torch.cuda.current_stream())

    def _check_rows(self, what: str, t, heads: int) -> None:
        if t.shape != (1, heads, self._add.c.total_new, self.d):
            raise ValueError(f"PagedCache.{what}: expected rows {(1, heads, self._add.c.total_new, self.d)}, got {tuple(t.shape)}")

    def append(self, layer: int, k, v) -> None:
        """The step's new rows of a layer, [1][n_kv_heads][batch * tokens][head_dim], requests one behind the other; once a step (a
        second time open rows would be read that the first has moved on)."""
        if self._add is None:
            raise ValueError("PagedCache.append: no step has been begun")
        if self._has[layer] != self._steps - 1:
            raise ValueError(f"PagedCache.append: layer {layer} has the rows of {self._has[layer]} steps, this is step {self._steps}")
        self._check_rows("append", k, self.Hkv)
        self._check_rows("append", v, self.Hkv)
        self._read_here(self._add, self._step_on)
        fb.finch_pages_append(self._ctx, self._of_layer[layer], self._add, k, v, rope=self.rope)
        self._has[layer] = self._steps

    def attend(self, layer: int, q, out, row_lse=None) -> None:
        """Attention of the step's query rows, [1][n_q_heads][batch * tokens][head_dim], over the layer's cache, the step's rows among
        it."""
        if self._see is None:
            raise ValueError("PagedCache.attend: no step has been begun")
        if self._has[layer] != self._steps:
            raise ValueError(f"PagedCache.attend: layer {layer} has the rows of {self._has[layer]} steps, this is step {self._steps}")
        self._check_rows("attend", q, self.Hq)
        self._read_here(self._see, self._step_on)
        fb.finch_pages_attend(self._ctx, self._of_layer[layer], self._see, q, out, row_lse, ws=self._ws)
