"""Further turns on paged caches: questions that follow an answer, several answers from one cache, requests that end.

``TurnCache`` is a ``PagedCache`` whose requests may continue one another, be taken back and end;
``TurnStep`` is a pass of new rows over it, as ``DraftStep`` is, for models that norm their queries and keys,
for chunks of many rows (a question, a prompt), for layers with a window, and with the step from logits to the
probabilities that drafted tokens are verified against:

  plan    qcf_page_plan
  per layer:
    store   qcf_norm_rope_store (qcf_rope_store without norms)
    attend  qcf_chunk_attn (qcf_tree_attn for drafted trees and few rows)
  shape   qcf_shape_logits       penalties, biases, a grammar's mask, temperature
  verify, commit                 as in DraftStep

Nothing waits for the GPU, and every buffer stays where it is, so that a pass can be captured into a graph and
replayed.
"""
from __future__ import annotations

import torch

from . import qcf
from .draft import DraftStep, PagedCache

__all__ = ["TurnCache", "TurnStep"]

# Query vectors per KV head (rows times the heads that share it) up to which qcf_tree_attn takes a pass: it reads the
# whole rectangle, but its units hold fewer vectors and its work begins faster.  Over 2000 to 8000 tokens, 16 requests,
# 32/8 heads of 128, us: 64 vectors 79 / 80 with qcf_chunk_attn, 128 91 / 95, 256 128 / 125, 512 233 / 214; one request of
# 30000 tokens, 64/8 heads: 128 vectors 41 / 62, 256 55 / 61.
FEW_VECTORS = 256


class TurnCache(PagedCache):
    """Pages of ``n_layers`` layers for up to ``batch`` requests, which may share pages.  ``pages_missing``: pages that the
    last change of requests, and the passes since the one before, asked for when none was free (their tokens
    are not seen); after a change ``free_head`` counts what is free again."""

    def __init__(self, n_layers, n_pages, page_size, n_kv_heads, head_dim, batch, max_pages,
                 dtype=torch.bfloat16, device="cuda"):
        super().__init__(n_layers, n_pages, page_size, n_kv_heads, head_dim, batch, max_pages, dtype, device)
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=self.device)
        self._pools = qcf.PoolSet(self.k + self.v)
        self._table, self._kv, self._held, self._head = i32(batch, max_pages), i32(batch), i32(batch), i32(1)
        self._head_after, self.pages_missing = i32(1), i32(1)
        self._copy_src, self._copy_dst, self._copy_rows = i32(batch), i32(batch), i32(batch)
        self._itself = torch.arange(batch, dtype=torch.int32, device=self.device)
        need = qcf.qcf_page_release_workspace_size(batch, max_pages, n_pages)
        self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)

    def continue_from(self, source, keep_len=None):
        """Request b becomes a continuation of request source[b] (int32; itself, another's, or -1: it ends) at its
        first keep_len[b] tokens (all of them without keep_len).  Full pages are shared, started ones
        copied in every layer, and pages that no request holds any more become free, pages beyond the tokens
        (rejected drafts) among them; the copies' pages are taken before."""
        qcf.qcf_page_fork(self._table, self._kv, self._held, self.block_table, self.kv_len, source, self.free_pages,
                          self.page_size, self.n_pages, keep_len=keep_len, free_head=self.free_head,
                          free_head_out=self._head, copy_src=self._copy_src, copy_dst=self._copy_dst,
                          copy_rows=self._copy_rows)
        qcf.qcf_copy_pages(self._pools, self._copy_src, self._copy_dst, self.page_size, rows=self._copy_rows)
        qcf.qcf_page_release(self.block_table, self.pages_held, self._table, self._held, self.free_pages, self._head,
                             self._head_after, self.n_pages, workspace=self._ws)
        self.block_table.copy_(self._table)
        self.kv_len.copy_(self._kv)
        self.pages_held.copy_(self._held)
        self.free_head.copy_(self._head_after)
        torch.sub(self._head, self.n_pages, out=self.pages_missing).clamp_(min=0)

    def keep(self, keep_len):
        """Every request keeps its first keep_len[b] tokens (0: it ends)."""
        self.continue_from(self._itself, keep_len)


class TurnStep(DraftStep):
    """One pass of up to ``max_rows`` packed new rows, at most ``max_new`` per request, over a ``TurnCache`` (or
    a ``PagedCache``).

    ``q_norm``, ``k_norm``: each layer's weights of the norms per head ([head_dim] or [heads, head_dim]), with ``eps``;
    or None.  ``window``: tokens that rows see, the same for all layers or one per layer (0: all).
    ``shape``'s probabilities are ``target``, which ``verify`` takes."""

    def __init__(self, cache: PagedCache, max_rows, max_new, n_q_heads, freq, interleaved=False, magnitude=1.0,
                 scale=None, vocab=None, q_norm=None, k_norm=None, eps=1e-6, window=0):
        super().__init__(cache, max_rows, max_new, n_q_heads, freq, interleaved, magnitude, scale, vocab)
        n = len(cache.k)
        self.window = [int(window)] * n if isinstance(window, int) else [int(w) for w in window]
        if len(self.window) != n:
            raise qcf.QcfError("window needs one number, or one per layer")
        if (q_norm is None) != (k_norm is None) or (q_norm is not None and (len(q_norm) != n or len(k_norm) != n)):
            raise qcf.QcfError("q_norm and k_norm go together, with one weight per layer")
        self.q_norm, self.k_norm, self.eps = q_norm, k_norm, float(eps)
        group = n_q_heads // cache.n_kv_heads
        # few rows, and pages of fewer than 16, are the tree call's
        self.few = self.max_new * group <= FEW_VECTORS or cache.page_size < 16
        if cache.page_size < 16 and any(self.window):
            raise qcf.QcfError("layers with a window need pages of at least 16 rows")
        # (68 MB in bf16 at head size 128, whatever the sizes)
        self.ws_chunk = None
        if not self.few or any(self.window):
            need = qcf.qcf_chunk_attn_workspace_size(cache.batch, self.max_new, self.max_kv, n_q_heads,
                                                     cache.n_kv_heads, cache.head_dim, cache.dtype)
            self.ws_chunk = torch.empty(max(need, 256), dtype=torch.uint8, device=cache.device)
        self.target = self.ws_shape = None
        self._shaped = {}  # target and workspace of each vocabulary
        if vocab is not None:
            self._shaping(vocab)

    def _shaping(self, vocab):
        """Room for probabilities over ``vocab`` tokens; each vocabulary keeps its own, for a captured pass may write to it."""
        if vocab not in self._shaped:
            dev = self.cache.device
            need = qcf.qcf_shape_logits_workspace_size(self.max_rows, vocab)
            self._shaped[vocab] = (torch.zeros((self.max_rows, vocab), dtype=torch.float32, device=dev),
                                   torch.empty(max(need, 256), dtype=torch.uint8, device=dev))
        self.target, self.ws_shape = self._shaped[vocab]

    def store(self, layer, q, k, v):
        if self.q_norm is None:
            return super().store(layer, q, k, v)
        c, n = self.cache, q.shape[0]
        qcf.qcf_norm_rope_store(c.k[layer], c.v[layer], k, v, self.slots[:n], self.positions[:n], self.freq,
                                interleaved=self.interleaved, magnitude=self.magnitude, q_new=q, q_out=self.q[:n],
                                q_weight=self.q_norm[layer], k_weight=self.k_norm[layer], eps=self.eps)

    def attend(self, layer):
        window = self.window[layer]
        if self.tree and window:
            raise qcf.QcfError("a layer with a window takes chunks, not trees")
        if self.tree or (self.few and not window):
            return super().attend(layer)
        c = self.cache
        qcf.qcf_chunk_attn(self.out, self.q, self.cu, c.k[layer], c.v[layer], c.block_table, c.kv_len, c.page_size,
                           self.max_new, self.max_kv, self.scale, window=window, workspace=self.ws_chunk)
        return self.out

    def shape(self, logits, tokens=None, history=None, prompt_len=None, **shaping):
        """``target`` [max_rows, vocab] <- the probabilities of the model's logits [max_rows, vocab] after the planned
        rows: of all of them, for drafted tokens.  (After a question or a prompt, of which each request's last row
        alone is drawn from, qcf.qcf_shape_logits takes those rows, with the question in the history.)  ``tokens`` are the rows' tokens and ``history`` [batch, width] those of the requests' cached tokens, in
        their order, of which the first prompt_len[b] count as the prompt (so before ``commit``); the rest as
        qcf.qcf_shape_logits takes it (repetition, presence, frequency, bias_*, allowed, temperature)."""
        self._shaping(logits.shape[1])
        qcf.qcf_shape_logits(self.target, logits, self.cu, history=history, prompt_len=prompt_len,
                             hist_len=None if history is None else self.cache.kv_len, tokens=tokens,
                             tree_mask=self.mask if self.tree and tokens is not None else None, workspace=self.ws_shape,
                             **shaping)
        return self.target
