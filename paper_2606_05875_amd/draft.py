"""Answering from the fused caches: a paged cache and one pass of drafted tokens over it.

After the fusion step a request's cache is complete and its answer is decoded from it (Section 3.5, the
decode that follows the cache fusion).  ``PagedCache`` holds the layers' keys and values in pages with the
block tables and the free list on the GPU; ``DraftStep`` is one pass of the model's new rows over it, as a
stream-ordered chain of libqcf calls:

  plan    qcf_page_plan      pages, slots, positions and tree masks of the new rows
  per layer:
    store   qcf_rope_store   rotate the new rows' queries and keys, keys and values into their slots
    attend  qcf_tree_attn    the new rows over the pages
  verify  qcf_verify_drafts  which drafted tokens stay, and the next token
  commit  qcf_gather_rows + qcf_rope_store per layer: the rows that stay move to the front of the new
          rows' slots (trees only: a chain's are there already); the lengths grow

A fused cache moves in with ``plan`` (its lengths as new rows) and ``fill``.  Nothing waits for the GPU, and
every buffer stays where it is, so that a pass can be captured into a graph and replayed.
"""
from __future__ import annotations

import math

import torch

from . import qcf
from .step import kv_buffer

__all__ = ["PagedCache", "DraftStep"]


class PagedCache:
    """Pages of ``n_layers`` layers for up to ``batch`` requests of up to ``max_pages`` pages each."""

    def __init__(self, n_layers, n_pages, page_size, n_kv_heads, head_dim, batch, max_pages,
                 dtype=torch.bfloat16, device="cuda"):
        self.n_pages, self.page_size, self.batch, self.max_pages = n_pages, page_size, batch, max_pages
        self.n_kv_heads, self.head_dim, self.dtype, self.device = n_kv_heads, head_dim, dtype, torch.device(device)
        pool = lambda: kv_buffer(n_pages * page_size, n_kv_heads, head_dim, dtype, self.device)
        self.k = [pool() for _ in range(n_layers)]
        self.v = [pool() for _ in range(n_layers)]
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=self.device)
        self.block_table = i32(batch, max_pages).fill_(-1)
        self.kv_len, self.pages_held = i32(batch), i32(batch)
        self.free_pages = torch.arange(n_pages, dtype=torch.int32, device=self.device)
        self.free_head = i32(1)  # entries of free_pages before it are taken; above n_pages: they ran out


class DraftStep:
    """One pass of up to ``max_rows`` packed new rows, at most ``max_new`` per request.

    ``freq``: the model's rotary frequencies (qcf.rope_frequencies), with ``interleaved`` and ``magnitude`` as
    qcf_rope_store takes them.  ``vocab``: entries of the probabilities that verify takes; without it, and for more,
    the first such verify allocates their workspace.  Inputs of a pass are given to its stages and are only read
    by them."""

    def __init__(self, cache: PagedCache, max_rows, max_new, n_q_heads, freq, interleaved=False, magnitude=1.0,
                 scale=None, vocab=None):
        self.cache, self.max_rows, self.max_new = cache, int(max_rows), int(max_new)
        self.freq, self.interleaved, self.magnitude = freq, bool(interleaved), float(magnitude)
        d, hkv, dt, dev, B = cache.head_dim, cache.n_kv_heads, cache.dtype, cache.device, cache.batch
        self.scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=dev)
        self.slots, self.positions, self.cu = i32(max_rows), i32(max_rows), i32(B + 1)
        self.mask = i32(max_rows, (self.max_new + 31) // 32)
        self.kv_end, self._held, self._head = i32(B), i32(B), i32(1)
        self.q = torch.zeros((max_rows, n_q_heads, d), dtype=dt, device=dev)
        self.out = torch.zeros((max_rows, n_q_heads, d), dtype=dt, device=dev)
        self.max_kv = cache.max_pages * cache.page_size
        need = qcf.qcf_tree_attn_workspace_size(B, self.max_new, self.max_kv, n_q_heads, hkv, d, dt)
        self.ws_attn = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        self.n_out, self.path, self.tokens_out = i32(B), i32(B, self.max_new), i32(B, self.max_new)
        self.move_src, self.move_dst = i32(B, self.max_new), i32(B, self.max_new)
        self.ws_verify, self._outgrown = None, []
        if vocab is not None:
            self._room(vocab)
        self.k_move, self.v_move = (torch.zeros((B * self.max_new, hkv, d), dtype=dt, device=dev) for _ in range(2))
        self.tree = False

    def _room(self, vocab):
        """ws_verify for ``vocab``; one that became too small is kept, for a captured pass may write to it."""
        need = max(qcf.qcf_verify_drafts_workspace_size(self.cache.batch, vocab), 256)
        if self.ws_verify is None or self.ws_verify.numel() < need:
            self._outgrown.append(self.ws_verify)
            self.ws_verify = torch.empty(need, dtype=torch.uint8, device=self.cache.device)

    def plan(self, new_len, parents=None):
        """Pages and slots for ``new_len`` rows of each request: drafted trees (``parents``, see
        qcf_page_plan), or chains, single tokens, prompts.  The pages are taken at once."""
        c = self.cache
        self.tree = parents is not None
        qcf.qcf_page_plan(c.block_table, c.kv_len, new_len, c.free_pages, self.slots, self.positions, self.cu,
                          c.page_size, c.n_pages, self.max_new, pages_held=c.pages_held, free_head=c.free_head,
                          kv_end=self.kv_end, pages_held_out=self._held, free_head_out=self._head,
                          parents=parents, tree_mask=self.mask if self.tree else None)
        c.pages_held.copy_(self._held)
        c.free_head.copy_(self._head)

    def fill(self, layer, k, v, rows):
        """Keys and values as they are (a fused cache's) into the planned slots: slot of packed row i
        gets row ``rows[i]`` of k and v; packed rows beyond len(rows) are not filled."""
        c = self.cache
        qcf.qcf_rope_store(c.k[layer], c.v[layer], k, v, self.slots[:rows.numel()], src_idx=rows)

    def store(self, layer, q, k, v):
        """The new rows' projections [rows, heads, head_dim] (rows of max_rows, dense or strided): queries
        turned into ``self.q``, keys turned and values into the layer's pages."""
        c = self.cache
        n = q.shape[0]
        qcf.qcf_rope_store(c.k[layer], c.v[layer], k, v, self.slots[:n], self.positions[:n], self.freq,
                           interleaved=self.interleaved, magnitude=self.magnitude, q_new=q, q_out=self.q[:n])

    def attend(self, layer):
        """Attention of the stored rows over the layer's pages; returns [max_rows, H_q, head_dim]
        (rows behind the batch's last are left as they were)."""
        c = self.cache
        qcf.qcf_tree_attn(self.out, self.q, self.cu, c.k[layer], c.v[layer], c.block_table, c.kv_len, c.page_size,
                          self.max_new, self.max_kv, self.scale, tree_mask=self.mask if self.tree else None,
                          workspace=self.ws_attn)
        return self.out

    def verify(self, target, tokens, u_accept, u_next, draft=None, parents=None):
        """Accepted rows (``path``), their tokens and the next one (``tokens_out``), ``n_out`` per request;
        ``parents`` as given to plan."""
        if (parents is not None) != self.tree:
            raise qcf.QcfError("verify takes the parents that plan was given")
        self._room(target.shape[1])
        qcf.qcf_verify_drafts(self.n_out, self.path, self.tokens_out, target, tokens, self.cu, u_accept, u_next,
                              draft=draft, parents=parents, slots=self.slots, move_src=self.move_src,
                              move_dst=self.move_dst, workspace=self.ws_verify)

    def commit(self, all_rows=False):
        """The rows that verify accepted become part of the requests (or, with ``all_rows``, every
        planned row: prompts, fused caches, tokens that need no check)."""
        c = self.cache
        if all_rows:
            c.kv_len.copy_(self.kv_end)
            return
        if self.tree:
            src, dst = self.move_src.view(-1), self.move_dst.view(-1)
            for k, v in zip(c.k, c.v):
                # out of the slots first: a row's slot may be another's destination
                qcf.qcf_gather_rows(self.k_move, k, src)
                qcf.qcf_gather_rows(self.v_move, v, src)
                qcf.qcf_rope_store(k, v, self.k_move, self.v_move, dst)
        c.kv_len.add_(self.n_out)
