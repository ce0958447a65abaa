"""Answering from fused caches: the decoding calls together, over several passes, against the float64
oracle; and captured into a graph."""
import math

import numpy as np
import pytest
import torch

from oracle import decode as D
from paper_2606_05875_amd import qcf
from paper_2606_05875_amd.draft import DraftStep, PagedCache
from paper_2606_05875_amd.step import FusionStep
from paper_2606_05875_amd.workloads import make_workload
from test_gpu_decode import DT, HALF, host, i32, random_parents, say, within

pytestmark = pytest.mark.gpu


def token_rows(cache, b, n):
    """Slots of request b's first n tokens."""
    t = cache.block_table[b].cpu().numpy().astype(np.int64)
    j = np.arange(n)
    return t[j // cache.page_size] * cache.page_size + j % cache.page_size


class Inputs:
    """One pass's random inputs of fixed sizes."""

    def __init__(self, rng, B, max_new, rows, hq, hkv, d, dtype, vocab, tree, draft):
        self.new = rng.integers(0, max_new + 1, B)
        self.new[rng.integers(B)] = max_new
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        par = np.full(rows, -1, np.int32)
        par[:self.cu[-1]] = random_parents(rng, self.new, 3)
        for a, m in zip(self.cu, self.new):                     # one root per request
            par[a + 1:a + m] = np.maximum(par[a + 1:a + m], 0)
        self.parents_h = par
        self.parents = i32(par) if tree else None
        t = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(DT[dtype]).cuda()
        qkv = t(rows, (hq + 2 * hkv) * d)
        q, k, v = qkv.split([hq * d, hkv * d, hkv * d], 1)
        self.q, self.k, self.v = q.view(rows, hq, d), k.view(rows, hkv, d), v.view(rows, hkv, d)
        self.new_len = i32(self.new)
        z = 2 * torch.from_numpy(rng.standard_normal((rows, vocab))).cuda()
        self.target = torch.softmax(z, 1).float()
        self.draft = torch.softmax(z + 0.5 * torch.from_numpy(rng.standard_normal((rows, vocab))).cuda(), 1).float() if draft else None
        up = par if tree else np.concatenate([np.arange(-1, m - 1) for m in self.new] + [np.full(rows, -1)])[:rows]
        base = np.repeat(self.cu[:-1], self.new)
        tok = rng.integers(0, vocab, rows)
        top = torch.argsort(self.target, 1, descending=True).cpu().numpy()
        for r in range(self.cu[-1]):                            # likely children of the row's parent
            tok[r] = top[base[r] + max(up[r], 0), rng.integers(0, 3)]
        self.tokens_h, self.tokens = tok, i32(tok)
        self.u_h = rng.random(rows).astype(np.float32) * np.float32(0.3)
        self.un_h = rng.random(B).astype(np.float32)
        self.u, self.un = torch.from_numpy(self.u_h).cuda(), torch.from_numpy(self.un_h).cuda()


@pytest.mark.parametrize("dtype,tree,draft,interleaved,rotary", [
    ("bf16", True, False, False, 128), ("bf16", False, True, True, 64), ("f32", True, True, True, 48),
    ("f32", False, False, False, 64)])
def test_answering_from_fused_caches(dtype, tree, draft, interleaved, rotary):
    say("answering from fused caches", dtype, tree, draft, interleaved, rotary)
    name, kw = (("c2", dict(chunk_lens=[[150, 77], [40], [129, 1, 60]], q_lens=[9, 20, 5], anchors_per_chunk=3))
                if dtype == "bf16" else ("c1", {}))
    w = make_workload(name, **kw)
    step = FusionStep(w)
    step.run()
    B, hq, hkv, d, vocab, max_new, layers = w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, 501, 9, 2
    lens = np.diff(w.cu_kv)
    ps, max_pages = 16, 60
    cache = PagedCache(layers, B * max_pages, ps, hkv, d, B, max_pages, DT[dtype])
    rng = np.random.default_rng(1)
    cache.free_pages.copy_(i32(rng.permutation(B * max_pages)))
    freq = qcf.rope_frequencies(rotary, 1e4, scaling="by_parts", factor=4.0, trained_len=256)
    # the fused caches move into pages
    move = DraftStep(cache, int(lens.sum()) + 3, int(lens.max()), hq, freq)
    move.plan(i32(lens))
    for layer in range(layers):
        move.fill(layer, step.k, step.v, i32(np.arange(w.n_rows)))
    move.commit(all_rows=True)
    kept = [[(host(step.k)[a:z], host(step.v)[a:z]) for a, z in zip(w.cu_kv[:-1], w.cu_kv[1:])] for _ in range(layers)]
    rows = B * max_new + 4
    s = DraftStep(cache, rows, max_new, hq, freq, interleaved=interleaved, magnitude=1.1)
    lengths = lens.astype(np.int64).copy()
    grown = 0
    for turn in range(5):
        x = Inputs(rng, B, max_new, rows, hq, hkv, d, dtype, vocab, tree, draft)
        s.plan(x.new_len, x.parents)
        outs = []
        for layer in range(layers):
            s.store(layer, x.q, x.k, x.v)
            s.out.fill_(7.0)
            outs.append(host(s.attend(layer)))
        s.verify(x.target, x.tokens, x.u, x.un, draft=x.draft, parents=x.parents)
        n = int(x.cu[-1])
        np.testing.assert_array_equal(s.cu.cpu().numpy(), x.cu)
        depth = np.array([0 if i == x.cu[b] else -1 for b in range(B) for i in range(x.cu[b], x.cu[b + 1])])
        for b in range(B):
            for i in range(x.cu[b] + 1, x.cu[b + 1]):
                depth[i] = depth[x.cu[b] + x.parents_h[i]] + 1 if tree else i - x.cu[b]
        pos = depth + np.repeat(lengths, x.new)
        np.testing.assert_array_equal(s.positions.cpu().numpy()[:n], pos)
        fr = freq.cpu().numpy()
        kr, ksize = D.rope(host(x.k)[:n], pos, fr, interleaved, 1.1)
        qr = host(s.q)[:n]
        w_q, qsize = D.rope(host(x.q)[:n], pos, fr, interleaved, 1.1)
        within(qr, w_q, HALF[dtype] * np.abs(w_q) + 4 * 2.0 ** -24 * qsize, "queries")
        used = []
        for b in range(B):
            a, z, m, L = x.cu[b], x.cu[b + 1], x.new[b], int(lengths[b])
            slot = token_rows(cache, b, L + m)
            used += list(slot)
            np.testing.assert_array_equal(s.slots.cpu().numpy()[a:z], slot[L:])
            see = D.chain_see(m, L)
            if tree:
                see[:, L:] = False
                for i in range(m):
                    up = i
                    while up >= 0:
                        see[i, L + up] = True
                        up = x.parents_h[a + up]
            wp, wt = D.verify(host(x.target)[a:z], host(x.draft)[a:z] if draft else None, x.tokens_h[a:z],
                              x.parents_h[a:z] if tree else None, x.u_h[a:z], x.un_h[b])
            assert int(s.n_out[b]) == len(wp)
            np.testing.assert_array_equal(s.path[b].cpu().numpy(), wp + [-1] * (max_new - len(wp)))
            np.testing.assert_array_equal(s.tokens_out[b].cpu().numpy(), wt + [-1] * (max_new - len(wt)))
            for layer in range(layers):
                K, V = host(cache.k[layer])[slot], host(cache.v[layer])[slot]
                np.testing.assert_array_equal(K[:L], kept[layer][b][0])
                np.testing.assert_array_equal(V[:L], kept[layer][b][1])
                within(K[L:], kr[a:z], HALF[dtype] * np.abs(kr[a:z]) + 4 * 2.0 ** -24 * ksize[a:z], "keys")
                np.testing.assert_array_equal(V[L:], host(x.v)[a:z])
                if m:
                    want, lse, absv, absx = D.tree_attention(qr[a:z], K, V, see, s.scale)
                    off = d * 2.0 ** -24 * absx + 3 * 2.0 ** -23 * (np.abs(lse) + absx) + (L + m + 16) * 2.0 ** -24
                    within(outs[layer][a:z], want, HALF[dtype] * np.abs(want) + (2 * off + (2.0 ** -8 if dtype == "bf16" else 0))[..., None] * absv,
                           f"request {b} layer {layer}")
                keep = np.concatenate([np.arange(L), L + np.array(wp, np.int64)])
                kept[layer][b] = (K[keep], V[keep])
            grown += len(wp)
            lengths[b] += len(wp)
        assert len(set(used)) == len(used)                      # no slot belongs to two tokens
        assert all((o[n:] == 7.0).all() for o in outs)          # rows behind the last request
        s.commit()
        np.testing.assert_array_equal(cache.kv_len.cpu().numpy(), lengths)
        assert int(cache.free_head[0]) == int(cache.pages_held.sum()) == int((cache.block_table >= 0).sum())
    assert grown > 5 * B                                        # drafts were accepted
    for layer in range(layers):                                 # after the last move
        for b in range(B):
            slot = token_rows(cache, b, int(lengths[b]))
            np.testing.assert_array_equal(host(cache.k[layer])[slot], kept[layer][b][0])
            np.testing.assert_array_equal(host(cache.v[layer])[slot], kept[layer][b][1])


def test_a_pass_in_a_graph():
    """Plan to commit captured once and replayed with new inputs in place: the same state and outputs as eager
    passes from the same start, which run in between."""
    say("a draft pass in a graph")
    B, hq, hkv, d, vocab, max_new, ps = 4, 8, 2, 128, 700, 6, 32
    rows = B * max_new + 2
    freq = qcf.rope_frequencies(d, 1e4)

    def start():
        rng = np.random.default_rng(5)
        cache = PagedCache(1, 200, ps, hkv, d, B, 40)
        for x in (cache.k[0], cache.v[0]):
            x.copy_(torch.from_numpy(rng.standard_normal(x.shape)))
        cache.free_pages.copy_(i32(rng.permutation(200)))
        s = DraftStep(cache, rows, max_new, hq, freq)
        m = DraftStep(cache, 1000, 500, hq, freq)
        m.plan(i32([300, 500, 3, 0]))
        m.commit(all_rows=True)
        return cache, s

    def one(s, x):
        s.plan(x.new_len, x.parents)
        s.store(0, x.q, x.k, x.v)
        s.attend(0)
        s.verify(x.target, x.tokens, x.u, x.un, parents=x.parents)
        s.commit()

    rng = np.random.default_rng(6)
    feed = [Inputs(rng, B, max_new, rows, hq, hkv, d, "bf16", vocab, True, False) for _ in range(5)]
    buf = Inputs(rng, B, max_new, rows, hq, hkv, d, "bf16", vocab, True, False)
    eager_cache, eager = start()
    warm_cache, warm = start()
    cache, s = start()
    one(warm, buf)                                              # (loads the kernels)
    s.ws_verify = torch.empty_like(warm.ws_verify)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        one(s, buf)
    for turn, x in enumerate(feed):
        for name in ("q", "k", "v", "target", "tokens", "u", "un", "parents", "new_len"):
            getattr(buf, name).copy_(getattr(x, name))
        g.replay()
        torch.cuda.synchronize()
        one(eager, x)
        torch.cuda.synchronize()
        n = int(x.cu[-1])
        for name in ("slots", "positions", "cu", "n_out", "path", "tokens_out", "mask"):
            assert torch.equal(getattr(s, name), getattr(eager, name)), (turn, name)
        assert torch.equal(s.out[:n], eager.out[:n]), turn
        for name in ("block_table", "kv_len", "pages_held", "free_head"):
            assert torch.equal(getattr(cache, name), getattr(eager_cache, name)), (turn, name)
        assert torch.equal(cache.k[0], eager_cache.k[0]) and torch.equal(cache.v[0], eager_cache.v[0]), turn


def test_verify_takes_the_plans_parents():
    cache = PagedCache(1, 8, 16, 2, 64, 2, 4)
    s = DraftStep(cache, 8, 4, 4, qcf.rope_frequencies(64, 1e4))
    s.plan(i32([2, 3]))
    x = torch.zeros((8, 5), device="cuda")
    with pytest.raises(qcf.QcfError):
        s.verify(x, i32([0] * 8), x[:, 0].contiguous(), x[:2, 0].contiguous(), parents=i32([-1] * 8))
