"""Batches of the decoding calls that are large, wide, empty or have holes: more requests than a block has threads,
vocabularies of more pieces than a wave has lanes, masks of many words, missing pages of every size."""
import numpy as np
import pytest
import torch

from paper_2606_05875_amd import qcf
from paper_2606_05875_amd.draft import DraftStep, PagedCache
from test_gpu_decode import Batch, _verify, host, i32, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,top,most", [(300, 3, None), (700, 2, None), (300, 14, None), (300, 25, None), (530, 40, 140000)])
def test_attention_of_many_requests(batch, top, most, dtype):
    """More requests than threads, many without new rows, a few long ones: shares begin anywhere among them."""
    say("attention of many requests", batch, top, most, dtype)
    rng = np.random.default_rng(51)
    new = np.where(rng.random(batch) < 0.8, 0, rng.integers(0, 3, batch))
    new[[0, batch // 2, batch - 3]] = top
    kv = np.where(rng.random(batch) < 0.5, 0, rng.integers(0, 70, batch))
    kv[[0, 17, batch // 2, batch - 3]] = 2200, 2300, 700, 1
    x = Batch([int(v) for v in kv], [int(v) for v in new], 8, 2, 64, dtype, 16, True, seed=52)
    g = dict(max_kv=most) if most else {}
    a, b = x.call(**g), x.call(**g)
    x.check(*a)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_without_new_rows(dtype):
    say("attention without new rows", dtype)
    for kv, most in (([5, 0, 90], 100), ([3000, 7], 3000)):
        x = Batch(kv, [0] * len(kv), 8, 2, 64, dtype, 16, False, seed=53)
        x.check(*x.call(max_q=4, max_kv=most))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_of_many_words(dtype):
    """More than 1024 rows with a mask; words behind the rows' own; fewer words than rows (the rest is not seen)."""
    say("masks of many words", dtype)
    x = Batch([40], [1100], 2, 1, 64, dtype, 32, "random", seed=54)
    x.check(*x.call())
    x = Batch([100, 0], [9, 40], 4, 2, 128, dtype, 16, True, seed=55, words=6)
    x.check(*x.call())
    x.mask = x.mask[:, :1].contiguous()
    see = [s.copy() for s in x.see]
    see[1][:, 32:] = False
    x.check(*x.call(), see=see)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [1, 4, 32, 256])
@pytest.mark.parametrize("hq,new", [(8, 2), (8, 13), (16, 15), (16, 30)])
def test_missing_pages_of_every_size(ps, hq, new, dtype):
    say("missing pages", ps, hq, new, dtype)
    x = Batch([900, 2500], [new, 1], hq, 2, 64, dtype, ps, True, seed=56)
    rng = np.random.default_rng(57)
    t, see = x.table_h.copy(), [s.copy() for s in x.see]
    for b in range(2):
        pages = -(-x.end[b] // ps)
        for p in rng.permutation(pages)[:max(1, pages // 5)]:
            t[b, p] = (-1, 2 ** 30)[int(p) % 2]
            see[b][:, p * ps:(p + 1) * ps] = False
    x.check(*x.call(table=i32(t)), see=see)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft,tree", [(False, False), (True, True), (False, True), (True, False)])
def test_verify_large_vocabularies(dtype, draft, tree):
    """More than 64 pieces of 4096 tokens; numbers near 0 and 1 draw from the first and the last of them."""
    say("verify large vocabularies", dtype, draft, tree)

    def ends(t, dr, tokens, u, un, parents, cu):
        un[:] = (2.0 ** -20, 0.5, 1 - 2.0 ** -20)
    for vocab, pad in ((262137, 0), (262145, 3), (600001, 5)):
        _verify([1, 3, 2], vocab, dtype, draft, tree, seed=vocab, pad=pad, spare=0)
        _verify([1, 3, 2], vocab, dtype, draft, tree, seed=vocab + 1, pad=pad, spare=0, mutate=ends)


def test_a_pass_without_rows():
    """No request brings a row: nothing changes."""
    say("a pass without rows")
    cache = PagedCache(2, 8, 16, 2, 64, 3, 4)
    s = DraftStep(cache, 6, 2, 4, qcf.rope_frequencies(64, 1e4))
    s.plan(i32([2, 0, 1]))
    s.commit(all_rows=True)
    before = [t.clone() for t in (cache.kv_len, cache.pages_held, cache.free_head, cache.block_table, *cache.k, *cache.v)]
    s.out.fill_(7.0)
    for parents in (None, i32([-1] * 6)):
        s.plan(i32([0, 0, 0]), parents)
        one = torch.ones((6, 4, 64), device="cuda").bfloat16()
        for layer in range(2):
            s.store(layer, one, one[:, :2].contiguous(), one[:, 2:].contiguous())
            s.attend(layer)
        x = torch.full((6, 5), 0.2, device="cuda")
        s.verify(x, i32([0] * 6), x[:, 0].contiguous(), x[:3, 0].contiguous(), parents=parents)
        s.commit()
        assert (s.n_out == 0).all() and (s.path == -1).all() and (s.tokens_out == -1).all() and (s.out == 7.0).all()
    for a, b in zip(before, (cache.kv_len, cache.pages_held, cache.free_head, cache.block_table, *cache.k, *cache.v)):
        bits = lambda t: t.contiguous().view(torch.int16)       # (slots without a token may hold NaN)
        assert torch.equal(bits(a), bits(b))
