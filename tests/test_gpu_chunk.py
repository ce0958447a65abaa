"""Attention of a chunk of new rows over a paged cache (qcf_chunk_attn) against the float64 oracle, with the
tolerances of test_gpu_decode: every row up to its own token, or a window of the last ones."""
import math

import numpy as np
import pytest
import torch

from oracle import turns as T
from paper_2606_05875_amd import qcf
from test_gpu_decode import DT, GEO, Batch, host, i32, say

pytestmark = pytest.mark.gpu


class Chunk(Batch):
    def __init__(self, kv, new, hq, hkv, d, dtype, ps, window=0, **kw):
        super().__init__(kv, new, hq, hkv, d, dtype, ps, False, **kw)
        self.window = window
        self.see = [T.chunk_see(m, k, window) for m, k in zip(new, kv)]

    def call(self, out=None, lse=None, ws=None, **kw):
        out = torch.full_like(self.q, 5.0) if out is None else out
        lse = torch.full(self.q.shape[:2], 5.0, device="cuda") if lse is None else lse
        g = dict(max_q=self.max_q, max_kv=self.max_kv, table=self.table)
        g.update(kw)
        qcf.qcf_chunk_attn(out, self.q, i32(self.cu), self.k, self.v, g["table"], i32(self.kv), self.ps, g["max_q"],
                           g["max_kv"], self.scale, window=self.window, lse=lse, workspace=ws)
        return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", GEO)
@pytest.mark.parametrize("window", [0, 1, 50])
def test_chunk_attn(dtype, hq, hkv, d, window):
    say("chunk attention", dtype, hq, hkv, d, window)
    for i, (kv, new, ps) in enumerate(((
            [0, 1, 31, 32, 33, 63, 64, 65, 127, 200], [1, 2, 3, 1, 5, 8, 1, 4, 9, 7], 16),
            ([300, 5, 0], [1, 1, 1], 32), ([130, 0, 17], [33, 0, 64], 16), ([0], [140], 64), ([500, 40], [8, 16], 128))):
        x = Chunk(kv, new, hq, hkv, d, dtype, ps, window, seed=i, pad=(0, d, 8, 0, 16)[i], q_scale=(1.5, 1.5, 4.0, 1.5, 0.2)[i])
        x.check(*x.call())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv,new,hq,hkv,d,ps,window", [
    ([9000], [1], 8, 2, 64, 16, 0), ([5000, 100, 0, 2500], [3, 1, 200, 40], 8, 2, 128, 64, 0), ([0], [700], 4, 1, 128, 16, 0),
    ([3000, 2000], [140, 30], 8, 2, 128, 16, 300), ([2100], [65], 16, 4, 64, 32, 64), ([33, 1500], [270, 130], 8, 4, 64, 16, 1000),
    ([0, 900], [500, 300], 2, 2, 128, 128, 129), ([4000], [77], 32, 1, 64, 16, 33), ([0], [1000], 2, 1, 64, 16, 2000)])
def test_chunk_attn_long(dtype, kv, new, hq, hkv, d, ps, window):
    """Tiles that are cut over blocks, chunks of several tiles; twice over a dirty workspace: the same bits."""
    say("chunk attention long", dtype, kv, new, hq, hkv, d, ps, window)
    x = Chunk(kv, new, hq, hkv, d, dtype, ps, window, seed=5)
    x.check(*x.call())
    need = qcf.qcf_chunk_attn_workspace_size(len(kv), x.max_q, x.max_kv, hq, hkv, d, DT[dtype])
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    a, b = x.call(ws=ws), x.call(ws=ws)
    x.check(*a)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    # larger bounds than the batch needs: within the same tolerances
    x.check(*x.call(max_q=x.max_q + 9, max_kv=x.max_kv + 5000))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv,new,hq,hkv,d,window", [(70, 90, 8, 2, 64, 0), (300, 150, 4, 1, 128, 100), (5, 40, 32, 1, 64, 9), (900, 70, 2, 2, 128, 0)])
def test_unseen_values_stay_out(dtype, kv, new, hq, hkv, d, window):
    """Infinities and NaN in keys and values reach the rows that see their token and no other."""
    say("chunk attention unseen values", dtype, kv, new, hq, hkv, d, window)
    x = Chunk([kv], [new], hq, hkv, d, dtype, 16, window, seed=8)
    clean = host(x.call()[0])[:new]
    for at in (kv + new // 2, kv + new - 1, max(0, kv + new // 2 - window) if window else kv):
        slot = int(x.slot[0][at])
        sees = x.see[0][:, at]
        for value in (math.inf, -math.inf, math.nan):
            for cache in (x.v, x.k):
                keep = cache[slot].clone()
                cache[slot, :, 3] = value
                o = host(x.call()[0])[:new]
                cache[slot] = keep
                np.testing.assert_array_equal(o[~sees], clean[~sees])
                if cache is x.v:
                    np.testing.assert_array_equal(o[sees][..., 3], np.full_like(o[sees][..., 3], value))
                    rest = [j for j in range(d) if j != 3]
                    assert np.isfinite(o[sees][..., rest]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps,window", [(16, 0), (32, 70), (64, 0), (128, 40)])
def test_missing_pages_and_short_bounds(dtype, ps, window):
    """Tokens in pages that are not there, behind the table or behind max_kv are not seen; a row that sees none gives zeros."""
    say("chunk attention missing pages", dtype, ps, window)
    kv, new = [300, 40, 0], [60, 9, 200]
    x = Chunk(kv, new, 8, 2, 128, dtype, ps, window, seed=9)
    for bad in (-1, 10 ** 6):
        t = x.table_h.copy()
        t[0, 0], t[0, 300 // ps], t[2, 1] = bad, bad, bad
        see = [s.copy() for s in x.see]
        for b, p in ((0, 0), (0, 300 // ps), (2, 1)):
            see[b][:, p * ps:(p + 1) * ps] = False
        x.check(*x.call(table=i32(t)), see=see)
    cols = 256 // ps
    see = [s.copy() for s in x.see]
    for s in see:
        s[:, cols * ps:] = False
    x.check(*x.call(table=x.table[:, :cols]), see=see)
    see = [s.copy() for s in x.see]
    for s in see:
        s[:, 310:] = False
    x.check(*x.call(max_kv=310), see=see)
    t = torch.full_like(x.table, -1)
    x.check(*x.call(table=t), see=[np.zeros_like(s) for s in x.see])
    x.check(*x.call(table=t[:, :0]), see=[np.zeros_like(s) for s in x.see])
    # rows behind max_q are left alone
    o, e = x.call(max_q=50)
    assert (host(o)[50:60] == 5.0).all() and (host(e)[50:60] == 5.0).all() and (host(o)[:50] != 5.0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,window", [(64, 0), (128, 20)])
def test_no_tokens_at_all(dtype, d, window):
    """max_kv = 0, or an empty pool: every row gives zeros and a log-sum-exp of -infinity; a workspace of the asked size is
    enough, and nothing is written behind it."""
    say("chunk attention without tokens", dtype, d, window)
    x = Chunk([300, 0, 40, 7], [60, 9, 0, 200], 8, 2, d, dtype, 16, window, seed=14)
    rows = int(x.cu[-1])
    need = qcf.qcf_chunk_attn_workspace_size(4, 200, 0, 8, 2, d, DT[dtype])
    ws = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    for how in (dict(max_kv=0, ws=ws[:need]), dict(max_kv=0), dict(max_kv=0, table=x.table[:, :0])):
        o, e = x.call(**how)
        assert (o[:rows] == 0).all() and (e[:rows] == -math.inf).all() and (o[rows:] == 5.0).all() and (e[rows:] == 5.0).all()
    x.k, x.v = x.k[:0], x.v[:0]
    o, e = x.call()
    assert (o[:rows] == 0).all() and (e[:rows] == -math.inf).all()
    assert (ws[need:] == 0x5A).all()


@pytest.mark.parametrize("d", [64, 128])
def test_float32_weights_stay_above_zero_in_merged_parts(d):
    """Parts of a row that weigh 2^-135 of it, in a row that is cut over blocks and in one that is not: weights are
    subnormal numbers (14 bits), so that large values count and infinite ones are infinite."""
    say("chunk attention small weights", d)
    for kv in (40, 9000):
        x = Chunk([kv], [1], 8, 2, d, "f32", 16, seed=15)
        at = torch.from_numpy(x.slot[0][:kv // 2]).cuda()
        low = np.float32(-135 / (x.scale * math.log2(math.e)))
        x.k.zero_()
        x.k[at, :, 0] = float(low)
        x.q[:1] = 0
        x.q[0, :, 0] = 1.0
        x.v[:, :, 5] = 0
        x.v[at, :, 5] = 3e34                                             # (4500 of them, weighed 1 in a part, are below 3.4e38)
        x.v[at[0], :, 3] = math.inf
        o = host(x.call()[0])[0]
        weight = 2.0 ** (float(low) * x.scale * math.log2(math.e))
        want = weight * float(np.float32(3e34)) * (kv // 2) / (kv + 1 - kv // 2)
        assert (o[:, 3] == math.inf).all()
        # half a step of the weight is 2^-15 of it at most, of two factors in a row 2^-14; the rest is below 2^-16
        np.testing.assert_allclose(o[:, 5], want, rtol=2.0 ** -14 + 2.0 ** -16)
        assert np.isfinite(np.delete(o, 3, axis=1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_any_size(dtype):
    """One row and head with logits beyond 2^28: the others' bits are those of a call without it; rows that see only
    logits of -infinity or NaN are NaN."""
    say("chunk attention logits of any size", dtype)
    for kv, new, hq, hkv, d, window in ((70, 40, 8, 2, 64, 0), (2500, 33, 16, 4, 128, 0), (600, 100, 4, 4, 128, 90)):
        x = Chunk([kv], [new], hq, hkv, d, dtype, 16, window, seed=12)
        was = x.call()
        for row, head in ((0, 1), (new - 1, hq - 1)):
            keep = x.q[row, head].clone()
            x.q[row, head] = 1e18
            now = x.call()
            x.q[row, head] = math.nan
            nan = x.call()
            x.q[row, head] = keep
            rest = torch.ones(was[1].shape, dtype=torch.bool, device="cuda")
            rest[row, head] = False
            assert now[1][row, head].abs() > 1e15 and torch.isfinite(now[0][row, head]).all()
            assert torch.isnan(nan[0][row, head]).all() and torch.isnan(nan[1][row, head])
            for a, b, c in zip(was, now, nan):
                assert torch.equal(a[:new][rest[:new]], b[:new][rest[:new]]) and torch.equal(a[:new][rest[:new]], c[:new][rest[:new]])
    # infinite keys that all logits of a row meet
    x = Chunk([0], [3], 2, 1, 64, dtype, 16, 1, seed=13)
    x.q[1] = x.q[1].abs() + 0.1
    x.k[int(x.slot[0][1])] = -math.inf
    o, e = x.call()
    assert torch.isnan(o[1]).all() and torch.isnan(e[1]).all() and torch.isfinite(o[[0, 2]]).all()


@pytest.mark.parametrize("dtype,window", [("bf16", 0), ("f32", 30), ("bf16", 70)])
def test_more_requests_than_threads(dtype, window):
    """700 requests, many without rows: three of them to a thread that adds up the work."""
    say("chunk attention many requests", dtype, window)
    rng = np.random.default_rng(16)
    new, kv = rng.choice([0, 0, 1, 1, 2, 40], 700), rng.choice([0, 1, 15, 16, 100, 300], 700)
    new[0], new[-1] = 0, 40
    x = Chunk(kv.tolist(), new.tolist(), 8, 2, 64, dtype, 16, window, seed=17)
    x.check(*x.call())


def test_the_same_as_the_tree_call_without_a_mask():
    """Rows of a decoded token, a chain and a prompt: what qcf_tree_attn gives, within both calls' roundings."""
    say("chunk and tree attention")
    for dtype in ("bf16", "f32"):
        x = Chunk([200, 0, 31], [1, 70, 5], 8, 2, 128, dtype, 32, seed=3)
        a, b = x.call(), Batch.call(x)
        x.check(*a)
        x.check(*b)


def test_chunk_attn_refuses():
    x = Chunk([20], [3], 8, 2, 64, "bf16", 16)
    for kw in (dict(page=8), dict(page=24), dict(window=-1), dict(scale=0.0), dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda")),
               dict(q=x.q.float()), dict(q=x.q[:, ::2]), dict(cu=i32([0])), dict(out=x.q)):
        out = torch.empty_like(x.q)
        with pytest.raises(qcf.QcfError):
            qcf.qcf_chunk_attn(kw.get("out", out), kw.get("q", x.q), kw.get("cu", i32(x.cu)), x.k, x.v, x.table, i32(x.kv),
                               kw.get("page", 16), 3, 23, kw.get("scale", 0.1), window=kw.get("window", 0), workspace=kw.get("ws"))
