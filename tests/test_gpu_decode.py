"""The decoding calls (include/qcf_decode.h) against the float64 oracle, at the sizes and masks where
they can go wrong.

Tolerances, per element, from the roundings made (a rounding to a type is off by at most half a step:
2^-8 of the value for bf16, 2^-24 for float32):
  rotation   cosine and sine are rounded to float32 once, then a product and a fused multiply-add:
             4 * 2^-24 * magnitude * (|x1| + |x2|), and one rounding to the storage type
  attention  a logit is a float32 sum of d products, at most d * 2^-24 of the sum of magnitudes off, and
             three more roundings (scale, exponent's argument, exponential) of 2^-23 of the largest logit;
             a weight is off by that factor in numerator and sum.  A sum over n tokens adds at
             most (n + 16) * 2^-24, the weights' rounding to bf16 2^-8, the output one rounding.
  integers   equal.
"""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import decode as D
from paper_2606_05875_amd import qcf

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def host(t):
    return t.double().cpu().numpy()


def cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int64)


def rows_of(rng, shape, dtype, pad=0, scale=1.0):
    """A [rows, heads, d] tensor with `pad` elements between rows, and its values in float64."""
    x = torch.from_numpy(rng.standard_normal((shape[0], int(np.prod(shape[1:])) + pad)) * scale).to(DT[dtype]).cuda()
    v = x[:, :int(np.prod(shape[1:]))].view(shape)
    return v, host(v)


def within(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want)):.3g} "
                           f"at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}")


def random_parents(rng, new, back=5):
    return np.concatenate([[-1 if i == 0 else rng.integers(max(-1, i - back), i) for i in range(n)] for n in new]
                          + [[]]).astype(np.int32)


# -- pages ------------------------------------------------------------------------
def _plan(kv, new, ps, n_rows=None, tree=False, spare=0, free=None, held=None, head=None, cols=None, seed=0,
          words=None, back=5):
    rng = np.random.default_rng(seed)
    B, kv, new = len(kv), np.asarray(kv), np.asarray(new)
    have = [max(-(-max(int(k), 0) // ps), 0 if held is None else int(h)) for k, h in
            zip(kv, kv if held is None else held)]
    need = [max(h, -(-(max(int(k), 0) + max(int(n), 0)) // ps)) for k, n, h in zip(kv, new, have)]
    cols = max(need + [1]) + 1 if cols is None else cols
    pages = sum(need) + 20
    order = rng.permutation(pages)
    table, at = np.full((B, cols), -7), 0
    for b, h in enumerate(have):
        table[b, :min(h, cols)] = order[at:at + min(h, cols)]
        at += h
    free = order[at:] if free is None else free(order[at:], pages)
    total = int(np.maximum(new, 0).sum())
    n_rows = total + spare if n_rows is None else n_rows
    parents = None
    if tree:
        parents = np.full(n_rows, 5, np.int32)
        parents[:total] = random_parents(rng, np.maximum(new, 0), back)[:n_rows]
        words = (int(max(new)) + 31) // 32 if words is None else words
    full = lambda *shape: torch.full(shape, -9, dtype=torch.int32, device="cuda")
    wide = torch.full((B, cols + 3), -11, dtype=torch.int32, device="cuda")     # columns beyond the table stay
    wide[:, :cols] = i32(table) if B else wide[:, :cols]
    t, slots, pos, cu, end, ho, fo = wide[:, :cols], full(n_rows), full(n_rows), full(B + 1), full(B), full(B), full(1)
    mask = full(n_rows, words) if tree else None
    kw = dict(pages_held=None if held is None else i32(held), free_head=None if head is None else i32([head]),
              kv_end=end, pages_held_out=ho, free_head_out=fo)
    if tree:
        kw.update(parents=i32(parents), tree_mask=mask)
    qcf.qcf_page_plan(t, i32(kv), i32(new), i32(free), slots, pos, cu, ps, pages, int(max(list(new) + [0])), **kw)
    want = D.page_plan(table, kv, new, free, ps, pages, n_rows, held, head or 0, parents, words or 0)
    got = [host(x).astype(np.int64) for x in (t, slots, pos, cu, end, ho)]
    for g, w, name in zip(got, [want[0], want[1], want[2], want[4], want[5], want[6]],
                          ("table", "slots", "positions", "cu", "end", "held")):
        np.testing.assert_array_equal(g, w, err_msg=name)
    assert int(fo[0]) == want[7]
    if tree:
        np.testing.assert_array_equal(mask.cpu().numpy(), D.pack_bits(want[3]) if words else mask.cpu().numpy())
    assert (wide[:, cols:] == -11).all()


@pytest.mark.parametrize("ps", [1, 2, 16, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_page_plan(ps, tree):
    say("page plan", ps, tree)
    rng = np.random.default_rng(7)
    _plan([0, 1, ps, ps - 1, 5 * ps, 7, 0], [1, 0, 3, 1, ps + 1, 70, 0], ps, tree=tree, spare=5)
    _plan([13], [1], ps, tree=tree)
    _plan([0], [0], ps, tree=tree, spare=3, words=1)
    _plan(rng.integers(0, 300, 700), rng.integers(0, 9, 700), ps, tree=tree, spare=1000)     # several scans
    _plan(rng.integers(0, 60, 40), rng.integers(0, 200, 40), ps, tree=tree)                  # several tiles


def test_page_plan_lengths():
    say("page plan lengths")
    _plan([], [], 16, spare=4)                                       # no request: only padding
    _plan([0, 0], [30000, 12345], 64)                                # prompts
    _plan([-5, 3], [-1, 2], 16, spare=2)                             # negative lengths count as zero
    _plan([5, 9, 0], [4, 4, 4], 4, held=[5, 1, 0], head=3)           # more pages than tokens; fewer than tokens
    _plan([2 ** 30], [3], 2 ** 20)                                   # far positions
    _plan([4, 4], [1024, 1000], 16, tree=True, back=40)              # the largest trees
    _plan([4, 4], [1024, 1000], 16, tree=True, back=1)               # as chains: every earlier row is an ancestor
    _plan([4], [40], 16, tree=True, words=4)                         # a wider mask than needed
    _plan([7, 2], [9, 3], 4, n_rows=6, held=[5, 2])                  # fewer packed rows than new ones (no page begins there)


def test_page_plan_runs_out():
    say("page plan runs out")
    _plan([3, 9, 0], [9, 30, 50], 8, free=lambda f, n: f[:4])                         # the free list ends
    _plan([3, 9, 0], [9, 30, 50], 8, free=lambda f, n: np.where(np.arange(f.size) % 3 == 1, n + 5, f))  # no such page
    _plan([3, 9, 0], [9, 30, 50], 8, free=lambda f, n: np.where(np.arange(f.size) % 3 == 1, -2, f))
    _plan([3, 9, 0], [9, 30, 50], 8, cols=4)                                          # the table ends
    _plan([0, 0], [9, 9], 8, free=lambda f, n: f[:0], head=0)
    _plan([0, 0], [9, 9], 8, head=10 ** 6)
    _plan([0, 0], [9, 9], 8, head=-3)


# -- rotary ------------------------------------------------------------------------
def _rope(rows, hq, hkv, d, dtype, R, inter, kv=True, q=True, gather=False, pad=0, magnitude=1.0, top=40000,
          extra=0, seed=0, freq=None, pos=None):
    rng = np.random.default_rng(seed)
    src = rows + 9 if gather else rows + extra
    n_slots = rows + 13
    k, kh = rows_of(rng, (src, hkv, d), dtype, pad)
    v, vh = rows_of(rng, (src, hkv, d), dtype, pad)
    x, xh = rows_of(rng, (src, hq, d), dtype, 2 * pad)
    kc, vc = rows_of(rng, (n_slots, hkv, d), dtype, 3 * pad), rows_of(rng, (n_slots, hkv, d), dtype, 3 * pad)
    slots = rng.permutation(n_slots)[:rows]
    if rows > 3:
        slots[1], slots[2] = -1, n_slots                      # stored nowhere
    idx = rng.permutation(src)[:rows]
    pos = rng.integers(-20, top, rows) if pos is None else pos
    freq = D.rope_frequencies(R, 1e4) if freq is None else freq
    out = torch.full((rows, hq, d), 3.0, dtype=DT[dtype], device="cuda")
    kw = dict(q_new=x, q_out=out) if q else {}
    args = (kc[0], vc[0], k, v, i32(slots)) if kv else (None,) * 5
    qcf.qcf_rope_store(*args, *((i32(pos), torch.from_numpy(freq).cuda()) if R else ()), interleaved=inter,
                       magnitude=magnitude, src_idx=i32(idx) if gather else None, **kw)
    at = idx if gather else np.arange(rows)
    turn = lambda y: D.rope(y[at], pos, freq, inter, magnitude) if R else (y[at], 0 * y[at])
    tol = lambda w, size: HALF[dtype] * np.abs(w) + (4 * 2.0 ** -24 * size if R else 0)
    if kv:
        ok = (slots >= 0) & (slots < n_slots)
        w, size = turn(kh)
        want, bound = kc[1].copy(), np.zeros_like(kc[1])
        want[slots[ok]], bound[slots[ok]] = w[ok], tol(w, size)[ok]
        within(host(kc[0]), want, bound, "keys")               # rows without a slot keep their bits
        want = vc[1].copy()
        want[slots[ok]] = vh[at][ok]
        np.testing.assert_array_equal(host(vc[0]), want)
    if q:
        w, size = turn(xh)
        within(host(out), w, tol(w, size), "queries")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (32, 8, 128), (16, 1, 128), (5, 5, 64), (64, 8, 128)])
@pytest.mark.parametrize("inter", [False, True])
def test_rope_store(dtype, hq, hkv, d, inter):
    say("rope store", dtype, hq, hkv, d, inter)
    for rows, R, kw in ((1, d, {}), (5, 16, dict(pad=8)), (37, d - 16, dict(gather=True, magnitude=1.25)),
                        (300, d, dict(pad=16, extra=4)), (11, 48, dict(kv=False)), (12, 32, dict(q=False, gather=True)),
                        (1030, d // 2, dict(q=rows_even(hq)))):
        _rope(rows, hq, hkv, d, dtype, R, inter, seed=rows, **kw)


def rows_even(x):
    return x % 2 == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_store_copies(dtype):
    """Without positions rows are copied as they are (into pages, or from slot to slot)."""
    say("rope store copies", dtype)
    for rows in (1, 6, 130):
        _rope(rows, 8, 8, 128, dtype, 0, False, gather=rows == 6, pad=8, seed=rows)


def test_rope_store_far_positions():
    """Angles up to 2^31 keep float64's precision; other frequencies are taken as given; an angle that
    is not finite gives NaN in its pairs and nothing else."""
    say("rope store far positions")
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 123456789, 0, 1])
    _rope(6, 4, 2, 64, "f32", 64, False, pos=pos)
    freq = np.concatenate([np.linspace(0, 3, 16)])
    _rope(6, 4, 2, 64, "f32", 32, True, pos=np.array([5, 6, 7, 8, 9, 1000]), freq=freq)
    x = torch.ones((2, 1, 64), device="cuda")
    out = torch.empty_like(x)
    freq = torch.tensor([math.inf] + [1.0] * 7, dtype=torch.float64, device="cuda")
    qcf.qcf_rope_store(None, None, None, None, None, i32([1, 3]), freq, q_new=x, q_out=out)
    got = host(out)[:, 0]
    assert np.isnan(got[:, [0, 8]]).all() and np.isfinite(np.delete(got, [0, 8], 1)).all()


def test_rope_store_skips_missing_sources():
    say("rope store missing sources")
    rng = np.random.default_rng(3)
    x, xh = rows_of(rng, (4, 2, 64), "f32")
    out = torch.full((5, 2, 64), 3.0, device="cuda")
    qcf.qcf_rope_store(None, None, None, None, None, i32([0] * 5), torch.ones(8, dtype=torch.float64, device="cuda"),
                       q_new=x, q_out=out, src_idx=i32([3, -1, 4, 0, 3]))
    got = host(out)
    assert (got[[1, 2]] == 3.0).all()
    np.testing.assert_array_equal(got[[0, 3, 4]], xh[[3, 0, 3]])


def test_rope_store_empty():
    e = torch.empty((0, 2, 64), device="cuda")
    qcf.qcf_rope_store(None, None, None, None, None, i32([]), torch.ones(8, dtype=torch.float64, device="cuda"),
                       q_new=e, q_out=e.clone())


# -- attention ------------------------------------------------------------------------
class Batch:
    """A paged batch in torch and its tokens in float64, with scattered pages."""

    def __init__(self, kv, new, hq, hkv, d, dtype, ps, tree, seed=0, pad=0, spare=3, q_scale=1.5, back=5, fill=None,
                 words=None, big=0):
        rng = self.rng = np.random.default_rng(seed)
        self.kv, self.new, self.hq, self.hkv, self.d, self.dtype, self.ps = kv, new, hq, hkv, d, dtype, ps
        self.end = [a + b for a, b in zip(kv, new)]
        need = [-(-e // ps) for e in self.end]
        pages = sum(need) + 4
        order = rng.permutation(pages)
        if big:                                                # pages far into a large pool
            order = order + big
            pages += big
        table, at = np.full((len(kv), max(need + [0]) + 2), -1), 0
        for b, h in enumerate(need):
            table[b, :h] = order[at:at + h]
            at += h
        self.table_h, self.table = table, i32(table)
        slot = [np.array([t[j // ps] * ps + j % ps for j in range(e)], np.int64) for t, e in zip(table, self.end)]
        self.slot = slot
        width = hkv * d + pad
        pool = lambda: torch.full((pages * ps, width), float("nan"), dtype=DT[dtype], device="cuda") if not big else \
            torch.empty((pages * ps, width), dtype=DT[dtype], device="cuda")
        self.kbuf, self.vbuf = pool(), pool()                  # rows without a token hold NaN
        self.k, self.v = (x[:, :hkv * d].view(-1, hkv, d) for x in (self.kbuf, self.vbuf))
        self.kh, self.vh = [], []
        for s in slot:
            for cache, lst in ((self.k, self.kh), (self.v, self.vh)):
                x = torch.from_numpy(rng.standard_normal((s.size, hkv, d))).to(DT[dtype])
                if fill is not None:
                    fill(x, cache is self.v)
                cache[torch.from_numpy(s).cuda()] = x.cuda()
                lst.append(x.double().numpy())
        self.cu = cum(new)
        n = int(self.cu[-1])
        self.q = torch.from_numpy(rng.standard_normal((n + spare, hq, d)) * q_scale).to(DT[dtype]).cuda()
        self.q[n:] = float("nan")
        self.see, self.mask = [], None
        bits = np.zeros((n + spare, 32 * (words or (max(new + [1]) + 31) // 32)), bool)
        for b, m in enumerate(new):
            see = D.chain_see(m, kv[b])
            if tree == "random":                               # any mask, rows that see no draft among them
                see[:, kv[b]:] = rng.random((m, m)) < 0.4
                if m:
                    see[m // 2, kv[b]:] = False
            elif tree:
                par = random_parents(rng, [m], back)
                see[:, kv[b]:] = False
                for i in range(m):
                    a = i
                    while a >= 0:
                        see[i, kv[b] + a] = True
                        a = par[a]
            self.see.append(see)
            bits[self.cu[b]:self.cu[b + 1], :m] = see[:, kv[b]:]
            bits[self.cu[b]:self.cu[b + 1], m:] = rng.random((m, bits.shape[1] - m)) < 0.5    # beyond the request: unseen
        if tree:
            self.mask = i32(D.pack_bits(bits))
        self.scale = 1 / math.sqrt(d)
        self.max_q, self.max_kv = max(new + [0]), max(self.end + [0])

    def call(self, out=None, lse=None, ws=None, **kw):
        out = torch.full_like(self.q, 5.0) if out is None else out
        lse = torch.full(self.q.shape[:2], 5.0, device="cuda") if lse is None else lse
        g = dict(max_q=self.max_q, max_kv=self.max_kv, table=self.table)
        g.update(kw)
        qcf.qcf_tree_attn(out, self.q, i32(self.cu), self.k, self.v, g["table"], i32(self.kv), self.ps, g["max_q"],
                          g["max_kv"], self.scale, tree_mask=self.mask, lse=lse, workspace=ws)
        return out, lse

    def check(self, out, lse, see=None):
        n = int(self.cu[-1])
        o, e = host(out), host(lse)
        assert (o[n:] == 5.0).all() and (e[n:] == 5.0).all()   # rows behind the last request
        for b in range(len(self.kv)):
            a, z = self.cu[b], self.cu[b + 1]
            if a == z:
                continue
            s = self.see[b] if see is None else see[b]
            q = host(self.q[a:z])
            want, wl, absv, absx = D.tree_attention(q, np.nan_to_num(self.kh[b], nan=0.0), self.vh[b], s, self.scale)
            seen = s.any(1)
            assert (o[a:z][~seen] == 0).all() and (e[a:z][~seen] == -np.inf).all()
            top = np.where(np.isfinite(wl), np.abs(wl), 0) + absx
            off = self.d * 2.0 ** -24 * absx + 3 * 2.0 ** -23 * top + (s.shape[1] + 16) * 2.0 ** -24
            within(e[a:z][seen], wl[seen], (off + 2.0 ** -22 * np.abs(wl))[seen], f"request {b} lse")
            tol = HALF[self.dtype] * np.abs(want) + (2 * off + (2.0 ** -8 if self.dtype == "bf16" else 0))[..., None] * absv
            within(o[a:z], want, tol, f"request {b}")


GEO = [(8, 2, 64), (32, 8, 128), (32, 1, 64), (4, 4, 128), (64, 8, 128), (16, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", GEO)
@pytest.mark.parametrize("tree", [False, True, "random"])
def test_tree_attn(dtype, hq, hkv, d, tree):
    say("tree attention", dtype, hq, hkv, d, tree)
    for i, (kv, new, ps) in enumerate(((
            [0, 1, 31, 32, 33, 63, 64, 65, 127, 200], [1, 2, 3, 1, 5, 8, 1, 4, 9, 7], 16),
            ([300, 5, 0], [1, 1, 1], 1), ([130, 0, 17], [33, 0, 64], 8), ([0], [40], 64), ([500, 40], [8, 16], 128))):
        x = Batch(kv, new, hq, hkv, d, dtype, ps, tree, seed=i, pad=(0, d, 8, 0, 16)[i], q_scale=(1.5, 1.5, 4.0, 1.5, 0.2)[i])
        x.check(*x.call())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv,new,hq,hkv,d", [
    ([9000], [1], 8, 2, 64), ([5000, 100, 0, 2500], [3, 1, 2, 4], 8, 2, 128), ([4200], [17], 16, 2, 128),
    ([3000, 2000], [40, 30], 8, 2, 128), ([2100], [65], 16, 4, 64), ([33, 1500], [70, 130], 8, 4, 64)])
def test_tree_attn_long(dtype, kv, new, hq, hkv, d):
    """Caches that are cut over blocks, more query vectors than a tile holds; twice over a dirty workspace:
    the same bits."""
    say("tree attention long", dtype, kv, new, hq, hkv, d)
    x = Batch(kv, new, hq, hkv, d, dtype, 16, True, seed=5, back=9)
    x.check(*x.call())
    need = qcf.qcf_tree_attn_workspace_size(len(kv), x.max_q, x.max_kv, hq, hkv, d, DT[dtype])
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    a, b = x.call(ws=ws), x.call(ws=ws)
    x.check(*a)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    # larger bounds than the batch needs, another workspace: within the same tolerances
    x.check(*x.call(max_q=x.max_q + 9, max_kv=x.max_kv + 5000))


@pytest.mark.parametrize("kv,new,hq,hkv,d,ps", [
    ([3000, 2000], [40, 30], 16, 4, 128, 16), ([0, 700, 64, 1], [33, 1, 70, 0], 8, 2, 64, 64), ([4100], [130], 8, 4, 64, 128),
    ([40, 2500, 9], [17, 20, 1], 64, 4, 128, 128), ([90, 5], [65, 3], 4, 1, 128, 4), ([900], [300], 2, 1, 64, 8)])
@pytest.mark.parametrize("tree", [False, True, "random"])
def test_tree_attn_many_keys_by_the_bounds(kv, new, hq, hkv, d, ps, tree):
    """More than 128 vectors per KV head and bounds that promise many keys: units of 256 vectors.  Values that are
    not seen, pages that are not there, twice over a dirty workspace."""
    say("tree attention many keys", kv, new, hq, hkv, d, ps, tree)
    x = Batch(kv, new, hq, hkv, d, "bf16", ps, tree, seed=15, back=9)
    most = 64 * (-(-8192 // (len(kv) * hkv)) + 1)
    assert x.max_q * (hq // hkv) > 128 and most > x.max_kv
    need = qcf.qcf_tree_attn_workspace_size(len(kv), x.max_q, most, hq, hkv, d, DT["bf16"])
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    a, b = x.call(ws=ws, max_kv=most), x.call(ws=ws, max_kv=most)
    x.check(*a)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    bad = new[0] // 2
    if new[0] > 1:
        slot, sees = int(x.slot[0][kv[0] + bad]), x.see[0][:, kv[0] + bad]
        for value in (math.inf, math.nan):
            keep = x.v[slot].clone()
            x.v[slot, :, 3] = value
            o, c = host(x.call(max_kv=most)[0])[:new[0]], host(a[0])[:new[0]]
            x.v[slot] = keep
            np.testing.assert_array_equal(o[~sees], c[~sees])
            np.testing.assert_array_equal(o[sees][..., 3], np.full_like(o[sees][..., 3], value))
    t = x.table_h.copy()
    t[0, 1] = -1
    see = [s.copy() for s in x.see]
    see[0][:, ps:2 * ps] = False
    x.check(*x.call(table=i32(t), max_kv=most), see=see)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_attn_unseen_values_stay_out(dtype):
    """Infinities and NaN in keys and values of drafted tokens reach the rows that see them and no other."""
    say("tree attention unseen values", dtype)
    for hq, hkv, d, kv, new in ((8, 2, 64, 70, 9), (8, 1, 128, 30, 12), (32, 1, 64, 5, 40), (16, 2, 128, 1000, 7)):
        x = Batch([kv], [new], hq, hkv, d, dtype, 16, True, seed=8, back=9)
        clean, _ = x.call()
        bad = new // 2                                          # one drafted token
        slot = int(x.slot[0][kv + bad])
        sees = x.see[0][:, kv + bad]
        assert sees.any() and not sees.all()
        for value in (math.inf, -math.inf, math.nan):
            for cache in (x.v, x.k):
                keep = cache[slot].clone()
                cache[slot, :, 3] = value
                out, _ = x.call()
                cache[slot] = keep
                o, c = host(out)[:new], host(clean)[:new]
                np.testing.assert_array_equal(o[~sees], c[~sees])
                if cache is x.v:
                    want = np.full_like(o[sees][..., 3], value)
                    np.testing.assert_array_equal(o[sees][..., 3], want)
                    rest = [j for j in range(d) if j != 3]
                    # (the one bad token is added on its own there, which rounds its weight later)
                    np.testing.assert_allclose(o[sees][..., rest], c[sees][..., rest],
                                               rtol=2.0 ** -6, atol=2.0 ** -6)


def test_tree_attn_large_logits():
    """Logits of +-1e30 and more, and a row whose logits are all far below zero, are ordinary numbers."""
    say("tree attention large logits")
    for dtype in ("bf16", "f32"):
        x = Batch([50], [3], 4, 2, 64, dtype, 16, True, seed=9)
        for scale in (1e18, 1e33):
            sign = torch.sign(x.q[:3].double().sum(-1, keepdim=True)).to(DT[dtype])
            x.q[:3] = (sign * scale).expand(3, 4, 64)           # every logit of a row: scale * sum of a key
            out, lse = x.call()
            q = host(x.q[:3])
            want, wl, _, _ = D.tree_attention(q, x.kh[0], x.vh[0], x.see[0], x.scale)
            one = np.sort(np.abs(x.kh[0].sum(-1)), axis=0)
            assert np.isfinite(host(out[:3])).all()
            np.testing.assert_allclose(host(lse[:3]), wl, rtol=64 * 2.0 ** -24 * 64)
            within(host(out[:3]), want, 2.0 ** -7 * np.abs(want) + 1e-30, "one token takes all")


def test_tree_attn_bad_pages():
    """Tokens in pages outside the pool, or beyond the table, are not seen."""
    say("tree attention bad pages")
    for dtype in ("bf16", "f32"):
        x = Batch([100, 40], [4, 3], 8, 2, 64, dtype, 16, True, seed=10)
        for bad in (-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1):
            t = x.table_h.copy()
            t[0, 2], t[1, 0] = bad, bad
            see = [s.copy() for s in x.see]
            see[0][:, 32:48] = False
            see[1][:, :16] = False
            x.check(*x.call(table=i32(t)), see=see)
        see = [s.copy() for s in x.see]
        see[0][:, 48:] = False
        x.check(*x.call(table=x.table[:, :3]), see=see)         # a view with the table's row stride
        see = [s.copy() for s in x.see]
        see[0][:, 50:] = False
        x.check(*x.call(max_kv=50), see=see)                    # fewer keys than there are


def test_tree_attn_no_pool():
    say("tree attention without a pool")
    x = Batch([0, 0], [2, 1], 8, 2, 64, "bf16", 16, False, seed=11)
    out, lse = torch.full_like(x.q, 5.0), torch.full(x.q.shape[:2], 5.0, device="cuda")
    qcf.qcf_tree_attn(out, x.q, i32(x.cu), x.k[:7], x.v[:7], x.table, i32(x.kv), 16, 2, 2, 0.1, lse=lse)
    assert (out[:3] == 0).all() and (lse[:3] == -math.inf).all() and (out[3:] == 5.0).all()
    qcf.qcf_tree_attn(out[:0], x.q[:0], i32(x.cu), x.k, x.v, x.table, i32(x.kv), 16, 2, 2, 0.1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_attn_offsets_past_32_bits(dtype):
    """Pages more than 4 GiB into the pool."""
    say("tree attention far pages", dtype)
    big = 5 * 2 ** 30 // (16 * 2 * 64 * (2 if dtype == "bf16" else 4))
    x = Batch([900, 20], [5, 2], 8, 2, 64, dtype, 16, True, seed=12, big=big)
    x.check(*x.call())


# -- verification ------------------------------------------------------------------------
def _verify(new, vocab, dtype, draft, tree, seed=0, pad=0, spare=2, sharp=3.0, noise=1.0, mutate=None, max_rows=None,
            back=4, slots=True):
    rng = np.random.default_rng(seed)
    cu = cum(new)
    n = int(cu[-1]) + spare
    soft = lambda z: np.exp(z - z.max(1, keepdims=True)) / np.exp(z - z.max(1, keepdims=True)).sum(1, keepdims=True)
    z = sharp * rng.standard_normal((n, vocab))
    put = lambda x: torch.from_numpy(np.pad(x, ((0, 0), (0, pad)), constant_values=0.7)).to(DT[dtype]).cuda()[:, :vocab]
    t, dr = put(soft(z)), put(soft(z + noise * rng.standard_normal((n, vocab))))
    parents = np.concatenate([random_parents(rng, new, back), np.zeros(spare)]).astype(np.int32) if tree else None
    base = np.concatenate([np.repeat(cu[:-1], new), np.zeros(spare)]).astype(np.int64)
    up = parents if tree else np.concatenate([np.arange(-1, m - 1) for m in new] + [np.zeros(spare)]).astype(np.int64)
    p = host(dr)[base + np.maximum(up, 0)]
    c = np.cumsum(p, 1)
    tokens = np.minimum((c < rng.random((n, 1)) * c[:, -1:]).sum(1), vocab - 1).astype(np.int32)
    u, un = rng.random(n).astype(np.float32), rng.random(len(new)).astype(np.float32)
    if mutate is not None:
        mutate(t=t, dr=dr, tokens=tokens, u=u, un=un, parents=parents, cu=cu)
    W = max(new + [0]) if max_rows is None else max_rows
    full = lambda *s: torch.full(s, -9, dtype=torch.int32, device="cuda")
    n_out, path, toks, ms, md = full(len(new)), full(len(new), W), full(len(new), W), full(len(new), W), full(len(new), W)
    slot = rng.permutation(10 * n)[:n].astype(np.int32)
    kw = dict(slots=i32(slot), move_src=ms, move_dst=md) if slots else {}
    f = lambda a: torch.from_numpy(a).cuda()
    qcf.qcf_verify_drafts(n_out, path, toks, t, i32(tokens), i32(cu), f(u), f(un), draft=dr if draft else None,
                          parents=i32(parents) if tree else None, **kw)
    th, dh = host(t), host(dr)
    lens = []
    for b, m in enumerate(new):
        a, m = cu[b], min(m, W)
        wp, wt = D.verify(th[a:a + m], dh[a:a + m] if draft else None, tokens[a:a + m],
                          parents[a:a + m] if tree else None, u[a:a + m], un[b])
        k = len(wp)
        lens.append(k)
        row = lambda x: x[b].cpu().numpy()
        assert int(n_out[b]) == k, (b, int(n_out[b]), wp, wt)
        np.testing.assert_array_equal(row(path), wp + [-1] * (W - k), err_msg=f"request {b}")
        np.testing.assert_array_equal(row(toks), wt + [-1] * (W - k), err_msg=f"request {b}")
        if slots:
            src = [slot[a + x] if x != i else -1 for i, x in enumerate(wp)]
            dst = [slot[a + i] if x != i else -1 for i, x in enumerate(wp)]
            np.testing.assert_array_equal(row(ms), src + [-1] * (W - k))
            np.testing.assert_array_equal(row(md), dst + [-1] * (W - k))
    return lens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("tree", [False, True])
def test_verify(dtype, draft, tree):
    say("verify", dtype, draft, tree)
    lens = []
    for i, (new, vocab, pad) in enumerate((([1], 1, 0), ([1, 2, 5, 0, 9, 3], 7, 0), ([6] * 40, 50, 3), ([26, 4], 4095, 1),
                                           ([5, 5, 5, 8], 4097, 0), ([3], 150001, 7), ([9, 70, 130], 333, 0))):
        for seed in range(3):
            lens += _verify(new, vocab, dtype, draft, tree, seed=10 * i + seed, pad=pad,
                            noise=(0.3, 1.0, 2.5)[seed], back=(2, 4, 8)[seed])
    assert len(set(lens)) > 3                                   # walks of several lengths came up


def test_verify_borders():
    say("verify borders")

    def certain(t, dr, tokens, u, un, parents, cu):             # one-hot rows: greedy decoding
        x = torch.from_numpy(tokens).long().cuda().roll(-1)
        t.zero_()
        t[torch.arange(t.shape[0]), x] = 1.0
        u[:] = np.float32(1 - 2.0 ** -24)
        un[:] = np.float32(1 - 2.0 ** -24)
    assert _verify([6, 3], 999, "f32", False, False, mutate=certain) == [6, 3]

    def same(t, dr, tokens, u, un, parents, cu):                # P = D: R is empty after a rejection
        t.copy_(dr)
        u[:] = 1.0
    assert _verify([4, 4], 64, "f32", True, False, mutate=same) == [1, 1]

    def nothing(t, dr, tokens, u, un, parents, cu):             # no probabilities at all: token -1
        t.zero_()
    _verify([3, 2], 77, "bf16", True, True, mutate=nothing)

    def odd(t, dr, tokens, u, un, parents, cu):                 # NaN and negative entries count as zero
        t[:, 3] = math.nan
        t[:, 5] = -1.0
        dr[:, 2] = math.nan
        tokens[1], tokens[3] = 3, 77
        tokens[2] = -1
    _verify([5, 4], 77, "f32", True, True, mutate=odd)
    _verify([5, 4], 77, "f32", False, True, mutate=odd)

    def zero_u(t, dr, tokens, u, un, parents, cu):
        t[:, :4] = 0.0
        u[:] = 0.0
        un[:] = 0.0
    _verify([5, 4], 77, "f32", True, True, mutate=zero_u)

    def one(t, dr, tokens, u, un, parents, cu):                 # a number of 1: the last token that can be drawn
        u[:] = 1.0
        un[:] = 1.0
        t[:, -3:] = 0.0
        t[:] = torch.round(t * 1024) / 1024                     # sums are exact
    _verify([5, 4], 5000, "f32", False, True, mutate=one)

    def twins(t, dr, tokens, u, un, parents, cu):               # the same token twice among siblings
        parents[1:] = 0
        tokens[1:4] = 9
        u[:] = 0.99
    for draft in (False, True):
        _verify([6], 40, "f32", draft, True, mutate=twins)
    _verify([6, 2], 40, "f32", True, True, max_rows=4)          # further rows are ignored
    _verify([2, 2], 40, "f32", True, True, max_rows=9, slots=False)

    def lost(t, dr, tokens, u, un, parents, cu):                # parents that are no parents
        parents[:] = [-1, 5, 1, 0, -3, 3, 0, 0]
    _verify([6], 40, "f32", True, True, mutate=lost)


def test_verify_large_trees():
    say("verify large trees")
    for draft in (False, True):
        _verify([1024, 700, 65, 64], 97, "f32", draft, True, back=60, noise=0.4)
        _verify([1024, 5], 97, "f32", draft, False, noise=0.05)


# -- refusals of the binding --
def test_binding_refusals():
    say("binding refusals")
    i, w = i32([0, 1, 2, 3]), i32([[0, 1], [2, 3]])
    f, h = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, 2, 64, device="cuda").bfloat16()
    freq = qcf.rope_frequencies(64, 1e4)
    plan = lambda table=w, kv=i[:2], new=i[:2], slots=i, pos=i, cu=i[:3], **k: \
        qcf.qcf_page_plan(table, kv, new, i, slots, pos, cu, 16, 4, 1, **k)
    rope = lambda kc=f, vc=f, kn=f, vn=f, slots=i, pos=i, fr=freq, **k: qcf.qcf_rope_store(kc, vc, kn, vn, slots, pos, fr, **k)
    attn = lambda out=f, q=f.clone(), cu=i[:3], kc=f, vc=f, table=w, kv=i[:2], **k: \
        qcf.qcf_tree_attn(out, q, cu, kc, vc, table, kv, 2, 2, 4, 0.1, **k)
    t = torch.zeros(4, 5, device="cuda")
    u = t[:, 0].contiguous()
    ver = lambda n=i[:2], path=w, toks=w, target=t, tokens=i, cu=i[:3], ua=u, un=u[:2], **k: \
        qcf.qcf_verify_drafts(n, path, toks, target, tokens, cu, ua, un, **k)
    for call in (lambda: plan(table=w[:1]), lambda: plan(table=w.t()), lambda: plan(kv=i[:2].long()), lambda: plan(cu=i),
                 lambda: plan(pos=i[:3]), lambda: plan(parents=i), lambda: plan(tree_mask=w), lambda: plan(kv=i[::2]),
                 lambda: plan(parents=i, tree_mask=w), lambda: plan(free_head=i), lambda: plan(pages_held=i),
                 lambda: rope(kc=h), lambda: rope(kc=None), lambda: rope(slots=None), lambda: rope(pos=None),
                 lambda: rope(fr=None), lambda: rope(slots=i[:3]), lambda: rope(fr=freq.float()), lambda: rope(fr=freq[::2]),
                 lambda: rope(kn=f[:3], vn=f[:3]), lambda: rope(q_new=f), lambda: rope(q_new=f, q_out=f[:3]),
                 lambda: rope(kn=f[:, :1]), lambda: rope(vn=f.transpose(0, 1)), lambda: rope(src_idx=i[:2]),
                 lambda: rope(kn=f, vn=f),                       # the cache itself
                 lambda: attn(out=f[:3]), lambda: attn(q=h), lambda: attn(cu=i), lambda: attn(table=w[:1]),
                 lambda: attn(kc=f[:, :1]), lambda: attn(tree_mask=w), lambda: attn(lse=u), lambda: attn(kv=i),
                 lambda: attn(workspace=torch.zeros(4, dtype=torch.uint8)), lambda: attn(q=f.transpose(0, 1)),
                 lambda: attn(out=f, q=f),                       # in place
                 lambda: ver(path=w[:1]), lambda: ver(toks=i32([[0], [1]])), lambda: ver(target=t[:3]), lambda: ver(ua=u[:3]),
                 lambda: ver(un=u), lambda: ver(tokens=i.long()), lambda: ver(draft=t[:, :4]), lambda: ver(draft=t.bfloat16()),
                 lambda: ver(slots=i), lambda: ver(parents=i[:3]), lambda: ver(target=t.t().contiguous().t())):
        with pytest.raises(qcf.QcfError):
            call()
    torch.cuda.synchronize()


# -- streams and graphs ------------------------------------------------------------------------
def test_calls_on_another_stream_and_in_a_graph():
    """A captured pass, replayed with other inputs in place and eager calls in between, gives what eager
    calls give."""
    say("decode calls in a graph")
    x = Batch([3000, 70, 0], [5, 1, 3], 8, 2, 128, "bf16", 16, True, seed=20)
    need = qcf.qcf_tree_attn_workspace_size(3, x.max_q, x.max_kv, 8, 2, 128)
    ws, ws2 = (torch.empty(need + 256, dtype=torch.uint8, device="cuda") for _ in range(2))
    out, lse = torch.full_like(x.q, 5.0), torch.full(x.q.shape[:2], 5.0, device="cuda")
    cu, kv = i32(x.cu), i32(x.kv)
    target = torch.softmax(2 * torch.randn(12, 5000, device="cuda"), 1)
    u, un = torch.rand(12, device="cuda"), torch.rand(3, device="cuda")
    tokens, par = i32(np.arange(12)), i32([-1, 0, 0, 1, 1, -1, -1, 0, 0, 0, 0, 0])
    e = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    n_out, path, toks = e(3), e(3, 5), e(3, 5)
    vws = torch.empty(qcf.qcf_verify_drafts_workspace_size(3, 5000), dtype=torch.uint8, device="cuda")
    freq = qcf.rope_frequencies(128, 1e4)
    pos, slots = i32(np.arange(12) % 7), i32(np.concatenate([x.slot[b][x.kv[b]:] for b in range(3)] + [[-1] * 3]))
    raw = torch.randn(12, 8, 128, device="cuda").bfloat16()
    kn = torch.randn(12, 2, 128, device="cuda").bfloat16()

    def step(o, l, q, w, no, pa, to):
        qcf.qcf_rope_store(x.k, x.v, kn, kn, slots, pos, freq, q_new=raw, q_out=q)
        qcf.qcf_tree_attn(o, q, cu, x.k, x.v, x.table, kv, 16, x.max_q, x.max_kv, 0.09, tree_mask=x.mask, lse=l,
                          workspace=w)
        qcf.qcf_verify_drafts(no, pa, to, target, tokens, cu, u, un, parents=par, workspace=vws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, lse, x.q, ws, n_out, path, toks)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out, lse, x.q, ws, n_out, path, toks)
    for turn in range(4):
        raw.copy_(torch.randn(12, 8, 128, device="cuda"))
        kn.copy_(torch.randn(12, 2, 128, device="cuda"))
        u.copy_(torch.rand(12, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        o2, l2, q2 = torch.full_like(out, 5.0), torch.full_like(lse, 5.0), torch.empty_like(x.q)
        no, pa, to = e(3), e(3, 5), e(3, 5)
        step(o2, l2, q2, ws2, no, pa, to)
        torch.cuda.synchronize()
        assert torch.equal(out, o2) and torch.equal(lse, l2), turn
        assert torch.equal(n_out, no) and torch.equal(path, pa) and torch.equal(toks, to), turn
