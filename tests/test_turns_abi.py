"""The calls for further turns are declared, exported and reject bad host arguments before launching (no GPU)."""
import math
import os
import re

import pytest
import torch

from paper_2606_05875_amd import qcf

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qcf_turns.h")
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
A, B, C, MIS = 0x10000, 0x20000, 0x30000, 0x10004    # fake addresses: these calls never get to a kernel
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(qcf.lib_path()):
        from paper_2606_05875_amd.build import build
        build(verbose=False)
    return qcf.lib()


def test_declared_and_bound(L):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    decl = {m.group(1): m.group(2).count(",") + 1
            for m in re.finditer(r"\b(?:qcf_status|size_t)\s+(qcf_\w+)\s*\(([^;]*?)\)\s*;", text, re.S)}
    assert set(decl) == {"qcf_norm_rope_store", "qcf_chunk_attn_workspace_size", "qcf_chunk_attn",
                         "qcf_shape_logits_workspace_size", "qcf_shape_logits", "qcf_page_fork", "qcf_copy_pages",
                         "qcf_page_release_workspace_size", "qcf_page_release"}
    for name, nargs in decl.items():
        assert hasattr(L, name) and len(qcf.EXPORTS[name][1]) == nargs, name
        assert name in qcf.__all__, name


def test_norm_rope_store_refusals(L):
    def call(**k):
        g = k.get
        return L.qcf_norm_rope_store(
            g("kc", A), g("vc", B), g("slots_n", 100), g("cs", 1024), g("qo", A), g("kn", C), g("vn", C), g("ns", 1024),
            g("qn", C), g("qs", 4096), g("src_n", 10), g("src"), g("dt", BF16), g("n", 10), g("slots", A), g("pos", A),
            g("freq", A), g("dim", 128), 0, g("mag", 1.0), g("qw", B), g("qws", 0), g("kw", B), g("kws", 128),
            g("eps", 1e-6), g("hq", 32), 8, g("d", 128), None)
    for bad in (dict(kc=None), dict(vc=None), dict(kn=None), dict(vn=None), dict(slots=None), dict(cs=1000),
                dict(ns=1028), dict(qn=None), dict(qo=MIS), dict(qs=4000), dict(pos=None), dict(freq=None),
                dict(dim=0), dict(dim=144), dict(dim=-16), dict(mag=math.nan), dict(n=-1), dict(src_n=-1),
                dict(slots_n=-1), dict(hq=30), dict(kn=A), dict(vn=B), dict(qn=A), dict(freq=MIS), dict(kc=MIS),
                dict(src=MIS + 1), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(qw=MIS), dict(kw=MIS),
                dict(qws=64), dict(qws=-128), dict(kws=132), dict(qw=None, qws=128), dict(kw=None)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dt=5), dict(d=96), dict(hq=24), dict(dim=24)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(n=0) == OK and call(src_n=0) == OK and call(n=0, eps=0.0, qw=None, kw=None, kws=0) == OK
    assert call(kc=None, vc=None, qo=None, kn=None, vn=None, slots=None) == OK


def test_chunk_attn_refusals(L):
    need = L.qcf_chunk_attn_workspace_size(4, 8, 1 << 20, 32, 8, 128, BF16)
    assert L.qcf_chunk_attn_workspace_size(4, 8, 100, 32, 8, 96, BF16) == 0
    assert L.qcf_chunk_attn_workspace_size(0, 8, 100, 32, 8, 128, BF16) == 0

    def call(**k):
        g = k.get
        return L.qcf_chunk_attn(g("out", A), g("lse"), g("q", B), g("n", 32), g("cu", A), g("kc", A + 4096), g("vc", C),
                                g("slots", 1 << 20), g("stride", 1024), g("table", A), g("ts", 70000),
                                g("cols", 70000), g("ps", 16), g("kv", A), g("window", 0), g("dt", BF16),
                                g("batch", 4), g("max_q", 8), g("max_kv", 1 << 20), g("hq", 32), 8, g("d", 128),
                                g("scale", 0.1), g("ws", A), g("wsb", need), None)
    for bad in (dict(out=None), dict(q=None), dict(cu=None), dict(kc=None), dict(vc=None), dict(table=None),
                dict(kv=None), dict(out=B), dict(out=C), dict(q=MIS), dict(lse=MIS + 1), dict(stride=1000), dict(ts=69999),
                dict(ps=0), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(n=-1), dict(window=-1),
                dict(batch=-1), dict(max_q=-1), dict(max_kv=-1), dict(slots=-1), dict(hq=36)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dt=5), dict(d=96), dict(hq=24), dict(ps=48), dict(ps=8), dict(ps=1), dict(stride=1 << 26),
                dict(max_kv=2 ** 31 - 5), dict(max_q=(1 << 20) + 1), dict(batch=1 << 20, max_q=1 << 20),
                dict(batch=(1 << 30) + 1, max_q=1, hq=8)):
        assert call(**bad) == UNSUPPORTED, bad
    if need:
        for bad in (dict(ws=None), dict(ws=A + 16), dict(wsb=need - 1)):
            assert call(**bad) == WORKSPACE, bad
    for nothing in (dict(n=0), dict(batch=0), dict(max_q=0)):
        assert call(**nothing, out=None, q=None, ws=None, wsb=0) == OK


def test_chunk_attn_without_tokens_needs_its_workspace(L):
    """Rows that see no token (max_kv = 0, no table, no pool) go through the same kernels, which use the workspace."""
    for dt in (F32, BF16):
        for d in (64, 128):
            need = L.qcf_chunk_attn_workspace_size(4, 8, 0, 32, 8, d, dt)
            assert 0 < need <= L.qcf_chunk_attn_workspace_size(4, 8, 1, 32, 8, d, dt)

            def call(**k):
                g = k.get
                return L.qcf_chunk_attn(A, None, B, 32, A, g("kc"), g("kc"), g("slots", 1 << 20), 8 * d, g("table"), g("cols", 70000),
                                        g("cols", 70000), 16, A, 0, dt, 4, 8, g("max_kv", 0), 32, 8, d, 0.1, g("ws"),
                                        g("wsb", 0), None)
            pool = dict(kc=C, table=A)
            for nothing in ({}, pool, dict(cols=0, max_kv=100), dict(slots=15, max_kv=100), dict(pool, slots=0, cols=0)):
                for bad in (dict(), dict(wsb=need), dict(ws=A + 16, wsb=need), dict(ws=A, wsb=need - 1)):
                    assert call(**nothing, **bad) == WORKSPACE, (nothing, bad)
    for x in ((0, 8, 0), (4, 0, 0), (-1, 8, 0), (4, -1, 0)):
        assert L.qcf_chunk_attn_workspace_size(*x, 32, 8, 128, BF16) == 0


def test_chunk_attn_workspace_grows_from_no_tokens_on(L):
    for dt in (F32, BF16):
        for batch, max_q in ((1, 1), (16, 9), (300, 4000)):
            sizes = [L.qcf_chunk_attn_workspace_size(batch, max_q, kv, 32, 8, 64, dt) for kv in (0, 1, 63, 64, 4096, 33000)]
            assert sizes == sorted(sizes) and sizes[0] > 0


def test_chunk_attn_workspace_is_monotone(L):
    """The size for (batch, max_q, max_kv) covers every smaller call."""
    for dt in (F32, BF16):
        for d in (64, 128):
            values = [(b, q, kv) for b in (1, 2, 16, 300) for q in (1, 9, 200, 4000) for kv in (1, 64, 1000, 4096, 33000)]
            got = {x: L.qcf_chunk_attn_workspace_size(*x, 32, 8, d, dt) for x in values}
            for x in values:
                for y in values:
                    if all(a <= b for a, b in zip(x, y)):
                        assert got[x] <= got[y], (x, y, got[x], got[y])


def test_shape_logits_refusals(L):
    vocab = 100000
    need = L.qcf_shape_logits_workspace_size(20, vocab)
    assert need > 0 and L.qcf_shape_logits_workspace_size(0, vocab) == 0 and L.qcf_shape_logits_workspace_size(3, 10) == 0
    assert L.qcf_shape_logits_workspace_size(21, vocab) >= need

    def call(**k):
        g = k.get
        return L.qcf_shape_logits(
            g("out", A), g("os", vocab), g("odt", F32), g("z", B), g("zs", vocab), g("dt", F32), g("n", 20),
            g("vocab", vocab), g("batch", 4), g("cu", A), g("hist", A), g("hs", 50), g("width", 50), g("prompt", A),
            g("hl", A), g("tok", A), g("mask", A), g("words", 1), g("rep"), g("pres"), g("freq"), g("bs", A), g("bt", A),
            g("bv", A), g("nb", 5), g("allowed", A), g("aw", 3125), g("temp", A), g("prob", 1), g("ws", A),
            g("wsb", need), None)
    for bad in (dict(out=None), dict(z=None), dict(out=MIS + 1), dict(z=MIS + 2), dict(os=vocab - 1), dict(zs=vocab - 1),
                dict(n=-1), dict(vocab=0), dict(batch=-1), dict(cu=None), dict(hist=None), dict(hl=None), dict(hs=49),
                dict(width=-1), dict(tok=None), dict(words=0), dict(bs=None), dict(bt=None), dict(bv=None), dict(nb=-1),
                dict(aw=3124), dict(z=A, odt=BF16), dict(z=A, os=vocab + 8), dict(rep=MIS + 1), dict(temp=MIS + 2),
                dict(allowed=MIS + 1), dict(hist=None, hl=None, prompt=None), dict(hist=None, hl=None, width=0)):
        assert call(**bad) == INVALID, bad
    assert call(dt=3) == UNSUPPORTED and call(odt=2) == UNSUPPORTED
    assert call(vocab=(1 << 28) + 1, os=1 << 29, zs=1 << 29) == UNSUPPORTED
    assert call(batch=(1 << 30) + 1) == UNSUPPORTED and call(width=(1 << 30) + 1, hs=1 << 31) == UNSUPPORTED
    for bad in (dict(ws=None), dict(ws=A + 16), dict(wsb=need - 1)):
        assert call(**bad) == WORKSPACE, bad
    for nothing in (dict(n=0), dict(batch=0)):
        assert call(**nothing, out=None, z=None, cu=None, ws=None, wsb=0) == OK


def test_page_fork_refusals(L):
    def call(**k):
        g = k.get
        return L.qcf_page_fork(g("to", A), g("tos", 10), g("kvo", A + 64), g("ho", A + 128), g("table", B), g("ts", 10),
                               g("cols", 10), g("batch", 4), g("kv", B + 64), g("src", B + 128), g("keep"), g("free", C),
                               g("n_free", 8), g("head"), g("pages", 100), g("ps", 16), g("fo", A + 192), g("cs", A + 256),
                               g("cd", A + 320), g("cr", A + 384), None)
    for bad in (dict(to=None), dict(kvo=None), dict(ho=None), dict(table=None), dict(kv=None), dict(src=None),
                dict(free=None), dict(fo=None), dict(cs=None), dict(cd=None), dict(cr=None), dict(tos=9), dict(ts=9),
                dict(batch=-1), dict(n_free=-1), dict(pages=-1), dict(ps=0), dict(pages=1 << 28), dict(to=B),
                dict(kvo=B + 64), dict(ho=B + 64), dict(head=A + 192), dict(keep=A + 64), dict(fo=C), dict(kv=MIS + 1),
                dict(kvo=A), dict(cs=A + 128), dict(cr=A + 320), dict(fo=A + 64)):
        assert call(**bad) == INVALID, bad
    assert call(ps=24) == UNSUPPORTED and call(batch=1 << 22) == UNSUPPORTED


def test_copy_pages_refusals(L):
    def call(**k):
        g = k.get
        return L.qcf_copy_pages(g("pools", A), g("n", 4), g("slots", 1024), g("rb", 2048), g("rs", 2304), g("ps", 16),
                                g("src", B), g("dst", C), g("rows"), g("pairs", 5), None)
    for bad in (dict(pools=None), dict(pools=MIS), dict(src=None), dict(dst=None), dict(n=-1), dict(slots=-1), dict(rb=0),
                dict(rb=2040), dict(rs=2040), dict(rs=2312), dict(ps=0), dict(pairs=-1), dict(rows=MIS + 1)):
        assert call(**bad) == INVALID, bad
    assert call(ps=24) == UNSUPPORTED and call(pairs=1 << 30) == UNSUPPORTED
    for nothing in (dict(n=0), dict(pairs=0), dict(slots=8)):
        assert call(**nothing, pools=None, src=None, dst=None) == OK


def test_page_release_refusals(L):
    need = L.qcf_page_release_workspace_size(400, 1000, 100000)
    assert need > 0 and L.qcf_page_release_workspace_size(4, 10, 100) == 0 and L.qcf_page_release_workspace_size(0, 10, 5) == 0
    assert need <= L.qcf_page_release_workspace_size(401, 1001, 100001)

    def call(**k):
        g = k.get
        return L.qcf_page_release(g("tb", A), g("bs", 1000), g("hb", A + 64), g("ta", A), g("as_", 1000), g("ha", A + 128),
                                  g("cols", 1000), g("batch", 400), g("free", B), g("n_free", 8), g("head", C),
                                  g("fo", C + 64), g("pages", 100000), g("ws", B + 256), g("wsb", need), None)
    for bad in (dict(tb=None), dict(hb=None), dict(ta=None), dict(ha=None), dict(free=None), dict(head=None),
                dict(fo=None), dict(bs=999), dict(as_=999), dict(batch=-1), dict(cols=-1), dict(n_free=-1), dict(pages=-1),
                dict(pages=1 << 31), dict(fo=C), dict(free=A), dict(hb=MIS + 1), dict(free=C)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(batch=1 << 22), dict(batch=1 << 12, cols=1 << 21, bs=1 << 21, as_=1 << 21)):
        assert call(**bad) == UNSUPPORTED, bad
    for bad in (dict(ws=None), dict(ws=B + 16), dict(wsb=need - 1)):
        assert call(**bad) == WORKSPACE, bad


def test_page_release_outputs_are_not_one_another(L):
    """The new head is written while other threads write the list."""
    call = lambda free, out: L.qcf_page_release(A, 10, A + 64, A, 10, A + 128, 10, 4, free, 8, C, out, 100, None, 0, None)
    assert call(B, B) == INVALID


def test_the_binding_refuses_host_tensors():
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64)
    t = i.view(2, 2)
    for call in (lambda: qcf.qcf_norm_rope_store(f, f, f, f, i, i, torch.ones(32, dtype=torch.float64)),
                 lambda: qcf.qcf_norm_rope_store(None, None, None, None, None),
                 lambda: qcf.qcf_chunk_attn(f, f, i, f, f, t, i, 16, 1, 4, 0.1),
                 lambda: qcf.qcf_shape_logits(f[0], f[0], i),
                 lambda: qcf.qcf_page_fork(t, i, i, t, i, i, i, 16, 4),
                 lambda: qcf.PoolSet([f]), lambda: qcf.PoolSet([]),
                 lambda: qcf.qcf_copy_pages([f], i, i, 16),
                 lambda: qcf.qcf_page_release(t, i, t, i, i, i[:1], i[:1], 4)):
        with pytest.raises(qcf.QcfError):
            call()
