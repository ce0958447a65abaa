"""The decoding calls are declared, exported and reject bad host arguments before launching (no GPU)."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2606_05875_amd import qcf

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qcf_decode.h")
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
    assert set(decl) == {"qcf_page_plan", "qcf_rope_frequencies", "qcf_rope_store", "qcf_tree_attn_workspace_size",
                         "qcf_tree_attn", "qcf_verify_drafts_workspace_size", "qcf_verify_drafts"}
    for name, nargs in decl.items():
        assert hasattr(L, name) and len(qcf.EXPORTS[name][1]) == nargs, name


def test_page_plan_refusals(L):
    def call(**k):
        g = k.get
        return L.qcf_page_plan(g("table", A), g("stride", 10), g("cols", 10), g("batch", 4), g("kv", A), g("new", A),
                               g("held"), g("free", A), g("n_free", 8), g("head"), g("pages", 100), g("ps", 16),
                               g("max_new", 8), g("par"), g("mask"), g("words", 0), g("slots", A), g("pos", A),
                               g("n", 32), g("cu", A), g("end"), g("held_out"), g("head_out"), None)
    for bad in (dict(table=None), dict(kv=None), dict(new=None), dict(free=None), dict(slots=None), dict(pos=None),
                dict(cu=None), dict(stride=9), dict(batch=-1), dict(n=-1), dict(n_free=-1), dict(pages=-1), dict(ps=0),
                dict(ps=-16), dict(par=A), dict(mask=A), dict(par=A, mask=A, words=0), dict(par=A, mask=A, words=-1),
                dict(par=A, mask=A, words=1, max_new=33), dict(kv=MIS + 1), dict(pages=1 << 28, ps=16),
                dict(head=A, head_out=A), dict(held=B, held_out=B), dict(held_out=A), dict(end=A), dict(end=MIS + 1)):
        assert call(**bad) == INVALID, bad
    assert call(ps=24) == UNSUPPORTED
    assert call(par=A, mask=A, words=33, max_new=1025) == UNSUPPORTED


def test_rope_frequency_refusals(L):
    buf = (ctypes.c_double * 64)()
    f = lambda dim=128, theta=1e4, sc=0, factor=2.0, lo=1.0, hi=4.0, tl=100.0, p=buf: \
        L.qcf_rope_frequencies(p, dim, theta, sc, factor, lo, hi, tl)
    assert f() == OK and f(sc=1) == OK and f(sc=2) == OK
    for bad in (dict(p=None), dict(dim=0), dict(dim=7), dict(theta=0.0), dict(theta=math.inf), dict(theta=math.nan),
                dict(sc=1, factor=0.0), dict(sc=2, factor=math.inf), dict(sc=2, lo=4.0), dict(sc=2, tl=0.0)):
        assert f(**bad) == INVALID, bad
    assert f(sc=3) == UNSUPPORTED and f(sc=-1) == UNSUPPORTED
    with pytest.raises(qcf.QcfError):
        qcf.qcf_rope_frequencies(torch.empty(4), 1e4)
    with pytest.raises(qcf.QcfError):
        qcf.rope_frequencies(16, 1e4, device="cpu", scaling="cubic")
    with pytest.raises(qcf.QcfError):
        qcf.rope_frequencies(15, 1e4, device="cpu")


def test_rope_store_refusals(L):
    def call(**k):
        g = k.get
        return L.qcf_rope_store(g("kc", A), g("vc", B), g("slots_n", 100), g("cs", 1024), g("qo", A), g("kn", C),
                                g("vn", C), g("ns", 1024), g("qn", C), g("qs", 4096), g("src_n", 10), g("src"),
                                g("dt", BF16), g("n", 10), g("slots", A), g("pos", A), g("freq", A), g("dim", 128), 0,
                                g("mag", 1.0), g("hq", 32), 8, g("d", 128), None)
    for bad in (dict(kc=None), dict(vc=None), dict(kn=None), dict(vn=None), dict(slots=None), dict(cs=1000),
                dict(ns=1028), dict(qn=None), dict(qo=MIS), dict(qs=4000), dict(pos=None), dict(freq=None),
                dict(dim=0), dict(dim=144), dict(dim=-16), dict(mag=math.nan), dict(mag=math.inf), dict(n=-1),
                dict(src_n=-1), dict(slots_n=-1), dict(hq=30), dict(kn=A), dict(vn=B), dict(qn=A), dict(freq=MIS),
                dict(kc=MIS), dict(pos=None, freq=None, dim=0, mag=2.0), dict(src=MIS + 1)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dt=5), dict(d=96), dict(hq=24), dict(dim=24)):
        assert call(**bad) == UNSUPPORTED, bad
    # nothing to do
    assert call(n=0) == OK and call(src_n=0) == OK
    assert call(kc=None, vc=None, qo=None, kn=None, vn=None, slots=None) == OK


def test_tree_attn_refusals(L):
    need = L.qcf_tree_attn_workspace_size(4, 8, 1 << 20, 32, 8, 128, BF16)
    assert L.qcf_tree_attn_workspace_size(4, 8, 100, 32, 8, 96, BF16) == 0

    def call(**k):
        g = k.get
        return L.qcf_tree_attn(g("out", A), g("lse"), g("q", B), g("n", 32), g("cu", A), g("kc", A + 4096), g("vc", C),
                               g("slots", 1 << 20), g("stride", 1024), g("table", A), g("ts", 70000),
                               g("cols", 70000), g("ps", 16), g("kv", A), g("mask"), g("words", 0), g("dt", BF16),
                               g("batch", 4), g("max_q", 8), g("max_kv", 1 << 20), g("hq", 32), 8, g("d", 128),
                               g("scale", 0.1), g("ws", A), g("wsb", need), None)
    for bad in (dict(out=None), dict(q=None), dict(cu=None), dict(kc=None), dict(vc=None), dict(table=None),
                dict(kv=None), dict(out=B), dict(q=MIS), dict(lse=MIS + 1), dict(stride=1000), dict(ts=69999),
                dict(ps=0), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(mask=A), dict(n=-1),
                dict(batch=-1), dict(max_q=-1), dict(max_kv=-1), dict(slots=-1), dict(hq=36)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dt=5), dict(d=96), dict(hq=24), dict(ps=48), dict(stride=1 << 26), dict(max_kv=2 ** 31 - 5),
                dict(batch=1 << 14, max_q=1 << 14)):
        assert call(**bad) == UNSUPPORTED, bad
    if need:
        for bad in (dict(ws=None), dict(ws=A + 16), dict(wsb=need - 1)):
            assert call(**bad) == WORKSPACE, bad
    for nothing in (dict(n=0), dict(batch=0), dict(max_q=0)):
        assert call(**nothing, out=None, q=None, ws=None, wsb=0) == OK


def test_tree_attn_workspace_is_monotone(L):
    """The size for (batch, max_q, max_kv) covers every smaller call."""
    size = lambda b, q, kv, d=128, dt=BF16: L.qcf_tree_attn_workspace_size(b, q, kv, 32, 8, d, dt)
    for dt in (F32, BF16):
        for d in (64, 128):
            values = [(b, q, kv) for b in (1, 2, 3, 16, 64, 300) for q in (1, 2, 5, 8, 9, 17, 40, 64, 200)
                      for kv in (1, 63, 64, 257, 1000, 4096, 33000, 140000)]
            got = {x: size(*x, d, dt) for x in values}
            for x in values:
                for y in values:
                    if all(a <= b for a, b in zip(x, y)):
                        assert got[x] <= got[y], (x, y, got[x], got[y])


def test_verify_refusals(L):
    need = L.qcf_verify_drafts_workspace_size(4, 1000)
    assert need > 0 and L.qcf_verify_drafts_workspace_size(0, 1000) == 0

    def call(**k):
        g = k.get
        return L.qcf_verify_drafts(g("n_out", A), g("path", A), g("out", A), g("target", A), g("draft", A),
                                   g("stride", 1000), g("dt", F32), g("n", 20), g("vocab", 1000), g("tok", A),
                                   g("par"), g("batch", 4), g("cu", A), g("max_rows", 8), g("u", A), g("un", A),
                                   g("slots"), g("ms"), g("md"), g("ws", A), g("wsb", need), None)
    for bad in (dict(n_out=None), dict(path=None), dict(out=None), dict(target=None), dict(target=MIS), dict(draft=MIS),
                dict(stride=999), dict(n=-1), dict(vocab=0), dict(tok=None), dict(batch=-1), dict(cu=None),
                dict(max_rows=-1), dict(u=None), dict(un=None), dict(slots=A), dict(ms=A), dict(md=A),
                dict(slots=A, ms=A), dict(par=MIS + 1)):
        assert call(**bad) == INVALID, bad
    assert call(dt=3) == UNSUPPORTED and call(max_rows=1025) == UNSUPPORTED
    assert call(vocab=(1 << 28) + 1, stride=1 << 29) == UNSUPPORTED
    for bad in (dict(ws=None), dict(ws=A + 16), dict(wsb=need - 1)):
        assert call(**bad) == WORKSPACE, bad
    assert call(batch=0, n_out=None, path=None, out=None, target=None, tok=None, ws=None, wsb=0) == OK


def test_the_binding_refuses_host_tensors():
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64)
    for call in (lambda: qcf.qcf_page_plan(i.view(2, 2), i, i, i, i, i, i, 16, 4, 1),
                 lambda: qcf.qcf_rope_store(f, f, f, f, i, i, torch.ones(32, dtype=torch.float64)),
                 lambda: qcf.qcf_rope_store(None, None, None, None, None),
                 lambda: qcf.qcf_tree_attn(f, f, i, f, f, i.view(2, 2), i, 16, 1, 4, 0.1),
                 lambda: qcf.qcf_verify_drafts(i, i.view(2, 2), i.view(2, 2), f, i, i, f, f)):
        with pytest.raises(qcf.QcfError):
            call()
