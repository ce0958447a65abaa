"""Further turns on paged caches, the calls together: questions, drafted answers from shaped probabilities, requests that
continue others, are taken back and end; against the float64 oracle, and captured into a graph."""
import math

import numpy as np
import pytest
import torch

from oracle import decode as D
from oracle import turns as T
from paper_2606_05875_amd import qcf
from paper_2606_05875_amd.turns import FEW_VECTORS, TurnCache, TurnStep
from test_gpu_decode import DT, HALF, host, i32, say, within
from test_gpu_draft import token_rows

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.float32))).cuda()


class Model:
    """Random projections, logits and weights of a pass of fixed size."""

    def __init__(self, rng, dtype, layers, hq, hkv, d, vocab, norms=True):
        self.rng, self.dtype, self.layers, self.hq, self.hkv, self.d, self.vocab = rng, dtype, layers, hq, hkv, d, vocab
        w = lambda: torch.from_numpy(1 + 0.3 * rng.standard_normal(d)).to(DT[dtype]).cuda()
        self.qn, self.kn = ([w() for _ in range(layers)] for _ in range(2)) if norms else (None, None)

    def rows(self, n):
        qkv = torch.from_numpy(self.rng.standard_normal((n, (self.hq + 2 * self.hkv) * self.d))).to(DT[self.dtype]).cuda()
        q, k, v = qkv.split([self.hq * self.d, self.hkv * self.d, self.hkv * self.d], 1)
        return q.view(n, self.hq, self.d), k.view(n, self.hkv, self.d), v.view(n, self.hkv, self.d)


class Mirror:
    """What every request holds, on the host: its tokens' keys and values per layer."""

    def __init__(self, layers, batch, hkv, d):
        e = lambda: np.zeros((0, hkv, d))
        self.k = [[e() for _ in range(batch)] for _ in range(layers)]
        self.v = [[e() for _ in range(batch)] for _ in range(layers)]

    def lengths(self):
        return np.array([x.shape[0] for x in self.k[0]])

    def continue_from(self, source, keep):
        for lst in (self.k, self.v):
            for layer in range(len(lst)):
                old = lst[layer]
                lst[layer] = [old[s][:max(0, keep[b])].copy() if 0 <= s < len(old) else old[0][:0].copy()
                              for b, s in enumerate(source)]


def check_cache(cache, mirror):
    """Tables, lengths, free list and contents: every page is free or held, started pages belong to one request."""
    kv, held = cache.kv_len.cpu().numpy(), cache.pages_held.cpu().numpy()
    np.testing.assert_array_equal(kv, mirror.lengths())
    table, ps = cache.block_table.cpu().numpy(), cache.page_size
    assert (held * ps >= kv).all()
    head = int(cache.free_head[0])
    free = cache.free_pages.cpu().numpy()[head:]
    used = {int(p) for b in range(len(kv)) for p in table[b, :held[b]]}
    assert len(set(free)) == len(free) and not used & set(free.tolist()) and len(used) + len(free) == cache.n_pages
    owners = [int(table[b, kv[b] // ps]) for b in range(len(kv)) if kv[b] % ps]
    assert len(set(owners)) == len(owners)
    for b in range(len(kv)):
        if not kv[b]:
            continue
        at = torch.from_numpy(token_rows(cache, b, int(kv[b]))).cuda()
        for layer in range(len(cache.k)):
            np.testing.assert_array_equal(host(cache.k[layer][at]), mirror.k[layer][b])
            np.testing.assert_array_equal(host(cache.v[layer][at]), mirror.v[layer][b])


def run_pass(step, model, new, mirror, rng, check=True):
    """A pass of chunks; the mirror gets the stored rows; outputs against the oracle."""
    cache = step.cache
    lens, cu = mirror.lengths(), np.concatenate([[0], np.cumsum(new)])
    step.plan(i32(new))
    outs, stored = [], []
    for layer in range(model.layers):
        q, k, v = model.rows(step.max_rows)
        step.store(layer, q, k, v)
        n = int(cu[-1])
        pos = np.concatenate([np.arange(a) + b for a, b in zip(new, lens)] + [[]]).astype(np.int64)
        np.testing.assert_array_equal(step.positions.cpu().numpy()[:n], pos)
        slots = step.slots.cpu().numpy()[:n]
        fr = step.freq.cpu().numpy()
        for got, src, w in ((host(step.q)[:n], q, model.qn), (host(cache.k[layer])[slots], k, model.kn)):
            y, size = T.norm_rope(host(src)[:n], pos, fr, None if w is None else host(w[layer]), step.eps if w else 0.0,
                                  step.interleaved, step.magnitude) if w else D.rope(host(src)[:n], pos, fr, step.interleaved, step.magnitude)
            within(got, y, HALF[model.dtype] * np.abs(y) + (model.d / 2 + 9) * E * size * 1.01, "rows")
        np.testing.assert_array_equal(host(cache.v[layer])[slots], host(v)[:n])
        step.out.fill_(7.0)
        out = host(step.attend(layer))
        assert (out[n:] == 7.0).all()
        outs.append(out)
        stored.append((host(cache.k[layer])[slots], host(cache.v[layer])[slots], host(step.q)[:n]))
    for layer, (k, v, q) in enumerate(stored):
        for b in range(len(new)):
            a, z = cu[b], cu[b + 1]
            mk = np.concatenate([mirror.k[layer][b], k[a:z]])
            mv = np.concatenate([mirror.v[layer][b], v[a:z]])
            if z > a and check:
                see = T.chunk_see(new[b], int(lens[b]), step.window[layer])
                want, _, absv, absx = D.tree_attention(q[a:z], mk, mv, see, step.scale)
                off = model.d * E * absx + 3 * 2.0 ** -23 * 2 * absx + (see.shape[1] + 16) * E
                within(outs[layer][a:z], want, HALF[model.dtype] * np.abs(want)
                       + (2 * off + (2.0 ** -8 if model.dtype == "bf16" else 0))[..., None] * absv, f"layer {layer} request {b}")
            mirror.k[layer][b], mirror.v[layer][b] = mk, mv


@pytest.mark.parametrize("dtype,ps,window,norms,interleaved", [("bf16", 16, (0, 24), True, False), ("f32", 32, 0, True, True),
                                                               ("bf16", 64, 0, False, False), ("f32", 16, (40, 0), False, False)])
def test_turns(dtype, ps, window, norms, interleaved):
    say("turns", dtype, ps, window, norms, interleaved)
    rng = np.random.default_rng(5)
    layers, hq, hkv, d, B, vocab, pages = 2, 8, 2, 64, 6, 700, 60
    model = Model(rng, dtype, layers, hq, hkv, d, vocab, norms)
    cache = TurnCache(layers, pages, ps, hkv, d, B, 30, DT[dtype])
    cache.free_pages.copy_(i32(rng.permutation(pages)))
    freq = qcf.rope_frequencies(48, 1e4)
    step = TurnStep(cache, 300, 130, hq, freq, interleaved=interleaved, magnitude=1.1, vocab=vocab, q_norm=model.qn, k_norm=model.kn,
                    window=window)
    assert step.max_new * hq // hkv > FEW_VECTORS
    mirror = Mirror(layers, B, hkv, d)
    run_pass(step, model, [130, 40, 7, 0, 64, 1], mirror, rng)          # prompts
    step.commit(all_rows=True)
    check_cache(cache, mirror)
    # request 3 is empty: it and request 5 continue request 0, request 2 ends, 4 is taken back
    L = mirror.lengths()
    source, keep = [0, 1, -1, 0, 4, 0], [130, 40, 9, 130, 33, 77]
    cache.continue_from(i32(source), i32(keep))
    mirror.continue_from(source, keep)
    check_cache(cache, mirror)
    run_pass(step, model, [3, 20, 50, 11, 0, 90], mirror, rng)          # questions, some over shared pages
    step.commit(all_rows=True)
    check_cache(cache, mirror)
    # everyone continues someone else, in a ring; then all but two end, and the cache fills up again
    source = [1, 2, 3, 4, 5, 0]
    cache.continue_from(i32(source))
    mirror.continue_from(source, [10 ** 6] * B)
    check_cache(cache, mirror)
    keep = [0, 10 ** 6, 0, 0, 5, 0]
    cache.keep(i32(keep))
    mirror.continue_from(list(range(B)), keep)
    check_cache(cache, mirror)
    run_pass(step, model, [30, 2, 100, 30, 9, 100], mirror, rng)
    step.commit(all_rows=True)
    check_cache(cache, mirror)
    cache.keep(i32([0] * B))
    mirror.continue_from(list(range(B)), [0] * B)
    check_cache(cache, mirror)
    assert int(cache.free_head[0]) == 0 and sorted(cache.free_pages.tolist()) == list(range(pages))


def test_an_answer_from_shaped_probabilities():
    """Drafted chains verified against shaped probabilities: history in the cache, drafts along the rows, pages of rejected
    drafts given back."""
    say("answers from shaped probabilities")
    rng = np.random.default_rng(6)
    layers, hq, hkv, d, B, vocab, max_new = 1, 4, 2, 64, 3, 500, 5
    cache = TurnCache(layers, 40, 16, hkv, d, B, 12, torch.float32)
    freq = qcf.rope_frequencies(64, 1e4)
    model = Model(rng, "f32", layers, hq, hkv, d, vocab, False)
    prompt, step = TurnStep(cache, 60, 30, hq, freq), TurnStep(cache, B * max_new + 2, max_new, hq, freq, vocab=vocab)
    mirror = Mirror(layers, B, hkv, d)
    lens = [17, 30, 4]
    run_pass(prompt, model, lens, mirror, rng)
    prompt.commit(all_rows=True)
    history = rng.integers(0, 40, (B, 100))
    said = [list(history[b, :lens[b]]) for b in range(B)]
    hist = i32(history)
    pen = dict(repetition=f32([1.3, 1.0, 2.0]), presence=f32([0.5, 0, 0.1]), frequency=f32([0.2, 0.3, 0]),
               temperature=f32([1.0, 0.7, 0.0]))
    for turn in range(6):
        new = np.array([5, 3, 4])
        cu = np.concatenate([[0], np.cumsum(new)])
        lens_now = mirror.lengths()
        run_pass(step, model, new, mirror, rng)
        rows = step.max_rows
        logits = torch.from_numpy(2 * rng.standard_normal((rows, vocab))).float().cuda()
        tokens = rng.integers(0, 40, rows)
        target = host(step.shape(logits, tokens=i32(tokens), history=hist, prompt_len=i32(lens), **pen))
        want = []
        for b in range(B):
            for i in range(new[b]):
                p, _ = T.shape_logits(host(logits)[cu[b] + i], said[b][:lens[b]], said[b][lens[b]:] + list(tokens[cu[b]:cu[b] + i + 1]),
                                      *(float(pen[k][b]) for k in ("repetition", "presence", "frequency")),
                                      temperature=float(pen["temperature"][b]))
                want.append(p)
        # (test_gpu_turns' bound: |z| below 12, T from 0.7, so 4 * 8 * 2^-24 * 12 / 0.7 and (2 * 24 / 0.7 + 71) * 2^-24)
        np.testing.assert_allclose(target[:cu[-1]], np.array(want), rtol=4.2e-5, atol=2.0 ** -125)
        u, un = rng.random(rows).astype(np.float32) * np.float32(0.05), rng.random(B).astype(np.float32)
        step.verify(step.target, i32(tokens), f32(u), f32(un))
        step.commit()
        n_out, toks = step.n_out.cpu().numpy(), step.tokens_out.cpu().numpy()
        for b in range(B):
            path, out = D.verify(target[cu[b]:cu[b + 1]], None, tokens[cu[b]:cu[b + 1]], None, u[cu[b]:cu[b + 1]], un[b])
            assert n_out[b] == len(path) and list(toks[b, :len(out)]) == out
            row = [int(tokens[cu[b]])] + out[:-1]
            said[b] += row
            history[b, lens_now[b]:lens_now[b] + len(row)] = row
        hist = i32(history)
        keep = lens_now + n_out
        cache.keep(i32(keep))                                           # rejected rows' pages go back
        mirror.continue_from(list(range(B)), keep)
        check_cache(cache, mirror)


def test_the_first_token_after_a_question():
    """One row of logits per request, its last: the question is cached by then, so its tokens count from the history."""
    say("the first token after a question")
    rng = np.random.default_rng(12)
    layers, hq, hkv, d, B, vocab = 1, 8, 2, 64, 3, 9000
    cache = TurnCache(layers, 40, 16, hkv, d, B, 12)
    model = Model(rng, "bf16", layers, hq, hkv, d, vocab)
    step = TurnStep(cache, 260, 100, hq, qcf.rope_frequencies(64, 1e4), q_norm=model.qn, k_norm=model.kn)
    mirror = Mirror(layers, B, hkv, d)
    history, prompt = rng.integers(0, 60, (B, 192)), [10, 0, 100]
    for new in ([10, 90, 100], [70, 1, 66]):
        run_pass(step, model, new, mirror, rng)
        step.commit(all_rows=True)
    logits, rep, freq, temp = rng.standard_normal((B, vocab)).astype(np.float32), [1.3, 0.8, 1.0], [0.2, 0.1, -0.3], [1.0, 0.5, 2.0]
    rows, target = i32(np.arange(B + 1)), torch.empty((B, vocab), device="cuda")
    qcf.qcf_shape_logits(target, f32(logits), rows, history=i32(history), prompt_len=i32(prompt), hist_len=cache.kv_len,
                         repetition=f32(rep), frequency=f32(freq), temperature=f32(temp))
    want = np.array([T.shape_logits(logits[b], history[b, :prompt[b]], history[b, prompt[b]:n], float(np.float32(rep[b])), 0.0,
                                    float(np.float32(freq[b])), temperature=temp[b])[0] for b, n in enumerate(mirror.lengths())])
    # (test_gpu_turns' bound: |z| below 5 + 0.3 * 170, T from 0.5, so 4 * 8 * 2^-24 * 56 / 0.5 and (2 * 61 / 0.5 + 79) * 2^-24)
    np.testing.assert_allclose(host(target), want, rtol=2.4e-4, atol=2.0 ** -125)
    n_out, path, toks = i32([0] * B), i32([[0]] * B), i32([[0]] * B)
    u = np.array([0.1, 0.5, 0.9])
    qcf.qcf_verify_drafts(n_out, path, toks, target, i32([0] * B), rows, f32([0.5] * B), f32(u))
    for b, t in enumerate(toks.view(-1).tolist()):                      # drawn where the running sum passes u
        c = np.cumsum(want[b])
        assert c[t] >= u[b] - 1e-3 and (t == 0 or c[t - 1] <= u[b] + 1e-3)


def test_turns_in_a_graph():
    """A captured turn (fork, chunk, shaped probabilities) replays beside eager ones with the same results."""
    say("turns in a graph")
    rng = np.random.default_rng(7)
    layers, hq, hkv, d, B, vocab = 2, 8, 2, 64, 4, 9000
    model = Model(rng, "bf16", layers, hq, hkv, d, vocab)
    freq = qcf.rope_frequencies(64, 1e4)
    rows = [model.rows(400) for _ in range(layers)]
    logits = torch.from_numpy(rng.standard_normal((400, vocab))).bfloat16().cuda()
    tokens, history = i32(rng.integers(0, vocab, 400)), i32(rng.integers(0, 50, (B, 600)))
    rep = f32([1.2] * B)
    new, source, keep = i32([100, 0, 100, 80]), i32([0, 0, 2, 0]), i32([500, 70, 40, 33])

    def fresh():
        cache = TurnCache(layers, 90, 16, hkv, d, B, 40)
        for x in cache.k + cache.v:
            x.zero_()
        return cache, TurnStep(cache, 400, 100, hq, freq, vocab=vocab, q_norm=model.qn, k_norm=model.kn, window=[0, 50])

    def turn(cache, step):
        step.plan(new)
        outs = []
        for layer in range(layers):
            step.store(layer, *rows[layer])
            outs.append(step.attend(layer).clone())
        target = step.shape(logits, tokens=tokens, history=history, repetition=rep).clone()
        step.commit(all_rows=True)
        cache.continue_from(source, keep)
        return outs + [target, cache.block_table, cache.kv_len, cache.pages_held, cache.free_head, cache.free_pages]

    state = lambda c: [c.block_table, c.kv_len, c.pages_held, c.free_pages, c.free_head] + c.k + c.v
    cache, step = fresh()
    start = [x.clone() for x in state(cache)]
    eager = []
    for _ in range(3):
        eager.append([x.clone() for x in turn(cache, step)])
    for x, y in zip(state(cache), start):
        x.copy_(y)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        turn(cache, step)
        for x, y in zip(state(cache), start):
            x.copy_(y)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = turn(cache, step)
    for x, y in zip(state(cache), start):
        x.copy_(y)
    n = 280
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            rows_of = n if a.dim() > 1 and a.shape[0] == 400 else None
            assert torch.equal(a[:rows_of], b[:rows_of])


def test_alternating_vocabularies_keep_their_buffers():
    """Each vocabulary has one target and workspace, however often it comes; a captured pass finds its own again."""
    say("turns, alternating vocabularies")
    freq = qcf.rope_frequencies(64, 1e4)
    cache = TurnCache(1, 8, 16, 2, 64, 2, 4)
    step = TurnStep(cache, 6, 3, 4, freq, vocab=500)
    step.plan(i32([3, 2]))
    logits = {v: torch.randn(6, v, device="cuda") for v in (500, 20000, 9001)}
    first = {v: step.shape(x) for v, x in logits.items()}
    want = {v: t.clone() for v, t in first.items()}
    at = {v: t.data_ptr() for v, t in first.items()}
    assert first[500].shape == (6, 500) and len(set(at.values())) == 3
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for _ in range(3):
        for v in (20000, 500, 9001):
            got = step.shape(logits[v])
            assert got.data_ptr() == at[v] == step.target.data_ptr() and torch.equal(got[:5], want[v][:5])
        assert all(torch.equal(first[v][:5], want[v][:5]) for v in first)
        del got
    assert torch.cuda.memory_allocated() == held


def test_steps_of_few_rows_hold_no_workspace_they_never_use():
    """Layers that see all tokens of few rows take the tree call; one with a window takes the chunk call, and its rows see
    the window's tokens."""
    say("turns of few rows")
    rng = np.random.default_rng(10)
    freq = qcf.rope_frequencies(48, 1e4)
    for ps, window, holds in ((16, 0, False), (8, 0, False), (16, (0, 40), True)):
        model = Model(rng, "bf16", 2, 8, 2, 64, 100)
        cache = TurnCache(2, 60, ps, 2, 64, 3, 30)
        mirror = Mirror(2, 3, 2, 64)
        first = TurnStep(cache, 300, 130, 8, freq, q_norm=model.qn, k_norm=model.kn, window=window)
        assert first.ws_chunk is not None or ps < 16
        run_pass(first, model, [100, 7, 90], mirror, rng)
        first.commit(all_rows=True)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        step = TurnStep(cache, 12, 4, 8, freq, q_norm=model.qn, k_norm=model.kn, window=window)
        assert step.few and (step.ws_chunk is not None) == holds
        if not holds:
            need = qcf.qcf_chunk_attn_workspace_size(3, 4, 30 * ps, 8, 2, 64, torch.bfloat16)
            assert torch.cuda.memory_allocated() - before < need
        for new in ([1, 1, 1], [4, 0, 3]):
            run_pass(step, model, new, mirror, rng)
            step.commit(all_rows=True)
            check_cache(cache, mirror)


def test_a_cache_that_runs_out_of_pages_says_so():
    """Continuations that find no page: how many were missing is kept (free_head counts free pages alone again), and the list is
    whole afterwards."""
    say("turns, pages run out")
    rng = np.random.default_rng(11)
    freq = qcf.rope_frequencies(48, 1e4)
    cache = TurnCache(1, 8, 16, 2, 64, 4, 6)
    model = Model(rng, "bf16", 1, 4, 2, 64, 100, False)
    step = TurnStep(cache, 120, 90, 4, freq)
    mirror = Mirror(1, 4, 2, 64)
    run_pass(step, model, [84, 7, 0, 0], mirror, rng)                   # 6 + 1 of 8 pages
    step.commit(all_rows=True)
    assert int(cache.pages_missing[0]) == 0
    cache.continue_from(i32([0, 0, 0, 0]))                              # three copies, one page (and the one that 1 gives up, later)
    assert int(cache.pages_missing[0]) == 2
    table = cache.block_table.cpu().numpy()
    assert (table[:, 5] >= 0).sum() == 2 and (table[2:, 5] == -1).all()
    head, held = int(cache.free_head[0]), {int(p) for p in table.ravel() if p >= 0}
    assert len(held) + 8 - head == 8 and not held & set(cache.free_pages.tolist()[head:])
    cache.keep(i32([84, 80, 80, 0]))
    assert int(cache.pages_missing[0]) == 0
    mirror.continue_from([0, 0, 0, 0], [84, 80, 80, 0])
    check_cache(cache, mirror)
    # planned rows that found no page: free_head says so until requests change, then that change
    step.plan(i32([10, 1, 1, 40]))
    assert int(cache.free_head[0]) == cache.n_pages + 3
    step.commit(all_rows=True)
    cache.keep(i32([84, 80, 80, 0]))
    assert int(cache.pages_missing[0]) == 3 and int(cache.free_head[0]) <= cache.n_pages
    mirror.continue_from([0, 1, 2, 3], [84, 80, 80, 0])
    check_cache(cache, mirror)


def test_turn_step_refusals():
    freq = qcf.rope_frequencies(64, 1e4)
    cache = TurnCache(2, 8, 8, 2, 64, 2, 4)
    with pytest.raises(qcf.QcfError):
        TurnStep(cache, 8, 4, 8, freq, window=5)                        # pages of 8 rows
    cache = TurnCache(2, 8, 16, 2, 64, 2, 4)
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(window=[1]), dict(q_norm=[w, w]), dict(q_norm=[w], k_norm=[w])):
        with pytest.raises(qcf.QcfError):
            TurnStep(cache, 8, 4, 8, freq, **bad)
    step = TurnStep(cache, 8, 4, 8, freq, window=[0, 5])
    step.plan(i32([2, 2]), parents=i32([-1, 0, -1, 0, -1, -1, -1, -1]))
    step.attend(0)
    with pytest.raises(qcf.QcfError):
        step.attend(1)                                                  # a tree over a window


def test_calls_on_another_stream():
    """The calls take torch's current stream: work on a side stream, ordered by events alone."""
    say("turns on another stream")
    rng = np.random.default_rng(8)
    model = Model(rng, "bf16", 1, 8, 2, 64, 100)
    freq = qcf.rope_frequencies(64, 1e4)
    results = []
    for side in (False, True):
        rng2 = np.random.default_rng(9)
        model.rng = rng2
        cache = TurnCache(1, 40, 16, 2, 64, 3, 12)
        cache.k[0].zero_(), cache.v[0].zero_()
        step = TurnStep(cache, 300, 90, 8, freq, q_norm=model.qn, k_norm=model.kn)
        data = model.rows(300)
        s = torch.cuda.Stream() if side else torch.cuda.current_stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step.plan(i32([90, 80, 70]))
            step.store(0, *data)
            out = step.attend(0).clone()
            step.commit(all_rows=True)
            cache.continue_from(i32([2, 2, 0]))
        torch.cuda.current_stream().wait_stream(s)
        results.append([x.clone() for x in (out[:240], cache.k[0], cache.block_table, cache.free_pages)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
