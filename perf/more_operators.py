"""A further turn on the paged caches: the operators around the answering calls, in use.

A request's fused cache lives on in pages after its first answer.  The next question is a chunk of new rows, models
norm the queries and keys of every head before they are rotated, answers are drawn from logits that
penalties, biases and a grammar have shaped, one cache is continued by several answers, and requests end.  The
cases are one pass each of

  norm     qcf_norm_rope_store: per-head norms and rotary positions of new rows, keys and values into their slots
  chunk    qcf_chunk_attn: attention of the new rows over a paged cache, each up to its own token, or a window of them
  shape    qcf_shape_logits: logits to the probabilities that drafts are verified against
  fork     qcf_page_fork and qcf_copy_pages: requests that continue others, their started pages copied in all layers
  release  qcf_page_release: pages that no request holds any more go back to the free list

``run`` computes them in plain torch operations, or with ``own`` set through
``paper_2606_05875_amd.qcf``.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1.0e-6


def listed():
    case = lambda name, kind, **kw: dict(kw, name=name, kind=kind)
    return [
        # one decoded token of each of 48 requests; a weight for every head, half of it rotated in adjacent pairs (latency)
        case("norm_decode", "norm", rows=48, slots=4096, pos_hi=33000, hq=32, hkv=8, d=128, rotary=64,
             interleaved=True, weights="heads", gather=True, dtype="bf16"),
        # a 32K-token prompt with 64/8 heads of 128
        case("norm_prompt", "norm", rows=32896, slots=33024, pos_hi=32896, hq=64, hkv=8, d=128, rotary=128,
             interleaved=False, weights="shared", gather=False, dtype="bf16"),
        # a test-sized model in float32: three further questions
        case("chunk_small_f32", "chunk", batch=3, new_lo=5, new_hi=70, ctx_lo=33, ctx_hi=700, page=16, window=0,
             hq=8, hkv=2, d=64, dtype="f32", layout=4),
        # a further question of each request of a ragged serving batch, over its fused cache and first answer
        case("chunk_questions", "chunk", batch=16, new_lo=16, new_hi=128, ctx_lo=2000, ctx_hi=12700, page=64, window=0,
             hq=32, hkv=8, d=128, dtype="bf16", layout=5),
        # prompts of several lengths in a layer whose rows see the last 1024 tokens
        case("chunk_window", "chunk", batch=6, new_lo=700, new_hi=4000, ctx_lo=0, ctx_hi=6000, page=16, window=1024,
             hq=32, hkv=8, d=64, dtype="bf16", layout=6),
        # a chunk of a long prompt that enters in pieces of 2048 rows, 64/8 heads of 128
        case("chunk_prefill", "chunk", batch=1, new_lo=2048, new_hi=2048, ctx_lo=30848, ctx_hi=30848, page=128, window=0,
             hq=64, hkv=8, d=128, dtype="bf16", layout=7),
        # one row of logits for each of 64 requests, penalties over what was said so far
        case("shape_decode", "shape", batch=64, new_lo=1, new_hi=1, hist_lo=512, hist_hi=8192, vocab=128000,
             penalties=True, bias=0, grammar=False, tree=False, dtype="f32", out="f32", layout=8),
        # trees of drafts in bfloat16 under a grammar, with biases and penalties along every path
        case("shape_tree", "shape", batch=16, new_lo=10, new_hi=26, hist_lo=2000, hist_hi=12700, vocab=150001,
             penalties=True, bias=200, grammar=True, tree=True, dtype="bf16", out="f32", layout=9),
        # four requests of eight beams each: every beam continues one of its request's
        case("fork_beams", "fork", batch=32, group=8, ctx_lo=300, ctx_hi=900, page=16, layers=12, hkv=8, d=128,
             cut=False, layout=10),
        # eight answers from one fused cache
        case("fork_answers", "fork", batch=8, group=8, ctx_lo=12000, ctx_hi=12000, page=128, layers=16, hkv=8, d=128,
             cut=False, layout=11),
        # the end of a ragged serving batch's turn: some requests end, some are taken back to an earlier token
        case("release_turn", "release", batch=16, ctx_lo=2000, ctx_hi=12700, page=64, group=1, layout=12),
        # a large batch in small pages, groups of four with a common context
        case("release_shared", "release", batch=256, ctx_lo=0, ctx_hi=14000, page=16, group=4, layout=13),
    ]


def draw(rng):
    """Another case of the ranges the listed ones stand for."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["norm", "chunk", "chunk", "chunk", "shape", "shape", "fork", "release"])
    layout = rng.randrange(20, 1 << 20)
    heads = [(8, 2, 64), (16, 4, 64), (32, 8, 64), (8, 8, 128), (16, 1, 128), (32, 8, 128), (32, 8, 128),
             (40, 10, 128), (64, 8, 128)]
    hq, hkv, d = rng.choice(heads)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "norm":
        rows = log(1, 12000 if dtype == "f32" else 30000)
        return dict(kind=kind, rows=rows, slots=rows + rng.randint(0, 3000), pos_hi=log(1000, 130000), hq=hq,
                    hkv=hkv, d=d, rotary=16 * rng.randint(1, d // 16), interleaved=rng.random() < 0.5,
                    weights=rng.choice(["shared", "heads", "none"]), gather=rng.random() < 0.3, dtype=dtype)
    if kind == "chunk":
        # rows times tokens of the whole batch, bounded so that no draw costs more than the largest case
        area = log(3e3, 4e6 if dtype == "f32" else 3e7)
        batch = rng.choice([1, 1, 2, 3, log(4, 24)])
        hi = min(log(1, 4000), max(1, int(math.sqrt(area / batch))))
        top = min(32000, max(0, area // (batch * hi) - hi))
        return dict(kind=kind, batch=batch, new_lo=rng.choice([1, max(1, hi // 3), hi]), new_hi=hi,
                    ctx_lo=rng.choice([0, top // 4, top]), ctx_hi=top, page=rng.choice([16, 16, 32, 64, 128]),
                    window=rng.choice([0, 0, 1, log(2, 5000)]) if rng.random() < 0.6 else 0, hq=hq, hkv=hkv, d=d,
                    dtype=dtype, layout=layout)
    if kind == "shape":
        hi = rng.randint(1, 12)
        vocab = log(900, 150000)
        batch = max(1, min(log(1, 64), 30_000_000 // (hi * vocab)))
        top = log(1, 12000)
        return dict(kind=kind, batch=batch, new_lo=rng.randint(1, hi), new_hi=hi, hist_lo=rng.choice([0, top // 3]),
                    hist_hi=top, vocab=vocab, penalties=rng.random() < 0.8, bias=rng.choice([0, log(1, 500)]),
                    grammar=rng.random() < 0.4, tree=rng.random() < 0.4, dtype=rng.choice(["f32", "bf16"]),
                    out=rng.choice(["f32", "f32", "bf16"]), layout=layout)
    page = rng.choice([8, 16, 32, 64, 128])
    if kind == "fork":
        group = rng.choice([1, 2, 4, 8])
        batch = group * log(1, 8)
        top = log(20, 24000 // batch)
        return dict(kind=kind, batch=batch, group=group, ctx_lo=rng.choice([0, top // 3, top]), ctx_hi=top, page=page,
                    layers=rng.randint(1, 12), hkv=hkv, d=d, cut=rng.random() < 0.5, layout=layout)
    batch = log(1, 400)
    return dict(kind=kind, batch=batch, ctx_lo=0, ctx_hi=log(100, 15000), page=max(16, page), group=rng.choice([1, 4]),
                layout=layout)


# ---------------------------------------------------------------------------
# lengths and what a pass cannot do without (from the case alone)
# ---------------------------------------------------------------------------
def lengths(c, lo="ctx_lo", hi="ctx_hi"):
    """(new rows, tokens held) per request; the extremes occur where there is room for them."""
    r = random.Random(c["layout"])
    new = [r.randint(c.get("new_lo", 1), c.get("new_hi", 1)) for _ in range(c["batch"])]
    ctx = [r.randint(c[lo], c[hi]) for _ in range(c["batch"])]
    new[0], ctx[0] = c.get("new_hi", 1), c[hi]
    if c["batch"] > 2:
        new[-1], ctx[-1] = c.get("new_lo", 1), c[lo]
    return new, ctx


def continuing(c):
    """Who continues whom, and at how many tokens (for cut cases)."""
    r = random.Random(c["layout"] + 1)
    g = c["group"]
    if g == c["batch"]:
        source = [0] * c["batch"]
    else:
        source = [b // g * g + r.randrange(g) for b in range(c["batch"])]
    _, ctx = lengths(c)
    keep = [r.randint(0, ctx[s] + 5) if c["cut"] else ctx[s] for s in source]
    return source, keep


def work(c):
    es = 2 if c.get("dtype") == "bf16" else 4
    if c["kind"] == "norm":
        row = (c["hq"] + 2 * c["hkv"]) * c["d"] * es
        n = (c["hq"] + c["hkv"]) * c["d"]
        return {"bytes": c["rows"] * (2 * row + 8 + (4 if c["gather"] else 0)), "flops": c["rows"] * 6 * n}
    if c["kind"] == "release":
        _, ctx = lengths(c)
        return {"bytes": 8 * sum(-(-x // c["page"]) for x in ctx) + 12 * c["batch"], "flops": 0}
    new, ctx = lengths(c) if c["kind"] != "shape" else lengths(c, "hist_lo", "hist_hi")
    n = sum(new)
    if c["kind"] == "chunk":
        w = c["window"] or 1 << 40
        keys = sum(min(a + b, a - 1 + w) for a, b in zip(new, ctx))
        seen = sum(sum(min(b + i + 1, w) for i in range(a)) for a, b in zip(new, ctx))
        return {"bytes": keys * 2 * c["hkv"] * c["d"] * es + n * c["hq"] * (2 * c["d"] * es + 4),
                "flops": 4 * c["hq"] * c["d"] * seen}
    if c["kind"] == "shape":
        eo = 2 if c["out"] == "bf16" else 4
        return {"bytes": n * c["vocab"] * (es + eo + (0.125 if c["grammar"] else 0)) + 4 * sum(ctx), "flops": 6 * n * c["vocab"]}
    source, keep = continuing(c)
    ps, moved, pages = c["page"], 0, 0
    for b, (s, k) in enumerate(zip(source, keep)):
        at = min(k, ctx[s])
        pages += -(-at // ps)
        if not (s == b and at // ps == ctx[b] // ps):
            moved += at % ps
    return {"bytes": 8 * pages + 16 * c["batch"] + moved * c["hkv"] * c["d"] * 2 * 2 * 2 * c["layers"], "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to(DEV)


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.float32))).to(DEV)


def empty_i32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def cumulated(x):
    return np.concatenate([[0], np.cumsum(x)])


def grow_trees(rng, new):
    """Parents (index within the request, -1 for the first row) of ragged trees."""
    return np.concatenate([[-1] + [int(rng.integers(max(0, i - 6), i)) for i in range(1, n)] for n in new]).astype(np.int32)


def ancestor_bits(parents, new):
    """[rows, words] bits of each row's ancestors and itself."""
    m = np.zeros((len(parents), (max(new) + 31) // 32), np.uint32)
    base = 0
    for n in new:
        for i in range(n):
            if parents[base + i] >= 0:
                m[base + i] = m[base + parents[base + i]]
            m[base + i, i // 32] |= np.uint32(1 << (i % 32))
        base += n
    return m.view(np.int32)


def pool(slots, hkv, d, dtype):
    """K or V pages as a user lays them out: rows padded to an odd number of head slices."""
    width = (hkv + 1 - hkv % 2) * d
    return torch.zeros((slots, width), dtype=dtype, device=DEV)[:, :hkv * d].view(slots, hkv, d)


def prepare(c, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)
    s = {"case": c}
    globals()["prepare_" + c["kind"]](c, s, rng, normal)
    if own:
        from paper_2606_05875_amd import qcf
        s["calls"] = globals()["own_" + c["kind"]](c, s, qcf)
    return s


def prepare_norm(c, s, rng, normal):
    dt = DT[c["dtype"]]
    src = c["rows"] + 100 if c["gather"] else c["rows"]
    # the rows of one product x W_qkv: queries, keys and values side by side; rows of different sizes
    qkv = (normal(src, (c["hq"] + 2 * c["hkv"]) * c["d"]) * torch.exp(normal(src, 1))).to(dt)
    q, k, v = qkv.split([c["hq"] * c["d"], c["hkv"] * c["d"], c["hkv"] * c["d"]], dim=1)
    s.update(q=q.view(src, c["hq"], c["d"]), k=k.view(src, c["hkv"], c["d"]), v=v.view(src, c["hkv"], c["d"]))
    own_heads = c["weights"] == "heads"
    weight = lambda h: None if c["weights"] == "none" else (1 + 0.2 * normal(*((h,) if own_heads else ()), c["d"])).to(dt)
    s["q_weight"], s["k_weight"] = weight(c["hq"]), weight(c["hkv"])
    s["slots"] = i32(rng.permutation(c["slots"])[:c["rows"]])
    s["positions"] = i32(rng.integers(0, c["pos_hi"], c["rows"]) if c["rows"] != c["pos_hi"] else np.arange(c["rows"]))
    s["src"] = i32(rng.permutation(src)[:c["rows"]]) if c["gather"] else None
    s["inv_freq"] = torch.from_numpy(1.0e6 ** (-np.arange(0, c["rotary"], 2, dtype=np.float64) / c["rotary"])).to(DEV)
    s["k_cache"], s["v_cache"] = (pool(c["slots"], c["hkv"], c["d"], dt) for _ in range(2))
    s["q_out"] = torch.empty((c["rows"], c["hq"], c["d"]), dtype=dt, device=DEV)


def prepare_chunk(c, s, rng, normal):
    dt = DT[c["dtype"]]
    new, ctx = lengths(c)
    ps = c["page"]
    need = [-(-(a + b) // ps) for a, b in zip(new, ctx)]
    pages = sum(need) + 5
    order = rng.permutation(pages)
    table = np.full((c["batch"], max(need) + 2), -1, np.int32)
    at = 0
    for b, h in enumerate(need):
        table[b, :h] = order[at:at + h]
        at += h
    n = sum(new)
    s["k_cache"], s["v_cache"] = (pool(pages * ps, c["hkv"], c["d"], dt) for _ in range(2))
    s["k_cache"].copy_(normal(pages * ps, c["hkv"], c["d"]))
    s["v_cache"].copy_(normal(pages * ps, c["hkv"], c["d"]))
    s["q"] = (2.0 * normal(n, c["hq"], c["d"])).to(dt)  # logits spread over a few units
    s["out"] = torch.empty((n, c["hq"], c["d"]), dtype=dt, device=DEV)
    s["lse"] = torch.empty((n, c["hq"]), device=DEV)
    s.update(table=i32(table), kv_len=i32(ctx), cu=i32(cumulated(new)), new=new, ctx=ctx, scale=1.0 / math.sqrt(c["d"]))


def prepare_shape(c, s, rng, normal):
    new, ctx = lengths(c, "hist_lo", "hist_hi")
    n, V, B = sum(new), c["vocab"], c["batch"]
    s["logits"] = (3.0 * normal(n, V) - 2.0).to(DT[c["dtype"]])
    # what was said: some tokens often, most never (the logits of those are high)
    said = np.minimum(V - 1, (V ** rng.random((B, max(ctx) + 1))).astype(np.int64))
    said = (said * 7919 + 11) % V
    s["history"] = i32(said)
    s["hist_len"], s["prompt_len"] = i32(ctx), i32([int(x * r) for x, r in zip(ctx, rng.random(B))])
    tokens = np.concatenate([rng.choice(said[b], a) for b, a in enumerate(new)])
    s["tokens"] = i32(tokens)
    s["cu"] = i32(cumulated(new))
    s["new"], s["ctx"] = new, ctx
    s["parents"] = grow_trees(rng, new) if c["tree"] else None
    s["mask"] = i32(ancestor_bits(s["parents"], new)) if c["tree"] else None
    some = lambda lo, hi: f32(rng.uniform(lo, hi, B))
    for name, lo, hi in (("repetition", 1.0, 1.5), ("presence", 0.0, 1.0), ("frequency", 0.0, 0.5)):
        s[name] = some(lo, hi) if c["penalties"] else None
    s["temperature"] = some(0.5, 1.3)
    s["bias_start"] = s["bias_token"] = s["bias_value"] = s["allowed"] = None
    if c["bias"]:
        each = [min(V, int(rng.integers(0, 2 * c["bias"]))) for _ in range(B)]
        s["bias_start"] = i32(cumulated(each))
        s["bias_token"] = i32(np.concatenate([rng.permutation(V)[:k] for k in each] + [[0]])[:sum(each)])
        s["bias_value"] = f32(rng.normal(0, 4, sum(each)))
    if c["grammar"]:  # from a few to most of the tokens are allowed
        words = (V + 31) // 32
        a = rng.integers(0, 1 << 32, (n, words), dtype=np.uint64) & rng.integers(0, 1 << 32, (n, words), dtype=np.uint64)
        a[: n // 3] &= np.where(rng.random((n // 3, words)) < 0.02, np.uint64(0xffffffff), np.uint64(0))
        s["allowed"] = i32(a.astype(np.uint32).view(np.int32))
    s["out"] = torch.empty((n, V), dtype=DT[c["out"]], device=DEV)


def prepare_fork(c, s, rng, normal):
    _, ctx = lengths(c)
    ps, B = c["page"], c["batch"]
    source, keep = continuing(c)
    held = [-(-x // ps) for x in ctx]
    pages = sum(held) + B + 6
    order = rng.permutation(pages)
    table = np.full((B, max(held) + 3), -1, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    s.update(table=i32(table), kv_len=i32(ctx), source=i32(source), keep=i32(keep) if c["cut"] else None,
             free=i32(order), head=i32([at]), pages=pages)
    P, width = 2 * c["layers"], (c["hkv"] + 1 - c["hkv"] % 2) * c["d"]
    s["all"] = torch.empty((P, pages * ps, width), dtype=torch.bfloat16, device=DEV)
    for p in range(P):
        s["all"][p] = normal(pages * ps, width)
    s["pools"] = [x[:, :c["hkv"] * c["d"]].view(pages * ps, c["hkv"], c["d"]) for x in s["all"]]
    s.update(table_out=empty_i32(*table.shape), kv_out=empty_i32(B), held_out=empty_i32(B), head_out=empty_i32(1),
             copy_src=empty_i32(B), copy_dst=empty_i32(B), copy_rows=empty_i32(B))


def prepare_release(c, s, rng, normal):
    _, ctx = lengths(c)
    ps, B = c["page"], c["batch"]
    held = [-(-x // ps) for x in ctx]
    table = np.full((B, max(held) + 2), -1, np.int32)
    pages = sum(held) + 20
    order = rng.permutation(pages)
    at = 0
    for b, h in enumerate(held):
        first = b // c["group"] * c["group"]
        same = min(held[first], h) // 2 if b != first else 0  # the group's shared context
        table[b, :same] = table[first, :same]
        table[b, same:h] = order[at:at + h - same]
        at += h - same
    after, held_after = np.full_like(table, -1), list(held)
    for b in range(B):
        fate = rng.random()
        if fate < 0.25:
            held_after[b] = 0                                     # ended
        elif fate < 0.4:
            held_after[b] = int(rng.integers(0, held[b] + 1))     # taken back to an earlier token
        after[b, :held_after[b]] = table[b, :held_after[b]]
    s.update(table=i32(table), held=i32(held), after=i32(after), held_after=i32(held_after), free_list=i32(order),
             head=i32([at]), pages=pages, head_out=empty_i32(1))


# ---------------------------------------------------------------------------
# the framework's operators: each call is validated once and replayed, as its steps do
# ---------------------------------------------------------------------------
def own_norm(c, s, qcf):
    return [qcf.prepare(qcf.qcf_norm_rope_store, s["k_cache"], s["v_cache"], s["k"], s["v"], s["slots"], s["positions"],
                        s["inv_freq"], interleaved=c["interleaved"], q_new=s["q"], q_out=s["q_out"], src_idx=s["src"],
                        q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)]


def own_chunk(c, s, qcf):
    new, ctx = s["new"], s["ctx"]
    max_kv = max(a + b for a, b in zip(new, ctx))
    need = qcf.qcf_chunk_attn_workspace_size(c["batch"], max(new), max_kv, c["hq"], c["hkv"], c["d"], DT[c["dtype"]])
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    return [qcf.prepare(qcf.qcf_chunk_attn, s["out"], s["q"], s["cu"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"],
                        c["page"], max(new), max_kv, s["scale"], window=c["window"], lse=s["lse"], workspace=s["ws"])]


def own_shape(c, s, qcf):
    need = qcf.qcf_shape_logits_workspace_size(s["out"].shape[0], c["vocab"])
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    return [qcf.prepare(qcf.qcf_shape_logits, s["out"], s["logits"], s["cu"], history=s["history"],
                        prompt_len=s["prompt_len"], hist_len=s["hist_len"], tokens=s["tokens"], tree_mask=s["mask"],
                        repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                        bias_start=s["bias_start"], bias_token=s["bias_token"], bias_value=s["bias_value"],
                        allowed=s["allowed"], temperature=s["temperature"], workspace=s["ws"])]


def own_fork(c, s, qcf):
    s["pool_set"] = qcf.PoolSet(s["pools"])
    return [qcf.prepare(qcf.qcf_page_fork, s["table_out"], s["kv_out"], s["held_out"], s["table"], s["kv_len"], s["source"],
                        s["free"], c["page"], s["pages"], keep_len=s["keep"], free_head=s["head"],
                        free_head_out=s["head_out"], copy_src=s["copy_src"], copy_dst=s["copy_dst"],
                        copy_rows=s["copy_rows"]),
            qcf.prepare(qcf.qcf_copy_pages, s["pool_set"], s["copy_src"], s["copy_dst"], c["page"], rows=s["copy_rows"])]


def own_release(c, s, qcf):
    return [qcf.prepare(qcf.qcf_page_release, s["table"], s["held"], s["after"], s["held_after"], s["free_list"],
                        s["head"], s["head_out"], s["pages"])]


OUT = {"norm": ("k_cache", "v_cache", "q_out"), "chunk": ("out", "lse"), "shape": ("out",),
       "fork": ("table_out", "kv_out", "held_out", "head_out", "copy_src", "copy_dst", "copy_rows", "all"),
       "release": ("free_list", "head_out")}


def run(s):
    c = s["case"]
    if own:
        for call in s["calls"]:
            call()
        return [s[k] for k in OUT[c["kind"]]]
    return globals()["plain_" + c["kind"]](c, s)


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def plain_norm(c, s):
    R, rows = c["rotary"], s["slots"].long()
    src = s["src"].long() if c["gather"] else torch.arange(c["rows"], device=DEV)
    angle = s["positions"].double()[:, None] * s["inv_freq"][None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]

    def turn(x, weight):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if weight is not None:
            x = x * weight.float()
        a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
        y, z = a * cos - b * sin, a * sin + b * cos
        y = torch.stack([y, z], -1).flatten(-2) if c["interleaved"] else torch.cat([y, z], -1)
        return torch.cat([y, x[..., R:]], -1).to(DT[c["dtype"]])

    s["k_cache"][rows] = turn(s["k"][src], s["k_weight"])
    s["v_cache"][rows] = s["v"][src]
    return [s["k_cache"], s["v_cache"], turn(s["q"][src], s["q_weight"])]


def plain_chunk(c, s):
    ps, g = c["page"], c["hq"] // c["hkv"]
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    base = 0
    for b, (n, held) in enumerate(zip(s["new"], s["ctx"])):
        lo = max(0, held - c["window"] + 1) if c["window"] else 0                  # the first token that a row sees
        j = torch.arange(lo, held + n, device=DEV)
        slot = s["table"][b, torch.div(j, ps, rounding_mode="floor")].long() * ps + j % ps
        k = s["k_cache"][slot].float().permute(1, 2, 0).contiguous()                # [hkv, d, keys]
        v = s["v_cache"][slot].float().transpose(0, 1).contiguous()
        q = s["q"][base:base + n].float().view(n, c["hkv"], g, -1).permute(1, 2, 0, 3).reshape(c["hkv"], g * n, -1)
        x = torch.matmul(q, k).view(c["hkv"], g, n, -1) * s["scale"]
        at = held + torch.arange(n, device=DEV)[:, None]
        see = j[None, :] <= at
        if c["window"]:
            see = see & (j[None, :] > at - c["window"])
        x = torch.where(see, x, -math.inf)
        top = x.amax(-1, keepdim=True)
        e = torch.exp(x - top)
        tot = e.sum(-1, keepdim=True)
        o = torch.matmul(e.view(c["hkv"], g * n, -1), v).view(c["hkv"], g, n, -1) / tot
        out[base:base + n] = o.permute(2, 0, 1, 3).reshape(n, c["hq"], -1).to(out.dtype)
        lse[base:base + n] = (top + torch.log(tot)).squeeze(-1).permute(2, 0, 1).reshape(n, -1)
        base += n
    return [out, lse]


def plain_shape(c, s):
    V, B, n = c["vocab"], c["batch"], s["logits"].shape[0]
    cu = s["cu"].long()
    req = torch.searchsorted(cu, torch.arange(n, device=DEV), right=True) - 1
    z = s["logits"].float()
    if c["penalties"]:
        said = s["history"].long()
        at = torch.arange(said.shape[1], device=DEV)[None, :]
        there = at < s["hist_len"][:, None]
        answer = there & (at >= s["prompt_len"][:, None])
        zero = torch.zeros((B, V), device=DEV)
        count = zero.scatter_add(1, said, answer.float())[req]
        seen = zero.scatter_add(1, said, there.float())[req]
        # the rows of the pass that a row follows, itself among them
        first = cu[req]
        j = torch.arange(max(s["new"]), device=DEV)[None, :]
        own_row = torch.arange(n, device=DEV) - first
        if c["tree"]:
            follows = (s["mask"][:, torch.div(j[0], 32, rounding_mode="floor")] >> (j % 32)) & 1 == 1
        else:
            follows = j <= own_row[:, None]
        t = s["tokens"].long()[(first[:, None] + j).clamp(max=n - 1)]
        count = count.scatter_add_(1, t, follows.float())
        seen = seen + count
        r = s["repetition"][req][:, None]
        z = torch.where(seen > 0, torch.where(z > 0, z / r, z * r), z)
        z = z - s["frequency"][req][:, None] * count - s["presence"][req][:, None] * (count > 0)
    if c["bias"]:
        start = s["bias_start"].long()
        who = torch.searchsorted(start, torch.arange(s["bias_token"].numel(), device=DEV), right=True) - 1
        bias = torch.zeros((B, V), device=DEV)
        bias[who, s["bias_token"].long()] = s["bias_value"]
        z = z + bias[req]
    if c["grammar"]:
        t = torch.arange(V, device=DEV)
        z = torch.where((s["allowed"][:, torch.div(t, 32, rounding_mode="floor")] >> (t % 32)) & 1 == 1, z, -math.inf)
    z = z / s["temperature"][req][:, None]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    tot = e.sum(1, keepdim=True)
    return [torch.where(tot > 0, e / tot, torch.zeros_like(e)).to(DT[c["out"]])]


def plain_fork(c, s):
    ps, B = c["page"], c["batch"]
    kv, src = s["kv_len"].long(), s["source"].long()
    at = kv[src] if s["keep"] is None else torch.minimum(kv[src], s["keep"].long())
    me = torch.arange(B, device=DEV)
    full, part = torch.div(at, ps, rounding_mode="floor"), at % ps
    fresh = (part > 0) & ~((src == me) & (full == torch.div(kv, ps, rounding_mode="floor")))
    held = full + (part > 0).long()
    place = s["head"].long() + torch.cumsum(fresh.long(), 0) - fresh.long()
    page = s["free"].long()[place.clamp(max=s["free"].numel() - 1)]
    col = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    table = torch.where(col < held[:, None], s["table"].long()[src], -1)
    last = table.gather(1, full.clamp(max=table.shape[1] - 1)[:, None]).squeeze(1)
    table = torch.where(fresh[:, None] & (col == full[:, None]), page[:, None], table)
    none = torch.full_like(last, -1)
    copy_src, copy_dst, rows = torch.where(fresh, last, none), torch.where(fresh, page, none), torch.where(fresh, part, 0)
    width = c["hkv"] * c["d"]
    pages = s["all"].view(s["all"].shape[0], s["pages"], ps, -1)
    pair, row = torch.nonzero(torch.arange(ps, device=DEV)[None, :] < rows[:, None], as_tuple=True)
    pages[:, copy_dst[pair], row, :width] = pages[:, copy_src[pair], row, :width]
    head = s["head"] + fresh.sum().int()
    return [table.int(), at.int(), held.int(), head, copy_src.int(), copy_dst.int(), rows.int(), s["all"]]


def plain_release(c, s):
    col = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    mark = lambda table, held: torch.zeros(s["pages"] + 1, dtype=torch.bool, device=DEV).index_fill_(
        0, torch.where(col < held[:, None], table, s["pages"]).long().view(-1), True)[:-1]
    gone = mark(s["table"], s["held"]) & ~mark(s["after"], s["held_after"])
    page = torch.nonzero(gone).squeeze(1)
    head = s["head"] - page.numel()
    s["free_list"][head.long() + torch.arange(page.numel(), device=DEV)] = page.int()
    return [s["free_list"], head]


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(c, seed):
    return globals()["exact_" + c["kind"]](c, prepare(c, seed))


def exact_norm(c, s):
    src = s["src"].long() if c["gather"] else slice(None)
    R = c["rotary"]
    w = torch.exp(1j * s["positions"].double()[:, None, None] * s["inv_freq"])

    def turn(x, weight):
        x = x[src].double()
        x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["d"] + EPS)
        y = x if weight is None else x * weight.double()
        y = y.clone()
        if c["interleaved"]:
            z = torch.view_as_complex(y[..., :R].unflatten(-1, (R // 2, 2)).contiguous()) * w
            y[..., :R] = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * w
            y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
        return y

    out = []
    for new in (turn(s["k"], s["k_weight"]), s["v"][src].double()):
        cache = torch.zeros((c["slots"], c["hkv"], c["d"]), dtype=torch.double, device=DEV)
        out.append(cache.index_copy_(0, s["slots"].long(), new))
    return out + [turn(s["q"], s["q_weight"])]


def exact_chunk(c, s):
    outs, lses = [], []
    base, g = 0, c["hq"] // c["hkv"]
    table = s["table"].cpu().numpy().astype(np.int64)
    for b, (n, held) in enumerate(zip(s["new"], s["ctx"])):
        slot = np.array([table[b, j // c["page"]] * c["page"] + j % c["page"] for j in range(held + n)], np.int64)
        slot = torch.from_numpy(slot).to(DEV)
        hide = torch.ones((n, held + n), dtype=torch.bool, device=DEV).triu(held + 1)
        if c["window"]:
            hide |= torch.ones_like(hide).tril(held - c["window"])
        o = torch.empty((n, c["hq"], c["d"]), dtype=torch.double, device=DEV)
        e = torch.empty((n, c["hq"]), dtype=torch.double, device=DEV)
        for h in range(c["hq"]):
            k, v = (s[name][slot, h // g].double() for name in ("k_cache", "v_cache"))
            x = (s["q"][base:base + n, h].double() @ k.T * s["scale"]).masked_fill_(hide, -math.inf)
            e[:, h] = torch.logsumexp(x, 1)
            o[:, h] = torch.exp(x - e[:, h, None]) @ v
        outs.append(o)
        lses.append(e)
        base += n
    return [torch.cat(outs), torch.cat(lses)]


def exact_shape(c, s):
    n64 = lambda k: s[k].cpu().numpy().astype(np.int64)
    f64 = lambda k, b: float(s[k][b])
    said, prompt, tokens = n64("history"), n64("prompt_len"), n64("tokens")
    V, base, rows = c["vocab"], 0, []
    for b, (n, long) in enumerate(zip(s["new"], s["ctx"])):
        for i in range(n):
            path, up = [], i
            while up >= 0:
                path.append(tokens[base + up])
                up = s["parents"][base + up] if c["tree"] else up - 1
            z = s["logits"][base + i].double()
            if c["penalties"]:
                answer = np.bincount(np.concatenate([said[b, prompt[b]:long], path]), minlength=V)
                seen = answer + np.bincount(said[b, :prompt[b]], minlength=V)
                k = torch.from_numpy(answer).to(DEV).double()
                r = torch.where(torch.from_numpy(seen > 0).to(DEV), f64("repetition", b), 1.0).double()
                z = torch.where(z > 0, z / r, z * r) - f64("frequency", b) * k - f64("presence", b) * (k > 0).double()
            if c["bias"]:
                a, e = int(s["bias_start"][b]), int(s["bias_start"][b + 1])
                z = z.index_add(0, s["bias_token"][a:e].long(), s["bias_value"][a:e].double())
            if c["grammar"]:
                bits = np.unpackbits(s["allowed"][base + i].cpu().numpy().view(np.uint8), bitorder="little")[:V]
                z = z.masked_fill(torch.from_numpy(bits == 0).to(DEV), -math.inf)
            p = torch.softmax(z / f64("temperature", b), 0)
            rows.append(torch.nan_to_num(p, nan=0.0))  # (a row of which nothing is allowed)
        base += n
    return [torch.stack(rows)]


def exact_fork(c, s):
    ps, table, kv = c["page"], s["table"].cpu().numpy(), s["kv_len"].cpu().numpy()
    source, keep = continuing(c)
    free, head = s["free"].cpu().numpy(), int(s["head"][0])
    new, lens, held, moves = np.full_like(table, -1), [], [], []
    every = s["all"].clone()
    for b, src in enumerate(source):
        n = min(int(kv[src]), keep[b])
        pages = [int(x) for x in table[src, :-(-n // ps)]]
        move = (-1, -1, 0)
        if n % ps and not (src == b and n // ps == kv[b] // ps):
            move = (pages[-1], int(free[head]), n % ps)
            head += 1
            a, z, w = move[0] * ps, move[1] * ps, c["hkv"] * c["d"]
            every[:, z:z + move[2], :w] = s["all"][:, a:a + move[2], :w]
            pages[-1] = move[1]
        new[b, :len(pages)] = pages
        lens.append(n)
        held.append(len(pages))
        moves.append(move)
    return [i32(new), i32(lens), i32(held), i32([head])] + [i32([m[k] for m in moves]) for k in range(3)] + [every]


def exact_release(c, s):
    rows = lambda t, held: {int(p) for row, h in zip(s[t].cpu().numpy(), s[held].cpu().numpy()) for p in row[:h]}
    gone = sorted(rows("table", "held") - rows("after", "held_after"))
    free, head = s["free_list"].cpu().numpy().copy(), int(s["head"][0]) - len(gone)
    free[head:head + len(gone)] = gone
    return [i32(free), i32([head])]
