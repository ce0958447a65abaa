"""Answering from the fused cache: the operators that come after the fusion step, in use.

When a request's cache is fused, its answer is decoded from it: the cache lives on in pages, a
pass of the model sees a few new rows per request (one token, or a tree of drafted ones), and
the drafted tokens are checked against the model's probabilities.  The cases are one call each of

  plan    qcf_page_plan: pages for the new rows, their slots, positions and tree masks
  rope    qcf_rope_store: rotary positions of new rows, keys and values into their slots
  attn    qcf_tree_attn: attention of the new rows over a paged cache
  verify  qcf_verify_drafts: which drafted tokens stay, and the next token

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


def listed():
    case = lambda name, kind, **kw: dict(kw, name=name, kind=kind)
    return [
        # one more token for each request of a running batch (the smallest call: latency)
        case("plan_decode", "plan", batch=64, new_lo=1, new_hi=1, ctx_lo=200, ctx_hi=9000, page=64,
             tree=False, layout=1),
        # a tree of drafted tokens for each request of a large batch, with the masks
        case("plan_trees", "plan", batch=256, new_lo=1, new_hi=40, ctx_lo=0, ctx_hi=14000, page=16,
             tree=True, layout=2),
        # a ragged serving batch whose fused caches move into pages: 16 requests, about 117K rows
        case("plan_admit", "plan", batch=16, new_lo=2000, new_hi=12700, ctx_lo=0, ctx_hi=0, page=64,
             tree=False, layout=3),
        # one decoded token of each of 48 requests; adjacent pairs, half of every head rotated
        case("rope_decode", "rope", rows=48, slots=4096, pos_hi=33000, hq=32, hkv=8, d=128, rotary=64,
             interleaved=True, scaling="none", theta=1.0e4, gather=False, dtype="bf16"),
        # float32 rows read through an index, a quarter of each 64-wide head rotated
        case("rope_f32", "rope", rows=2500, slots=6000, pos_hi=12000, hq=16, hkv=4, d=64, rotary=16,
             interleaved=False, scaling="linear", theta=1.0e6, gather=True, dtype="f32"),
        # a 32K-token prompt with 64/8 heads of 128, frequencies stretched by parts
        case("rope_prompt", "rope", rows=32896, slots=33024, pos_hi=32896, hq=64, hkv=8, d=128,
             rotary=128, interleaved=False, scaling="parts", theta=5.0e5, gather=False, dtype="bf16"),
        # a test-sized model in float32: three requests, small trees
        case("attn_small_f32", "attn", batch=3, new_lo=2, new_hi=8, ctx_lo=33, ctx_hi=700, page=16,
             tree=True, hq=8, hkv=2, d=64, dtype="f32", layout=4),
        # decoding: 64 requests, one token each
        case("attn_decode", "attn", batch=64, new_lo=1, new_hi=1, ctx_lo=512, ctx_hi=8192, page=64,
             tree=False, hq=32, hkv=8, d=128, dtype="bf16", layout=5),
        # drafted trees over a ragged serving batch
        case("attn_tree", "attn", batch=16, new_lo=8, new_hi=40, ctx_lo=2000, ctx_hi=12700, page=64,
             tree=True, hq=32, hkv=8, d=128, dtype="bf16", layout=6),
        # one 32K-token request with 64/8 heads and a wide tree
        case("attn_long_tree", "attn", batch=1, new_lo=64, new_hi=64, ctx_lo=32896, ctx_hi=32896, page=128,
             tree=True, hq=64, hkv=8, d=128, dtype="bf16", layout=7),
        # chains of four drafted tokens with the draft's own probabilities
        case("verify_chain", "verify", batch=64, new_lo=5, new_hi=5, vocab=128000, draft=True, tree=False,
             dtype="f32", layout=8),
        # trees drafted without probabilities, a large vocabulary in bfloat16
        case("verify_tree", "verify", batch=16, new_lo=10, new_hi=26, vocab=150001, draft=False, tree=True,
             dtype="bf16", layout=9),
    ]


def draw(rng):
    """Another case of the ranges the listed ones stand for."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["plan", "rope", "attn", "attn", "attn", "verify"])
    layout = rng.randrange(10, 1 << 20)
    if kind == "plan":
        if rng.random() < 0.3:  # prompts
            batch = log(1, 24)
            hi = log(50, 120000 // batch)
            return dict(kind=kind, batch=batch, new_lo=max(1, hi // 6), new_hi=hi, ctx_lo=0, ctx_hi=0,
                        page=rng.choice([16, 32, 64, 128]), tree=False, layout=layout)
        hi = rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 64)])
        return dict(kind=kind, batch=log(1, 400), new_lo=rng.randint(min(1, hi - 1), hi), new_hi=hi, ctx_lo=0,
                    ctx_hi=log(100, 15000), page=rng.choice([8, 16, 32, 64, 128]),
                    tree=hi > 1 and rng.random() < 0.7, layout=layout)
    heads = [(8, 2, 64), (16, 4, 64), (32, 8, 64), (8, 8, 128), (16, 1, 128), (32, 8, 128), (32, 8, 128),
             (40, 10, 128), (64, 8, 128)]
    hq, hkv, d = rng.choice(heads)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "rope":
        rows = log(1, 12000 if dtype == "f32" else 30000)
        return dict(kind=kind, rows=rows, slots=rows + rng.randint(0, 3000), pos_hi=log(1000, 130000), hq=hq,
                    hkv=hkv, d=d, rotary=16 * rng.randint(1, d // 16), interleaved=rng.random() < 0.5,
                    scaling=rng.choice(["none", "linear", "parts"]), theta=rng.choice([1.0e4, 5.0e5, 1.0e6]),
                    gather=rng.random() < 0.3, dtype=dtype)
    if kind == "attn":
        hi = rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 40)])
        # keys of the whole batch, bounded so that no draw costs more than the largest case
        keys = log(200, 20000 if dtype == "f32" else 170000 if hi <= 8 else 60000)
        batch = min(rng.choice([1, 2, log(1, 64)]), max(1, keys // 40))
        top = max(2, keys // batch)
        return dict(kind=kind, batch=batch, new_lo=max(1, hi // 3), new_hi=hi, ctx_lo=rng.choice([0, 1, top // 4]),
                    ctx_hi=top, page=rng.choice([8, 16, 32, 64, 128]), tree=hi > 1 and rng.random() < 0.7,
                    hq=hq, hkv=hkv, d=d, dtype=dtype, layout=layout)
    hi = rng.randint(1, 12)
    vocab = log(900, 150000)
    batch = max(1, min(log(1, 64), 30_000_000 // (hi * vocab)))
    return dict(kind=kind, batch=batch, new_lo=rng.randint(1, hi), new_hi=hi, vocab=vocab,
                draft=rng.random() < 0.6, tree=rng.random() < 0.5, dtype=rng.choice(["f32", "bf16"]),
                layout=layout)


# ---------------------------------------------------------------------------
# lengths (from the case alone)
# ---------------------------------------------------------------------------
def lengths(c):
    """(new rows, rows held) per request; the extremes occur where there is room for them."""
    r = random.Random(c["layout"])
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["batch"])]
    ctx = [r.randint(c.get("ctx_lo", 0), c.get("ctx_hi", 0)) for _ in range(c["batch"])]
    new[0], ctx[0] = c["new_hi"], c.get("ctx_hi", 0)
    if c["batch"] > 2:
        new[-1], ctx[-1] = c["new_lo"], c.get("ctx_lo", 0)
    return new, ctx


def work(c):
    if c["kind"] == "rope":
        es = 2 if c["dtype"] == "bf16" else 4
        row = (c["hq"] + 2 * c["hkv"]) * c["d"] * es
        turned = (c["hq"] + c["hkv"]) * c["rotary"]
        return {"bytes": c["rows"] * (2 * row + 8 + (4 if c["gather"] else 0)), "flops": 3 * c["rows"] * turned}
    new, ctx = lengths(c)
    n = sum(new)
    if c["kind"] == "plan":
        pages = [-(-(a + b) // c["page"]) - (-(-b // c["page"])) for a, b in zip(new, ctx)]
        words = (max(new) + 31) // 32 if c["tree"] else 0
        return {"bytes": c["batch"] * 24 + n * (8 + (4 + 4 * words if c["tree"] else 0)) + sum(pages) * 8,
                "flops": 4 * n}
    if c["kind"] == "attn":
        es = 2 if c["dtype"] == "bf16" else 4
        keys = sum(a + b for a, b in zip(new, ctx))
        # a row sees the rows held, itself and, of the drafted ones, at least its parent's chain
        seen = sum(a * (b + (a + 1) / 2) for a, b in zip(new, ctx))
        return {"bytes": keys * 2 * c["hkv"] * c["d"] * es + n * c["hq"] * (2 * c["d"] * es + 4),
                "flops": 4 * c["hq"] * c["d"] * seen}
    es = 2 if c["dtype"] == "bf16" else 4
    two = 2 if c["draft"] else 1
    # one row of the target's (and the draft's) probabilities per request, a few numbers per drafted token
    return {"bytes": c["batch"] * c["vocab"] * es * two + n * (12 + es * two),
            "flops": c["batch"] * c["vocab"] * two}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to(DEV)


def grow_trees(rng, new):
    """Parents (index within the request, -1 for the first row) of ragged trees."""
    out = []
    for n in new:
        p = np.full(n, -1, np.int32)
        for i in range(1, n):
            p[i] = rng.integers(max(0, i - 6), i)
        out.append(p)
    return np.concatenate(out) if out else np.zeros(0, np.int32)


def ancestor_bits(parents, new, words):
    """[rows, words] bits of each row's ancestors and itself."""
    m = np.zeros((len(parents), words), np.uint32)
    base = 0
    for n in new:
        for i in range(n):
            r = base + i
            if parents[r] >= 0:
                m[r] = m[base + parents[r]]
            m[r, i // 32] |= np.uint32(1 << (i % 32))
        base += n
    return m.view(np.int32)


def rotary_frequencies(c):
    """Angular frequencies of the case in float64 (one per rotated pair)."""
    R = c["rotary"]
    w = c["theta"] ** (-np.arange(0, R, 2, dtype=np.float64) / R)
    if c["scaling"] == "linear":
        return w / 4.0
    if c["scaling"] == "parts":  # slow turns are stretched by 8, fast ones kept, in between blended
        turns = 8192.0 * w / (2.0 * math.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return (1.0 - keep) * w / 8.0 + keep * w
    return w


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
        s["call"] = globals()["own_" + c["kind"]](c, s, qcf)
    return s


def prepare_plan(c, s, rng, normal):
    new, ctx = lengths(c)
    ps = c["page"]
    held = [-(-x // ps) for x in ctx]
    need = [-(-(a + b) // ps) for a, b in zip(new, ctx)]
    width = max(need) + 3
    pages = sum(need) + 50
    order = rng.permutation(pages)
    table = np.full((c["batch"], width), -1, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    n = sum(new)
    rows = n + 7  # the packed rows of a replayed step: a few behind the last request stay unused
    s.update(kv_len=i32(ctx), new_len=i32(new), table=i32(table), free=i32(order[at:]), pages=pages, rows=rows,
             max_new=max(new), held=i32(held), head=i32([0]))
    e = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)
    s.update(slots=e(rows), positions=e(rows), cu_new=e(c["batch"] + 1), kv_end=e(c["batch"]),
             held_out=e(c["batch"]), head_out=e(1))
    s["words"] = (max(new) + 31) // 32
    if c["tree"]:
        s["parents"] = i32(np.concatenate([grow_trees(rng, new), np.full(7, -1, np.int32)]))
        s["mask"] = e(rows, s["words"])


def prepare_rope(c, s, rng, normal):
    dt = DT[c["dtype"]]
    src = c["rows"] + 100 if c["gather"] else c["rows"]
    # the rows of one product x W_qkv: queries, keys and values side by side
    qkv = (normal(src, (c["hq"] + 2 * c["hkv"]) * c["d"])).to(dt)
    q, k, v = qkv.split([c["hq"] * c["d"], c["hkv"] * c["d"], c["hkv"] * c["d"]], dim=1)
    s.update(q=q.view(src, c["hq"], c["d"]), k=k.view(src, c["hkv"], c["d"]), v=v.view(src, c["hkv"], c["d"]))
    s["slots"] = i32(rng.permutation(c["slots"])[:c["rows"]])
    pos = rng.integers(0, c["pos_hi"], c["rows"]) if c["rows"] != c["pos_hi"] else np.arange(c["rows"])
    s["positions"] = i32(pos)
    s["src"] = i32(rng.permutation(src)[:c["rows"]]) if c["gather"] else None
    s["inv_freq"] = torch.from_numpy(rotary_frequencies(c)).to(DEV)
    s["magnitude"] = 1.0 if c["scaling"] != "parts" else 0.1 * math.log(8.0) + 1.0
    s["k_cache"], s["v_cache"] = (pool(c["slots"], c["hkv"], c["d"], dt) for _ in range(2))
    s["q_out"] = torch.empty((c["rows"], c["hq"], c["d"]), dtype=dt, device=DEV)


def prepare_attn(c, s, rng, normal):
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
    s.update(table=i32(table), kv_len=i32(ctx), cu=i32(np.concatenate([[0], np.cumsum(new)])), new=new, ctx=ctx,
             scale=1.0 / math.sqrt(c["d"]), mask=None, parents=None)
    if c["tree"]:
        s["parents"] = grow_trees(rng, new)
        s["mask"] = i32(ancestor_bits(s["parents"], new, (max(new) + 31) // 32))


def prepare_verify(c, s, rng, normal):
    dt = DT[c["dtype"]]
    new, _ = lengths(c)
    n, V = sum(new), c["vocab"]
    # the draft's logits are the target's with some noise
    z = 3.0 * normal(n, V)
    target = torch.softmax(z, 1)
    z += normal(n, V)
    draft = torch.softmax(z, 1)
    del z
    if c["tree"]:
        parents = grow_trees(rng, new)
    else:
        parents = np.concatenate([np.arange(-1, m - 1) for m in new]).astype(np.int32)
    base = np.repeat(np.concatenate([[0], np.cumsum(new)[:-1]]), new)
    up = torch.from_numpy(base + np.maximum(parents, 0)).to(DEV)
    if c["draft"]:  # drawn from the draft's probabilities at the parent
        seed = int(rng.integers(1 << 31))
        pick = torch.multinomial(draft, 16, replacement=True,
                                 generator=torch.Generator(device=DEV).manual_seed(seed))
    else:           # the most likely ones at the parent
        pick = torch.topk(draft, 16, dim=1).indices
    nth = np.zeros(n, np.int64)
    seen = {}
    for r in range(n):
        key = (base[r], parents[r])
        nth[r] = seen.get(key, 0) % 16
        seen[key] = seen.get(key, 0) + 1
    tokens = pick[up, torch.from_numpy(nth).to(DEV)].to(torch.int32)
    s.update(target=target.to(dt), draft=draft.to(dt) if c["draft"] else None, tokens=tokens,
             parents=i32(parents) if c["tree"] else None, cu=i32(np.concatenate([[0], np.cumsum(new)])), new=new,
             u=torch.from_numpy(rng.random(n, dtype=np.float32)).to(DEV),
             u_last=torch.from_numpy(rng.random(c["batch"], dtype=np.float32)).to(DEV))
    e = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)
    s.update(n_out=e(c["batch"]), path=e(c["batch"], max(new)), out_tokens=e(c["batch"], max(new)))


# ---------------------------------------------------------------------------
# the framework's operators: each call is validated once and replayed, as its steps do
# ---------------------------------------------------------------------------
def own_plan(c, s, qcf):
    tree = dict(parents=s["parents"], tree_mask=s["mask"]) if c["tree"] else {}
    return qcf.prepare(qcf.qcf_page_plan, s["table"], s["kv_len"], s["new_len"], s["free"], s["slots"],
                       s["positions"], s["cu_new"], c["page"], s["pages"], s["max_new"], pages_held=s["held"],
                       free_head=s["head"], kv_end=s["kv_end"], pages_held_out=s["held_out"],
                       free_head_out=s["head_out"], **tree)


def own_rope(c, s, qcf):
    return qcf.prepare(qcf.qcf_rope_store, s["k_cache"], s["v_cache"], s["k"], s["v"], s["slots"], s["positions"],
                       s["inv_freq"], interleaved=c["interleaved"], magnitude=s["magnitude"], q_new=s["q"],
                       q_out=s["q_out"], src_idx=s["src"])


def own_attn(c, s, qcf):
    new, ctx = s["new"], s["ctx"]
    max_kv = max(a + b for a, b in zip(new, ctx))
    need = qcf.qcf_tree_attn_workspace_size(c["batch"], max(new), max_kv, c["hq"], c["hkv"], c["d"], DT[c["dtype"]])
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    return qcf.prepare(qcf.qcf_tree_attn, s["out"], s["q"], s["cu"], s["k_cache"], s["v_cache"], s["table"],
                       s["kv_len"], c["page"], max(new), max_kv, s["scale"], tree_mask=s["mask"], lse=s["lse"],
                       workspace=s["ws"])


def own_verify(c, s, qcf):
    need = qcf.qcf_verify_drafts_workspace_size(c["batch"], c["vocab"])
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    return qcf.prepare(qcf.qcf_verify_drafts, s["n_out"], s["path"], s["out_tokens"], s["target"], s["tokens"],
                       s["cu"], s["u"], s["u_last"], draft=s["draft"], parents=s["parents"], workspace=s["ws"])


OUT = {"plan": ("slots", "positions", "cu_new", "kv_end", "held_out", "head_out", "table"),
       "rope": ("k_cache", "v_cache", "q_out"), "attn": ("out", "lse"), "verify": ("n_out", "path", "out_tokens")}


def run(s):
    c = s["case"]
    if own:
        s["call"]()
        names = OUT[c["kind"]] + (("mask",) if c["kind"] == "plan" and c["tree"] else ())
        return [s[k] for k in names]
    return globals()["plain_" + c["kind"]](c, s)


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def plain_plan(c, s):
    ps = c["page"]
    kv, new, held = s["kv_len"].long(), s["new_len"].long(), s["held"].long()
    rows, B = s["rows"], c["batch"]
    need = torch.maximum(torch.div(kv + new + ps - 1, ps, rounding_mode="floor"), held)
    fresh = need - held
    first = s["head"].long() + torch.cumsum(fresh, 0) - fresh      # place in the free list
    cu = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    col = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    at = first[:, None] + col - held[:, None]
    take = (col >= held[:, None]) & (col < need[:, None])
    page = s["free"].long()[at.clamp(0, s["free"].numel() - 1)]
    table = torch.where(take, page, s["table"].long())
    t = torch.arange(rows, device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    used = t < cu[-1]
    bb = b.clamp(0, B - 1)
    i = t - cu[bb]
    logical = kv[bb] + i
    pg = torch.div(logical, ps, rounding_mode="floor").clamp(0, table.shape[1] - 1)
    slot = table[bb, pg] * ps + logical % ps
    depth = i
    out = []
    if c["tree"]:
        bits = torch.zeros((rows, s["words"] * 32), dtype=torch.long, device=DEV)
        at, depth = torch.where(used, i, -1), torch.full_like(i, -1)
        par = s["parents"].long()
        for _ in range(s["max_new"]):
            live = at >= 0
            bits.scatter_reduce_(1, at.clamp(min=0)[:, None], live.long()[:, None], "amax")
            depth = depth + live.long()
            at = torch.where(live, par[(cu[bb] + at).clamp(0, rows - 1)], at)
        two = torch.ones(32, dtype=torch.long, device=DEV) << torch.arange(32, device=DEV)
        w = (bits.view(rows, s["words"], 32) * two).sum(2)
        out = [torch.where(w >= 1 << 31, w - (1 << 32), w).int()]
    none = torch.full_like(t, -1)
    return [torch.where(used, slot, none).int(), torch.where(used, kv[bb] + depth, none).int(), cu.int(),
            (kv + new).int(), need.int(), (s["head"].long() + fresh.sum()).int(), table.int()] + out


def plain_rope(c, s):
    R, rows = c["rotary"], s["slots"].long()
    src = s["src"].long() if c["gather"] else torch.arange(c["rows"], device=DEV)
    angle = s["positions"].double()[:, None] * s["inv_freq"][None, :]
    cos = (torch.cos(angle) * s["magnitude"]).float()[:, None, :]
    sin = (torch.sin(angle) * s["magnitude"]).float()[:, None, :]

    def turn(x):
        x = x.float()
        a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
        y, z = a * cos - b * sin, a * sin + b * cos
        y = torch.stack([y, z], -1).flatten(-2) if c["interleaved"] else torch.cat([y, z], -1)
        return torch.cat([y, x[..., R:]], -1).to(DT[c["dtype"]])

    s["k_cache"][rows] = turn(s["k"][src])
    s["v_cache"][rows] = s["v"][src]
    return [s["k_cache"], s["v_cache"], turn(s["q"][src])]


def plain_attn(c, s):
    ps, g = c["page"], c["hq"] // c["hkv"]
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    base = 0
    for b, (n, held) in enumerate(zip(s["new"], s["ctx"])):
        j = torch.arange(held + n, device=DEV)
        slot = s["table"][b, torch.div(j, ps, rounding_mode="floor")].long() * ps + j % ps
        k = s["k_cache"][slot].float().transpose(0, 1)                              # [hkv, keys, d]
        v = s["v_cache"][slot].float().transpose(0, 1).contiguous()
        q = s["q"][base:base + n].float().view(n, c["hkv"], g, -1).permute(1, 2, 0, 3).reshape(c["hkv"], g * n, -1)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) * s["scale"]
        t = torch.arange(n, device=DEV)
        if s["mask"] is None:
            see = t[None, :] <= t[:, None]
        else:
            see = (s["mask"][base:base + n][:, torch.div(t, 32, rounding_mode="floor")] >> (t % 32)) & 1 == 1
        x = x.view(c["hkv"], g, n, held + n)
        x[..., held:] = torch.where(see, x[..., held:], -math.inf)
        top = x.amax(-1, keepdim=True)
        e = torch.exp(x - top)
        tot = e.sum(-1, keepdim=True)
        o = torch.matmul((e / tot).view(c["hkv"], g * n, -1), v).view(c["hkv"], g, n, -1)
        out[base:base + n] = o.permute(2, 0, 1, 3).reshape(n, c["hq"], -1).to(out.dtype)
        lse[base:base + n] = (top + torch.log(tot)).squeeze(-1).permute(2, 0, 1).reshape(n, -1)
        base += n
    return [out, lse]


def plain_verify(c, s):
    """All requests in step over their rows' indices; sums and comparisons in 64 bits."""
    B, V, W = c["batch"], c["vocab"], max(s["new"])
    cu = s["cu"].long()
    new = cu[1:] - cu[:-1]
    req = torch.arange(B, device=DEV)
    cur, count = torch.zeros(B, dtype=torch.long, device=DEV), torch.ones(B, dtype=torch.long, device=DEV)
    Z, coef = torch.ones(B, dtype=torch.double, device=DEV), torch.zeros(B, dtype=torch.double, device=DEV)
    path = torch.full((B, W), -1, dtype=torch.long, device=DEV)
    toks = torch.full((B, W + 1), -1, dtype=torch.long, device=DEV)
    path[:, 0] = 0
    last = cu[-1] - 1
    gone = torch.zeros((B, V), dtype=torch.bool, device=DEV)       # tokens refused at the current row
    pos = lambda x: torch.where(x > 0, x, torch.zeros_like(x))
    chain = torch.arange(W, device=DEV) - 1

    def residual():
        p = pos(s["target"][cu[:-1] + cur].double())
        if c["draft"]:
            return pos(p - coef[:, None] * pos(s["draft"][cu[:-1] + cur].double()))
        return torch.where(gone, torch.zeros_like(p), p)

    for j in range(1, W):
        row = torch.minimum(cu[:-1] + j, last)
        par = s["parents"][row].long() if c["tree"] else chain[j].expand(B)
        test = (j < new) & (par == cur)
        x = s["tokens"][row].long()
        at = cu[:-1] + cur
        p = pos(s["target"][at, x].double())
        if c["draft"]:
            qx = pos(s["draft"][at, x].double())
            rx = pos(p - coef * qx)
        else:
            qx = torch.ones_like(p)
            rx = torch.where(gone[req, x], torch.zeros_like(p), p)
        yes = test & (s["u"][row].double() * Z * qx < rx)
        no = test & ~yes
        if c["draft"]:
            coef = torch.where(no, coef + Z, coef)
            if c["tree"]:
                Z = torch.where(no, residual().sum(1), Z)
        else:
            Z = torch.where(no, pos(Z - rx), Z)
            gone[req, x] |= no
        toks[req, torch.where(yes, count - 1, W)] = x
        path[req, torch.where(yes, count, 0)] = torch.where(yes, j, 0)
        count = count + yes.long()
        cur = torch.where(yes, j, cur)
        Z, coef = torch.where(yes, 1.0, Z), torch.where(yes, 0.0, coef)
        gone &= ~yes[:, None]
    r = residual()
    empty = r.sum(1, keepdim=True) == 0
    r = torch.where(empty, pos(s["target"][cu[:-1] + cur].double()), r)
    cum = torch.cumsum(r, 1)
    over = cum > s["u_last"].double()[:, None] * cum[:, -1:]
    toks[req, count - 1] = over.int().argmax(1)
    return [count.int(), path.int(), toks[:, :W].int()]


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(c, seed):
    if c["kind"] == "attn":
        new, ctx = lengths(c)
        if sum(a * (a + b) for a, b in zip(new, ctx)) * c["hq"] * c["d"] > 2e11:
            return None
    s = prepare(c, seed)
    return globals()["exact_" + c["kind"]](c, s)


def exact_plan(c, s):
    n = lambda t: t.cpu().numpy().astype(np.int64)
    kv, new, held, free, table = n(s["kv_len"]), n(s["new_len"]), n(s["held"]), n(s["free"]), n(s["table"])
    ps, rows = c["page"], s["rows"]
    slots, positions = np.full(rows, -1), np.full(rows, -1)
    mask = np.zeros((rows, s["words"] * 32), np.uint8)
    cu, held_out = [0], held.copy()
    head = at = 0
    par = n(s["parents"]) if c["tree"] else None
    for b in range(c["batch"]):
        while held_out[b] * ps < kv[b] + new[b]:
            table[b, held_out[b]] = free[head]
            held_out[b] += 1
            head += 1
        level = []
        for i in range(new[b]):
            where = kv[b] + i
            slots[at] = table[b, where // ps] * ps + where % ps
            if c["tree"]:
                up = par[at]
                level.append(0 if up < 0 else level[up] + 1)
                if up >= 0:
                    mask[at] = mask[at - i + up]
                mask[at, i] = 1
            positions[at] = kv[b] + (level[i] if c["tree"] else i)
            at += 1
        cu.append(at)
    out = [slots, positions, cu, kv + new, held_out, [head], table]
    if c["tree"]:
        out.append(np.packbits(mask, axis=1, bitorder="little").view(np.int32))
    return [i32(x) for x in out]


def exact_rope(c, s):
    src = s["src"].long() if c["gather"] else slice(None)
    R = c["rotary"]
    w = torch.exp(1j * s["positions"].double()[:, None, None] * s["inv_freq"]) * s["magnitude"]

    def turn(x):
        x = x[src].double()
        y = x.clone()
        if c["interleaved"]:
            z = torch.view_as_complex(x[..., :R].unflatten(-1, (R // 2, 2)).contiguous()) * w
            y[..., :R] = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * w
            y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
        return y

    out = []
    for new in (turn(s["k"]), s["v"][src].double()):
        cache = torch.zeros((c["slots"], c["hkv"], c["d"]), dtype=torch.double, device=DEV)
        out.append(cache.index_copy_(0, s["slots"].long(), new))
    return out + [turn(s["q"])]


def exact_attn(c, s):
    outs, lses = [], []
    base, g = 0, c["hq"] // c["hkv"]
    table = s["table"].cpu().numpy().astype(np.int64)
    for b, (n, held) in enumerate(zip(s["new"], s["ctx"])):
        slot = np.array([table[b, j // c["page"]] * c["page"] + j % c["page"] for j in range(held + n)], np.int64)
        slot = torch.from_numpy(slot).to(DEV)
        see = np.zeros((n, held + n), bool)
        see[:, :held] = True
        for i in range(n):
            up = i
            while up >= 0:
                see[i, held + up] = True
                up = s["parents"][base + up] if s["parents"] is not None else up - 1
        hide = torch.from_numpy(~see).to(DEV)
        o = torch.empty((n, c["hq"], c["d"]), dtype=torch.double, device=DEV)
        e = torch.empty((n, c["hq"]), dtype=torch.double, device=DEV)
        for h in range(c["hq"]):
            k, v = (s[name][slot, h // g].double() for name in ("k_cache", "v_cache"))
            x = (s["q"][base:base + n, h].double() @ k.T * s["scale"]).masked_fill(hide, -math.inf)
            e[:, h] = torch.logsumexp(x, 1)
            o[:, h] = torch.exp(x - e[:, h, None]) @ v
        outs.append(o)
        lses.append(e)
        base += n
    return [torch.cat(outs), torch.cat(lses)]


def exact_verify(c, s):
    B, W = c["batch"], max(s["new"])
    n_out, path, toks = np.zeros(B, np.int64), np.full((B, W), -1), np.full((B, W), -1)
    tokens, u, u_last = (s[k].cpu().numpy() for k in ("tokens", "u", "u_last"))
    parents = s["parents"].cpu().numpy() if c["tree"] else None
    base = 0
    for b, n in enumerate(s["new"]):
        cur, went = 0, [0]
        dist = lambda name, row: s[name][base + row].double().cpu().numpy()
        p = r = dist("target", 0)
        q = dist("draft", 0) if c["draft"] else None
        Z, refused = 1.0, 0.0
        for j in range(1, n):
            if (parents[base + j] if c["tree"] else j - 1) != cur:
                continue
            x = tokens[base + j]
            if float(u[base + j]) * Z * (q[x] if c["draft"] else 1.0) < r[x]:
                cur = j
                went.append(j)
                toks[b, len(went) - 2] = x
                p = r = dist("target", cur)
                q = dist("draft", cur) if c["draft"] else None
                Z, refused = 1.0, 0.0
            elif c["draft"]:
                refused += Z
                r = np.maximum(p - refused * q, 0.0)
                Z = math.fsum(r) if c["tree"] else Z
            else:
                Z = max(Z - r[x], 0.0)
                r = r.copy()
                r[x] = 0.0
        if not r.any():
            r = p
        cum = np.cumsum(r)
        toks[b, len(went) - 1] = int(np.searchsorted(cum, float(u_last[b]) * cum[-1], side="right"))
        n_out[b] = len(went)
        path[b, :len(went)] = went
        base += n
    return [i32(n_out), i32(path), i32(toks)]
