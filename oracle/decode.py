"""Oracle of the decoding operators (NumPy, float64): written from their definitions, one request,
row and token at a time; shares no code with the HIP path."""
import math

import numpy as np


def page_plan(table, kv_len, new_len, free, page_size, n_pages, n_rows, held=None, head=0, parents=None, words=0):
    """(table, slots, positions, mask bits [rows, 32 * words], cu, kv_end, held, head) after a plan."""
    table = np.array(table, np.int64)
    B, cols = table.shape
    slots, positions = np.full(n_rows, -1, np.int64), np.full(n_rows, -1, np.int64)
    mask = np.zeros((n_rows, 32 * words), bool)
    cu, out_held, end = [0], [], []
    for b in range(B):
        kv, new = max(int(kv_len[b]), 0), max(int(new_len[b]), 0)
        mine = max(-(-kv // page_size), int(held[b]) if held is not None else 0)
        mine = min(mine, cols)
        need = max(mine, min(-(-(kv + new) // page_size), cols))
        for c in range(mine, need):
            page = int(free[head]) if 0 <= head < len(free) else -1
            table[b, c] = page if 0 <= page < n_pages else -1
            head += 1
        depth = []
        for i in range(new):
            r = cu[-1] + i
            up = int(parents[r]) if parents is not None and r < n_rows else -1
            up = up if 0 <= up < i else -1
            depth.append(i if parents is None else 0 if up < 0 else depth[up] + 1)
            if r >= n_rows:
                continue
            t = kv + i
            page = table[b, t // page_size] if t // page_size < need else -1
            if 0 <= page < n_pages:
                slots[r] = page * page_size + t % page_size
            positions[r] = kv + depth[i]
            if parents is not None:
                if up >= 0:
                    mask[r] = mask[cu[-1] + up]
                if i < mask.shape[1]:
                    mask[r, i] = True
        cu.append(cu[-1] + new)
        out_held.append(need)
        end.append(kv + new)
    return table, slots, positions, mask, np.array(cu), np.array(end), np.array(out_held), head


def pack_bits(mask):
    """[rows, 32 w] booleans as int32 words."""
    return np.packbits(mask.astype(np.uint8), axis=1, bitorder="little").view(np.int32)


def rope_frequencies(rotary_dim, theta, scaling="none", factor=1.0, low_turns=1.0, high_turns=4.0, trained_len=0.0):
    out = []
    for j in range(rotary_dim // 2):
        w = theta ** (-2 * j / rotary_dim)
        if scaling == "linear":
            w /= factor
        elif scaling == "by_parts":
            g = min(max((trained_len / (2 * math.pi / w) - low_turns) / (high_turns - low_turns), 0.0), 1.0)
            w = (1 - g) * (w / factor) + g * w
        out.append(w)
    return np.array(out)


def rope(x, pos, freq, interleaved=False, magnitude=1.0):
    """Turned rows [n, heads, d] (float64) and the sum of magnitudes that bounds their rounding."""
    y, size = np.array(x, np.float64), np.abs(np.array(x, np.float64))
    R = 2 * len(freq)
    for j, w in enumerate(freq):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + R // 2)
        ang = np.asarray(pos, np.float64) * w
        c, s = magnitude * np.cos(ang)[:, None], magnitude * np.sin(ang)[:, None]
        xa, xb = np.array(x[..., a], np.float64), np.array(x[..., b], np.float64)
        y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
        size[..., a] = size[..., b] = abs(magnitude) * (np.abs(xa) + np.abs(xb))
    return y, size


def tree_attention(q, k, v, see, scale):
    """q [n, hq, d] over a request's tokens k, v [t, hkv, d]; see [n, t] booleans.  Returns the output,
    the log-sum-exp, and per (row, head): sum of weights times |v|, and the largest sum |q||k| scale."""
    n, hq, d = q.shape
    g = hq // k.shape[1] if k.shape[0] else 1
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    absv, absx = np.zeros((n, hq, d)), np.zeros((n, hq))
    for h in range(hq):
        for i in range(n):
            t = np.nonzero(see[i])[0]
            if t.size == 0:
                continue
            kk, vv = k[t, h // g], v[t, h // g]
            x = kk @ q[i, h] * scale
            top = x.max()
            e = np.exp(x - top)
            w = e / e.sum()
            out[i, h] = w @ vv
            lse[i, h] = top + np.log(e.sum())
            absv[i, h] = w @ np.abs(vv)
            absx[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, lse, absv, absx


def chain_see(n, kv):
    return np.concatenate([np.ones((n, kv), bool), np.tril(np.ones((n, n), bool))], 1)


def verify(target, draft, tokens, parents, u_accept, u_next):
    """One request: (rows that stay, tokens that come out)."""
    n, vocab = target.shape
    if n == 0:
        return [], []
    zero = lambda x: np.where(x > 0, x, 0.0).astype(np.float64)
    cur, path, out = 0, [0], []
    while True:
        P = zero(target[cur])
        D = zero(draft[cur]) if draft is not None else None
        R, Z, c = P.copy(), 1.0, 0.0
        step = None
        for j in range(cur + 1, n):
            if (parents[j] if parents is not None else j - 1) != cur or not 0 <= tokens[j] < vocab:
                continue
            x = tokens[j]
            if float(u_accept[j]) * Z * (D[x] if D is not None else 1.0) < R[x]:
                step = j
                break
            if D is not None:
                c += Z
                R = np.maximum(P - c * D, 0.0)
                Z = math.fsum(R)
            else:
                Z = max(Z - R[x], 0.0)
                R[x] = 0.0
        if step is None:
            break
        cur = step
        path.append(step)
        out.append(int(tokens[step]))
    if not R.any():
        R = P
    cum = np.cumsum(R)
    if not R.any():
        return path, out + [-1]
    t = int(np.searchsorted(cum, float(u_next) * cum[-1], side="right"))
    return path, out + [t if t < vocab else int(np.nonzero(R)[0][-1])]
