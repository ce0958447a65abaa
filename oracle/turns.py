"""Oracle of the calls for further turns (NumPy, float64): written from their definitions, one request,
row and token at a time; shares no code with the HIP path."""
import numpy as np

from .decode import rope


def norm(x, weight=None, eps=0.0):
    """Rows [n, heads, d] over their root mean square per head, times the weight ([d] or [heads, d])."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if weight is None else y * weight


def norm_rope(x, pos, freq, weight=None, eps=0.0, interleaved=False, magnitude=1.0):
    """Normed and turned rows, and the sum of magnitudes of what was turned."""
    y = norm(x, weight, eps)
    return rope(y, pos, freq, interleaved, magnitude) if len(freq) else (y, np.abs(y))


def chunk_see(n, kv, window=0):
    """[n, kv + n]: which tokens each new row sees."""
    see = np.zeros((n, kv + n), bool)
    for i in range(n):
        lo = max(0, kv + i - window + 1) if window else 0
        see[i, lo:kv + i + 1] = True
    return see


def said_by(row, request, history, prompt_len, hist_len, tokens, first, follows):
    """Tokens said in the prompt and in the answer before the row's next one."""
    prompt, answer = [], []
    if history is not None:
        for i in range(max(0, min(int(hist_len), history.shape[1]))):
            (prompt if i < prompt_len else answer).append(int(history[request, i]))
    if tokens is not None:
        answer += [int(tokens[first + j]) for j in follows]
    return prompt, answer


def shape_logits(z, prompt=(), answer=(), repetition=1.0, presence=0.0, frequency=0.0, bias=(), allowed=None,
                 temperature=None):
    """One row: shaped logits (float64), or with a temperature probabilities; and the largest magnitude that each
    token's logit passed through."""
    z = np.array(z, np.float64)
    size = np.abs(z)
    for t in sorted({x for x in list(prompt) + list(answer) if 0 <= x < z.size}):
        c = sum(1 for x in answer if x == t)
        z[t] = z[t] / repetition if z[t] > 0 else z[t] * repetition
        size[t] = max(size[t], abs(z[t]))
        z[t] -= frequency * c
        size[t] = max(size[t], abs(z[t]))
        z[t] -= presence * (c > 0)
        size[t] = max(size[t], abs(z[t]))
    for t, v in dict(bias).items():  # (of several entries the last)
        if 0 <= t < z.size:
            z[t] += v
            size[t] = max(size[t], abs(z[t]), abs(v))
    if allowed is not None:
        z[~allowed] = -np.inf
        size[~allowed] = 0.0
    if temperature is None:
        return z, size
    p = np.zeros_like(z)
    top = z.max()
    if temperature == 0:
        if np.nanmax(z) > -np.inf:
            p[int(np.nanargmax(z))] = 1.0
    elif np.isnan(z).any() or top == np.inf:
        p[:] = np.nan
    elif top > -np.inf:
        p = np.exp((z - top) / temperature)
        p /= p.sum()
    return p, size


def page_fork(table, kv_len, source, free, page_size, n_pages, keep=None, head=0):
    """(table, lengths, held, head, copies [(from, to, rows)]) of the requests that continue others."""
    B, cols = table.shape
    new, lens, held, copies = np.full_like(table, -1), [], [], []
    for b in range(B):
        s = int(source[b])
        n = max(0, int(kv_len[s])) if 0 <= s < B else 0
        if keep is not None:
            n = min(n, max(0, int(keep[b])))
        pages = min(-(-n // page_size), cols)
        if pages:
            new[b, :pages] = table[s, :pages]
        copy = (-1, -1, 0)
        at, part = divmod(n, page_size)
        if part and at < cols and not (s == b and at == max(0, int(kv_len[b])) // page_size):
            page = int(table[s, at])
            if 0 <= page < n_pages:
                to = int(free[head]) if 0 <= head < len(free) else -1
                head += 1
                to = to if 0 <= to < n_pages else -1
                new[b, at] = to
                if to >= 0:
                    copy = (page, to, part)
        lens.append(n)
        held.append(pages)
        copies.append(copy)
    return new, np.array(lens, np.int64), np.array(held, np.int64), head, copies


def page_release(before, held_before, after, held_after, free, head, n_pages):
    """(free list, head) with the pages that only the first table names."""
    cols = before.shape[1]
    named = lambda t, h: {int(p) for row, k in zip(t, h) for p in row[:min(max(int(k), 0), cols)] if 0 <= p < n_pages}
    gone = sorted(named(before, held_before) - named(after, held_after))
    free = np.array(free)
    at = min(max(int(head), 0), len(free)) - len(gone)
    for k, page in enumerate(gone):
        if at + k >= 0:
            free[at + k] = page
    return free, max(at, 0)
