"""Float64 CPU statement of the operators around a round: appending to a paged
cache with the position rotation, attention over that cache, and sampling; the cache in 8 bits
and the pages of a batch.

Written from their definitions, token by token; it shares no code with the CUDA
path.  Caches are [pages, page_size, kv_heads, head_dim], a position p of
sequence b lies in slot p % page_size of page table[b, p // page_size], and it
has no place where that page is outside the cache or the table ends before it.
"""

from __future__ import annotations

import numpy as np


def place(table, pages, page_size, b, p):
    """(page, slot) of position p of sequence b, or None."""
    if p < 0 or p // page_size >= table.shape[1]:
        return None
    page = int(table[b, p // page_size])
    return (page, p % page_size) if 0 <= page < pages else None


def rotate(x, cs, interleaved):
    """The head x [D] with its pairs turned by cs [rot/2, 2] (cos, sin)."""
    y = np.array(x, dtype=np.float64)
    half = cs.shape[0]
    for a in range(half):
        i, j = (2 * a, 2 * a + 1) if interleaved else (a, a + half)
        c, s = float(cs[a, 0]), float(cs[a, 1])
        y[i], y[j] = x[i] * c - x[j] * s, x[j] * c + x[i] * s
    return y


def append(q, k, v, k_cache, v_cache, table, starts, cache_len, rope, interleaved):
    """(q_out, k_cache, v_cache) after the append; the caches are copied."""
    kc, vc, qo = np.array(k_cache, np.float64), np.array(v_cache, np.float64), np.zeros(q.shape)
    for b in range(len(cache_len)):
        for t in range(starts[b], starts[b + 1]):
            p = int(cache_len[b]) + t - starts[b]
            if p < 0 or (rope is not None and p >= rope.shape[0]):
                continue
            cs = np.zeros((0, 2)) if rope is None else rope[p]
            for h in range(q.shape[1]):
                qo[t, h] = rotate(q[t, h], cs, interleaved)
            at = place(table, kc.shape[0], kc.shape[1], b, p)
            if at is None:
                continue
            for h in range(k.shape[1]):
                kc[at][h] = rotate(k[t, h], cs, interleaved)
                vc[at][h] = v[t, h]
    return qo, kc, vc


def attend(q, k_cache, v_cache, table, starts, cache_len, scale, window=0, sinks=0, causal=True):
    """(out, spread): the attention of every token, and sum_j p_j |v_j|, which bounds
    what rounding the weights can change."""
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    pages, page_size, kv_heads, _ = k_cache.shape
    group = q.shape[1] // kv_heads
    for b in range(len(cache_len)):
        n, c = starts[b + 1] - starts[b], int(cache_len[b])
        places = {j: place(table, pages, page_size, b, j) for j in range(max(0, c + n))}
        for i in range(n):
            p = c + i
            seen = [j for j, at in places.items()
                    if at is not None and (j <= p or not causal) and (window <= 0 or j > p - window or j < sinks)]
            if not seen:
                continue
            pg, sl = (np.array(x) for x in zip(*(places[j] for j in seen)))
            k, v = k_cache[pg, sl].astype(np.float64), v_cache[pg, sl].astype(np.float64)
            for h in range(q.shape[1]):
                s = scale * (k[:, h // group] @ q[starts[b] + i, h].astype(np.float64))
                w = np.exp(s - s.max())
                w /= w.sum()
                out[starts[b] + i, h] = w @ v[:, h // group]
                spread[starts[b] + i, h] = w @ np.abs(v[:, h // group])
    return out, spread


def kept_tokens(x, temperature, top_k, top_p, min_p):
    """(tokens, probabilities) that the filters keep, in descending order of the logits."""
    x = np.array(x, np.float64)
    x[np.isnan(x)] = -np.inf
    top = x.max()
    if top == -np.inf:
        return np.zeros(0, np.int64), np.zeros(0)
    order = np.argsort(-x, kind="stable")
    if not temperature > 0:
        return order[:1], np.ones(1)
    d = np.where(x == top, 0.0, x - top) / temperature
    w = np.exp(d[order])
    if 0 < top_k < x.size:
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        before = np.cumsum(w) - w
        keep = before < top_p * w.sum()
        keep[0] = True
        order, w = order[keep], w[keep]
    if min_p > 0:
        keep = w >= min(min_p, 1.0)
        order, w = order[keep], w[keep]
    return order, w / w.sum()


def sample(x, u, temperature, top_k, top_p, min_p):
    """(token, probability) of one row."""
    tokens, probs = kept_tokens(x, temperature, top_k, top_p, min_p)
    if not tokens.size:
        return -1, 0.0
    by_index = np.argsort(tokens)
    run = np.cumsum(probs[by_index])
    at = min(int(np.searchsorted(run, u, side="right")), tokens.size - 1)
    return int(tokens[by_index[at]]), float(probs[by_index[at]])


def e4m3(x):
    """The e4m3 number nearest to each x, of two equally near ones the even one; beyond 448 the largest."""
    x = np.array(x, np.float64)
    _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.clip(np.rint(x / step) * step, -448.0, 448.0)


def page_exponent(x):
    """The least e in [-40, 40] with max |x| <= 448 * 2 ** e (NaN does not count)."""
    a = np.abs(np.asarray(x, np.float64))
    a = float(np.max(np.where(np.isnan(a), 0.0, a), initial=0.0))
    e = -40
    while e < 40 and a > 448.0 * 2.0**e:
        e += 1
    return e


def append_fp8(q, k, v, k_codes, v_codes, k_exp, v_exp, table, starts, cache_len, rope, interleaved,
               rounded=True):
    """(q_out, k_codes, v_codes, k_exp, v_exp) after the append.  Codes are e4m3 numbers as float64; not `rounded`:
    those of the new tokens as they are before their rounding."""
    codes = [np.array(x, np.float64) for x in (k_codes, v_codes)]
    exps = [np.array(x, np.int64) for x in (k_exp, v_exp)]
    qo = np.zeros(q.shape)
    pages, size = codes[0].shape[:2]
    for b in range(len(cache_len)):
        written = {}  # page: [(slot, token)]
        rows = {}
        for t in range(starts[b], starts[b + 1]):
            p = int(cache_len[b]) + t - starts[b]
            if p < 0 or (rope is not None and p >= rope.shape[0]):
                continue
            cs = np.zeros((0, 2)) if rope is None else rope[p]
            qo[t] = [rotate(x, cs, interleaved) for x in q[t]]
            rows[t] = (np.array([rotate(x, cs, interleaved) for x in k[t]]), np.array(v[t], np.float64))
            at = place(table, pages, size, b, p)
            if at is not None:
                written.setdefault(at[0], []).append((at[1], t))
        for page, tokens in written.items():
            first = min(slot for slot, _ in tokens)
            for i in range(2):
                for h in range(k.shape[1]):
                    e = page_exponent([rows[t][i][h] for _, t in tokens])
                    if first > 0:
                        old = min(max(int(exps[i][page, h]), -40), 40)
                        e = max(e, old)
                        if e > old:
                            codes[i][page, :first, h] = e4m3(codes[i][page, :first, h] * 2.0 ** (old - e))
                    for slot, t in tokens:
                        x = rows[t][i][h] * 2.0**-e
                        codes[i][page, slot, h] = e4m3(x) if rounded else x
                    exps[i][page, h] = e
    return qo, *codes, *exps


def reserve(cache_len, new_len, page_size, table, held, free, tokens):
    """(table, held, free, missing, starts, slots) after a call; `free` is a list whose end is the top, `tokens` the
    length of slots."""
    table, held, free = np.array(table), list(held), list(free)
    missing, given, starts, slots = 0, [], [0], []
    for b, (c, n) in enumerate(zip(cache_len, new_len)):
        n = max(int(n), 0)
        need = -(-min(max(int(c) + n, 0), table.shape[1] * page_size) // page_size)
        given += table[b, need:held[b]].tolist()
        table[b, need:held[b]] = -1
        held[b] = min(held[b], need)
        for i in range(held[b], need):
            if free:
                table[b, i] = free.pop()
                held[b] = i + 1
            else:
                table[b, i] = -1
                missing += 1
        for i in range(n):
            at = place(table, 1 << 31, page_size, b, int(c) + i)
            slots.append(-1 if at is None else at[0] * page_size + at[1])
        starts.append(min(starts[-1] + n, tokens))
    return table, held, free + given[::-1], missing, starts, (slots + [-1] * tokens)[:tokens]
