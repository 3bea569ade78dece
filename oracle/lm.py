"""Plain fp64 forms of the language model's own step: cache append, attention of drafts, weights of cached keys,
eviction, adjusted scores, sampling.

numpy on the host, one row, head and token after the other; tensors come as fp64 arrays of the values that the element
type holds.
"""
from __future__ import annotations

import math

import numpy as np


def sequence_of(row_offsets, t: int) -> int:
    """The sequence that owns row t, or -1 for a row behind the last one."""
    for s in range(len(row_offsets) - 1):
        if row_offsets[s] <= t < row_offsets[s + 1]:
            return s
    return -1


def rotate(x, position: float, inv_freq, interleaved: bool):
    """One head [d] with its first 2 len(inv_freq) elements rotated by position * inv_freq."""
    out = np.array(x, np.float64)
    half = len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = float(position) * float(inv_freq[i])
        c, s = math.cos(angle), math.sin(angle)
        out[a], out[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return out


def append(q, k, v, k_cache, v_cache, pages, row_offsets, cache_lens, rows: int, q_out=None, positions=None,
           inv_freq=None, interleaved=False, source_rows=None):
    """(q_out, k_cache, v_cache) after the append, as new arrays; caches [pages, heads, page size, d]."""
    k_cache, v_cache = np.array(k_cache, np.float64), np.array(v_cache, np.float64)
    q_out = None if q is None else np.array(q_out, np.float64)
    freq = np.zeros(0) if inv_freq is None else np.asarray(inv_freq, np.float64)
    n_pages, heads, page_size, _ = k_cache.shape
    for t in range(rows):
        s = sequence_of(row_offsets, t)
        if s < 0:
            continue
        src = t if source_rows is None else int(source_rows[t])
        if not 0 <= src < k.shape[0]:
            continue
        c = int(cache_lens[s]) + t - int(row_offsets[s])
        p = c if positions is None else int(positions[t])
        if q is not None:
            for h in range(q.shape[1]):
                q_out[t, h] = rotate(q[src, h], p, freq, interleaved)
        if not 0 <= c < pages.shape[1] * page_size:
            continue
        page = int(pages[s, c // page_size])
        if not 0 <= page < n_pages:
            continue
        for h in range(heads):
            k_cache[page, h, c % page_size] = rotate(k[src, h], p, freq, interleaved)
            v_cache[page, h, c % page_size] = v[src, h]
    return q_out, k_cache, v_cache


def attend(q, k_cache, v_cache, pages, row_offsets, cache_lens, scale: float, tree=None, out=None):
    """(out [rows, heads, d], lse [rows, heads]): every row over the keys it sees.

    tree: [rows, drafts] truth values (row i sees its sequence's draft j), or None: drafts up to itself.  A key whose
    page is none is seen by no row.  Rows behind the last sequence keep what `out` holds (lse: NaN).
    """
    rows, heads, d = q.shape
    n_pages, kv_heads, page_size, _ = k_cache.shape
    group = heads // kv_heads
    out = np.zeros((rows, heads, d)) if out is None else np.array(out, np.float64)
    lse = np.full((rows, heads), np.nan)
    for s in range(len(row_offsets) - 1):
        r0, r1, length = int(row_offsets[s]), int(row_offsets[s + 1]), int(cache_lens[s])
        n = r1 - r0
        if n == 0:
            continue
        at = np.arange(length + n)
        entry = at // page_size
        page = np.where(entry < pages.shape[1], pages[s, np.minimum(entry, pages.shape[1] - 1)], -1)
        real = (page >= 0) & (page < n_pages)
        page = np.where(real, page, 0)
        for i in range(n):
            sees = real.copy()
            for j in range(n):
                sees[length + j] &= bool(tree[r0 + i, j]) if tree is not None else j <= i
            where = np.nonzero(sees)[0]
            for h in range(heads):
                kk = k_cache[page[where], h // group, where % page_size]
                vv = v_cache[page[where], h // group, where % page_size]
                if len(where) == 0:
                    out[r0 + i, h], lse[r0 + i, h] = 0.0, -np.inf
                    continue
                x = kk @ q[r0 + i, h] * scale
                top = x.max()
                w = np.exp(x - top)
                out[r0 + i, h] = (w / w.sum()) @ vv
                lse[r0 + i, h] = top + math.log(w.sum())
    return out, lse


def place(pages, s: int, c: int, n_pages: int, page_size: int):
    """(page, slot) of cache index c of sequence s, or None where that is no page."""
    entry = c // page_size
    if not 0 <= entry < pages.shape[1] or not 0 <= int(pages[s, entry]) < n_pages:
        return None
    return int(pages[s, entry]), c % page_size


def key_weights(q, lse, k_cache, pages, row_offsets, cache_lens, mass, scale: float, decay=1.0, tree=None,
                source_rows=None, key_positions=None, positions=None):
    """(mass, key_positions, terms): what the rows put on each key, added to decay * mass of the cached ones.

    tree: [rows, drafts] truth values or None, as in attend.  terms [like mass]: the sum of w (|x| + |lse| + d scale
    sum |q k|) over what was added, which an error in the scores is measured by.
    """
    mass, terms = np.array(mass, np.float64), np.zeros(np.shape(mass))
    key_positions = None if key_positions is None else np.array(key_positions)
    n_pages, kv_heads, page_size, d = k_cache.shape
    group = q.shape[1] // kv_heads
    for s in range(len(row_offsets) - 1):
        r0, r1, length = int(row_offsets[s]), int(row_offsets[s + 1]), max(0, int(cache_lens[s]))
        if r1 <= r0:
            continue
        for c in range(length + r1 - r0):
            at = place(pages, s, c, n_pages, page_size)
            if at is None:
                continue
            page, slot = at
            rows = [t for t in range(r0, r1) if c < length or (
                bool(tree[t, c - length]) if tree is not None else c - length <= t - r0)]
            source = [t if source_rows is None else int(source_rows[t]) for t in rows]
            source = [t for t in source if 0 <= t < q.shape[0]]
            for h in range(kv_heads):
                key, some = k_cache[page, h, slot], slice(h * group, (h + 1) * group)
                ls = lse[source, some]
                fine = np.isfinite(ls)
                x = np.where(fine, q[source, some] @ key * scale, 0.0)
                ls = np.where(fine, ls, 0.0)
                w = np.where(fine, np.exp(x - ls), 0.0)
                mass[page, h, slot] = w.sum() + (
                    decay * mass[page, h, slot] if c < length and decay != 0.0 else 0.0)
                far = np.where(fine, np.abs(q[source, some]) @ np.abs(key), 0.0)
                terms[page, h, slot] = (w * (np.abs(x) + np.abs(ls) + d * abs(scale) * far)).sum()
                if c >= length and key_positions is not None:
                    key_positions[page, h, slot] = c if positions is None else positions[r0 + c - length]
    return mass, key_positions, terms


def evict(k_cache, v_cache, mass, key_positions, pages, cache_lens, budgets, next_positions=None, sinks=0, recent=0,
          max_keys=None, mass_out=None, positions_out=None):
    """(k_cache, v_cache, mass, key_positions, new_lens) after the eviction, as new arrays; mass_out and positions_out:
    what a ledger that is not written in place holds before."""
    k, v = np.array(k_cache), np.array(v_cache)
    mass_to = np.array(mass if mass_out is None else mass_out)
    positions_to = None if key_positions is None else np.array(key_positions if positions_out is None else positions_out)
    n_pages, kv_heads, page_size, _ = k.shape
    room = pages.shape[1] * page_size
    most = room if max_keys is None else min(room, max_keys)
    new_lens = np.array(cache_lens)
    for s, n in enumerate(int(x) for x in cache_lens):
        where = [place(pages, s, c, n_pages, page_size) for c in range(max(0, min(n, room)))]
        stay = len(where)
        if 0 <= budgets[s] < n <= most and None not in where:
            stay = new_lens[s] = int(budgets[s])
        nxt = n if next_positions is None else int(next_positions[s])
        for h in range(kv_heads):
            def order(c):
                page, slot = where[c]
                m = float(mass[page, h, slot])
                p = c if key_positions is None else int(key_positions[page, h, slot])
                fixed = p < sinks or p >= nxt - recent
                return not fixed, math.isnan(m), 0.0 if math.isnan(m) else -m, c

            source = list(range(stay))
            if stay < len(where):
                kept = set(sorted(range(len(where)), key=order)[:stay])
                behind = iter(sorted(c for c in kept if c >= stay))
                source = [c if c in kept else next(behind) for c in range(stay)]
            for c, from_c in enumerate(source):
                if where[c] is None:
                    continue
                (page, slot), (fp, fs) = where[c], where[from_c]
                mass_to[page, h, slot] = mass[fp, h, fs]
                if positions_to is not None:
                    positions_to[page, h, slot] = key_positions[fp, h, fs]
                if c != from_c:
                    k[page, h, slot], v[page, h, slot] = k_cache[fp, h, fs], v_cache[fp, h, fs]
    return k, v, mass_to, positions_to, new_lens


def adjust(scores, probabilities=False, prompt=(), output=(), repetition=1.0, presence=0.0, frequency=0.0, bias=(),
           allowed=None):
    """One row's adjusted scores.  prompt, output: tokens (an output token as often as it is there); bias: (token, value)
    pairs, of which the last of a token counts; allowed: a truth value for each token, or None."""
    x = np.array(scores, np.float64)
    V = len(x)
    count, there = [0] * V, set()
    for v in output:
        if 0 <= v < V:
            count[v] += 1
            there.add(int(v))
    there |= {int(v) for v in prompt if 0 <= v < V}
    last = {int(v): float(b) for v, b in bias if 0 <= v < V}
    repetition = repetition if math.isfinite(repetition) and repetition > 0 else 1.0
    presence = presence if math.isfinite(presence) else 0.0
    frequency = frequency if math.isfinite(frequency) else 0.0
    with np.errstate(all="ignore"):
        for v in there | set(last):
            if probabilities and not x[v] > 0:
                continue
            y = np.log(x[v]) if probabilities else x[v]
            if v in there:
                y = y / repetition if y > 0 else y * repetition
            if count[v]:
                y = y - presence - frequency * count[v]
            if v in last:
                y = y + last[v]
            x[v] = np.exp(y) if probabilities else y
    if allowed is not None:
        x[~np.asarray(allowed, bool)] = 0.0 if probabilities else -np.inf
    return x


def sample(scores, uniform: float, probabilities: bool, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, its probability among the kept ones, how many are kept) of one row; (-1, 0, 0) if it holds none.

    scores: logits (present unless NaN or -inf), or probabilities (present if > 0).  If the largest is +inf only the
    +inf ones are present.  Weights (x / max)^(1 / T) or exp((x - max) / T); T <= 0: the first maximum.  Order: larger
    first, lower index first among equals.  The first top_k (0: all); of those the ones before which less than
    top_p of their weight lies; of those the ones of weight min_p and more.  The token is the first kept one, by index,
    at which the running weight exceeds uniform times their sum.
    """
    x = np.asarray(scores, np.float64)
    present = (x > 0) if probabilities else (~np.isnan(x) & (x > -np.inf))
    if np.any(present & (x == np.inf)):
        present &= x == np.inf
    index = np.nonzero(present)[0]
    if len(index) == 0:
        return -1, 0.0, 0
    y = x[index]
    order = index[np.argsort(-y, kind="stable")]
    first = x[order[0]]
    if not temperature > 0:
        return int(order[0]), 1.0, 1
    if first == np.inf:
        w = np.ones(len(x))
    elif probabilities:
        with np.errstate(divide="ignore", invalid="ignore"):
            w = np.exp(np.log(x / first) / temperature) if temperature != 1.0 else x / first
    else:
        with np.errstate(invalid="ignore"):
            w = np.exp((x - first) / temperature)
    n = len(order)
    if top_k > 0:
        n = min(n, int(top_k))
    if top_p < 1.0:
        running = np.cumsum(w[order[:n]])
        before = np.concatenate([[0.0], running[:-1]])
        n = max(1, int(np.sum(before < top_p * running[-1])))
    if min_p > 0.0:
        n = max(1, int(np.sum(w[order[:n]] >= min_p)))
    kept = np.sort(order[:n])
    running = np.cumsum(w[kept])
    u = min(max(uniform, 0.0), 1.0) if uniform == uniform else 0.0
    heavy = np.nonzero(w[kept] > 0)[0]
    i = min(int(np.sum(running <= u * running[-1])), int(heavy[-1]))
    return int(kept[i]), float(w[kept[i]] / running[-1]), n
