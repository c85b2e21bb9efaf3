"""The serving operators in plain numpy, fp64: request by request, token by
token, from their definitions (include/streambeam.h)."""
from __future__ import annotations

import math

import numpy as np


def plan_pages(lens, add, free, table, page_size, token_cap):
    """free: the free list's n_free entries. Returns (lens, granted, free,
    table, slots, positions, q_start) after the step."""
    lens, free, table = list(lens), list(free), np.array(table)
    room = table.shape[1] * page_size
    for b, n in enumerate(add):
        if n < 0:
            free += [int(x) for x in table[b, :-(-lens[b] // page_size)]]
            lens[b] = 0
    granted, slots, positions, q_start, stopped, asked, wanted = [], [], [], [0], False, 0, 0
    n_free = len(free)
    for b, n in enumerate(add):
        n = n if n > 0 and lens[b] + n <= room else 0
        held = -(-lens[b] // page_size)
        need = -(-(lens[b] + n) // page_size) - held if n else 0
        asked, wanted = asked + n, wanted + need
        stopped = stopped or asked > token_cap or wanted > n_free
        if stopped:
            n = need = 0
        for c in range(held, held + need):
            table[b, c] = free.pop()
        for pos in range(lens[b], lens[b] + n):
            slots.append(int(table[b, pos // page_size]) * page_size + pos % page_size)
            positions.append(pos)
        lens[b] += n
        granted.append(n)
        q_start.append(q_start[-1] + n)
    pad = [-1] * (token_cap - len(slots))
    return lens, granted, free, table, slots + pad, positions + pad, q_start


def rotate(x, position, inv_freq, layout, mscale):
    """One head's row. Returns (rotated, |a| + |b| of every value's pair)."""
    x = np.asarray(x, np.float64)
    n = len(inv_freq)
    out, size = x.copy(), np.abs(x)
    for i, f in enumerate(inv_freq):
        a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = mscale * math.cos(position * f), mscale * math.sin(position * f)
        out[a], out[b] = x[a] * c - x[b] * s, x[a] * s + x[b] * c
        size[a] = size[b] = mscale * (abs(x[a]) + abs(x[b]))
    return out, size


def attention(q, k_cache, v_cache, table, lens, q_start, window, sinks, scale):
    """q [tokens, q_heads, D]; caches [pages, page_size, kv_heads, D]. Returns
    (out, sum of weights times |v|, largest sum of |q||k| of a score); rows of no
    request are NaN."""
    q, k_cache, v_cache = (np.asarray(t, np.float64) for t in (q, k_cache, v_cache))
    T, Hq, D = q.shape
    pages, page, Hkv, _ = k_cache.shape
    out, size, big = (np.full(q.shape, np.nan) for _ in range(3))
    for b, n in enumerate(lens):
        m = q_start[b + 1] - q_start[b]
        for t in range(q_start[b], q_start[b + 1]):
            p = n - m + t - q_start[b]
            out[t] = size[t] = big[t] = 0
            keys = [j for j in range(p + 1) if (window == 0 or j > p - window or j < sinks) and 0 <= table[b][j // page] < pages]
            if not keys:
                continue
            at = [(table[b][j // page], j % page) for j in keys]
            K, V = np.stack([k_cache[i] for i in at]), np.stack([v_cache[i] for i in at])   # [keys, Hkv, D]
            for h in range(Hq):
                hk = h // (Hq // Hkv)
                s = K[:, hk] @ q[t, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ V[:, hk]
                size[t, h] = w @ np.abs(V[:, hk])
                big[t, h] = np.max(np.abs(K[:, hk]) @ np.abs(q[t, h]))
    return out, size, big


def shared_attention(q, k_cache, v_cache, prefix_table, prefix_lens, group_start, table, lens, q_start, scale):
    """As attention, over the group's prefix and the request's own tokens."""
    q, k_cache, v_cache = (np.asarray(t, np.float64) for t in (q, k_cache, v_cache))
    T, Hq, D = q.shape
    pages, page, Hkv, _ = k_cache.shape
    out, size, big = (np.full(q.shape, np.nan) for _ in range(3))
    for b, n in enumerate(lens):
        m = q_start[b + 1] - q_start[b]
        ahead = []
        for g, length in enumerate(prefix_lens):
            if group_start[g] <= b < group_start[g + 1]:
                ahead = [(prefix_table[g][j // page], j % page) for j in range(length)]
        for t in range(q_start[b], q_start[b + 1]):
            p = n - m + t - q_start[b]
            out[t] = size[t] = big[t] = 0
            at = [i for i in ahead + [(table[b][j // page], j % page) for j in range(p + 1)] if 0 <= i[0] < pages]
            if not at:
                continue
            i, j = np.array(at).T
            K, V = k_cache[i, j], v_cache[i, j]   # [keys, Hkv, D]
            for h in range(Hq):
                hk = h // (Hq // Hkv)
                s = K[:, hk] @ q[t, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ V[:, hk]
                size[t, h] = w @ np.abs(V[:, hk])
                big[t, h] = np.max(np.abs(K[:, hk]) @ np.abs(q[t, h]))
    return out, size, big


def page_bounds(k_cache, table, lens, q_start, bounds):
    """bounds [pages, 2, kv_heads, D] after the step."""
    k_cache, bounds = np.asarray(k_cache, np.float64), np.array(bounds, np.float64)
    pages, page = k_cache.shape[:2]
    for b, n in enumerate(lens):
        m = q_start[b + 1] - q_start[b]
        for c in sorted({j // page for j in range(max(n - m, 0), n)}):
            at = table[b][c]
            if 0 <= at < pages:
                keys = k_cache[at, :min(page, n - c * page)]
                bounds[at, 0], bounds[at, 1] = keys.min(0), keys.max(0)   # (NaN where one is)
    return bounds


def select_pages(q, bounds, table, lens, q_start, page_size, top, first, last):
    """(pages [tokens, kv_heads, first + top + last], kept [tokens])."""
    q, bounds = np.asarray(q, np.float64), np.asarray(bounds, np.float64)
    T, Hq, D = q.shape
    n_pages, _, Hkv, _ = bounds.shape
    width = first + top + last
    pages, kept = np.full((T, Hkv, width), -1), np.full(T, -1)
    for b, n in enumerate(lens):
        m = q_start[b + 1] - q_start[b]
        for t in range(q_start[b], q_start[b + 1]):
            p = n - m + t - q_start[b]
            seen = p // page_size + 1 if p >= 0 else 0
            kept[t] = max(p + 1, 0) if seen <= width else (width - 1) * page_size + p % page_size + 1
            for h in range(Hkv):
                cols = list(range(seen))
                if seen > width:
                    mine = q[t, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)]
                    up, down = np.where(mine < 0, 0, mine).sum(0), np.where(mine > 0, 0, mine).sum(0)   # (NaN stays)
                    score = {}
                    for c in range(first, seen - last):
                        at = table[b][c]
                        if not 0 <= at < n_pages:
                            score[c] = (-1, 0.0)
                            continue
                        with np.errstate(invalid="ignore"):
                            s = float(np.sum(bounds[at, 1, h] * up + bounds[at, 0, h] * down))
                        score[c] = (1, 0.0) if math.isnan(s) else (0, s)
                    best = sorted(score, key=lambda c: (score[c][0], score[c][1]), reverse=True)   # (stable: of equal ones the first)
                    cols = sorted(cols[:first] + best[:top] + cols[seen - last:])
                pages[t, h, :len(cols)] = [table[b][c] for c in cols]
    return pages, kept


def selected_attention(q, k_cache, v_cache, pages, kept, scale):
    """As attention, over the first kept[t] keys of pages[t][h]; rows with kept
    below 0 are NaN."""
    q, k_cache, v_cache = (np.asarray(t, np.float64) for t in (q, k_cache, v_cache))
    T, Hq, D = q.shape
    n_pages, page, Hkv, _ = k_cache.shape
    out, size, big = (np.full(q.shape, np.nan) for _ in range(3))
    for t in range(T):
        if kept[t] < 0:
            continue
        out[t] = size[t] = big[t] = 0
        for hk in range(Hkv):
            n = min(kept[t], page * len(pages[t][hk]))
            at = [(pages[t][hk][j // page], j % page) for j in range(n) if 0 <= pages[t][hk][j // page] < n_pages]
            if not at:
                continue
            i, j = np.array(at).T
            K, V = k_cache[i, j, hk], v_cache[i, j, hk]
            for h in range(hk * (Hq // Hkv), (hk + 1) * (Hq // Hkv)):
                s = K @ q[t, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h], size[t, h], big[t, h] = w @ V, w @ np.abs(V), np.max(np.abs(K) @ np.abs(q[t, h]))
    return out, size, big


def sample(z, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob) of one row."""
    z = np.asarray(z, np.float64).copy()
    z[np.isnan(z)] = -np.inf
    order = np.argsort(-z, kind="stable")
    top = z[order[0]]
    if top == -np.inf:
        return -1, -math.inf
    if not T > 0:
        return int(order[0]), 0.0
    x = np.where(z == top, 0.0, z - (top if np.isfinite(top) else 0.0))
    x[(z != top) & (~np.isfinite(z) | (top == np.inf))] = -np.inf
    w = np.zeros(len(z), dtype=object)
    for i in np.flatnonzero(x > -np.inf):
        e = x[i] / T * math.log2(math.e) if T < np.inf else 0.0
        w[i] = int(np.rint(2.0 ** (e + 44))) if e > -64 else 0
    kept = list(order[:top_k] if 0 < top_k < len(z) else order)
    if top_p < 1:
        limit, before, prefix = float(top_p) * float(sum(w[i] for i in kept)), 0, []
        for i in kept:
            if prefix and not before < limit:
                break
            prefix.append(i)
            before += w[i]
        kept = prefix
    if min_p > 0:
        kept = [i for i in kept if w[i] >= min(min_p, 1.0) * 2.0 ** 44]
    kept = sorted(i for i in kept if w[i] > 0)
    total = sum(w[i] for i in kept)
    u = 0.0 if not u > 0 else min(u, 1.0)
    mass = 0
    for i in kept:
        mass += w[i]
        if mass > float(u) * float(total):
            break
    return int(i), float(x[i] / T - math.log(total / 2.0 ** 44)) if x[i] < 0 else -math.log(total / 2.0 ** 44)


def quantize_rows(x):
    """(codes [rows, cols rounded up to 16], scales [rows]) of fp64 rows that
    hold values of at most 24 bits: their quotients with an fp32 scale are no
    nearer to a border than 2^-33 unless they are on it, and fp64 tells them apart."""
    x = np.asarray(x, np.float64)
    codes, scales = np.zeros((x.shape[0], -(-x.shape[1] // 16) * 16), np.int64), np.zeros(x.shape[0], np.float32)
    for r, row in enumerate(x):
        if not np.all(np.isfinite(row)):
            scales[r] = np.nan
            continue
        scales[r] = np.float32(np.max(np.abs(row)) / 127)
        if scales[r] > 0:
            codes[r, :len(row)] = np.clip(np.rint(row / np.float64(scales[r])), -127, 127)
    return codes, scales


def linear(x, x_scale, w, w_scale, bias=None):
    """(out, the size of the product alone) in fp64; the sums as whole numbers."""
    sums = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T   # (below 2^53: exact)
    out = sums * np.asarray(x_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)
    return out + (0 if bias is None else np.asarray(bias, np.float64)), np.abs(out)
