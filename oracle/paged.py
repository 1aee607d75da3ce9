"""fp64 reference of the paged cache's calls -- TEST INFRASTRUCTURE ONLY, like the package.

Plain numpy, one unit (layer, sequence, KV head) at a time, from the definitions: the rows of a
sequence are looked up through its table one by one, attention is a softmax over the rows that a
query sees, and the eviction sorts.
"""
from __future__ import annotations

import numpy as np


def rows_of(pool, table_row, layer, h, js):
    """Rows js of one unit: [len(js), d] float64."""
    page = pool.shape[3]
    return np.array([pool[layer, table_row[j // page], h, j % page] for j in js], np.float64).reshape(len(js), -1)


def visible(n, window, sinks):
    """Indices of the rows a query sees among n."""
    return [j for j in range(n) if window == 0 or j < sinks or j >= n - window]


def decode(K, V, table, lens, q, kn, vn, scale, window=0, sinks=0, weights=None):
    """One token.  K and V (and weights, lens) are numpy arrays and are updated in place; kn and vn may
    be None.  Returns out, lse and, for error bounds, per query head the largest
    scale * sum_i |q_i k_ji|, the rows seen, and sum_j p_j |v_j| per output element."""
    Ly, B, Hq, d = q.shape
    H, page = K.shape[2], K.shape[3]
    G = Hq // H
    out, lse = np.zeros((Ly, B, Hq, d)), np.full((Ly, B, Hq), -np.inf)
    big, seen, absv = np.zeros((Ly, B, Hq)), np.zeros((Ly, B, Hq), int), np.zeros((Ly, B, Hq, d))
    for ly in range(Ly):
        for b in range(B):
            for h in range(H):
                n = int(lens[ly, b, h])
                if kn is not None:
                    K[ly, table[b, n // page], h, n % page] = kn[ly, b, h]
                    V[ly, table[b, n // page], h, n % page] = vn[ly, b, h]
                    if weights is not None:
                        weights[ly, b, h, n] = 0.0
                    n += 1
                    lens[ly, b, h] = n
                js = visible(n, window, sinks)
                if not js:
                    continue
                k, v = rows_of(K, table[b], ly, h, js), rows_of(V, table[b], ly, h, js)
                for g in range(G):
                    x = q[ly, b, h * G + g].astype(np.float64)
                    z = scale * (k @ x)
                    m = z.max()
                    e = np.exp(z - m)
                    p = e / e.sum()
                    i = (ly, b, h * G + g)
                    out[i], lse[i] = p @ v, m + np.log(e.sum())
                    big[i], seen[i], absv[i] = scale * (np.abs(k) @ np.abs(x)).max(), len(js), p @ np.abs(v)
                    if weights is not None:
                        weights[ly, b, h, js] += p / G
    return out, lse, big, seen, absv


def evict(K, V, weights, table, lens, budget, w, sinks):
    """Cuts K, V, weights and lens in place; returns the kept rows of every unit that was cut."""
    Ly, H, page = K.shape[0], K.shape[2], K.shape[3]
    kept = {}
    for ly in range(Ly):
        for b in range(len(budget)):
            for h in range(H):
                L, m = int(lens[ly, b, h]), int(budget[b])
                if L <= m:
                    continue
                between = range(sinks, L - w)
                best = sorted(between, key=lambda j: (-float(weights[ly, b, h, j]), j))[:m - sinks - w]
                rows = sorted(list(range(sinks)) + best + list(range(L - w, L)))
                for pool in (K, V):
                    moved = [pool[ly, table[b, j // page], h, j % page].copy() for j in rows]
                    for r, x in enumerate(moved):
                        pool[ly, table[b, r // page], h, r % page] = x
                weights[ly, b, h, :m] = weights[ly, b, h, rows]
                lens[ly, b, h] = m
                kept[ly, b, h] = np.array(rows)
    return kept


def rotate(x, pos, inv_freq, interleaved):
    """Rows x [..., d] turned by the position pos: pairs (i, i + rot / 2), or neighbours; float64."""
    x = np.array(x, np.float64)
    half = len(inv_freq)
    a = float(pos) * np.asarray(inv_freq, np.float64)
    c, s = np.cos(a), np.sin(a)
    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, v = x[..., lo].copy(), x[..., hi].copy()
    x[..., lo], x[..., hi] = u * c - v * s, v * c + u * s
    return x


def append(K, V, table, lens, k, v, starts, pos=None, inv_freq=(), interleaved=False, q=None, q_out=None):
    """New tokens' rows into K and V (and q_out), updated in place with lens; k, v, q are [layers, T, heads, d]."""
    Ly, H, page = K.shape[0], K.shape[2], K.shape[3]
    for b in range(len(starts) - 1):
        for t in range(starts[b], starts[b + 1]):
            s = 0 if pos is None else pos[t]
            for ly in range(Ly):
                if q is not None:
                    q_out[ly, t] = rotate(q[ly, t], s, inv_freq, interleaved)
                for h in range(H):
                    r = lens[ly, b, h] + t - starts[b]
                    K[ly, table[b, r // page], h, r % page] = rotate(k[ly, t, h], s, inv_freq, interleaved)
                    V[ly, table[b, r // page], h, r % page] = v[ly, t, h]
        lens[:, b] += starts[b + 1] - starts[b]


def prefix_lead(group):
    """The first sequence of each sequence's group (equal values next to each other)."""
    lead = list(range(len(group)))
    for b in range(1, len(group)):
        if group[b] == group[b - 1]:
            lead[b] = lead[b - 1]
    return lead


def prefix_decode(K, V, table, lens, q, kn, vn, scale, group, shared, skip=()):
    """One token of sequences that share prefixes: decode(), the rows below shared[b] looked up in the table of
    the group's first sequence.  Units in `skip` (layer, b, h) are left alone (zeros, -inf)."""
    Ly, B, Hq, d = q.shape
    H, page = K.shape[2], K.shape[3]
    G = Hq // H
    lead = prefix_lead(group)
    out, lse = np.zeros((Ly, B, Hq, d)), np.full((Ly, B, Hq), -np.inf)
    big, seen, absv = np.zeros((Ly, B, Hq)), np.zeros((Ly, B, Hq), int), np.zeros((Ly, B, Hq, d))
    for ly, b, h in np.ndindex(Ly, B, H):
        if (ly, b, h) in skip:
            continue
        n = int(lens[ly, b, h])
        if kn is not None:
            K[ly, table[b, n // page], h, n % page] = kn[ly, b, h]
            V[ly, table[b, n // page], h, n % page] = vn[ly, b, h]
            n += 1
            lens[ly, b, h] = n
        if n == 0:
            continue
        j = np.arange(n)
        ids = np.where(j < shared[b], table[lead[b], j // page], table[b, j // page])
        k, v = K[ly, ids, h, j % page].astype(np.float64), V[ly, ids, h, j % page].astype(np.float64)
        for g in range(G):
            i = (ly, b, h * G + g)
            z = scale * (k @ q[i].astype(np.float64))
            m = z.max()
            with np.errstate(invalid="ignore"):  # logits that are all -inf
                e = np.exp(z - m) if m > -np.inf or np.isnan(m) else np.zeros(n)
            if e.sum() == 0:
                continue
            p = e / e.sum()
            out[i], lse[i] = p @ v, m + np.log(e.sum())
            big[i], seen[i], absv[i] = abs(scale) * (np.abs(k) @ np.abs(q[i])).max(), n, p @ np.abs(v)
    return out, lse, big, seen, absv
