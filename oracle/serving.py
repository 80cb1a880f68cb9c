"""Decoding over a paged cache and prefill attention in fp64: plain definitions for tests.

Test infrastructure only.  Written from the formulas alone, in numpy, one sequence, head and row at a time
where that is clearest; shares nothing with the CUDA path.  Pages are arrays [num_pages][H_kv][page_size][d]; a
table entry outside [0, num_pages) is no page.
"""
from __future__ import annotations

import numpy as np


def rotate(x, weight, eps, table_rows, interleaved):
    """Norm and rotation of rows x [T][H][d]; table_rows [T][rot] (cosines, then sines) or None."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if table_rows is None:
        return y
    half = table_rows.shape[1] // 2
    out = y.copy()
    for i in range(half):
        c, s = table_rows[:, i, None], table_rows[:, half + i, None]
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        out[:, :, a] = y[:, :, a] * c - y[:, :, b] * s
        out[:, :, b] = y[:, :, b] * c + y[:, :, a] * s
    return out


def place(table_row, slot, page_size, num_pages):
    """(page, slot within it), or None where the slot has no page."""
    if slot < 0 or slot >= len(table_row) * page_size:
        return None
    page = int(table_row[slot // page_size])
    return (page, slot % page_size) if 0 <= page < num_pages else None


def append(k_pages, v_pages, weights, table, lens, cu, positions, max_positions, k, v):
    """Stores rotated keys and values k, v [T][H_kv][d] in place; lens count the new tokens already."""
    num_pages, _, page_size, _ = k_pages.shape
    for s in range(len(lens)):
        for t in range(int(cu[s]), int(cu[s + 1])):
            if not 0 <= positions[t] < max_positions:
                continue
            at = place(table[s], int(lens[s]) - (int(cu[s + 1]) - t), page_size, num_pages)
            if at is None:
                continue
            k_pages[at[0], :, at[1]] = k[t]
            v_pages[at[0], :, at[1]] = v[t]
            if weights is not None:
                weights[at[0], :, at[1]] = 0.0


def e4m3(x):
    """x rounded to the nearest e4m3 number, ties to even: steps of 2^(e - 3) from 2^e on, of 2^-9 below 2^-6; 448 at most."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.clip(np.floor(np.log2(np.abs(x))), -6, None)
    e = np.where(np.isfinite(e), e, -6)
    step = 2.0 ** (e - 3)
    return np.clip(np.round(x / step) * step, -448.0, 448.0)


def scale_of(y):
    """The factor of rows y [...][d] of a cache of 8 bits, before its own rounding."""
    return np.maximum(np.abs(y).max(axis=-1) / 448.0, 2.0 ** -126)


def paged_read(k_pages, v_pages, table, lens, first, cu, num_rows, fill):
    """Packed rows (k, v) [num_rows][H_kv][d] of pages that hold the values themselves; `fill` behind the last sequence."""
    num_pages, Hkv, page_size, d = k_pages.shape
    k, v = (np.full((num_rows, Hkv, d), float(fill)) for _ in range(2))
    for s in range(len(lens)):
        for t in range(int(cu[s]), min(int(cu[s + 1]), num_rows)):
            slot = int(first[s]) + t - int(cu[s])
            at = place(table[s], slot, page_size, num_pages) if slot < int(lens[s]) else None
            k[t] = 0.0 if at is None else k_pages[at[0], :, at[1]]
            v[t] = 0.0 if at is None else v_pages[at[0], :, at[1]]
    return k, v


def softmax(x):
    """Rows of x; (weights, ln of the sum).  A row of minus infinities has no weights."""
    m = np.max(x, axis=-1, keepdims=True, initial=-np.inf)
    e = np.exp(x - np.where(np.isneginf(m), 0.0, m))
    z = e.sum(axis=-1, keepdims=True)
    with np.errstate(divide="ignore"):
        return e / np.where(z == 0, 1.0, z), (np.where(np.isneginf(m), 0.0, m) + np.log(z))[..., 0]


def paged_decode(q, k_pages, v_pages, weights, table, lens, max_len, window, sinks, scale):
    """out [batch][H_q][d]; adds the attention weights to `weights` in place (None: not kept)."""
    num_pages, Hkv, page_size, d = k_pages.shape
    batch, Hq, _ = q.shape
    g = Hq // Hkv
    out = np.zeros((batch, Hq, d))
    for s in range(batch):
        n = min(max(int(lens[s]), 0), max_len)
        seen = [j for j in range(n) if not window or j >= n - window or j < sinks]
        at = [place(table[s], j, page_size, num_pages) for j in seen]
        at = [p for p in at if p is not None]
        if not at:
            continue
        pages, ofs = np.array(at).T
        for h in range(Hkv):
            k, v = k_pages[pages, h, ofs], v_pages[pages, h, ofs]
            p, _ = softmax(scale * (q[s, h * g:(h + 1) * g] @ k.T))
            out[s, h * g:(h + 1) * g] = p @ v
            if weights is not None:
                weights[pages, h, ofs] += p.sum(axis=0)
    return out


def shared_decode(q, k_pages, v_pages, weights, table, lens, max_len, prefix_table, prefix_lens, cu, max_prefix, scale,
                  pool=None):
    """paged_decode where sequences cu[r] .. cu[r + 1] - 1 see the slots of row r of prefix_table before their own; these are
    in the same pages, or in those of pool, (k, v)."""
    num_pages, Hkv, page_size, d = k_pages.shape
    pk, pv = (k_pages, v_pages) if pool is None else pool
    batch, Hq, _ = q.shape
    g = Hq // Hkv
    out = np.zeros((batch, Hq, d))
    for s in range(batch):
        group = [r for r in range(len(cu) - 1) if cu[r] <= s < cu[r + 1]]
        before = []
        if group:
            n = min(max(int(prefix_lens[group[0]]), 0), max_prefix)
            before = [place(prefix_table[group[0]], j, pk.shape[2], pk.shape[0]) for j in range(n)]
        own = [place(table[s], j, page_size, num_pages) for j in range(min(max(int(lens[s]), 0), max_len))]
        before, own = ([p for p in x if p is not None] for x in (before, own))
        if not before and not own:
            continue
        for h in range(Hkv):
            k = np.array([pk[p, h, o] for p, o in before] + [k_pages[p, h, o] for p, o in own])
            v = np.array([pv[p, h, o] for p, o in before] + [v_pages[p, h, o] for p, o in own])
            p, _ = softmax(scale * (q[s, h * g:(h + 1) * g] @ k.T))
            out[s, h * g:(h + 1) * g] = p @ v
            if weights is not None and own:
                pages, ofs = np.array(own).T
                weights[pages, h, ofs] += p.sum(axis=0)[len(before):]
    return out


def evict(k_pages, v_pages, weights, table, lens, new_table, max_len, budget, sinks, recent):
    """(new_lens, kept); moves the kept rows in place."""
    num_pages, Hkv, page_size, _ = k_pages.shape
    batch = len(lens)
    new_lens = np.zeros(batch, dtype=np.int32)
    kept = np.full((batch, Hkv, budget), -1, dtype=np.int32)
    for s in range(batch):
        n = min(max(int(lens[s]), 0), max_len)
        m = min(n, budget)
        new_lens[s] = m
        at = [place(table[s], j, page_size, num_pages) for j in range(n)]
        for h in range(Hkv):
            if n <= budget:
                keep = list(range(n))
            else:
                always = [j for j in range(n) if j < sinks or j >= n - recent]

                def rank(j):
                    w = -np.inf if at[j] is None else weights[at[j][0], h, at[j][1]]
                    return (-(-np.inf if np.isnan(w) else w), j)

                others = sorted((j for j in range(n) if sinks <= j < n - recent), key=rank)
                keep = sorted(always + others[:budget - len(always)])
            kept[s, h, :m] = keep
            for j, src in enumerate(keep):
                dst = place(new_table[s], j, page_size, num_pages)
                if at[src] is None or dst is None:
                    continue
                for x in (k_pages, v_pages, weights):
                    x[dst[0], h, dst[1]] = x[at[src][0], h, at[src][1]]
    return new_lens, kept


def prefill(q, k, v, cu_q, cu_k, window, sinks, scale):
    """(out [T_q][H_q][d], lse [T_q][H_q]) of packed sequences, row by row over the keys that it sees."""
    Tq, Hq, d = q.shape
    Hkv = k.shape[1]
    g = Hq // Hkv
    out, lse = np.zeros((Tq, Hq, d)), np.full((Tq, Hq), -np.inf)
    for s in range(len(cu_q) - 1):
        q0, q1, k0, k1 = int(cu_q[s]), int(cu_q[s + 1]), int(cu_k[s]), int(cu_k[s + 1])
        for i in range(q1 - q0):
            p = (k1 - k0) - (q1 - q0) + i
            seen = np.array([t for t in range(p + 1) if not window or t > p - window or t < sinks], dtype=int)
            if not len(seen):
                continue
            for h in range(Hkv):
                x = scale * (q[q0 + i, h * g:(h + 1) * g] @ k[k0 + seen, h].T)
                w, z = softmax(x)
                out[q0 + i, h * g:(h + 1) * g] = w @ v[k0 + seen, h]
                lse[q0 + i, h * g:(h + 1) * g] = z
    return out, lse
