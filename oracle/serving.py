"""Serving operators around the packed cache: attention behind a sliding
window with sinks, attention of trees of drafted tokens, acceptance of a path
of a tree, forking and compaction of page pools.  Plain loops in fp64 (and
whole numbers); test infrastructure only.

Attention is App. A on the visible positions (see oracle.attention): with y =
R_g q_h, x_j = scale s^K_j (y . C[codeK_j]) and alpha = softmax over the
visible j, o = R_g^T sum_j alpha_j s^V_j C[codeV_j]; nothing visible gives 0.
"""

from __future__ import annotations

import numpy as np

from . import compress as _cz
from . import rotation as _rot


def _attend(y, k, v, see, scale):
    """y [R][d] rotated queries, k / v [n][d] rotated records, see [R][n]:
    (o [R][d] rotated, B [R], W [R]) with B the largest sum of |products| of a
    visible score and W the weighted mean of the visible values' norms, which
    bound rounding errors (see error_bound)."""
    out = np.zeros_like(y)
    big, mean = np.zeros(len(y)), np.zeros(len(y))
    for r in range(len(y)):
        j = np.flatnonzero(see[r])
        if j.size == 0:
            continue
        x = (k[j] @ y[r]) * scale
        e = np.exp(x - x.max())
        a = e / e.sum()
        out[r] = a @ v[j]
        big[r] = (np.abs(k[j]) @ np.abs(y[r])).max() * scale
        mean[r] = a @ np.linalg.norm(v[j], axis=-1)
    return out, big, mean


def error_bound(big, mean):
    """2-norm by which a row computed in fp32 from (hi, lo) fp16 pairs may be
    off: a score of 128 products has an error of sqrt(128) roundings of 2^-24 of
    its partial sums (at most B), four times that (2.7e-6 B) holding for every
    score of a test; operands are pairs of 22 bits and weights, sums and the
    rotation are rounded a few times more (1e-6 in all).  A relative error d of
    the weights moves the mean of values by at most 2 d times the mean of their
    norms."""
    return 2.0 * (2.7e-6 * np.asarray(big) + 1e-6) * np.asarray(mean) + 1e-30


def window_visible(length, window, n_sinks):
    """Which positions 0 .. length - 1 the query of the last one sees."""
    j = np.arange(length)
    return (j >= length - window) | (j < n_sinks)


def decode_window(q, k_rec, k_norms, v_rec, v_norms, seq_lens, quats, levels, window, n_sinks,
                  scale=None):
    """q [B][H_q][d], caches as for oracle.attention.decode_fused; (out, B, W)
    per query head."""
    q = np.asarray(q, np.float64)
    b_, hq, d = q.shape
    hkv = k_rec.shape[1]
    group, bits = hq // hkv, _cz.bits_of(levels)
    rots = _rot.rotation_matrices(np.asarray(quats))
    scale = d ** -0.5 if not scale or scale <= 0 else scale
    out, big, mean = np.zeros_like(q), np.zeros((b_, hq)), np.zeros((b_, hq))
    for b in range(b_):
        n = int(seq_lens[b])
        see = window_visible(n, window, n_sinks)
        j = np.flatnonzero(see)
        for g in range(hkv):
            hs = slice(g * group, (g + 1) * group)
            k = _cz.dequantize_rotated(_cz.unpack(k_rec[b, g, j], d, bits), k_norms[b, g, j],
                                       levels)
            v = _cz.dequantize_rotated(_cz.unpack(v_rec[b, g, j], d, bits), v_norms[b, g, j],
                                       levels)
            o, big[b, hs], mean[b, hs] = _attend(q[b, hs] @ rots[g].T, k, v,
                                                 np.ones((group, len(j)), bool), scale)
            out[b, hs] = o @ rots[g]
    return out, big, mean


def tree_visible(words, length, window, n_sinks):
    """(cached [T][length], nodes [T][T]) booleans of what each node sees."""
    t_ = len(words)
    full = (1 << t_) - 1
    words = [int(w) & ((1 << 64) - 1) & full for w in words]
    pos = [length + bin(w & ~(1 << t)).count("1") for t, w in enumerate(words)]
    cached, nodes = np.zeros((t_, length), bool), np.zeros((t_, t_), bool)
    j = np.arange(length)
    for t, w in enumerate(words):
        if w == 0:
            continue
        cached[t] = True if window == 0 else (j > pos[t] - window) | (j < n_sinks)
        for u in range(t_):
            nodes[t, u] = bool(w >> u & 1) and (window == 0 or pos[u] > pos[t] - window or
                                                pos[u] < n_sinks)
    return cached, nodes


def decode_tree(q, k_rec, k_norms, v_rec, v_norms, seq_lens, dk_rec, dk_norms, dv_rec, dv_norms,
                words, quats, levels, window=0, n_sinks=0, scale=None):
    """q [B][T][H_q][d], words [B][T] (integers), drafts' records [B][H_kv][>=
    T][..]; (out, B, W) per node and query head."""
    q = np.asarray(q, np.float64)
    b_, t_, hq, d = q.shape
    hkv = k_rec.shape[1]
    group, bits = hq // hkv, _cz.bits_of(levels)
    rots = _rot.rotation_matrices(np.asarray(quats))
    scale = d ** -0.5 if not scale or scale <= 0 else scale
    out, big, mean = np.zeros_like(q), np.zeros((b_, t_, hq)), np.zeros((b_, t_, hq))
    for b in range(b_):
        n = int(seq_lens[b])
        cached, nodes = tree_visible(words[b], n, window, n_sinks)
        see = np.concatenate((cached, nodes), 1)
        used = see.any(0)                       # a record that nobody sees is not looked at
        jc, jd = np.flatnonzero(used[:n]), np.flatnonzero(used[n:])
        see = np.repeat(see[:, used], group, axis=0)
        for g in range(hkv):
            hs = slice(g * group, (g + 1) * group)

            def side(rec, nrm, drec, dnrm):
                r = np.concatenate((rec[b, g, jc], drec[b, g, jd]))
                s = np.concatenate((nrm[b, g, jc], dnrm[b, g, jd]))
                return _cz.dequantize_rotated(_cz.unpack(r, d, bits), s, levels)

            y = q[b, :, hs].reshape(-1, d) @ rots[g].T
            o, bb, mm = _attend(y, side(k_rec, k_norms, dk_rec, dk_norms),
                                side(v_rec, v_norms, dv_rec, dv_norms), see, scale)
            out[b, :, hs] = (o @ rots[g]).reshape(t_, group, d)
            big[b, :, hs], mean[b, :, hs] = bb.reshape(t_, group), mm.reshape(t_, group)
    return out, big, mean


def accept(draft, path, n_accept, cache, seq_lens, tables=None):
    """draft / cache: lists of arrays [..][H][positions][..]; copies in place,
    returns (lengths, status)."""
    lens, status = np.array(seq_lens), 0
    dcap, page = draft[0].shape[2], cache[0].shape[2]
    cap = page if tables is None else tables.shape[1] * page
    for b in range(len(lens)):
        n, at = int(n_accept[b]), int(lens[b])
        if n < 0 or n > path.shape[1] or at < 0:
            status |= 1
            continue
        if at + n > cap:
            status |= 5
            continue
        nodes = [int(x) for x in path[b, :n]]
        bad = any(x < 0 or x >= dcap for x in nodes)
        lost = False
        if tables is not None:
            pages = [int(tables[b, (at + i) // page]) for i in range(n)]
            lost = any(p < 0 or p >= cache[0].shape[0] for p in pages)
        if bad or lost:
            status |= (1 if bad else 0) | (5 if lost else 0)
            continue
        for i, node in enumerate(nodes):
            for src, dst in zip(draft, cache):
                if tables is None:
                    dst[b, :, at + i] = src[b, :, node]
                else:
                    dst[pages[i], :, (at + i) % page] = src[b, :, node]
        lens[b] = at + n
    return lens, status


def fork(pool, tables, seq_lens, parents, refs, page, reserve=0):
    """(tables, lengths, refs, status); the copies are made in `pool` (arrays
    [pages][H][page][..]) in place."""
    n_pages, width = len(refs), tables.shape[1]
    there = lambda p: 0 <= p < n_pages  # noqa: E731
    refs0, refs = np.array(refs), np.array(refs)
    for p in tables.ravel():
        if there(p):
            refs[p] -= 1
    new = np.full((len(parents), width), -1, np.int32)
    lens, status = np.zeros(len(parents), np.int32), 0
    fresh, sources, seen = [], {}, set()
    for i, par in enumerate(parents):
        if par >= len(tables):
            status |= 1
        if par < 0 or par >= len(tables):
            continue
        n = min(max(int(seq_lens[par]), 0), width * page)
        lens[i] = n
        full, need = n // page, -(-min(n + reserve, width * page) // page)
        for k in range(need):
            p = int(tables[par, k])
            if k < full:
                new[i, k] = p if there(p) else -1
            elif par not in seen and there(p) and refs0[p] == 1:
                new[i, k] = p
            else:
                fresh.append((i, k))
                if k == full and n % page and there(p):
                    sources[i, k] = p
            if new[i, k] >= 0:
                refs[new[i, k]] += 1
        seen.add(par)
    busy = refs.copy()
    for p in sources.values():
        busy[p] += 1
    free = [int(p) for p in np.flatnonzero(busy <= 0)]
    for (i, k), p in zip(fresh, free + [-1] * len(fresh)):
        new[i, k] = p
        full = lens[i] // page
        if p < 0:
            status |= 5
            if k == full:
                lens[i] = full * page
            continue
        refs[p] = 1
        if (i, k) in sources:
            n = lens[i] % page
            for a in pool:
                a[p, :, :n] = a[sources[i, k], :, :n]
    return new, lens, refs, status


def compact(pool, tables, refs):
    """(tables, refs, map, n_live); pages are moved in `pool` in place."""
    refs = np.array(refs)
    live = refs > 0
    n = int(live.sum())
    p = np.arange(len(refs))
    movers, takers = p[live & (p >= n)], p[~live & (p < n)]
    page_map = np.where(live, p, -1).astype(np.int32)
    page_map[movers] = takers
    out = refs.copy()
    out[takers] = refs[movers]
    out[movers] = 0
    t = np.array(tables)
    inside = (t >= 0) & (t < len(refs))
    t[inside] = page_map[t[inside]]
    for a in pool:
        a[takers] = a[movers]
    return t, out, page_map, n
