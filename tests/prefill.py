"""Shared helpers of the tests of prompts in chunks: plain implementations in 64 bits of page
assignment, rotary positions and causal attention of many sequences, and their tolerances."""

from __future__ import annotations

import numpy as np
import torch

from oracle import compress as ocz
from oracle import rotation as orot
from tests import serving as sv

D = 128


def extend(tables, lens, new, refs, page, n_tokens):
    """What iq_extend_pages returns, sequence by sequence: (row_starts, slots, positions, tables,
    lens, refs, status)."""
    tables, lens, refs = tables.copy(), lens.copy(), refs.copy()
    b, width = tables.shape
    n_pages = len(refs)
    free = [p for p in range(n_pages) if refs[p] <= 0]
    slots = np.full(n_tokens, -1, np.int64)
    positions = np.zeros(n_tokens, np.int32)
    starts, status, asked, taken = [0], 0, 0, 0
    total = 0
    for i in range(b):
        length, n = int(lens[i]), int(new[i])
        sane = length >= 0 and n >= 0
        n = max(n, 0)
        end = total + n
        room = n == 0 or length + n <= width * page
        ks = []
        if sane and room and n:
            ks = [k for k in range(length // page, -(-(length + n) // page))
                  if not 0 <= tables[i, k] < n_pages]
        asked += len(ks)
        served = not ks or asked <= len(free)
        held = end <= n_tokens
        if not sane or not held:
            status |= 1
        if sane and (not room or not served):
            status |= 5
        fits = sane and room and held and served
        if fits:
            for k in ks:
                tables[i, k] = free[taken]
                refs[free[taken]] = 1
                taken += 1
            lens[i] = length + n
        for j in range(n):
            t = total + j
            if t < n_tokens:
                positions[t] = length + j
                if fits:
                    p = length + j
                    slots[t] = int(tables[i, p // page]) * page + p % page
        total = end
        starts.append(min(total, n_tokens))
    return np.array(starts, np.int32), slots, positions, tables, lens, refs, status


def rope(x, positions, freqs, layout, amplitude=1.0):
    """Rotary positions of x [n][heads][dim] in 64 bits."""
    x = np.asarray(x, np.float64).copy()
    m = 2 * len(freqs)
    angle = positions.astype(np.float64)[:, None] * np.asarray(freqs)[None]
    c, s = amplitude * np.cos(angle)[:, None], amplitude * np.sin(angle)[:, None]
    if layout == "half":
        i, j = np.arange(m // 2), np.arange(m // 2) + m // 2
    else:
        i, j = np.arange(0, m, 2), np.arange(1, m, 2)
    a, b = x[..., i].copy(), x[..., j].copy()
    x[..., i], x[..., j] = a * c - b * s, a * s + b * c
    return x


def attention(q, rows, starts, lens, quats, hkv, window=0, sinks=0, scale=D ** -0.5):
    """Attention of tokens q [n][Hq][128] over records rows = (k_codes, k_norms, v_codes,
    v_norms), [B][H][cap][..], in the original space and 64 bits: (outputs, for every row the
    largest |q| |k| scale of its seen positions and the weighted mean of |v|)."""
    n, hq, _ = q.shape
    group = hq // hkv
    lv = sv.levels(3).astype(np.float64)
    rots = orot.rotation_matrices(quats)
    out = np.zeros((n, hq, D))
    big, mean = np.zeros((n, hq)), np.zeros((n, hq))
    for b in range(len(lens)):
        s, e, length = int(starts[b]), int(starts[b + 1]), int(lens[b])
        for g in range(hkv):
            k = lv[ocz.unpack(rows[0][b, g, :length])] * rows[1][b, g, :length, None].astype(
                np.float64)
            v = lv[ocz.unpack(rows[2][b, g, :length])] * rows[3][b, g, :length, None].astype(
                np.float64)
            k, v = k @ rots[g], v @ rots[g]
            kn, vn = np.linalg.norm(k, axis=1), np.linalg.norm(v, axis=1)
            for t in range(s, e):
                p = length - (e - s) + (t - s)
                if p < 0:
                    continue
                j = np.arange(p + 1)
                if window:
                    j = j[(j > p - window) | (j < sinks)]
                for h in range(g * group, (g + 1) * group):
                    x = np.asarray(q[t, h], np.float64)
                    a = k[j] @ x * scale
                    w = np.exp(a - a.max())
                    w /= w.sum()
                    out[t, h] = w @ v[j]
                    big[t, h] = np.linalg.norm(x) * kn[j].max() * scale
                    mean[t, h] = w @ vn[j]
    return out, big, mean


def check_attention(got, want, dtype, label):
    """Every output row within its bound.

    fp32: that of the other operators with pairs of parts (serving.check_rows).
    fp16: with u = 2^-11 (half a step of fp16, relative), a rotated query's entries are off by u
    each, so a score by at most u sum |q_i| |k_i| scale <= u B, B the largest |q| |k| scale; a
    weight by a relative 2 u B (its own score's and its sum's), its product with the value scale
    by u more, values are exact.  The output is off by at most (2 u B + u) W, W the weighted mean
    of |v|, in the 2-norm, and by u |out| at its own rounding, |out| <= W: u (2 B + 2) W in all,
    to the first order; 1.01 for the others, and for the 32-bit sums.  Entries below 2^-14 are
    rounded by 2^-25 instead: 2^-25 128^(1/2) more.
    In all (the 2-norm over every row) errors of random sign stay far below: the query's add up to
    u B / 128^(1/2) of a score, in which |k| and |q| of random directions make B about 11 times a
    score's spread; 8e-4 of the outputs, against 2.1e-4 (0.29 of a step's half at random) for the
    last rounding alone."""
    ref, big, mean = want
    if dtype == torch.float32:
        return sv.check_rows(got, want, label)
    got = got.cpu().numpy().astype(np.float64)
    assert np.all(np.isfinite(got)), f"{label}: not finite"
    u = 2.0 ** -11
    err = np.linalg.norm(got - ref, axis=-1)
    tol = 1.01 * u * (2 * big + 2) * mean + 2.0 ** -25 * D ** 0.5
    worst = float((err / tol).max()) if err.size else 0.0
    print(f"[rows] {label}: worst error {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{label}: error {worst:.2f} times its bound"
    if err.size and np.any(ref):
        rel = np.linalg.norm(err) / np.linalg.norm(ref)
        print(f"[rows] {label}: {rel:.2e} off in all", flush=True)
        assert rel <= 8e-4 * max(1.0, big.max() / 32), f"{label}: {rel:.2e} off in all"
    assert np.all(got[mean == 0] == 0), f"{label}: a row that sees nothing is not zero"
