"""Shared helpers of the tests of the serving operators: caches of random
records (codes of Gaussian coordinates, scales like the norms of keys), the
same on page pools, and the comparison with the oracle."""

from __future__ import annotations

import numpy as np
import torch

from oracle import codebook as ocb
from oracle import compress as ocz
from oracle import rotation as orot
from oracle import serving as osv

DEV = torch.device("cuda:0")
D = 128
NAMES = ("k_codes", "k_norms", "v_codes", "v_norms")


def levels(bits):
    return ocb.isoquant_codebook(D, bits)[0]


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def records(rng, shape, bits=3):
    """Random records [*shape][16 bits] and scales [*shape] of a cache's four
    arrays, as numpy."""
    thr = ocb.isoquant_codebook(D, bits)[1]
    out = []
    for _ in range(2):
        y = rng.standard_normal((*shape, D)) * D ** -0.5
        codes = np.searchsorted(thr, y, side="right").astype(np.uint8)
        out.append(ocz.pack(codes, bits))
        out.append((np.exp(0.35 * rng.standard_normal(shape)) * 14.0).astype(np.float32))
    return out


def rotation(rng_seed, hkv):
    return orot.make_quaternions(rng_seed, hkv)


def to_pool(rng, rows, lens, page, max_pages, extra=2):
    """The rows' arrays [B][H][cap][..] on a pool of `extra` pages too many, in
    no order: (pool arrays, tables); the unused slots and pages hold NaN
    scales."""
    used = [-(-int(n) // page) for n in lens]
    n_pages = sum(used) + extra
    order = list(rng.permutation(n_pages))
    tables = np.full((len(lens), max_pages), -1, np.int32)
    pool = []
    for a in rows:
        shape = (n_pages, a.shape[1], page) + a.shape[3:]
        pool.append(np.full(shape, np.nan if a.dtype == np.float32 else 255, a.dtype))
    for b, n in enumerate(lens):
        for k in range(used[b]):
            p = order.pop()
            tables[b, k] = p
            m = min(page, int(n) - k * page)
            for a, x in zip(pool, rows):
                a[p, :, :m] = x[b, :, k * page:k * page + m]
    return pool, tables


def as_dict(arrays):
    return {n: dev(a) for n, a in zip(NAMES, arrays)}


def check_rows(got, want, label):
    """Every row of got [..][128] within the bound of the oracle's (out, B, W)."""
    ref, big, mean = want
    got = got.cpu().numpy().astype(np.float64)
    assert np.all(np.isfinite(got)), f"{label}: not finite"
    err = np.linalg.norm(got - ref, axis=-1)
    tol = osv.error_bound(big, mean)
    worst = float((err / tol).max()) if err.size else 0.0
    print(f"[rows] {label}: worst error {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{label}: error {worst:.2f} times its bound"
    # all rows together: correct kernels of pairs and 32-bit sums are 2e-7 to 6e-7
    # off in the 2-norm (scores up to B of 16), two orders of the sums twice that;
    # an operand without its lo part is 1e-4 off
    if err.size and np.any(ref):
        rel = np.linalg.norm(err) / np.linalg.norm(ref)
        assert rel <= 4e-6 * max(1.0, big.max() / 16), f"{label}: {rel:.2e} off in all"
    none = mean == 0
    assert np.all(got[none] == 0), f"{label}: a row that sees nothing is not zero"
