"""Forking and compaction at the ends of their documented ranges."""

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2608_08081_amd import api
from tests import serving as sv
from tests.test_gpu_pages import check_fork, i32, same, state

pytestmark = pytest.mark.gpu


def bytes_pool(rng, n_pages, page):
    """Pools of any bytes (what moves is not looked at)."""
    return [rng.integers(0, 256, (n_pages, 1, page, 48), dtype=np.uint8),
            rng.random((n_pages, 1, page), dtype=np.float32),
            rng.integers(0, 256, (n_pages, 1, page, 48), dtype=np.uint8),
            rng.random((n_pages, 1, page), dtype=np.float32)]


def test_fork_asks_for_more_than_32_bits_of_pages():
    """65535 rows that each reserve 33000 pages: 2.2e9 pages asked for, of which
    the pool has 64.  (Tables of 8.7 GB; what is expected of them is written down
    here: the first row keeps its parent's page and takes the free ones, every
    other row has nothing.)"""
    page, rows, width, n_pages = 16, 65535, 33000, 64
    free_bytes, _ = torch.cuda.mem_get_info()
    if free_bytes < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    rng = np.random.default_rng(41)
    pool = sv.as_dict(sv.records(rng, (n_pages, 1, page)))
    before = {n: a.clone() for n, a in pool.items()}
    tables = torch.full((1, width), -1, dtype=torch.int32, device=sv.DEV)
    tables[0, 0] = 7
    refs = torch.zeros(n_pages, dtype=torch.int32, device=sv.DEV)
    refs[7] = 1
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    out_tables = torch.empty((rows, width), dtype=torch.int32, device=sv.DEV)
    print("[fork] 65535 rows of 33000 pages", flush=True)
    t, lens, refs = api.iq_fork_pages(
        pool, tables, i32([5]), torch.zeros(rows, dtype=torch.int32, device=sv.DEV), refs,
        out_tables=out_tables, reserve=width * page, status=status)
    torch.cuda.synchronize()
    others = [p for p in range(n_pages) if p != 7]
    assert t[0, :n_pages].tolist() == [7] + others
    assert int(t[0, n_pages:].max()) == -1 and int(t[0, n_pages:].min()) == -1
    for r0 in range(1, rows, 8192):
        block = t[r0:r0 + 8192]
        assert int(block.max()) == -1 and int(block.min()) == -1
    assert lens[0].item() == 5 and int(lens[1:].max()) == 0 and int(lens[1:].min()) == 0
    assert refs.tolist() == [1] * n_pages and status.item() == 5
    for n, a in pool.items():
        assert torch.equal(a, before[n])


def test_fork_many_pages():
    """Free pages are found past 64 chunks of 2048 (131072 pages), the first of
    them far behind and in words of few."""
    rng = np.random.default_rng(42)
    page, n_pages = 16, 140000
    lens = [int(n) for n in rng.integers(0, 60, 40)]
    _, tables, refs = state(rng, lens, page, 12, 0, n_pages)
    pool = bytes_pool(rng, n_pages, page)
    refs[:139000] = np.maximum(refs[:139000], 1)     # held by somebody else
    refs[rng.integers(0, 139000, 60)] = 0
    tables[refs[np.maximum(tables, 0)] == 0] = -1    # (a page that was freed is nobody's)
    parents = rng.integers(-1, 40, 64)
    want = check_fork(rng, pool, tables, lens, parents, refs, page, reserve=100)
    assert want[0].max() > 131072 and want[3] == 0


@pytest.mark.parametrize("share", [0.2, 0.8])
def test_compact_many_pages(share):
    """More chunks than a wave has lanes, movers and takers in many of them."""
    rng = np.random.default_rng([43, int(10 * share)])
    n_pages, page = 140000, 16
    refs = ((rng.random(n_pages) < share) * rng.integers(1, 4, n_pages)).astype(np.int32)
    tables = rng.choice(np.flatnonzero(refs > 0), (50, 40)).astype(np.int32)
    pool = bytes_pool(rng, n_pages, page)
    got, t, r = sv.as_dict(pool), i32(tables), i32(refs)
    print(f"[compact] 140000 pages, {share} of them live", flush=True)
    ot, orefs, page_map, n_live = api.iq_compact_pages(got, t, r)
    want = osv.compact(pool, tables, refs)
    same(ot, want[0], "tables")
    same(orefs, want[1].astype(np.int32), "counts")
    same(page_map, want[2], "map")
    assert n_live.item() == want[3]
    for x, name in zip(pool, sv.NAMES):
        same(got[name], x, name)
