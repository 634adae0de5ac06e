"""Forking and compaction at the ends of their documented ranges."""

import numpy as np
import pytest
import torch

from paper_2608_08081_amd import api
from tests import serving as sv
from tests.test_gpu_pages import i32

pytestmark = pytest.mark.gpu


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
