"""Records moved between caches: acceptance, forking and compaction, against
the oracle's whole numbers, bit for bit."""

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2608_08081_amd import api
from tests import serving as sv

pytestmark = pytest.mark.gpu


def same(got, want, label):
    got = got.cpu().numpy() if hasattr(got, "cpu") else np.asarray(got)
    want = np.asarray(want)
    assert got.shape == want.shape and got.dtype == want.dtype, label
    assert np.array_equal(got.view(np.uint8), want.view(np.uint8)), label


def i32(x):
    return sv.dev(np.asarray(x, np.int32))


# ---------------------------------------------------------------- acceptance

@pytest.mark.parametrize("bits", [3, 2, 4])
@pytest.mark.parametrize("in_place", [False, True])
def test_accept_on_rows(bits, in_place):
    rng = np.random.default_rng(bits)
    b, hkv, cap, t = 9, 3, 70, 12
    draft, cache = sv.records(rng, (b, hkv, t + 1), bits), sv.records(rng, (b, hkv, cap), bits)
    # sequence: none, all, one, does not fit, exactly fits, bad node, bad count, twice the same
    lens = np.asarray([0, 10, 69, 69, 64, 5, 6, 7, -3], np.int32)
    count = np.asarray([0, 12, 1, 2, 6, 3, 13, 4, 1], np.int32)
    path = np.asarray([rng.permutation(t) for _ in range(b)], np.int32)
    path[5, 2] = t + 1
    path[7, :4] = [3, 3, 0, 3]
    path[1, 0] = t                     # the draft cache's last record
    path[0] = -7                       # not read
    got, seq = [sv.dev(a) for a in cache], i32(lens)
    out = seq if in_place else torch.full((b,), 77, dtype=torch.int32, device=sv.DEV)
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    print(f"[accept] rows bits={bits}", flush=True)
    ret = api.iq_accept_tree(sv.as_dict(draft), i32(path), i32(count), *got, seq,
                             None if in_place else out, status, bits=bits)
    assert ret is out
    want_lens, want_status = osv.accept(draft, path, count, cache, lens)
    same(out, want_lens, "lengths")
    assert status.item() == want_status == 5
    for a, x, n in zip(got, cache, sv.NAMES):
        same(a, x, n)


@pytest.mark.parametrize("page", [16, 32])
def test_accept_on_pools(page):
    rng = np.random.default_rng(page)
    b, hkv, t = 7, 2, 64
    lens = [0, 15, 16, 100, 120, 31, 64]
    cap = 128
    rows = sv.records(rng, (b, hkv, cap))
    # room for the accepted tokens except in sequence 5
    pool, tables = sv.to_pool(rng, rows, [cap if i != 5 else n for i, n in enumerate(lens)], page,
                              cap // page)
    draft = sv.records(rng, (b, hkv, t))
    count = np.asarray([64, 1, 16, 28, 9, 2, 0], np.int32)
    path = np.asarray([rng.permutation(t) for _ in range(b)], np.int32)
    got, seq = sv.as_dict(pool), i32(lens)
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    print(f"[accept] pool page={page}", flush=True)
    out = api.iq_accept_tree_paged(sv.as_dict(draft), i32(path), i32(count), got, i32(tables), seq,
                                   status=status)
    want_lens, want_status = osv.accept(draft, path, count, pool, lens, tables)
    assert out is seq
    same(seq, want_lens.astype(np.int32), "lengths")
    assert status.item() == want_status == 5
    for x, n in zip(pool, sv.NAMES):
        same(got[n], x, n)


def test_accept_of_nothing():
    """Paths of no node: the lengths and records stay; a count that names one is
    refused."""
    rng = np.random.default_rng(8)
    draft, cache = sv.records(rng, (2, 1, 3)), sv.records(rng, (2, 1, 16))
    got, seq = [sv.dev(a) for a in cache], i32([4, 16])
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    print("[accept] nothing", flush=True)
    path = torch.empty((2, 0), dtype=torch.int32, device=sv.DEV)
    api.iq_accept_tree(sv.as_dict(draft), path, i32([0, 0]), *got, seq, None, status)
    assert seq.tolist() == [4, 16] and status.item() == 0
    api.iq_accept_tree(sv.as_dict(draft), path, i32([0, 1]), *got, seq, None, status)
    assert seq.tolist() == [4, 16] and status.item() == 1
    for a, x in zip(got, cache):
        same(a, x, "records")


# ------------------------------------------------------------------- forking

def state(rng, lens, page, width, hkv, n_pages, prompt=0):
    """Sequences of given lengths on a pool, with `prompt` leading pages shared
    by all of them: (pool, tables, refs)."""
    order = list(rng.permutation(n_pages))
    shared = [order.pop() for _ in range(prompt)]
    tables, refs = np.full((len(lens), width), -1, np.int32), np.zeros(n_pages, np.int32)
    for b, n in enumerate(lens):
        k = -(-n // page)
        row = (shared + [order.pop() for _ in range(max(0, k - prompt))])[:k]
        tables[b, :k] = row
        refs[row] += 1
    return sv.records(rng, (n_pages, hkv, page)), tables, refs


def check_fork(rng, pool, tables, lens, parents, refs, page, reserve=0, in_place=False):
    got = sv.as_dict(pool)
    r = i32(refs)
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    out_refs = None if in_place else torch.full_like(r, 99)
    print(f"[fork] rows={len(parents)} pages={len(refs)} page={page} reserve={reserve}", flush=True)
    t, n, o = api.iq_fork_pages(got, i32(tables), i32(lens), i32(parents), r, out_refs=out_refs,
                                reserve=reserve, status=status)
    assert (o is r) == in_place
    want = osv.fork(pool, tables, lens, parents, refs, page, reserve)
    same(t, want[0], "tables")
    same(n, want[1], "lengths")
    same(o, want[2], "counts")
    if not in_place:
        same(r, np.asarray(refs, np.int32), "counts before")
    assert status.item() == want[3]
    for x, name in zip(pool, sv.NAMES):
        same(got[name], x, name)
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page,hkv,n_pages,reserve", [(16, 1, 200, 0), (16, 3, 4100, 5),
                                                     (64, 2, 130, 64), (32, 4, 2048, 100)])
def test_fork(page, hkv, n_pages, reserve, in_place):
    rng = np.random.default_rng([page, hkv, reserve])
    lens = [0, 1, page - 1, page, page + 1, 3 * page, 5 * page + 7, 4 * page - 1]
    pool, tables, refs = state(rng, lens, page, 12, hkv, n_pages)
    # freed, kept, several of one, changed places, empty rows, more rows than before
    parents = [6, 6, -1, 0, 2, 6, 5, 5, 7, -1, 3, 1, 6, 0]
    check_fork(rng, pool, tables, lens, parents, refs, page, reserve, in_place)


@pytest.mark.parametrize("beams", [2, 4, 7])
def test_beam_search(beams):
    """Rounds of reordering; what the tables say afterwards is what each beam
    wrote."""
    rng = np.random.default_rng(beams)
    page, hkv, width, n_pages = 16, 2, 8, 64
    lens = [37] * beams
    pool, tables, refs = state(rng, lens, page, width, hkv, n_pages, prompt=1)
    for _ in range(4):
        parents = rng.integers(0, beams, beams).astype(np.int32)
        want = check_fork(rng, pool, tables, lens, parents, refs, page, reserve=1)
        tables, lens, refs = want[0], [int(n) for n in want[1]], want[2]
        count = np.bincount(tables[tables >= 0], minlength=n_pages)
        assert np.array_equal(count, refs)
        for b, n in enumerate(lens):           # each beam's next token, in its own page
            p = tables[b, n // page]
            assert refs[p] == 1
            for a in pool:
                a[p, :, n % page] = rng.integers(0, 200)
        lens = [n + 1 for n in lens]


def test_fork_full_pool():
    """No page is free but for those that the call frees, and too few."""
    rng = np.random.default_rng(1)
    page, lens = 16, [20, 30, 40, 5]
    pool, tables, refs = state(rng, lens, page, 4, 2, 8)
    assert (refs > 0).all()
    check_fork(rng, [a.copy() for a in pool], tables, lens, [2, 2, 0, 0], refs, page)
    want = check_fork(rng, pool, tables, lens, [0, 0, 1, 1, 1, 2, 2, 2], refs, page)
    assert want[3] == 5 and 16 in want[1]


def test_fork_pages_held_elsewhere():
    """A partly filled page that somebody else counts is copied even for the
    first row; one that two rows hold is kept by neither; entries outside the
    pool and a parent past the rows."""
    rng = np.random.default_rng(2)
    page, lens = 16, [20, 25, 40, 9]
    pool, tables, refs = state(rng, lens, page, 4, 2, 40)
    refs[tables[0, 1]] += 1
    tables[3, 0] = tables[1, 1]
    refs[tables[1, 1]] += 1
    tables[2, 1] = 40
    tables[2, 3] = -9
    check_fork(rng, pool, tables, lens, [0, 0, 1, 3, 2, 2, 4, 2 ** 30], refs, page, reserve=3)


def test_fork_lengths_outside_the_tables():
    rng = np.random.default_rng(12)
    page, lens = 16, [20, 33, 64]
    pool, tables, refs = state(rng, lens, page, 4, 1, 30)
    check_fork(rng, pool, tables, [-5, 1000, 64], [0, 1, 1, 2], refs, page, reserve=1000)


def test_fork_one_large_page():
    """A page of many pieces."""
    rng = np.random.default_rng(13)
    page = 4096
    pool, tables, refs = state(rng, [5000, 4096], page, 2, 2, 5)
    check_fork(rng, pool, tables, [5000, 4096], [0, 0, 0], refs, page)


def test_fork_many_rows():
    rng = np.random.default_rng(14)
    b, page = 700, 16
    lens = [int(n) for n in rng.integers(0, 50, b)]
    pool, tables, refs = state(rng, lens, page, 5, 1, 6000)
    parents = rng.integers(-1, b, 900)
    check_fork(rng, pool, tables, lens, parents, refs, page, reserve=2)


# ---------------------------------------------------------------- compaction

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n_pages,share", [(1, 0.0), (1, 1.0), (63, 0.5), (64, 0.5), (65, 0.3),
                                           (2048, 0.9), (2049, 0.1), (5000, 0.5), (300, 0.0),
                                           (300, 1.0)])
def test_compact(n_pages, share, in_place):
    rng = np.random.default_rng([n_pages, int(share * 10)])
    hkv, page, width = 2, 16, 9
    refs = (rng.random(n_pages) < share) * rng.integers(1, 4, n_pages)
    refs = (refs - (rng.random(n_pages) < 0.05) * 4).clip(-1).astype(np.int32)
    live = np.flatnonzero(refs > 0)
    tables = np.full((11, width), -1, np.int32)
    if live.size:
        tables[:] = rng.choice(live, tables.shape)
    tables[0, :4] = [-1, -5, n_pages, 2 ** 31 - 1]
    free = np.flatnonzero(refs <= 0)
    if free.size:
        tables[1, 0] = free[0]
    pool = sv.records(rng, (n_pages, hkv, page))
    got, t, r = sv.as_dict(pool), i32(tables), i32(refs)
    print(f"[compact] {n_pages} pages, {live.size} live", flush=True)
    kw = {} if in_place else {"out_tables": torch.zeros_like(t), "out_refs": torch.zeros_like(r)}
    ot, orefs, page_map, n_live = api.iq_compact_pages(got, t, r, **kw)
    assert (ot is t) == in_place and (orefs is r) == in_place
    want = osv.compact(pool, tables, refs)
    same(ot, want[0], "tables")
    same(orefs, want[1].astype(np.int32), "counts")
    same(page_map, want[2], "map")
    assert n_live.item() == want[3]
    for x, name in zip(pool, sv.NAMES):
        same(got[name], x, name)


def test_compact_large_pages():
    rng = np.random.default_rng(21)
    refs = np.asarray([0, 0, 1, 0, 2, 1], np.int32)
    pool = sv.records(rng, (6, 3, 2048))
    got = sv.as_dict(pool)
    t = i32([[2, 4, 5, -1]])
    api.iq_compact_pages(got, t, i32(refs))
    want = osv.compact(pool, np.asarray([[2, 4, 5, -1]], np.int32), refs)
    same(t, want[0], "tables")
    for x, name in zip(pool, sv.NAMES):
        same(got[name], x, name)
