"""The windowed steps and trees where the work is cut differently: rows of many
parts, lengths at their bound, waves with more batches than a load of the page
table holds, values that are not finite in one part of many, more sequences than
a workgroup has threads.  Against the oracle in 64 bits."""

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2608_08081_amd import api
from tests import serving as sv
from tests.test_gpu_tree import case, check, hide, oracle, run
from tests.test_gpu_window import _hide

pytestmark = pytest.mark.gpu


def i32(x):
    return sv.dev(np.asarray(x, np.int32))


def steps(rng, cache, read, step, lens, cap, hkv, group, quats, window, sinks, bits, count,
          most=None):
    """`count` steps in a row: what each writes is what the one-token compression
    writes, what it returns is the oracle's attention of the advanced rows (of
    `most` positions at most)."""
    b = len(lens)
    seq = i32(lens)
    after = list(lens)
    for s in range(count):
        q = rng.standard_normal((b, hkv * group, sv.D)).astype(np.float32)
        new = [sv.dev(rng.standard_normal((b, hkv, sv.D)).astype(np.float32)) for _ in range(2)]
        before = read()
        print(f"[edges] step {s} cap={cap} window={window}+{sinks} bits={bits}", flush=True)
        got = step(sv.dev(q), new, seq)
        rows = read()
        for i, n in enumerate(after):
            if n >= cap:
                continue
            one = [x[i:i + 1].unsqueeze(2).contiguous() for x in new]
            c = [sv.dev(a[i:i + 1, :, n:n + 1]) for a in before]
            api.iq_compress_kv_bits(*one, quats, *c, bits=bits)
            for a, x in zip(before, c):
                a[i:i + 1, :, n:n + 1] = x.cpu().numpy()
            after[i] = n + 1
        assert seq.tolist() == after
        for a, x in zip(rows, before):
            assert np.array_equal(a.view(np.uint8), x.view(np.uint8))
        seen = [min(n, most or cap) for n in after]
        want = osv.decode_window(q, *rows, seen, quats.cpu().numpy(), sv.levels(bits), window,
                                 sinks)
        sv.check_rows(got, want, f"step {s}")


@pytest.mark.parametrize("bits,hkv,group,cap,lens,window,sinks", [
    (3, 2, 8, 8192, [8190], 4096, 4),           # 32 parts and the new token's
    (2, 1, 8, 8192, [8191], 4096, 4),
    (4, 2, 5, 8192, [8190], 4096, 16),
    (3, 1, 16, 4096, [4000, 31], 2500, 40),     # two groups of heads
    (3, 1, 8, 4096, [0], 4096, 0),              # nothing cached
    (3, 4, 8, 2048, [2047, 600], 1000, 7),      # 7 parts
])
def test_step_on_rows_of_many_parts(bits, hkv, group, cap, lens, window, sinks):
    rng = np.random.default_rng([bits, hkv, cap, window])
    rows = sv.records(rng, (len(lens), hkv, cap), bits)
    _hide(rows, lens, window, sinks, span=3)
    quats = sv.dev(sv.rotation(21, hkv))
    cache = [sv.dev(a) for a in rows]
    steps(rng, cache, lambda: [a.cpu().numpy() for a in cache],
          lambda q, new, seq: api.iq_decode_step_window(q, *new, *cache, seq, quats, window, sinks,
                                                        bits=bits),
          lens, cap, hkv, group, quats, window, sinks, bits, 3)


def pool_reader(pool, tables, hkv, page):
    """The sequences' rows [B][H][capacity] as they stand on the pool (a row's
    entries outside it: NaN scales)."""
    def read():
        out = []
        for n in sv.NAMES:
            a = pool[n].cpu().numpy()
            shape = (len(tables), hkv, tables.shape[1] * page) + a.shape[3:]
            r = np.full(shape, np.nan if a.dtype == np.float32 else 0, a.dtype)
            for b, row in enumerate(tables):
                for k, p in enumerate(row):
                    if 0 <= p < len(a):
                        r[b, :, k * page:(k + 1) * page] = a[p]
            out.append(r)
        return out
    return read


@pytest.mark.parametrize("hkv,group,page,cap,lens,window,sinks", [
    (2, 8, 32, 8192, [8190], 4096, 4),          # 32 parts
    (1, 16, 16, 4096, [4094, 15], 2500, 40),
    (4, 8, 64, 2048, [2045, 640], 1000, 7),
])
def test_step_on_pools_of_many_parts(hkv, group, page, cap, lens, window, sinks):
    rng = np.random.default_rng([hkv, page, cap, window])
    rows = sv.records(rng, (len(lens), hkv, cap))
    _hide(rows, lens, window, sinks, span=3)
    arrays, tables = sv.to_pool(rng, rows, [min(n + 3, cap) for n in lens], page, cap // page)
    pool, quats, tab = sv.as_dict(arrays), sv.dev(sv.rotation(22, hkv)), sv.dev(tables)
    steps(rng, pool, pool_reader(pool, tables, hkv, page),
          lambda q, new, seq: api.iq_decode_step_window_paged(q, *new, pool, tab, seq, quats, window,
                                                              sinks),
          lens, cap, hkv, group, quats, window, sinks, 3, 2)


@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 3), (200, 0), (7, 150)])
@pytest.mark.parametrize("paged", [False, True])
def test_step_at_the_bound_of_the_lengths(window, sinks, paged):
    """Rows below, at and above max_seq_len: the token is written, and attended
    only where it is before the bound."""
    rng = np.random.default_rng([window, sinks, paged])
    hkv, group, cap, most, page = 2, 4, 256, 150, 16
    lens = [148, 149, 150, 151, 200, 0, 255, 256]
    rows = sv.records(rng, (len(lens), hkv, cap))
    quats = sv.dev(sv.rotation(23, hkv))
    if paged:
        arrays, tables = sv.to_pool(rng, rows, [cap] * len(lens), page, cap // page)
        pool, tab = sv.as_dict(arrays), sv.dev(tables)
        read = pool_reader(pool, tables, hkv, page)

        def step(q, new, seq):
            return api.iq_decode_step_window_paged(q, *new, pool, tab, seq, quats, window, sinks,
                                                   max_seq_len=most)
    else:
        cache = [sv.dev(a) for a in rows]

        def read():
            return [a.cpu().numpy() for a in cache]

        def step(q, new, seq):
            return api.iq_decode_step_window(q, *new, *cache, seq, quats, window, sinks,
                                             max_seq_len=most)
    steps(rng, None, read, step, lens, cap, hkv, group, quats, window, sinks, 3, 3, most)


@pytest.mark.parametrize("bits", [2, 4])
def test_long_rows_of_other_widths(bits):
    rng = np.random.default_rng([24, bits])
    hkv, group, cap, lens, window, sinks = 1, 8, 8192, [8192, 5000], 4096, 4
    rows = sv.records(rng, (2, hkv, cap), bits)
    quats = sv.rotation(24, hkv)
    q = rng.standard_normal((2, hkv * group, sv.D)).astype(np.float32)
    want = osv.decode_window(q, *rows, lens, quats, sv.levels(bits), window, sinks)
    _hide(rows, lens, window, sinks)
    print(f"[edges] rows of 8192 at {bits} bits", flush=True)
    got = api.iq_decode_attention_window(sv.dev(q), *map(sv.dev, rows), i32(lens), sv.dev(quats),
                                         window, sinks, bits=bits)
    sv.check_rows(got, want, f"{bits} bits")


def test_more_batches_than_a_load_of_the_table():
    """264 rows of one part, 65 and 66 batches to a wave: the page table is read
    again behind the hole.  (The sequences share the pool's pages in orders of
    their own; a page without a visible position is not mapped.)"""
    rng = np.random.default_rng(25)
    b, hkv, group, page, cap, window, sinks = 33, 8, 2, 16, 9008, 8300, 20
    n_pages, width = 700, cap // page
    arrays = sv.records(rng, (n_pages, hkv, page))
    lens = [int(n) for n in rng.integers(8400, cap + 1, b)]
    lens[3:6] = [cap, 17, 8300]
    tables = np.stack([rng.permutation(n_pages)[:width] for _ in range(b)]).astype(np.int32)
    for i, n in enumerate(lens):
        see = np.zeros(cap, bool)
        see[:n] = osv.window_visible(n, window, sinks)
        tables[i, ~see.reshape(width, page).any(1)] = -1
    assert (tables < 0).sum() > 100
    quats = sv.rotation(25, hkv)
    q = rng.standard_normal((b, hkv * group, sv.D)).astype(np.float32)
    pool = sv.as_dict(arrays)
    print("[edges] 264 rows of 8320 positions", flush=True)
    got = api.iq_decode_attention_window_paged(sv.dev(q), pool, sv.dev(tables), i32(lens),
                                               sv.dev(quats), window, sinks)
    some = [0, 3, 4, 5, 13, 32]       # (the oracle takes a second per sequence)
    rows = [np.ascontiguousarray(a[np.maximum(tables[some], 0)].swapaxes(1, 2)).reshape(
        (len(some), hkv, cap) + a.shape[3:]) for a in arrays]
    want = osv.decode_window(q[some], *rows, [lens[i] for i in some], quats, sv.levels(3), window,
                             sinks)
    sv.check_rows(got[some], want, "long waves")
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("cap,window", [(1024, 600), (8192, 4096)])     # 4 and 32 parts
def test_not_finite_in_one_part(cap, window):
    """A NaN key scale, a value scale that is not finite, and keys that are NaN
    in a whole part or everywhere show in the rows that attend them and in no
    other, with the step's merge and without."""
    rng = np.random.default_rng([26, cap])
    b, hkv, group, sinks, n = 6, 2, 8, 4, cap - 5
    rows = sv.records(rng, (b, hkv, cap))
    rows[1][0, 1, n - 100] = np.nan                      # a key
    rows[3][1, 0, 2] = np.inf                            # a sink's value
    rows[3][2, 1, n - window + 3] = np.nan               # a value at the window's start
    rows[1][3, 0, n - 300:n - 100] = np.nan              # all keys of a part
    rows[1][4, 1, :] = np.nan                            # all keys
    rows[1][5, :, sinks:n - window - 2] = np.nan         # behind the hole: nobody's
    rows[3][5, :, sinks:n - window - 2] = np.inf
    quats = sv.dev(sv.rotation(26, hkv))
    q = sv.dev(rng.standard_normal((b, hkv * group, sv.D)).astype(np.float32))
    bad = np.zeros((b, hkv, group), bool)
    for i, g in ((0, 1), (1, 0), (2, 1), (3, 0), (4, 1)):
        bad[i, g] = True
    cache = [sv.dev(a) for a in rows]
    print(f"[edges] not finite, window {window}", flush=True)
    got = api.iq_decode_attention_window(q, *cache, i32([n] * b), quats, window, sinks)
    finite = np.isfinite(got.cpu().numpy()).all(-1).reshape(bad.shape)
    assert np.array_equal(~finite, bad)
    new = [sv.dev(rng.standard_normal((b, hkv, sv.D)).astype(np.float32)) for _ in range(2)]
    got = api.iq_decode_step_window(q, *new, *cache, i32([n] * b), quats, window, sinks)
    finite = np.isfinite(got.cpu().numpy()).all(-1).reshape(bad.shape)
    assert np.array_equal(~finite, bad)


@pytest.mark.parametrize("b,t,page", [(300, 5, 0), (600, 3, 16), (513, 17, 0)])
def test_trees_of_many_sequences(b, t, page):
    """More sequences than a workgroup that plans has threads: the pieces of each
    round of 256."""
    rng = np.random.default_rng(b)
    lens = [int(n) for n in rng.integers(0, 91, b)]
    lens[256:260] = [0, 90, 1, 64]
    cap = 96
    c = case(b + t, lens, 1, 2 if t < 10 else 8, cap, t, padding=1)
    if not page:
        return check(c, f"{b} sequences")
    want = oracle(c)
    hide(c)
    c["pool"], c["tables"] = sv.to_pool(rng, c["rows"], lens, page, cap // page)
    print(f"[tree] {b} sequences on pools", flush=True)
    sv.check_rows(run(c), want, f"{b} sequences on pools")
