"""Attention behind a sliding window with sinks: rows and pools, decode and the
fused step, against the oracle in 64 bits.  Everything outside what a row sees
has NaN scales, so that a position too many shows."""

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2608_08081_amd import api
from tests import serving as sv

pytestmark = pytest.mark.gpu


def _hide(rows, lens, window, sinks, span=0):
    """NaN scales wherever no row sees (lengths up to lens + span)."""
    for b, n in enumerate(lens):
        see = np.zeros(rows[1].shape[2], bool)
        for m in range(n, n + span + 1):
            v = osv.window_visible(m, window, sinks)
            see[:m] |= v[:len(see)]
        see[n:] = False
        rows[1][b][:, ~see] = np.nan
        rows[3][b][:, ~see] = np.nan


SHAPES = [
    # hkv, group, cap, lengths, window, sinks
    (1, 1, 16, [0, 1, 2, 15, 16], 1, 0),
    (2, 8, 64, [0, 1, 5, 16, 17, 31, 32, 33, 48, 64], 16, 1),
    (2, 4, 256, [100, 255, 256, 3, 130], 33, 5),
    (1, 16, 512, [512, 511, 400, 77], 100, 4),
    (4, 5, 1024, [1024, 1000, 129, 128, 127, 64], 127, 63),
    (1, 9, 1040, [1040, 1039, 600], 65, 130),        # sinks beyond a chunk
    (8, 8, 2048, [2048, 1500], 700, 16),
    (2, 8, 4096, [4096, 4095, 37], 4096, 0),         # a window of the whole row
    (2, 3, 320, [320, 17, 200], 7, 320),             # sinks of the whole row
    (1, 8, 8192, [8192], 4096, 4),
]


@pytest.mark.parametrize("bits", [3, 2, 4])
@pytest.mark.parametrize("hkv,group,cap,lens,window,sinks", SHAPES)
def test_rows(hkv, group, cap, lens, window, sinks, bits):
    if bits != 3 and cap > 2048:
        pytest.skip("the widths share the walk; long rows at 3 bits")
    rng = np.random.default_rng([hkv, group, cap, window, sinks, bits])
    b, hq = len(lens), hkv * group
    rows = sv.records(rng, (b, hkv, cap), bits)
    quats = sv.rotation(5, hkv)
    q = rng.standard_normal((b, hq, sv.D)).astype(np.float32)
    want = osv.decode_window(q, *rows, lens, quats, sv.levels(bits), window, sinks)
    _hide(rows, lens, window, sinks)
    print(f"[window] hkv={hkv} group={group} cap={cap} window={window} sinks={sinks} bits={bits}",
          flush=True)
    args = (sv.dev(q), *map(sv.dev, rows), sv.dev(np.asarray(lens, np.int32)), sv.dev(quats),
            window, sinks)
    got = api.iq_decode_attention_window(*args, bits=bits)
    sv.check_rows(got, want, f"window {window}+{sinks}")
    assert torch.equal(got, api.iq_decode_attention_window(*args, bits=bits))


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("hkv,group,cap,lens,window,sinks", [
    (2, 8, 256, [0, 1, 17, 100, 255, 256], 40, 3),
    (1, 4, 1024, [1024, 1000, 513, 30], 300, 70),
    (3, 12, 4096, [4096, 2000, 64], 1000, 16),
])
def test_pools(hkv, group, cap, lens, window, sinks, page):
    rng = np.random.default_rng([hkv, group, cap, page])
    b, hq = len(lens), hkv * group
    rows = sv.records(rng, (b, hkv, cap))
    quats = sv.rotation(6, hkv)
    q = rng.standard_normal((b, hq, sv.D)).astype(np.float32)
    want = osv.decode_window(q, *rows, lens, quats, sv.levels(3), window, sinks)
    _hide(rows, lens, window, sinks)
    pool, tables = sv.to_pool(rng, rows, lens, page, cap // page)
    # pages without a visible position need not be mapped
    for i, n in enumerate(lens):
        see = osv.window_visible(n, window, sinks)
        for k in range(-(-n // page)):
            if not see[k * page:(k + 1) * page].any():
                tables[i, k] = [-1, 2 ** 31 - 1][k % 2]
    if not (tables == 0).any():        # (entries outside the pool read page 0)
        pool[1][0] = pool[3][0] = np.nan
    print(f"[window] pool page={page} cap={cap} window={window} sinks={sinks}", flush=True)
    got = api.iq_decode_attention_window_paged(
        sv.dev(q), sv.as_dict(pool), sv.dev(tables), sv.dev(np.asarray(lens, np.int32)),
        sv.dev(quats), window, sinks)
    sv.check_rows(got, want, f"paged window {window}+{sinks}")


@pytest.mark.parametrize("scale,most", [(0.3, None), (0.0, 150)])
def test_scale_and_bound_of_the_lengths(scale, most):
    """Lengths above max_seq_len count as max_seq_len (the window ends there)."""
    rng = np.random.default_rng(11)
    lens, hkv = [200, 256, 90], 2
    rows = sv.records(rng, (3, hkv, 256))
    quats = sv.rotation(1, hkv)
    q = rng.standard_normal((3, 16, sv.D)).astype(np.float32)
    seen = [min(n, most or 256) for n in lens]
    want = osv.decode_window(q, *rows, seen, quats, sv.levels(3), 50, 2, scale)
    got = api.iq_decode_attention_window(
        sv.dev(q), *map(sv.dev, rows), sv.dev(np.asarray(lens, np.int32)), sv.dev(quats), 50, 2,
        max_seq_len=most, softmax_scale=scale)
    sv.check_rows(got, want, "scale")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("bits,hkv,group,cap,lens,window,sinks", [
    (3, 2, 8, 64, [0, 1, 15, 16, 40, 63, 64], 16, 1),
    (3, 4, 4, 512, [511, 512, 300, 0], 1, 0),
    (2, 1, 9, 256, [255, 100, 17], 64, 4),
    (4, 3, 5, 1024, [1000, 1023, 5], 500, 20),
])
def test_step_on_rows(bits, hkv, group, cap, lens, window, sinks, dtype):
    """The step writes what iq_append_token / the bulk compression writes and
    attends the advanced rows; a full row drops its token and attends as it is."""
    rng = np.random.default_rng([bits, hkv, cap, window])
    b, hq = len(lens), hkv * group
    rows = sv.records(rng, (b, hkv, cap), bits)
    _hide(rows, lens, window, sinks, span=1)
    quats = sv.dev(sv.rotation(7, hkv))
    q = rng.standard_normal((b, hq, sv.D)).astype(np.float32)
    new = [torch.from_numpy(rng.standard_normal((b, hkv, sv.D))).to(sv.DEV, dtype)
           for _ in range(2)]
    cache = [sv.dev(a) for a in rows]
    seq = sv.dev(np.asarray(lens, np.int32))
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    print(f"[window step] bits={bits} cap={cap} window={window}", flush=True)
    got = api.iq_decode_step_window(sv.dev(q), *new, *cache, seq, quats, window, sinks,
                                    status=status, bits=bits)
    fits = [n < cap for n in lens]
    after = [n + f for n, f in zip(lens, fits)]
    assert seq.tolist() == after
    assert status.item() == (0 if all(fits) else 5)
    # what was written: one-token bulk compression, sequence by sequence
    want_rows = [sv.dev(a) for a in rows]
    for i, n in enumerate(lens):
        if fits[i]:
            one = [x[i:i + 1].unsqueeze(2).contiguous() for x in new]
            c = [a[i:i + 1] for a in want_rows]
            api.iq_compress_kv_bits(*one, quats, c[0], c[1], c[2], c[3], dst_offset=n, bits=bits)
    for a, x in zip(cache, want_rows):
        assert torch.equal(a.view(torch.uint8), x.view(torch.uint8))
    want = osv.decode_window(q, *[a.cpu().numpy() for a in cache], after, quats.cpu().numpy(),
                             sv.levels(bits), window, sinks)
    sv.check_rows(got, want, "step")


def test_step_on_pools():
    """Pool steps: tokens across page borders, a page that is not mapped, a full
    sequence."""
    rng = np.random.default_rng(3)
    hkv, group, page, cap, window, sinks = 2, 8, 16, 128, 30, 5
    lens = [0, 15, 16, 31, 100, 127, 128]
    rows = sv.records(rng, (len(lens), hkv, cap))
    _hide(rows, lens, window, sinks, span=1)
    pool, tables = sv.to_pool(rng, rows, lens, page, cap // page, extra=8)
    free = sorted(set(range(len(pool[0]))) - set(tables.ravel()))
    for b, n in enumerate(lens):
        if n < cap and tables[b, n // page] < 0 and b != 2:   # sequence 2: not mapped
            tables[b, n // page] = free.pop()
    quats = sv.rotation(8, hkv)
    q = rng.standard_normal((len(lens), hkv * group, sv.D)).astype(np.float32)
    new = [rng.standard_normal((len(lens), hkv, sv.D)).astype(np.float32) for _ in range(2)]
    out = {}
    for name in ("window", "plain"):
        p, seq = sv.as_dict(pool), sv.dev(np.asarray(lens, np.int32))
        status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
        args = (sv.dev(q), *map(sv.dev, new), p, sv.dev(tables), seq, sv.dev(quats))
        if name == "window":
            got = api.iq_decode_step_window_paged(*args, window, sinks, status=status)
        else:
            api.iq_decode_step_paged(*args, status=status)
        out[name] = [p[n].cpu().numpy() for n in sv.NAMES] + [seq.cpu().numpy(),
                                                               status.cpu().numpy()]
    for a, x in zip(out["window"], out["plain"]):
        assert np.array_equal(a.view(np.uint8), x.view(np.uint8))
    after = out["window"][4]
    assert list(after) == [1, 16, 16, 32, 101, 128, 128] and out["window"][5][0] == 5
    got = got.cpu()
    flat = []
    for a in out["window"][:4]:
        r = np.zeros((len(lens), hkv, cap) + a.shape[3:], a.dtype)
        for b, n in enumerate(after):
            for k in range(-(-int(n) // page)):
                r[b, :, k * page:(k + 1) * page] = a[tables[b, k]]
        flat.append(r)
    want = osv.decode_window(q, *flat, after, quats, sv.levels(3), window, sinks)
    sv.check_rows(got, want, "pool step")


def test_not_finite_where_seen_only():
    """A NaN query, key scale or value scale inside the window shows in the rows
    that attend it and in no other."""
    rng = np.random.default_rng(4)
    lens, hkv, window, sinks = [300, 300, 300, 300], 2, 100, 4
    rows = sv.records(rng, (4, hkv, 320))
    quats = sv.rotation(9, hkv)
    q = rng.standard_normal((4, 16, sv.D)).astype(np.float32)
    rows[1][0, 1, 250] = np.nan          # a key in the window: sequence 0, heads 8 .. 15
    rows[3][1, 0, 2] = np.inf            # a sink's value: sequence 1, heads 0 .. 7
    q[2, 5, 7] = np.nan
    got = api.iq_decode_attention_window(
        sv.dev(q), *map(sv.dev, rows), sv.dev(np.asarray(lens, np.int32)), sv.dev(quats), window,
        sinks).cpu().numpy()
    bad = ~np.isfinite(got).all(-1)
    want = np.zeros((4, 16), bool)
    want[0, 8:] = want[1, :8] = want[2, 5] = True
    # (an infinite value scale times a weight of any size is not finite)
    assert np.array_equal(bad, want)


def test_many_rows():
    """More rows than workgroups: one part per row, several rounds."""
    rng = np.random.default_rng(5)
    b, hkv, cap = 150, 4, 96
    lens = rng.integers(0, cap + 1, b)
    rows = sv.records(rng, (b, hkv, cap))
    quats = sv.rotation(10, hkv)
    q = rng.standard_normal((b, hkv, sv.D)).astype(np.float32)
    want = osv.decode_window(q, *rows, lens, quats, sv.levels(3), 20, 3)
    got = api.iq_decode_attention_window(
        sv.dev(q), *map(sv.dev, rows), sv.dev(lens.astype(np.int32)), sv.dev(quats), 20, 3)
    sv.check_rows(got, want, "many rows")
