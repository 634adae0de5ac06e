"""Attention of trees of drafted tokens against the oracle in 64 bits: group
sizes and numbers of nodes around the kernel's tile and row counts, rows of any
capacity and pools, windows, padding.  What no node sees has NaN scales."""

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2608_08081_amd import api
from tests import serving as sv

pytestmark = pytest.mark.gpu


def random_tree(rng, t, padding=0):
    """Mask words of a random tree of t nodes, the last `padding` of them not
    there."""
    parents = [-1] + [int(rng.integers(max(-1, i - 5), i)) for i in range(1, t)]
    for i in range(t - padding, t):
        parents[i] = -2
    return api.tree_mask(np.asarray(parents)).numpy()


def case(seed, lens, hkv, group, cap, t, window=0, sinks=0, bits=3, dcap=None, padding=0):
    rng = np.random.default_rng(seed)
    b = len(lens)
    c = {"lens": lens, "rows": sv.records(rng, (b, hkv, cap), bits),
         "draft": sv.records(rng, (b, hkv, dcap or t), bits), "quats": sv.rotation(seed, hkv),
         "q": rng.standard_normal((b, t, hkv * group, sv.D)).astype(np.float32),
         "words": np.stack([random_tree(rng, t, padding if i % 2 else 0) for i in range(b)]),
         "window": window, "sinks": sinks, "bits": bits, "rng": rng}
    return c


def oracle(c):
    seen = [min(n, c["rows"][1].shape[2]) for n in c["lens"]]
    return osv.decode_tree(c["q"], *c["rows"], seen, *c["draft"], c["words"], c["quats"],
                           sv.levels(c["bits"]), c["window"], c["sinks"])


def hide(c):
    """NaN scales where no node sees."""
    for b, n in enumerate(c["lens"]):
        cached, nodes = osv.tree_visible(c["words"][b], n, c["window"], c["sinks"])
        for a, see in ((c["rows"], cached.any(0)), (c["draft"], nodes.any(0))):
            full = np.zeros(a[1].shape[2], bool)
            full[:len(see)] = see
            a[1][b][:, ~full] = np.nan
            a[3][b][:, ~full] = np.nan


def run(c, **kw):
    args = (sv.dev(np.asarray(c["lens"], np.int32)), sv.as_dict(c["draft"]), sv.dev(c["words"]),
            sv.dev(c["quats"]))
    kw = {"window": c["window"], "n_sinks": c["sinks"], **kw}
    if "tables" in c:
        return api.iq_decode_attention_tree_paged(sv.dev(c["q"]), sv.as_dict(c["pool"]),
                                                  sv.dev(c["tables"]), *args, **kw)
    return api.iq_decode_attention_tree(sv.dev(c["q"]), *map(sv.dev, c["rows"]), *args,
                                        bits=c["bits"], **kw)


def check(c, label):
    want = oracle(c)
    hide(c)
    print(f"[tree] {label}", flush=True)
    got = run(c)
    sv.check_rows(got, want, label)
    assert torch.equal(got, run(c))


@pytest.mark.parametrize("t,hkv,group,cap,lens", [
    (1, 1, 1, 1, [0]),
    (1, 2, 8, 40, [0, 1, 31, 32, 33, 40]),
    (2, 1, 16, 33, [33, 7]),
    (5, 2, 7, 100, [100, 99, 64, 3]),
    (8, 4, 8, 257, [257, 256, 255, 0]),
    (9, 1, 8, 96, [96, 95]),                # 72 rows: a block of four waves, not full
    (13, 2, 5, 700, [700, 650]),
    (16, 1, 8, 1000, [1000]),               # 128 rows
    (17, 2, 8, 500, [500, 31]),             # 136 rows
    (33, 1, 1, 64, [64, 63, 1]),            # two tiles of nodes, few rows
    (32, 2, 8, 320, [320, 300]),            # 256 rows
    (40, 1, 16, 130, [130, 17]),            # 640 rows: three blocks
    (64, 2, 4, 600, [600, 599]),
    (64, 1, 16, 200, [200]),                # 1024 rows
])
def test_rows(t, hkv, group, cap, lens):
    check(case(t * 1000 + cap, lens, hkv, group, cap, t), f"T={t} {hkv}x{group} {lens}")


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("t,group,cap,lens", [(3, 4, 90, [90, 45]), (12, 5, 333, [333, 12]),
                                              (24, 8, 256, [256, 1])])
def test_widths(t, group, cap, lens, bits):
    check(case(t + bits, lens, 2, group, cap, t, bits=bits), f"T={t} bits={bits}")


@pytest.mark.parametrize("t,group,cap,lens,window,sinks", [
    (1, 8, 64, [64, 10, 0], 1, 0),
    (6, 4, 200, [200, 199, 5, 0], 3, 0),
    (6, 4, 200, [200, 199, 5, 0], 3, 2),
    (13, 5, 1000, [1000, 700, 64], 100, 4),
    (24, 8, 600, [600, 33], 64, 40),
    (64, 2, 400, [400, 100], 33, 1),
    (20, 8, 128, [128, 3], 500, 4),         # a window past every row
    (20, 8, 128, [128, 3], 9, 500),         # sinks past every row
])
def test_windows(t, group, cap, lens, window, sinks):
    check(case(t * 7 + window, lens, 2, group, cap, t, window=window, sinks=sinks),
          f"T={t} window={window}+{sinks}")


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("t,group,lens,window,sinks", [
    (4, 8, [100, 128, 0, 17], 0, 0), (24, 4, [700, 31], 0, 0), (24, 4, [700, 31], 200, 5),
    (64, 8, [300, 301], 0, 0)])
def test_pools(t, group, lens, window, sinks, page):
    cap = -(-max(lens) // page) * page + page
    c = case(t + page, lens, 2, group, cap, t, window=window, sinks=sinks, dcap=t + 3)
    want = oracle(c)
    hide(c)
    c["pool"], c["tables"] = sv.to_pool(c["rng"], c["rows"], lens, page, cap // page)
    print(f"[tree] pool T={t} page={page} window={window}", flush=True)
    sv.check_rows(run(c), want, "pool")


@pytest.mark.parametrize("t,group,lens,window,sinks,page", [
    (33, 4, [64, 33, 32, 31, 0, 1], 0, 0, 16),       # 132 rows; pairs of tiles that end anywhere
    (40, 8, [700, 95, 96, 97, 128], 0, 0, 32),       # 320 rows
    (64, 4, [500, 401, 160], 100, 5, 16),            # 256 rows, a window
    (50, 16, [1000, 3], 70, 40, 64),                 # 800 rows
    (40, 8, [700, 95, 96, 97, 128], 0, 0, 0),
    (64, 4, [500, 401, 160], 100, 5, 0),
])
def test_many_rows(t, group, lens, window, sinks, page):
    """More than 128 rows of a KV head, on pools and rows."""
    hkv, width = 2, 64
    cap = width * page if page else max(lens) + 3
    c = case(t * 31 + group + page, lens, hkv, group, cap, t, window=window, sinks=sinks)
    label = f"many rows T={t} group={group} page={page} window={window}"
    if not page:
        return check(c, label)
    want = oracle(c)
    hide(c)
    c["pool"], c["tables"] = sv.to_pool(c["rng"], c["rows"], lens, page, width)
    print(f"[tree] {label}", flush=True)
    got = run(c)
    sv.check_rows(got, want, label)
    assert torch.equal(got, run(c))


def test_padding_and_general_words():
    """Padded nodes give zero rows; a word need not be a tree's: nodes without
    themselves, roots in several places, bits past the nodes."""
    c = case(3, [50, 0, 65], 2, 4, 70, 11, padding=4, dcap=20)
    c["words"][0] = [1, 1, 0b100, 0b110, 0, 1 << 4, ~0, 0b1 | 1 << 40, 1 << 11, 1 << 9, 0b1000]
    check(c, "words")
    c = case(4, [0, 0], 1, 8, 16, 8, padding=8)
    c["words"][:] = 0
    check(c, "nothing at all")


def test_chain_is_multi_token_decode():
    """A chain of nodes gives what multi-token decode gives on a cache that
    holds them (both within their bounds of the oracle)."""
    c = case(5, [200, 333], 2, 8, 352, 4)
    c["words"][:] = np.asarray([1, 3, 7, 15])
    want = oracle(c)
    for b, n in enumerate(c["lens"]):
        for a, d in zip(c["rows"], c["draft"]):
            a[b, :, n:n + 4] = d[b]
    multi = api.iq_decode_attention_multi(
        sv.dev(c["q"]), *map(sv.dev, c["rows"]),
        sv.dev(np.asarray(c["lens"], np.int32) + 4), sv.dev(c["quats"]))
    sv.check_rows(multi, want, "multi-token")
    sv.check_rows(run(c), want, "tree")


def test_not_finite_where_seen_only():
    """A value or key scale that is not finite, at a node that some see, and a
    query that is not, show in those rows and nowhere else."""
    c = case(6, [100], 2, 4, 100, 10)
    c["words"][0] = [1, 0b11, 0b101, 0b1001, 0b10011, 0b100011, 0b1000101, 0b10001001, 0b100000001,
                     0b1000000001]
    want = oracle(c)
    for side, node, value in ((1, 2, np.nan), (3, 1, np.inf), (3, 3, np.nan)):
        d = [a.copy() for a in c["draft"]]
        d[side][0, 1, node] = value
        q = c["q"].copy()
        q[0, 8, 0, 3] = np.inf
        got = run({**c, "draft": d, "q": q}).cpu().numpy()
        _, nodes = osv.tree_visible(c["words"][0], 100, 0, 0)
        bad = np.zeros((10, 8), bool)
        bad[nodes[:, node], 4:] = True
        bad[8, 0] = True
        assert np.array_equal(~np.isfinite(got[0]).all(-1), bad)
        ok = ~bad
        err = np.linalg.norm(got[0][ok] - want[0][0][ok], axis=-1)
        assert np.all(err <= osv.error_bound(want[1][0][ok], want[2][0][ok]))


def test_large_scores_and_scales():
    """Weights far apart: a peaked softmax, value scales over many orders of
    magnitude (within 2^15), zero value scales, large and small queries."""
    c = case(7, [500, 480], 2, 4, 512, 9)
    r = c["rng"]
    c["rows"][3][:] *= np.exp(2.5 * r.standard_normal(c["rows"][3].shape)).astype(np.float32)
    c["rows"][3][0, 0] = 0
    c["draft"][3][0, 0] = 0
    c["q"][0] *= 8
    c["q"][1, 3] *= 1e-20
    check(c, "scales")


def test_scale_bound_and_other_stream():
    """softmax_scale, max_seq_len below the lengths, and a call on a side
    stream."""
    c = case(8, [300, 120], 1, 8, 304, 12)
    cut = {**c, "lens": [150, 120]}
    want = osv.decode_tree(c["q"], *c["rows"], [150, 120], *c["draft"], c["words"], c["quats"],
                           sv.levels(3), 0, 0, 0.25)
    assert oracle(cut)[0].shape == want[0].shape
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run(c, max_seq_len=150, softmax_scale=0.25)
    side.synchronize()
    sv.check_rows(got, want, "scale")


def test_many_sequences():
    rng = np.random.default_rng(9)
    lens = [int(n) for n in rng.integers(0, 90, 70)]
    check(case(9, lens, 3, 2, 90, 6, padding=2), "70 sequences")
