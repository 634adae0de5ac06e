"""GPU tests of prompts in chunks on page pools: pages and slots, rotary positions, compression
into slots and attention of chunks, against plain implementations in 64 bits."""

import numpy as np
import pytest
import torch

from oracle import codebook as ocb
from oracle import compress as ocz
from oracle import rotation as orot
from paper_2608_08081_amd import api
from tests import prefill as pf
from tests import serving as sv

pytestmark = pytest.mark.gpu
D = 128


# ---- pages and slots ------------------------------------------------------------------------
def extend_case(rng, rows, page, width, n_pages, context, new, reserve=0, bad=False):
    """Tables, lengths, new lengths and counts; some rows have pages beyond their length."""
    order = list(rng.permutation(n_pages))
    tables = np.full((rows, width), -1, np.int32)
    refs = np.where(rng.random(n_pages) < 0.1, -rng.integers(0, 3, n_pages), 0).astype(np.int32)
    lens = rng.integers(0, context + 1, rows).astype(np.int32)
    more = rng.integers(0, new + 1, rows).astype(np.int32)
    for b in range(rows):
        used = -(-int(lens[b]) // page)
        extra = int(rng.integers(0, reserve + 1))
        for k in range(min(width, used + extra)):
            if k >= used and rng.random() < 0.4:
                continue                        # a hole in what is reserved
            if not order:
                break
            p = order.pop()
            tables[b, k] = p
            refs[p] = 1
    for p in order[:len(order) // 6]:
        refs[p] += 2
    if bad:
        lens[rng.integers(0, rows)] = -3
        more[rng.integers(0, rows)] = -1
        more[rng.integers(0, rows)] = width * page + 1
        tables[0, -1] = n_pages
    return tables, lens, more, refs


EXTEND = [
    (1, 16, 4, 9, 20, 30, 0, False, 0), (7, 16, 20, 150, 200, 60, 0, False, 5),
    (64, 64, 8, 600, 400, 1, 0, False, 0), (65, 32, 12, 900, 200, 150, 3, False, 1),
    (33, 16, 40, 700, 300, 300, 5, False, 0), (300, 16, 30, 5000, 300, 100, 4, True, 9),
    (5, 16, 700, 4000, 2000, 9000, 40, False, 0), (1500, 16, 3, 2500, 20, 20, 1, False, 3),
    (3, 1024, 2, 5, 1500, 500, 0, False, 0), (70, 16, 20, 800, 160, 150, 6, False, -200)]


@pytest.mark.parametrize("rows,page,width,n_pages,context,new,reserve,bad,pad", EXTEND)
@pytest.mark.parametrize("in_place", [False, True])
def test_extend(rows, page, width, n_pages, context, new, reserve, bad, pad, in_place):
    rng = np.random.default_rng([rows, page, n_pages])
    tables, lens, more, refs = extend_case(rng, rows, page, width, n_pages, context, new, reserve,
                                           bad)
    n = max(0, int(np.maximum(more, 0).sum()) + pad)
    want = pf.extend(tables, lens, more, refs, page, n)
    t, ln, m, r = (sv.dev(x) for x in (tables, lens, more, refs))
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    kw = {} if in_place else {"out_tables": torch.full_like(t, 77), "out_lens": torch.full_like(ln, 77),
                              "out_refs": torch.full_like(r, 77)}
    got = api.iq_extend_pages(t, ln, m, r, page, n_tokens=n, status=status, **kw)
    for name, x, y in zip(("row_starts", "slots", "positions", "tables", "lens", "refs"), got, want):
        assert np.array_equal(x.cpu().numpy(), y), name
    assert int(status) == want[6]
    if not in_place:
        for x, y in ((t, tables), (ln, lens), (r, refs)):
            assert np.array_equal(x.cpu().numpy(), y), "an input changed"


# ---- rotary positions -----------------------------------------------------------------------
def rope_tolerance(x, dtype, amplitude):
    """Of values a cos - b sin with |a|, |b| <= x: the angle's rest is off by 2^-25 of at most pi /
    4, cos and sin by 4 units of 2^-24 (the functions' documented bound of 2, and the amplitude),
    their products by 2^-23 together, all of |x| 2^(1/2) amplitude; then half a step of the type
    of the result (fp16: at least 2^-25)."""
    m = np.sqrt(2.0) * np.abs(x).max() * abs(amplitude)
    t = m * (2.0 ** -25 + 4 * 2.0 ** -24 + 2.0 ** -23)
    return t + (m * 2.0 ** -11 + 2.0 ** -25 if dtype == torch.float16 else m * 2.0 ** -24)


@pytest.mark.parametrize("n,hq,hkv,dim,m,far", [
    (1, 32, 4, 128, 128, 32768), (3, 5, 1, 128, 64, 1 << 20), (5, 1, 1, 128, 16, 100),
    (130, 8, 8, 128, 96, 1 << 30), (17, 16, 1, 64, 64, 70000), (9, 3, 2, 64, 48, 5000),
    (1025, 4, 2, 128, 128, 1 << 31)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_rotate(n, hq, hkv, dim, m, far, layout, dtype):
    rng = np.random.default_rng([n, dim, m])
    x = torch.from_numpy(rng.standard_normal((n, hq + 2 * hkv, dim)) * 3).to(dtype)
    pos = rng.integers(-far, far, n).astype(np.int32)
    pos[0] = 0 if n > 1 else far - 1
    freqs = api.iq_rope_frequencies(m)
    xd = x.to(sv.DEV)
    q, k = xd[:, :hq], xd[:, hq:hq + hkv]        # slices of one tensor
    amplitude = 1.0 if n % 2 else 1.25
    kw = {"layout": layout, "amplitude": amplitude}
    qo, ko = api.iq_rotate_positions(q, k, sv.dev(pos), freqs.to(sv.DEV), **kw)
    for got, part in ((qo, x[:, :hq]), (ko, x[:, hq:hq + hkv])):
        want = pf.rope(part.double().numpy(), pos, freqs.numpy(), layout, amplitude)
        err = np.abs(got.cpu().double().numpy() - want).max()
        assert got.dtype == dtype and err <= rope_tolerance(want, dtype, amplitude), err
        assert torch.equal(got[..., m:].cpu(), part[..., m:])
    # in place on the slices: the same, and the rest as it was
    api.iq_rotate_positions(q, k, sv.dev(pos), freqs.to(sv.DEV), q_out=q, k_out=k, **kw)
    assert torch.equal(xd[:, :hq], qo) and torch.equal(xd[:, hq:hq + hkv], ko)
    assert torch.equal(xd[:, hq + hkv:].cpu(), x[:, hq + hkv:])
    # one of the two alone, contiguous
    only, none = api.iq_rotate_positions(x[:, :hq].contiguous().to(sv.DEV), None, sv.dev(pos),
                                         freqs.to(sv.DEV), **kw)
    assert none is None and torch.equal(only, qo)


def test_rotate_nonfinite():
    """A NaN or infinity stays in its pair."""
    x = torch.randn(2, 2, 128, dtype=torch.float32)
    x[0, 1, 5] = float("nan")
    x[1, 0, 70] = float("inf")
    pos = np.array([3, 4], np.int32)
    f = api.iq_rope_frequencies(128).to(sv.DEV)
    got, _ = api.iq_rotate_positions(x.to(sv.DEV), None, sv.dev(pos), f)
    bad = ~torch.isfinite(got.cpu())
    want = torch.zeros_like(bad)
    want[0, 1, [5, 69]] = True
    want[1, 0, [6, 70]] = True
    assert torch.equal(bad, want)


# ---- compression into slots -----------------------------------------------------------------
@pytest.mark.parametrize("n,hkv,page,dtype", [
    (1, 1, 16, torch.float16), (3, 4, 16, torch.float32), (64, 8, 64, torch.float16),
    (129, 2, 32, torch.float32), (700, 3, 16, torch.float16)])
@pytest.mark.parametrize("sides", ["kv", "k", "v"])
def test_compress_slots(n, hkv, page, dtype, sides):
    """Records bit by bit those of the bulk compression of the same vectors."""
    rng = np.random.default_rng([n, hkv, page])
    n_pages = -(-n // page) + 3
    slots = rng.permutation(n_pages * page)[:n].astype(np.int64)
    if n > 2:
        slots[n // 2] = -1
        slots[n - 1] = n_pages * page
    x = torch.from_numpy(rng.standard_normal((n, 2 * hkv + 1, D)) * np.exp(
        rng.standard_normal((n, 2 * hkv + 1, 1)))).to(dtype).to(sv.DEV)
    k, v = x[:, :hkv], x[:, hkv:2 * hkv]
    if n > 8:
        k[3] = 0
    quats = sv.dev(sv.rotation(5, hkv))
    pool = {}
    for s in "kv":
        pool[s + "_codes"] = torch.full((n_pages, hkv, page, 48), 171, dtype=torch.uint8,
                                        device=sv.DEV)
        pool[s + "_norms"] = torch.full((n_pages, hkv, page), -7.0, device=sv.DEV)
    want = {s: a.clone() for s, a in pool.items()}
    cache = api.alloc_cache(1, hkv, -(-n // 16) * 16, sv.DEV)
    api.iq_compress_kv(k.transpose(0, 1).contiguous()[None], v.transpose(0, 1).contiguous()[None],
                       quats, cache["k_codes"], cache["k_norms"], cache["v_codes"],
                       cache["v_norms"])
    keep = torch.from_numpy((slots >= 0) & (slots < n_pages * page)).to(sv.DEV)
    at = sv.dev(slots)[keep]
    for s in sides:
        for part in ("_codes", "_norms"):
            src = cache[s + part][0].transpose(0, 1)[:n][keep]
            want[s + part][at // page, :, at % page] = src
    api.iq_compress_kv_slots(k if "k" in sides else None, v if "v" in sides else None, quats, pool,
                             sv.dev(slots))
    for s in pool:
        assert torch.equal(pool[s], want[s]), s


# ---- attention --------------------------------------------------------------------------------
def attention_case(rng, seqs, hq, hkv, page, dtype, pad=0, norm=1.0):
    lens = np.array([t for _, t in seqs], np.int32)
    starts = np.concatenate(([0], np.cumsum([x for x, _ in seqs]))).astype(np.int32)
    rows = sv.records(rng, (len(seqs), hkv, max(1, int(lens.max()))))
    width = -(-int(lens.max()) // page) + 1
    pool, tables = sv.to_pool(rng, rows, lens, page, width)
    quats = sv.rotation(11, hkv)
    q = torch.from_numpy(rng.standard_normal((int(starts[-1]) + pad, hq, D)) * norm).to(dtype)
    return rows, lens, starts, pool, tables, quats, q


SEQS = [
    [(1, 1)], [(1, 33)], [(5, 5)], [(3, 100), (1, 64), (0, 50), (7, 7)],
    [(40, 300)], [(64, 64), (33, 97)], [(130, 130), (1, 500), (17, 1000)],
    [(200, 777), (1, 1), (300, 300)], [(2, 2), (0, 0), (3, 0)], [(9, 4), (5, 40)]]


@pytest.mark.parametrize("seqs", SEQS, ids=[str(i) for i in range(len(SEQS))])
@pytest.mark.parametrize("hq,hkv,page", [(16, 2, 16), (4, 4, 64), (5, 1, 32)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_attention(seqs, hq, hkv, page, dtype):
    rng = np.random.default_rng([hq, page, seqs[0][1]])
    pad = hq % 3
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, hq, hkv, page, dtype, pad)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, hkv)
    out = torch.full(q.shape, 9.0, dtype=dtype, device=sv.DEV)
    api.iq_prefill_attention_paged(q.to(sv.DEV), sv.as_dict(pool), sv.dev(tables), sv.dev(starts),
                                   sv.dev(lens), sv.dev(quats), out=out)
    n = int(starts[-1])
    pf.check_attention(out[:n], tuple(x[:n] for x in want), dtype, f"{seqs} {hq}/{hkv}")
    assert torch.all(out[n:] == 9.0), "padding was written"


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 2), (32, 0), (100, 40), (64, 33), (5000, 3)])
@pytest.mark.parametrize("seqs", [[(70, 300), (1, 90)], [(150, 150)], [(12, 700)]],
                         ids=["a", "b", "c"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_attention_window(window, sinks, seqs, dtype):
    rng = np.random.default_rng([window, sinks])
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 8, 2, 16, dtype)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2, window, sinks)
    out = api.iq_prefill_attention_paged(q.to(sv.DEV), sv.as_dict(pool), sv.dev(tables),
                                         sv.dev(starts), sv.dev(lens), sv.dev(quats),
                                         window=window, n_sinks=sinks)
    pf.check_attention(out, want, dtype, f"window {window} {sinks} {seqs}")


@pytest.mark.parametrize("tokens", [1, 3, 4])
def test_attention_as_decode(tokens):
    """Chunks of a few tokens against the multi-token decode of the same pools."""
    rng = np.random.default_rng(tokens)
    seqs = [(tokens, 900), (tokens, 100), (tokens, 4000)]
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 16, 2, 32, torch.float32)
    p = sv.as_dict(pool)
    want = api.iq_decode_attention_multi_paged(q.to(sv.DEV).view(3, tokens, 16, D), p,
                                               sv.dev(tables), sv.dev(lens), sv.dev(quats))
    got = api.iq_prefill_attention_paged(q.to(sv.DEV), p, sv.dev(tables), sv.dev(starts),
                                         sv.dev(lens), sv.dev(quats))
    # (both are within 4e-6 of the exact result, in the 2-norm)
    rel = (got - want.view(got.shape)).norm() / want.norm()
    assert float(rel) <= 8e-6
