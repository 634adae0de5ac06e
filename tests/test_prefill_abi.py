"""CPU tests of the entry points of prompts in chunks: refusals before any launch (with addresses
that are never read), workspace sizes, rotary frequencies against their formulas, the binding's
native checks, and the kernels' resources."""

import ctypes
import itertools
import math

import numpy as np
import pytest
import torch

from paper_2608_08081_amd import _lib, api
from tests import prefill as pf
from tests.test_kernel_resources import LDS_PER_CU, _device_asm, _kernels
from tests.test_serving_sizes import grows

L = _lib.lib()
P = ctypes.c_void_p
OK, ARG, UNSUP, SMALL = 0, 1, 2, 3


def at(i, off=0):
    """Distinct, aligned addresses."""
    return P((i + 1 << 40) + off)


# ---- refusals -----------------------------------------------------------------------------------
EXTEND = dict(page=16, n_pages=100, tables=at(0), lens=at(1), more=at(2), batch=3, max_pages=5,
              refs=at(3), n=50, out_tables=at(4), out_lens=at(5), out_refs=at(6), starts=at(7),
              slots=at(8), positions=at(9), ws=at(10), nbytes=1 << 30, status=at(11), stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(page=24), ARG), (dict(page=8), ARG), (dict(n_pages=0), ARG), (dict(tables=None), ARG),
    (dict(max_pages=0), ARG), (dict(batch=0), ARG), (dict(batch=-1), ARG), (dict(n=-1), ARG),
    (dict(n=1 << 31), ARG), (dict(batch=65536), UNSUP), (dict(lens=None), ARG),
    (dict(more=at(2, 2)), ARG), (dict(refs=None), ARG), (dict(out_tables=None), ARG),
    (dict(out_lens=at(5, 1)), ARG), (dict(out_refs=None), ARG), (dict(starts=None), ARG),
    (dict(slots=None), ARG), (dict(slots=at(8, 4)), ARG), (dict(positions=at(9, 2)), ARG),
    (dict(status=at(11, 2)), ARG), (dict(ws=None), ARG), (dict(ws=at(10, 64)), ARG),
    (dict(nbytes=64), SMALL), (dict(n_pages=(1 << 30) + 1), UNSUP),
    # memory in common: outputs with each other and with inputs of another kind
    (dict(out_lens=at(2)), ARG), (dict(out_lens=at(0, 56)), ARG), (dict(out_tables=at(1)), ARG),
    (dict(out_tables=at(0, 4)), ARG), (dict(out_refs=at(3, 396)), ARG), (dict(starts=at(2, -12)), ARG),
    (dict(starts=at(5, 8)), ARG), (dict(slots=at(9, 192)), ARG), (dict(positions=at(8, 396)), ARG),
    (dict(status=at(1, 8)), ARG), (dict(ws=at(3)), ARG), (dict(slots=at(10, 256)), ARG),
    (dict(out_refs=at(6), out_lens=at(6, 396)), ARG)])
def test_extend_refusals(kw, want):
    assert L.iq_extend_pages(*dict(EXTEND, **kw).values()) == want


ROTATE = dict(q=at(0), qs=2048, qo=at(1), qos=2048, hq=16, k=at(2), ks=256, ko=at(3), kos=256, hkv=2,
              dtype=1, n=9, hd=128, pos=at(4), freqs=at(5), m=128, layout=0, amp=1.0, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), UNSUP), (dict(layout=2), UNSUP), (dict(layout=-1), UNSUP), (dict(hd=96), UNSUP),
    (dict(m=8), UNSUP), (dict(m=24), UNSUP), (dict(m=144), UNSUP), (dict(hd=64, m=80), UNSUP),
    (dict(n=-1), ARG), (dict(n=(1 << 24) + 1), UNSUP), (dict(q=None), ARG), (dict(qo=None), ARG),
    (dict(k=None), ARG), (dict(ko=None), ARG), (dict(q=None, qo=None, k=None, ko=None), ARG),
    (dict(hq=0), ARG), (dict(hkv=-1), ARG), (dict(hq=70000, qs=1 << 24, qos=1 << 24), ARG),
    (dict(qs=2040), ARG), (dict(qs=2052), ARG), (dict(kos=255), ARG), (dict(q=at(0, 8)), ARG),
    (dict(ko=at(3, 4)), ARG), (dict(pos=None), ARG), (dict(pos=at(4, 2)), ARG), (dict(freqs=None), ARG),
    (dict(freqs=at(5, 4)), ARG), (dict(qs=1 << 40), ARG),
    # memory in common
    (dict(qo=at(0, 16)), ARG), (dict(qo=at(0), qos=4096), ARG), (dict(ko=at(0)), ARG),
    (dict(ko=at(1, 4096)), ARG), (dict(qo=at(2)), ARG), (dict(qo=at(4)), ARG), (dict(ko=at(5)), ARG),
    (dict(n=0), OK)])
def test_rotate_refusals(kw, want):
    assert L.iq_rotate_positions(*dict(ROTATE, **kw).values()) == want


SLOTS = dict(k=at(0), ks=256, v=at(1), vs=256, dtype=1, n=9, hkv=2, hd=128, quats=at(2), kc=at(3),
             kn=at(4), vc=at(5), vn=at(6), page=16, n_pages=5, slots=at(7), stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=5), UNSUP), (dict(hd=64), UNSUP), (dict(n=-1), ARG), (dict(hkv=0), ARG),
    (dict(hkv=70000, ks=1 << 24, vs=1 << 24), UNSUP), (dict(n=(1 << 24) + 1), UNSUP),
    (dict(page=20), ARG), (dict(n_pages=0), ARG), (dict(k=None, v=None), ARG), (dict(kc=None), ARG),
    (dict(kn=None), ARG), (dict(vc=at(5, 8)), ARG), (dict(vn=at(6, 2)), ARG), (dict(ks=255), ARG),
    (dict(vs=260), ARG), (dict(k=at(0, 8)), ARG), (dict(quats=None), ARG), (dict(quats=at(2, 8)), ARG),
    (dict(slots=None), ARG), (dict(slots=at(7, 4)), ARG), (dict(n=0), OK)])
def test_slots_refusals(kw, want):
    assert L.iq_compress_kv_slots(*dict(SLOTS, **kw).values()) == want


PREFILL = dict(q=at(0), qs=2048, dtype=1, kc=at(1), kn=at(2), vc=at(3), vn=at(4), page=16, n_pages=9,
               tables=at(5), max_pages=4, starts=at(6), lens=at(7), n=20, most=64, window=0, sinks=0,
               quats=at(8), batch=2, hq=16, hkv=2, hd=128, scale=0.0, out=at(9), os=2048, ws=at(10),
               nbytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(hd=64), UNSUP), (dict(dtype=2), UNSUP), (dict(hkv=0), ARG), (dict(window=-1), ARG),
    (dict(sinks=-1), ARG), (dict(page=12), ARG), (dict(n_pages=0), ARG), (dict(tables=None), ARG),
    (dict(max_pages=0), ARG), (dict(batch=-1), ARG), (dict(n=-1), ARG), (dict(hq=0), ARG),
    (dict(hq=17), ARG), (dict(hq=34), UNSUP), (dict(batch=65536), UNSUP), (dict(most=-1), ARG),
    (dict(most=65), ARG), (dict(n=1 << 24, batch=3), UNSUP), (dict(q=None), ARG), (dict(out=None), ARG),
    (dict(q=at(0, 8)), ARG), (dict(qs=2047), ARG), (dict(os=2052), ARG), (dict(kc=None), ARG),
    (dict(kn=at(2, 4)), ARG), (dict(vc=at(3, 8)), ARG), (dict(vn=None), ARG), (dict(quats=None), ARG),
    (dict(starts=None), ARG), (dict(lens=at(7, 2)), ARG), (dict(starts=at(6, 1)), ARG),
    (dict(ws=None), ARG), (dict(ws=at(10, 128)), ARG), (dict(nbytes=4096), SMALL),
    (dict(out=at(0)), ARG), (dict(out=at(0, 19 * 4096)), ARG), (dict(batch=0), OK), (dict(n=0), OK)])
def test_prefill_refusals(kw, want):
    assert L.iq_prefill_attention_paged(*dict(PREFILL, **kw).values()) == want


def test_rows_between_rows():
    """Outputs may lie between the rows of an input of the same stride, not on them."""
    def call(off, **kw):
        a = dict(PREFILL, qs=8192, os=8192, out=at(0, off), nbytes=0)
        return L.iq_prefill_attention_paged(*dict(a, **kw).values())

    assert call(4096) == SMALL and call(16384 - 4096) == SMALL and call(-4096) == SMALL
    assert call(4080) == ARG and call(16384 - 4080) == ARG and call(5 * 16384) == ARG
    assert call(4096, os=8208) == ARG


# ---- sizes --------------------------------------------------------------------------------------
def test_prefill_sizes_grow():
    size = api.iq_prefill_workspace_bytes
    batches = [1, 2, 3, 7, 31, 32, 33, 64, 255, 256, 300, 1024, 1025, 4095, 4096, 4097, 9000, 65535]
    tokens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 100, 511, 513, 4096, 100000]
    lengths = [0, 1, 31, 4096, 4097, 100000, 1 << 20]
    for hq, hkv in ((32, 4), (8, 8), (40, 8), (16, 1), (5, 1)):
        for n, t in itertools.product(lengths, tokens):
            grows([size(b, t, hq, hkv, n) for b in batches], ("batch", n, t))
        for n, b in itertools.product(lengths, batches):
            grows([size(b, t, hq, hkv, n) for t in tokens], ("tokens", n, b))
        for t, b in itertools.product(tokens, batches):
            grows([size(b, t, hq, hkv, n) for n in lengths], ("length", t, b))


def test_prefill_sizes_of_other_shapes():
    assert api.iq_prefill_workspace_bytes(1, 1, 34, 2, 64) == 0
    assert api.iq_prefill_workspace_bytes(1, 1, 17, 2, 64) == 0
    assert api.iq_prefill_workspace_bytes(65536, 1, 16, 2, 64) == 0
    assert api.iq_prefill_workspace_bytes(1, 1 << 24, 16, 2, 64) == 0
    assert L.iq_prefill_workspace_bytes(1, 1, 16, 2, 64, 64) == 0


def test_extend_sizes_grow():
    size = api.iq_extend_workspace_bytes
    rows = (0, 1, 63, 64, 65, 8192, 8193, 65535)
    pages = (1, 2, 63, 64, 2047, 2048, 2049, 140000, 5000000)
    for r in rows:
        grows([size(n, r) for n in pages], ("pages", r))
    for n in pages:
        grows([size(n, r) for r in rows], ("rows", n))
    assert size(0, 1) == size(1, -1) == size(1, 65536) == size((1 << 30) + 1, 1) == 0


# ---- frequencies ----------------------------------------------------------------------------------
@pytest.mark.parametrize("m,theta,factor", [(128, 10000.0, 1.0), (64, 5e5, 8.0), (16, 1e6, 0.5),
                                            (96, 10000.0, 32.0), (4, 100.0, 3.0)])
def test_rope_frequencies(m, theta, factor):
    """Against the formulas in Python's doubles: powers are within a few units of 2^-53, and the
    exponent's rounding moves them by ln(theta) units more."""
    def same(a, b):
        b = np.array(b)
        assert np.abs(a.numpy() - b).max() <= 64 * 2.0 ** -53 * np.abs(b).max()
        assert np.all(np.abs(a.numpy() - b) <= 64 * 2.0 ** -53 * np.abs(b))

    plain = [theta ** (-2.0 * i / m) for i in range(m // 2)]
    same(api.iq_rope_frequencies(m, theta), plain)
    same(api.iq_rope_frequencies(m, theta, "linear", factor), [f / factor for f in plain])
    base = theta * factor ** (m / (m - 2))
    got = api.iq_rope_frequencies(m, theta, "base", factor)
    same(got, [base ** (-2.0 * i / m) for i in range(m // 2)])
    assert math.isclose(float(got[-1]), plain[-1] / factor, rel_tol=1e-13)
    bands = []
    for f in plain:
        r = 2048.0 * f / (2 * math.pi)
        w = min(1.0, max(0.0, (r - 1.0) / (32.0 - 1.0)))
        bands.append(w * f + (1 - w) * f / factor)
    same(api.iq_rope_frequencies(m, theta, "bands", factor, 1.0, 32.0, 2048.0), bands)


FREQS = dict(theta=1e4, m=128, scaling=0, factor=2.0, low=1.0, high=32.0, most=4096.0)


@pytest.mark.parametrize("kw,want", [
    (dict(scaling=4), UNSUP), (dict(scaling=-1), UNSUP), (dict(m=0), ARG), (dict(m=3), ARG),
    (dict(m=(1 << 20) + 2), ARG), (dict(theta=0.0), ARG), (dict(theta=-1.0), ARG),
    (dict(theta=math.inf), ARG), (dict(theta=math.nan), ARG), (dict(scaling=1, factor=0.0), ARG),
    (dict(scaling=2, factor=math.nan), ARG), (dict(scaling=2, m=2), ARG),
    (dict(scaling=3, low=-1.0), ARG), (dict(scaling=3, low=32.0), ARG), (dict(scaling=3, low=math.nan), ARG),
    (dict(scaling=3, high=math.inf), ARG), (dict(scaling=3, most=0.0), ARG),
    (dict(factor=math.nan), OK), (dict(scaling=1, low=math.nan), OK)])
def test_rope_frequency_refusals(kw, want):
    out = np.zeros(64)
    ptr = out.ctypes.data_as(P)
    assert L.iq_rope_frequencies(*dict(FREQS, **kw).values(), ptr) == want
    assert want == OK or not out.any()
    assert L.iq_rope_frequencies(*FREQS.values(), None) == ARG


# ---- the binding ----------------------------------------------------------------------------------
def test_everything_else_goes_to_the_general_path():
    nat = _lib.native()
    t = torch.zeros(1, 16, 128)
    for fn, n in (("extend", 14), ("rotate", 8), ("compress_slots", 8), ("prefill", 15)):
        f = getattr(nat, fn)
        assert f(*[None] * n) is None
        assert f(*[t] * n) is None
        assert f(*[object()] * n) is None
        assert f() is None and f(t) is None


def test_host_tensors_are_refused():
    i = torch.zeros(2, dtype=torch.int32)
    tables, refs = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(9, dtype=torch.int32)
    with pytest.raises(ValueError):
        api.iq_extend_pages(tables, i, i, refs, 16, n_tokens=4)
    with pytest.raises(ValueError):
        api.iq_extend_pages(tables, i, i, refs, 16)               # no n_tokens, no slots
    q = torch.zeros(4, 16, 128)
    with pytest.raises(ValueError):
        api.iq_rotate_positions(q, None, torch.zeros(4, dtype=torch.int32), torch.zeros(64).double())
    with pytest.raises(ValueError):
        api.iq_rotate_positions(None, None, i, torch.zeros(64).double())
    with pytest.raises(KeyError):
        api.iq_rotate_positions(q, None, i, torch.zeros(64).double(), layout="other")
    pool = {"k_codes": torch.zeros(5, 2, 16, 48, dtype=torch.uint8), "k_norms": torch.zeros(5, 2, 16)}
    with pytest.raises(ValueError):
        api.iq_compress_kv_slots(q, None, torch.zeros(2, 32, 2, 4), pool, torch.zeros(4).long())
    with pytest.raises(ValueError):
        api.iq_compress_kv_slots(None, None, torch.zeros(2, 32, 2, 4), pool, torch.zeros(4).long())
    pool["v_codes"], pool["v_norms"] = pool["k_codes"], pool["k_norms"]
    with pytest.raises(ValueError):
        api.iq_prefill_attention_paged(q, pool, tables, torch.zeros(3, dtype=torch.int32), i,
                                       torch.zeros(2, 32, 2, 4))
    with pytest.raises(KeyError):
        api.iq_rope_frequencies(64, scaling="other")


# ---- the plain forms ------------------------------------------------------------------------------
def test_plain_extend():
    """The plain form itself, on a case by hand: pages of 16, the free ones 1, 4 and 5; the second
    sequence fills its last page, the third finds one page too few, the fourth needs none."""
    tables = np.array([[0, -1], [2, -1], [-1, -1], [3, -1]], np.int32)
    lens, new = np.array([16, 10, 0, 3], np.int32), np.array([2, 22, 20, 4], np.int32)
    refs = np.array([1, 0, 1, 1, 0, -1], np.int32)
    starts, slots, pos, t, ln, r, status = pf.extend(tables, lens, new, refs, 16, 50)
    assert starts.tolist() == [0, 2, 24, 44, 48]
    assert t.tolist() == [[0, 1], [2, 4], [-1, -1], [3, -1]] and ln.tolist() == [18, 32, 0, 7]
    assert r.tolist() == [1, 1, 1, 1, 1, -1] and status == 5
    assert slots[:3].tolist() == [16, 17, 42] and slots[7:9].tolist() == [47, 64]
    assert (slots[24:44] == -1).all() and pos[24:44].tolist() == list(range(20))
    assert slots[44:].tolist() == [51, 52, 53, 54, -1, -1] and pos[44:].tolist() == [3, 4, 5, 6, 0, 0]


# ---- resources ------------------------------------------------------------------------------------
@pytest.mark.parametrize("src,most", [("iq_extend.hip", 128), ("iq_positions.hip", 128),
                                      ("iq_prefill.hip", 256)])
def test_no_scratch(src, most, tmp_path):
    """Registers for the waves that each kernel is launched with, and no scratch."""
    ks = _kernels(_device_asm(src, tmp_path))
    assert ks
    for name, (vgprs, lds, scratch) in ks.items():
        assert vgprs <= most and lds <= LDS_PER_CU, name
        assert scratch == 0, name
