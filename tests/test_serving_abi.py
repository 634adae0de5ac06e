"""CPU tests of the serving operators' entry points: refusals before any launch
(with addresses that are never read), workspace sizes, mask words, the oracle
against the oracle of the operators that were there, and the kernels' resources."""

import ctypes
import re

import numpy as np
import pytest
import torch

from oracle import attention as oatt
from oracle import serving as osv
from paper_2608_08081_amd import _lib, api
from tests import serving as sv
from tests.test_kernel_resources import _device_asm, _kernels

L = _lib.lib()
P = ctypes.c_void_p


def at(i, off=0):
    """Distinct, aligned addresses."""
    return P((i + 1 << 32) + off)


WINDOW = dict(q=at(0), kc=at(1), kn=at(2), vc=at(3), vn=at(4), lens=at(5), cap=64, most=64, window=8,
              sinks=2, quats=at(6), batch=2, hq=16, hkv=2, hd=128, scale=0.0, out=at(7), ws=at(8),
              nbytes=1 << 30, bits=3, stream=None)


def window(**kw):
    a = dict(WINDOW, **kw)
    return L.iq_decode_attention_window(*a.values())


def window_step(**kw):
    a = dict(WINDOW, k=at(9), v=at(10), dtype=1, status=None)
    a.update(kw)
    return L.iq_decode_step_window(a["q"], a["k"], a["v"], a["dtype"], *[a[n] for n in list(WINDOW)[1:19]],
                                   a["status"], a["bits"], a["stream"])


@pytest.mark.parametrize("kw,want", [
    (dict(window=0), 1), (dict(window=-1), 1), (dict(sinks=-1), 1), (dict(hd=64), 2),
    (dict(bits=5), 2), (dict(hq=15), 1), (dict(hq=34), 2), (dict(cap=60, most=60), 2),
    (dict(most=65), 1), (dict(most=-1), 1), (dict(batch=-1), 1), (dict(q=None), 1),
    (dict(kn=at(2, 4)), 2), (dict(kc=at(1, 8)), 1), (dict(ws=at(8, 128)), 1), (dict(nbytes=64), 3),
    (dict(batch=0), 0), (dict(batch=70000), 2)])
def test_window_refusals(kw, want):
    assert window(**kw) == want
    if kw.get("batch") != 0:
        assert window_step(**kw) == want


def test_window_step_refusals():
    assert window_step(k=None) == 1
    assert window_step(v=at(10, 8)) == 1
    assert window_step(dtype=3) == 2
    assert window_step(status=at(11, 2)) == 1
    assert window_step(most=0) == 1
    assert window_step(batch=0) == 0


PAGED = dict(q=at(0), kc=at(1), kn=at(2), vc=at(3), vn=at(4), page=16, n_pages=9, tables=at(11),
             max_pages=4, lens=at(5), most=64, window=8, sinks=2, quats=at(6), batch=2, hq=16, hkv=2,
             hd=128, scale=0.0, out=at(7), ws=at(8), nbytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(window=0), 1), (dict(sinks=-2), 1), (dict(page=24), 1), (dict(page=8), 1),
    (dict(n_pages=0), 1), (dict(tables=None), 1), (dict(max_pages=0), 1), (dict(most=65), 1),
    (dict(hq=34), 2), (dict(nbytes=8), 3), (dict(batch=0), 0)])
def test_window_paged_refusals(kw, want):
    assert L.iq_decode_attention_window_paged(*dict(PAGED, **kw).values()) == want


TREE = dict(q=at(0), kc=at(1), kn=at(2), vc=at(3), vn=at(4), lens=at(5), cap=50, most=50, dkc=at(12),
            dkn=at(13), dvc=at(14), dvn=at(15), dcap=8, mask=at(16), window=0, sinks=0, quats=at(6),
            batch=2, t=8, hq=16, hkv=2, hd=128, scale=0.0, out=at(7), ws=at(8), nbytes=1 << 30,
            bits=3, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(t=0), 1), (dict(t=65, dcap=65), 2), (dict(dcap=7), 1), (dict(window=-1), 1),
    (dict(sinks=-1), 1), (dict(hq=17), 1), (dict(hq=34), 2), (dict(hkv=0), 1), (dict(hd=96), 2),
    (dict(bits=1), 2), (dict(most=51), 1), (dict(mask=None), 1), (dict(mask=at(16, 4)), 1),
    (dict(dkc=None), 1), (dict(dvn=at(15, 2)), 1), (dict(out=at(7, 4)), 1), (dict(ws=None), 1),
    (dict(nbytes=100), 3), (dict(batch=-2), 1), (dict(batch=0), 0),
    (dict(cap=2 ** 31 - 1, most=2 ** 31 - 1), 1), (dict(batch=2 ** 23, hq=256, hkv=16), 2)])
def test_tree_refusals(kw, want):
    assert L.iq_decode_attention_tree(*dict(TREE, **kw).values()) == want


TREE_PAGED = dict(q=at(0), kc=at(1), kn=at(2), vc=at(3), vn=at(4), page=16, n_pages=9, tables=at(11),
                  max_pages=4, lens=at(5), most=64, dkc=at(12), dkn=at(13), dvc=at(14), dvn=at(15),
                  dcap=8, mask=at(16), window=0, sinks=0, quats=at(6), batch=2, t=8, hq=16, hkv=2,
                  hd=128, scale=0.0, out=at(7), ws=at(8), nbytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(page=17), 1), (dict(hkv=0), 1), (dict(most=65), 1), (dict(tables=None), 1),
    (dict(tables=at(11, 2)), 1), (dict(t=65, dcap=99), 2), (dict(dvc=None), 1), (dict(batch=0), 0)])
def test_tree_paged_refusals(kw, want):
    assert L.iq_decode_attention_tree_paged(*dict(TREE_PAGED, **kw).values()) == want


ACCEPT = dict(dkc=at(12), dkn=at(13), dvc=at(14), dvn=at(15), dcap=8, path=at(16), most=8,
              n=at(17), kc=at(1), kn=at(2), vc=at(3), vn=at(4), cap=50, lens=at(5), out=at(5),
              batch=2, hkv=2, hd=128, status=None, bits=3, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(hd=64), 2), (dict(bits=6), 2), (dict(most=65), 2), (dict(most=-1), 1), (dict(dcap=-1), 1),
    (dict(hkv=0), 1), (dict(path=None), 1), (dict(n=at(17, 1)), 1), (dict(dkc=at(12, 4)), 1),
    (dict(kn=None), 1), (dict(out=None), 1), (dict(status=at(18, 3)), 1), (dict(batch=0), 0)])
def test_accept_refusals(kw, want):
    assert L.iq_accept_tree(*dict(ACCEPT, **kw).values()) == want


FORK = dict(kc=at(1), kn=at(2), vc=at(3), vn=at(4), page=16, n_pages=9, hkv=2, hd=128, tables=at(5),
            lens=at(6), batch=2, max_pages=4, parents=at(7), rows=3, reserve=0, refs=at(8),
            out=at(9), out_lens=at(10), out_refs=at(8), ws=at(11), nbytes=1 << 30, status=None,
            stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(hd=64), 2), (dict(page=12), 1), (dict(batch=0), 1), (dict(rows=0), 1),
    (dict(reserve=-1), 1), (dict(out=at(5)), 1), (dict(out=at(5, 16)), 1),
    (dict(out_lens=at(6, 4)), 1), (dict(out_refs=at(8, 4)), 1), (dict(parents=None), 1),
    (dict(kn=at(2, 4)), 1), (dict(refs=None), 1), (dict(nbytes=1000), 3), (dict(ws=at(11, 8)), 1),
    (dict(n_pages=2 ** 30 + 1), 2)])
def test_fork_refusals(kw, want):
    assert L.iq_fork_pages(*dict(FORK, **kw).values()) == want


COMPACT = dict(kc=at(1), kn=at(2), vc=at(3), vn=at(4), page=16, n_pages=9, hkv=2, hd=128, tables=at(5),
               batch=2, max_pages=4, refs=at(8), out=at(5), out_refs=at(8), map=at(9), live=at(10),
               ws=at(11), nbytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(hd=64), 2), (dict(page=0), 1), (dict(batch=0), 1), (dict(out=at(5, 4)), 1),
    (dict(out_refs=at(8, 32)), 1), (dict(map=at(8)), 1), (dict(map=None), 1), (dict(live=None), 1),
    (dict(nbytes=0), 3), (dict(vn=None), 1)])
def test_compact_refusals(kw, want):
    assert L.iq_compact_pages(*dict(COMPACT, **kw).values()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(batch=65536), 2), (dict(path=None, most=0), 0), (dict(dkc=at(1)), 1),
    (dict(dvc=at(1, 16)), 1), (dict(dkn=at(4)), 1), (dict(dvn=at(2, 4)), 1)])
def test_accept_overlaps_and_sizes(kw, want):
    """(one that nothing refuses has no sequences: nothing is launched)"""
    batch = {} if want else {"batch": 0}
    assert L.iq_accept_tree(*dict(ACCEPT, **kw, **batch).values()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(batch=65536), 2), (dict(rows=65536), 2), (dict(out_lens=at(7)), 1),
    (dict(out=at(7)), 1), (dict(out=at(8)), 1), (dict(out_refs=at(5)), 1), (dict(out_refs=at(9)), 1),
    (dict(out_lens=at(9, 32)), 1)])
def test_fork_overlaps_and_sizes(kw, want):
    assert L.iq_fork_pages(*dict(FORK, **kw).values()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(batch=65536), 2), (dict(out=at(8)), 1), (dict(map=at(5)), 1), (dict(live=at(8)), 1),
    (dict(live=at(9, 4)), 1), (dict(out_refs=at(5)), 1)])
def test_compact_overlaps_and_sizes(kw, want):
    assert L.iq_compact_pages(*dict(COMPACT, **kw).values()) == want


def test_tree_batch_limit():
    assert L.iq_decode_attention_tree(*dict(TREE, batch=65536, t=1).values()) == 2
    assert api.iq_decode_tree_workspace_bytes(65536, 1, 16, 2, 1000) == 0
    assert api.iq_pages_workspace_bytes(9, 65536) == 0


def test_workspace_sizes():
    w = api.iq_decode_window_workspace_bytes
    assert w(2, 16, 2, 1024, 64, 4) > 0 and w(0, 16, 2, 1024, 64) >= 0
    assert w(2, 16, 2, 1024, 0) == 0 and w(2, 16, 3, 1024, 8) == 0 and w(2, 16, 2, 1024, 8, -1) == 0
    assert w(1, 32, 4, 32768, 1 << 62, 1 << 62) == w(1, 32, 4, 32768, 32768, 32768)
    t = api.iq_decode_tree_workspace_bytes
    assert t(2, 8, 16, 2, 1000) > 0 and t(2, 65, 16, 2, 1000) == 0 and t(2, 0, 16, 2, 1000) == 0
    assert t(2, 8, 34, 2, 1000) == 0 and t(2, 8, 16, 2, 1000, -1) == 0
    assert t(1, 64, 32, 4, 32768, 1 << 62, 1 << 62) > 0
    p = api.iq_pages_workspace_bytes
    assert p(1, 1) > 0 and p(0, 1) == 0 and p(1 << 31, 1) == 0 and p(5, -1) == 0


def test_tree_mask():
    m = api.tree_mask([[-1, 0, 0, 1, 3, -2], [-1, -1, 1, 2, 3, 4]])
    assert m.dtype == torch.int64 and m.tolist() == [[1, 3, 5, 11, 27, 0], [1, 2, 6, 14, 30, 62]]
    chain = api.tree_mask(np.arange(-1, 63))
    assert chain[63].item() == -1 and chain[62].item() == 2 ** 63 - 1
    for bad in ([0], [-1, 1], [-1, 2, 0], [-3], [-1, -2, 1], [], np.zeros(65, int) - 1):
        with pytest.raises(ValueError):
            api.tree_mask(bad)


def test_python_refusals():
    """Tensors on the host are refused by every entry point."""
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: z(*s, dt=torch.int32)  # noqa: E731
    cache = {"k_codes": z(1, 1, 16, 48, dt=torch.uint8), "k_norms": z(1, 1, 16),
             "v_codes": z(1, 1, 16, 48, dt=torch.uint8), "v_norms": z(1, 1, 16)}
    rows = list(cache.values())
    quats, q = z(1, 32, 2, 4), z(1, 8, 128)
    calls = [
        lambda: api.iq_decode_attention_window(q, *rows, i(1), quats, 4),
        lambda: api.iq_decode_attention_window_paged(q, cache, i(1, 1), i(1), quats, 4),
        lambda: api.iq_decode_step_window(q, z(1, 1, 128), z(1, 1, 128), *rows, i(1), quats, 4),
        lambda: api.iq_decode_step_window_paged(q, z(1, 1, 128), z(1, 1, 128), cache, i(1, 1), i(1),
                                                quats, 4),
        lambda: api.iq_decode_attention_tree(q.unsqueeze(1), *rows, i(1), cache,
                                             z(1, 1, dt=torch.int64), quats),
        lambda: api.iq_decode_attention_tree_paged(q.unsqueeze(1), cache, i(1, 1), i(1), cache,
                                                   z(1, 1, dt=torch.int64), quats),
        lambda: api.iq_accept_tree(cache, i(1, 4), i(1), *rows, i(1)),
        lambda: api.iq_accept_tree_paged(cache, i(1, 4), i(1), cache, i(1, 1), i(1)),
        lambda: api.iq_fork_pages(cache, i(1, 1), i(1), i(1), i(1)),
        lambda: api.iq_compact_pages(cache, i(1, 1), i(1)),
    ]
    for call in calls:
        with pytest.raises(ValueError, match="device tensor"):
            call()
    del cache["v_norms"]
    for call in calls[4:]:
        with pytest.raises(ValueError, match="v_norms|device tensor"):
            call()


def test_oracle_agrees_with_what_was_there():
    rng = np.random.default_rng(0)
    rows = sv.records(rng, (2, 2, 40))
    quats, q = sv.rotation(3, 2), rng.standard_normal((2, 4, 6, 128))
    lv = sv.levels(3)
    lens = [40, 17]
    full, _, _ = osv.decode_window(q[:, 0], *rows, lens, quats, lv, 100, 0)
    assert np.allclose(full, oatt.decode_fused(q[:, 0], *rows, lens, quats, lv), atol=1e-12)
    one, _, _ = osv.decode_window(q[:, 0], *rows, lens, quats, lv, 5, 0)
    cut = [np.stack([a[b, :, n - 5:n] for b, n in enumerate(lens)]) for a in rows]
    assert np.allclose(one, oatt.decode_fused(q[:, 0], *cut, [5, 5], quats, lv), atol=1e-12)
    draft = [np.stack([a[b, :, n - 4:n] for b, n in enumerate(lens)]) for a in rows]
    chain = api.tree_mask([[-1, 0, 1, 2]] * 2).numpy()
    tree, _, _ = osv.decode_tree(q, *rows, [36, 13], *draft, chain, quats, lv)
    assert np.allclose(tree, oatt.decode_multi(q, *rows, lens, quats, lv), atol=1e-12)


def test_kernel_resources(tmp_path):
    """No scratch; eight waves on a CU at least."""
    ks = _kernels(_device_asm("iq_decode_window.hip", tmp_path))
    win = {n: v for n, v in ks.items() if "decode_window_kernel" in n}
    assert len(win) == 12
    for name, (vg, lds, priv) in win.items():
        assert priv == 0 and vg <= 128 and 2 * lds <= 160 * 1024, (name, vg, lds, priv)
    ks = _kernels(_device_asm("iq_decode_tree.hip", tmp_path))
    tree = {n: v for n, v in ks.items() if re.search("11tree_kernel", n)}
    assert len(tree) == 16
    for name, (vg, lds, priv) in tree.items():
        per_cu = 1 if "kernelILi8E" in name else 2   # (of eight waves, and of four)
        assert priv == 0 and vg <= 256 and per_cu * lds <= 160 * 1024, (name, vg, lds, priv)
    for name, (vg, lds, priv) in _kernels(_device_asm("iq_pages.hip", tmp_path)).items():
        assert priv == 0 and vg <= 64, (name, vg, priv)
