"""CPU tests: acceptance, forking and compaction refuse arrays that share memory
with what they write (addresses that are never read)."""

import pytest

from tests.test_serving_abi import ACCEPT, COMPACT, FORK, L, at

# ACCEPT: path [2][8] at 16, n_accept [2] at 17, seq_lens [2] at 5


@pytest.mark.parametrize("kw", [
    dict(out=at(17)), dict(out=at(17, 4)), dict(out=at(16)), dict(out=at(16, 60)),
    dict(out=at(5, 4)), dict(lens=at(5, 4)), dict(status=at(5)), dict(status=at(5, 4)),
    dict(status=at(17)), dict(status=at(16, 8))])
def test_accept(kw):
    assert L.iq_accept_tree(*dict(ACCEPT, **kw).values()) == 1
    a = dict(ACCEPT, **kw)
    paged = dict(dkc=a["dkc"], dkn=a["dkn"], dvc=a["dvc"], dvn=a["dvn"], dcap=a["dcap"],
                 path=a["path"], most=a["most"], n=a["n"], kc=a["kc"], kn=a["kn"], vc=a["vc"],
                 vn=a["vn"], page=16, n_pages=9, tables=at(20), max_pages=4, lens=a["lens"],
                 out=a["out"], batch=2, hkv=2, hd=128, status=a["status"], stream=None)
    assert L.iq_accept_tree_paged(*paged.values()) == 1


def test_accept_page_table():
    paged = dict(dkc=at(12), dkn=at(13), dvc=at(14), dvn=at(15), dcap=8, path=at(16), most=8,
                 n=at(17), kc=at(1), kn=at(2), vc=at(3), vn=at(4), page=16, n_pages=9, tables=at(20),
                 max_pages=4, lens=at(5), out=at(5), batch=2, hkv=2, hd=128, status=None,
                 stream=None)
    for kw in (dict(out=at(20)), dict(out=at(20, 28)), dict(status=at(20, 12))):
        assert L.iq_accept_tree_paged(*dict(paged, **kw).values()) == 1


@pytest.mark.parametrize("kw", [
    dict(status=at(5)), dict(status=at(6, 4)), dict(status=at(7, 8)), dict(status=at(8, 32)),
    dict(status=at(9, 44)), dict(status=at(10)), dict(status=at(8), out_refs=at(12))])
def test_fork_status(kw):
    assert L.iq_fork_pages(*dict(FORK, **kw).values()) == 1


def test_what_may_be_shared():
    """(no sequences: nothing is launched)"""
    assert L.iq_accept_tree(*dict(ACCEPT, batch=0, out=at(5), status=at(19)).values()) == 0
    assert L.iq_accept_tree(*dict(ACCEPT, batch=0, out=at(18)).values()) == 0
    # compaction in place is checked up to the workspace's size
    assert L.iq_compact_pages(*dict(COMPACT, nbytes=0).values()) == 3
    assert L.iq_fork_pages(*dict(FORK, nbytes=0, status=at(13)).values()) == 3
