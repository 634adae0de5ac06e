"""CPU tests of the serving operators' workspace sizes: a workspace of a large
shape serves every smaller one, and covers the call's own use of it."""

import itertools

import pytest

from paper_2608_08081_amd import api

HEADS = [(32, 4), (8, 1), (40, 8), (64, 8), (16, 1), (5, 5)]
BATCHES = [1, 2, 3, 7, 8, 9, 16, 31, 64, 100, 129, 255, 256, 257, 300, 512, 700]
NODES = [1, 2, 3, 4, 5, 8, 13, 15, 16, 17, 24, 31, 32, 33, 48, 63, 64]
LENGTHS = [0, 1, 16, 31, 100, 1000, 4097, 8192, 32768]
WINDOWS = [1, 16, 33, 127, 128, 129, 1000, 4096, 10000, 32768]   # then none
SINKS = [0, 1, 4, 16, 60, 130, 5000]


def grows(sizes, label):
    assert all(a > 0 for a in sizes), label
    for (i, a), b in zip(enumerate(sizes), sizes[1:]):
        assert a <= b, (label, i, a, b)


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_tree_sizes_grow(hq, hkv):
    size = api.iq_decode_tree_workspace_bytes
    for n, t in itertools.product(LENGTHS, NODES):
        grows([size(b, t, hq, hkv, n) for b in BATCHES], ("batch", n, t))
    for n, b in itertools.product(LENGTHS, BATCHES):
        grows([size(b, t, hq, hkv, n) for t in range(1, 65)], ("nodes", n, b))
    for b, t in itertools.product(BATCHES, NODES):
        grows([size(b, t, hq, hkv, n) for n in LENGTHS], ("length", b, t))
        grows([size(b, t, hq, hkv, 32768, w, 4) for w in WINDOWS + [0]], ("window", b, t))
        grows([size(b, t, hq, hkv, 32768, 100, s) for s in SINKS], ("sinks", b, t))


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_window_sizes_grow(hq, hkv):
    size = api.iq_decode_window_workspace_bytes
    for n, w in itertools.product(LENGTHS, WINDOWS):
        grows([size(b, hq, hkv, n, w, 4) for b in range(1, 701)], ("batch", n, w))
    for b, w in itertools.product(BATCHES, WINDOWS):
        grows([size(b, hq, hkv, n, w, 4) for n in LENGTHS], ("length", b, w))
    for b, n in itertools.product(BATCHES, LENGTHS):
        grows([size(b, hq, hkv, n, w, 4) for w in WINDOWS], ("window", b, n))
        grows([size(b, hq, hkv, n, 100, s) for s in SINKS], ("sinks", b, n))


def test_page_sizes_grow():
    size = api.iq_pages_workspace_bytes
    for rows in (0, 1, 63, 64, 65, 1000, 65535):
        grows([size(n, rows) for n in (1, 2, 63, 64, 2047, 2048, 2049, 140000)], ("pages", rows))
    for n in (1, 2048, 140000):
        grows([size(n, r) for r in (0, 1, 63, 64, 65, 1000, 65535)], ("rows", n))
