"""CPU tests of the largest sizes of the operators of prompts in chunks, on both sides of each
documented limit (with addresses that are never read; what is within the limits is refused for
something else before a launch)."""

import pytest

from paper_2608_08081_amd import api
from tests.test_prefill_abi import ARG, L, PREFILL, ROTATE, SLOTS, SMALL, UNSUP


def pieces(batch, n, hq, hkv):
    """P of the header."""
    rows = n * (hq // hkv)
    block = next((r for r in (32, 64, 128) if r >= rows // batch), 256)
    return rows // block + min(batch, n) + 2 * max(1, (256 if block == 256 else 512) // hkv)


# (batch, n_tokens, query heads, KV heads), within the limits or not; of pieces for instance
# (968 + 1000 + 2) 2047 < 2^22, (65536 + 65535 + 16) 62 and (4000 + 4000 + 2) 960 above
ATTENTION = [
    (4096, 1, 2047, 2047, True), (4096, 1, 2048, 2048, False), (1, 1, 2048, 2048, False),
    (8192, 1, 1023, 1023, True), (8192, 1, 1024, 1024, False), (65535, 1, 128, 128, True),
    (65535, 1, 129, 129, False),
    (65535, 65535, 62, 62, True), (65535, 65535, 63, 63, False), (65535, 65535, 64, 64, False),
    (1000, 31000, 2117, 2117, False), (1000, 31000, 2047, 2047, True), (2, 60000, 2047, 2047, True),
    (2, 1 << 27, 1, 1, True), (2, 1 << 26, 2, 1, True), (2, 1 << 26, 2, 2, True),
    (2, (1 << 27) + 1, 1, 1, False), (4000, 1 << 22, 32, 32, True), (65535, 1 << 21, 62, 62, False),
    (65535, 1 << 21, 64, 64, False), (4000, 128000, 960, 960, False)]


@pytest.mark.parametrize("batch,n,hq,hkv,within", ATTENTION)
def test_attention_limits(batch, n, hq, hkv, within):
    said = (n * hq <= 1 << 27 and hkv * max(batch, 4096) < 1 << 23 and
            hkv * pieces(batch, n, hq, hkv) < 1 << 22)
    assert said == within
    kw = dict(batch=batch, n=n, hq=hq, hkv=hkv, qs=128 * hq, os=128 * hq, nbytes=4096,
              q=ctypes_at(1), out=ctypes_at(60))
    got = L.iq_prefill_attention_paged(*dict(PREFILL, **kw).values())
    assert got == (SMALL if within else UNSUP)
    assert (api.iq_prefill_workspace_bytes(batch, n, hq, hkv, 64) > 0) == within


def ctypes_at(i):
    """Addresses far enough apart for the largest arrays."""
    return type(PREFILL["q"])(i << 56)


@pytest.mark.parametrize("n,heads,want", [
    (1 << 24, 63, ARG), (1 << 24, 64, UNSUP), ((1 << 24) + 1, 1, UNSUP), (128, 65535, ARG),
    (128 * 128, 65535, ARG), (128 * 128 + 1, 65535, UNSUP), (129 * 128, 65535, UNSUP),
    (128, 65536, UNSUP), ((1 << 24) - 127, 64, UNSUP), ((1 << 24) - 128, 64, ARG)])
def test_compression_limits(n, heads, want):
    """(Without keys and values: ARG within the limits.)"""
    kw = dict(n=n, hkv=heads, k=None, v=None)
    assert L.iq_compress_kv_slots(*dict(SLOTS, **kw).values()) == want


@pytest.mark.parametrize("n,heads,want", [(1 << 24, 16, ARG), ((1 << 24) + 1, 16, UNSUP),
                                          (9, 65535, ARG), (9, 65536, ARG)])
def test_rotation_limits(n, heads, want):
    kw = dict(n=n, hq=heads, qs=heads * 128, qos=heads * 128, k=None, ko=None, pos=None)
    assert L.iq_rotate_positions(*dict(ROTATE, **kw).values()) == want
