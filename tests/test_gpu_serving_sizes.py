"""One workspace, sized for the largest call, serves the smaller ones: the same
results bit for bit as with a workspace of their own, nothing written behind it."""

import numpy as np
import pytest
import torch

from paper_2608_08081_amd import api
from tests import serving as sv

pytestmark = pytest.mark.gpu

GUARD = 4096


def guarded(nbytes):
    buf = torch.full((nbytes + GUARD,), 0xA5, dtype=torch.uint8, device=sv.DEV)
    return buf, buf[:nbytes]


def cut(rows, b):
    return [a[:b].contiguous() for a in rows]


def test_tree():
    rng = np.random.default_rng(31)
    b, hkv, group, cap, t = 5, 1, 8, 16384, 33
    hq = hkv * group
    rows = [sv.dev(a) for a in sv.records(rng, (b, hkv, cap))]
    draft = [sv.dev(a) for a in sv.records(rng, (b, hkv, t))]
    quats = sv.dev(sv.rotation(1, hkv))
    q = sv.dev(rng.standard_normal((b, t, hq, sv.D)).astype(np.float32))
    lens = sv.dev(rng.integers(cap // 2, cap + 1, b).astype(np.int32))
    words = sv.dev(np.tile((1 << np.arange(1, t + 1)) - 1, (b, 1)))
    buf, ws = guarded(api.iq_decode_tree_workspace_bytes(b, t, hq, hkv, cap))
    for nb, nt, window, most in ((5, 33, 0, None), (1, 16, 0, None), (1, 17, 0, None),
                                 (1, 32, 0, None), (4, 8, 0, 1000), (3, 4, 100, None),
                                 (5, 1, 0, None), (2, 24, 500, 1500)):
        print(f"[sizes] tree batch={nb} nodes={nt} window={window}", flush=True)
        args = (q[:nb, :nt].contiguous(), *cut(rows, nb), lens[:nb],
                dict(zip(sv.NAMES, cut(draft, nb))), words[:nb, :nt].contiguous(), quats)
        kw = {"window": window, "n_sinks": 4 if window else 0, "max_seq_len": most}
        got = api.iq_decode_attention_tree(*args, workspace=ws, **kw)
        assert torch.equal(got, api.iq_decode_attention_tree(*args, **kw))
        assert (buf[len(ws):] == 0xA5).all()


def test_window():
    rng = np.random.default_rng(32)
    b, hkv, group, cap = 130, 2, 8, 1024
    hq = hkv * group
    rows = [sv.dev(a) for a in sv.records(rng, (b, hkv, cap))]
    quats = sv.dev(sv.rotation(2, hkv))
    q = sv.dev(rng.standard_normal((b, hq, sv.D)).astype(np.float32))
    lens = sv.dev(rng.integers(0, cap + 1, b).astype(np.int32))
    buf, ws = guarded(api.iq_decode_window_workspace_bytes(b, hq, hkv, cap, 600, 16))
    for nb, window, sinks in ((130, 600, 16), (128, 600, 16), (129, 500, 0), (85, 600, 4),
                              (64, 600, 16), (3, 600, 16), (1, 17, 1)):
        print(f"[sizes] window batch={nb} window={window}", flush=True)
        args = (q[:nb].contiguous(), *cut(rows, nb), lens[:nb], quats, window, sinks)
        got = api.iq_decode_attention_window(*args, workspace=ws)
        assert torch.equal(got, api.iq_decode_attention_window(*args))
        assert (buf[len(ws):] == 0xA5).all()
