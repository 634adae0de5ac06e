"""GPU tests of windowed chunks with sinks of a turn of four tiles (128 positions) and more: a token
sees the sinks up to its own position only, and nothing behind its sequence's end."""

import numpy as np
import pytest
import torch

from tests import prefill as pf
from tests.test_gpu_prefill import attention_case
from tests.test_gpu_prefill_edges import attend

pytestmark = pytest.mark.gpu

# (a sequence of 1000 makes room for sinks behind the end of the others)
SEQS = {"fresh": [(300, 300)], "pair": [(260, 260), (230, 230)], "room": [(230, 230), (300, 1000)],
        "few": [(1, 230), (2, 250), (400, 1000), (1, 100)], "short": [(100, 129), (200, 200)]}


@pytest.mark.parametrize("window,sinks", [(64, 127), (64, 128), (64, 129), (1, 256), (200, 256),
                                          (33, 300), (100, 5000)])
@pytest.mark.parametrize("seqs", list(SEQS))
@pytest.mark.parametrize("hq,hkv", [(2, 2), (16, 2)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_sinks_of_whole_turns(window, sinks, seqs, hq, hkv, dtype):
    rng = np.random.default_rng([window, sinks, hq])
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, SEQS[seqs], hq, hkv, 16, dtype)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, hkv, window, sinks)
    out = attend(q, pool, tables, starts, lens, quats, window=window, n_sinks=sinks)
    pf.check_attention(out, want, dtype, f"{seqs} {window}/{sinks}")
