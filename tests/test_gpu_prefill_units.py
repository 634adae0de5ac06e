"""GPU tests of the unit that value scales share in chunk attention: what no row sees does not enter
it, however large, and scales near the end of fp32's range keep it finite."""

import numpy as np
import pytest
import torch

from tests import prefill as pf
from tests import serving as sv
from tests.test_gpu_prefill import attention_case
from tests.test_gpu_prefill_edges import attend

pytestmark = pytest.mark.gpu
LARGEST = float(np.finfo(np.float32).max)


def with_first_page(pool, tables, scale):
    """The pools with a page more, of index 0 and on no table, whose scales are `scale`."""
    first = [np.full((1, *a.shape[1:]), scale if a.dtype == np.float32 else 90, a.dtype) for a in pool]
    return ([np.concatenate([f, a]) for f, a in zip(first, pool)],
            np.where(tables >= 0, tables + 1, tables).astype(np.int32))


@pytest.mark.parametrize("large", [1e6, 2.0 ** 40, 1e30, LARGEST])
@pytest.mark.parametrize("window,sinks", [(100, 20), (256, 0), (33, 200)])
@pytest.mark.parametrize("seqs", [[(90, 1000)], [(9, 1000)], [(200, 5000), (1, 700), (60, 700)]],
                         ids=["many", "few", "mixed"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_large_finite_scales_in_unseen_places(dtype, seqs, window, sinks, large):
    """Scales between the sinks and the first token's window, those of page 0 behind entries outside
    the pools, and those behind the end: any finite value, the same bits."""
    rng = np.random.default_rng(31)
    rows, lens, starts, _, _, quats, q = attention_case(rng, seqs, 16, 2, 16, dtype)
    width = -(-int(lens.max()) // 16) + 1
    outs = []
    for x in (14.0, large):
        order = np.random.default_rng(32)
        given = [a.copy() for a in rows]
        for b, (n, total) in enumerate(seqs):
            lo = max(sinks, total - n - window + 1)
            for i in (1, 3):
                given[i][b, :, sinks:lo] = x
        pool, tables = sv.to_pool(order, given, lens, 16, width)
        for a in pool:
            if a.dtype == np.float32:
                a[np.isnan(a)] = x                # behind the ends, and pages on no table
        pool, tables = with_first_page(pool, tables, x)
        for b, (n, total) in enumerate(seqs):
            lo = max(sinks, total - n - window + 1)
            for k in range(-(-sinks // 16), lo // 16):        # pages without a seen position
                tables[b, k] = (-1, 1 << 30, -(1 << 31))[k % 3]
        outs.append(attend(q, pool, tables, starts, lens, quats, window=window, n_sinks=sinks).cpu())
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2, window, sinks)
    pf.check_attention(outs[0], want, dtype, f"ordinary {seqs}")
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("large", [2.0 ** 125, 2.0 ** 126, 2.0 ** 127, LARGEST])
@pytest.mark.parametrize("seqs", [[(300, 300)], [(40, 700), (3, 90)], [(9, 100)]],
                         ids=["many", "mixed", "few"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_scales_near_the_end_of_the_range(dtype, seqs, large):
    """A finite scale of the first sequence's last position, which its last token alone sees: the
    others' outputs stay finite (beside it their scales have no bits left), those of other sequences
    keep their bounds, and what the last token attends is not lost."""
    rng = np.random.default_rng(33)
    rows, lens, starts, _, _, quats, q = attention_case(rng, seqs, 16, 2, 16, dtype)
    rows[3][0, :, seqs[0][1] - 1] = large
    pool, tables = sv.to_pool(rng, rows, lens, 16, -(-int(lens.max()) // 16) + 1)
    out = attend(q, pool, tables, starts, lens, quats).cpu()
    n = seqs[0][0]
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2)
    assert torch.isfinite(out[:n - 1]).all()
    pf.check_attention(out[n:], tuple(x[n:] for x in want), dtype, f"beside {large}")
    last = tuple(x[n - 1] for x in want)
    if dtype == torch.float16:
        assert np.abs(last[0]).max(-1).min() > 2 * 65504      # beyond fp16 in every head
        assert (~torch.isfinite(out[n - 1])).any(-1).all()
    else:
        pf.check_attention(out[n - 1], last, dtype, f"with {large}")
