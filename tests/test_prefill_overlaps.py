"""CPU tests of memory that the operators of prompts in chunks may not share (addresses that are
never read: every call is refused before a launch, or asks for a larger workspace)."""

import pytest

from tests.test_prefill_abi import ARG, EXTEND, L, SMALL, at

INPUTS = ["tables", "lens", "more", "refs"]
OUTPUTS = ["out_tables", "out_lens", "out_refs", "starts", "slots", "positions", "status", "ws"]
IN_PLACE = {("tables", "out_tables"), ("lens", "out_lens"), ("refs", "out_refs")}


def call(**kw):
    # (a workspace that is too small is found after all memory in common)
    return L.iq_extend_pages(*dict(EXTEND, nbytes=256, **kw).values())


def test_nothing_shared():
    assert call() == SMALL


@pytest.mark.parametrize("given", INPUTS)
@pytest.mark.parametrize("out", OUTPUTS)
def test_extend_outputs_on_inputs(given, out):
    """An output where an input begins: allowed for the three that may be done in place alone."""
    want = SMALL if (given, out) in IN_PLACE else ARG
    assert call(**{out: EXTEND[given]}) == want
