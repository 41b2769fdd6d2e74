"""Tensors that require gradients are not turned without a word (no GPU: the refusal comes before the device is looked at)."""
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2503_10501_amd", "libtokencarve.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libtokencarve.so not built (run __graft_entry__.build())")


def test_tensors_that_require_gradients_are_refused_unless_these_are_off():
    from paper_2503_10501_amd import binding as tc
    r, table = tc.make_rope(64), torch.zeros(1, 2, 32)
    plain, leaf = torch.zeros(1, 3, 2, 64), torch.zeros(1, 3, 2, 64, requires_grad=True)
    for x, y in ((leaf, None), (leaf, plain), (plain, leaf), (leaf * 2, plain)):
        for transposed in (False, True):
            with pytest.raises(ValueError, match="gradients"):
                tc.tc_rope_apply(r, x, table, table, y, transposed=transposed)
    with torch.no_grad():
        with pytest.raises(ValueError, match="GPU"):   # as for any tensor on the CPU
            tc.tc_rope_apply(r, leaf, table, table)
    with pytest.raises(ValueError, match="GPU"):
        tc.tc_rope_apply(r, plain, table, table)
    with torch.no_grad():   # what was made there does not require them
        y = leaf * 2
    with pytest.raises(ValueError, match="GPU"):
        tc.tc_rope_apply(r, y, table, table)


@pytest.mark.gpu
def test_a_parameter_is_turned_where_gradients_are_off():
    from paper_2503_10501_amd import binding as tc
    r = tc.make_rope(64)
    c, s = torch.empty(1, 5, 32, device="cuda"), torch.empty(1, 5, 32, device="cuda")
    tc.tc_rope_tables(r, torch.arange(5, dtype=torch.int32, device="cuda")[None], c, s)
    x = torch.nn.Parameter(torch.randn(1, 2, 5, 64, device="cuda"))
    y = torch.empty(1, 2, 5, 64, device="cuda")
    tc.tc_rope_apply(r, x.detach(), c, s, y)
    with torch.no_grad():
        tc.tc_rope_apply(r, x, c, s)
    assert torch.equal(x, y)
