"""Rows that are written must differ (no GPU: the refusal comes before any launch)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2503_10501_amd", "libtokencarve.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libtokencarve.so not built (run __graft_entry__.build())")
FAKE = 4096   # never dereferenced: the call must fail before any launch


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("in_place", [True, False])
def test_rows_that_overlap_are_refused_as_output(d, which, in_place):
    from paper_2503_10501_amd import binding as tc
    lib, F = tc.load_library(), FAKE
    r = ctypes.byref(tc.make_rope(d))
    good = [d * 16, d * 4, d]
    bad = list(good)
    for stride in (0, 8, d // 2, d - 8):
        bad[which] = stride
        st = ctypes.byref(tc.tc_strides(*bad))
        xs = st if in_place else ctypes.byref(tc.tc_strides(*good))
        assert lib.tc_rope_apply(r, tc.TC_BF16, 2, 4, 4, F, xs, F, F, F if in_place else 2 * F, st, 0, None) == -2
        # along an axis of one entry the stride says nothing: the next check is reached (tables that are not aligned)
        sizes = [1 if i == which else 4 for i in range(3)]
        assert lib.tc_rope_apply(r, tc.TC_BF16, *sizes, F, xs, F + 4, F, F if in_place else 2 * F, st, 0, None) == -6
