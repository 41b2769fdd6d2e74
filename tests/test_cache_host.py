"""Host checks (no GPU) of the entry points behind the compression: structures, refusals before any launch, and pins of their oracle."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import cache_oracle as orc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2503_10501_amd", "libtokencarve.so")
needs_library = pytest.mark.skipif(not os.path.exists(LIB), reason="libtokencarve.so not built (run __graft_entry__.build())")
FAKE = 4096   # never dereferenced: the call must fail before any launch


def _binding():
    from paper_2503_10501_amd import binding
    binding.load_library()
    return binding


def _fields(name):
    header = open(os.path.join(ROOT, "include", "tokencarve.h")).read()
    body = header[:header.index("} %s;" % name)]
    body = re.sub(r"/\*.*?\*/", "", body[body.rindex("typedef struct {"):], flags=re.S)
    return [(t, f.strip()) for t, names in re.findall(r"(int32_t|int64_t|float)\s+([\w ,]+);", body) for f in names.split(",")]


@needs_library
@pytest.mark.parametrize("name", ["tc_rope", "tc_strides"])
def test_structures_match_the_header(name):
    tc = _binding()
    kinds = {ctypes.c_int32: "int32_t", ctypes.c_int64: "int64_t", ctypes.c_float: "float"}
    assert _fields(name) == [(kinds[t], f) for f, t in getattr(tc, name)._fields_]


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), -2), (dict(rot_dim=3), -2), (dict(rot_dim=130), -2), (dict(rot_dim=-2), -2), (dict(layout=2), -4), (dict(scaling=4), -4),
    (dict(scaling=-1), -4), (dict(base=1.0), -4), (dict(base=float("nan")), -4), (dict(base=float("inf")), -4), (dict(magnitude=-1.0), -4),
    (dict(scaling=1, factor=0.5), -4), (dict(scaling=2, factor=2.0, rot_dim=2), -4), (dict(scaling=3, factor=2.0, high=4.0), -4),
    (dict(scaling=3, factor=2.0, original_len=10, low=4.0, high=4.0), -4), (dict(scaling=3, factor=float("nan"), original_len=10, high=4.0), -4)])
def test_rotary_parameters_out_of_range(kw, status):
    tc = _binding()
    r = tc.make_rope(**dict(dict(head_dim=128), **kw))
    lib, st = tc.load_library(), ctypes.byref(tc.tc_strides(128, 128, 128))
    assert lib.tc_rope_tables(ctypes.byref(r), FAKE, 4, FAKE, FAKE, None) == status
    assert lib.tc_rope_apply(ctypes.byref(r), tc.TC_BF16, 1, 1, 1, FAKE, st, FAKE, FAKE, FAKE, st, 0, None) == status


@needs_library
def test_rotary_entry_points_check_their_arguments():
    tc = _binding()
    lib, r, F = tc.load_library(), ctypes.byref(tc.make_rope(128)), FAKE
    s = ctypes.byref(tc.tc_strides(128 * 16 * 4, 128, 128 * 4))
    assert lib.tc_rope_tables(None, F, 4, F, F, None) == -1
    assert lib.tc_rope_tables(r, None, 4, F, F, None) == lib.tc_rope_tables(r, F, 4, None, F, None) == lib.tc_rope_tables(r, F, 4, F, None, None) == -1
    assert lib.tc_rope_tables(r, F + 4, 4, F, F, None) == lib.tc_rope_tables(r, F, 4, F, F + 8, None) == -6
    assert lib.tc_rope_tables(r, F, -1, F, F, None) == -2
    assert lib.tc_rope_tables(r, None, 0, None, None, None) == 0

    def apply(dtype=tc.TC_BF16, B=2, H=4, T=16, x=F, xs=s, c=F, sn=F, y=F, ys=s):
        return lib.tc_rope_apply(r, dtype, B, H, T, x, xs, c, sn, y, ys, 0, None)

    assert apply(dtype=3) == -3
    assert apply(B=-1) == apply(B=1 << 17) == apply(H=0) == apply(H=1025) == apply(T=-1) == apply(T=(1 << 20) + 1) == -2
    for what in ("x", "xs", "c", "sn", "y", "ys"):
        assert apply(**{what: None}) == -1
    for what in ("x", "c", "sn", "y"):
        assert apply(**{what: F + 8}) == -6
    for bad in ((-128, 128, 128), (100, 128, 128), (128, 4, 128), (128, 128, 1 << 50)):
        st = ctypes.byref(tc.tc_strides(*bad))
        assert apply(xs=st) == apply(ys=st) == -2
    for i in range(3):   # written rows must differ, rows that are read need not
        v = [8192, 128, 512]
        v[i] = 0
        assert apply(ys=ctypes.byref(tc.tc_strides(*v))) == -2
        assert apply(xs=ctypes.byref(tc.tc_strides(*v))) == -4    # (got as far as the check of calls in place)
    assert apply(B=0, x=None) == apply(T=0, x=None) == 0


def test_oracle_turns_pairs_by_their_angle():
    th = orc.rope_theta(8, base=100.0)
    assert np.allclose(th, [1.0, 100.0 ** -0.25, 100.0 ** -0.5, 100.0 ** -0.75])
    c, s = orc.rope_tables([0, 5], th)
    assert np.allclose(c[0], 1) and np.allclose(s[0], 0) and np.allclose(c[1, 2], np.cos(0.5))
    x = np.arange(10.0)
    y = orc.rope_apply(x, c[1], s[1])
    z = orc.rope_apply(x, c[1], s[1], interleaved=True)
    for k in range(4):
        assert np.allclose([y[k], y[k + 4]], [x[k] * c[1, k] - x[k + 4] * s[1, k], x[k + 4] * c[1, k] + x[k] * s[1, k]])
        assert np.allclose([z[2 * k], z[2 * k + 1]], [x[2 * k] * c[1, k] - x[2 * k + 1] * s[1, k], x[2 * k + 1] * c[1, k] + x[2 * k] * s[1, k]])
    assert np.array_equal(y[8:], x[8:]) and np.array_equal(z[8:], x[8:])
    assert np.allclose(orc.rope_apply(y, c[1], s[1], transposed=True), x)
    # the product of a query and a key turned by their positions depends on the distance alone
    q, k = np.arange(8.0), np.cos(np.arange(8.0))
    at = lambda v, p: orc.rope_apply(v, *orc.rope_tables(p, th))  # noqa: E731
    assert np.isclose(at(q, 17) @ at(k, 12), at(q, 5) @ at(k, 0))


def test_oracle_scalings():
    plain = orc.rope_theta(16)
    assert np.allclose(orc.rope_theta(16, scaling=orc.LINEAR, factor=4.0) * 4, plain)
    by_base = orc.rope_theta(16, scaling=orc.BASE, factor=4.0)
    assert np.isclose(by_base[0], plain[0]) and np.isclose(by_base[-1] * 4, plain[-1])
    bands = orc.rope_theta(16, scaling=orc.BANDS, factor=4.0, original_len=1000, low=1.0, high=4.0)
    turns = 1000 * plain / (2 * np.pi)
    assert np.allclose(bands[turns >= 4], plain[turns >= 4]) and np.allclose(4 * bands[turns <= 1], plain[turns <= 1])
    assert (turns >= 4).any() and (turns <= 1).any() and np.all(np.diff(bands) < 0)
