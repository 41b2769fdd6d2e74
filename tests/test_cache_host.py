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
@pytest.mark.parametrize("name", ["tc_rope", "tc_strides", "tc_cache"])
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


CACHE = dict(batch=4, n_heads=8, n_kv_heads=2, head_dim=64, dtype=1, n_query=3, capacity=100, n_prefixes=2, prefix_len=10, budget=40, n_sink=4,
             n_recent=8)


def _calls(tc, **change):
    """Every entry point on a cache, with arguments that name no memory; `change` replaces some of them."""
    lib, F = tc.load_library(), FAKE
    st = ctypes.byref(tc.tc_strides(1024, 64, 256))
    a = dict(c=None, r=ctypes.byref(tc.make_rope(64)), Q=F, qs=st, K=F, ks=st, V=F, vs=st, cos=F, sin=F, pos=F, len=F, q_len=F, Qo=F, Kc=F, Vc=F,
             sp=F, w=F, Kp=F, Vp=F, O=2 * F, Ko=2 * F, Vo=2 * F, po=2 * F, wo=2 * F, cap=50, lo=2 * F, ws=F, bytes=1 << 40)
    a.update(change)
    v = lambda *names: [a[n] for n in names]  # noqa: E731
    return {
        "append": lambda: lib.tc_cache_append(*v("c", "r", "Q", "qs", "K", "ks", "V", "vs", "cos", "sin", "pos", "len", "q_len", "Qo", "Kc", "Vc", "sp", "w"), None),
        "attention": lambda: lib.tc_cache_attention(*v("c", "Q", "Kp", "Vp", "Kc", "Vc", "len", "q_len", "O", "w", "ws", "bytes"), None),
        "evict": lambda: lib.tc_cache_evict(*v("c", "len", "Kc", "Vc", "sp", "w", "Ko", "Vo", "po", "wo", "cap", "lo", "ws", "bytes"), None),
    }


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), -2), (dict(batch=(1 << 16) + 2), -2), (dict(n_heads=0), -2), (dict(n_heads=2048), -2), (dict(n_kv_heads=3), -2),
    (dict(n_kv_heads=0), -2), (dict(head_dim=96), -2), (dict(n_query=0), -2), (dict(n_query=(1 << 20) + 1), -2), (dict(capacity=0), -2),
    (dict(capacity=(1 << 24) + 1), -2), (dict(max_len=101), -2), (dict(max_len=-1), -2), (dict(n_prefixes=3), -2), (dict(n_prefixes=-1), -2),
    (dict(n_prefixes=0), -2), (dict(prefix_len=-1), -2), (dict(prefix_len=(1 << 24) + 1), -2), (dict(dtype=3), -3), (dict(softmax_scale=-1.0), -4),
    (dict(softmax_scale=float("inf")), -4), (dict(softmax_scale=float("nan")), -4), (dict(budget=101), -4), (dict(budget=-1), -4),
    (dict(n_sink=-1), -4), (dict(n_recent=-1), -4), (dict(n_sink=33), -4), (dict(n_sink=2 ** 31 - 1, n_recent=2 ** 31 - 1), -4),
    (dict(batch=1 << 16, n_heads=1024, n_kv_heads=1024, n_query=1 << 20), -2)])
def test_cache_parameters_out_of_range(kw, status):
    tc = _binding()
    c = tc.make_cache(**dict(CACHE, **kw))
    assert tc.tc_cache_workspace_bytes(c) == 0
    for name, call in _calls(tc, c=ctypes.byref(c)).items():
        assert call() == status, name


@needs_library
def test_cache_entry_points_check_their_arguments():
    tc = _binding()
    c = tc.make_cache(**CACHE)
    ok = ctypes.byref(c)
    needed = {"append": ("Q", "qs", "K", "ks", "V", "vs", "cos", "sin", "pos", "len", "Qo", "Kc", "Vc", "sp", "w"),
              "attention": ("Q", "Kp", "Vp", "Kc", "Vc", "len", "O", "ws"),
              "evict": ("len", "Kc", "Vc", "sp", "w", "Ko", "Vo", "po", "wo", "lo", "ws")}
    for entry, names in needed.items():
        for name in names:
            assert _calls(tc, c=ok, **{name: None})[entry]() == -1, (entry, name)
            if name not in ("qs", "ks", "vs"):
                assert _calls(tc, c=ok, **{name: FAKE + 8})[entry]() == -6, (entry, name)
        assert _calls(tc, c=None)[entry]() == -1
        empty = ctypes.byref(tc.make_cache(**dict(CACHE, batch=0)))
        assert _calls(tc, c=empty, **{name: None for name in names})[entry]() == 0
    assert _calls(tc, c=ok, w=FAKE + 4)["attention"]() == -6 and _calls(tc, c=ok, q_len=FAKE + 4)["attention"]() == -6
    assert _calls(tc, c=ok, bytes=tc.tc_cache_workspace_bytes(c) - 1)["attention"]() == -5
    odd = ctypes.byref(tc.tc_strides(1024, 64, 4))
    for name in ("qs", "ks", "vs"):
        assert _calls(tc, c=ok, **{name: odd})["append"]() == -2
    assert _calls(tc, c=ok, r=ctypes.byref(tc.make_rope(128)))["append"]() == -2
    assert _calls(tc, c=ok, r=ctypes.byref(tc.make_rope(64, rot_dim=1)))["append"]() == -2
    assert _calls(tc, c=ok, r=None)["append"]() == -1    # tables without what they are of
    assert _calls(tc, c=ok, cap=39)["evict"]() == -2
    assert _calls(tc, c=ok, bytes=tc.tc_cache_workspace_bytes(c) - 1)["evict"]() == -5
    assert _calls(tc, c=ok, lo=FAKE)["evict"]() == -4     # the lengths are read while they are written
    assert _calls(tc, c=ok, Ko=FAKE)["evict"]() == -4     # half in place
    assert _calls(tc, c=ok, Ko=FAKE, Vo=FAKE, po=FAKE, wo=FAKE, cap=99)["evict"]() == -4
    assert _calls(tc, c=ctypes.byref(tc.make_cache(**dict(CACHE, budget=0, n_sink=0, n_recent=0))))["evict"]() == -4


@needs_library
def test_what_no_grid_holds_is_refused():
    """A grid counts its threads in 32 bits."""
    tc = _binding()
    lib, F = tc.load_library(), FAKE
    big = dict(batch=1 << 16, n_heads=1024, n_kv_heads=1024, head_dim=64, dtype=1, n_query=1, capacity=4)
    for kw in (dict(big, budget=2), dict(big, budget=4, batch=1 << 15, n_heads=512, n_kv_heads=512)):
        calls = _calls(tc, c=ctypes.byref(tc.make_cache(**kw)), Kp=None, Vp=None, bytes=1 << 60)
        assert calls["attention"]() == calls["evict"]() == -2
    c = tc.make_cache(**dict(big, batch=1, n_query=1 << 20))
    assert _calls(tc, c=ctypes.byref(c))["append"]() == -2
    st = ctypes.byref(tc.tc_strides(1 << 30, 128, 1 << 17))
    r = ctypes.byref(tc.make_rope(128, rot_dim=2))
    assert lib.tc_rope_apply(r, tc.TC_BF16, 1 << 8, 1024, 1 << 13, F, st, F, F, F, st, 0, None) == -2
    assert lib.tc_rope_tables(r, F, 1 << 36, F, F, None) == -2


@needs_library
def test_cache_workspace_grows_with_the_cache_and_not_with_the_call():
    tc = _binding()
    size = lambda **kw: tc.tc_cache_workspace_bytes(tc.make_cache(**dict(CACHE, **kw)))  # noqa: E731
    assert size() % 256 == 0
    assert size(max_len=1) == size(max_len=50) == size(max_len=100) == size()
    for name, values in (("capacity", (40, 4096, 32768, 32769, 1 << 20)), ("budget", (12, 40, 100))):
        sizes = [size(**{name: x}) for x in values]
        assert sizes == sorted(sizes), name


def test_oracle_appends_the_last_slots():
    K, V, p, w = np.zeros((2, 5, 3)), np.zeros((2, 5, 3)), np.full((2, 5), -1), np.ones((2, 5))
    k = np.arange(12.0).reshape(2, 2, 3)
    orc.append(K, V, p, w, k, -k, [7, 9], 4)
    assert np.array_equal(K[:, 2:4], k) and np.array_equal(V[:, 2:4], -k) and p.tolist() == [[-1, -1, 7, 9, -1]] * 2
    assert w.tolist() == [[1, 1, 0, 0, 1]] * 2 and not K[:, [0, 1, 4]].any()
    orc.append(K, V, p, w, k, -k, [7, 9], 6)    # the second one falls behind the cache
    assert np.array_equal(K[:, 4], k[:, 0])


def test_oracle_attention_by_a_softmax_and_closed_forms():
    g = np.random.default_rng(4)
    q, K, V, Kp, Vp = (g.normal(size=s) for s in ((4, 3, 8), (2, 10, 8), (2, 10, 8), (2, 5, 8), (2, 5, 8)))
    O, W = orc.attention(q, K, V, 7, 3, Kp, Vp)
    for h in range(4):
        j = h // 2
        keys, vals = np.concatenate([Kp[j], K[j, :7]]), np.concatenate([Vp[j], V[j, :7]])
        s = q[h] @ keys.T / np.sqrt(8)
        for t in range(3):
            s[t, 5 + 7 - 3 + t + 1:] = -np.inf
        p = np.exp(s) / np.exp(s).sum(1, keepdims=True)
        assert np.allclose(O[:, h], p @ vals)
    assert np.isclose(W[:, :7].sum() + _prefix_share(q, K, Kp), 12.0) and not W[:, 7:].any()
    # equal keys: the mean of the values seen; no key at all: zero; padded rows: zero
    O, W = orc.attention(q, np.ones_like(K), V, 2, 2)
    assert np.allclose(O[0, 0], V[0, 0]) and np.allclose(O[1, 3], V[1, :2].mean(0)) and not O[2].any()
    assert np.allclose(W[0, :2], [2 * 1.5, 2 * 0.5])
    O, W = orc.attention(q, K, V, 0, 3)
    assert not O.any() and not W.any()
    O, W = orc.attention(q, K, V, 2, 3)        # the first of three tokens lies in front of the cache
    assert not O[0].any() and np.allclose(O[1, 0], V[0, 0])


def _prefix_share(q, K, Kp):
    total = 0.0
    for h in range(4):
        for t in range(3):
            s = np.exp(np.concatenate([Kp[h // 2], K[h // 2, :5 + t]]) @ q[h, t] / np.sqrt(8))
            total += s[:5].sum() / s.sum()
    return total


@pytest.mark.parametrize("mistake", ["later", "prefix", "head", "scale", "weight"])
def test_planted_mistakes_move_the_oracle(mistake):
    """What the comparisons on the GPU rest on: each of these mistakes, planted here, is far outside their bounds."""
    g = np.random.default_rng(5)
    q, K, V, Kp, Vp = (g.normal(size=s) for s in ((4, 3, 64), (2, 40, 64), (2, 40, 64), (2, 20, 64), (2, 20, 64)))
    O, W = orc.attention(q, K, V, 30, 3, Kp, Vp)
    if mistake == "later":       # the rows see one slot too many
        P, X = orc.attention(q, K, V, 31, 3, Kp, Vp)
    elif mistake == "prefix":    # a prefix without its last key
        P, X = orc.attention(q, K, V, 30, 3, Kp[:, :-1], Vp[:, :-1])
    elif mistake == "head":      # heads dealt to key heads in turn
        P, X = orc.attention(q[[0, 2, 1, 3]], K, V, 30, 3, Kp, Vp)
    elif mistake == "scale":
        P, X = orc.attention(q, K, V, 30, 3, Kp, Vp, scale=0.13)
    else:                        # a row of a head that does not share the slot
        P, X = O, orc.attention(q[[0, 0, 2, 3]], K, V, 30, 3, Kp, Vp)[1]
    assert np.abs(O - P).max() > 0.02 or np.abs(W - X).max() > 0.02


def test_oracle_evicts_by_protection_weight_and_slot():
    pos, w = [0, 1, 2, 3, 4, 5, 6, 7], [0.1, 5.0, 2.0, 2.0, float("nan"), 2.0, 0.3, 0.0]
    # slot 0 and 7 are protected, 1 has the most, of 2, 3, 5 the first two stay
    assert orc.evict(pos, w, 8, 5, 1, 1) == [0, 1, 2, 3, 7]
    assert orc.evict(pos, w, 8, 4, 1, 1) == [0, 1, 2, 7]
    assert orc.evict(pos, w, 8, 3, 0, 0) == [3, 1, 2]    # no one is protected: slot 3 comes to the freed slot 0
    assert orc.evict(pos, w, 8, 2, 0, 1) == [7, 1]
    assert orc.evict(pos, w, 5, 5, 0, 0) == [0, 1, 2, 3, 4] and orc.evict(pos, w, 0, 5, 0, 0) == []
    assert orc.evict(pos, [0.0, -0.0] * 4, 8, 3, 0, 0) == [0, 1, 2]


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
