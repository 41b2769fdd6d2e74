"""Attention over a shared prefix and the cache against the float64 oracle: types, heads, lengths, masks, what may not be seen, weights."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _tc():
    from oracle import cache_oracle as orc
    from paper_2503_10501_amd import binding as tc
    tc.load_library()
    return tc, orc


def make(dtype, d, B, H, Hk, T, cap, lens, q_len=None, images=0, P=0, max_len=0, scale=0.0, weights=True, seed=0, spread=1.0):
    """A call's tensors.  Slots behind a sequence's length hold NaN: nothing may come from there."""
    tc, _ = _tc()
    g, sd = torch.Generator().manual_seed(seed), DTYPES[dtype]
    s = dict(c=tc.make_cache(B, H, Hk, d, tc._DTYPES[dtype], T, cap, max_len=max_len, n_prefixes=images, prefix_len=P, softmax_scale=scale))
    normal = lambda *shape: torch.randn(*shape, generator=g).to(sd)  # noqa: E731
    s["Q"], K, V = normal(B, H, T, d) * spread, normal(B, Hk, cap, d), normal(B, Hk, cap, d)
    for b in range(B):
        K[b, :, max(0, min(lens[b], max_len or cap)):], V[b, :, max(0, min(lens[b], max_len or cap)):] = float("nan"), float("nan")
    s["K"], s["V"] = K, V
    s["Kp"], s["Vp"] = (normal(images, Hk, P, d), normal(images, Hk, P, d)) if P else (None, None)
    s["w"] = torch.rand(B, Hk, cap, generator=g) if weights else None
    s["lens"], s["q_len"] = torch.tensor(lens, dtype=torch.int32), None if q_len is None else torch.tensor(q_len, dtype=torch.int32)
    for k in s:
        if k != "c" and s[k] is not None:
            s[k] = s[k].cuda()
    s["O"] = torch.full((B, T, H * d), 7.0, dtype=sd, device="cuda")
    s["ws"] = torch.full((tc.tc_cache_workspace_bytes(s["c"]),), 0xff, dtype=torch.uint8, device="cuda")
    return s


def call(s):
    tc, _ = _tc()
    tc.tc_cache_attention(s["c"], s["Q"], s["K"], s["V"], s["lens"], s["O"], s["ws"], K_prefix=s["Kp"], V_prefix=s["Vp"], weight=s["w"],
                          q_len=s["q_len"])


def check(s, before=None):
    """Runs the call and compares.  The bound of an output, A = sum p |v| of its row:
      half a step of the storage type of O; of the probabilities too, where they enter the products rounded once (p (1 + e), |e| <= h each: off
      by h A at most), which they do in tiles of more than 16 rows: those of a sequence, or of all sequences of an image at its prefix;
      scores: d + 4 roundings of float32 of at most scale sum |q k|, in the exponent, so relative to p, numerator and sum: twice;
      2^-20 for the exponentials (an ulp or two each) and sums; half storage: probabilities below its normal numbers, 2^-25 each."""
    _, orc = _tc()
    c, sd = s["c"], s["O"].dtype
    h, sixteen = torch.finfo(sd).eps / 2, sd != torch.float32
    w0 = None if s["w"] is None else s["w"].clone()
    call(s)
    torch.cuda.synchronize()
    B, H, Hk, T, d = c.batch, c.n_heads, c.n_kv_heads, c.n_query, c.head_dim
    host = {k: None if s[k] is None else s[k].cpu().double().numpy() for k in ("Q", "K", "V", "Kp", "Vp", "O", "w")}
    scale = float(np.float32(c.softmax_scale)) or 1.0 / np.sqrt(d)
    for b in range(B):
        n = min(max(int(s["lens"][b]), 0), c.max_len or c.capacity)
        m = T if s["q_len"] is None else min(max(int(s["q_len"][b]), 0), T)
        img = b // (B // c.n_prefixes) if c.prefix_len else None
        Kp, Vp = (None, None) if img is None else (host["Kp"][img], host["Vp"][img])
        K, V = host["K"][b, :, :n], host["V"][b, :, :n]
        want, grow = orc.attention(host["Q"][b], K, V, n, m, Kp, Vp, scale)
        A, _ = orc.attention(host["Q"][b], K, np.abs(V), n, m, Kp, None if Vp is None else np.abs(Vp), scale)
        keys = K if Kp is None else np.concatenate([Kp, K], axis=1)
        vals = V if Vp is None else np.concatenate([Vp, V], axis=1)
        es = 0.0 if keys.shape[1] == 0 or m == 0 else 2.0 ** -24 * (d + 4) * scale * max(
            np.abs(host["Q"][b, x, :m]).dot(np.abs(keys[x // (H // Hk)]).T).max() for x in range(H))
        rel = 2 * (es + 2.0 ** -20)
        tile = H // Hk * T * (B // c.n_prefixes if c.prefix_len else 1)
        bound = h * np.abs(want) + ((h if tile > 16 else h * h) if sixteen else 0) * A + rel * A
        if sd == torch.float16 and keys.shape[1]:
            bound = bound + 2.0 ** -25 * (1 + np.abs(vals).sum(1).max())
        got = host["O"][b].reshape(T, H, d)
        assert np.all(np.abs(got - want) <= bound), (b, np.max(np.abs(got - want) - bound))
        assert not got[m:].any()
        if w0 is not None:
            base, new = w0[b].cpu().double().numpy(), host["w"][b]
            off = np.abs(new[:, :n] - base[:, :n] - grow)
            assert np.all(off <= 2 * rel * grow + 2.0 ** -24 * (np.abs(new[:, :n]) + 64 * grow)), (b, off.max())
            assert np.array_equal(new[:, n:], base[:, n:])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 2), (8, 1)])
@pytest.mark.parametrize("T", [1, 3, 20])
def test_types_heads_and_rows(dtype, d, H, Hk, T):
    check(make(dtype, d, 3, H, Hk, T, 100, [100, T, 57], seed=T))
    check(make(dtype, d, 4, H, Hk, T, 90, [90, 33, 64, T], [T, max(1, T - 1), (T + 1) // 2, 0], images=2, P=41, seed=T + 1))


@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
@pytest.mark.parametrize("P", [0, 1, 31, 32, 33, 65])
def test_lengths_of_one_token(n, P):
    check(make("bf16", 64, 2, 2, 1, 1, max(n, 1), [n, n], images=1 if P else 0, P=P, seed=n + 7 * P))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,lens,q_len", [(5, [3, 0, 5, 4], None), (40, [70, 12, 40, 0], [40, 12, 39, 40]), (130, [130, 200, 64, 131], [130, 129, 64, 1]),
                                          (33, [33, 99, 5, 7], [0, 0, 0, 1]), (70, [-4, 500, 200, 77], [-1, 99, 70, 70])])
@pytest.mark.parametrize("P", [0, 50])
def test_rows_that_see_little_or_nothing(dtype, T, lens, q_len, P):
    # more rows than slots, none of either, lengths out of range
    check(make(dtype, 64, 4, 2, 1, T, 200, lens, q_len, images=4 if P else 0, P=P))


@pytest.mark.parametrize("dtype,d,H,Hk", [("bf16", 128, 8, 2), ("f16", 64, 4, 4), ("f32", 128, 2, 1)])
def test_long_caches_and_prefixes(dtype, d, H, Hk):
    check(make(dtype, d, 1, H, Hk, 1, 6000, [5999]))
    check(make(dtype, d, 2, H, Hk, 1, 2500, [2500, 3], images=1, P=3100))
    check(make(dtype, d, 2, H, Hk, 7, 1500, [1500, 700], [7, 5], images=2, P=1001))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("each,T", [(1, 1), (3, 1), (16, 1), (21, 2), (40, 1), (5, 30), (2, 70)])
def test_sequences_of_an_image_share_its_prefix(dtype, each, T):
    B = 2 * each
    g = np.random.default_rng(each)
    lens = [int(x) for x in g.integers(T, T + 60, B)]
    check(make(dtype, 64, B, 2, 1, T, T + 60, lens, [int(x) for x in g.integers(0, T + 1, B)], images=2, P=70, seed=each))


@pytest.mark.parametrize("dtype,d,H,Hk,each,T,P", [
    ("bf16", 128, 8, 8, 3, 1, 2100), ("bf16", 64, 16, 16, 8, 2, 1200), ("f16", 64, 8, 8, 12, 5, 1500), ("f16", 128, 16, 4, 10, 1, 1777),
    ("f32", 64, 8, 8, 9, 1, 1100), ("f32", 128, 4, 4, 20, 2, 500), ("bf16", 64, 8, 8, 33, 16, 300)])
def test_prefixes_large_enough_to_be_read_once(dtype, d, H, Hk, each, T, P):
    """From 32 MB on that would be read again: rows of all sequences of an image as one matrix, of up to and over 16 rows."""
    B = 2 * each
    g = np.random.default_rng(each + T)
    assert 2 * (each - 1) * Hk * P * d * 2 * torch.finfo(DTYPES[dtype]).bits // 8 >= 32e6
    lens = [int(x) for x in g.integers(0, T + 60, B)]
    q_len = [int(x) for x in g.integers(0, T + 1, B)]
    check(make(dtype, d, B, H, Hk, T, T + 60, lens, q_len, images=2, P=P, seed=each))
    check(make(dtype, d, B, H, Hk, T, T + 300, [x + 230 for x in lens], images=2, P=P, seed=each, weights=False))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("n,P", [(2040, 0), (2048, 0), (2049, 0), (1000, 1040), (1000, 1060), (130, 0), (128, 0), (129, 0), (0, 2000), (1, 127)])
def test_one_sequence_with_and_without_parts(dtype, d, n, P):
    # the largest cache of one sweep, and the smallest that is cut
    check(make(dtype, d, 1, 4, 2, 1, max(n, 1), [n], images=1 if P else 0, P=P))
    check(make(dtype, d, 1, 2, 2, 3, n + 2, [n], images=1 if P else 0, P=P, weights=False))


@pytest.mark.parametrize("T", [1, 6, 90, 300])
def test_many_rows_without_weights(T):
    check(make("bf16", 128, 2, 4, 2, T, 400, [400, 333], images=1, P=37, weights=False))
    check(make("f16", 64, 3, 3, 3, T, 350, [350, 301, 300], weights=False))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T", [3, 60])
def test_what_is_not_seen_has_no_influence(dtype, T):
    """NaN and infinities in later tokens' keys and values, in padded rows of queries, and values that some rows see."""
    _, orc = _tc()
    for bad in (float("nan"), float("inf"), -float("inf")):
        s = make(dtype, 64, 2, 4, 2, T, 100, [90, 80], [T, T - 1], images=1, P=40, seed=5)
        call(s)
        clean, weight = s["O"].clone(), s["w"].clone()
        t = make(dtype, 64, 2, 4, 2, T, 100, [90, 80], [T, T - 1], images=1, P=40, seed=5)
        t["Q"][1, :, T - 1] = bad                   # a padded row
        t["K"][0, :, 89], t["V"][0, :, 88] = bad, bad     # keys of the last token, values of the one before it
        call(t)
        torch.cuda.synchronize()
        assert torch.equal(t["O"][1], clean[1]) and torch.equal(t["w"][1], weight[1])
        assert torch.equal(t["O"][0, :T - 2], clean[0, :T - 2])
        late = t["O"][0, T - 2].float()              # sees the value, not the key
        assert (late.isnan().all() if bad != bad else (late == bad).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 40])
def test_values_at_the_end_of_the_range(dtype, T):
    # sums of weighted values stay within float32 where their mean does
    s = make(dtype, 64, 1, 2, 1, T, 500, [500], images=1, P=300, spread=0.01, weights=False)
    big = float(torch.finfo(DTYPES[dtype]).max) * 0.9
    s["V"].fill_(big)
    s["Vp"].fill_(big)
    call(s)
    torch.cuda.synchronize()
    assert ((s["O"].double() / big - 1).abs() <= 2.0 ** -7 if dtype == "bf16" else (s["O"].double() / big - 1).abs() <= 2.0 ** -18).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_peaked_and_scaled_scores(dtype):
    check(make(dtype, 128, 2, 4, 1, 2, 200, [200, 111], scale=0.7, spread=6.0))
    check(make(dtype, 64, 2, 2, 2, 33, 200, [200, 111], scale=1e-3, images=1, P=64))


@pytest.mark.parametrize("dtype,d,G,T,P", [("bf16", 64, 1, 20, 0), ("f16", 64, 2, 32, 70), ("bf16", 128, 1, 33, 0), ("f16", 128, 4, 25, 40)])
def test_heads_enough_that_keys_are_one_part(dtype, d, G, T, P):
    # (what the slots gather is then added by the kernel that attends, several tiles of keys one after another)
    g = np.random.default_rng(T)
    B, Hk, cap = 16, 32, 330
    lens = [330, 0, 1, 64, 65, 128, 129, 192, 193] + [int(x) for x in g.integers(0, cap + 1, B - 9)]
    check(make(dtype, d, B, G * Hk, Hk, T, cap, lens, [T, 0, T] + [int(x) for x in g.integers(0, T + 1, B - 3)], images=4 if P else 0, P=P, seed=T))


@pytest.mark.parametrize("dtype,d,B,G,T,cap,images,P", [
    ("bf16", 128, 24, 1, 1, 40, 0, 0), ("f16", 128, 20, 4, 3, 170, 4, 20), ("bf16", 128, 24, 2, 1, 320, 0, 0), ("f16", 64, 40, 1, 2, 130, 0, 0),
    ("bf16", 64, 40, 1, 1, 300, 8, 10), ("f32", 64, 24, 1, 1, 100, 2, 33), ("f32", 128, 12, 2, 5, 290, 0, 0), ("bf16", 128, 64, 1, 1, 60, 8, 40),
    ("f16", 128, 64, 1, 1, 250, 8, 40)])
def test_more_heads_than_fit_at_once(dtype, d, B, G, T, cap, images, P):
    # (one or two wavefronts have a head's keys)
    g = np.random.default_rng(cap)
    lens = [cap, 0, 1, 33] + [int(x) for x in g.integers(0, cap + 1, B - 4)]
    check(make(dtype, d, B, 32 * G, 32, T, cap, lens, [int(x) for x in g.integers(0, T + 1, B)] if T > 1 else None, images=images, P=P, seed=cap))


@pytest.mark.parametrize("T", [1, 16, 40, 80])
def test_many_halves_far_below_the_largest(T):
    """One key has all but a thousandth of the attention, 40000 others 2^-25.4 of its each: rounded to halves as they are they would be nothing.
    They are rounded as multiples of 2^-24 after a factor: 2^15 in small tiles, whose remainder is exact to half a step, 2^-40 of the largest;
    2^7 at least in large ones, 2^-32."""
    _, orc = _tc()
    n = 40000
    s = make("f16", 64, 1, 1, 1, T, n, [n])
    s["Q"].zero_(), s["K"].zero_()
    s["Q"][..., 0], s["K"][0, 0, 0, 0], s["V"][0, 0, 0], s["V"][0, 0, 1:] = 16.0, 8.8, 0.0, 1.0
    call(s)
    want, _ = orc.attention(*(s[k][0].cpu().double().numpy() for k in ("Q", "K", "V")), n, T)
    got = s["O"][0].cpu().double().numpy()
    want = np.asarray(want).reshape(T, 64)
    h, rel = 2.0 ** -11, 2 * (2.0 ** -24 * 68 * 17.6 + 2.0 ** -20)
    bound = (h + (h if T > 16 else h * h) + rel) * want + n * (2.0 ** -32 if T > 16 else 2.0 ** -40)
    assert 8e-4 < want.min() and np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / want)


def test_weights_gather_over_calls_and_are_the_same_each_time():
    s = make("bf16", 128, 3, 8, 2, 1, 700, [700, 650, 9], images=1, P=128)
    start = s["w"].clone()
    call(s)
    once, O = s["w"].clone(), s["O"].clone()
    for _ in range(3):
        s["w"].copy_(start)
        call(s)
        assert torch.equal(s["w"], once) and torch.equal(s["O"], O)
    s["w"].copy_(start)
    for _ in range(3):
        call(s)
    grown = once.double() - start.double()
    assert ((s["w"].double() - start.double()) - 3 * grown).abs().max() <= 6 * 2.0 ** -23


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 elements: the last sequence's rows are found."""
    cap, B = 1 << 20, 33
    s = make("bf16", 128, 1, 1, 1, 1, 64, [60], weights=False)
    call(s)
    tc, _ = _tc()
    K, V = (torch.zeros(B, 1, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K[-1, :, :64], V[-1, :, :64] = s["K"][0], s["V"][0]
    c = tc.make_cache(B, 1, 1, 128, tc.TC_BF16, 1, cap, max_len=64)
    O = torch.empty(B, 1, 128, dtype=torch.bfloat16, device="cuda")
    lens = torch.full((B,), 60, dtype=torch.int32, device="cuda")
    tc.tc_cache_attention(c, s["Q"].expand(B, 1, 1, 128).contiguous(), K, V, lens, O, tc.new_cache_workspace(c))
    torch.cuda.synchronize()
    assert (O[-1].float() - s["O"][0].float()).abs().max() <= 2.0 ** -7 * s["O"].float().abs().max() and not O[:-1].any()


def test_the_largest_numbers_of_sequences_rows_and_heads():
    tc, _ = _tc()
    new = lambda *s, dtype=torch.bfloat16: torch.randn(*s, device="cuda").to(dtype)  # noqa: E731
    for B, H, Hk, T, cap in ((65536, 1, 1, 1, 3), (1, 1, 1, 1 << 20, 40), (2, 1024, 1, 1, 70), (2, 1024, 1024, 1, 5)):
        c = tc.make_cache(B, H, Hk, 64, tc.TC_BF16, T, cap, budget=2)
        Q, K, V = new(B, H, T, 64), new(B, Hk, cap, 64), new(B, Hk, cap, 64)
        lens, q_len = torch.full((B,), cap, dtype=torch.int32, device="cuda"), torch.full((B,), min(T, 2), dtype=torch.int32, device="cuda")
        O, w, ws = torch.empty(B, T, H * 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, Hk, cap, device="cuda"), tc.new_cache_workspace(c)
        tc.tc_cache_attention(c, Q, K, V, lens, O, ws, weight=w, q_len=q_len)
        m = min(T, 2)
        x = (Q[:, :, :m].double().view(B, Hk, -1, 64) @ K.double().transpose(2, 3).contiguous()) / 8
        if m == 2:
            x[:, :, 0, cap - 1] = -float("inf")   # (one head) the first of two rows does not see the last slot
        p = x.softmax(-1)
        want = (p @ V.double()).view(B, H, m, 64).transpose(1, 2).reshape(B, m, H * 64)
        # one rounding of the output and one of the probabilities, of values of at most 5.6
        assert (O[:, :m].double() - want).abs().max() <= 2 * 2.0 ** -8 * 5.6 and not O[:, m:].any()
        assert (w.double() - p.sum(2)).abs().max() <= 2.0 ** -16 * p.sum(2).max()
        sp, left = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(B, Hk, 1), torch.empty(B, dtype=torch.int32, device="cuda")
        tc.tc_cache_evict(c, lens, K, V, sp, w, left, ws)
        best = p.sum(2).topk(2, dim=-1).values.sum(-1)
        assert (w[:, :, :2].double().sum(-1) - best).abs().max() <= 2.0 ** -15 * best.max() and (left == 2).all()


def test_refusals():
    tc, _ = _tc()
    s = make("bf16", 64, 2, 4, 2, 3, 20, [20, 9], [3, 1], images=1, P=7)
    s["K"], s["V"] = s["K"].nan_to_num(), s["V"].nan_to_num()
    call(s)
    for name in ("Q", "K", "V", "Kp", "Vp", "w", "lens", "q_len", "O", "ws"):
        bads = [s[name].cpu(), s[name].double()] + ([s[name][:1] if name != "Kp" and name != "Vp" else s[name][:, :, :5]] if name != "ws" else [])
        for bad in bads:
            with pytest.raises(ValueError):
                call(dict(s, **{name: bad}))
    with pytest.raises(ValueError):
        call(dict(s, Kp=None))
    with pytest.raises(ValueError):
        call(dict(s, Q=s["Q"].transpose(1, 2).contiguous().transpose(1, 2)))
    with pytest.raises(tc.TokenCarveError) as e:
        call(dict(s, ws=s["ws"][:256]))
    assert e.value.status == -5
