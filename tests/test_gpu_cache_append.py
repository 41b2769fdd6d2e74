"""New tokens into the cache against the float64 oracle: types, layouts, lengths, rows that do not fit, slots that stay as they are."""
import numpy as np
import pytest
import torch

from tests.test_gpu_rope import DTYPES, _near

pytestmark = pytest.mark.gpu


def _tc():
    from oracle import cache_oracle as orc
    from paper_2503_10501_amd import binding as tc
    tc.load_library()
    return tc, orc


def _run(dtype, d, rot, inter, B, H, Hk, T, cap, lens, q_len, seed=0, max_len=0, turned=True):
    tc, orc = _tc()
    g, sd = torch.Generator().manual_seed(seed), DTYPES[dtype]
    qkv = torch.randn(B, T, (H + 2 * Hk) * d, generator=g).to(sd).cuda()
    q, k, v = qkv.split([H * d, Hk * d, Hk * d], dim=2)
    q, k, v = (x.reshape(B, T, -1, d).transpose(1, 2) if B * T == 1 else x.view(B, T, -1, d).transpose(1, 2) for x in (q, k, v))
    pos = torch.randint(0, 4000, (B, T), generator=g, dtype=torch.int32).cuda()
    K, V = (torch.randn(B, Hk, cap, d, generator=g).to(sd).cuda() for _ in range(2))
    sp = torch.randint(0, 99, (B, Hk, cap), generator=g, dtype=torch.int32).cuda()
    w = torch.rand(B, Hk, cap, generator=g).cuda() + 1
    Qo = torch.full((B, H, T, d), 5.0, dtype=sd, device="cuda")
    r = tc.make_rope(d, rot_dim=rot, layout=int(inter)) if turned else None
    co = si = None
    if turned:
        co, si = torch.empty(B, T, rot // 2, device="cuda"), torch.empty(B, T, rot // 2, device="cuda")
        tc.tc_rope_tables(r, pos, co, si)
    c = tc.make_cache(B, H, Hk, d, tc._DTYPES[dtype], T, cap, max_len=max_len)
    want = [x.cpu().clone().double().numpy() for x in (K, V, sp, w)]
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    m = None if q_len is None else torch.tensor(q_len, dtype=torch.int32, device="cuda")
    tc.tc_cache_append(c, r, q, k, v, co, si, pos, n, Qo, K, V, sp, w, q_len=m)
    torch.cuda.synchronize()
    hq, hk, hv = (x.cpu().double().numpy() for x in (q, k, v))
    if turned:
        ch, sh = co.cpu().double().numpy()[:, None], si.cpu().double().numpy()[:, None]
        hq, hk = orc.rope_apply(hq, ch, sh, inter), orc.rope_apply(hk, ch, sh, inter)
    most = max_len or cap
    for b in range(B):
        mb = T if q_len is None else min(max(q_len[b], 0), T)
        hq[b, :, mb:] = 0
        orc.append(*(x[b] for x in want), hk[b][:, :mb], hv[b][:, :mb], pos[b].tolist(), min(max(lens[b], 0), most))
    assert _near(Qo, hq, sd)
    assert _near(K, want[0], sd)
    assert np.array_equal(V.cpu().double().numpy(), want[1])    # values are copied
    assert np.array_equal(sp.cpu().double().numpy(), want[2]) and np.array_equal(w.cpu().double().numpy(), want[3])
    if q_len is not None:   # rows behind the last token: exactly zero
        for b in range(B):
            assert not Qo[b, :, min(max(q_len[b], 0), T):].any()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 20), (128, 128), (128, 32), (128, 34)])
def test_types_layouts_and_shares(dtype, inter, d, rot):
    _run(dtype, d, rot, inter, 3, 4, 2, 5, 40, [5, 17, 40], [5, 2, 1])


@pytest.mark.parametrize("T,cap,lens,q_len,max_len", [
    (1, 1, [1], None, 0), (1, 9, [0], None, 0), (1, 9, [9], [0], 0),             # the first, no slot at all, no token
    (4, 9, [2, 9], None, 0), (4, 9, [12, -3], None, 0), (4, 9, [9, 9], [7, -2], 0),   # rows in front of the cache; lengths out of range
    (4, 9, [9, 6], None, 6), (33, 64, [33, 64, 40], [33, 31, 1], 0)])
def test_lengths(T, cap, lens, q_len, max_len):
    _run("bf16", 64, 64, False, len(lens), 2, 1, T, cap, lens, q_len, max_len=max_len)


@pytest.mark.parametrize("H,Hk", [(1, 1), (5, 5), (32, 8), (7, 1)])
def test_heads(H, Hk):
    _run("f16", 128, 128, False, 2, H, Hk, 3, 20, [20, 11], None, seed=H)


def test_many_tokens_of_an_odd_number_of_heads():
    _run("bf16", 128, 128, False, 8, 33, 3, 200, 256, [256, 200, 230, 201, 255, 240, 210, 220], [200, 1, 100, 199, 7, 200, 150, 0])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_without_tables_rows_are_copied(dtype):
    _run(dtype, 64, 64, False, 2, 3, 1, 4, 12, [12, 7], [4, 3], turned=False)


def test_the_largest_number_of_sequences_and_rows():
    tc, orc = _tc()
    for B, T in ((65536, 1), (1, 1 << 20)):
        q = torch.randn(B, 1, T, 64, device="cuda").bfloat16()
        c = tc.make_cache(B, 1, 1, 64, tc.TC_BF16, T, T + 1)
        pos = torch.arange(B * T, dtype=torch.int32, device="cuda").view(B, T)
        K, V = torch.zeros(B, 1, T + 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, 1, T + 1, 64, dtype=torch.bfloat16, device="cuda")
        sp, w = torch.full((B, 1, T + 1), -1, dtype=torch.int32, device="cuda"), torch.ones(B, 1, T + 1, device="cuda")
        lens, out = torch.full((B,), T + 1, dtype=torch.int32, device="cuda"), torch.empty_like(q)
        r, co, si = tc.make_rope(64), torch.empty(B, T, 32, device="cuda"), torch.empty(B, T, 32, device="cuda")
        tc.tc_rope_tables(r, pos, co, si)
        tc.tc_cache_append(c, r, q, q, q, co, si, pos, lens, out, K, V, sp, w)
        want = torch.empty_like(q)
        tc.tc_rope_apply(r, q, co, si, want)
        assert torch.equal(out, want) and torch.equal(K[:, :, 1:], want) and torch.equal(V[:, :, 1:], q) and not K[:, :, 0].any()
        assert torch.equal(sp[:, 0, 1:], pos) and not w[:, :, 1:].any() and (w[:, :, 0] == 1).all() and (sp[:, :, 0] == -1).all()
        i = B * T - 1
        wc, ws = orc.rope_tables(np.array([i]), orc.rope_theta(64))
        row = orc.rope_apply(q.view(-1, 64)[i].double().cpu().numpy()[None], wc, ws)
        assert _near(out.view(-1, 64)[i][None], row, torch.bfloat16)


def test_refusals():
    tc, _ = _tc()
    c = tc.make_cache(1, 2, 1, 64, tc.TC_BF16, 2, 8)
    sd = torch.bfloat16
    t = dict(Q=torch.zeros(1, 2, 2, 64, dtype=sd, device="cuda"), K=torch.zeros(1, 1, 2, 64, dtype=sd, device="cuda"),
             V=torch.zeros(1, 1, 2, 64, dtype=sd, device="cuda"), cos=None, sin=None, pos_ids=torch.zeros(1, 2, dtype=torch.int32, device="cuda"),
             lens=torch.ones(1, dtype=torch.int32, device="cuda"), Q_out=torch.zeros(1, 2, 2, 64, dtype=sd, device="cuda"),
             K_cache=torch.zeros(1, 1, 8, 64, dtype=sd, device="cuda"), V_cache=torch.zeros(1, 1, 8, 64, dtype=sd, device="cuda"),
             slot_pos=torch.zeros(1, 1, 8, dtype=torch.int32, device="cuda"), weight=torch.zeros(1, 1, 8, device="cuda"))
    tc.tc_cache_append(c, None, **t)
    for name in t:
        if t[name] is None:
            continue
        for bad in (t[name].cpu(), t[name].double(), t[name][..., :-1] if name != "lens" else t[name][:0]):
            with pytest.raises(ValueError):
                tc.tc_cache_append(c, None, **dict(t, **{name: bad}))
    with pytest.raises(ValueError):   # a cache that is a view
        wide = torch.zeros(1, 1, 8, 128, dtype=sd, device="cuda")
        tc.tc_cache_append(c, None, **dict(t, K_cache=wide[..., :64]))
    with pytest.raises(tc.TokenCarveError):
        tc.tc_cache_append(tc.make_cache(1, 2, 1, 64, tc.TC_BF16, 2, 8, max_len=9), None, **t)
