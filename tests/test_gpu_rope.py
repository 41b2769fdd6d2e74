"""Rotary positions on the GPU against the float64 oracle: tables at any position and scaling, rows of every type, layout, stride and rotated share."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SCALINGS = [dict(), dict(scaling=1, factor=4.0), dict(scaling=2, factor=3.5), dict(scaling=3, factor=8.0, original_len=8192, low=1.0, high=4.0),
            dict(scaling=3, factor=16.0, original_len=4096, low=0.0, high=32.0, base=500000.0)]


def _tc():
    from oracle import cache_oracle as orc
    from paper_2503_10501_amd import binding as tc
    tc.load_library()
    assert torch.cuda.is_available()
    return tc, orc


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("how", range(len(SCALINGS)))
@pytest.mark.parametrize("rot", [2, 24, 64, 128])
def test_tables_at_any_position(rot, how):
    tc, orc = _tc()
    kw = dict(SCALINGS[how])
    if kw.get("scaling") == 2 and rot == 2:
        pytest.skip("the base is not scaled for a single pair")
    r = tc.make_rope(128, rot_dim=rot, magnitude=1.25 if how == 3 else 0.0, **kw)
    pos = np.concatenate([np.arange(-3, 700), [4095, 32767, 131071, 1 << 24, (1 << 31) - 1, -(1 << 31)]]).astype(np.int32)
    c = torch.full((len(pos), rot // 2), 7.0, device="cuda")
    s = torch.full_like(c, 7.0)
    tc.tc_rope_tables(r, torch.from_numpy(pos).cuda(), c, s)
    m = 1.25 if how == 3 else 1.0
    wc, ws = orc.rope_tables(pos, orc.rope_theta(rot, **kw), m)
    # one rounding of a value of at most m, and the angle: pos theta, theta a few roundings of float64 off (the power's exponent is at
    # most 13: 13 + 3 steps of 2^-53 between the two sides)
    bound = half_step(torch.float32) * m + m * np.abs(pos.astype(np.float64))[:, None] * 32 * 2.0 ** -53
    assert np.all(np.abs(c.cpu().numpy().astype(np.float64) - wc) <= bound)
    assert np.all(np.abs(s.cpu().numpy().astype(np.float64) - ws) <= bound)


def test_many_positions_and_none():
    tc, orc = _tc()
    r = tc.make_rope(64)
    pos = torch.arange(70001, dtype=torch.int32, device="cuda")   # threads with several positions
    c, s = torch.empty(70001, 32, device="cuda"), torch.empty(70001, 32, device="cuda")
    tc.tc_rope_tables(r, pos, c, s)
    wc, ws = orc.rope_tables(np.arange(70001), orc.rope_theta(64))
    assert np.abs(c.cpu().numpy() - wc).max() <= 2.0 ** -24 + 70001 * 2.0 ** -48
    assert np.abs(s.cpu().numpy() - ws).max() <= 2.0 ** -24 + 70001 * 2.0 ** -48
    tc.tc_rope_tables(r, pos[:0], c[:0], s[:0])


def _case(tc, orc, dtype, d, rot, inter, B, H, T, seed, transposed, order):
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, 5000, (B, T), generator=g, dtype=torch.int32)
    r = tc.make_rope(d, rot_dim=rot, layout=int(inter))
    c, s = torch.empty(B, T, rot // 2, device="cuda"), torch.empty(B, T, rot // 2, device="cuda")
    tc.tc_rope_tables(r, pos.cuda(), c, s)
    x = torch.randn(B, H, T, d, generator=g).to(dtype)
    wide = torch.full((B, T, H + 1, d) if order == "token" else (B, H, T + 2, d), 3.0, dtype=dtype, device="cuda")
    xin = wide[:, :, 1:].transpose(1, 2) if order == "token" else wide[:, :, 1:T + 1]
    xin.copy_(x)
    want = orc.rope_apply(x.double().numpy(), c.cpu().double().numpy()[:, None], s.cpu().double().numpy()[:, None], inter, transposed)
    return r, c, s, xin, wide, want


def _near(y, want, dtype):
    # the result's rounding, and those of the two products and the sum in float32 (each at most |x| of the pair, here below 1.5 |y|max of a pair)
    y = y.double().cpu().numpy()
    size = np.abs(want) + 4 * np.sqrt(2.0)   # a pair's elements: |a cos|, |b sin| <= 5.7 for the normal draws used here
    return np.all(np.abs(y - want) <= half_step(dtype) * np.abs(want) + 3 * 2.0 ** -24 * size + (2.0 ** -25 if dtype == torch.float16 else 0))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (64, 2), (64, 24), (64, 40), (128, 128), (128, 20), (128, 96), (128, 126)])
def test_rows_of_every_type_layout_and_share(dtype, inter, d, rot):
    tc, orc = _tc()
    for B, H, T, order, transposed in ((2, 3, 5, "token", False), (1, 1, 1, "head", True), (3, 5, 33, "head", False)):
        r, c, s, x, wide, want = _case(tc, orc, DTYPES[dtype], d, rot, inter, B, H, T, d + rot, transposed, order)
        before = wide.clone()
        y = torch.full((B, T, H, d), 9.0, dtype=DTYPES[dtype], device="cuda").transpose(1, 2)
        tc.tc_rope_apply(r, x, c, s, y, transposed=transposed)
        assert _near(y, want, DTYPES[dtype])
        assert torch.equal(y[..., rot:], x[..., rot:]) and torch.equal(wide, before)   # copies bit for bit, the input as it was
        tc.tc_rope_apply(r, x, c, s, transposed=transposed)                            # in place: the same, and nothing beside it
        assert torch.equal(x, y)
        x.copy_(torch.zeros_like(x))
        before_rows = before[:, :, 1:].transpose(1, 2) if order == "token" else before[:, :, 1:T + 1]
        before_rows.copy_(torch.zeros_like(x))
        assert torch.equal(wide, before)


def test_many_rows_of_an_odd_number_of_heads():
    tc, orc = _tc()
    r, c, s, x, wide, want = _case(tc, orc, torch.bfloat16, 128, 128, False, 4, 33, 300, 3, False, "token")
    y = torch.empty(4, 33, 300, 128, dtype=torch.bfloat16, device="cuda")
    tc.tc_rope_apply(r, x, c, s, y)
    assert _near(y, want, torch.bfloat16)


def test_a_row_for_all_sequences_and_heads():
    tc, orc = _tc()
    r = tc.make_rope(64)
    c, s = torch.empty(2, 3, 32, device="cuda"), torch.empty(2, 3, 32, device="cuda")
    tc.tc_rope_tables(r, torch.tensor([[0, 1, 2], [7, 8, 9]], dtype=torch.int32, device="cuda"), c, s)
    x = torch.randn(1, 1, 3, 64, device="cuda").expand(2, 4, 3, 64)
    y = torch.empty(2, 4, 3, 64, device="cuda")
    tc.tc_rope_apply(r, x, c, s, y)
    want = orc.rope_apply(x.cpu().double().numpy(), c.cpu().double().numpy()[:, None], s.cpu().double().numpy()[:, None])
    assert _near(y, want, torch.float32)
    with pytest.raises(tc.TokenCarveError):   # written rows must differ
        tc.tc_rope_apply(r, y, c, s, x)


@pytest.mark.parametrize("inter", [False, True])
def test_transposed_is_the_gradient_by_formula_and_by_differences(inter):
    tc, orc = _tc()
    B, H, T, d, rot = 1, 2, 3, 64, 20
    r, c, s, x, wide, want = _case(tc, orc, torch.float32, d, rot, inter, B, H, T, 5, False, "head")
    g = torch.randn(B, H, T, d, device="cuda")
    dx, y = torch.empty_like(g), torch.empty_like(g)
    tc.tc_rope_apply(r, g, c, s, dx, transposed=True)
    # <g, R e> for each unit vector e, R linear: differences of the forward pass without a step's error
    eye = torch.zeros(d, H, T, d, device="cuda")
    eye[torch.arange(d), :, :, torch.arange(d)] = 1.0
    ye = torch.empty_like(eye)
    tc.tc_rope_apply(r, eye, c.expand(d, T, rot // 2).contiguous(), s.expand(d, T, rot // 2).contiguous(), ye)
    by_difference = (ye.double() * g.double()).sum(-1).permute(1, 2, 0)[None]
    assert (dx.double() - by_difference).abs().max() <= 4 * 2.0 ** -24 * 2 * g.abs().max()
    formula = orc.rope_apply(g.cpu().double().numpy(), c.cpu().double().numpy()[:, None], s.cpu().double().numpy()[:, None], inter, True)
    assert _near(dx, formula, torch.float32)
    # there and back again: magnitude 1, so the transposed turn undoes the turn
    tc.tc_rope_apply(r, x, c, s, y)
    tc.tc_rope_apply(r, y, c, s, y, transposed=True)
    assert (y - x).abs().max() <= 8 * 2.0 ** -24 * x.abs().max()


def test_positions_kept_by_the_compression_turn_as_its_tables_say():
    """The tables of tc_assemble_sequence are those of tc_rope_tables at its position ids."""
    tc, orc = _tc()
    from workloads import CONFIGS
    w = CONFIGS["tiny"]
    p = tc.params_for(w, batch=2)
    Ln = w.seq_len - w.n_vis + w.k_final
    H = torch.randn(2, w.seq_len, w.hidden, device="cuda")
    X = torch.randn(2, w.k_final, w.hidden, device="cuda")
    kept = torch.stack([torch.randperm(w.n_vis)[:w.k_final].sort().values for _ in range(2)]).to(torch.int32).cuda()
    Hn, pos = torch.empty(2, Ln, w.hidden, device="cuda"), torch.empty(2, Ln, dtype=torch.int32, device="cuda")
    c0, s0 = torch.empty(2, Ln, 32, device="cuda"), torch.empty(2, Ln, 32, device="cuda")
    tc.tc_assemble_sequence(p, H, X, kept, Hn, pos, 10000.0, c0, s0)
    c, s = torch.empty_like(c0), torch.empty_like(s0)
    tc.tc_rope_tables(tc.make_rope(64), pos, c, s)
    assert (c - c0).abs().max() <= 2.0 ** -24 and (s - s0).abs().max() <= 2.0 ** -24


def test_captured_calls_on_a_stream_of_their_own():
    tc, orc = _tc()
    r = tc.make_rope(128)
    pos = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    x = torch.randn(2, 4, 1, 128, device="cuda").bfloat16()
    c, s, y = torch.empty(2, 1, 64, device="cuda"), torch.empty(2, 1, 64, device="cuda"), torch.empty_like(x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        tc.tc_rope_tables(r, pos, c, s)
        tc.tc_rope_apply(r, x, c, s, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pos.add_(1)
        tc.tc_rope_tables(r, pos, c, s)
        tc.tc_rope_apply(r, x, c, s, y)
    for step in range(1, 4):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert int(pos[0, 0]) == step
        wc, ws = orc.rope_tables(pos.cpu().numpy(), orc.rope_theta(128))
        want = orc.rope_apply(x.double().cpu().numpy(), wc[:, None], ws[:, None])
        assert _near(y, want, torch.bfloat16)


def test_tensors_that_do_not_fit_are_refused():
    tc, _ = _tc()
    r = tc.make_rope(64)
    x = torch.zeros(2, 3, 5, 64, device="cuda")
    c = torch.zeros(2, 5, 32, device="cuda")
    for bad in ((x.half(), c, c, x), (x, c[:, :4], c, x), (x, c.double(), c, x), (x[..., :32], c, c, x[..., :32]), (x, c, c, x[:, :2]),
                (x, c.cpu(), c, x), (x.cpu(), c, c, x), (x.double(), c, c, x.double()), (x.transpose(2, 3), c, c, x)):
        with pytest.raises(ValueError):
            tc.tc_rope_apply(r, *bad)
    odd = torch.zeros(2, 3, 5, 66, device="cuda")[..., :64]   # rows of 264 bytes
    for bad in ((odd, x), (x, odd)):
        with pytest.raises(tc.TokenCarveError) as e:
            tc.tc_rope_apply(r, bad[0], c, c, bad[1])
        assert e.value.status == -2
    with pytest.raises(tc.TokenCarveError) as e:   # in place with other strides
        tc.tc_rope_apply(r, x, c, c, x.view(3, 2, 5, 64).transpose(0, 1))
    assert e.value.status == -4
    with pytest.raises(ValueError):
        tc.tc_rope_tables(r, torch.zeros(4, dtype=torch.int64, device="cuda"), c[0, :4], c[0, :4])
    tc.tc_rope_apply(r, x[:0], c[:0], c[:0], x[:0])
    tc.tc_rope_apply(r, x[:, :, :0], c[:, :0], c[:, :0], x[:, :, :0])
