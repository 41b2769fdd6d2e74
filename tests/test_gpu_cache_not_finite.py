"""Infinities and NaN among the values that attention over the cache reads: they reach every row that sees them, in the element they are in, and nothing else."""
import pytest
import torch

from tests.test_gpu_cache_attention import call, make

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def planted(s, spots):
    """Plants (tensor, sequence or image, key, element, value) in all heads and returns, per output, the sum of what its row sees of them (0: nothing)."""
    c = s["c"]
    B, T, H, d = c.batch, c.n_query, c.n_heads, c.head_dim
    seen = torch.zeros(B, T, H, d)
    t = torch.arange(T)
    for name, i, key, e, value in spots:
        s[name][i, :, key, e] = value
        for b in range(B):
            n, m = int(s["lens"][b]), T if s["q_len"] is None else int(s["q_len"][b])
            if name == "Vp":
                rows = (t < m) & (b // (B // c.n_prefixes) == i)
            else:
                rows = (t < m) & (key <= n - m + t) & (b == i)
            seen[b, rows, :, e] += value
    return seen.cuda()


def compare(build, spots, before=None):
    """Outputs and weights with the values and without: what sees none of them is the same bit by bit."""
    s, t = build(), build()
    if before is not None:
        before(s)
        before(t)
    seen = planted(t, spots)
    call(s)
    call(t)
    torch.cuda.synchronize()
    clean, got = (x["O"].view(seen.shape) for x in (s, t))
    assert clean.isfinite().all()
    touched = seen != 0     # (NaN too)
    assert touched.any() and torch.equal(got[~touched], clean[~touched])
    hit, want = got[touched].float(), seen[touched]
    lost = torch.where(want.isnan(), ~hit.isnan(), hit != want)
    assert not lost.any(), "%d of %d" % (int(lost.sum()), lost.numel())
    if s["w"] is not None:
        assert torch.equal(s["w"], t["w"])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("T,n,P,spot", [
    (20, 30, 40, ("Vp", 3)), (60, 70, 40, ("Vp", 3)), (20, 30, 100, ("Vp", 70)),         # a prefix that ends inside a tile, two wavefronts share its keys
    (60, 90, 0, ("V", 5)), (40, 90, 100, ("V", 10)), (40, 90, 100, ("Vp", 95)),          # slots that the first rows of a tile do not see all of
    (128, 256, 0, ("V", 140)), (128, 228, 0, ("V", 70)), (128, 228, 0, ("V", 101)),      # 128 rows: wavefronts of rows that see the tile whole
    (300, 340, 33, ("V", 200)), (300, 340, 33, ("V", 339)), (576, 640, 0, ("V", 77))])
def test_many_rows_that_see_a_tile_whole_beside_rows_that_do_not(dtype, d, value, T, n, P, spot):
    compare(lambda: make(dtype, d, 2, 1, 1, T, n + 5, [n, n - 3], [T, T - 2], images=1 if P else 0, P=P, seed=T), [(spot[0], 0, spot[1], 11, value)])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,T,G", [(64, 40, 1), (64, 100, 1), (128, 40, 1), (64, 25, 4), (128, 300, 2)])
@pytest.mark.parametrize("B,Hk", [(2, 2), (16, 32)])
def test_many_rows_and_several_values_at_once(dtype, d, T, G, B, Hk):
    # infinities of both signs in one element are no number, in others they stay apart; keys in parts (few heads) and in one part
    n = T + 140
    spots = [("Vp", 0, 3, 0, INF), ("V", 0, 70, 1, -INF), ("V", 0, n - T + 2, 1, -INF), ("V", 0, n - 1, 2, NAN), ("V", 1, 100, 3, INF),
             ("V", 1, n - T + 5, 3, -INF), ("Vp", 0, 50, d - 1, -INF)]
    compare(lambda: make(dtype, d, B, G * Hk, Hk, T, n, [n] * B, images=2, P=52, seed=d), spots)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("T,n,P,spots", [
    (1, 300, 0, [("V", 0), ("V", 299)]), (1, 300, 0, [("V", 70)]), (1, 8, 200, [("Vp", 5)]), (1, 8, 200, [("Vp", 199)]), (3, 130, 40, [("Vp", 33), ("V", 129)]),
    (16, 90, 0, [("V", 40)]), (16, 90, 70, [("V", 80), ("Vp", 64)]), (1, 7000, 0, [("V", 4000)]), (5, 7000, 100, [("Vp", 10)])])
def test_few_rows_wherever_the_value_lies(dtype, d, value, T, n, P, spots):
    # a tile that all rows see whole, one that they do not, keys of one workgroup and in parts
    spots = [(name, 0, key, 3 + i, value) for i, (name, key) in enumerate(spots)]
    compare(lambda: make(dtype, d, 2, 2, 1, T, n, [n, n - 1], images=1 if P else 0, P=P, seed=n), spots)


@pytest.mark.parametrize("dtype,d,each,T", [("bf16", 128, 20, 1), ("bf16", 128, 7, 2), ("f16", 64, 40, 2), ("f32", 64, 20, 1)])
def test_a_prefix_that_is_read_once(dtype, d, each, T):
    P, Hk = 1200, 16
    assert 2 * (each - 1) * Hk * P * d * 2 * torch.finfo({"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]).bits // 8 >= 32e6
    g = torch.Generator().manual_seed(each)
    lens = [int(x) for x in torch.randint(T, 60, (2 * each,), generator=g)]
    spots = [("Vp", 0, 5, 0, INF), ("Vp", 1, 700, 1, NAN), ("Vp", 1, P - 1, 2, -INF), ("V", 3, 0, 3, INF), ("Vp", 0, 9, 3, -INF)]
    compare(lambda: make(dtype, d, 2 * each, Hk, Hk, T, 60, lens, images=2, P=P, seed=each), spots)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,n,P", [(1, 300, 0), (4, 90, 200), (1, 7000, 0), (40, 300, 0), (40, 90, 100), (200, 700, 0)])
@pytest.mark.parametrize("rising", [True, False])
def test_however_small_its_probability_is(dtype, T, n, P, rising):
    """Scores along the keys rise or fall by 640, so that probabilities of float32 are 0 at one end, and what was summed there is scaled to 0 on the way."""
    def ramp(s):
        s["Q"].zero_()
        s["Q"][..., 0] = 64.0
        for name, keys in (("Kp", P), ("K", n)):
            if keys:
                x = torch.linspace(-40.0, 40.0, P + n)[:P] if name == "Kp" else torch.linspace(-40.0, 40.0, P + n)[P:]
                s[name][..., :keys, 0] = (x if rising else -x).to(s[name].dtype).cuda()
    spots = [("V", 0, 2, 0, INF), ("V", 0, n - T, 1, -INF), ("V", 1, n // 2 - T, 2, NAN)] + ([("Vp", 0, 7, 3, INF), ("Vp", 0, P - 1, 4, -INF)] if P else [])
    compare(lambda: make(dtype, 64, 2, 2, 2, T, n, [n, n], images=1 if P else 0, P=P, seed=n), spots, ramp)
