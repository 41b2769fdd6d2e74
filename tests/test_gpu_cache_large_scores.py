"""Finite queries and keys whose scores are far beyond what a softmax in float32 can tell apart: equal keys share the attention, and nothing becomes infinite or NaN."""
import pytest
import torch

from tests.test_gpu_cache_attention import DTYPES, call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,size", [("f16", x) for x in (100.0, 700.0, 1100.0, 1500.0, 3000.0, 9000.0, 30000.0, 65000.0)] +
                         [(t, x) for t in ("bf16", "f32") for x in (100.0, 3e3, 1e4, 3e4, 1e5, 1e8, 1e12, 1e16)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("T,n", [(1, 300), (3, 5000), (40, 340), (200, 500), (20, 4000)])
def test_equal_keys_of_any_size_share_the_attention(dtype, size, sign, T, n):
    """Four keys have scores of 64 size^2 / 8 and all others 0 (sign > 0), or all others minus that (sign < 0): what the rest has of the attention is
    2^-50000 and less.  The mean of four values: probabilities of a quarter, whose power of two is exact, times values of at most 6, and the output's rounding.
    (Size 100: scores of 115416 in base 2, whose product is off by up to 2^-8 from the rounded maximum.  Tiles of more than 16 rows form probabilities of it,
    2^x for x up to 2^-8 beside a whole number: no powers of two, so they round to 16 bits, half a step each, h times the mean of |v|.)"""
    sd = DTYPES[dtype]
    for seed in range(6):
        s = make(dtype, 64, 2, 2, 1, T, n, [n, n - 1], seed=seed)
        at = torch.tensor([3, 77, 150, n - T - 2], device="cuda")
        q = min(size * (1 + 0.03 * seed), float(torch.finfo(torch.float16).max)) if dtype == "f16" else size * (1 + 0.03 * seed)
        s["Q"].fill_(q)
        s["K"].fill_(0.0 if sign > 0 else -size)
        s["K"][:, :, at] = size if sign > 0 else 0.0
        s["w"].zero_()
        call(s)
        torch.cuda.synchronize()
        v = s["V"][:, 0, at].double()
        want = v.mean(1)[:, None, None]
        got = s["O"].double().view(2, T, 2, 64)
        rounded = torch.finfo(sd).eps / 2 * v.abs().mean(1)[:, None, None] if dtype != "f32" and 2 * T > 16 and size == 100.0 else 0.0
        assert ((got - want).abs() <= torch.finfo(sd).eps / 2 * want.abs() + rounded + 2.0 ** -20 * 6).all(), (seed, (got - want).abs().max())
        assert s["w"].isfinite().all() and (s["w"] >= 0).all() and (s["w"] <= 2 * T).all()   # a probability for each of 2 T rows at most
