"""Where probabilities enter the products as a head and a remainder, the outputs are held to that; rounded once only where the rows of a tile are more than 16."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from tests.test_gpu_cache_attention import DTYPES, call, make


def bound_of(dtype, d, G, T, each, images, Hk, q, K, V, n, m, Kp, Vp, scale):
    """Half a step of O; of the probabilities, by how the rows are tiled: G T rows of a sequence, or, where these are 16 at most and re-reading the prefix
    would take 32 MB and more, at the prefix the rows of all sequences of an image.  Tiles of up to 16 rows: a remainder of at most h p is rounded, h h p; larger ones:
    h p.  Scores: d + 4 roundings of float32 of at most scale sum |q k|, in numerator and sum; 2^-20 for exponentials and sums; half storage: 2^-25
    for each probability below its normal numbers."""
    sd = DTYPES[dtype]
    h = torch.finfo(sd).eps / 2
    want, _ = orc.attention(q, K, V, n, m, Kp, Vp, scale)
    A, _ = orc.attention(q, K, np.abs(V), n, m, Kp, None if Vp is None else np.abs(Vp), scale)
    once = 0.0 * A
    packed = Vp is not None and G * T <= 16 and images * (each - 1) * Hk * Vp.shape[1] * d * 2.0 * torch.finfo(sd).bits / 8 >= 32e6
    if G * T > 16:
        once = A
    elif packed and each * G * T > 16:
        once, _ = orc.attention(q, K, 0 * V, n, m, Kp, np.abs(Vp), scale)   # the prefix's share
    keys = K if Kp is None else np.concatenate([Kp, K], axis=1)
    es = 0.0 if m == 0 or keys.shape[1] == 0 else 2.0 ** -24 * (d + 4) * scale * max(np.abs(q[x, :m]).dot(np.abs(keys[x // G]).T).max() for x in range(q.shape[0]))
    bound = h * np.abs(want) + 2 * (es + 2.0 ** -20) * A
    if sd != torch.float32:
        bound = bound + h * h * A + h * once
    if sd == torch.float16:
        vals = V if Vp is None else np.concatenate([Vp, V], axis=1)
        bound = bound + 2.0 ** -25 * (1 + np.abs(vals).sum(1).max())
    return want, bound


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("d,G,T,each,images,Hk,P,n", [
    (64, 1, 1, 40, 2, 1, 70, 60), (64, 2, 2, 21, 2, 1, 70, 60), (128, 2, 8, 5, 2, 1, 41, 90), (64, 1, 16, 9, 1, 2, 130, 40),     # read once for each sequence
    (64, 1, 1, 12, 2, 16, 1000, 50), (128, 1, 2, 5, 2, 16, 900, 40),                                                          # once for all, up to 16 rows
    (64, 1, 2, 24, 2, 16, 1000, 50), (128, 2, 3, 7, 2, 16, 900, 40),                                                          # ... and more
    (64, 1, 3, 2, 2, 2, 0, 500), (128, 4, 4, 2, 1, 1, 0, 3000), (64, 1, 17, 2, 1, 1, 33, 90)])
def test_outputs_are_as_exact_as_their_tiles(dtype, d, G, T, each, images, Hk, P, n):
    B = each * images
    g = np.random.default_rng(each + T)
    lens, q_len = [int(x) for x in g.integers(T, n + 1, B)], [int(x) for x in g.integers(1, T + 1, B)]
    s = make(dtype, d, B, G * Hk, Hk, T, n, lens, q_len, images=images if P else 0, P=P, seed=d + T)
    call(s)
    torch.cuda.synchronize()
    host = {k: None if s[k] is None else s[k].cpu().double().numpy() for k in ("Q", "K", "V", "Kp", "Vp", "O")}
    for b in range(B):
        i = b // each
        want, bound = bound_of(dtype, d, G, T, each, images, Hk, host["Q"][b], host["K"][b, :, :lens[b]], host["V"][b, :, :lens[b]], lens[b], q_len[b],
                               host["Kp"][i] if P else None, host["Vp"][i] if P else None, 1.0 / np.sqrt(d))
        off = np.abs(host["O"][b].reshape(T, G * Hk, d) - want)
        assert np.all(off <= bound), (b, np.max(off / np.maximum(bound, 1e-30)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P", [0, 70])
def test_probabilities_rounded_once_fall_outside_the_bound_of_small_tiles(dtype, P):
    """The mistake planted in the oracle: rows of 60 slots and a prefix, probabilities (scaled as the largest is, to its power of two) rounded to 16 bits."""
    sd, d = DTYPES[dtype], 64
    g = torch.Generator().manual_seed(P)
    normal = lambda *shape: torch.randn(*shape, generator=g).to(sd).double().numpy()  # noqa: E731
    q, K, V = normal(2, 1, d), normal(1, 60, d), normal(1, 60, d)
    Kp, Vp = (normal(1, P, d), normal(1, P, d)) if P else (None, None)
    want, bound = bound_of(dtype, d, 2, 1, 8, 1, 1, q, K, V, 60, 1, Kp, Vp, 1.0 / np.sqrt(d))
    keys, vals = (K[0], V[0]) if P == 0 else (np.concatenate([Kp[0], K[0]]), np.concatenate([Vp[0], V[0]]))
    s = q[:, 0] @ keys.T / np.sqrt(d)
    p = np.exp(s - s.max(1, keepdims=True))
    once = torch.from_numpy(p).to(sd).double().numpy()
    good = torch.from_numpy((p / p.sum(1, keepdims=True)) @ vals).to(sd).double().numpy()
    bad = torch.from_numpy((once @ vals) / p.sum(1, keepdims=True)).to(sd).double().numpy()
    assert np.all(np.abs(good - want[0]) <= bound[0]) and not np.all(np.abs(bad - want[0]) <= bound[0])
