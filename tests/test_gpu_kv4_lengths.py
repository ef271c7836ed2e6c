"""GPU parity of attention over the last tokens of a sequence of 2^31 - 1 whose
other pages are none, and over the same tokens as a short sequence, with the
definition in 64 bits on the values that the cache holds (u = 2^-24).

Tolerance: z_j = scale q k_j is a sum of G groups of exact whole numbers: with
A = the largest scale sum |q k_j|, q's 2^-31 and the groups' and the factor's
roundings, d = (G + 5) u A.  With Z = the largest |z|, a difference to a reference (2 Z),
the exponential and the value's scale leave a weight within eps = d + 2 u Z + 6 u of
itself.  A sum takes two roundings for each of a wave's tiles of 64 tokens (2047 are 32,
were they all one wave's), each of the 4 waves and each part that holds tokens (at most
33): n = 64 + 8 + 66.  So a result of terms of absolute sum S is within
(2 eps + n u) S + 2 u of itself, and the lse within eps + n u + 2 u |lse|."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_fp32_at_the_end_of_32_bits(dim):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13511_amd import binding as ext
    page, heads, n, short = 1024, 32, (1 << 31) - 1, 2047
    rng = np.random.default_rng(dim + 1)
    cuda = lambda x, t: torch.from_numpy(np.asarray(x)).to(t).cuda()
    cache = ext.kv4_cache(2, 1, dim, page)
    table, lens, far_lens = cuda([[1, 0]], torch.int32), cuda([short], torch.int32), cuda([n], torch.int32)
    far = torch.full((1, 1 << 21), -1, dtype=torch.int32, device="cuda")
    far[0, -2:] = table[0]
    every = cuda([0, short], torch.int32)
    k, v = (cuda(rng.standard_normal((short, 1, dim)), torch.float32) for _ in range(2))
    ext.kv4_append(cache, k, v, table, lens, starts=every)
    k, v = (x[:, 0].double().cpu().numpy() for x in ext.kv4_read(cache, table, lens, dim, starts=every, tokens=short))
    q = rng.standard_normal((1, heads, dim)).astype(np.float32)
    z = q[0].astype(np.float64) @ k.T / math.sqrt(dim)
    w = np.exp(z - z.max(-1, keepdims=True))
    lse, w = np.log(w.sum(-1)) + z.max(-1), w / w.sum(-1, keepdims=True)
    want, S = w @ v, w @ np.abs(v)
    A = (np.abs(q[0].astype(np.float64)) @ np.abs(k).T / math.sqrt(dim)).max(-1)
    eps = (dim / 64 + 5) * U * A + 2 * U * np.abs(z).max(-1) + 6 * U
    adds = (64 + 8 + 66) * U
    for t, l in ((far, far_lens), (table, lens)):
        out, got = ext.kv4_attention(cache, cuda(q, torch.float32), t, l, starts=cuda([0, 1], torch.int32), max_new=1, max_len=10 ** 6)
        torch.cuda.synchronize()
        err = np.abs(out[0].double().cpu().numpy() - want)
        bound = (2 * eps[:, None] + adds) * S + 2 * U * np.abs(want)
        assert (err <= bound).all(), (err / bound).max()
        assert (np.abs(got[0].double().cpu().numpy() - lse) <= eps + adds + 2 * U * np.abs(lse)).all()
