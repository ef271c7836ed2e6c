"""GPU parity of the head's operators where sizes, addresses or types come to
their limits, with the same definitions in 64 bits (u = 2^-24)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


@pytest.fixture(scope="module")
def ext():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13511_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1 << 24), (3, (1 << 24) + 13)])
def test_rows_of_G_past_31_bits(ext, dtype, rows, vocab):
    """Few rows of a vocabulary whose G lies in one piece: 64 rows of it are more than 2^31 bytes.

    Logits are exact but for the scale (whole numbers), p carries (n / 64 + 40) u + 8 u (Z + |lse|) < 0.02 of itself
    (n / 64 u = 2^-6 alone is what a plain order may lose); G is rounded to e of itself, an entry of grad_weight is a sum of
    at most three terms, rounded once."""
    rng = np.random.default_rng(rows)
    t, e = TYPES[dtype]
    x = torch.from_numpy(rng.integers(-3, 4, (rows, 16)) * 0.25).to(t).cuda()
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = (torch.randint(-3, 4, (vocab, 16), generator=gen, device="cuda") * 0.125).to(t)
    y = torch.from_numpy(np.array([vocab - 1, 5, 1 << 23][:rows])).cuda()
    g = torch.from_numpy(-rng.uniform(0.5, 1.0, rows).astype(np.float32)).cuda()
    got = ext.linear_logprobs(x, w, y)
    _, gw = ext.linear_logprobs_backward(x, w, y, got.lse, got.entropy, g, need_x=False)
    torch.cuda.synchronize()
    for v0 in range(0, vocab, 1 << 22):
        part = w[v0:v0 + (1 << 22)].double()
        p = torch.exp(x.double() @ part.t().contiguous() - got.lse.double()[:, None])
        G = -g.double()[:, None] * p
        for r in range(rows):
            if v0 <= y[r] < v0 + len(part):
                G[r, y[r] - v0] += g[r].double()
        want, size = G.t().contiguous() @ x.double(), G.abs().t().contiguous() @ x.double().abs()
        err = (gw[v0:v0 + (1 << 22)].double() - want).abs()
        assert (err <= e * 1.01 * want.abs() + (e * 1.01 + 0.02) * size + 2.0 ** -25).all(), v0
