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


def spread_gradients(kind, rows, rng):
    sign = rng.choice([-1.0, 1.0], rows)
    if kind == "loss scale":                       # a loss scaled up by 2^16, whose rows weigh it from all to 2^-16
        return sign * 2.0 ** 14 * 2.0 ** -np.linspace(0, 16, rows)
    if kind == "two":
        return sign * np.where(np.arange(rows) % 2, 1e-2, 1e3)
    if kind == "past 2^24":
        return sign * np.where(np.arange(rows) % 2, 2e-4, 1e4)
    return sign * np.logspace(-2, 4, rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["log", "loss scale", "two", "past 2^24"])
@pytest.mark.parametrize("rows,width,vocab", [(2, 40, 300), (50, 264, 900), (50, 261, 900), (300, 512, 8192), (2100, 72, 9000)])
def test_rows_whose_gradients_differ_in_size(ext, dtype, kind, rows, width, vocab):
    """With an lse far above the logits all p are 0: each target's row of grad_weight is one term, scale g x, and grad_x
    scale g weight.  G's rounding is given back to e of itself (e e is left, of fp32's parts 2^-21), the product, the scale
    and its kind take 8 u, and the result is rounded once, or by half its type's smallest number (2^-25 in fp16).  In fp16 x
    enters grad_weight with a power of two for each row, such that the largest of all |x g| is above 2^14 times 2^14: what
    that takes below 2^-14 is rounded by 2^-25, which leaves 2^-38 of the largest |x g|."""
    t, e = TYPES[dtype]
    rng = np.random.default_rng(rows)
    x = torch.from_numpy(rng.standard_normal((rows, width))).to(t).cuda()
    w = torch.from_numpy(rng.standard_normal((vocab, width)) / math.sqrt(width)).to(t).cuda()
    y = rng.permutation(vocab)[:rows]
    g = spread_gradients(kind, rows, rng).astype(np.float32)
    scale = 0.75
    far = torch.full((rows,), 400.0, device="cuda")
    gx, gw = ext.linear_logprobs_backward(x, w, torch.from_numpy(y).cuda(), far, far, torch.from_numpy(g).cuda(), scale=scale)
    g, xx, ww = g.astype(np.float64), x.double().cpu().numpy(), w.double().cpu().numpy()
    rest = 2.0 ** -21 if dtype == "fp32" else 1.01 * e * e
    tiny = 2.0 ** -25 if dtype == "fp16" else 2.0 ** -126
    want = scale * g[:, None] * ww[y]
    assert (np.abs(gx.double().cpu().numpy() - want) <= (e + rest + 8 * U) * np.abs(want) + tiny).all()
    want = np.zeros((vocab, width))
    want[y] = scale * g[:, None] * xx
    left = 2.0 ** -38 * scale * np.abs(g[:, None] * xx).max() if dtype == "fp16" else 0.0
    err = np.abs(gw.double().cpu().numpy() - want)
    bound = (e + rest + 8 * U) * np.abs(want) + tiny + left
    assert (err <= bound).all(), (err / bound).max()


def test_rows_of_zeros_and_infinities_in_fp16(ext):
    """What scales fp16's x for grad_weight follows from finite entries: a row of zeros, one of its type's smallest number,
    and one with an infinite entry (in its own column, where weight is negative: its logits are -infinity) leave the others
    exact to the result's rounding (as above)."""
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((30, 64))).half().cuda()
    x[:, 3] = 1.0
    x[4] = 0
    x[5] = 2.0 ** -24
    x[6, 3] = math.inf
    w = torch.from_numpy(rng.standard_normal((200, 64))).half().cuda()
    w[:, 3] = -1.0
    y = torch.arange(30, device="cuda")
    far, g = torch.full((30,), 400.0, device="cuda"), torch.logspace(-3, 0, 30, device="cuda")
    gx, gw = ext.linear_logprobs_backward(x, w, y, far, far, g)
    keep = torch.arange(64, device="cuda") != 3
    want = (g[:, None].double() * x.double())[:, keep]
    left = 2.0 ** -38 * float(want.abs().max())
    err = (gw.double()[:30][:, keep] - want).abs()
    assert (err <= (2.0 ** -11 + 1.01 * 2.0 ** -22 + 8 * U) * want.abs() + 2.0 ** -25 + left).all() and (gw[30:][:, keep] == 0).all()
    for rows in (x[4:5], x[4:5] * 0 + math.nan):      # no finite entry but zeros, or none
        gx, gw = ext.linear_logprobs_backward(rows.contiguous(), w, y[:1], far[:1], far[:1], g[:1])
        assert (gw[0] == 0).all() if rows[0, 0] == 0 else gw[0].isnan().all()


@pytest.mark.parametrize("dtype,width", [("fp32", 4), ("bf16", 5)])
def test_the_largest_launch(ext, dtype, width):
    """8192 rows of 2^25 columns in tiles of 128 rows, which one launch cannot hold.  Logits are exact (whole numbers); lse
    carries (n / 64 + 40) u + 4 u (1 + Z) of the sum of n exponentials and 2 u of itself: n / 64 u = 2^-5."""
    vocab, rows = 1 << 25, 8192
    t = TYPES[dtype][0]
    gen = torch.Generator(device="cuda").manual_seed(5)
    w = (torch.randint(-3, 4, (vocab, width), generator=gen, device="cuda") * 0.5).to(t)
    few = (torch.randint(-3, 4, (4, width), generator=gen, device="cuda") * 0.5).to(t)
    y = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    y[0], y[rows - 1] = vocab - 1, 0
    got = ext.linear_logprobs(few.repeat(rows // 4, 1), w, y)
    torch.cuda.synchronize()
    total = torch.zeros(4, dtype=torch.float64, device="cuda")
    for v0 in range(0, vocab, 1 << 22):
        total += torch.exp(few.double() @ w[v0:v0 + (1 << 22)].double().t().contiguous()).sum(1)
    lse = torch.log(total).repeat(rows // 4)
    z = (few.double().repeat(rows // 4, 1) * w[y].double()).sum(1)
    assert ((got.lse - lse).abs() <= 2.0 ** -5 + 100 * U * (1 + lse.abs())).all()
    assert ((got.logprob - (z - lse)).abs() <= 2.0 ** -5 + 100 * U * (1 + lse.abs() + z.abs())).all()
