"""GPU parity of the log probabilities of given tokens and their gradient
(externd_token_logprobs, _backward) with the oracle's fp64 form.

Tolerance (u = 2^-24, Z the largest finite |scale x| of the row, n its
length): z = scale x is rounded once (u Z), its difference to the maximum
once more (2 u Z), the exponential is within 4 u, and at least 64 partial
sums are joined by a tree: a sum of n exponentials carries s = 4 u + 4 u Z +
(n / 64 + 24) u of itself, so lse moves by s + 2 u Z + u |lse|, a log
probability by u Z more, and the entropy, whose sum weighs each term with up
to 2 Z beside the maximum, by (2 + 4 Z) s + 4 u Z.  Gradients: p carries
s + 6 u Z, ln p + entropy moves by the sum of the two bounds above, and the
result is rounded once to its type."""
import math

import numpy as np
import pytest

import oracle.decode_oracle as ref

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


def bounds(z, n, lse):
    Z = np.max(np.where(np.isfinite(z), np.abs(z), 0), -1)
    s = 4 * U + 4 * U * Z + (n / 64 + 24) * U
    dl = s + 2 * U * Z + U * np.where(np.isfinite(lse), np.abs(lse), 0)
    return Z, s, dl, dl + U * Z, (2 + 4 * Z) * s + 4 * U * Z


def near(got, want, tol):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    ok = np.isfinite(want)
    assert np.array_equal(got[~ok & ~np.isnan(want)], want[~ok & ~np.isnan(want)])
    assert np.all(np.abs(got - want)[ok] <= np.broadcast_to(tol, want.shape)[ok]), np.max(np.abs(got - want)[ok])


def make(rows, n, dtype, seed=0, ties=False):
    rng = np.random.default_rng(seed)
    x = 3 * rng.standard_normal((rows, n))
    if ties:
        x = np.round(x)                              # a handful of distinct logits: most of the best are equal
    y = rng.integers(0, n, rows)
    y[rng.random(rows) < 0.2] = -1
    return torch.from_numpy(x).to(TYPES[dtype][0]).cuda(), torch.from_numpy(y).cuda()


def check(ext, x, y, top, scale=1.0):
    got = ext.token_logprobs(x, y, top=top, scale=scale)
    torch.cuda.synchronize()
    X, n = x.double().cpu().numpy(), x.shape[1]
    s32 = float(np.float32(scale))
    lp, h, lse, tl, ti, _ = ref.logprobs(X, y.cpu().numpy(), s32, top)
    _, _, dl, dp, dh = bounds(s32 * X, n, lse)
    near(got.lse, lse, dl)
    near(got.logprob, lp, dp)
    near(got.entropy, h, dh)
    near(got.top_logprobs, tl, dp[:, None])
    assert got.top_ids.dtype is torch.int64 and np.array_equal(got.top_ids.cpu().numpy(), ti)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,top", [
    (1, 1, 1), (3, 2, 2), (2, 63, 5), (5, 64, 64), (4, 65, 1), (7, 1000, 20), (300, 129, 3), (1, 65537, 64), (9, 32000, 33),
    (2, 40001, 0), (1, 8192, 8), (2, 8191, 8), (6, 10007, 10), (1030, 777, 5), (64, 20003, 2)])
def test_matches_oracle(ext, dtype, rows, n, top):
    check(ext, *make(rows, n, dtype), top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,top", [(4, 5000, 40), (2, 70, 64), (1, 40003, 64), (3, 64, 7)])
def test_ties_go_to_the_lowest_index(ext, dtype, rows, n, top):
    check(ext, *make(rows, n, dtype, ties=True), top)
    x = torch.zeros((rows, n), device="cuda", dtype=TYPES[dtype][0])
    x[:, ::3] = -0.0                                  # equal to zero
    got = ext.token_logprobs(x, top=top)
    assert got.logprob is None
    assert torch.equal(got.top_ids, torch.arange(top, device="cuda").expand(rows, top))


@pytest.mark.parametrize("dtype", TYPES)
def test_orders_that_keep_the_list_busy(ext, dtype):
    """Rising logits (every one enters the list) and falling ones, the largest last or first in each stretch."""
    n = 20000
    up = torch.arange(n, device="cuda", dtype=torch.float32) * 1e-3
    for x in (up, up.flip(0), up.view(100, 200).t().reshape(-1)):
        x = x.to(TYPES[dtype][0])[None].contiguous()
        check(ext, x, torch.tensor([5], device="cuda"), 64)


@pytest.mark.parametrize("dtype", TYPES)
def test_masks_and_nonfinite(ext, dtype):
    """Masked logits (-infinity, and the type's lowest value), rows with one or no logit left, infinities and NaN."""
    t = TYPES[dtype][0]
    x, _ = make(8, 3001, dtype, 3)
    x[0, 100:] = -math.inf
    x[1, :] = -math.inf
    x[1, 2999] = 2.0
    x[2, :] = -math.inf
    x[3, 10:] = torch.finfo(t).min
    x[4, 7] = math.nan
    x[5, 8] = math.inf
    x[6, :] = torch.finfo(t).min
    y = torch.tensor([50, 2999, 4, 3, 0, 8, 12, -1], device="cuda")
    got = ext.token_logprobs(x, y, top=6)
    X = x.double().cpu().numpy()
    keep = [0, 1, 3, 7] if dtype != "fp16" else [0, 1, 3, 6, 7]       # the lowest fp16 value is an ordinary number
    lp, h, lse, tl, ti, _ = ref.logprobs(X[keep], y.cpu().numpy()[keep], 1.0, 6)
    _, _, dl, dp, dh = bounds(np.where(X[keep] < -1e4, 0, X[keep]), 3001, lse)      # entries below leave no trace
    for i, r in enumerate(keep):
        if r == 6:
            continue
        assert abs(got.lse[r].item() - lse[i]) <= dl[i] and abs(got.logprob[r].item() - lp[i]) <= dp[i]
        assert abs(got.entropy[r].item() - h[i]) <= dh[i]
        assert got.top_ids[r].tolist() == ti[i].tolist()
    assert got.entropy[1].item() == 0.0 and got.logprob[1].item() == 0.0
    assert torch.isneginf(got.top_logprobs[1, 1:]).all()
    # nothing left
    assert got.lse[2].item() == -math.inf and got.logprob[2].item() == -math.inf and got.entropy[2].item() == 0.0
    assert torch.isneginf(got.top_logprobs[2]).all() and got.top_ids[2].tolist() == [0, 1, 2, 3, 4, 5]
    for r in (4, 5):
        assert all(math.isnan(v[r].item()) for v in (got.lse, got.logprob, got.entropy)) and torch.isnan(got.top_logprobs[r]).all()
    assert got.top_ids[4, 0].item() == 7 and got.top_ids[5, 0].item() == 8
    # all equal at the lowest value: uniform
    assert abs(got.entropy[6].item() - math.log(3001)) <= (2 + 4) * (3001 / 64 + 40) * U
    # targets outside
    y = torch.tensor([3001, 1 << 40, -1, -(1 << 40), 5, 5, 5, 3000], device="cuda")
    got = ext.token_logprobs(x, y)
    assert math.isnan(got.logprob[0].item()) and math.isnan(got.logprob[1].item())
    assert got.logprob[2].item() == 0.0 and got.logprob[3].item() == 0.0 and math.isfinite(got.logprob[7].item())


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_scale_and_alignment(ext, dtype):
    x, y = make(9, 1300, dtype, 4)
    for view in (x[:, 1:1200], x[::2, 3:1300], x[:, :1299], x[1:2, 5:]):
        yy = y[:view.shape[0]].clamp(max=view.shape[1] - 1)
        check(ext, view, yy, 7, scale=0.7)
        check(ext, view, yy, 7, scale=3.0)


def test_same_bits_every_time_and_on_other_streams(ext):
    for rows, n in ((1, 100003), (40, 5003)):
        x, y = make(rows, n, "bf16", 8)
        a = ext.token_logprobs(x, y, top=16)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            b = ext.token_logprobs(x, y, top=16)
        s.synchronize()
        for f in ("logprob", "entropy", "lse", "top_logprobs", "top_ids"):
            assert torch.equal(getattr(a, f), getattr(b, f)), f
        ws = torch.empty(max(256, ext.lib().externd_token_logprobs_workspace_bytes(rows, n, 16)), dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c = ext.token_logprobs(x, y, top=16, workspace=ws)
        for _ in range(3):
            x.normal_()
            g.replay()
            torch.cuda.synchronize()
            d = ext.token_logprobs(x, y, top=16)
            assert torch.equal(c.logprob, d.logprob) and torch.equal(c.top_ids, d.top_ids) and torch.equal(c.entropy, d.entropy)


# ---------------------------------------------------------------------------
# gradient
# ---------------------------------------------------------------------------
def check_backward(ext, x, y, g, ge, scale, unit, **kw):
    fwd = ext.token_logprobs(x, y, scale=scale)
    X, Y = x.double().cpu().numpy(), y.cpu().numpy()
    s32 = float(np.float32(scale))
    zero = np.zeros(len(Y))
    G, E = (zero if v is None else v.double().cpu().numpy() for v in (g, ge))
    want = ref.logprobs_backward(X, Y, s32, G, E)
    _, h, lse, _, _, p = ref.logprobs(X, Y, s32, 0)
    Z, s, dl, dp, dh = bounds(s32 * X, x.shape[1], lse)
    got = ext.token_logprobs_backward(x, y, fwd.lse, fwd.entropy, g, ge, scale=scale, **kw).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        lp = np.where(p > 0, np.abs(s32 * X - lse[:, None]), 0)
    part = np.abs(G)[:, None] + np.abs(E)[:, None] * (lp + np.abs(h)[:, None])
    bound = s32 * (p * part * (s + dl + 8 * U * (1 + Z))[:, None] + p * (np.abs(E) * (dp + dh))[:, None]
                   + 4 * U * (np.abs(G)[:, None] + p * part)) + unit * np.abs(want) + (2.0 ** -25 if unit == 2.0 ** -11 else 1e-38)
    assert np.all(np.abs(got - want) <= bound)
    return fwd


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (2, 64), (5, 1001), (70, 513), (2, 40001), (3, 8192)])
def test_gradient_matches_oracle(ext, dtype, rows, n):
    x, y = make(rows, n, dtype, 1)
    g, ge = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    unit = TYPES[dtype][1]
    fwd = check_backward(ext, x, y, g, ge, 0.8, unit)
    check_backward(ext, x, y, g, None, 1.0, unit)
    check_backward(ext, x, y, None, ge, 1.0, unit)
    # into the logits themselves, and into a slice: the same bits
    want = ext.token_logprobs_backward(x, y, fwd.lse, fwd.entropy, g, ge, scale=0.8)
    into = torch.zeros((rows, n + 3), device="cuda", dtype=x.dtype)
    ext.token_logprobs_backward(x, y, fwd.lse, fwd.entropy, g, ge, scale=0.8, out=into[:, 1:n + 1])
    assert torch.equal(into[:, 1:n + 1], want) and (into[:, 0] == 0).all() and (into[:, n + 1:] == 0).all()
    x2 = x.clone()
    ext.token_logprobs_backward(x2, y, fwd.lse, fwd.entropy, g, ge, scale=0.8, out=x2)
    assert torch.equal(x2, want)


def test_gradient_against_differences(ext):
    """Central differences of the fp64 loss around the same logits: the step 1e-4 leaves 1e-8 of third derivatives."""
    x, y = make(4, 33, "fp32", 2)
    y[:3] = torch.tensor([3, -1, 32], device="cuda")
    g, ge = torch.randn(4, device="cuda"), torch.randn(4, device="cuda")
    fwd = ext.token_logprobs(x, y)
    d = ext.token_logprobs_backward(x, y, fwd.lse, fwd.entropy, g, ge).double().cpu().numpy()
    X, Y, G, E = x.double().cpu().numpy(), y.cpu().numpy(), g.double().cpu().numpy(), ge.double().cpu().numpy()

    def loss(X):
        lp, h, *_ = ref.logprobs(X, Y, 1.0, 0)
        return (G * lp + E * h).sum()
    for i in np.ndindex(X.shape):
        e = np.zeros_like(X)
        e[i] = 1e-4
        assert abs((loss(X + e) - loss(X - e)) / 2e-4 - d[i]) < 1e-5      # fp32 sums of entries up to a few units


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_masks(ext, dtype):
    x, y = make(3, 500, dtype, 5)
    x[0, 100:] = -math.inf
    x[1, :] = -math.inf
    y[0], y[1], y[2] = 5, 7, 600
    g, ge = torch.ones(3, device="cuda"), torch.ones(3, device="cuda")
    fwd = ext.token_logprobs(x, y)
    d = ext.token_logprobs_backward(x, y, fwd.lse, fwd.entropy, g, ge)
    assert torch.isfinite(d).all() and (d[0, 100:] == 0).all()
    assert (d[1, :7] == 0).all() and (d[1, 8:] == 0).all() and d[1, 7].item() == 1.0
    check_backward(ext, x[:1], y[:1], g[:1], ge[:1], 1.0, TYPES[dtype][1])


def test_refusals(ext):
    x, y = make(4, 50, "fp32")
    for f in (lambda: ext.token_logprobs(x.double(), y), lambda: ext.token_logprobs(x, y.int()), lambda: ext.token_logprobs(x.t(), y),
              lambda: ext.token_logprobs(x, y[:2]), lambda: ext.token_logprobs(x[0], y), lambda: ext.token_logprobs(x.cpu(), y),
              lambda: ext.token_logprobs_backward(x, y, x[:, 0], x[:, 0].contiguous())):
        with pytest.raises(ValueError):
            f()
    for kw in (dict(top=51), dict(top=-1), dict(top=65), dict(scale=0.0), dict(scale=math.nan)):
        with pytest.raises(ext.ExterndError):
            ext.token_logprobs(x, y, **kw)
    with pytest.raises(ext.ExterndError):
        ext.token_logprobs_backward(x, y, None, None, x[:, 0].contiguous())
    e = ext.token_logprobs(x[:0], y[:0], top=3)
    assert e.logprob.shape == (0,) and e.top_ids.shape == (0, 3)
