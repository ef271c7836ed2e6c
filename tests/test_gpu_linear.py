"""GPU parity of the log probabilities behind a dense head and their gradients
(externd_linear_logprobs, _backward) with the oracle's fp64 form.

Tolerance (u = 2^-24, K the width, S = scale sum |x_k w_k| of a logit, Z the
row's largest |z|, n the vocabulary): a logit is a sum of K products in fp32 in
some order, exact in the 16-bit types (K roundings of at most S; fp32 parts
leave out and round 2^-21 S more), times scale: d = (K + 8) u S, and 0 but for
the scale's u Z where all sums are whole numbers below 2^24.  Differences to a
reference and exponentials are within 4 u + 4 u Z of themselves and at least 64
partial sums are joined by a tree, so a sum of n exponentials carries
s = d + 4 u + 4 u Z + (n / 64 + 40) u; lse moves by s + 2 u |lse|, a log probability by d + u Z more,
the entropy by (2 + 4 Z) s + 4 u (Z + |lse|).

Gradients: p carries q = d + (lse's error) + 4 u (Z + |lse|) + 4 u and ln p + entropy moves by
h = q + (the entropy's error), so that G moves by
D = (|g| p + |ge| p (|ln p + H| + 1)) q + |ge| p h + 4 u |G|, is rounded to e |G| (2^-8, 2^-11, 2^-21 for fp32's
three parts; in fp16 also 2^-39 of the row's largest), and a product of m terms of
absolute sum T adds (m + 64) u T; the result is rounded once."""
import math

import numpy as np
import pytest

import oracle.ends_oracle as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}
ROUND_G = {"fp32": 2.0 ** -21, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def ext():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13511_amd import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().double().cpu().numpy()


def make(rows, width, vocab, dtype, seed=0, whole=False):
    """whole: small whole numbers, whose products and sums fp32 holds exactly."""
    rng = np.random.default_rng(seed)
    if whole:
        x, w = rng.integers(-3, 4, (rows, width)) * 0.25, rng.integers(-3, 4, (vocab, width)) * 0.125
    else:
        x, w = rng.standard_normal((rows, width)), rng.standard_normal((vocab, width)) * 2.0 / math.sqrt(width)
    y = rng.integers(0, vocab, rows)
    y[rng.random(rows) < 0.2] = -1
    t = TYPES[dtype][0]
    return torch.from_numpy(x).to(t).cuda(), torch.from_numpy(w).to(t).cuda(), torch.from_numpy(y).cuda()


class Bounds:
    def __init__(self, x, w, scale, whole=False):
        self.z, S = ref.linear(f64(x), f64(w), scale)
        self.lse, self.entropy, self.p = ref.softmax_moments(self.z)
        n, K = w.shape
        Z = np.abs(self.z).max(-1)
        self.d = (0 if whole else (K + 8) * U * S.max(-1)) + U * Z
        self.s = self.d + 4 * U + 4 * U * Z + (n / 64 + 40) * U
        self.dl = self.s + 2 * U * np.abs(self.lse)
        self.dp = self.dl + self.d + U * Z
        self.dh = (2 + 4 * Z) * self.s + 4 * U * (Z + np.abs(self.lse))
        self.q = self.d + self.dl + 4 * U * (Z + np.abs(self.lse)) + 4 * U


def check(ext, x, w, y, scale=1.0, whole=False):
    got = ext.linear_logprobs(x, w, y, scale=scale)
    b = Bounds(x, w, float(np.float32(scale)), whole)
    rows, yy = np.arange(x.shape[0]), y.cpu().numpy()
    lp = np.where(yy >= 0, b.z[rows, np.maximum(yy, 0)] - b.lse, 0.0)
    for name, g, want, tol in (("lse", got.lse, b.lse, b.dl), ("logprob", got.logprob, lp, b.dp), ("entropy", got.entropy, b.entropy, b.dh)):
        err = np.abs(f64(g) - want)
        assert np.all(err <= tol), (name, np.max(err / tol))
    assert got.top_ids is None and got.top_logprobs is None
    return got


SIZES = [(1, 1, 1), (1, 8, 1), (3, 7, 5), (2, 64, 256), (5, 65, 257), (1, 2560, 1000), (8, 256, 3001), (16, 1001, 600), (17, 33, 2049),
         (33, 130, 513), (64, 512, 300), (65, 96, 1025), (200, 72, 700), (255, 264, 511), (257, 2560, 513), (700, 40, 1031), (1030, 8, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", SIZES)
def test_forward(ext, dtype, rows, width, vocab):
    check(ext, *make(rows, width, vocab, dtype, rows), scale=0.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", [(1, 9, 70), (7, 128, 300), (300, 200, 1300), (40, 1024, 515)])
def test_forward_whole_numbers(ext, dtype, rows, width, vocab):
    check(ext, *make(rows, width, vocab, dtype, rows, True), whole=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", [(1, 16, 70001), (3, 40, 9000), (8, 65, 20011), (32, 24, 65537), (31, 7, 8193)])
def test_few_rows_of_a_large_vocabulary(ext, dtype, rows, width, vocab):
    """Tiles of less than 256 columns; every target's own logit, one by one the columns around the tiles' ends."""
    x, w, _ = make(rows, width, vocab, dtype, rows, True)
    for first in (0, 130, 255, vocab - rows):
        check(ext, x, w, torch.arange(first, first + rows, device="cuda"), whole=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [264, 261])
def test_last_columns_by_themselves(ext, dtype, width):
    """128 tiles for each of two row tiles, and one column more."""
    x, w, y = make(300, width, 32769, dtype, 20, True)
    y[7], y[8] = 32768, 32767
    check(ext, x, w, y, whole=True)
    check_backward(ext, x, w, y, *gradients(300, y, 21, "ge"), dtype, whole=True)


def gradients(rows, y, seed, kind):
    rng = np.random.default_rng(seed)
    g = (rng.standard_normal(rows) / rows).astype(np.float32) if "g" in kind else None
    ge = (0.3 * rng.standard_normal(rows) / rows).astype(np.float32) if "e" in kind else None
    if "0" in kind:
        for a in (g, ge):
            if a is not None:
                a[rng.random(rows) < 0.4] = 0
    return tuple(None if a is None else torch.from_numpy(a).cuda() for a in (g, ge))


def check_backward(ext, x, w, y, g, ge, dtype, scale=1.0, whole=False, given=None, **kw):
    s32, rows = float(np.float32(scale)), x.shape[0]
    fwd = ext.linear_logprobs(x, w, y, scale=scale)
    gx, gw = given or ext.linear_logprobs_backward(x, w, y, fwd.lse, fwd.entropy, g, ge, scale=scale, **kw)
    b = Bounds(x, w, s32, whole)
    yy = y.cpu().numpy()
    asked = (yy >= 0) & (yy < w.shape[0])
    G = ref.logits_gradient(b.z, yy, None if g is None else f64(g), None if ge is None else f64(ge))
    gg = np.zeros(rows) if g is None else np.abs(f64(g)) * asked
    hh = np.zeros(rows) if ge is None else np.abs(f64(ge))
    lp = np.where(b.p > 0, b.z - b.lse[:, None], 0.0)
    col = lambda v: v[:, None]
    D = (col(gg) + col(hh) * (np.abs(lp + col(b.entropy)) + 1)) * b.p * col(b.q) + col(hh) * b.p * col(b.q + b.dh) + 4 * U * np.abs(G)
    D = D + ROUND_G[dtype] * np.abs(G)
    if dtype == "fp16":
        D = D + 2.0 ** -39 * col(gg + hh * (1 + np.abs(b.entropy)))
    D[(gg == 0) & (hh == 0)] = 0
    A, e = np.abs(G), TYPES[dtype][1]
    out = []
    for got, left, right in ((gx, (G, A, D), f64(w)), (gw, (G.T, A.T, D.T), np.where(((gg != 0) | (hh != 0))[:, None], f64(x), 0))):
        if got is None:
            continue
        want, size, off = (s32 * (m @ r) for m, r in zip(left, (right, np.abs(right), np.abs(right))))
        tol = off + (right.shape[0] + 64) * U * (size + off) + e * (np.abs(want) + off + 64 * U * size) + (2.0 ** -25 if dtype == "fp16" else 2.0 ** -126)
        err = np.abs(f64(got) - want)
        assert np.all(err <= tol), np.max(err / tol)
        out.append(got)
    return gx, gw


LARGE = [(100, 72, 16500), (100, 73, 16500), (128, 8, 16500), (300, 136, 6700), (300, 71, 6700), (512, 64, 4200)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", LARGE)
def test_large_tiles(ext, dtype, rows, width, vocab):
    """More than 1024 tiles of 64 columns and 32 rows: these calls take the large ones, aligned or not."""
    assert -(-vocab // 64) * -(-rows // 32) > 1024
    x, w, y = make(rows, width, vocab, dtype, rows, True)
    check(ext, x, w, y, scale=0.7)
    check_backward(ext, x, w, y, *gradients(rows, y, 1, "ge"), dtype, scale=0.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", SIZES)
def test_backward(ext, dtype, rows, width, vocab):
    x, w, y = make(rows, width, vocab, dtype, rows)
    check_backward(ext, x, w, y, *gradients(rows, y, 1, "ge"), dtype, scale=0.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["g", "e", "g0", "ge0"])
@pytest.mark.parametrize("need", [(True, False), (False, True)])
def test_backward_parts(ext, dtype, kind, need):
    x, w, y = make(70, 136, 901, dtype, 3, True)
    gx, gw = check_backward(ext, x, w, y, *gradients(70, y, 2, kind), dtype, whole=True, need_x=need[0], need_weight=need[1])
    assert (gx is None) == (not need[0]) and (gw is None) == (not need[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_and_pieces(ext, dtype):
    """More rows than one pass of the forward call takes, and a vocabulary of several pieces."""
    x, w, y = make(8200, 16, 300, dtype, 4, True)
    check(ext, x, w, y, whole=True)
    x, w, y = make(8200, 24, 9000, dtype, 5, True)
    g = torch.zeros(8200, device="cuda")
    g[::97] = 0.01
    fwd = ext.linear_logprobs(x, w, y)
    gx, gw = ext.linear_logprobs_backward(x, w, y, fwd.lse, fwd.entropy, g)
    some = torch.arange(0, 8200, 97, device="cuda")
    # rows that take no part add zeros, which round nothing: the bounds are those of the others alone
    check_backward(ext, x[some].contiguous(), w, y[some].contiguous(), g[some].contiguous(), None, dtype, whole=True, given=(gx[some], gw))
    rest = torch.ones(8200, dtype=torch.bool, device="cuda")
    rest[some] = False
    assert (gx[rest] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", [(70, 256, 1000), (40, 900, 1300), (452, 1002, 1030), (7, 300, 257), (3, 40, 129)])
def test_splits_behind_the_end(ext, dtype, rows, width, vocab):
    """The last of the splits of grad_x's sum have nothing to add (and weight ends where its memory does)."""
    x, w, y = make(rows, width, vocab, dtype, 23, True)
    check_backward(ext, x, w, y, *gradients(rows, y, 24, "ge"), dtype, whole=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_last_pass_of_few_rows(ext, dtype):
    """8192 rows and three more, whose tiles outnumber the CUs."""
    x, w, y = make(8195, 64, 70001, dtype, 22, True)
    y[8192:] = torch.tensor([70000, 5, 300], device="cuda")
    got = ext.linear_logprobs(x, w, y)
    last = Bounds(x[8192:], w, 1.0, True)
    for g, want, tol in ((got.lse, last.lse, last.dl), (got.entropy, last.entropy, last.dh),
                         (got.logprob, last.z[np.arange(3), [70000, 5, 300]] - last.lse, last.dp)):
        assert np.all(np.abs(f64(g[8192:]) - want) <= tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,vocab", [(3, 24, 1000), (40, 72, 8192), (200, 300, 8200), (2500, 1031, 8200)])
@pytest.mark.parametrize("one", [False, True])
def test_the_targets_entry_is_not_rounded(ext, dtype, rows, width, vocab, one):
    """Of G's entries g (1 at the target - p) with p = 1 / vocab, all logits being 0.
    A 16-bit G rounds the target's to e of itself, and its rest, which is added,
    to e of that: e e of the target's share is left, and e of the others' (p's
    rounding; none in grad_x, whose weights cancel in pairs), of the scale and
    its kind 8 u, of m terms (m + 64) u; and the result is rounded once."""
    t, e = TYPES[dtype]
    rng = np.random.default_rng(rows)
    y = np.full(rows, vocab - 3) if one else rng.integers(0, vocab, rows)
    y[::7] = vocab - 1
    g, scale = rng.uniform(1, 2, rows).astype(np.float32), 1.37
    lse, H = torch.full((rows,), math.log(vocab), device="cuda"), torch.full((rows,), math.log(vocab), device="cuda")
    where = torch.from_numpy(y).cuda(), lse, H, torch.from_numpy(g).cuda()
    g = g.astype(np.float64)

    half = torch.from_numpy(rng.uniform(1, 2, (vocab // 2, width))).to(t).cuda()
    w = torch.stack((half, -half), 1).reshape(vocab, width)
    x = torch.zeros((rows, width), dtype=t, device="cuda")
    gx, _ = ext.linear_logprobs_backward(x, w, *where, scale=scale, need_weight=False)
    share = scale * g[:, None] * f64(w)[y]
    terms = scale * g[:, None] / vocab * np.abs(f64(w)).sum(0)
    off = np.abs(f64(gx) - share)
    assert (off <= e * np.abs(share) + (e * e + 8 * U + 64 * U) * np.abs(share) * 1.01 + (vocab + 72) * U * terms).all()

    x = torch.from_numpy(rng.uniform(1, 2, (rows, width))).to(t).cuda()
    _, gw = ext.linear_logprobs_backward(x, torch.zeros_like(w), *where, scale=scale, need_x=False)
    first = np.zeros((vocab, width))
    np.add.at(first, y, scale * g[:, None] * f64(x))
    second = scale / vocab * (g[:, None] * f64(x)).sum(0)
    want, parts = first - second, first + second
    bound = e * np.abs(want) + (e * second + e * e * parts) * 1.01 + (rows + 72 + 8 * math.log(vocab)) * U * parts
    assert (np.abs(f64(gw) - want) <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", [(9, 256, 20000), (58, 521, 3607), (130, 264, 8000), (300, 512, 2000), (700, 1000, 5000)])
def test_both_gradients_at_once(ext, dtype, rows, width, vocab):
    """Sizes whose tiles of both products the CUs hold together, and each by itself."""
    x, w, y = make(rows, width, vocab, dtype, 27)
    g = gradients(rows, y, 28, "ge")
    check_backward(ext, x, w, y, *g, dtype)
    got = ext.linear_logprobs(x, w, y)
    lse, H = got.lse, got.entropy
    _, gw = ext.linear_logprobs_backward(x, w, y, lse, H, *g)
    assert torch.equal(gw, ext.linear_logprobs_backward(x, w, y, lse, H, *g, need_x=False)[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("vocab,width", [(38000, 96), (38000, 44), (45000, 100), (45000, 260), (32769, 300), (20118, 132), (20148, 40)])
def test_few_rows_and_pieces_of_a_tile(ext, dtype, whole, vocab, width):
    """Tiles, or last ones, of five and six pieces of 32 columns, of which waves share the last; odd numbers of steps."""
    x, w, y = make(9, width, vocab, dtype, 25, whole)
    y[3], y[4], y[5] = vocab - 1, 130, 165
    check(ext, x, w, y, whole=whole)
    check_backward(ext, x, w, y, *gradients(9, y, 26, "ge"), dtype, whole=whole)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,gap", [(1, 0), (0, 1), (3, 5), (2, 6), (8, 8), (5, 11)])
def test_strides(ext, dtype, offset, gap):
    """Rows that begin anywhere, with gaps that hold NaN; outputs between other columns."""
    for rows, width, vocab in ((70, 200, 530), (5, 129, 300)):
        x0, w0, y = make(rows, width, vocab, dtype, 6)
        bufs = [torch.full((t.shape[0], width + gap + offset), math.nan, device="cuda", dtype=t.dtype) for t in (x0, w0)]
        x, w = (b[:, offset:offset + width] for b in bufs)
        x.copy_(x0), w.copy_(w0)
        got, want = check(ext, x, w, y), ext.linear_logprobs(x0, w0, y)
        g, ge = gradients(rows, y, 7, "ge")
        outs = [torch.full_like(b, 9.0) for b in bufs]
        views = [b[:, offset:offset + width] for b in outs]
        gx, gw = check_backward(ext, x, w, y, g, ge, dtype, out=tuple(views))
        assert gx is views[0] and gw is views[1]
        for o in outs:
            assert (o[:, :offset] == 9).all() and (o[:, offset + width:] == 9).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [3, 70])
def test_padding_rows_may_hold_anything(ext, dtype, rows):
    """Rows without gradients: x, lse and entropy there may be NaN or infinite; forward, only their own results are."""
    x, w, y = make(rows, 96, 400, dtype, 8)
    y[1], y[2] = -1, 5
    g, ge = gradients(rows, y, 9, "g")[0], torch.zeros(rows, device="cuda")
    g[2] = 0
    fwd = ext.linear_logprobs(x, w, y)
    want = ext.linear_logprobs_backward(x, w, y, fwd.lse, fwd.entropy, g, ge)
    x[1], x[2] = math.nan, math.inf
    bad = ext.linear_logprobs(x, w, y)
    assert torch.isnan(bad.lse[1:3]).all() and torch.isnan(bad.entropy[1:3]).all() and bad.logprob[1] == 0 and torch.isnan(bad.logprob[2])
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[1:3] = False
    assert torch.equal(bad.lse[keep], fwd.lse[keep]) and torch.equal(bad.logprob[keep], fwd.logprob[keep])
    got = ext.linear_logprobs_backward(x, w, y, bad.lse, bad.entropy, g, ge)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (got[0][1:3] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_nonfinite(ext, dtype):
    """A NaN in weight reaches every row; targets past the vocabulary; logits that overflow the type but not fp32."""
    x, w, y = make(6, 64, 130, dtype, 10)
    y[0], y[1] = 130, 1 << 40
    got = ext.linear_logprobs(x, w, y)
    assert torch.isnan(got.logprob[:2]).all() and torch.isfinite(got.lse).all()
    g = torch.ones(6, device="cuda")
    gx, gw = ext.linear_logprobs_backward(x, w, y, got.lse, got.entropy, g)
    assert (gx[:2] == 0).all() and torch.isfinite(gx).all() and torch.isfinite(gw).all()
    w2 = w.clone()
    w2[77, 5] = math.nan
    bad = ext.linear_logprobs(x, w2, y)
    assert torch.isnan(bad.lse).all() and torch.isnan(bad.entropy).all()
    big = make(6, 64, 130, dtype, 11, True)
    big = (big[0] * 64, big[1] * 64, big[2])      # one logit stands out by thousands: probabilities of 0 and 1
    check(ext, *big, whole=True)
    fwd = ext.linear_logprobs(*big)
    gx, gw = ext.linear_logprobs_backward(*big, fwd.lse, fwd.entropy, g, g)
    assert torch.isfinite(gx).all() and torch.isfinite(gw).all()


def test_logits_of_minus_infinity(ext):
    """An infinite entry of weight that meets positive entries: probability 0, in the 16-bit types."""
    for dtype in ("bf16", "fp16"):
        x, w, y = make(40, 32, 100, dtype, 12)
        x = x.abs() + 0.125
        want = ext.linear_logprobs(x, torch.cat([w[:50], w[51:]]), None)
        w[50, 3] = -math.inf
        got = ext.linear_logprobs(x, w, torch.full((40,), 50, device="cuda"))
        assert torch.isneginf(got.logprob).all() and (got.lse - want.lse).abs().max() < 1e-5 and (got.entropy - want.entropy).abs().max() < 1e-4
        only = torch.full((3, 32), -math.inf, device="cuda", dtype=x.dtype)
        got = ext.linear_logprobs(x, only, torch.zeros(40, dtype=torch.int64, device="cuda"))
        assert torch.isneginf(got.lse).all() and (got.entropy == 0).all() and torch.isneginf(got.logprob).all()


def test_small_gradients_keep_their_bits_in_fp16(ext):
    """Gradients down to 1e-12 beside ones of 1: each row's own scale carries them."""
    x, w, y = make(64, 64, 2000, "fp16", 13, True)
    y = y.clamp_min(0)
    g = torch.logspace(-12, 0, 64, device="cuda")
    fwd = ext.linear_logprobs(x, w, y)
    gx, _ = ext.linear_logprobs_backward(x, w * 0 + w, y, fwd.lse, fwd.entropy, g, need_weight=False)
    check_backward(ext, x, w, y, g, None, "fp16", whole=True)
    check_backward(ext, x, w, y, torch.full((64,), 1e-9, device="cuda"), None, "fp16", whole=True)
    assert (gx[40:] != 0).any(-1).all()


def test_gradient_against_differences(ext):
    """A step along the gradients changes the loss by their squared length (fp32; central differences)."""
    x, w, y = make(24, 48, 150, "fp32", 14)
    y = y.clamp_min(0)
    g, ge = gradients(24, y, 15, "ge")

    def loss(x, w):
        z = f64(x) @ f64(w).T * 0.9
        lse, entropy, _ = ref.softmax_moments(z)
        return float((f64(g) * (z[np.arange(24), y.cpu().numpy()] - lse)).sum() + (f64(ge) * entropy).sum())
    fwd = ext.linear_logprobs(x, w, y, scale=0.9)
    gx, gw = ext.linear_logprobs_backward(x, w, y, fwd.lse, fwd.entropy, g, ge, scale=0.9)
    for dx, dw in ((gx, None), (None, gw)):
        step = 1e-3
        a = loss(x.double() + step * dx.double() if dx is not None else x, w.double() + step * dw.double() if dw is not None else w)
        c = loss(x.double() - step * dx.double() if dx is not None else x, w.double() - step * dw.double() if dw is not None else w)
        want = sum(float((d.double() ** 2).sum()) for d in (dx, dw) if d is not None)
        # third derivatives of a loss of weights ~1 / 24 along a step of 1e-3 |gradient| < 1e-3
        assert abs((a - c) / (2 * step) - want) <= 1e-4 * want + 1e-9


def test_nothing(ext):
    w = torch.ones((5, 8), device="cuda")
    x, none = torch.empty((0, 8), device="cuda"), torch.empty((0,), device="cuda")
    got = ext.linear_logprobs(x, w, torch.empty((0,), dtype=torch.int64, device="cuda"))
    assert got.lse.shape == got.logprob.shape == (0,)
    gx, gw = ext.linear_logprobs_backward(x, w, None, none, none, None, none)
    assert gx.shape == (0, 8) and gw.shape == (5, 8) and (gw == 0).all()
    x = torch.ones((3, 8), device="cuda")
    got = ext.linear_logprobs(x, w)
    assert got.logprob is None
    gx, gw = ext.linear_logprobs_backward(x, w, None, got.lse, got.entropy)
    assert (gx == 0).all() and (gw == 0).all()
    assert ext.linear_logprobs_backward(x, w, None, got.lse, got.entropy, need_x=False, need_weight=False) == (None, None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [4, 300])
def test_streams_graphs_and_repeats(ext, dtype, rows):
    x, w, y = make(rows, 264, 1500, dtype, 16)
    g, ge = gradients(rows, y, 17, "ge")

    def both(**kw):
        f = ext.linear_logprobs(x, w, y, **kw)
        return (f.lse, f.logprob, f.entropy, *ext.linear_logprobs_backward(x, w, y, f.lse, f.entropy, g, ge, **kw))
    want = both()
    assert all(torch.equal(a, b) for a, b in zip(both(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(3):
        x.mul_(0.9)
        g.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_given_workspaces_may_hold_anything(ext):
    """Workspaces of NaN, of the size that the library asks for and a byte less."""
    x, w, y = make(100, 136, 700, "bf16", 18)
    g = gradients(100, y, 19, "g")[0]
    f = ext.linear_logprobs(x, w, y)
    want = ext.linear_logprobs_backward(x, w, y, f.lse, f.entropy, g)
    L = ext.lib()
    a, b = L.externd_linear_logprobs_workspace_bytes(1, 100, 700, 136), L.externd_linear_logprobs_backward_workspace_bytes(1, 100, 700, 136, 1, 1)
    wa, wb = (torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (a, b))
    assert torch.equal(ext.linear_logprobs(x, w, y, workspace=wa).lse, f.lse)
    got = ext.linear_logprobs_backward(x, w, y, f.lse, f.entropy, g, workspace=wb)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for call in (lambda: ext.linear_logprobs(x, w, y, workspace=wa[:-1]),
                 lambda: ext.linear_logprobs_backward(x, w, y, f.lse, f.entropy, g, workspace=wb[:-1])):
        with pytest.raises(ext.ExterndError):
            call()


def test_refusals(ext):
    x, w, y = make(4, 16, 20, "fp32")
    e = torch.zeros(4, device="cuda")
    for call in (lambda: ext.linear_logprobs(x.double(), w, y), lambda: ext.linear_logprobs(x, w.half(), y),
                 lambda: ext.linear_logprobs(x, w[:, :8], y), lambda: ext.linear_logprobs(x, w.t(), y),
                 lambda: ext.linear_logprobs(x, w, y.int()), lambda: ext.linear_logprobs(x, w, y[:3]),
                 lambda: ext.linear_logprobs(x.cpu(), w, y), lambda: ext.linear_logprobs(x, w.cpu(), y),
                 lambda: ext.linear_logprobs_backward(x, w, y, e[:3], e, e), lambda: ext.linear_logprobs_backward(x, w, y, e, e, e.half()),
                 lambda: ext.linear_logprobs_backward(x, w, y, e, e, e, out=(x, None)),
                 lambda: ext.linear_logprobs_backward(x, w, y, e, e, e, out=(None, w)),
                 lambda: ext.linear_logprobs_backward(x, w, y, e, e, e, out=(torch.empty_like(x[:3]), None)),
                 lambda: ext.linear_logprobs(x, w, y, workspace=torch.empty(1 << 20))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ext.linear_logprobs(x, w, y, scale=0.0), lambda: ext.linear_logprobs(x, w, y, scale=math.inf),
                 lambda: ext.linear_logprobs(x, w[:0], y), lambda: ext.linear_logprobs_backward(x, w, None, e, e, e),
                 lambda: ext.linear_logprobs_backward(x, w, y, None, e, e), lambda: ext.linear_logprobs_backward(x, w, y, e, None, e, e),
                 lambda: ext.linear_logprobs_backward(x, w, y, e, e, e, scale=math.nan)):
        with pytest.raises(ext.ExterndError):
            call()
