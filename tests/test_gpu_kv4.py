"""GPU parity of the 4-bit cache (externd_kv4_append, _read) and attention
over it (externd_kv4_attention) with the oracle's fp64 forms.

Cache: scale, zero point and codes are rounded quotients.  For bf16 and fp16
inputs, and fp32 inputs of at most 12 significant bits, an fp32 quotient
rounds to a tie or to a seven-bit scale only where the exact one is there, so
the stored values are the oracle's bit for bit; for other fp32 inputs a value
is within s / 2 (1 + 2^-20) of its input.

Attention over given values (u = 2^-24, n visible keys, D channels, unit t of
the result's type: 2^-24, 2^-8, 2^-11): a score's products and sums in fp32,
or its query as 31-bit integers, are within e = (D + 16) u scale sum |q k^|
of the exact score, the largest such sum a row sees taken for all; softmax
weights then carry 2 e + (n / 64 + 80) u (exponential, sums over at least 64
partial sums, joining of parts), and 2^-11 where 16-bit queries take fp16
weights on the matrix cores (below 2^-14: 2^-25 of the largest value).  So
  |out - exact| <= (2 e + (n / 64 + 80) u + w) sum p |v| + w2 max |v| + t |out|
  |lse - exact| <= e + (n / 64 + 80) u + 2 u |lse|
with w = 2^-11, w2 = n 2^-25 for 16-bit types and 0 for fp32."""
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


class Pool:
    """A pool of pages in random order over arbitrary bytes, on the host and on the GPU."""

    def __init__(self, lens, news, heads, dim, page, seed, spare=2):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.news, self.heads, self.dim, self.page = lens, news, heads, dim, page
        need = [-(-max(n, 0) // page) for n in lens]
        width = max(need + [1])
        order = rng.permutation(sum(need) + spare)
        self.table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.cache = rng.integers(0, 256, (len(order), heads, page * (dim + dim // 16)), dtype=np.uint8)
        self.starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)

    def fill(self, scale=1.0):
        """Stores random whole sequences with the oracle."""
        for b, n in enumerate(self.lens):
            if n > 0:
                loud = 1 + 5 * (self.rng.random((1, self.heads, self.dim)) < 0.05)
                k = scale * (self.rng.standard_normal((n, self.heads, self.dim)) * loud + 0.5 * loud)
                v = scale * self.rng.standard_normal((n, self.heads, self.dim))
                ref.kv4_encode(self.cache, self.page, k, v, self.table[b], 0, self.heads)
        return self

    def gpu(self):
        one = all(n == 1 for n in self.news)
        return (torch.from_numpy(self.cache).cuda(), torch.from_numpy(self.table).cuda(),
                torch.tensor(self.lens, dtype=torch.int32, device="cuda"), None if one else torch.from_numpy(self.starts).cuda())

    def places(self):
        """(token, sequence, position) of each new token."""
        return [(self.starts[b] + i, b, self.lens[b] - self.news[b] + i) for b in range(len(self.lens)) for i in range(self.news[b])]


def inputs(rng, shape, dtype):
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.exp(rng.uniform(-3, 3, shape[:2] + (1,))))
    if dtype == "fp32":
        x = x.to(torch.bfloat16).float()          # few significant bits: see the top
    return x.to(TYPES[dtype][0])


# ---------------------------------------------------------------------------
# append and read
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,page,heads,lens,news", [
    (64, 16, 1, [1], [1]), (128, 16, 8, [5, 17, 16, 0, 33], [1, 1, 1, 1, 1]), (128, 64, 2, [70, 3, 129], [70, 2, 65]),
    (256, 32, 3, [31, 40, 0, 2], [31, 7, 0, 5]), (64, 1024, 5, [1030, 12], [9, 12]), (128, 32, 1, [200], [200])])
def test_append_matches_oracle(ext, dtype, dim, page, heads, lens, news):
    pool = Pool(lens, news, heads, dim, page, 7)
    n = int(pool.starts[-1])
    k, v = inputs(pool.rng, (n, heads, dim), dtype), inputs(pool.rng, (n, heads, dim), dtype)
    cache, table, dlens, starts = pool.gpu()
    ext.kv4_append(cache, k.cuda(), v.cuda(), table, dlens, starts=starts)
    want = pool.cache.copy()
    K, V = k.double().numpy(), v.double().numpy()
    for t, b, p in pool.places():
        if p >= 0:
            ref.kv4_encode(want, page, K[t:t + 1], V[t:t + 1], pool.table[b], p, heads)
    assert np.array_equal(cache.cpu().numpy(), want)                 # the tokens' bytes, and no other byte
    kept = np.array([p >= 0 for _, _, p in pool.places()])[:, None, None]
    for got, x in zip(ext.kv4_read(cache, table, dlens, dim, starts=starts, tokens=n), (K, V)):
        assert np.array_equal(got.double().cpu().numpy(), np.where(kept, ref.kv4_values(x), 0))
    for t in (torch.bfloat16, torch.float16):
        a, b = ext.kv4_read(cache, table, dlens, dim, starts=starts, tokens=n), ext.kv4_read(cache, table, dlens, dim, starts=starts,
                                                                                            tokens=n, dtype=t)
        assert torch.equal(a[0].to(t), b[0]) and torch.equal(a[1].to(t), b[1])


def test_append_any_fp32(ext):
    """fp32 inputs of any bits, sizes from subnormal to beyond what the cache holds."""
    rng = np.random.default_rng(11)
    n, dim = 400, 128
    size = np.exp(rng.uniform(math.log(1e-12), math.log(1.6e4), (n, 1, 1)))     # spans up to 64000
    x = (size * np.clip(rng.standard_normal((n, 2, dim)), -2, 2)).astype(np.float32)
    pool = Pool([n], [n], 2, dim, 32, 3)
    cache, table, lens, starts = pool.gpu()
    X = torch.from_numpy(x).cuda()
    ext.kv4_append(cache, X, -X, table, lens, starts=starts)
    for got, want in zip(ext.kv4_read(cache, table, lens, dim, starts=starts, tokens=n), (x, -x)):
        got, want = got.double().cpu().numpy().reshape(n, 2, 2, 64), want.astype(np.float64).reshape(n, 2, 2, 64)
        span = np.maximum(want.max(-1), 0) - np.minimum(want.min(-1), 0)
        # the step: fifteenth of the span (one fp32 rounding of the span, one of the quotient) and its rounding up
        step = np.maximum(span / 15 * (1 + 2.0 ** -22) * (1 + 2.0 ** -6), span / 15 + 2.0 ** -20)
        assert np.all(np.abs(got - want) <= (step / 2 * (1 + 2.0 ** -20))[..., None])
    big = torch.tensor([1e9, -1e9, 65280.0, 70000.0], device="cuda").repeat(64).view(1, 2, 128)
    ext.kv4_append(cache, big, big, table, torch.tensor([1], dtype=torch.int32, device="cuda"))
    got, _ = ext.kv4_read(cache, table, torch.tensor([1], dtype=torch.int32, device="cuda"), dim)
    assert torch.isfinite(got).all() and got.abs().max().item() <= 65280.0       # beyond its range it saturates


@pytest.mark.parametrize("dtype", TYPES)
def test_append_strides_and_nonfinite(ext, dtype):
    """k and v as slices of a fused projection at odd places; groups with a NaN or an infinity read as NaN."""
    t = TYPES[dtype][0]
    rng = np.random.default_rng(5)
    n, heads, dim = 21, 2, 128
    flat = inputs(rng, (n, 1, 3 + 2 * heads * dim), dtype)[:, 0].clone()
    flat[4, 3 + 7] = math.nan
    flat[9, 3 + 64 + 1] = math.inf
    flat[12, 3 + heads * dim + 200] = -math.inf
    flat = flat.cuda()
    k, v = flat[:, 3:3 + heads * dim].unflatten(1, (heads, dim)), flat[:, 3 + heads * dim:].unflatten(1, (heads, dim))
    assert k.dtype is t
    pool = Pool([40], [n], heads, dim, 16, 1)
    cache, table, lens, starts = pool.gpu()
    ext.kv4_append(cache, k, v, table, lens, starts=starts)
    for got, x in zip(ext.kv4_read(cache, table, lens, dim, starts=starts, tokens=n), (k, v)):
        want = ref.kv4_values(x.double().cpu().numpy())
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
        assert np.isnan(want).sum() in (128, 64)


def test_places_outside_the_cache(ext):
    """Pages beyond the pool and lengths beyond the table reach no memory: nothing is stored, zeros are read."""
    dim, heads, page = 64, 2, 16
    pool = Pool([20, 40, 5], [20, 8, 5], heads, dim, page, 2)
    pool.table[0, 1], pool.table[2, 0] = 10 ** 6, -7
    pool.lens = [20, 60, 5]                          # table rows hold 48 tokens: the last 8 of 60 are in none
    cache, table, lens, starts = pool.gpu()
    n = 33
    k = torch.randn((n, heads, dim), device="cuda")
    before = cache.clone()
    ext.kv4_append(cache, k, k, table, lens, starts=starts)
    K, _ = ext.kv4_read(cache, table, lens, dim, starts=starts, tokens=n)
    assert (K[:16] != 0).any() and (K[16:] == 0).all()
    page0 = int(pool.table[0, 0])
    others = [i for i in range(cache.shape[0]) if i != page0]
    assert torch.equal(cache[others], before[others])


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def check_attention(ext, pool, heads_q, dtype, window=0, scale=None, cache=None, seed=0, hints=True, q=None):
    t, unit = TYPES[dtype]
    n, dim, each = int(pool.starts[-1]), pool.dim, heads_q // pool.heads
    rng = np.random.default_rng(seed)
    if q is None:
        q = torch.from_numpy(rng.standard_normal((n, heads_q, dim)).astype(np.float32)).to(t).cuda()
    dcache, table, lens, starts = pool.gpu()
    kw = dict(max_new=max(pool.news), max_len=max(pool.lens)) if hints else {}
    out, lse = ext.kv4_attention(dcache, q, table, lens, starts=starts, window=window, scale=scale, **kw)
    torch.cuda.synchronize()
    out, lse, Q = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    s = float(np.float32(dim ** -0.5 if scale is None else scale))
    for b in range(len(pool.lens)):
        if not pool.news[b]:
            continue
        rows = slice(int(pool.starts[b]), int(pool.starts[b + 1]))
        at = [p for _, c, p in pool.places() if c == b]
        held = min(max(pool.lens[b], 0), pool.table.shape[1] * pool.page)
        for h in range(pool.heads):
            K, V, there = ref.kv4_decode(pool.cache, pool.page, dim, pool.table[b], held, h)
            for j in range(h * each, (h + 1) * each):
                o, e, mass, reach = ref.attention(Q[rows, j], K, V, there, at, s, window)
                err = ((dim + 16) * U * reach)[:, None]
                sums = (held / 64 + 80) * U
                w, w2 = (0.0, 0.0) if dtype == "fp32" else (2.0 ** -11, held * 2.0 ** -25)
                bound = (2 * err + sums + w) * mass + w2 * (np.abs(V[there]).max() if there.any() else 0) + unit * np.abs(o) + 1e-30
                assert np.all(np.abs(out[rows, j] - o) <= bound), (b, j, np.max(np.abs(out[rows, j] - o) / bound))
                none = np.isneginf(e)
                assert np.array_equal(np.isneginf(lse[rows, j]), none) and np.all(out[rows, j][none] == 0)
                with np.errstate(invalid="ignore"):
                    off = np.abs(lse[rows, j] - e)
                assert np.all(off[~none] <= (err[:, 0] + sums + 2 * U * np.abs(e))[~none])
    return out


SHAPES = [
    # heads of a model of this width at one token each: every length around a tile, an empty sequence
    (128, 16, 8, 32, [1, 15, 16, 17, 63, 64, 65, 0, 127, 128, 300], [1] * 11, 0),
    (64, 32, 2, 2, [5, 100, 64], [1, 1, 1], 0),                      # each query head its own cache head
    (256, 16, 1, 4, [33, 500], [1, 1], 0),
    (128, 64, 1, 8, [200, 70], [1, 1], 0),
    (64, 16, 1, 5, [90, 31], [1, 1], 0),                             # five query heads a cache head
    (128, 32, 1, 16, [250], [1], 0),
    (64, 16, 1, 64, [70], [1], 0),
    # drafted tokens, some sequences without any, one with fewer tokens held than new
    (128, 16, 2, 8, [40, 7, 0, 130, 3], [3, 0, 0, 5, 5], 0),
    (64, 64, 2, 4, [200, 64], [9, 2], 33),                           # windows, odd
    (128, 16, 1, 4, [1000], [1], 1), (128, 16, 2, 8, [700, 90], [1, 1], 100),
    (256, 32, 1, 2, [120], [7], 5),
    # chunks: a whole prompt, a chunk behind others, odd numbers of rows
    (128, 64, 2, 8, [150, 97, 260], [150, 33, 64], 0), (64, 16, 1, 1, [257], [257], 0), (256, 32, 1, 4, [140], [100], 0),
    (128, 32, 1, 5, [222], [77], 60), (64, 128, 2, 6, [300, 41], [130, 41], 0), (128, 1024, 1, 3, [515], [129], 0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,page,heads,heads_q,lens,news,window", SHAPES)
def test_attention_matches_oracle(ext, dtype, dim, page, heads, heads_q, lens, news, window):
    pool = Pool(lens, news, heads, dim, page, dim + len(lens)).fill()
    check_attention(ext, pool, heads_q, dtype, window)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_long(ext, dtype):
    """Lengths past what one workgroup takes, without the launch hints too."""
    pool = Pool([4500, 1, 2777], [1, 1, 1], 1, 128, 64, 1).fill()
    a = check_attention(ext, pool, 4, dtype)
    b = check_attention(ext, pool, 4, dtype, hints=False)
    assert np.allclose(a, b, rtol=2.0 ** -7, atol=2.0 ** -10)
    check_attention(ext, Pool([3001, 900], [6, 3], 1, 64, 16, 2).fill(), 2, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_wrong_hints(ext, dtype):
    """Hints below the truth change the launch, not the result."""
    pool = Pool([900, 333], [70, 3], 1, 128, 32, 4).fill()
    t = TYPES[dtype][0]
    q = torch.randn((73, 4, 128), device="cuda").to(t)
    cache, table, lens, starts = pool.gpu()
    want, wl = ext.kv4_attention(cache, q, table, lens, starts=starts)
    for mn, ml in ((1, 1), (2, 64), (100000, 10 ** 6)):
        got, gl = ext.kv4_attention(cache, q, table, lens, starts=starts, max_new=mn, max_len=ml)
        # two results within the bound of the exact one: here a few units of the type at most
        assert torch.allclose(got.float(), want.float(), rtol=2.0 ** -7 if dtype != "fp32" else 1e-4, atol=2e-3 if dtype != "fp32" else 1e-5)
        assert torch.allclose(gl, wl, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [2.0 ** -12, 200.0])
def test_attention_small_and_large_values(ext, dtype, size):
    """Values near the smallest steps, and large scores (one key takes all the weight)."""
    pool = Pool([130, 20], [1, 1], 2, 128, 16, 9).fill(size)
    check_attention(ext, pool, 8, dtype)
    pool = Pool([200, 20], [90, 20], 1, 128, 16, 9).fill(size)
    check_attention(ext, pool, 4, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("news", [[1, 1], [60, 40]])
def test_attention_nonfinite(ext, dtype, news):
    """NaN in what no row sees changes nothing; in a seen key or value it makes the rows NaN that see it; a NaN or
    an infinity in q makes that row NaN alone."""
    dim, page, heads = 128, 16, 1
    t = TYPES[dtype][0]
    pool = Pool([100, 90], news, heads, dim, page, 6).fill()
    cache, table, lens, starts = pool.gpu()
    q = torch.randn((sum(news), 4, dim), device="cuda").to(t)
    want, wl = ext.kv4_attention(cache, q, table, lens, starts=starts)
    assert torch.isfinite(want).all() and torch.isfinite(wl).all()
    nan = torch.full((2, 1, dim), math.nan, device="cuda")
    # the place behind each sequence's last token
    beyond = torch.tensor([101, 91], dtype=torch.int32, device="cuda")
    dirty = cache.clone()
    ext.kv4_append(dirty, nan, nan, table, beyond)
    got, gl = ext.kv4_attention(dirty, q, table, lens, starts=starts)
    assert torch.equal(got, want) and torch.equal(gl, wl)
    # position 95 of the first sequence
    for kk, vv in ((nan[:1], torch.ones_like(nan[:1])), (torch.ones_like(nan[:1]), nan[:1])):
        dirty = cache.clone()
        ext.kv4_append(dirty, kk, vv, table[:1], torch.tensor([96], dtype=torch.int32, device="cuda"))
        got, gl = ext.kv4_attention(dirty, q, table, lens, starts=starts)
        sees = torch.tensor([p >= 95 and b == 0 for _, b, p in pool.places()], device="cuda")
        assert torch.isnan(got[sees]).all()
        assert torch.equal(got[~sees], want[~sees]) and torch.equal(gl[~sees], wl[~sees])
    for bad in (math.nan, math.inf, -math.inf):
        q2 = q.clone()
        q2[0, 2, 5] = bad
        got, gl = ext.kv4_attention(cache, q2, table, lens, starts=starts)
        assert torch.isnan(got[0, 2]).all() and torch.isnan(gl[0, 2])
        other = torch.ones((sum(news), 4), dtype=torch.bool, device="cuda")
        other[0, 2] = False
        assert torch.equal(got[other], want[other]) and torch.equal(gl[other], wl[other])


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_pages_without_tokens(ext, dtype):
    """Pages outside the pool count as masked; a row that sees only such pages is empty; lengths above the table."""
    pool = Pool([100, 30, 80], [1, 1, 1], 1, 64, 16, 8).fill()
    pool.table[0, 2], pool.table[1, :] = 10 ** 7, -1
    check_attention(ext, pool, 4, dtype)
    pool.lens = [100, 30, 10 ** 6]
    dcache, table, lens, starts = pool.gpu()
    out, lse = ext.kv4_attention(dcache, torch.ones((3, 4, 64), device="cuda", dtype=TYPES[dtype][0]), table, lens)
    assert torch.isfinite(out).all() and (out[1] == 0).all() and torch.isneginf(lse[1]).all()
    pool = Pool([100, 64], [50, 64], 1, 64, 16, 8).fill()
    pool.table[0, 2], pool.table[1, 0] = 10 ** 7, -1
    check_attention(ext, pool, 4, dtype)


@pytest.mark.parametrize("news", [[1], [40]])
def test_attention_strides_and_scale(ext, news):
    """q as a slice of a fused projection at an odd place; another scale, zero among them."""
    pool = Pool([77], news, 2, 64, 16, 3).fill()
    cache, table, lens, starts = pool.gpu()
    for dtype, (t, _) in TYPES.items():
        flat = torch.randn((news[0], 5 + 4 * 64 + 2 * 64), device="cuda").to(t)
        q = flat[:, 5:5 + 256].unflatten(1, (4, 64))
        a, al = ext.kv4_attention(cache, q, table, lens, starts=starts)
        b, bl = ext.kv4_attention(cache, q.contiguous(), table, lens, starts=starts)
        assert torch.equal(a, b) and torch.equal(al, bl)
        for scale in (0.02, 0.0, -0.1):
            check_attention(ext, pool, 4, dtype, scale=scale) if scale >= 0 else ext.kv4_attention(cache, q, table, lens, starts=starts, scale=scale)


def test_attention_far_pages(ext):
    """A cache past 4 GiB, the sequence in its last pages: offsets past 32 bits."""
    dim, page, heads = 128, 1024, 8
    per = page * (dim + dim // 16)
    pages = (5 << 30) // (per * heads)
    cache = torch.zeros((pages, heads, per), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    small = torch.zeros((2, heads, per), dtype=torch.uint8, device="cuda")
    near = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    n = 1100
    lens, starts = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    k, v = torch.randn((n, heads, dim), device="cuda"), torch.randn((n, heads, dim), device="cuda")
    for c, t in ((cache, table), (small, near)):
        ext.kv4_append(c, k, v, t, lens, starts=starts)
    assert torch.equal(cache[-2:], small)
    for dtype in (torch.float32, torch.bfloat16):
        for new in (1, 130):
            q = torch.randn((new, 32, dim), device="cuda").to(dtype)
            st = None if new == 1 else torch.tensor([0, new], dtype=torch.int32, device="cuda")
            a, b = ext.kv4_attention(cache, q, table, lens, starts=st), ext.kv4_attention(small, q, near, lens, starts=st)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_other_stream_graph_and_repeats(ext):
    pool = Pool([1500, 40, 0], [1, 1, 1], 2, 128, 32, 5).fill()
    cache, table, lens, starts = pool.gpu()
    q = torch.randn((3, 8, 128), device="cuda")
    want, wl = ext.kv4_attention(cache, q, table, lens)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, gl = ext.kv4_attention(cache, q, table, lens)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(gl, wl)
    out = torch.empty_like(q)
    ws = torch.empty(max(256, ext.kv4_attention_workspace_bytes(8, 2, 128, q.dtype, 3, 3, 1, 2048)), dtype=torch.uint8, device="cuda")
    k = torch.randn((3, 2, 128), device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):                          # one step: the new token enters the cache, then attention
        ext.kv4_append(cache, k, k, table, lens)
        ext.kv4_attention(cache, q, table, lens, out=out, max_len=2048, workspace=ws)
    for i in range(4):
        q.normal_()
        k.normal_()
        lens.add_(1)
        table[2, 0] = cache.shape[0] - 1
        g.replay()
        torch.cuda.synchronize()
        again, _ = ext.kv4_attention(cache, q, table, lens, max_len=2048)
        assert torch.equal(out, again)


def test_refusals(ext):
    pool = Pool([10, 20], [1, 1], 2, 64, 16, 1)
    cache, table, lens, _ = pool.gpu()
    q = torch.zeros((2, 4, 64), device="cuda")
    k = torch.zeros((2, 2, 64), device="cuda")
    bad = [lambda: ext.kv4_attention(cache, q.double(), table, lens), lambda: ext.kv4_attention(cache, q, table.long(), lens),
           lambda: ext.kv4_attention(cache, q, table, lens.long()), lambda: ext.kv4_attention(cache, q[:1], table, lens),
           lambda: ext.kv4_attention(cache[:, :, :-1], q, table, lens), lambda: ext.kv4_attention(cache.cpu(), q, table, lens),
           lambda: ext.kv4_attention(cache, q, table[:1], lens), lambda: ext.kv4_append(cache, k[:, :1], k[:, :1], table, lens),
           lambda: ext.kv4_append(cache, k, k[:1], table, lens), lambda: ext.kv4_append(cache, k.transpose(1, 2), k, table, lens),
           lambda: ext.kv4_read(cache, table, lens, 64, starts=lens)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ext.kv4_attention(cache, q[:, :3], table, lens), lambda: ext.kv4_attention(cache, q, table, lens, window=-1),
              lambda: ext.kv4_attention(cache, q, table, lens, scale=math.nan), lambda: ext.kv4_cache(4, 2, 96, 16),
              lambda: ext.kv4_cache(4, 2, 64, 24)):
        with pytest.raises(ext.ExterndError):
            f()
    assert ext.kv4_cache(3, 2, 64, 16).shape == (3, 2, 16 * 68)
