"""GPU parity of attention of many rows over the 4-bit cache (256 rows a
workgroup: the calls of bf16 and fp16 queries with many rows and enough
work) with its definition in 64 bits.

Bound (u = 2^-24, n visible keys, D channels, unit t of the result's type:
2^-8, 2^-11): a score's exact products are summed in fp32, so it is within
e = (D + 16) u scale sum |q k^| of the exact one, the largest such sum a row
sees taken for all; a weight carries 2 e + (n / 64 + 80) u (exponential, its
argument, sums and the joining of parts), and is rounded to fp16 for the
product with the values, 2^7 above its share of the reference and so at
least that of the row's largest: w = 2^-11 of itself (half a step of 11
bits), or half of fp16's smallest step, 2^-25 2^-7 of the largest weight.  So
  |out - exact| <= (2 e + (n / 64 + 80) u + w) sum p |v| + n 2^-32 max |v| + t |out|
  |lse - exact| <= e + (n / 64 + 80) u + 2 u |lse|.
The test of weak keys, whose weights are all one number, holds w = 2^-12."""
import math

import numpy as np
import pytest

import oracle.decode_oracle as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


@pytest.fixture(scope="module")
def ext():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13511_amd import binding
    binding.lib()
    return binding


class Cache:
    """Whole sequences of given k and v (a list of (tokens, heads, D) each), stored by the oracle in pages of a pool in
    random order over arbitrary bytes."""

    def __init__(self, ks, vs, news, page, seed=0):
        rng = np.random.default_rng(seed)
        self.news, self.lens, self.page = news, [len(k) for k in ks], page
        self.heads, self.dim = ks[0].shape[1:]
        need = [-(-n // page) for n in self.lens]
        order = rng.permutation(sum(need) + 2)
        self.table = np.full((len(ks), max(need + [1])), -1, np.int32)
        self.cache = rng.integers(0, 256, (len(order), self.heads, page * (self.dim + self.dim // 16)), dtype=np.uint8)
        at = 0
        for b, (k, v) in enumerate(zip(ks, vs)):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            if len(k):
                ref.kv4_encode(self.cache, page, k, v, self.table[b], 0, self.heads)
        self.starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.tokens = int(self.starts[-1])

    def gpu(self):
        return [torch.from_numpy(x).cuda() for x in (self.cache, self.table, np.array(self.lens, np.int32), self.starts)]


def exact(c, b, h, Q, scale, window):
    """The definition over what the cache holds, for the rows of sequence b and one cache head: Q (tokens, query heads of
    it, D) -> out, lse, and what the bounds need: sum p |v|, the largest sum of |q k| scale, the largest |v|, keys."""
    n, new = min(max(c.lens[b], 0), c.table.shape[1] * c.page), c.news[b]
    K, V, there = ref.kv4_decode(c.cache, c.page, c.dim, c.table[b], n, h)
    at, j = c.lens[b] - new + np.arange(new)[:, None], np.arange(n)[None]
    seen = ((j <= at) & there[None] & ((j > at - window) if window else True))[:, None]      # tokens, 1, keys
    K0, V0 = np.nan_to_num(K, nan=0.0), np.nan_to_num(V, nan=0.0)
    x = np.where(seen, scale * np.matmul(Q, K.T), -np.inf)
    top = x.max(-1, keepdims=True, initial=-np.inf)
    e = np.where(seen, np.exp(x - np.where(np.isneginf(top), 0, top)), 0.0)
    total = e.sum(-1)
    with np.errstate(divide="ignore"):
        lse = np.log(total) + np.where(np.isneginf(top), 0, top)[..., 0]
    p = e / np.where(total == 0, 1.0, total)[..., None]
    reach = abs(scale) * np.where(seen, np.matmul(np.abs(Q), np.abs(K0).T), 0.0).max(-1, initial=0.0)
    return np.matmul(p, V0), lse, np.matmul(p, np.abs(V0)), reach, np.abs(V0).max(initial=0.0), n


def check(ext, c, q, dtype, window=0, scale=None, max_len=None, out=None, weight=2.0 ** -11):
    """Attention of q (tokens, query heads, D) on the GPU against ``exact``; returns (out, lse)."""
    unit = TYPES[dtype][1]
    cache, table, lens, starts = c.gpu()
    got, lse = ext.kv4_attention(cache, q, table, lens, starts=starts, max_new=max(c.news), max_len=max_len, window=window,
                                 scale=scale, out=out)
    torch.cuda.synchronize()
    s = float(np.float32(c.dim ** -0.5 if scale is None else scale))
    G, L, Q = got.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    each = q.shape[1] // c.heads
    for b in range(len(c.lens)):
        rows = slice(int(c.starts[b]), int(c.starts[b + 1]))
        for h in range(c.heads):
            hs = slice(h * each, (h + 1) * each)
            o, e, mass, reach, big, n = exact(c, b, h, Q[rows, hs], s, window)
            err, sums = (c.dim + 16) * U * reach, (n / 64 + 80) * U
            bound = (2 * err + sums + weight)[..., None] * mass + n * 2.0 ** -32 * big + unit * np.abs(o)
            assert np.all(np.abs(G[rows, hs] - o) <= bound), (b, h, np.max(np.abs(G[rows, hs] - o) / (bound + 1e-300)))
            none = np.isneginf(e)
            assert np.array_equal(np.isneginf(L[rows, hs]), none)
            assert np.all(np.abs(L[rows, hs][~none] - e[~none]) <= (err + sums + 2 * U * np.abs(e))[~none])
    return got, lse


def random_cache(lens, news, heads, dim, page, seed):
    rng = np.random.default_rng(seed)
    loud = 1 + 5 * (rng.random((1, heads, dim)) < 0.05)
    ks = [rng.standard_normal((n, heads, dim)) * loud + 0.5 * loud for n in lens]
    return Cache(ks, [rng.standard_normal((n, heads, dim)) for n in lens], news, page, seed)


# ---------------------------------------------------------------------------
# small weights
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nats", [9.0, 13.0, 17.0, 17.5, 20.0])
def test_weak_keys_beside_a_dominating_one(ext, dtype, nats):
    """One key far above all others, its value zero: the result is the others' weights alone, each e^-nats of the
    largest.  (As fp16 numbers below the largest weight itself, those of 17 nats lost a fifth and those of 20 all.)"""
    dim, n, new, heads_q, rng = 128, 800, 400, 8, np.random.default_rng(3)
    k, v = np.zeros((n, 1, dim)), rng.standard_normal((n, 1, dim)) + 1.0
    k[0, 0, 0], v[0] = 1.0, 0.0
    c = Cache([k], [v], [new], 64)
    held = ref.kv4_values(k[:1])[0, 0, 0]
    q = torch.from_numpy(rng.standard_normal((new, heads_q, dim)))
    q[..., 0] = nats * math.sqrt(dim) / held
    q = q.to(TYPES[dtype][0]).cuda()
    # as many tiles as for 10^6 tokens: the form with 256 rows a workgroup, and parts that are joined
    assert ext.kv4_attention_workspace_bytes(heads_q, 1, dim, q.dtype, new, 1, new, 10 ** 6) > 768 * (8 * (dim + 4) * 4 + 32)
    check(ext, c, q, dtype, max_len=10 ** 6, weight=2.0 ** -12)


# ---------------------------------------------------------------------------
# windows
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("lens,news", [([7, 30], [12, 1]), ([500, 90], [505, 40])])
@pytest.mark.parametrize("window", [500, (1 << 31) - 1, (1 << 31) - 3, 1 << 31, (1 << 32) + 5, 1 << 40])
def test_windows_past_all_positions(ext, lens, news, window):
    """A window wider than any distance masks nothing, also where a sequence holds fewer tokens than it has new ones
    (positions below 0): the bits of the call without one."""
    rng = np.random.default_rng(1)
    ks, vs = ([rng.standard_normal((n, 2, 64)) for n in lens] for _ in range(2))
    cache, table, dlens, starts = Cache(ks, vs, news, 32).gpu()
    for dtype in (torch.float32, torch.bfloat16):
        q = torch.randn((sum(news), 32, 64), device="cuda").to(dtype)
        a, al = ext.kv4_attention(cache, q, table, dlens, starts=starts, max_new=max(news))
        b, bl = ext.kv4_attention(cache, q, table, dlens, starts=starts, max_new=max(news), window=window)
        assert torch.equal(a, b) and torch.equal(al, bl)
        assert torch.isneginf(al[:5]).all() and torch.isfinite(al[5:]).all()


# ---------------------------------------------------------------------------
# lengths up to 2^31 - 1
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_lengths_to_the_end_of_32_bits(ext, dim):
    """The last tokens of a sequence of 2^31 - 1 whose other pages are none, beside the same tokens in a short sequence:
    with a window the same tiles and bits, without one the same numbers (other parts are joined)."""
    page, heads_q = 1024, 32
    n, short = (1 << 31) - 1, 2047                        # alike modulo the page
    rng = np.random.default_rng(dim)
    c = Cache([rng.standard_normal((short, 1, dim))], [rng.standard_normal((short, 1, dim))], [1], page)
    cache, table, lens, _ = c.gpu()
    far = torch.full((1, 1 << 21), -1, dtype=torch.int32, device="cuda")
    far[0, -2:] = table[0]
    far_lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    for dtype, new in ((torch.float32, 1), (torch.bfloat16, 1), (torch.bfloat16, 40)):
        q = torch.randn((new, heads_q, dim), device="cuda").to(dtype)
        starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        kw = dict(starts=starts, max_new=new, max_len=10 ** 6)
        for window in (1, 100, 0):
            a, al = ext.kv4_attention(cache, q, far, far_lens, window=window, **kw)
            b, bl = ext.kv4_attention(cache, q, table, lens, window=window, **kw)
            torch.cuda.synchronize()
            assert torch.isfinite(bl).all()
            if window:
                assert torch.equal(a, b) and torch.equal(al, bl)
            else:      # sums of the same terms in another order: a few units of fp32, and one of the result's type
                unit = 2.0 ** -20 if dtype is torch.float32 else 2.0 ** -7
                assert torch.allclose(a.float(), b.float(), rtol=unit, atol=unit / 64) and torch.allclose(al, bl, rtol=1e-6, atol=1e-5)
    # whole sequences, new tokens and all: kept and read at the end
    k = torch.randn((3, 1, dim), device="cuda")
    starts = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    ext.kv4_append(cache, k, k, far, far_lens, starts=starts)
    got, _ = ext.kv4_read(cache, table, lens, dim, starts=starts, tokens=3)
    far_got, _ = ext.kv4_read(cache, far, far_lens, dim, starts=starts, tokens=3)
    assert torch.equal(got, far_got) and (got != 0).any()


# ---------------------------------------------------------------------------
# queries that are not finite
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("max_len", [None, 10 ** 6])      # one launch, and parts that are joined
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_nonfinite_queries_that_see_nothing(ext, dtype, max_len, bad):
    """A query that sees no key gives 0 and -infinity whatever it holds; one that sees any gives NaN; no other row changes."""
    lens, news, heads_q, dim = [500, 90], [505, 40], 16, 64
    c = random_cache(lens, news, 1, dim, 16, 4)
    c.table[1, 0] = -1                                    # the first 16 positions of the second sequence
    c.lens[1] = 20                                        # its first 36 new tokens see nothing, 4 see a page
    q = torch.randn((sum(news), heads_q, dim), device="cuda").to(TYPES.get(dtype, (torch.float32,))[0])
    cache, table, dlens, starts = c.gpu()
    kw = dict(starts=starts, max_new=max(news), max_len=max_len)
    want, wl = ext.kv4_attention(cache, q, table, dlens, **kw)
    sees = torch.tensor([t >= 5 for t in range(505)] + [t >= 36 for t in range(40)], device="cuda")
    assert torch.isfinite(want).all() and torch.equal(torch.isfinite(wl), sees[:, None].expand(-1, heads_q))
    hit = torch.zeros((sum(news), heads_q), dtype=torch.bool, device="cuda")
    hit[::3, 1::5] = True
    q2 = q.clone()
    q2[..., 7] = torch.where(hit, torch.full_like(q[..., 7], bad), q[..., 7])
    got, gl = ext.kv4_attention(cache, q2, table, dlens, **kw)
    nan = hit & sees[:, None]
    assert torch.isnan(got[nan]).all() and torch.isnan(gl[nan]).all()
    assert torch.equal(got[~nan], want[~nan]) and torch.equal(gl[~nan], wl[~nan])


# ---------------------------------------------------------------------------
# alignment
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("max_len", [None, 10 ** 6])
def test_results_at_any_place(ext, dtype, dim, max_len):
    """``out`` as a dense view that starts at any entry: the bits of an aligned one, and nothing beside it."""
    c = random_cache([300, 70], [300, 33], 1, dim, 32, 5)
    heads_q, n = 32, 333 * 32 * dim
    t = TYPES.get(dtype, (torch.float32,))[0]
    q = torch.randn((333, heads_q, dim), device="cuda").to(t)
    cache, table, lens, starts = c.gpu()
    kw = dict(starts=starts, max_new=300, max_len=max_len)
    want, wl = ext.kv4_attention(cache, q, table, lens, **kw)
    for lead in (1, 2, 3):
        flat = torch.zeros(n + 8, device="cuda", dtype=t)
        got, gl = ext.kv4_attention(cache, q, table, lens, out=flat[lead:lead + n].view(333, heads_q, dim), **kw)
        assert torch.equal(got, want) and torch.equal(gl, wl)
        assert (flat[:lead] == 0).all() and (flat[lead + n:] == 0).all()


# ---------------------------------------------------------------------------
# the kernel of 256 rows at every width, in one launch and with parts joined
# ---------------------------------------------------------------------------
FORMS = {"one launch": None, "joined": 10 ** 6}      # max_len: the longest length, or as many tiles as that has


def on_the_wide_kernel(ext, c, heads_q, dtype, form):
    """max_len of the form, once the plan is known to be that of 256 rows and of the form."""
    most = max(c.lens) if FORMS[form] is None else FORMS[form]
    args = (heads_q, c.heads, c.dim, TYPES[dtype][0], c.tokens, len(c.lens), max(c.news), most)
    assert ext.kv4_attention_block_rows(*args) == 256
    assert (ext.kv4_attention_workspace_bytes(*args) == 0) == (form == "one launch")
    return most


def queries(c, heads_q, dtype, seed=0):
    q = np.random.default_rng(seed).standard_normal((c.tokens, heads_q, c.dim)).astype(np.float32)
    return torch.from_numpy(q).to(TYPES[dtype][0]).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("heads,each,page,lens,news,window", [
    # prompts, a chunk behind held tokens, an empty sequence and one without new tokens
    (2, 12, 16, [300, 97, 0, 41, 9], [300, 33, 0, 41, 0], 0),
    (1, 32, 64, [450, 70], [200, 64], 0),
    # windows: one position, within a tile, over tiles, and longer than all
    (1, 32, 32, [333, 100], [240, 40], 1), (2, 16, 128, [400, 65], [222, 65], 37), (1, 32, 16, [500], [333], 200),
    (1, 24, 256, [511], [400], 5000),
    # fewer tokens held than new ones, lengths around tiles; five query heads a cache head
    (1, 32, 32, [65, 250, 64], [80, 129, 64], 0), (4, 5, 1024, [385, 129], [257, 129], 0), (3, 15, 16, [255], [255], 64)])
def test_wide_kernel_matches_definition(ext, dtype, dim, form, heads, each, page, lens, news, window):
    c = random_cache(lens, news, heads, dim, page, dim + len(lens))
    most = on_the_wide_kernel(ext, c, heads * each, dtype, form)
    check(ext, c, queries(c, heads * each, dtype), dtype, window=window, max_len=most)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_wide_kernel_long(ext, dtype, dim):
    """Several tiles a workgroup and row blocks that many share, their first and last rows in one."""
    c = random_cache([2100, 1500], [130, 3], 1, dim, 64, dim)
    most = on_the_wide_kernel(ext, c, 8, dtype, "joined")
    check(ext, c, queries(c, 8, dtype), dtype, max_len=most)
    c = random_cache([1700], [1700], 1, dim, 32, dim)      # one query head a cache head
    most = on_the_wide_kernel(ext, c, 1, dtype, "joined")
    check(ext, c, queries(c, 1, dtype), dtype, max_len=most, window=700)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", FORMS)
def test_wide_kernel_scales(ext, dtype, dim, form):
    c = random_cache([260, 90], [260, 50], 1, dim, 32, 2)
    most, q = on_the_wide_kernel(ext, c, 32, dtype, form), queries(c, 32, dtype)
    for scale in (0.0, -0.11, 3.0):
        check(ext, c, q, dtype, scale=scale, max_len=most)
    for size in (2.0 ** -18, 2.0 ** 6):                   # queries near the smallest and of large scores
        check(ext, c, q * size, dtype, max_len=most)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", FORMS)
def test_wide_kernel_pages_without_tokens(ext, dtype, dim, form):
    """Pages outside the pool are masked; rows that see only such pages are empty."""
    c = random_cache([300, 160], [280, 160], 1, dim, 16, 3)
    c.table[0, 2], c.table[0, 9], c.table[1, :3] = 10 ** 7, -1, -5
    most = on_the_wide_kernel(ext, c, 32, dtype, form)
    _, lse = check(ext, c, queries(c, 32, dtype), dtype, max_len=most)
    assert torch.isneginf(lse[280:280 + 48]).all() and torch.isfinite(lse[280 + 48:]).all()
    check(ext, c, queries(c, 32, dtype), dtype, max_len=most, window=20)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", FORMS)
def test_wide_kernel_strided_queries(ext, dtype, dim, form):
    """q as a slice of a fused projection at an odd place, and head by head in memory: the bits of a dense one."""
    c = random_cache([280, 30], [280, 25], 1, dim, 32, 6)
    most, q = on_the_wide_kernel(ext, c, 32, dtype, form), queries(c, 32, dtype)
    want, wl = check(ext, c, q, dtype, max_len=most)
    cache, table, lens, starts = c.gpu()
    flat = torch.zeros((c.tokens, 3 + 32 * dim + 2), device="cuda", dtype=q.dtype)
    flat[:, 3:3 + 32 * dim] = q.flatten(1)
    for other in (flat[:, 3:3 + 32 * dim].unflatten(1, (32, dim)), q.transpose(0, 1).contiguous().transpose(0, 1)):
        got, gl = ext.kv4_attention(cache, other, table, lens, starts=starts, max_new=max(c.news), max_len=most)
        assert torch.equal(got, want) and torch.equal(gl, wl)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window", [0, 90])
def test_wide_kernel_nan_in_the_cache(ext, dtype, dim, form, window):
    """64 channels of one token's key held as NaN make every row NaN that sees it; of its value, those 64 channels.  All
    else keeps its bits."""
    lens, news, each = [400, 120], [300, 120], 32
    c = random_cache(lens, news, 1, dim, 32, 8)
    most, q = on_the_wide_kernel(ext, c, each, dtype, form), queries(c, each, dtype)
    want, wl = check(ext, c, q, dtype, window=window, max_len=most)
    cache, table, dlens, starts = c.gpu()
    kw = dict(starts=starts, max_new=max(news), max_len=most, window=window)
    at = torch.tensor([p for b in range(2) for p in range(lens[b] - news[b], lens[b])], device="cuda")
    for token, group in ((3, 0), (200, dim // 64 - 1), (327, dim // 128), (399, 0)):
        sees = (at >= token) & (torch.arange(c.tokens, device="cuda") < news[0])
        sees &= (at < token + window) if window else True
        word = 32 * dim + 2 * ((token % 32 * 2) * (dim // 64) + group)
        for which in (0, 1):
            dirty = cache.clone()
            m = dirty[int(c.table[0, token // 32]), 0]
            m[word + which * (dim // 64) * 2 + 1] = 0x7E      # the scale word's upper byte: a NaN
            got, gl = ext.kv4_attention(dirty, q, table, dlens, **kw)
            assert torch.equal(got[~sees], want[~sees]) and torch.equal(gl[~sees], wl[~sees])
            if which == 0:
                assert torch.isnan(got[sees]).all() and torch.isnan(gl[sees]).all()
            else:
                hit = torch.zeros(dim, dtype=torch.bool, device="cuda")
                hit[group * 64:group * 64 + 64] = True
                assert torch.isnan(got[sees][..., hit]).all()
                assert torch.equal(got[sees][..., ~hit], want[sees][..., ~hit]) and torch.equal(gl, wl)


def test_wide_kernel_same_bits_every_time(ext):
    """Repeats, another stream, and replays of a graph."""
    c = random_cache([900, 300], [300, 300], 2, 128, 64, 9)
    cache, table, lens, starts = c.gpu()
    q = queries(c, 16, "bf16")
    most = on_the_wide_kernel(ext, c, 16, "bf16", "joined")
    kw = dict(starts=starts, max_new=300, max_len=most)
    want, wl = ext.kv4_attention(cache, q, table, lens, **kw)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got, gl = ext.kv4_attention(cache, q, table, lens, **kw)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(gl, wl)
    out = torch.empty_like(q)
    ws = torch.empty(ext.kv4_attention_workspace_bytes(16, 2, 128, q.dtype, 600, 2, 300, most), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ext.kv4_attention(cache, q, table, lens, out=out, workspace=ws, **kw)
    for _ in range(3):
        q.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ext.kv4_attention(cache, q, table, lens, **kw)[0])


def test_workspaces(ext):
    """A given workspace is device memory without gaps and is counted in bytes; any other is refused before a launch."""
    c = random_cache([900], [1], 1, 64, 64, 10)
    cache, table, lens, starts = c.gpu()
    q = queries(c, 8, "bf16")
    kw = dict(starts=starts, max_new=1, max_len=10 ** 5)
    need = ext.kv4_attention_workspace_bytes(8, 1, 64, q.dtype, 1, 1, 1, 10 ** 5)
    assert need > 0 and need % 256 == 0
    want, wl = ext.kv4_attention(cache, q, table, lens, **kw)
    for ws in (torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty(need // 4, device="cuda"),
               torch.empty((need // 512, 64), dtype=torch.float64, device="cuda")):
        got, gl = ext.kv4_attention(cache, q, table, lens, workspace=ws, **kw)
        assert torch.equal(got, want) and torch.equal(gl, wl)
    for ws in (torch.empty(need, dtype=torch.uint8), torch.empty((need, 2), dtype=torch.uint8, device="cuda")[:, 0]):
        with pytest.raises(ValueError):
            ext.kv4_attention(cache, q, table, lens, workspace=ws, **kw)
    for ws in (torch.empty(need - 256, dtype=torch.uint8, device="cuda"), torch.empty(need + 256, dtype=torch.uint8, device="cuda")[8:]):
        with pytest.raises(ext.ExterndError):
            ext.kv4_attention(cache, q, table, lens, workspace=ws, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [0, 30, 70])
@pytest.mark.parametrize("each", [4, 32])
def test_lengths_past_the_table(ext, dtype, window, each):
    """Positions come from the length as it is; those past the table hold nothing, and a query there sees what the table
    holds of its window."""
    c = random_cache([256, 96], [200, 60], 1, 64, 32, 11)
    c.lens = [256 + 50, 256 + 100]                         # tables hold 256: the second's pages from its fourth on are none
    check(ext, c, queries(c, each, dtype), dtype, window=window)
    cache, table, lens, starts = c.gpu()
    before = cache.clone()
    k = torch.randn((c.tokens, 1, 64), device="cuda")
    ext.kv4_append(cache, k, k, table, lens, starts=starts)
    got, _ = ext.kv4_read(cache, table, lens, 64, starts=starts, tokens=c.tokens)
    assert (got[:150] != 0).any(-1).all() and (got[150:] == 0).all()
    own = [int(p) for p in c.table[0]]
    assert torch.equal(cache[[i for i in range(cache.shape[0]) if i not in own]], before[[i for i in range(cache.shape[0]) if i not in own]])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", FORMS)
def test_wide_kernel_lse_of_equal_scores(ext, dtype, dim, form):
    """Queries of 0: every score is 0, every weight a power of two and their sum exact, so the lse is ln n within the
    logarithm's own error (one unit, 2 u of it), the constant's and the product's (u each)."""
    c = random_cache([400], [400], 1, dim, 64, 12)
    most = on_the_wide_kernel(ext, c, 32, dtype, form)
    cache, table, lens, starts = c.gpu()
    q = torch.zeros((400, 32, dim), device="cuda", dtype=TYPES[dtype][0])
    _, lse = ext.kv4_attention(cache, q, table, lens, starts=starts, max_new=400, max_len=most)
    want = np.log(np.arange(1.0, 401.0))[:, None]
    assert np.all(np.abs(lse.double().cpu().numpy() - want) <= 4 * U * want)
