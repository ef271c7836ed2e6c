"""GPU parity of attention of many rows over the 4-bit cache (256 rows a
workgroup: the calls of bf16 and fp16 queries with many rows and enough
work) with its definition in 64 bits.

Bound (u = 2^-24, n visible keys, D channels, unit t of the result's type:
2^-8, 2^-11): a score's exact products are summed in fp32, so it is within
e = (D + 16) u scale sum |q k^| of the exact one, the largest such sum a row
sees taken for all; a weight carries 2 e + (n / 64 + 80) u (exponential, its
argument, sums and the joining of parts), and is rounded to fp16 for the
product with the values, 2^7 above its share of the reference and so at
least that of the row's largest: 2^-12 of itself, or half of fp16's smallest
step, 2^-25 2^-7 of the largest weight.  So
  |out - exact| <= (2 e + (n / 64 + 80) u + 2^-12) sum p |v| + n 2^-32 max |v| + t |out|
  |lse - exact| <= e + (n / 64 + 80) u + 2 u |lse|."""
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


def check(ext, c, q, dtype, window=0, scale=None, max_len=None, out=None):
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
            bound = (2 * err + sums + 2.0 ** -12)[..., None] * mass + n * 2.0 ** -32 * big + unit * np.abs(o)
            assert np.all(np.abs(G[rows, hs] - o) <= bound), (b, h, np.max(np.abs(G[rows, hs] - o) / (bound + 1e-300)))
            none = np.isneginf(e)
            assert np.array_equal(np.isneginf(L[rows, hs]), none)
            assert np.all(np.abs(L[rows, hs] - e)[~none] <= (err + sums + 2 * U * np.abs(e))[~none])
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
    check(ext, c, q, dtype, max_len=10 ** 6)


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
