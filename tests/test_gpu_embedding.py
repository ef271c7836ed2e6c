"""GPU parity of the embedding and its gradient (externd_embedding, _backward)
with the oracle's fp64 form.

Tolerance (u = 2^-24): the embedding is one fp32 product rounded to its type
(u and half a step of the type).  A row's gradient of n terms is summed in
fp32 in some order (n - 1 roundings of sums of at most S = the terms'
absolute values), scaled or added with one more and rounded to its type:
(n + 1) u S, u |old + sum| and half a step."""
import math

import numpy as np
import pytest

import oracle.ends_oracle as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}
TINY = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -25}      # half a step of the smallest values, or more


@pytest.fixture(scope="module")
def ext():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13511_amd import binding
    binding.lib()
    return binding


def tensor(a, dtype):
    return torch.from_numpy(a).to(TYPES[dtype][0]).cuda()


def ids_of(kind, tokens, vocab, rng):
    if kind == "one":
        return np.full(tokens, vocab // 2)
    if kind == "none":
        return np.full(tokens, -1)
    if kind == "rising":
        return np.arange(tokens) % vocab
    if kind == "few":
        ids = rng.integers(0, min(3, vocab), tokens)
    else:
        ids = (rng.random(tokens) ** 6 * vocab).astype(np.int64)
    ids[rng.random(tokens) < 0.1] = -1
    ids[rng.random(tokens) < 0.05] = vocab          # outside too
    return ids


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,width,vocab", [(1, 1, 1), (3, 7, 5), (5, 64, 9), (33, 1001, 100), (2, 3, 40), (700, 72, 33), (257, 2560, 1000)])
def test_embedding(ext, dtype, tokens, width, vocab):
    rng = np.random.default_rng(tokens)
    table, ids = tensor(rng.standard_normal((vocab, width)), dtype), ids_of("skewed", tokens, vocab, rng)
    scale = float(np.float32(math.sqrt(width)))
    got = ext.embedding(table, torch.from_numpy(ids).cuda(), scale=scale).double().cpu().numpy()
    want = ref.embedding(table.double().cpu().numpy(), ids, scale)
    assert np.all(np.abs(got - want) <= (U + TYPES[dtype][1]) * np.abs(want) + TINY[dtype])


def test_embedding_strides_shapes_and_scales(ext):
    """Rows with gaps on either side, ids of two dimensions, scales of 0 and below (a missing row is +0), what is
    between the rows left as it was."""
    rng = np.random.default_rng(0)
    for dtype in TYPES:
        wide = tensor(rng.standard_normal((50, 131)), dtype)
        table = wide[:, 3:3 + 101]
        ids = torch.tensor([[4, -1, 49], [50, 0, 4]], device="cuda")
        for scale in (0.0, -1.5, 1.0):
            got = ext.embedding(table, ids, scale=scale)
            assert got.shape == (2, 3, 101)
            want = ref.embedding(table.double().cpu().numpy(), ids.view(-1).tolist(), scale)
            near = np.abs(got.double().cpu().numpy().reshape(6, 101) - want) <= (U + TYPES[dtype][1]) * np.abs(want)
            assert near.all() and not torch.signbit(got[0, 1]).any() and not torch.signbit(got[1, 0]).any()
        buf = torch.full((6, 119), 7.0, device="cuda", dtype=TYPES[dtype][0])
        assert ext.embedding(table, ids.view(-1), out=buf[:, 5:106]).data_ptr() == buf[:, 5:106].data_ptr()
        assert torch.equal(buf[:, 5:106], ext.embedding(table, ids.view(-1)))
        assert (buf[:, :5] == 7).all() and (buf[:, 106:] == 7).all()


def bound(dtype, want, size, count):
    n = count[:, None]
    return np.where(n > 0, (n + 1) * U * size + (U + TYPES[dtype][1]) * (np.abs(want) + (n + 2) * U * size) + TINY[dtype], 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,width,vocab,kind", [
    (1, 1, 1, "rising"), (3, 7, 5, "skewed"), (16, 64, 40, "rising"), (17, 65, 40, "one"), (33, 1001, 100, "skewed"),
    (300, 72, 33, "few"), (1000, 40, 70, "one"), (257, 2056, 1000, "skewed"), (64, 16, 8, "none"), (16383, 9, 3000, "skewed"),
    (16385, 8, 70000, "skewed"), (40000, 24, 3, "few"), (33000, 5, 600000, "rising"), (5000, 12, 513, "skewed")])
def test_backward(ext, dtype, tokens, width, vocab, kind):
    rng = np.random.default_rng(tokens + width)
    grad, ids = tensor(rng.standard_normal((tokens, width)), dtype), ids_of(kind, tokens, vocab, rng)
    scale, dev = float(np.float32(0.37)), torch.from_numpy(ids).cuda()
    got = ext.embedding_backward(grad, dev, vocab, scale=scale)
    assert torch.equal(got, ext.embedding_backward(grad, dev, vocab, scale=scale))
    want, size, count = ref.embedding_backward(grad.double().cpu().numpy(), ids, vocab, scale)
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound(dtype, want, size, count))


@pytest.mark.parametrize("dtype", TYPES)
def test_backward_accumulates(ext, dtype):
    """Into a table with gaps between its rows: rows without tokens, and the gaps, stay as they are."""
    rng = np.random.default_rng(5)
    for width in (65, 128):
        grad, ids = tensor(rng.standard_normal((400, width)), dtype), ids_of("skewed", 400, 90, rng)
        buf = tensor(rng.standard_normal((90, width + 9)), dtype)
        kept = buf.clone()
        old = kept[:, 4:4 + width].clone()
        got = ext.embedding_backward(grad, torch.from_numpy(ids).cuda(), 90, scale=2.0, out=buf[:, 4:4 + width], accumulate=True)
        want, size, count = ref.embedding_backward(grad.double().cpu().numpy(), ids, 90, 2.0)
        want = old.double().cpu().numpy() + want
        assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound(dtype, want, size, count))
        assert torch.equal(buf[:, :4], kept[:, :4]) and torch.equal(buf[:, 4 + width:], kept[:, 4 + width:])


@pytest.mark.parametrize("dtype", TYPES)
def test_backward_into_rows_with_gaps(ext, dtype):
    """Zeros reach the rows only."""
    rng = np.random.default_rng(6)
    grad, ids = tensor(rng.standard_normal((50, 33)), dtype), ids_of("skewed", 50, 70, rng)
    buf = torch.full((70, 50), 3.0, device="cuda", dtype=TYPES[dtype][0])
    got = ext.embedding_backward(grad, torch.from_numpy(ids).cuda(), 70, out=buf[:, 7:40])
    assert torch.equal(got, ext.embedding_backward(grad, torch.from_numpy(ids).cuda(), 70))
    assert (buf[:, :7] == 3).all() and (buf[:, 40:] == 3).all()


def test_padding_may_hold_anything(ext):
    """NaN and infinities where no id is; NaN where one is reaches that row only."""
    ids = torch.tensor([3, -1, 5, 9, 3], device="cuda")
    grad = torch.ones((5, 40), device="cuda")
    grad[1], grad[3] = math.nan, math.inf
    got = ext.embedding_backward(grad, ids, 9)
    assert torch.isfinite(got).all() and (got[3] == 2).all() and (got[5] == 1).all() and got.sum() == 120
    grad[2, 7] = math.nan
    got = ext.embedding_backward(grad, ids, 9)
    assert torch.isnan(got).sum() == 1 and torch.isnan(got[5, 7])


def test_nothing(ext):
    none = torch.empty((0,), dtype=torch.int64, device="cuda")
    table = torch.ones((4, 8), device="cuda")
    assert ext.embedding(table, none).shape == (0, 8)
    grad = torch.empty((0, 8), device="cuda")
    assert (ext.embedding_backward(grad, none, 4, out=table.clone()) == 0).all()
    assert torch.equal(ext.embedding_backward(grad, none, 4, out=table.clone(), accumulate=True), table)


def test_gradient_against_differences(ext):
    """The embedding is linear in its table: <grad, E(T + D) - E(T)> = <backward(grad), D>."""
    rng = np.random.default_rng(8)
    ids = torch.from_numpy(ids_of("skewed", 120, 30, rng)).cuda()
    table, grad, d = (torch.from_numpy(rng.integers(-8, 9, s).astype(np.float32)).cuda() for s in ((30, 20), (120, 20), (30, 20)))
    moved = ext.embedding(table + d, ids, scale=0.5) - ext.embedding(table, ids, scale=0.5)
    assert (grad * moved).sum().item() == (ext.embedding_backward(grad, ids, 30, scale=0.5) * d).sum().item()      # small whole numbers: exact


def test_other_streams_and_graphs(ext):
    """On a stream of its own with its own memory, and replayed from a graph on new contents with eager work in between."""
    rng = np.random.default_rng(9)
    ids = torch.from_numpy(ids_of("skewed", 500, 100, rng)).cuda()
    grad, table = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((500, 96), (100, 96)))
    want = ext.embedding(table, ids), ext.embedding_backward(grad, ids, 100)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ext.embedding(table, ids, stream=side), ext.embedding_backward(grad, ids, 100, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = ext.embedding(table, ids), ext.embedding_backward(grad, ids, 100)
    for i in range(3):
        ids.copy_(torch.from_numpy(ids_of("skewed" if i else "one", 500, 100, rng)).cuda())
        grad.mul_(1.5)
        g.replay()
        torch.cuda.synchronize()
        want = ext.embedding(table, ids), ext.embedding_backward(grad, ids, 100)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals(ext):
    t, ids = torch.ones((4, 8), device="cuda"), torch.zeros((3,), dtype=torch.int64, device="cuda")
    g = torch.ones((3, 8), device="cuda")
    bad = [lambda: ext.embedding(t.double(), ids), lambda: ext.embedding(t.t(), ids), lambda: ext.embedding(t, ids.int()),
           lambda: ext.embedding(t.cpu(), ids), lambda: ext.embedding(t, ids.cpu()), lambda: ext.embedding(t, ids, out=t[:3]),
           lambda: ext.embedding(t, ids, out=g[:2]), lambda: ext.embedding(t, ids, out=g.half()),
           lambda: ext.embedding_backward(g[:2], ids, 4), lambda: ext.embedding_backward(g, ids, 4, accumulate=True),
           lambda: ext.embedding_backward(g, ids, 4, out=g), lambda: ext.embedding_backward(g, ids, 4, out=t[:3]),
           lambda: ext.embedding_backward(g.t(), ids, 4), lambda: ext.embedding_backward(g, ids, 4, workspace=torch.empty(1 << 20))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ext.embedding(t, ids, scale=math.inf), lambda: ext.embedding(t[:0], ids), lambda: ext.embedding_backward(g, ids, 0),
                 lambda: ext.embedding_backward(g, ids, 4, scale=math.nan),
                 lambda: ext.embedding_backward(g, ids, 4, workspace=torch.empty(16, device="cuda"))):
        with pytest.raises(ext.ExterndError):
            call()


def test_rows_that_are_one(ext):
    """Expanded rows (a stride of 0) are refused, as table and as output, also where they overlap."""
    one, ids = torch.ones((1, 8), device="cuda"), torch.zeros((3,), dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        ext.embedding(one.expand(4, 8), ids, out=one.expand(3, 8))
    for call in (lambda: ext.embedding(one.expand(4, 8), ids), lambda: ext.embedding(one, ids, out=torch.ones((1, 8), device="cuda").expand(3, 8)),
                 lambda: ext.embedding_backward(one.expand(3, 8), ids, 4)):
        with pytest.raises(ext.ExterndError):
            call()
