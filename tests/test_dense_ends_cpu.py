"""Refusals of the operators at a model's dense ends before any device work,
their workspace sizes, and the oracle's gradients against differences (no GPU
needed)."""
import ctypes
import math

import numpy as np
import pytest

import oracle.ends_oracle as ref
from paper_2607_13511_amd import binding

D = ctypes.c_void_p(256)          # never dereferenced: validation fails first
BIG = 1 << 50
EINVAL, EWORKSPACE, EUNSUPPORTED = binding.EINVAL, binding.EWORKSPACE, binding.EUNSUPPORTED


def test_embedding_refuses_before_device_work():
    def f(table=D, dtype=1, vocab=10, width=8, stride=8, ids=D, tokens=3, scale=1.0, out=D, ostride=8):
        return binding.lib().externd_embedding(table, dtype, vocab, width, stride, ids, tokens, scale, out, ostride, None)
    assert f(tokens=0) == binding.OK and f(table=None, ids=None, out=None, tokens=0) == binding.OK
    for bad in (dict(table=None), dict(ids=None), dict(out=None), dict(dtype=3), dict(dtype=-1), dict(vocab=0), dict(width=0),
                dict(stride=7), dict(ostride=7), dict(tokens=-1), dict(scale=math.inf), dict(scale=math.nan)):
        assert f(**bad) == EINVAL, bad
    for bad in (dict(vocab=1 << 31), dict(tokens=1 << 31), dict(tokens=(1 << 31) - 1, width=1 << 20, stride=1 << 20, ostride=1 << 20)):
        assert f(**bad) == EUNSUPPORTED, bad


def test_embedding_backward_refuses_before_device_work():
    def f(grad=D, dtype=1, tokens=3, width=8, stride=8, ids=D, vocab=10, scale=1.0, acc=0, out=D, ostride=8, ws=D, n=BIG):
        return binding.lib().externd_embedding_backward(grad, dtype, tokens, width, stride, ids, vocab, scale, acc, out, ostride, ws, n, None)
    assert f(tokens=0, acc=1, grad=None, ids=None, ws=None, n=0) == binding.OK
    for bad in (dict(grad=None), dict(ids=None), dict(out=None), dict(dtype=3), dict(vocab=0), dict(width=0), dict(stride=7), dict(ostride=7),
                dict(tokens=-1), dict(scale=math.inf), dict(acc=2), dict(ws=ctypes.c_void_p(128))):
        assert f(**bad) == EINVAL, bad
    size = binding.lib().externd_embedding_backward_workspace_bytes
    assert f(ws=None) == EWORKSPACE and f(n=size(3, 10, 8) - 1) == EWORKSPACE
    for bad in (dict(vocab=(1 << 31) - 1), dict(tokens=(1 << 26) + 1), dict(width=(1 << 20) + 1, stride=1 << 21, ostride=1 << 21)):
        assert f(**bad) == EUNSUPPORTED, bad
    assert size(-1, 10, 8) == size(3, 0, 8) == size(3, 10, 0) == size((1 << 26) + 1, 10, 8) == 0
    assert size(1 << 26, (1 << 31) - 2, 64) > size(1 << 20, 1000, 64) > size(1000, 1000, 64) > 0


def _linear(x=D, xs=8, w=D, ws=8, dtype=1, rows=4, vocab=10, width=8, y=D, scale=1.0, lp=D, h=D, lse=D, work=D, n=BIG):
    return binding.lib().externd_linear_logprobs(x, xs, w, ws, dtype, rows, vocab, width, y, scale, lp, h, lse, work, n, None)


def _linear_backward(x=D, xs=8, w=D, ws=8, dtype=1, rows=4, vocab=10, width=8, y=D, scale=1.0, lse=D, h=D, g=D, ge=D, gx=D, gxs=8, gw=D,
                     gws=8, work=D, n=BIG):
    return binding.lib().externd_linear_logprobs_backward(x, xs, w, ws, dtype, rows, vocab, width, y, scale, lse, h, g, ge, gx, gxs, gw,
                                                          gws, work, n, None)


def test_linear_refuses_before_device_work():
    sizes = (dict(dtype=3), dict(rows=-1), dict(vocab=0), dict(width=0), dict(xs=7), dict(ws=7), dict(scale=0.0), dict(scale=-1.0),
             dict(scale=math.inf), dict(scale=math.nan), dict(x=None), dict(w=None), dict(work=ctypes.c_void_p(64)))
    for bad in sizes + (dict(y=None),):
        assert _linear(**bad) == EINVAL, bad
    for bad in sizes + (dict(lse=None), dict(y=None), dict(h=None), dict(gxs=7), dict(gws=7)):
        assert _linear_backward(**bad) == EINVAL, bad
    for f in (_linear, _linear_backward):
        for bad in (dict(rows=(1 << 22) + 1), dict(vocab=(1 << 25) + 1), dict(vocab=(1 << 31) - 1024), dict(rows=1 << 22, width=2049, xs=2049, ws=2049, **({} if f is _linear else dict(gxs=2049, gws=2049))),
                    dict(vocab=1 << 25, width=4097, xs=4097, ws=4097, **({} if f is _linear else dict(gxs=4097, gws=4097))), dict(width=(1 << 20) + 1, xs=1 << 21, ws=1 << 21, **({} if f is _linear else dict(gxs=1 << 21, gws=1 << 21))),
                    dict(xs=1 << 22), dict(ws=1 << 22)):
            assert f(**bad) == EUNSUPPORTED, bad
        assert f(work=None) == EWORKSPACE
    assert _linear(rows=0, x=None, w=None, work=None) == binding.OK
    assert _linear_backward(gx=None, gw=None) == binding.OK and _linear_backward(rows=0, gw=None) == binding.OK
    L = binding.lib()
    f, b = L.externd_linear_logprobs_workspace_bytes, L.externd_linear_logprobs_backward_workspace_bytes
    assert _linear(n=f(1, 4, 10, 8) - 1) == EWORKSPACE
    for gx, gw in ((D, D), (D, None), (None, D)):
        assert _linear_backward(gx=gx, gw=gw, n=b(1, 4, 10, 8, gx is not None, gw is not None) - 1) == EWORKSPACE
    for bad in ((3, 4, 10, 8), (1, -1, 10, 8), (1, 4, 0, 8), (1, 4, 10, 0), (1, (1 << 22) + 1, 10, 8), (1, 4, 1 << 31, 8)):
        assert f(*bad) == b(*bad, 1, 1) == 0


def test_the_logits_are_not_held():
    """Far less memory than the logits take."""
    L = binding.lib()
    for dtype, size in ((0, 4), (1, 2), (2, 2)):
        logits = 16384 * 150001 * size
        assert L.externd_linear_logprobs_workspace_bytes(dtype, 16384, 150001, 2560) < logits / 8
        assert L.externd_linear_logprobs_backward_workspace_bytes(dtype, 16384, 150001, 2560, 1, 1) < logits / 3


def test_clip_refuses_before_device_work():
    def f(ptrs=(256, 512), outs=None, sizes=(10, 10), types=(0, 1), max_norm=1.0, norm=D, ws=D, n=BIG, count=None):
        k = len(ptrs)
        a = (ctypes.c_void_p * k)(*ptrs)
        o = None if outs is None else (ctypes.c_void_p * k)(*outs)
        return binding.lib().externd_clip_gradients(k if count is None else count, a, o, (ctypes.c_int64 * k)(*sizes),
                                                    (ctypes.c_int32 * k)(*types), max_norm, norm, ws, n, None)
    for bad in (dict(ptrs=(None, 512)), dict(outs=(256, None)), dict(sizes=(10, -1)), dict(types=(0, 3)), dict(max_norm=-1.0),
                dict(max_norm=math.nan), dict(norm=None), dict(count=-1), dict(ptrs=(258, 512)), dict(ptrs=(256, 513)),
                dict(outs=(257, 512)), dict(ws=ctypes.c_void_p(8))):
        assert f(**bad) == EINVAL, bad
    assert f(ws=None) == EWORKSPACE and f(n=binding.lib().externd_clip_gradients_workspace_bytes(2) - 1) == EWORKSPACE
    assert f(count=(1 << 20) + 1) == EUNSUPPORTED and f(sizes=(10, 1 << 45)) == EUNSUPPORTED
    assert binding.lib().externd_clip_gradients_workspace_bytes(-1) == 0


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    x, w, y = rng.standard_normal((5, 6)), rng.standard_normal((9, 6)), np.array([3, -1, 8, 0, 9])
    g, ge = rng.standard_normal(5), rng.standard_normal(5)
    ge[1] = 0

    def loss(x, w):
        z, _ = ref.linear(x, w, 0.8)
        lse, h, _ = ref.softmax_moments(z)
        lp = np.array([z[r, t] - lse[r] if 0 <= t < 9 else 0.0 for r, t in enumerate(y)])
        return (g * lp).sum() + (ge * h).sum()
    G = 0.8 * ref.logits_gradient(ref.linear(x, w, 0.8)[0], y, g, ge)
    for a, grad in ((x, G @ w), (w, G.T @ x)):
        for i in np.ndindex(a.shape):
            kept, step = a[i], 1e-5
            a[i] = kept + step
            up = loss(x, w)
            a[i] = kept - step
            down = loss(x, w)
            a[i] = kept
            assert abs((up - down) / (2 * step) - grad[i]) < 1e-8
    assert (G[1] == 0).all()


def test_oracle_embedding_gradient_is_the_transpose():
    rng = np.random.default_rng(1)
    ids = np.array([0, 3, -1, 3, 7, 2, 3])
    table, grad = rng.standard_normal((7, 4)), rng.standard_normal((7, 4))
    back, size, count = ref.embedding_backward(grad, ids, 7, 1.7)
    assert abs((ref.embedding(table, ids, 1.7) * grad).sum() - (back * table).sum()) < 1e-12
    assert count.tolist() == [1, 0, 1, 3, 0, 0, 0] and np.all(size >= np.abs(back))


def test_oracle_clip():
    norm, got = ref.clip([[3.0, 0.0], [4.0]], 1.0)
    assert norm == 5 and np.allclose(got[0], [0.6, 0]) and np.allclose(got[1], [0.8])
    assert ref.clip([[3.0, 4.0]], 9.0)[1][0].tolist() == [3.0, 4.0] and ref.clip([[0.0]], 0.0)[1][0].tolist() == [0.0]


@pytest.mark.parametrize("many", [0, 100])
def test_what_is_written_twice(many):
    """Few spans and many, which are looked at differently; the others lie far behind."""
    def f(*spans):
        """(input, output, bytes) of each tensor."""
        spans = list(spans) + [(10000 + 10 * i,) * 2 + (10,) for i in range(many)]
        ins, ops, n = (list(c) for c in zip(*spans))
        return binding._written_twice(ins, ins if ins == ops else ops, n)
    assert not f((0, 0, 10), (10, 10, 10)) and not f((20, 20, 4), (0, 0, 20)) and not f((0, 0, 10), (0, 0, 0))
    assert f((0, 0, 10), (9, 9, 10)) and f((0, 0, 10), (0, 0, 10)) and f((0, 0, 100), (50, 50, 1))
    assert not f((0, 100, 10), (0, 200, 10))            # an input given twice, two outputs
    assert f((0, 100, 10), (0, 105, 10)) and f((0, 100, 10), (100, 200, 10)) and f((0, 5, 10))
    assert f((0, 500, 300), (900, 290, 10)) and not f((0, 500, 300), (900, 300, 10)) and f((0, 500, 300), (600, 300, 10))


@pytest.mark.parametrize("name", ["embedding", "embedding_backward", "linear_logprobs", "linear_logprobs_backward", "clip_gradients"])
def test_needs_a_gpu(name):
    """There is no fallback on the CPU."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is there")
    args = {"embedding": 2, "embedding_backward": 3, "linear_logprobs": 2, "linear_logprobs_backward": 5, "clip_gradients": 1}[name]
    with pytest.raises(RuntimeError):
        getattr(binding, name)(*[torch.ones(2, 2)] * args)


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("vocab", [(1 << 25) - 256, (1 << 25) - 255, 1 << 25])
@pytest.mark.parametrize("rows", [4097, 8064, 8065, 8192, 100000])
def test_a_pass_of_rows_is_one_launch(dtype, vocab, rows):
    """Tiles of 128 rows and 256 columns, 512 threads each, are fewer than 2^32 threads: from the workspace, which holds
    16 bytes for each of a pass's rows and tiles of columns and 4 for each row."""
    size = binding.lib().externd_linear_logprobs_workspace_bytes(dtype, rows, vocab, 64)
    tiles = -(-vocab // 256)
    of_a_pass = size // (16 * tiles)
    assert 2048 <= of_a_pass <= rows and -(-of_a_pass // 128) * tiles * 512 < 1 << 32


def test_views_of_one_buffer_overlap_where_bytes_are_shared():
    """Against the sets of their entries: columns side by side, rows apart, one row or many."""
    import torch
    buf = torch.zeros(6, 10)
    where = torch.arange(60).view(6, 10)
    cuts = [(r0, r1, c0, c1) for r0 in range(6) for r1 in range(r0, 7) if r1 - r0 in (0, 1, 2, 6) for c0, c1 in ((0, 4), (4, 10), (0, 10), (3, 5), (9, 10))]
    for a in cuts:
        for b in cuts:
            x, y = (buf[r0:r1, c0:c1] for r0, r1, c0, c1 in (a, b))
            shared = set(where[a[0]:a[1], a[2]:a[3]].flatten().tolist()) & set(where[b[0]:b[1], b[2]:b[3]].flatten().tolist())
            assert binding._overlaps(x, y) == bool(shared), (a, b)


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2), (2, 2)])
@pytest.mark.parametrize("vocab", [300, 2303, 2304, 40000])
@pytest.mark.parametrize("rows", [1, 3000, 40000, 1 << 20, 1 << 22])
def test_what_a_piece_of_G_takes(dtype, size, vocab, rows):
    """A piece is up to 2^26 entries or eight tiles of 256 columns, whichever is more, the last one up to 255 columns more, in
    rows an odd number of 256 entries apart: 512 more.  Beside it 40 bytes a row, grad_x's sums of up to 256 splits' tiles of
    rows x 8 columns, and 8 KB."""
    took = binding.lib().externd_linear_logprobs_backward_workspace_bytes(dtype, rows, vocab, 8, 1, 0)
    columns = min(max((1 << 26) // rows, 2048), -(-vocab // 256) * 256) + 512
    splits = max(1, 256 // -(-rows // 256))
    assert rows * vocab * size * (vocab <= 2303) <= took <= rows * columns * size + rows * 40 + splits * rows * 32 + 8192 + 4 * rows
