"""GPU parity of the norm over many tensors and of clipping by it
(externd_clip_gradients) with the oracle's fp64 form.

Tolerance (u = 2^-24): squares and sums are fp64 (n 2^-53 of sums of positive
terms, below u), so the norm is rounded once to fp32: 2 u.  A clipped entry is
rounded with the factor (u), in the product (u) and to its type."""
import math

import numpy as np
import pytest

import oracle.ends_oracle as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"fp32": (torch.float32, 0.0), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
EPS = {t: e for t, e in TYPES.values()}


@pytest.fixture(scope="module")
def ext():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13511_amd import binding
    binding.lib()
    return binding


def make(sizes, types=tuple(TYPES), seed=0, scale=1.0):
    rng = np.random.default_rng(seed)
    return [torch.from_numpy(scale * 10.0 ** rng.uniform(-3, 0) * rng.standard_normal(n)).to(TYPES[types[i % len(types)]][0]).cuda()
            for i, n in enumerate(sizes)]


def check(ext, tensors, max_norm, out=None):
    norm, want = ref.clip([t.double().cpu().numpy() for t in tensors], max_norm)
    got = ext.clip_gradients(tensors, max_norm, out=out)
    assert got.shape == () and got.dtype is torch.float32 and abs(got.item() - norm) <= 2 * U * norm
    for t, w in zip(tensors if out is None else out, want):
        err = np.abs(t.double().cpu().numpy() - w)
        assert np.all(err <= (2 * U + EPS[t.dtype]) * np.abs(w) * (1 + 4 * U) + TINY[t.dtype])


@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [3, 8191, 8192, 8193, 17], [1, 2, 3] * 40, [7] * 121, [100] * 500 + [70000], [20000000, 33, 5]])
@pytest.mark.parametrize("max_norm", [0.05, 1e6])
def test_matches_oracle(ext, sizes, max_norm):
    tensors = make(sizes)
    check(ext, [t.clone() for t in tensors], max_norm)                              # in place
    check(ext, tensors, max_norm, out=[torch.full_like(t, 9.0) for t in tensors])   # apart


@pytest.mark.parametrize("dtype", TYPES)
def test_every_alignment(ext, dtype):
    """Views that begin at any entry, in place and towards ones that begin elsewhere; what is around them stays."""
    for n in (1, 5, 40, 8200):
        for a in range(0, 9, 1 if n < 100 else 4):
            src = make([n + 32], (dtype,), a)[0]
            for b in (a, a + 1, a + 4):
                dst = torch.full_like(src, 5.0)
                check(ext, [src[a:a + n]], 1e-3, out=[dst[b:b + n]])
                assert (dst[:b] == 5).all() and (dst[b + n:] == 5).all()
            kept = src.clone()
            check(ext, [src[a:a + n]], 1e-3)
            assert torch.equal(src[:a], kept[:a]) and torch.equal(src[a + n:], kept[a + n:])


def test_unclipped_stays_as_it_is(ext):
    tensors = make([1000, 77])
    kept = [t.clone() for t in tensors]
    big = 1.5 * ext.clip_gradients(tensors).item()
    for m in (math.inf, big):
        ext.clip_gradients(tensors, m)
        assert all(torch.equal(a, b) for a, b in zip(tensors, kept))
    out = [torch.zeros_like(t) for t in tensors]
    ext.clip_gradients(tensors, big, out=out)
    assert all(torch.equal(a, b) for a, b in zip(out, kept))
    out = [torch.full_like(t, 4.0) for t in tensors]
    ext.clip_gradients(tensors, math.inf, out=out)                                  # only the norm
    assert all((o == 4).all() for o in out)


def test_zero_and_nonfinite_norms(ext):
    zeros = [torch.zeros(100, device="cuda"), torch.zeros(3, device="cuda", dtype=torch.float16)]
    for m in (0.0, 1.0, math.inf):
        assert ext.clip_gradients(zeros, m).item() == 0 and all((z == 0).all() for z in zeros)
    assert ext.clip_gradients([]).item() == 0 and ext.clip_gradients([torch.empty(0, device="cuda")], 1.0).item() == 0
    t = torch.ones(1000, device="cuda")
    assert ext.clip_gradients([t], 0.0).item() == pytest.approx(math.sqrt(1000), rel=2 * U) and (t == 0).all()
    t = torch.ones(1000, device="cuda")
    t[5] = -math.inf
    assert ext.clip_gradients([t]).item() == math.inf
    assert ext.clip_gradients([t], 1.0).item() == math.inf and torch.isnan(t[5]) and t.isnan().sum() == 1 and (t.nan_to_num() == 0).all()
    t = torch.ones(1000, device="cuda")
    t[999] = math.nan
    u = torch.ones(8, device="cuda", dtype=torch.bfloat16)
    assert math.isnan(ext.clip_gradients([t, u], 1.0).item()) and t.isnan().all() and u.isnan().all()


def test_squares_past_fp32(ext):
    """Entries whose squares are infinite, or 0, in fp32."""
    check(ext, [torch.full((100,), 1e25, device="cuda")], 1.0)
    check(ext, [torch.full((100,), 1e-30, device="cuda")], 1e-32)
    t = [torch.full((10000,), 3e38, device="cuda")]                                 # the norm itself is past fp32
    assert ext.clip_gradients(t, 1.0).item() == math.inf and (t[0] - 0.01).abs().max() <= 1e-8


def test_orders_of_dimensions(ext):
    a = torch.randn((30, 40), device="cuda").t()
    b = torch.randn((2, 8, 5, 3), device="cuda").to(memory_format=torch.channels_last)
    out = [torch.empty_like(a), torch.empty_like(b)]
    check(ext, [a, b], 0.5, out=out)
    check(ext, [a, b], 0.5)


def test_streams_graphs_and_repeats(ext):
    tensors = make([5000, 33, 100000] + [300] * 130)
    first, second = ([torch.empty_like(t) for t in tensors] for _ in range(2))
    want = ext.clip_gradients(tensors, 0.1, out=first)
    assert torch.equal(ext.clip_gradients(tensors, 0.1, out=second), want) and all(torch.equal(a, b) for a, b in zip(first, second))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ext.clip_gradients(tensors, 0.1, out=second, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(first, second))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ext.clip_gradients(tensors, 0.1, out=second)
    for _ in range(3):
        for t in tensors:
            t.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        want = ext.clip_gradients(tensors, 0.1, out=first)
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(first, second))


def test_refusals(ext):
    t, u = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    for call in (lambda: ext.clip_gradients([t.double()]), lambda: ext.clip_gradients([t.cpu()]), lambda: ext.clip_gradients([t[::2]]),
                 lambda: ext.clip_gradients([t, t], 1.0), lambda: ext.clip_gradients([t, t[5:]], 1.0),
                 lambda: ext.clip_gradients([t], 1.0, out=[u[:5]]), lambda: ext.clip_gradients([t], 1.0, out=[u.half()]),
                 lambda: ext.clip_gradients([t], 1.0, out=[]), lambda: ext.clip_gradients([t[:6]], 1.0, out=[t[2:8]]),
                 lambda: ext.clip_gradients([t, u], 1.0, out=[u, t]), lambda: ext.clip_gradients([t], workspace=torch.empty(1 << 20))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ext.clip_gradients([t], -1.0), lambda: ext.clip_gradients([t], math.nan),
                 lambda: ext.clip_gradients([t], workspace=torch.empty(16, device="cuda"))):
        with pytest.raises(ext.ExterndError):
            call()
    assert ext.clip_gradients([t, t]).item() == pytest.approx(math.sqrt(20), rel=2 * U)      # only read: twice is twice


def test_a_workspace_of_another_device(ext):
    class Elsewhere:
        device, is_cuda = torch.device("cuda", 1), True
        data_ptr, numel, element_size = (lambda s: 256), (lambda s: 1 << 20), (lambda s: 1)

        def is_contiguous(self):
            return True

    with pytest.raises(ValueError):
        ext.clip_gradients([torch.ones(10, device="cuda:0")], workspace=Elsewhere())
