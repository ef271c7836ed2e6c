"""The operators at a model's dense ends as a training step uses them together:
a model of one ternary factorization between an embedding and a head that are
the same matrix, in the order

    embedding -> apply -> linear_logprobs -> linear_logprobs_backward -> embedding_backward (onto the head's
    gradient) -> clip_gradients

against the same step in 64 bits, and against differences of its loss.

Tolerance (u = 2^-24): the logits' terms add up to S < 30 over width 64, apply
is within 600 u of its own terms, a row's probabilities move by at most
q = (2 * 72 + 700) u S + (n / 64 + 60) u < 2^-9, each gradient entry by q and
(n + 200) u of the sum of its terms' absolute values, and clipping by 4 u: in all
below 2^-8 of that sum for fp32 (2^-6 with bf16's and fp16's roundings of the
head, of the gradient's factor and of hidden states, each below 2^-8)."""
import math

import numpy as np
import pytest

import oracle.ends_oracle as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, 2.0 ** -8), "bf16": (torch.bfloat16, 2.0 ** -6), "fp16": (torch.float16, 2.0 ** -6)}
VOCAB, WIDTH, SCALE = 300, 64, 8.0


@pytest.fixture(scope="module")
def ext():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13511_amd import binding
    binding.lib()
    return binding


def dense(ext, f):
    B = ext.unpack_trits(f.B_packed.cpu().numpy(), f.k).astype(np.float64)
    C = ext.unpack_trits(f.C_packed.cpu().numpy(), WIDTH).astype(np.float64)
    return B @ (f.D.double().cpu().numpy()[:, None] * C)


def step(ext, E, f, M, ids, targets, max_norm, stream=None):
    """One step's loss and clipped gradient of E; M is the factorization's dense form, for its gradient."""
    t = E.dtype
    x = ext.embedding(E, ids, scale=SCALE)
    y = torch.cat([ext.apply(f.B_packed, f.C_packed, f.D, WIDTH, WIDTH, r.contiguous()) for r in x.float().split(8)])
    h = (x.float() + y).to(t)
    asked = int((targets >= 0).sum())
    got = ext.linear_logprobs(h, E, targets)
    g = torch.full((len(ids),), -1.0 / asked, device="cuda")
    gh, gE = ext.linear_logprobs_backward(h, E, targets, got.lse, got.entropy, g)
    gx = (gh.float() + gh.float() @ M).to(t)
    ext.embedding_backward(gx, ids, VOCAB, scale=SCALE, out=gE, accumulate=True)
    before = gE.clone()
    norm = ext.clip_gradients([gE], max_norm)
    return -got.logprob.sum().item() / asked, before, gE, norm


def exact(E, M, ids, targets):
    """(loss, gradient, sum of the absolute values of its terms) in 64 bits."""
    x = ref.embedding(E, ids, SCALE)
    h = x + x @ M.T
    z, _ = ref.linear(h, E, 1.0)
    lse, _, p = ref.softmax_moments(z)
    asked = int((targets >= 0).sum())
    loss = -sum(z[r, t] - lse[r] for r, t in enumerate(targets) if t >= 0) / asked
    G = ref.logits_gradient(z, targets, np.full(len(ids), -1.0 / asked), None)
    gh = G @ E
    gx = gh + gh @ M
    back, _, _ = ref.embedding_backward(gx, ids, len(E), SCALE)
    size, _, _ = ref.embedding_backward(np.abs(G) @ np.abs(E) @ (np.eye(WIDTH) + np.abs(M)), ids, len(E), SCALE)
    return loss, G.T @ h + back, np.abs(G).T @ np.abs(h) + size


def make(ext, dtype, seed=0):
    rng = np.random.default_rng(seed)
    f = ext.factorize(torch.from_numpy(rng.standard_normal((WIDTH, WIDTH)) * 0.1).float().cuda(), mu=1.5, tau=1.0, block=8, iters=4)
    E = torch.from_numpy(rng.standard_normal((VOCAB, WIDTH)) / 8).to(TYPES[dtype][0]).cuda()
    ids = rng.integers(0, VOCAB, 90)
    ids[:20] = 7                                       # a frequent token
    targets = np.roll(ids, -1)
    ids[80:], targets[79:] = -1, -1                    # padding
    M = dense(ext, f)
    return f, E, M, ids, targets, torch.from_numpy(M).float().cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(targets).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("max_norm", [0.25, 1e9])
def test_a_training_step_of_tied_ends(ext, dtype, max_norm):
    f, E, M, ids, targets, dM, di, dt = make(ext, dtype)
    loss, before, clipped, norm = step(ext, E, f, dM, di, dt, max_norm)
    want_loss, want, size = exact(E.double().cpu().numpy(), M, ids, targets)
    tol = TYPES[dtype][1]
    assert abs(loss - want_loss) <= tol * (1 + abs(want_loss))
    err = np.abs(before.double().cpu().numpy() - want)
    assert np.all(err <= tol * size + 1e-7), np.max(err / (size + 1e-9))
    n = float(np.sqrt((before.double().cpu().numpy() ** 2).sum()))
    assert abs(norm.item() - n) <= 1e-6 * n
    again = before.double().cpu().numpy() * min(1.0, max_norm / n)
    assert np.all(np.abs(clipped.double().cpu().numpy() - again) <= tol * np.abs(again) + 1e-7)
    assert all(torch.equal(a, b) for a, b in zip((before, clipped), step(ext, E, f, dM, di, dt, max_norm)[1:3]))


def test_the_gradient_of_tied_ends_against_differences(ext):
    """The oracle's loss along the step's gradient (central differences; third derivatives of a mean over 79 tokens
    along 1e-3 of a gradient of length about 1 are below 1e-5 of its square)."""
    f, E, M, ids, targets, dM, di, dt = make(ext, "fp32", 3)
    _, g, _, _ = step(ext, E, f, dM, di, dt, math.inf)
    E64, g64 = E.double().cpu().numpy(), g.double().cpu().numpy()
    up, down = (exact(E64 + s * g64, M, ids, targets)[0] for s in (1e-3, -1e-3))
    assert abs((up - down) / 2e-3 - (g64 ** 2).sum()) <= 1e-3 * (g64 ** 2).sum()


def test_replayed_steps(ext):
    """The whole step but for its host arithmetic in one graph, replayed on other tokens and weights."""
    f, E, M, ids, targets, dM, di, dt = make(ext, "bf16", 4)
    g = torch.full((len(ids),), -1.0 / 79, device="cuda")

    def run():
        h = ext.embedding(E, di, scale=SCALE)
        got = ext.linear_logprobs(h, E, dt)
        gh, gE = ext.linear_logprobs_backward(h, E, dt, got.lse, got.entropy, g)
        ext.embedding_backward(gh, di, VOCAB, scale=SCALE, out=gE, accumulate=True)
        return got.logprob, gE, ext.clip_gradients([gE, gh], 0.1)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(3):
        di.copy_(torch.roll(di, 3))
        dt.copy_(torch.roll(dt, 3))
        E.mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, run()))
