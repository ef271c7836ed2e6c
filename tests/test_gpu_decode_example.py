"""The decoding operators together, as examples/decode.py runs them: every stage of
a prompt's and of two single-token steps against its definition in 64 bits on the
stage's own inputs, so that the bounds are those of each stage (u = 2^-24):
* projections: as in the tests of apply: (n + k + 4) u |B| |D| |C| |x|;
* rotary: the turn of a pair has errors of a few u of |a| + |b| (4 u for two
  products and a sum, 2 u for sin and cos, and their 2^-32 turns, 1.5e-9);
* attention: a score is off by dx <= (D + 8) u scale sum |q k|; weights then by
  a factor e^(2 dx) at most, and n + 16 roundings in sums: (4 dx + (n + 16) u) max |v|
  (lse: 2 dx, the sum's roundings, 8 u of the largest score);
* log probabilities: sums of V entries, (V + 16) u, and 8 u of the largest |z|.
"""
import importlib.util
import os

import numpy as np
import pytest

from oracle import decode_oracle as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode.py")
    spec = importlib.util.spec_from_file_location("decode_example", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def f64(t):
    return t.double().cpu().numpy()


def check_projection(binding, fac, X, Y):
    k = fac.f.D.shape[0]
    B = binding.unpack_trits(fac.f.B_packed.cpu().numpy(), k).astype(np.float64)
    C = binding.unpack_trits(fac.f.C_packed.cpu().numpy(), fac.n).astype(np.float64)
    D, X = f64(fac.f.D), f64(X)
    want = (X @ C.T * D) @ B.T
    tol = (fac.n + k + 4) * U * ((np.abs(X) @ np.abs(C).T * np.abs(D)) @ np.abs(B).T)
    assert np.all(np.abs(f64(Y).reshape(want.shape) - want) <= tol)


def test_stages(example):
    binding = example.binding
    model, gen = example.Model(), torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, model.vocab, (n,), generator=gen).tolist() for n in (70, 23, 1)]
    session = example.Session(model, len(prompts))
    freqs = model.freqs.cpu().numpy().view(np.uint64)
    tokens, targets = prompts, [p[1:] + [-1] for p in prompts]
    for _ in range(3):
        out, s = session.step(tokens, targets)
        torch.cuda.synchronize()
        T = s["starts"][-1]
        for fac, name in ((model.q, "q0"), (model.k, "k0"), (model.v, "v")):
            check_projection(binding, fac, s["x"], s[name].reshape(T, -1))
        check_projection(binding, model.o, s["att"].reshape(T, -1), s["o"])
        check_projection(binding, model.head, s["y"], s["logits"])
        for a, b in (("q0", "q"), ("k0", "k")):
            want = ref.rotary(f64(s[a]), s["positions"], freqs, False, model.amplitude)
            big = np.abs(f64(s[a])).max(axis=-1, keepdims=True)
            assert np.all(np.abs(f64(s[b]) - want) <= 2 * big * model.amplitude * (6 * U + 2e-9))
        # what the cache holds: within half a step of what was stored, for the new tokens
        st = torch.tensor(s["starts"], dtype=torch.int32, device="cuda")
        kh, vh = binding.kv4_read(session.cache, s["table"], s["lens"], model.dim, starts=st, tokens=T)
        for got, x in ((f64(kh), f64(s["k"])), (f64(vh), f64(s["v"]))):
            span = np.maximum(x.max(-1, keepdims=True), 0) - np.minimum(x.min(-1, keepdims=True), 0)
            # the step is span / 15 rounded up to seven significant bits
            assert np.all(np.abs(got - x) <= span / 15 * (1 + 2.0 ** -6) * (0.5 + 2.0 ** -20))
        # attention over all that is held
        lens = session.lens
        whole = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
        K, V = binding.kv4_read(session.cache, s["table"], s["lens"], model.dim, starts=whole, tokens=sum(lens))
        K, V, q = f64(K), f64(V), f64(s["q"])
        scale, each, at = model.dim ** -0.5, model.heads // model.heads_kv, np.concatenate([[0], np.cumsum(lens)])
        for u in range(len(lens)):
            for t in range(s["starts"][u], s["starts"][u + 1]):
                n = s["positions"][t] + 1
                for h in range(model.heads):
                    k, v = K[at[u]:at[u] + n, h // each], V[at[u]:at[u] + n, h // each]
                    x = scale * (k @ q[t, h])
                    dx = (model.dim + 8) * U * scale * (np.abs(k) @ np.abs(q[t, h])).max()
                    p = np.exp(x - x.max())
                    want = p @ v / p.sum()
                    assert np.all(np.abs(f64(s["att"][t, h]) - want) <= (4 * dx + (n + 16) * U) * np.abs(v).max())
                    assert abs(float(s["lse"][t, h]) - (x.max() + np.log(p.sum()))) <= 2 * dx + (n + 16) * U + 8 * U * np.abs(x).max()
        y = np.array([t for ts in targets for t in ts]) if targets is not None else np.full(T, -1)
        lp, ent, lse, tl, ti, _ = ref.logprobs(f64(s["logits"]), y, 1.0, 5)
        z = np.abs(f64(s["logits"])).max()
        tol = (model.vocab + 16) * U + 8 * U * z
        if targets is not None:
            assert np.all(np.abs(f64(out.logprob) - lp) <= tol)
        assert np.all(np.abs(f64(out.top_logprobs) - tl) <= tol) and np.array_equal(out.top_ids.cpu().numpy(), ti)
        ends = [e - 1 for e in s["starts"][1:]]
        tokens, targets = [[t] for t in out.top_ids[ends, 0].tolist()], None


def test_pages_run_out(example):
    session = example.Session(example.Model(vocab=100), 1, pages=2)
    with pytest.raises(RuntimeError, match="no page left"):
        session.step([[1] * 33])


def test_main(example, capsys):
    example.main()
    assert "perplexity" in capsys.readouterr().out


def test_a_given_stream_has_its_own_memory(example):
    """With ``stream`` given, results and workspace come from that stream's memory: what the current
    stream has freed, with work on it pending, is not written.  The same bits as on the current one."""
    b, g = example.binding, torch.Generator().manual_seed(3)
    q, k = torch.randn((40, 8, 64), generator=g).cuda(), torch.randn((40, 2, 64), generator=g).cuda()
    x = torch.randn((40, 5000), generator=g).cuda()
    pos, freqs = torch.arange(40, device="cuda"), torch.from_numpy(b.rotary_frequencies(64)[0]).cuda()
    cache, table = b.kv4_cache(300, 2, 64, 16), torch.arange(300, dtype=torch.int32, device="cuda")[None].contiguous()
    lens, starts = torch.tensor([40], dtype=torch.int32, device="cuda"), torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    b.kv4_append(cache, k, k, table, lens, starts)
    y = torch.arange(40, device="cuda")
    lse, h = (lambda r: (r.lse, r.entropy))(b.token_logprobs(x, y))

    def calls(**kw):
        r = list(b.rotary(q, k, pos, freqs, **kw)) + list(b.rotary_backward(q, k, pos, freqs, **kw))
        r += list(b.kv4_read(cache, table, lens, 64, starts=starts, tokens=40, **kw))
        r += list(b.kv4_attention(cache, q, table, lens, starts=starts, **kw))
        t = b.token_logprobs(x, y, top=7, **kw)
        return r + [t.logprob, t.entropy, t.lse, t.top_logprobs, t.top_ids, b.token_logprobs_backward(x, y, lse, h, h, h, **kw)]
    want = calls()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls(stream=s)
    torch.cuda.synchronize()
    # memory that the current stream has freed must not come back for the other stream
    free = {torch.empty_like(t).data_ptr() for t in want for _ in range(4)}
    got = calls(stream=s)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert not free & {t.data_ptr() for t in got}
