"""Cases of the operators at a model's dense ends, which its factorization
leaves as they are: the embedding, the head with the log probabilities behind
it, and the norm of all gradients.

``embedding`` looks tokens up in a table and scales them;
``embedding_backward`` sums the gradients of each token's places.
``linear_logprobs`` gives the log probability of each row's target, the
entropy and the logarithm of the softmax's sum for the logits
``scale x W^T``, which are never held; ``linear_logprobs_backward`` gives the
gradients for x and for W.  ``clip_gradients`` is the norm over many tensors
and scales them down where it is above a bound.

``run`` computes an operator in plain torch operations, or, where ``own`` is
true, through ``paper_2607_13511_amd.binding``.  Widths are those of the
projections of the test configurations (2560, 1024, 4096, 9728) and odd ones.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _head(name, rows, width, vocab, dtype):
    return {"name": name, "op": "head", "rows": rows, "width": width, "vocab": vocab, "dtype": dtype}


def _head_backward(name, rows, width, vocab, dtype, frozen, entropy):
    """frozen: W is not trained, only x's gradient is asked for; entropy: its gradient is part of the loss."""
    return {"name": name, "op": "head_backward", "rows": rows, "width": width, "vocab": vocab, "dtype": dtype,
            "frozen": frozen, "entropy": entropy}


def _embed(name, tokens, width, vocab, dtype, backward, skew):
    """skew: ids are vocab u^skew for even u, so that larger ones repeat the low ids more."""
    return {"name": name, "op": "embed", "tokens": tokens, "width": width, "vocab": vocab, "dtype": dtype,
            "backward": backward, "skew": skew}


def _clip(name, layers, width, narrow, wide, vocab, dense, dtype, max_norm):
    """Gradients of a model of `layers` layers: two fp32 norm vectors and, for each of the seven projections, an
    fp32 vector of scales, or (dense) the matrix; and, where vocab > 0, an embedding and a head."""
    return {"name": name, "op": "clip", "layers": layers, "width": width, "narrow": narrow, "wide": wide, "vocab": vocab,
            "dense": dense, "dtype": dtype, "max_norm": max_norm}


def listed():
    return [
        # the next token of a single user, scored against a dense head
        _head("head_1_row", 1, 2560, 65536, "bf16"),
        # eight users' tokens in fp32, as apply returns hidden states; odd vocabulary
        _head("head_8_rows", 8, 2560, 65537, "fp32"),
        # perplexity of a text of 2048 tokens over a large vocabulary
        _head("head_2048_rows", 2048, 2560, 150001, "bf16"),
        # a training step of the head: gradients of hidden states and head, entropy in the loss
        _head_backward("head_backward_2048", 2048, 2560, 65537, "bf16", False, True),
        # hidden states' gradient through a head that is not trained
        _head_backward("head_backward_frozen", 4095, 1024, 32001, "fp16", True, False),
        # a small fp32 step, every size odd
        _head_backward("head_backward_fp32", 517, 1001, 8191, "fp32", False, True),
        # the newest tokens of 32 users
        _embed("embed_32_tokens", 32, 2560, 65536, "fp32", False, 1),
        # a batch of texts
        _embed("embed_8191_tokens", 8191, 2560, 150001, "bf16", False, 4),
        # their gradient: the whole table's, most rows of it zero
        _embed("embed_backward_8191", 8191, 2560, 65537, "bf16", True, 4),
        # a small vocabulary, whose few frequent tokens take most of a large batch; odd width
        _embed("embed_backward_repeats", 32001, 1001, 1000, "fp16", True, 16),
        # the scales and norms of a factored model: hundreds of short vectors
        _clip("clip_scales", 24, 2560, 1024, 9728, 0, False, "fp32", 1.0),
        # dense gradients of four layers, an embedding and a head
        _clip("clip_dense", 4, 2560, 1024, 9728, 65537, True, "bf16", 1.0),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Half of the widths as models have them (multiples of 64), half of any remainder."""
    n = _spread(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(("head", "head", "head_backward", "head_backward", "embed", "embed_backward", "clip"))
    dtype = rng.choice(tuple(TYPES))
    if op == "clip":
        dense = rng.random() < 0.5
        layers = _spread(rng, 1, 24)
        width = _width(rng, 64, 2560)
        narrow, wide = max(1, width * rng.choice((2, 4, 8)) // 8), width * rng.choice((2, 3, 4)) - rng.choice((0, 0, 1))
        vocab = rng.choice((0, _spread(rng, 1000, max(1001, min(65537, int(8e7 / width))))))
        if dense:
            layers = max(1, min(layers, int((1.6e8 if dtype == "fp32" else 4e8) / (width * (2 * width + 2 * narrow + 3 * wide)))))
        c = _clip("", layers, width, narrow, wide, vocab, dense, dtype if dense else "fp32", rng.choice((0.1, 1.0, 1.0, 1e9)))
    elif op.startswith("embed"):
        tokens, vocab = _spread(rng, 1, 32001), _spread(rng, 1000, 150001)
        width = _width(rng, 64, max(64, min(4096, int(1.6e8 / max(tokens, vocab)))))
        c = _embed("", tokens, width, vocab, dtype, op == "embed_backward", rng.choice((1, 4, 16)))
    else:
        vocab, width = _spread(rng, 1000, 150001), _width(rng, 64, 4096)
        most = int((7e11 if op == "head" else 2e11) / (vocab * width) / (6 if dtype == "fp32" else 1))
        rows = _spread(rng, 1, max(1, min(4096, most)))
        c = (_head("", rows, width, vocab, dtype) if op == "head" else
             _head_backward("", rows, width, vocab, dtype, rng.random() < 0.4, rng.random() < 0.4))
    del c["name"]
    return c


def _shapes(case):
    """(shape, type) of each gradient of a clip case."""
    w, n, f = case["width"], case["narrow"], case["wide"]
    matrices = [(w, w), (n, w), (n, w), (w, w), (f, w), (f, w), (w, f)]
    got = []
    for _ in range(case["layers"]):
        got += [((w,), "fp32"), ((w,), "fp32")]
        got += [(m, case["dtype"]) if case["dense"] else ((2 * min(m),), "fp32") for m in matrices]
    return got + [((case["vocab"], w), case["dtype"])] * (2 if case["vocab"] else 0)


def work(case):
    op, es = case["op"], BYTES[case["dtype"]]
    if op == "clip":
        sizes = [(math.prod(s), BYTES[t]) for s, t in _shapes(case)]
        return {"bytes": sum(2 * n * b for n, b in sizes), "flops": sum(3 * n for n, _ in sizes)}
    if op == "embed":
        some = case["tokens"] * case["width"] * es
        rest = case["vocab"] * case["width"] * es if case["backward"] else min(case["tokens"], case["vocab"]) * case["width"] * es
        return {"bytes": some + rest + 8 * case["tokens"], "flops": case["tokens"] * case["width"]}
    rows, width, vocab = case["rows"], case["width"], case["vocab"]
    product = 2 * rows * width * vocab
    if op == "head":
        return {"bytes": (rows + vocab) * width * es + 20 * rows, "flops": product + 6 * rows * vocab}
    return {"bytes": (2 * rows + (1 if case["frozen"] else 2) * vocab) * width * es + 24 * rows,
            "flops": (2 if case["frozen"] else 3) * product + 8 * rows * vocab}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    gen, op, t = _gen(seed), case["op"], TYPES[case["dtype"]]
    s = {"op": op}

    def normal(*shape, scale=1.0, dtype=t):
        return torch.randn(shape, generator=gen, device=DEV).mul_(scale).to(dtype)

    if op == "clip":
        # views of one buffer for each type, as a program keeps them; from tensor to tensor a gradient's size differs by a thousand
        shapes = _shapes(case)
        sizes = (10.0 ** (3.0 * torch.rand((len(shapes),), generator=gen, device=DEV) - 4.0)).tolist()
        s["grads"], s["clipped"], s["whole"], s["whole_clipped"] = [], [], {}, {}
        for dt in sorted({dt for _, dt in shapes}):
            parts = [normal(math.prod(shape), scale=z, dtype=TYPES[dt]) for (shape, d), z in zip(shapes, sizes) if d == dt]
            s["whole"][dt] = torch.cat(parts)
            s["whole_clipped"][dt] = torch.empty_like(s["whole"][dt])
            each = [math.prod(shape) for shape, d in shapes if d == dt]
            s["grads"] += s["whole"][dt].split(each)
            s["clipped"] += s["whole_clipped"][dt].split(each)
        s["max_norm"] = case["max_norm"]
        return s
    vocab, width = case["vocab"], case["width"]
    if op == "embed":
        u = torch.rand((case["tokens"],), generator=gen, device=DEV, dtype=torch.float64)
        s["ids"] = (u ** case["skew"] * vocab).long().clamp_(max=vocab - 1)
        s["ids"][torch.rand((case["tokens"],), generator=gen, device=DEV) < 0.02] = -1       # padding
        s["scale"], s["backward"], s["vocab"] = math.sqrt(width), case["backward"], vocab
        if case["backward"]:
            s["grad"] = normal(case["tokens"], width, scale=1e-2)
        else:
            s["table"] = normal(vocab, width, scale=width ** -0.5)
        return s
    # hidden states behind a norm; each leans towards its target's row, from not at all to strongly
    rows = case["rows"]
    s["weight"] = normal(vocab, width, scale=2.0 * width ** -0.5)
    s["targets"] = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
    lean = 3.0 * torch.rand((rows, 1), generator=gen, device=DEV)
    s["x"] = (normal(rows, width, dtype=torch.float32) + lean * s["weight"][s["targets"]].float()).to(t)
    s["targets"][torch.rand((rows,), generator=gen, device=DEV) < 0.05] = -1                 # places that ask for no token
    if op == "head_backward":
        # a mean over the tokens
        s["g_logprob"] = -(0.5 + torch.rand((rows,), generator=gen, device=DEV)) / rows
        s["g_entropy"] = normal(rows, scale=0.1 / rows, dtype=torch.float32) if case["entropy"] else None
        s["lse"], s["entropy"] = _moments(s["x"].float() @ s["weight"].float().t())
        s["frozen"] = case["frozen"]
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _moments(z):
    """lse and entropy of each row's softmax."""
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1)
    lse = torch.log(total) + top[:, 0]
    return lse, lse - (e * z).sum(-1) / total


def _plain_head(s):
    z = s["x"].to(torch.float32) @ s["weight"].to(torch.float32).t()
    lse, entropy = _moments(z)
    asked = s["targets"] >= 0
    lp = torch.gather(z, 1, s["targets"].clamp_min(0)[:, None])[:, 0] - lse
    return {"logprob": torch.where(asked, lp, torch.zeros_like(lp)), "entropy": entropy, "lse": lse}


def _plain_head_backward(s):
    x, w = s["x"].to(torch.float32), s["weight"].to(torch.float32)
    lp = (x @ w.t()).sub_(s["lse"][:, None])
    p = torch.exp(lp)
    g = torch.where(s["targets"] >= 0, s["g_logprob"], torch.zeros_like(s["g_logprob"]))
    if s["g_entropy"] is None:
        d = p.mul_(-g[:, None])
    else:
        d = p.mul_(-g[:, None] - s["g_entropy"][:, None] * lp.add_(s["entropy"][:, None]))
    d[torch.arange(d.shape[0], device=DEV), s["targets"].clamp_min(0)] += g
    gx = (d @ w).to(s["x"].dtype)
    return {"x": gx} if s["frozen"] else {"x": gx, "weight": (d.t() @ x).to(s["x"].dtype)}


def _plain_embed(s):
    asked = (s["ids"] >= 0)[:, None]
    if s["backward"]:
        g = s["grad"].to(torch.float32) * s["scale"]
        total = torch.zeros((s["vocab"], g.shape[1]), device=DEV)
        total.index_add_(0, s["ids"].clamp_min(0), torch.where(asked, g, torch.zeros_like(g)))
        return total.to(s["grad"].dtype)
    rows = s["table"][s["ids"].clamp_min(0)].to(torch.float32) * s["scale"]
    return torch.where(asked, rows, torch.zeros_like(rows)).to(s["table"].dtype)


def _plain_clip(s):
    total = torch.stack([g.to(torch.float32).square().sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = torch.sqrt(total)
    factor = torch.clamp(s["max_norm"] / norm, max=1.0).to(torch.float32)
    for g, c in zip(s["grads"], s["clipped"]):
        c.copy_(g.to(torch.float32) * factor)
    return {"norm": norm.to(torch.float32), **s["whole_clipped"]}


def run(s):
    op = s["op"]
    if not own:
        return {"head": _plain_head, "head_backward": _plain_head_backward, "embed": _plain_embed, "clip": _plain_clip}[op](s)
    from paper_2607_13511_amd import binding
    if op == "head":
        got = binding.linear_logprobs(s["x"], s["weight"], s["targets"])
        return {"logprob": got.logprob, "entropy": got.entropy, "lse": got.lse}
    if op == "head_backward":
        gx, gw = binding.linear_logprobs_backward(s["x"], s["weight"], s["targets"], s["lse"], s["entropy"],
                                                  grad_logprob=s["g_logprob"], grad_entropy=s["g_entropy"],
                                                  need_weight=not s["frozen"])
        return {"x": gx} if s["frozen"] else {"x": gx, "weight": gw}
    if op == "embed":
        if s["backward"]:
            return binding.embedding_backward(s["grad"], s["ids"], s["vocab"], scale=s["scale"])
        return binding.embedding(s["table"], s["ids"], scale=s["scale"])
    norm = binding.clip_gradients(s["grads"], s["max_norm"], out=s["clipped"])
    return {"norm": norm, **s["whole_clipped"]}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_head(s, backward):
    w = s["weight"].double()
    wt = w.t().contiguous()
    lse, entropy, logprob, gx, gw = [], [], [], [], 0.0
    step = max(1, min(256, int(1e8) // w.shape[0]))
    for a in range(0, s["x"].shape[0], step):
        x, y = s["x"][a:a + step].double(), s["targets"][a:a + step]
        lp = torch.log_softmax(x @ wt, -1)
        hot = torch.zeros_like(lp).scatter_(1, y.clamp(min=0)[:, None], (y >= 0).double()[:, None])
        if not backward:
            entropy.append(-(lp.exp() * lp).sum(-1))
            lse.append(torch.logsumexp(x @ wt, -1))
            logprob.append((hot * lp).sum(-1))
            continue
        p = lp.exp()
        d = s["g_logprob"][a:a + step].double()[:, None] * (hot - (y >= 0).double()[:, None] * p)
        if s["g_entropy"] is not None:
            h = -(p * lp).sum(-1, keepdim=True)
            d -= s["g_entropy"][a:a + step].double()[:, None] * p * (lp + h)
        gx.append(d @ w)
        if not s["frozen"]:
            gw = gw + d.t().contiguous() @ x
    if not backward:
        return {"logprob": torch.cat(logprob), "entropy": torch.cat(entropy), "lse": torch.cat(lse)}
    return {"x": torch.cat(gx)} if s["frozen"] else {"x": torch.cat(gx), "weight": gw}


def _exact_embed(s):
    ids = s["ids"]
    if not s["backward"]:
        padded = torch.cat([s["table"], torch.zeros_like(s["table"][:1])])
        return padded[torch.where(ids < 0, torch.full_like(ids, s["vocab"]), ids)].double() * s["scale"]
    # running sums over the tokens in the order of their ids; a token's sum is the difference of two of them
    order = torch.argsort(ids, stable=True)
    sums = torch.cumsum(s["grad"][order].double(), 0)
    sums = torch.cat([torch.zeros_like(sums[:1]), sums])
    upto = torch.searchsorted(ids[order], torch.arange(s["vocab"] + 1, device=DEV))
    return (sums[upto[1:]] - sums[upto[:-1]]) * s["scale"]


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "embed":
        return _exact_embed(s)
    if s["op"] == "clip":
        norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
        factor = min(1.0, s["max_norm"] / norm)
        return {"norm": torch.tensor(norm, dtype=torch.float64, device=DEV), **{t: g.double() * factor for t, g in s["whole"].items()}}
    return _exact_head(s, s["op"] == "head_backward")
