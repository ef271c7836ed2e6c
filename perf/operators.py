"""Cases of the decoding operators: rotary positions, the 4-bit cache,
attention over that cache, and log probabilities of given tokens.

They are what a model runs between and behind its factored projections:
``apply`` gives q, k and v, ``rotary`` turns q and k to their positions,
``kv4_append`` stores k and v in 4 bits, ``kv4_attention`` reads the cache,
and behind the last projection ``token_logprobs`` says how likely the given
next tokens were (perplexity), with the distribution's entropy and its most
likely tokens; ``token_logprobs_backward`` and ``rotary_backward`` are the
gradients.

``run`` computes an operator in plain torch operations, or, where ``own`` is
true, through ``paper_2607_13511_amd.binding``.  Head counts and widths are
those of the 2560 x 4096 and 2560 x 1024 attention projections of the test
configurations (32 query heads and 8 cache heads of 128 channels), and the
same rows split into heads of 64 and 256 channels.

The cache, per page of P tokens and cache head, holds P*D/2 bytes of K codes
(token by token; byte i is channel i in the low nibble and channel i + D/2 in
the high one), P*D/2 bytes of V codes (the same bytes, in blocks of 16
tokens with the tokens of one byte column side by side) and 16-bit words
[P][K, V][D/64]: the scale as fp16 whose low four mantissa bits hold the
zero point.  A value is scale * (code - zero point).
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
GROUP = 64                    # channels that share a scale
S_MAX = 4352.0                # 15 * S_MAX is the largest value an fp16 number with a 7-bit scale reaches
META_NAN = 0x7E00             # the word of a group that held an infinity or a NaN


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _rotary(name, tokens, heads, kv_heads, dim, rot, dtype, interleaved, backward, top_position):
    return {"name": name, "op": "rotary", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot,
            "dtype": dtype, "interleaved": interleaved, "backward": backward, "top_position": top_position}


def _append(name, batch, new, length, kv_heads, dim, page, dtype):
    return {"name": name, "op": "append", "batch": batch, "new": new, "length": length, "kv_heads": kv_heads, "dim": dim,
            "page": page, "dtype": dtype}


def _attention(name, batch, new, length, heads, kv_heads, dim, page, window, dtype):
    return {"name": name, "op": "attention", "batch": batch, "new": new, "length": length, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "window": window, "dtype": dtype}


def _logprobs(name, rows, vocab, top, dtype, backward):
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "backward": backward}


def listed():
    return [
        # q and k of one token, as apply returns them: the step of a single user
        _rotary("rotary_1_token", 1, 32, 8, 128, 128, "fp32", False, False, 4096),
        # gradients of q and k of a training batch: neighbouring pairs, half of each head turned, long positions
        _rotary("rotary_backward_8191", 8191, 32, 8, 128, 64, "bf16", True, True, 131072),
        # one new token each for 32 users, from apply's fp32 outputs
        _append("append_32_tokens", 32, 1, 2000, 8, 128, 32, "fp32"),
        # the prompts of three users enter the cache
        _append("append_prompts", 3, 2731, 2731, 8, 128, 64, "bf16"),
        # one token of a single user over a short cache, apply's fp32 types: latency
        _attention("attention_1_user_517", 1, 1, 517, 32, 8, 128, 16, 0, "fp32"),
        # one token each for 32 users at mixed lengths
        _attention("attention_32_users", 32, 1, 16384, 32, 8, 128, 32, 0, "bf16"),
        # one token over one very long cache
        _attention("attention_131071", 1, 1, 131071, 32, 8, 128, 256, 0, "fp16"),
        # a few drafted tokens each, verified at once; heads of 64, a window, odd lengths
        _attention("attention_drafts", 7, 5, 4001, 16, 2, 64, 16, 1500, "bf16"),
        # chunks of two prompts over what the cache already holds
        _attention("attention_chunks", 2, 2048, 12001, 32, 8, 128, 64, 0, "bf16"),
        # eight decoded tokens with their alternatives, fp32 logits
        _logprobs("logprobs_8_rows", 8, 65536, 5, "fp32", False),
        # perplexity of a text of 2048 tokens over a large vocabulary of odd size
        _logprobs("logprobs_2048_rows", 2048, 150001, 20, "bf16", False),
        # gradient of the text's log probabilities and entropies
        _logprobs("logprobs_backward", 2048, 65537, 0, "bf16", True),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotary", "append", "attention", "attention", "attention", "logprobs", "logprobs"))
    dtype = rng.choice(tuple(TYPES))
    dim = rng.choice((64, 128, 128, 256))
    kv_heads = rng.choice((1, 2, 4, 8))
    heads = kv_heads * rng.choice((1, 2, 4, 4, 5, 8))
    page = rng.choice((16, 32, 64, 128, 256))
    if op == "rotary":
        c = _rotary("", _spread(rng, 1, 8191), heads, kv_heads, dim, rng.choice((dim, dim // 2, dim - 14)), dtype,
                    rng.random() < 0.5, rng.random() < 0.5, _spread(rng, 100, 1 << 20))
    elif op == "append":
        new = _spread(rng, 1, 2731)
        batch = _spread(rng, 1, max(1, min(64, 8192 // new)))
        c = _append("", batch, new, new + _spread(rng, 1, 4000) - 1, kv_heads, dim, page, dtype)
    elif op == "attention":
        new = rng.choice((1, 1, 1, _spread(rng, 2, 8), _spread(rng, 2, 2048)))
        batch = _spread(rng, 1, 32) if new == 1 else _spread(rng, 1, max(1, min(16, 2048 // new)))
        length = new + _spread(rng, 1, min(131071, max(2, 200000 // batch)) if new < 9 else 12001) - 1
        c = _attention("", batch, new, length, heads, kv_heads, dim, page, rng.choice((0, 0, 0, _spread(rng, 1, 4096))), dtype)
    else:
        vocab = _spread(rng, 1000, 150001)
        backward = rng.random() < 0.4
        rows = _spread(rng, 1, min(2048, 500_000_000 // (vocab * BYTES[dtype] * (2 if backward else 1))))
        c = _logprobs("", rows, vocab, 0 if backward else rng.choice((0, 1, 5, 20, 33, 64)), dtype, backward)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# what a case's sequences are (from the case alone)
# ---------------------------------------------------------------------------
def _sequences(case):
    """(lengths, new tokens) of each sequence.  The first has the case's
    length and new tokens, the others from a quarter of it up; where there
    are five or more, one is empty and one has no new token."""
    r = random.Random("%d %d %d" % (case["batch"], case["new"], case["length"]))
    lens, news = [case["length"]], [case["new"]]
    for b in range(1, case["batch"]):
        n = case["new"] if case["new"] < 3 else r.randint(max(1, case["new"] // 4), case["new"])
        if b == 4:
            n = 0 if case["new"] > 1 else 1
        lens.append(0 if b == 3 and case["batch"] > 4 else max(n, r.randint(max(1, case["length"] // 4), case["length"])))
        news.append(0 if lens[-1] == 0 and case["new"] > 1 else n)
    return lens, news


def _visible(case):
    """(query, key) pairs that attention sees, and cache tokens that some query sees."""
    lens, news = _sequences(case)
    w = case.get("window", 0)
    pairs = keys = 0
    for n, q in zip(lens, news):
        for p in range(n - q, n):
            if p >= 0:
                pairs += min(p + 1, w) if w else p + 1
        if q and n:
            keys += min(n, w + q - 1) if w else n
    return pairs, keys


def work(case):
    op, es = case["op"], BYTES[case["dtype"]]
    if op == "rotary":
        both = case["heads"] + case["kv_heads"]
        return {"bytes": 2 * case["tokens"] * both * case["dim"] * es + 8 * case["tokens"],
                "flops": 4 * case["tokens"] * both * case["rot"]}
    if op == "logprobs":
        each = case["rows"] * case["vocab"]
        if case["backward"]:
            return {"bytes": 2 * each * es + 24 * case["rows"], "flops": 8 * each}
        return {"bytes": each * es + case["rows"] * (20 + 8 * case["top"]), "flops": 6 * each}
    dim, kv = case["dim"], case["kv_heads"]
    token = kv * (dim + dim // 16)                     # cache bytes of a token: K, V and their words
    lens, news = _sequences(case)
    if op == "append":                                 # written, and read back as values
        t = sum(news)
        return {"bytes": 2 * t * kv * dim * es * 2 + 2 * t * token, "flops": 2 * 6 * t * kv * dim}
    pairs, keys = _visible(case)
    t = sum(news)
    return {"bytes": keys * token + 2 * t * case["heads"] * dim * es + 4 * t * case["heads"],
            "flops": 4 * dim * case["heads"] * pairs}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _split(x):
    """(codes, words) of the values x (..., D) in fp32: see the top of this file."""
    xg = x.unflatten(-1, (-1, GROUP))
    fine = torch.isfinite(xg).all(-1)
    xg = torch.where(fine[..., None], xg, torch.zeros_like(xg))
    hi, lo = xg.amax(-1).clamp_min(0.0), xg.amin(-1).clamp_max(0.0)
    s = torch.div(hi - lo, torch.full_like(hi, 15.0))
    seven = ((s.view(torch.int32) + 0x1FFFF) & ~0x1FFFF).view(torch.float32)
    small = torch.ceil(s * 2.0 ** 20) * 2.0 ** -20
    s = torch.where(s < 2.0 ** -14, small, seven).clamp_max(S_MAX)
    by = torch.where(s > 0, s, torch.ones_like(s))
    z = torch.round(torch.div(-lo, by)).clamp(0.0, 15.0)
    c = (torch.round(torch.div(xg, by[..., None])) + z[..., None]).clamp(0.0, 15.0)
    word = (s.to(torch.float16).view(torch.int16).to(torch.int32) & 0xFFFF) | z.to(torch.int32)
    word = torch.where(fine, word, torch.full_like(word, META_NAN))
    c = torch.where(fine[..., None], c, torch.zeros_like(c))
    return c.flatten(-2).to(torch.uint8), word


def _page_bytes(page, dim):
    return page * (dim + dim // 16)


def _store(cache, slot, k, v, page):
    """Writes k and v (tokens, heads, D) in fp32 at the token slots (page * P + offset) of the cache."""
    pages, heads, _ = cache.shape
    dim = k.shape[-1]
    half, groups = dim // 2, dim // GROUP
    at, off = slot // page, slot % page
    words = cache[:, :, page * dim:].view(torch.int16).unflatten(-1, (page, 2, groups))
    kc, kw = _split(k)
    vc, vw = _split(v)
    cache[:, :, :page * half].unflatten(-1, (page, half))[at, :, off] = kc[..., :half] | (kc[..., half:] << 4)
    blocks = cache[:, :, page * half:page * dim].unflatten(-1, (page // 16, half, 16))
    blocks[at, :, off // 16, :, off % 16] = vc[..., :half] | (vc[..., half:] << 4)
    words[at, :, off, 0] = kw.to(torch.int16)
    words[at, :, off, 1] = vw.to(torch.int16)


def _load(cache, table, page, dim, only=None):
    """K and V as fp32 (sequences, tokens, heads, D) of the pages that `table` names."""
    half, groups = dim // 2, dim // GROUP
    got = cache[table]                                                       # B, n, H, bytes
    words = got[..., page * dim:].contiguous().view(torch.int16).to(torch.int32).unflatten(-1, (page, 2, groups))
    scale = (words & 0xFFF0).to(torch.int16).view(torch.float16).to(torch.float32)
    zero = (words & 15).to(torch.float32)
    kb = got[..., :page * half].unflatten(-1, (page, half))
    vb = got[..., page * half:page * dim].unflatten(-1, (page // 16, half, 16)).transpose(-1, -2).flatten(-3, -2)

    def values(b, which):
        c = torch.cat([b & 15, b >> 4], -1).to(torch.float32).unflatten(-1, (groups, GROUP))
        x = (scale[..., which, :, None] * (c - zero[..., which, :, None])).flatten(-2)
        return x.transpose(2, 3).flatten(1, 2)                               # B, n * P, H, D
    return values(kb, 0), values(vb, 1)


def _kv(gen, tokens, heads, dim, dtype):
    """k has channels that stand out, as keys behind rotary positions do; v is near normal."""
    loud = 1.0 + 4.0 * (torch.rand((1, heads, dim), generator=gen, device=DEV) < 0.04).float()
    shift = 0.5 * torch.randn((1, heads, dim), generator=gen, device=DEV) * loud
    k = torch.randn((tokens, heads, dim), generator=gen, device=DEV) * loud + shift
    v = 0.7 * torch.randn((tokens, heads, dim), generator=gen, device=DEV)
    return k.to(TYPES[dtype]), v.to(TYPES[dtype])


def _paged(case, gen):
    """An empty pool in random page order, with a table; what no sequence owns holds arbitrary bytes."""
    lens, news = _sequences(case)
    page = case["page"]
    need = [-(-n // page) for n in lens]
    width = max(max(need), 1)
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    table, at = torch.zeros((len(lens), width), dtype=torch.int32, device=DEV), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cache = torch.randint(0, 256, (pages, case["kv_heads"], _page_bytes(page, case["dim"])), generator=gen, device=DEV,
                          dtype=torch.uint8)
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    one = all(n == 1 for n in news)
    return {"cache": cache, "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV),
            "starts": None if one else torch.from_numpy(starts).to(DEV), "max_new": max(news), "tokens": int(starts[-1])}


def _places(table, first, lens, page):
    """Slots of the tokens first[b] <= position < lens[b] of every sequence, in order."""
    n = [max(0, e - f) for f, e in zip(first, lens)]
    b = torch.repeat_interleave(torch.arange(len(n), device=DEV), torch.tensor(n, device=DEV))
    begin = torch.tensor([0] + list(np.cumsum(n)[:-1]), device=DEV)
    p = torch.arange(sum(n), device=DEV) - begin[b] + torch.tensor(first, device=DEV)[b]
    return table[b, p // page].long() * page + p % page


def prepare(case, seed):
    gen, op, t = _gen(seed), case["op"], TYPES[case["dtype"]]
    s = {"op": op, "dtype": t}
    if op == "rotary":
        n, dim, rot = case["tokens"], case["dim"], case["rot"]
        s["q"] = torch.randn((n, case["heads"], dim), generator=gen, device=DEV).to(t)
        s["k"] = torch.randn((n, case["kv_heads"], dim), generator=gen, device=DEV).to(t)
        s["positions"] = torch.randint(0, case["top_position"], (n,), generator=gen, device=DEV, dtype=torch.int64)
        # turns a position in units of 2^-64, positions stretched fourfold as for a context of four times the trained one
        s["freqs"] = torch.tensor([int(round(2.0 ** 64 / (2 * math.pi) / 4.0 * 1e6 ** (-2.0 * i / rot))) for i in range(rot // 2)],
                                  dtype=torch.int64, device=DEV)
        s["interleaved"], s["backward"], s["amplitude"] = case["interleaved"], case["backward"], 0.1 * math.log(4.0) + 1.0
        return s
    if op == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        x = torch.randn((rows, vocab), generator=gen, device=DEV)
        x.mul_(2.0).add_(4.0 * (torch.rand((rows, vocab), generator=gen, device=DEV) < 3e-4).float())
        s["logits"] = x.to(t)
        s["targets"] = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
        s["targets"][torch.rand((rows,), generator=gen, device=DEV) < 0.05] = -1        # places that ask for no token
        s["top"], s["backward"] = case["top"], case["backward"]
        if case["backward"]:
            s["lse"], s["entropy"] = _moments(s["logits"])
            s["g_logprob"] = torch.randn((rows,), generator=gen, device=DEV)
            s["g_entropy"] = 0.1 * torch.randn((rows,), generator=gen, device=DEV)
        return s
    s.update(_paged(case, gen))
    lens, news = _sequences(case)
    page, dim, kv = case["page"], case["dim"], case["kv_heads"]
    s["dim"] = dim
    if op == "append":
        s["k"], s["v"] = _kv(gen, s["tokens"], kv, dim, case["dtype"])
        return s
    k, v = _kv(gen, sum(lens), kv, dim, "fp32")
    _store(s["cache"], _places(s["table"], [0] * len(lens), lens, page), k, v, page)
    del k, v
    s["q"] = torch.randn((s["tokens"], case["heads"], dim), generator=gen, device=DEV).to(t)
    s["window"] = case["window"]
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _turned(x, cos, sin, rot, interleaved, amplitude):
    y = x.to(torch.float32)
    r = y[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    c, d = amplitude * (a * cos - b * sin), amplitude * (b * cos + a * sin)
    r = torch.stack([c, d], -1).flatten(-2) if interleaved else torch.cat([c, d], -1)
    return torch.cat([r, y[..., rot:]], -1).to(x.dtype)


def _plain_rotary(s):
    turns = (s["positions"][:, None] * s["freqs"][None, :]) >> 32            # wraps at whole turns; 2^-32 turns
    angle = turns.to(torch.float32) * (2.0 * math.pi / 2.0 ** 32)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    sin = -sin if s["backward"] else sin
    rot = 2 * s["freqs"].numel()
    return [_turned(s[x], cos, sin, rot, s["interleaved"], s["amplitude"]) for x in ("q", "k")]


def _newest(s):
    """(sequence, position) of each new token; a position below zero is before the sequence."""
    batch = s["lens"].numel()
    if s["starts"] is None:
        b = torch.arange(batch, device=DEV)
        return b, s["lens"].long() - 1
    n = (s["starts"][1:] - s["starts"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(batch, device=DEV), n, output_size=s["tokens"])
    return b, torch.arange(s["tokens"], device=DEV) - s["starts"][1:][b].long() + s["lens"][b].long()


def _plain_append(s):
    page = s["cache"].shape[2] // (s["dim"] + s["dim"] // 16)
    b, p = _newest(s)
    kept = p >= 0
    slot = s["table"][b, p.clamp_min(0) // page].long() * page + p.clamp_min(0) % page
    _store(s["cache"], slot[kept], s["k"].to(torch.float32)[kept], s["v"].to(torch.float32)[kept], page)
    k, v = _at(s["cache"], slot, page, s["dim"])
    kept = kept[:, None, None]
    return [torch.where(kept, k, torch.zeros_like(k)).to(s["dtype"]), torch.where(kept, v, torch.zeros_like(v)).to(s["dtype"])]


def _at(cache, slot, page, dim):
    """K and V as fp32 (tokens, heads, D) at token slots."""
    half, groups = dim // 2, dim // GROUP
    at, off = slot // page, slot % page
    kb = cache[:, :, :page * half].unflatten(-1, (page, half))[at, :, off]
    vb = cache[:, :, page * half:page * dim].unflatten(-1, (page // 16, half, 16))[at, :, off // 16, :, off % 16]
    words = cache[:, :, page * dim:].view(torch.int16).unflatten(-1, (page, 2, groups))[at, :, off].to(torch.int32)
    scale = (words & 0xFFF0).to(torch.int16).view(torch.float16).to(torch.float32)
    zero = (words & 15).to(torch.float32)

    def values(b, which):
        c = torch.cat([b & 15, b >> 4], -1).to(torch.float32).unflatten(-1, (groups, GROUP))
        return (scale[..., which, :, None] * (c - zero[..., which, :, None])).flatten(-2)
    return values(kb, 0), values(vb, 1)


def _plain_attention(s):
    q, cache, lens = s["q"], s["cache"], s["lens"].long()
    tokens, heads, dim = q.shape
    kv, page = cache.shape[1], cache.shape[2] // (dim + dim // 16)
    batch, each = lens.numel(), heads // cache.shape[1]
    k, v = _load(cache, s["table"].long(), page, dim)
    length = k.shape[1]
    b, p = _newest(s)
    first = lens - (torch.bincount(b, minlength=batch) if s["starts"] is not None else 1)
    i = p - first[b]
    most = s["max_new"]
    rows = torch.zeros((batch, most, heads, dim), device=DEV)
    rows[b, i] = q.to(torch.float32)
    rows = rows.view(batch, most, kv, each, dim).transpose(1, 2).reshape(batch, kv, most * each, dim)
    t = torch.arange(length, device=DEV)
    here = (t[None] < lens[:, None])[:, :, None, None]
    k = torch.where(here, k, torch.zeros_like(k)).permute(0, 2, 3, 1).contiguous()
    v = torch.where(here, v, torch.zeros_like(v)).transpose(1, 2).contiguous()
    at = (first[:, None] + torch.arange(most, device=DEV)).repeat_interleave(each, 1)[:, :, None]     # B, most * each, 1
    seen = (t <= at) & (t < lens[:, None, None])
    seen = seen & (t > at - s["window"]) if s["window"] else seen
    x = torch.matmul(rows, k).mul_(1.0 / math.sqrt(dim)).masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.log(total) + top
    out = out.view(batch, kv, most, each, dim).transpose(1, 2).reshape(batch, most, heads, dim)[b, i]
    lse = lse.view(batch, kv, most, each).transpose(1, 2).reshape(batch, most, heads)[b, i]
    return {"out": out.to(s["dtype"]), "lse": lse}


def _moments(x):
    """lse and entropy of each row's softmax."""
    x = x.to(torch.float32)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1)
    lse = torch.log(total) + top[:, 0]
    mean = torch.where(e > 0, e * x, torch.zeros_like(e)).sum(-1) / total
    return lse, lse - mean


def _plain_logprobs(s):
    x, y = s["logits"].to(torch.float32), s["targets"]
    rows, vocab = x.shape
    asked = y >= 0
    if s["backward"]:
        lp = x - s["lse"][:, None]
        p = torch.exp(lp)
        g = torch.where(asked, s["g_logprob"], torch.zeros_like(s["g_logprob"]))
        d = -p * (g[:, None] + s["g_entropy"][:, None] * (lp + s["entropy"][:, None]))
        d[torch.arange(rows, device=DEV), y.clamp_min(0)] += g
        return d.to(s["dtype"])
    lse, entropy = _moments(x)
    lp = x[torch.arange(rows, device=DEV), y.clamp_min(0)] - lse
    r = {"logprob": torch.where(asked, lp, torch.zeros_like(lp)), "entropy": entropy, "lse": lse}
    if s["top"]:
        # the largest first, of equal ones the lowest index: both in one whole number
        bits = (x + 0.0).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
        keys = (bits << 32) | (0xFFFFFFFF - torch.arange(vocab, device=DEV))
        best = 0xFFFFFFFF - (torch.topk(keys, s["top"], dim=-1).values & 0xFFFFFFFF)
        r["top_ids"] = best
        r["top_logprobs"] = torch.gather(x, 1, best) - lse[:, None]
    return r


def run(s):
    op = s["op"]
    if not own:
        return {"rotary": _plain_rotary, "append": _plain_append, "attention": _plain_attention, "logprobs": _plain_logprobs}[op](s)
    from paper_2607_13511_amd import binding
    if op == "rotary":
        turn = binding.rotary_backward if s["backward"] else binding.rotary
        return list(turn(s["q"], s["k"], s["positions"], s["freqs"], interleaved=s["interleaved"], amplitude=s["amplitude"]))
    if op == "append":
        binding.kv4_append(s["cache"], s["k"], s["v"], s["table"], s["lens"], starts=s["starts"])
        return list(binding.kv4_read(s["cache"], s["table"], s["lens"], s["dim"], starts=s["starts"], tokens=s["tokens"],
                                     dtype=s["dtype"]))
    if op == "attention":
        out, lse = binding.kv4_attention(s["cache"], s["q"], s["table"], s["lens"], starts=s["starts"], max_new=s["max_new"],
                                         window=s["window"])
        return {"out": out, "lse": lse}
    if s["backward"]:
        return binding.token_logprobs_backward(s["logits"], s["targets"], s["lse"], s["entropy"], s["g_logprob"], s["g_entropy"])
    got = binding.token_logprobs(s["logits"], s["targets"], top=s["top"])
    r = {"logprob": got.logprob, "entropy": got.entropy, "lse": got.lse}
    return {**r, "top_ids": got.top_ids, "top_logprobs": got.top_logprobs} if s["top"] else r


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_rotary(s):
    turns = (s["positions"][:, None] * s["freqs"][None]).double() / 2.0 ** 64 * (-1.0 if s["backward"] else 1.0)
    turn = torch.polar(torch.full_like(turns, s["amplitude"]), 2 * math.pi * turns)[:, None]
    half, got = s["freqs"].numel(), []
    for x in (s["q"].double(), s["k"].double()):
        y = x.clone()
        if s["interleaved"]:
            y[..., :2 * half] = torch.view_as_real(torch.view_as_complex(x[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * turn).flatten(-2)
        else:
            w = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
            y[..., :half], y[..., half:2 * half] = w.real, w.imag
        got.append(y)
    return got


def _exact_store(x, kept):
    """The values that x (tokens, heads, D) in 64 bits stands for once it is held in 4 bits; 0 where a token is not kept."""
    got = torch.empty_like(x)
    for g in range(0, x.shape[-1], GROUP):
        y = x[..., g:g + GROUP]
        lo, hi = y.min(-1, keepdim=True)[0].clamp(max=0), y.max(-1, keepdim=True)[0].clamp(min=0)
        s = (hi - lo) / 15
        e = torch.frexp(s.clamp(min=2.0 ** -14)).exponent.long() - 7       # seven bits of s are whole in units of 2^e
        unit = ((e + 1023) << 52).view(torch.float64)
        s = (torch.ceil(s / unit) * unit).clamp(max=S_MAX)
        z = torch.where(s > 0, torch.round(-lo / s), torch.zeros_like(s)).clamp(0, 15)
        got[..., g:g + GROUP] = torch.where(s > 0, s * ((torch.round(y / s) + z).clamp(0, 15) - z), torch.zeros_like(y))
    return got * kept.double()[:, None, None]


def _exact_values(cache, b, table, n, page, dim, head, which):
    """K (which = 0) or V (1) of one sequence and head in 64 bits, by the nibbles' places."""
    t = torch.arange(n, device=DEV)
    rows = cache[table[b].long()[t // page], head]
    c = torch.arange(dim, device=DEV)
    i, o = c % (dim // 2), (t % page)[:, None]
    place = o * (dim // 2) + i if which == 0 else page * dim // 2 + (o // 16 * (dim // 2) + i) * 16 + o % 16
    code = (torch.gather(rows, 1, place) >> (4 * (c // (dim // 2))).to(torch.uint8)) & 15
    w = page * dim + 2 * ((o * 2 + which) * (dim // GROUP) + c // GROUP)
    lo, hi = torch.gather(rows, 1, w).int(), torch.gather(rows, 1, w + 1).int()
    scale = ((lo & 0xF0) | (hi << 8)).to(torch.int16).view(torch.float16).double()
    return scale * (code.double() - (lo & 15).double())


def _exact_attention(s):
    q = s["q"].double()
    tokens, heads, dim = q.shape
    cache, page = s["cache"], s["cache"].shape[2] // (dim + dim // 16)
    each = heads // cache.shape[1]
    lens = s["lens"].tolist()
    starts = s["starts"].tolist() if s["starts"] is not None else list(range(len(lens) + 1))
    out, lse = torch.zeros_like(q), torch.full((tokens, heads), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        a, e = starts[b], starts[b + 1]
        if n == 0 or a == e:
            continue
        t = torch.arange(n, device=DEV)
        at = (n - (e - a) + torch.arange(e - a, device=DEV))[:, None]
        gone = (t > at) | ((t <= at - s["window"]) if s["window"] else torch.zeros_like(t > at))
        for h in range(cache.shape[1]):
            k = _exact_values(cache, b, s["table"], n, page, dim, h, 0).t().contiguous()
            v = _exact_values(cache, b, s["table"], n, page, dim, h, 1)
            for j in range(h * each, (h + 1) * each):
                x = (q[a:e, j] @ k / math.sqrt(dim)).masked_fill(gone, -math.inf)
                lse[a:e, j] = torch.logsumexp(x, -1)
                out[a:e, j] = torch.exp(x - lse[a:e, j, None]) @ v
    return {"out": out, "lse": lse}


def _exact_logprobs(s):
    kept = {"logprob": [], "entropy": [], "lse": [], "top_logprobs": []}
    grads = []
    for a in range(0, s["logits"].shape[0], 256):
        x, y = s["logits"][a:a + 256].double(), s["targets"][a:a + 256]
        lp = torch.log_softmax(x, -1)
        p = lp.exp()
        h = -(p * lp).sum(-1)
        asked = (y >= 0).double()
        if s["backward"]:
            g = s["g_logprob"][a:a + 256].double() * asked
            hot = torch.zeros_like(x).scatter_(1, y.clamp(min=0)[:, None], 1.0)
            grads.append(g[:, None] * (hot - p) - s["g_entropy"][a:a + 256].double()[:, None] * p * (lp + h[:, None]))
        kept["logprob"].append(lp.gather(1, y.clamp(min=0)[:, None])[:, 0] * asked)
        kept["entropy"].append(h)
        kept["lse"].append(torch.logsumexp(x, -1))
        kept["top_logprobs"].append(torch.sort(lp, -1, descending=True).values[:, :s["top"]])
    if s["backward"]:
        return torch.cat(grads)
    r = {n: torch.cat(v) for n, v in kept.items()}
    if not s["top"]:
        del r["top_logprobs"]
        return r
    return {**r, "top_ids": None}


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "rotary":
        return _exact_rotary(s)
    if s["op"] == "append":
        lens, news = _sequences(case)
        kept = torch.tensor([n >= e - i for n, e in zip(lens, news) for i in range(e)], device=DEV)
        return [_exact_store(s["k"].double(), kept), _exact_store(s["v"].double(), kept)]
    return _exact_attention(s) if s["op"] == "attention" else _exact_logprobs(s)
