"""Attention and its cache as cases to time: tokens entering a paged cache with their rotary
embedding, attention over whole packed prompts, a training step of it (results and gradients), and
attention of new tokens over the cache - from one token of one sequence to a chunk of a prompt.

`run` goes through the entry points of the package where `own` is true and through the operators'
plain forms, 32-bit torch operations over masked scores, where it is not.  Heads and widths are
those of the repository's 7b, 13b and 70B-shaped workloads (heads of 128 elements) next to smaller
and odd ones; lists of lengths are texts, one number per sequence.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
THETA = 10000.0


def _numbers(text):
    return [int(x) for x in text.split(",")]


def _text(numbers):
    return ",".join(str(n) for n in numbers)


def _ragged(rng, n, total, least=1):
    """n lengths of at least `least` that add up to about `total`, spread over a factor of ten and more, as a text."""
    w = [math.exp(rng.gauss(0.0, 0.8)) for _ in range(n)]
    lens = [max(least, int(total * x / sum(w))) for x in w]
    return _text(n | (n > 2048) for n in lens)      # long ones are odd


# ------------------------------------------------------------------ cases ---
def listed():
    many = random.Random(7)
    return [
        # one sequence's next token enters the cache, 13b: launch and latency
        {"name": "append 13b one token", "kind": "append", "new": "1", "past": "700", "heads": 40, "kv": 40, "dim": 128, "page": 16,
         "interleaved": False, "dtype": "f16", "fused": False},
        # a batch of prompts enters it, 70B-shaped, q, k and v in one buffer
        {"name": "append 70b 16 prompts", "kind": "append", "new": _ragged(many, 16, 6000), "past": _text([0] * 16), "heads": 64, "kv": 8,
         "dim": 128, "page": 64, "interleaved": True, "dtype": "bf16", "fused": True},
        # the ragged prompt of the repository's timed blocks
        {"name": "prompt 7b T333", "kind": "prompt", "lens": "333", "heads": 32, "kv": 32, "dim": 128, "causal": True, "dtype": "f16", "fused": False},
        # one long prompt, 70B-shaped, grouped heads
        {"name": "prompt 70b T8192", "kind": "prompt", "lens": "8192", "heads": 64, "kv": 8, "dim": 128, "causal": True, "dtype": "bf16", "fused": False},
        # packed texts of an encoder, every length its own, an empty one and one of a single token among them
        {"name": "packed 12x64 both ways", "kind": "prompt", "lens": "511,1,0,1290,77,1024,333,64,899,127,2001", "heads": 12, "kv": 4, "dim": 64,
         "causal": False, "dtype": "f16", "fused": True},
        # a small training step: heads of an odd width, two short sequences
        {"name": "grad 8x96 T230", "kind": "grad", "lens": "129,101", "heads": 8, "kv": 2, "dim": 96, "causal": True, "dtype": "f16", "fused": False},
        # the tokens of the repository's timed training step
        {"name": "grad 7b T512", "kind": "grad", "lens": "512", "heads": 32, "kv": 32, "dim": 128, "causal": True, "dtype": "f16", "fused": False},
        # packed training sequences, grouped heads
        {"name": "grad 32x128 packed", "kind": "grad", "lens": "2048,613,1500,1,1930", "heads": 32, "kv": 8, "dim": 128, "causal": True, "dtype": "bf16",
         "fused": True},
        # single-stream decoding, 7b
        {"name": "decode 7b one token", "kind": "paged", "new": "1", "past": "2000", "heads": 32, "kv": 32, "dim": 128, "page": 16, "dtype": "f16",
         "fused": False},
        # a serving batch, 70B-shaped, contexts of every length
        {"name": "decode 70b x48", "kind": "paged", "new": _text([1] * 48), "past": _ragged(many, 48, 250000), "heads": 64, "kv": 8, "dim": 128, "page": 64,
         "dtype": "bf16", "fused": False},
        # a chunk of a long prompt next to seven sequences that decode
        {"name": "chunk 512 and singles", "kind": "paged", "new": "512,1,1,1,1,1,1,1", "past": "7700,1,300,4100,950,2047,15,6400", "heads": 32, "kv": 8,
         "dim": 128, "page": 32, "dtype": "f16", "fused": True},
        # drafts of a few tokens to be verified, 13b
        {"name": "drafts 13b 6x5", "kind": "paged", "new": "5,5,3,5,4,5", "past": "1100,2900,17,640,3333,512", "heads": 40, "kv": 40, "dim": 128, "page": 16,
         "dtype": "bf16", "fused": False},
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    kv = rng.choice((1, 2, 4, 5, 8, 16, 32, 40))
    heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8, 16) if kv * g <= 64])
    c = {"kind": rng.choice(("append", "prompt", "prompt", "grad", "grad", "paged", "paged", "paged")), "heads": heads, "kv": kv,
         "dim": rng.choice((64, 64, 80, 96, 128, 128, 128)), "dtype": rng.choice(("f16", "bf16")), "fused": rng.random() < 0.3}
    c["dim"] = 80 if c["dim"] * heads == 3072 else c["dim"]
    n = log_int(1, 48)
    if c["kind"] in ("prompt", "grad"):
        n = min(n, 16)
        c["causal"] = rng.random() < 0.7
        total = log_int(n, 8192 if c["kind"] == "prompt" else 6000)
        while total > n and total * total * heads > (8192 ** 2 if c["kind"] == "prompt" else 4096 ** 2) * (64 if c["causal"] else 32):
            total = total * 3 // 4
        c["lens"] = _ragged(rng, n, max(total, n), rng.choice((0, 1)))
        if not any(_numbers(c["lens"])):
            c["lens"] = _text([1] * n)
        return c
    c["page"] = rng.choice((16, 16, 32, 64, 128))
    if c["kind"] == "append":
        c["interleaved"] = rng.random() < 0.5
        c["new"] = _text([1] * n) if rng.random() < 0.4 else _ragged(rng, n, log_int(n, 6000))
        c["past"] = _text([log_int(1, 1000) - 1 for _ in range(n)])
        return c
    which = rng.choice(("single", "few", "chunk", "mixed"))
    n = n if which != "chunk" else min(n, 4)
    new = {"single": [1] * n, "few": [rng.randint(1, 8) for _ in range(n)], "chunk": [log_int(9, 700) for _ in range(n)],
           "mixed": [log_int(9, 700)] + [1] * (min(n, 12) - 1)}[which]
    limit = int(250000 * 8 / max(kv, 8)) if max(new) <= 8 else 12000
    c["new"] = _text(new)
    c["past"] = _ragged(rng, len(new), log_int(len(new), limit), 0)
    return c


# ----------------------------------------------------------------- inputs ---
def _heads(gen, tokens, case, with_kv=True):
    """q [tokens][heads][dim], k and v [tokens][kv][dim]: outputs of three layers, or parts of one's."""
    h, kv, d, dtype = case["heads"], case["kv"], case["dim"], DTYPES[case["dtype"]]
    n = h + 2 * kv if with_kv else h
    x = torch.randn((tokens, n, d), device=DEVICE, generator=gen)
    x[:, :h] *= 2.0      # scores spread like N(0, 2^2): a few keys of a row carry most of it
    x = x.to(dtype)
    parts = (x,) if not with_kv else (x[:, :h], x[:, h:h + kv], x[:, h + kv:])
    return parts if case["fused"] or not with_kv else tuple(p.contiguous() for p in parts)


def _starts(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEVICE)


class _Pages:
    """A cache as two tensors [pages][page][kv][dim]."""

    def __init__(self, k, v):
        self.k, self.v = k, v


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = {"kind": case["kind"], "scale": 1.0 / math.sqrt(case["dim"])}
    if case["kind"] in ("prompt", "grad"):
        lens = _numbers(case["lens"])
        s["q"], s["k"], s["v"] = _heads(gen, sum(lens), case)
        s["first"], s["causal"] = _starts(lens), case["causal"]
        if case["kind"] == "grad":
            s["do"] = (0.01 * torch.randn((sum(lens), case["heads"], case["dim"]), device=DEVICE, generator=gen)).to(s["q"].dtype)
        return s
    new, past = _numbers(case["new"]), _numbers(case["past"])
    lengths, page, dtype = [a + b for a, b in zip(new, past)], case["page"], DTYPES[case["dtype"]]
    used = [-(-n // page) for n in lengths]
    pages = sum(used) + 3
    order = torch.randperm(pages, device=DEVICE, generator=gen).to(torch.int32)
    table = torch.full((len(new), max(used) + 1), -1, dtype=torch.int32, device=DEVICE)
    for i, n in enumerate(used):
        table[i, :n] = order[sum(used[:i]):sum(used[:i + 1])]
    cache = [torch.empty((pages, page, case["kv"], case["dim"]), dtype=dtype, device=DEVICE).normal_(generator=gen) for _ in range(2)]
    s.update(table=table, first=_starts(new), lengths=torch.tensor(lengths, dtype=torch.int32, device=DEVICE), longest=max(new))
    s["cache"] = _Pages(*cache)
    if case["kind"] == "append":
        s["q"], s["k"], s["v"] = _heads(gen, sum(new), case)
        s["interleaved"] = case["interleaved"]
        rate = THETA ** (-torch.arange(0, case["dim"], 2, device=DEVICE).double() / case["dim"])
        angle = torch.arange(max(lengths), device=DEVICE).double()[:, None] * rate
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    else:
        s["q"], = _heads(gen, sum(new), case, with_kv=False)
    return s


# -------------------------------------------------------------------- run ---
def run(state):
    s = state
    if own:
        import paper_2602_05367_amd as rb
        if s["kind"] == "prompt":
            return rb.rb_attn_prompt(s["q"], s["k"], s["v"], s["first"], causal=s["causal"], scale=s["scale"])
        if s["kind"] == "grad":
            o, lse = rb.rb_attn_prompt(s["q"], s["k"], s["v"], s["first"], causal=s["causal"], scale=s["scale"], want_lse=True)
            dq, dk, dv = rb.rb_attn_prompt_grad(s["do"], s["q"], s["k"], s["v"], o, lse, s["first"], causal=s["causal"], scale=s["scale"])
            return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
        cache = rb.Cache(s["cache"].k, s["cache"].v)
        if s["kind"] == "append":
            q = rb.rb_cache_append(cache, s["k"], s["v"], s["first"], s["lengths"], s["table"], q=s["q"], cos=s["cos"], sin=s["sin"],
                                   interleaved=s["interleaved"])
            return {"q": q, "k": cache.k, "v": cache.v}
        return rb.rb_attn_paged(cache, s["q"], s["first"], s["lengths"], s["table"], scale=s["scale"])
    return {"prompt": _plain_prompt, "grad": _plain_grad, "append": _plain_append, "paged": _plain_paged}[s["kind"]](s)


def _sequence_of(first, tokens):
    """Which sequence each of the packed tokens belongs to, and its place there."""
    at = torch.arange(tokens, device=first.device)
    seq = torch.searchsorted(first[1:].contiguous(), at, right=True)
    return seq, at - first[seq]


def _softmax(scores, visible):
    """Softmax over the visible places of each row, with its log-sum; a row without any is zero."""
    scores = scores.masked_fill(~visible, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total), (top + torch.log(total)).squeeze(-1)


def _by_kv_head(x, kv):
    """[tokens][heads][dim] -> 32-bit [kv][tokens * heads / kv][dim]"""
    t, h, d = x.shape
    return x.float().reshape(t, kv, h // kv, d).permute(1, 0, 2, 3).reshape(kv, t * (h // kv), d)


def _back(x, tokens, heads):
    kv, d = x.shape[0], x.shape[2]
    return x.reshape(kv, tokens, heads // kv, d).permute(1, 0, 2, 3).reshape(tokens, heads, d)


def _plain_prompt_parts(s):
    t, h, _ = s["q"].shape
    kv = s["k"].shape[1]
    q, k, v = (_by_kv_head(s[n], kv) for n in ("q", "k", "v"))
    seq, at = _sequence_of(s["first"], t)
    visible = seq[:, None] == seq[None]
    visible = visible & (at[:, None] >= at[None]) if s["causal"] else visible
    p, lse = _softmax(torch.matmul(q, k.transpose(1, 2)) * s["scale"], visible.repeat_interleave(h // kv, 0)[None])
    return q, k, v, p, torch.matmul(p, v), lse


def _plain_prompt(s):
    t, h, _ = s["q"].shape
    return _back(_plain_prompt_parts(s)[4], t, h).to(s["q"].dtype)


def _plain_grad(s):
    t, h, _ = s["q"].shape
    kv, dtype = s["k"].shape[1], s["q"].dtype
    q, k, v, p, o, lse = _plain_prompt_parts(s)
    do = _by_kv_head(s["do"], kv)
    dv = torch.matmul(p.transpose(1, 2), do)
    dp = torch.matmul(do, v.transpose(1, 2))
    ds = p * (dp - (do * o).sum(-1, keepdim=True)) * s["scale"]
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(1, 2), q)
    return {"o": _back(o, t, h).to(dtype), "lse": _back(lse[..., None], t, h)[..., 0].contiguous(), "dq": _back(dq, t, h).to(dtype),
            "dk": _back(dk, t, kv).to(dtype), "dv": _back(dv, t, kv).to(dtype)}


def _turn(x, cos, sin, interleaved):
    x = x.float()
    cos, sin = cos[:, None], sin[:, None]
    half = x.shape[-1] // 2
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    pair = (a * cos - b * sin, b * cos + a * sin)
    return torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1)


def _plain_append(s):
    cache, t = s["cache"], s["k"].shape[0]
    page = cache.k.shape[1]
    seq, at = _sequence_of(s["first"], t)
    at = at + s["lengths"][seq] - (s["first"][1:] - s["first"][:-1])[seq]
    where = s["table"][seq, at // page].long(), at % page
    cos, sin = s["cos"][at], s["sin"][at]
    cache.k[where] = _turn(s["k"], cos, sin, s["interleaved"]).to(cache.k.dtype)
    cache.v[where] = s["v"]
    return {"q": _turn(s["q"], cos, sin, s["interleaved"]).to(s["q"].dtype), "k": cache.k, "v": cache.v}


def _plain_paged(s):
    q, first, lengths, table, cache = s["q"], s["first"], s["lengths"], s["table"], s["cache"]
    (t, h, d), kv, n = q.shape, cache.k.shape[2], table.shape[0]
    g, pages = h // kv, table.clamp(min=0).long()
    k, v = (c[pages].flatten(1, 2).permute(0, 2, 1, 3).float() for c in (cache.k, cache.v))      # [n][kv][longest][d]
    seq, at = _sequence_of(first, t)
    new = first[1:] - first[:-1]
    longest = s["longest"]
    padded = q.new_zeros((n, longest, h, d), dtype=torch.float32)
    padded[seq, at] = q.float()
    rows = padded.view(n, longest, kv, g, d).permute(0, 2, 1, 3, 4).reshape(n, kv, longest * g, d)
    last = (lengths - new)[:, None] + torch.arange(longest, device=q.device)[None]
    visible = torch.arange(k.shape[2], device=q.device)[None, None] <= last[..., None]      # [n][longest][keys]
    p, _ = _softmax(torch.matmul(rows, k.transpose(2, 3)) * s["scale"], visible.repeat_interleave(g, 1)[:, None])
    v = torch.where((torch.arange(v.shape[2], device=q.device)[None] < lengths[:, None])[:, None, :, None], v, torch.zeros_like(v))
    o = torch.matmul(p, v).view(n, kv, longest, g, d).permute(0, 2, 1, 3, 4).reshape(n, longest, h, d)
    return o[seq, at].to(q.dtype)


# ------------------------------------------------------------------ exact ---
def _exact_head(q, k, v, hidden, scale):
    """One head of one sequence in 64 bits: results, weights, log-sums.  hidden: places that a row does not see."""
    if k.shape[0] == 0:
        return torch.zeros_like(q), q.new_zeros((q.shape[0], 0)), q.new_full((q.shape[0],), -math.inf)
    w = torch.mm(q, k.t().contiguous()).mul_(scale).masked_fill_(hidden, -math.inf)
    lse = torch.logsumexp(w, 1)
    w = torch.exp(w - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    return torch.mm(w, v), w, lse


def exact(case, seed):
    s = prepare(case, seed)
    h, kv, d, scale = case["heads"], case["kv"], case["dim"], s["scale"]
    g = h // kv
    if case["kind"] in ("prompt", "grad"):
        q, k, v = (s[n].double() for n in ("q", "k", "v"))
        out = {"o": torch.zeros_like(q), "lse": q.new_zeros(q.shape[:2]), "dq": torch.zeros_like(q), "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)}
        begin = 0
        for n in _numbers(case["lens"]):
            part = slice(begin, begin + n)
            begin += n
            hidden = torch.ones((n, n), dtype=torch.bool, device=DEVICE).triu(1) if case["causal"] else torch.zeros((n, n), dtype=torch.bool, device=DEVICE)
            for i in range(h if n else 0):
                o, w, lse = _exact_head(q[part, i], k[part, i // g], v[part, i // g], hidden, scale)
                out["o"][part, i], out["lse"][part, i] = o, lse
                if case["kind"] == "grad":
                    do = s["do"][part, i].double()
                    out["dv"][part, i // g] += torch.mm(w.t().contiguous(), do)
                    dw = torch.mm(do, v[part, i // g].t().contiguous())
                    dw = w * (dw - (dw * w).sum(1, keepdim=True)) * scale
                    out["dq"][part, i] = torch.mm(dw, k[part, i // g])
                    out["dk"][part, i // g] += torch.mm(dw.t().contiguous(), q[part, i])
        return out if case["kind"] == "grad" else out["o"]
    new, past = _numbers(case["new"]), _numbers(case["past"])
    page, table = case["page"], s["table"].tolist()
    if case["kind"] == "append":
        out = {"q": s["q"].double(), "k": s["cache"].k.double(), "v": s["cache"].v.double()}
        for i, n in enumerate(new):
            begin = sum(new[:i])
            at = torch.arange(past[i], past[i] + n, device=DEVICE)
            turn = torch.complex(s["cos"][at].double(), s["sin"][at].double())[:, None]
            turned = []
            for x in (s["q"][begin:begin + n].double(), s["k"][begin:begin + n].double()):
                x = x if case["interleaved"] else x.unflatten(-1, (2, d // 2)).transpose(-1, -2)
                x = torch.view_as_real(torch.view_as_complex(x.reshape(n, -1, d // 2, 2).contiguous()) * turn)
                turned.append(x.flatten(-2) if case["interleaved"] else x.transpose(-1, -2).flatten(-2))
            out["q"][begin:begin + n] = turned[0]
            where = torch.tensor(table[i], device=DEVICE)[at // page], at % page
            out["k"][where], out["v"][where] = turned[1], s["v"][begin:begin + n].double()
        return out
    out = s["q"].double()
    for i, n in enumerate(new):
        begin, total = sum(new[:i]), new[i] + past[i]
        pages = torch.tensor(table[i][:-(-total // page)], device=DEVICE, dtype=torch.long)
        k, v = (c[pages].flatten(0, 1)[:total].double() for c in (s["cache"].k, s["cache"].v))
        hidden = torch.arange(total, device=DEVICE)[None] > torch.arange(past[i], total, device=DEVICE)[:, None]
        hidden = hidden.repeat_interleave(g, 0)
        for j in range(kv):
            rows = s["q"][begin:begin + n, j * g:(j + 1) * g].double().reshape(n * g, d)
            out[begin:begin + n, j * g:(j + 1) * g] = _exact_head(rows, k[:, j].contiguous(), v[:, j].contiguous(), hidden, scale)[0].view(n, g, d)
    return out


# ------------------------------------------------------------------- work ---
def work(case):
    h, kv, d = case["heads"], case["kv"], case["dim"]
    if case["kind"] in ("prompt", "grad"):
        lens = _numbers(case["lens"])
        t = sum(lens)
        pairs = h * sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lens)
        if case["kind"] == "prompt":
            return {"bytes": 2 * t * d * (2 * h + 2 * kv), "flops": 4 * d * pairs}
        # q, do, o, dq; k, v, dk, dv; the log-sums.  Two products forward, five of the gradient's
        return {"bytes": 2 * t * d * (4 * h + 4 * kv) + 4 * t * h, "flops": 14 * d * pairs}
    new, past = _numbers(case["new"]), _numbers(case["past"])
    t, pages = sum(new), sum(-(-(a + b) // case["page"]) for a, b in zip(new, past))
    if case["kind"] == "append":
        # q, k, v in and out, the rows of both tables
        rows = len({p + i for n, p in zip(new, past) for i in range(n)})
        return {"bytes": 4 * t * d * (h + 2 * kv) + 4 * rows * d, "flops": 3 * t * d * (h + kv)}
    pairs = h * sum(a * b + a * (a + 1) // 2 for a, b in zip(new, past))
    return {"bytes": 4 * t * d * h + 4 * d * kv * sum(a + b for a, b in zip(new, past)) + 4 * pages, "flops": 4 * d * pairs}
