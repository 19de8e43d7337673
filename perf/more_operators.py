"""A cache of 8-bit keys and values and the next token as cases to time: tokens entering the cache and read back, whole sequences read back,
attention of new tokens over it - from one token of one sequence to a chunk of a prompt -, and sampling with temperature,
top-k, top-p and min-p from given random numbers.

`run` goes through the entry points of the package where `own` is true and through the operators' plain forms where it is not: 32-bit torch
operations, 64-bit ones where values lie next to a border (rotary angles before they are rounded to 8 bits, sums of a sampling's weights).  Heads and widths are
those of the repository's 7b, 13b and 70B-shaped workloads (heads of 128 elements) next to smaller and odd ones; lists of lengths are texts, one number per sequence.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
LARGEST = {torch.float16: 1.875 * 2.0 ** 15, torch.bfloat16: 1.875 * 2.0 ** 127}
E4M3 = torch.float8_e4m3fn
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
    many = random.Random(8)
    return [
        # one sequence's next token enters the cache, 13b: launch and latency
        {"name": "append 13b one token", "kind": "append", "new": "1", "past": "700", "heads": 40, "kv": 40, "dim": 128, "page": 16, "rotary": 128,
         "interleaved": False, "dtype": "f16", "fused": False},
        # a batch of prompts enters it and comes back for attention over the prompts, 70B-shaped, q, k and v in one buffer
        {"name": "append 70b 16 prompts", "kind": "append", "new": _ragged(many, 16, 6000), "past": _text([0] * 16), "heads": 64, "kv": 8,
         "dim": 128, "page": 64, "rotary": 128, "interleaved": True, "dtype": "bf16", "fused": True},
        # a short sequence is read back, heads of an odd width
        {"name": "read 12x80 T333", "kind": "read", "lens": "333", "kv": 12, "dim": 80, "page": 16, "dtype": "f16"},
        # a batch of long contexts, an empty one among them, is read back, 70B-shaped
        {"name": "read 70b 16 sequences", "kind": "read", "lens": _ragged(many, 15, 100000) + ",0", "kv": 8, "dim": 128, "page": 64, "dtype": "bf16"},
        # single-stream decoding, 7b
        {"name": "decode 7b one token", "kind": "attn", "new": "1", "past": "2000", "heads": 32, "kv": 32, "dim": 128, "page": 16, "dtype": "f16"},
        # a serving batch, 70B-shaped, contexts of every length
        {"name": "decode 70b x48", "kind": "attn", "new": _text([1] * 48), "past": _ragged(many, 48, 250000), "heads": 64, "kv": 8, "dim": 128, "page": 64,
         "dtype": "bf16"},
        # a chunk of a long prompt next to seven sequences that decode
        {"name": "chunk 512 and singles", "kind": "attn", "new": "512,1,1,1,1,1,1,1", "past": "7700,1,300,4100,950,2047,15,6400", "heads": 32, "kv": 8,
         "dim": 128, "page": 32, "dtype": "f16"},
        # drafts of a few tokens to be verified, 13b
        {"name": "drafts 13b 6x5", "kind": "attn", "new": "5,5,3,5,4,5", "past": "1100,2900,17,640,3333,512", "heads": 40, "kv": 40, "dim": 128, "page": 16,
         "dtype": "bf16"},
        # the next token of one sequence, all filters on: launch and latency
        {"name": "sample 1x32000", "kind": "sample", "rows": 1, "vocab": 32000, "dtype": "f16", "temperature": "0.8", "top_k": "40", "top_p": "0.95", "min_p": "0.05"},
        # a small batch without filters over an odd vocabulary
        {"name": "sample 7x50001 unfiltered", "kind": "sample", "rows": 7, "vocab": 50001, "dtype": "bf16", "temperature": "1.0", "top_k": "", "top_p": "", "min_p": ""},
        # a serving batch with top-p alone: a nucleus of thousands of tokens
        {"name": "sample 48x131071 top-p", "kind": "sample", "rows": 48, "vocab": 131071, "dtype": "f32", "temperature": "1.0", "top_k": "", "top_p": "0.92", "min_p": ""},
        # a large batch in which every request has parameters of its own, greedy ones among them
        {"name": "sample 256x128000 mixed", "kind": "sample", "rows": 256, "vocab": 128000, "dtype": "bf16", "temperature": "0,0.6,0.8,1.0,1.3", "top_k": "0,50,1,1000,20",
         "top_p": "1.0,0.9,0.5", "min_p": "0,0.02"},
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    kind = rng.choice(("append", "append", "read", "read", "attn", "attn", "attn", "attn", "sample", "sample", "sample", "sample"))
    if kind == "sample":
        rows = log_int(1, 256)
        some = lambda values: rng.choice(("", _text(rng.choices(values, k=rng.randint(1, 5)))))      # noqa: E731
        return {"kind": kind, "rows": rows, "vocab": log_int(300, 152000), "dtype": rng.choice(("f16", "bf16", "f32")),
                "temperature": some((0, 0.3, 0.7, 1.0, 1.5)), "top_k": some((0, 1, 7, 50, 300, 3000)), "top_p": some((0.3, 0.8, 0.9, 0.97, 1.0)),
                "min_p": some((0, 0.01, 0.1, 0.5))}
    kv = rng.choice((1, 2, 4, 5, 8, 16, 32, 40))
    heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8, 16) if kv * g <= 64])
    c = {"kind": kind, "kv": kv, "dim": rng.choice((64, 64, 80, 96, 128, 128, 128)), "dtype": rng.choice(("f16", "bf16")), "page": rng.choice((16, 16, 32, 64, 128))}
    n = log_int(1, 48)
    if kind == "read":
        c["lens"] = _ragged(rng, n, log_int(n, 100000 * 8 // max(kv, 8)), rng.choice((0, 1)))
        if not any(_numbers(c["lens"])):
            c["lens"] = _text([1] * n)
        return c
    c["heads"] = heads
    if kind == "append":
        c["interleaved"], c["fused"], c["rotary"] = rng.random() < 0.5, rng.random() < 0.3, rng.choice((c["dim"], c["dim"], c["dim"] // 2))
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
def _starts(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEVICE)


def _two_to(e):
    """2^e in 64 bits, exactly: a power function need not be."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x, dtype):
    """Heads x [...][dim] in 8 bits: elements e4m3, and per head the byte of the power of two that they are in units of, the smallest that holds the largest of them."""
    x = x.clamp(-LARGEST[dtype], LARGEST[dtype])
    m, e = torch.frexp(x.abs().amax(-1))
    e = (e - 9 + (m > 0.875)).clamp(min=-126)      # 448 = 0.875 * 2^9
    return (x * _two_to(-e).to(x.dtype)[..., None]).float().to(E4M3), (e + 127).to(torch.uint8)


def _heads_of_a_cache(gen, shape, spread, dtype):
    """Normal elements, the size of every head of every token its own; in 8 bits."""
    x = torch.empty(shape, dtype=dtype, device=DEVICE).normal_(generator=gen)
    x *= torch.exp(spread * torch.randn(shape[:3], device=DEVICE, generator=gen))[..., None].to(dtype)
    elements, exponents = torch.empty(shape, dtype=torch.uint8, device=DEVICE), torch.empty(shape[:3], dtype=torch.uint8, device=DEVICE)
    for i in range(0, shape[0], 512):
        a, b = _quantise(x[i:i + 512].float(), dtype)
        elements[i:i + 512], exponents[i:i + 512] = a.view(torch.uint8), b
    return elements.view(E4M3), exponents.transpose(1, 2).contiguous()


class _Pages:
    """A cache: elements [pages][page][kv][dim], exponents' bytes [pages][kv][page]."""

    def __init__(self, gen, pages, page, kv, dim, dtype):
        self.k, self.k_exp = _heads_of_a_cache(gen, (pages, page, kv, dim), 0.3, dtype)
        self.v, self.v_exp = _heads_of_a_cache(gen, (pages, page, kv, dim), 0.7, dtype)
        self.dtype = dtype


def _parameter(text, rows, dtype):
    """A request's parameter in every row, some values in turn; none where the text is empty."""
    if not text:
        return None
    values = [float(v) for v in text.split(",")]
    return torch.tensor([values[i % len(values)] for i in range(rows)], device=DEVICE).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    s = {"kind": case["kind"]}
    if case["kind"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        # most tokens far below the likely ones, as a model's logits are
        x = 2.0 * torch.randn((rows, vocab), device=DEVICE, generator=gen)
        x += 4.0 * torch.rand((rows, vocab), device=DEVICE, generator=gen) ** 8
        s["logits"], s["u"] = x.to(dtype), torch.rand(rows, device=DEVICE, generator=gen)
        for name in ("temperature", "top_p", "min_p"):
            s[name] = _parameter(case[name], rows, torch.float32)
        s["top_k"] = _parameter(case["top_k"], rows, torch.int32)
        return s
    kv, dim, page = case["kv"], case["dim"], case["page"]
    if case["kind"] == "read":
        lengths = new = _numbers(case["lens"])
    else:
        new, past = _numbers(case["new"]), _numbers(case["past"])
        lengths = [a + b for a, b in zip(new, past)]
    used = [-(-n // page) for n in lengths]
    pages = sum(used) + 3
    order = torch.randperm(pages, device=DEVICE, generator=gen).to(torch.int32)
    table = torch.full((len(new), max(used) + 1), -1, dtype=torch.int32, device=DEVICE)
    for i, n in enumerate(used):
        table[i, :n] = order[sum(used[:i]):sum(used[:i + 1])]
    s.update(cache=_Pages(gen, pages, page, kv, dim, dtype), table=table, first=_starts(new), lengths=torch.tensor(lengths, dtype=torch.int32, device=DEVICE),
             tokens=sum(new), longest=max(new))
    if case["kind"] == "read":
        return s
    heads, fused = case["heads"], case["kind"] == "append"
    x = torch.randn((sum(new), heads + 2 * kv * fused, dim), device=DEVICE, generator=gen)
    x[:, :heads] *= 2.0      # scores spread like N(0, 2^2): a few keys of a row carry most of it
    x = x.to(dtype)
    if case["kind"] == "attn":
        s["q"], s["scale"] = x, 1.0 / math.sqrt(dim)
        return s
    parts = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    s["q"], s["k"], s["v"] = parts if case["fused"] else (p.contiguous() for p in parts)
    s["interleaved"] = case["interleaved"]
    rate = THETA ** (-torch.arange(0, case["rotary"], 2, device=DEVICE).double() / case["rotary"])
    angle = torch.arange(max(lengths), device=DEVICE).double()[:, None] * rate
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


# -------------------------------------------------------------------- run ---
def run(state):
    s = state
    if own:
        import paper_2602_05367_amd as rb
        if s["kind"] == "sample":
            return rb.rb_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        c = s["cache"]
        cache = rb.Cache8(c.k, c.v, c.k_exp, c.v_exp, c.dtype)
        if s["kind"] == "attn":
            return rb.rb_attn_cache8(cache, s["q"], s["first"], s["lengths"], s["table"], scale=s["scale"])
        out = {}
        if s["kind"] == "append":
            out["q"] = rb.rb_cache8_append(cache, s["k"], s["v"], s["first"], s["lengths"], s["table"], q=s["q"], cos=s["cos"], sin=s["sin"],
                                           interleaved=s["interleaved"])
        out["k"], out["v"] = rb.rb_cache8_read(cache, s["first"], s["lengths"], s["table"], s["tokens"])
        return out
    return {"append": _plain_append, "read": _plain_read, "attn": _plain_attention, "sample": _plain_sample}[s["kind"]](s)


def _places(s):
    """The packed tokens' sequences and positions, and where those lie in the cache: page and place in it."""
    at = torch.arange(s["tokens"], device=DEVICE)
    first, page = s["first"], s["cache"].k.shape[1]
    seq = torch.searchsorted(first[1:].contiguous(), at, right=True)
    position = at - first[seq + 1] + s["lengths"][seq]
    return seq, position, s["table"][seq, position // page].long(), position % page


def _turn(x, cos, sin, interleaved):
    """64 bits: the result is rounded to few bits, and sizes are compared."""
    rotary = 2 * cos.shape[1]
    x, rest = x[..., :rotary].double(), x[..., rotary:].double()
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :rotary // 2], x[..., rotary // 2:])
    pair = (a * cos - b * sin, b * cos + a * sin)
    return torch.cat((torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1), rest), -1)


def _rows(elements, exponents, page, place):
    """Heads of some positions, the values they stand for in 32 bits: [...][kv][dim]"""
    return elements.view(torch.uint8)[page, place].view(E4M3).float() * _two_to(exponents[page, :, place].int() - 127).float()[..., None]


def _plain_append(s):
    cache = s["cache"]
    _, position, page, place = _places(s)
    cos, sin = s["cos"][position], s["sin"][position]
    for x, elements, exponents in ((_turn(s["k"], cos, sin, s["interleaved"]), cache.k, cache.k_exp), (s["v"].float(), cache.v, cache.v_exp)):
        a, b = _quantise(x, cache.dtype)
        elements.view(torch.uint8)[page, place] = a.view(torch.uint8)
        exponents[page, :, place] = b
    return {"q": _turn(s["q"], cos, sin, s["interleaved"]).to(s["q"].dtype), **_plain_read(s)}


def _plain_read(s):
    cache = s["cache"]
    _, _, page, place = _places(s)
    return {"k": _rows(cache.k, cache.k_exp, page, place).to(cache.dtype), "v": _rows(cache.v, cache.v_exp, page, place).to(cache.dtype)}


def _plain_attention(s):
    q, cache, table, lengths = s["q"], s["cache"], s["table"].clamp(min=0).long(), s["lengths"]
    (t, h, d), kv, n, longest = q.shape, cache.k.shape[2], table.shape[0], s["longest"]
    g = h // kv
    keys = torch.arange(table.shape[1] * cache.k.shape[1], device=DEVICE)
    page, place = table[:, keys // cache.k.shape[1]], (keys % cache.k.shape[1])[None].expand(n, -1)
    k, v = (_rows(a, b, page, place).transpose(1, 2) for a, b in ((cache.k, cache.k_exp), (cache.v, cache.v_exp)))      # [n][kv][keys][d]
    v = torch.where((keys[None] < lengths[:, None])[:, None, :, None], v, torch.zeros_like(v))
    seq, position, _, _ = _places(s)
    new = s["first"][1:] - s["first"][:-1]
    rows = q.new_zeros((n, longest, h, d), dtype=torch.float32)
    at = position - (lengths - new)[seq]
    rows[seq, at] = q.float()
    rows = rows.view(n, longest, kv, g, d).permute(0, 2, 1, 3, 4).reshape(n, kv, longest * g, d)
    last = (lengths - new)[:, None] + torch.arange(longest, device=DEVICE)[None]
    visible = (keys[None, None] <= last[..., None]).repeat_interleave(g, 1)[:, None]
    scores = (torch.matmul(rows, k.transpose(2, 3).contiguous()) * s["scale"]).masked_fill(~visible, -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    o = torch.matmul(p / p.sum(-1, keepdim=True), v.contiguous())
    return o.view(n, kv, longest, g, d).permute(0, 2, 1, 3, 4).reshape(n, longest, h, d)[seq, at].to(q.dtype)


def _plain_sample(s):
    x = s["logits"].double()
    rows, vocab = x.shape

    def of(name, default):
        return (torch.full((rows,), default, device=DEVICE) if s[name] is None else s[name]).double()[:, None]

    temperature, top_k, top_p, min_p = of("temperature", 1.0), of("top_k", 0.0), of("top_p", 1.0), of("min_p", 0.0)
    down, order = torch.sort(x, descending=True, stable=True)      # equal ones: the lowest index first
    greedy = temperature <= 0
    w = torch.exp((down - down[:, :1]) / torch.where(greedy, torch.ones_like(temperature), temperature))
    rank = torch.arange(vocab, device=DEVICE)[None]
    kept = (rank < torch.where(top_k > 0, top_k, vocab)) & (~greedy | (rank == 0))
    w = torch.where(kept, w, torch.zeros_like(w))
    before = torch.cumsum(w, 1) - w
    kept = kept & ((before < top_p * w.sum(1, keepdim=True)) | (top_p >= 1) | (rank == 0)) & (w >= min_p)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, torch.zeros_like(w)))
    upto = torch.cumsum(w, 1)
    return (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1).to(torch.int32)


# ------------------------------------------------------------------ exact ---
def _value(elements, exponents):
    return elements.double() * _two_to(exponents.int() - 127)[..., None]


def _rounded(x):
    """Heads in 64 bits as e4m3 times the head's power of two holds them: four bits of each element, or the smallest element's step."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True) / 448)
    unit = torch.where(m == 0.5, e - 1, e).clamp(min=-126)
    _, e = torch.frexp(x)
    step = _two_to(torch.maximum(e - 4, unit - 9))
    return torch.round(x / step) * step


def exact(case, seed):
    if case["kind"] == "sample":
        return None
    s = prepare(case, seed)
    cache, page, table, lengths, starts = s["cache"], case["page"], s["table"].tolist(), s["lengths"].tolist(), s["first"].tolist()
    kv, d = case["kv"], case["dim"]

    def positions(i, begin, end):
        at = torch.arange(begin, end, device=DEVICE)
        return torch.tensor(table[i], device=DEVICE)[at // page], at % page

    def whole(i, end):
        pages = torch.tensor(table[i][:-(-end // page)], device=DEVICE, dtype=torch.long)
        return [_value(a.view(torch.uint8)[pages].view(E4M3).flatten(0, 1), b[pages].transpose(1, 2).flatten(0, 1))[:end]
                for a, b in ((cache.k, cache.k_exp), (cache.v, cache.v_exp))]

    if case["kind"] == "read":
        out = [whole(i, n) for i, n in enumerate(lengths) if n]
        return {"k": torch.cat([k for k, _ in out]), "v": torch.cat([v for _, v in out])}
    if case["kind"] == "append":
        out, rotary = {n: s[n].double() for n in ("q", "k", "v")}, case["rotary"]
        for i, n in enumerate(lengths):
            part = slice(starts[i], starts[i + 1])
            at = slice(n - (starts[i + 1] - starts[i]), n)
            turn = torch.complex(s["cos"][at].double(), s["sin"][at].double())[:, None]
            for name in ("q", "k"):
                x = out[name][part]
                y = x[..., :rotary] if case["interleaved"] else x[..., :rotary].unflatten(-1, (2, rotary // 2)).transpose(-1, -2)
                y = torch.view_as_real(torch.view_as_complex(y.reshape(*x.shape[:2], rotary // 2, 2).contiguous()) * turn)
                x[..., :rotary] = y.flatten(-2) if case["interleaved"] else y.transpose(-1, -2).flatten(-2)
        return {"q": out["q"], "k": _rounded(out["k"]), "v": _rounded(out["v"])}
    h, scale = case["heads"], s["scale"]
    g, out = h // kv, s["q"].double()
    for i, total in enumerate(lengths):
        n = starts[i + 1] - starts[i]
        part = slice(starts[i], starts[i + 1])
        k, v = whole(i, total)
        hidden = (torch.arange(total, device=DEVICE)[None] > torch.arange(total - n, total, device=DEVICE)[:, None]).repeat_interleave(g, 0)
        for j in range(kv):
            rows = s["q"][part, j * g:(j + 1) * g].double().reshape(n * g, d)
            p = torch.softmax(torch.mm(rows, k[:, j].t().contiguous()).mul_(scale).masked_fill_(hidden, -math.inf), 1)
            out[part, j * g:(j + 1) * g] = torch.mm(p, v[:, j].contiguous()).view(n, g, d)
    return out


# ------------------------------------------------------------------- work ---
def work(case):
    if case["kind"] == "sample":
        # every logit once, the random number, the token and the parameters; a difference, an exponential, two sums of each
        n = case["rows"] * case["vocab"]
        given = 2 + sum(bool(case[p]) for p in ("temperature", "top_k", "top_p", "min_p"))
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + 4 * given * case["rows"], "flops": 4 * n}
    kv, d = case["kv"], case["dim"]
    if case["kind"] == "read":
        t = sum(_numbers(case["lens"]))
        return {"bytes": 2 * t * kv * (3 * d + 1), "flops": 2 * t * kv * d}
    new, past = _numbers(case["new"]), _numbers(case["past"])
    t, h = sum(new), case["heads"]
    if case["kind"] == "append":
        # q, k, v in, q out, the cache's new heads out and in again, k and v back; the rows of both tables
        rows = len({p + i for n, p in zip(new, past) for i in range(n)})
        return {"bytes": 4 * t * d * h + 4 * t * kv * d + 4 * t * kv * (d + 1) + 4 * t * kv * d + 4 * rows * case["rotary"], "flops": 3 * t * d * (h + kv) + 6 * t * kv * d}
    pairs = h * sum(a * b + a * (a + 1) // 2 for a, b in zip(new, past))
    pages = sum(-(-(a + b) // case["page"]) for a, b in zip(new, past))
    return {"bytes": 4 * t * d * h + 2 * (d + 1) * kv * sum(a + b for a, b in zip(new, past)) + 4 * pages, "flops": 4 * d * pairs}
