"""Attention between residual-binary layers, the two ways it is used.

serve(): decoder blocks (Llama-shaped: normalisation, q, k, v, rotary embedding, cache, attention, o, residual, feed-forward
part) over a batch of sequences that share a paged cache.  A step takes any mix of new tokens per sequence: prompts at once, a chunk of
one beside others that decode, single tokens.  The cache holds 16 bits an element, or 8 (in_8_bits).

generate(): prompts in, tokens out: embedding, the blocks, an output head of the same kind of layer in fp32, and the next token
of every sequence drawn with its own temperature, top-k, top-p and min-p; nothing goes through the host on the way.

train_step(): the projections in front of attention in training: cores derived from the shared weights, results, gradients
through attention, and from them those of the weights and scales.

The embedding, the random numbers and the optimiser are the program's own.

    python examples/attention.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2602_05367_amd as rb

EPS = 1e-5


def rotary_tables(positions: int, dim: int, theta: float = 10000.0, device="cuda"):
    """cos, sin fp32 [positions][dim / 2] of the angles position * theta^(-2 i / dim)."""
    rate = theta ** (-torch.arange(0, dim, 2, device=device, dtype=torch.float64) / dim)
    angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def random_layer(gen, out: int, inn: int, K: int = 2, rms: float = 1.0) -> rb.Layer:
    """A frozen layer from a Gaussian weight; inputs of RMS 1 give outputs of RMS about `rms`."""
    device = gen.device
    W = torch.randn((out, inn), device=device, generator=gen) * 0.02
    a = torch.tensor((0.016, 0.0097, 0.0058)[:K], device=device).sqrt()[:, None]
    g, h = a.expand(K, out).contiguous().half(), a.expand(K, inn).contiguous().half()
    _, native, _ = rb.rb_couple(W, g, h)
    return rb.Layer(native, (g.float() * (rms / (0.02 * math.sqrt(inn * 0.76)))).half(), h, K, out, inn)


class Blocks:
    """Decoder blocks with a cache each and one page table for all."""

    def __init__(self, blocks: int, heads: int, kv_heads: int, dim: int, ffn: int, pages: int, page_tokens: int, positions: int, seed: int = 0,
                 in_8_bits: bool = False):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        d = heads * dim
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.cos, self.sin = rotary_tables(positions, dim)
        self.append, self.attention = (rb.rb_cache8_append, rb.rb_attn_cache8) if in_8_bits else (rb.rb_cache_append, rb.rb_attn_paged)
        make = rb.Cache8.zeros if in_8_bits else rb.Cache.zeros
        self.blocks = []
        for _ in range(blocks):
            shapes = {"q": (d, d), "k": (kv_heads * dim, d), "v": (kv_heads * dim, d), "o": (d, d), "gate": (ffn, d), "up": (ffn, d), "down": (d, ffn)}
            layers = {n: random_layer(gen, out, inn) for n, (out, inn) in shapes.items()}
            norms = [(1 + 0.1 * torch.randn(d, device="cuda", generator=gen)).half() for _ in range(2)]
            self.blocks.append((layers, norms, make(pages, page_tokens, kv_heads, dim)))

    def step(self, x, first, lengths, table):
        """New tokens x fp16 [tokens][d] of packed sequences (first), which are the last of `lengths` positions each."""
        t = x.shape[0]
        for layers, norms, cache in self.blocks:
            n = rb.rb_rmsnorm(x, norms[0], EPS)
            q, k, v = (rb.rb_linear_gemm(layers[m], n).view(t, -1, self.dim) for m in ("q", "k", "v"))
            q = self.append(cache, k, v, first, lengths, table, q=q, cos=self.cos, sin=self.sin)
            o = self.attention(cache, q, first, lengths, table)
            x = rb.rb_add(rb.rb_linear_gemm(layers["o"], o.view(t, -1)), x)
            n = rb.rb_rmsnorm(x, norms[1], EPS)
            a = rb.rb_silu_mul(rb.rb_linear_gemm(layers["gate"], n), rb.rb_linear_gemm(layers["up"], n))
            x = rb.rb_add(rb.rb_linear_gemm(layers["down"], a), x)
        return x


def _starts(new):
    return torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")


def _table(used):
    """A page table int32 [sequences][most of `used`]: pages of a sequence need not follow each other."""
    table = torch.zeros((len(used), max(used)), dtype=torch.int32)
    for i, n in enumerate(used):
        table[i, :n] = torch.arange(n) * len(used) + i
    return table.cuda()


def serve(model: Blocks, inputs, chunks):
    """inputs: one fp16 tensor [length][d] per sequence.  chunks: per step, how many tokens of each sequence are new.
    Returns the blocks' results, one tensor per sequence."""
    page = model.blocks[0][2].k.shape[1]
    table, done, out = _table([-(-x.shape[0] // page) for x in inputs]), [0] * len(inputs), [[] for _ in inputs]
    for new in chunks:
        x = torch.cat([s[p:p + n] for s, p, n in zip(inputs, done, new)])
        done = [p + n for p, n in zip(done, new)]
        lengths = torch.tensor(done, dtype=torch.int32, device="cuda")
        y = model.step(x, _starts(new), lengths, table).split(list(new))
        for o, part in zip(out, y):
            o.append(part)
    return [torch.cat(o) for o in out]


def generate(model: Blocks, embedding, norm, head: rb.Layer, prompts, new: int, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """prompts: one int64 tensor of tokens per sequence; u fp32 [new][sequences] in [0, 1); the others one number per sequence, or None.
    Returns the tokens int32 [new][sequences] that follow."""
    page = model.blocks[0][2].k.shape[1]
    table = _table([-(-(p.shape[0] + new) // page) for p in prompts])
    first = _starts([p.shape[0] for p in prompts])
    lengths, x, tokens = first.diff(), embedding[torch.cat(list(prompts))], []
    for i in range(new):
        y = model.step(x, first, lengths, table)
        logits = rb.rb_linear_gemm(head, rb.rb_rmsnorm(y[first[1:] - 1], norm, EPS), out_dtype=torch.float32)
        tokens.append(rb.rb_sample(logits, u[i], temperature, top_k, top_p, min_p))
        x, first, lengths = embedding[tokens[-1]], torch.arange(len(prompts) + 1, dtype=torch.int32, device="cuda"), lengths + 1
    return torch.stack(tokens)


def train_step(weights, scales, X, go, lens, heads: int, kv_heads: int):
    """weights: fp32 Wq, Wk, Wv; scales: fp16 (g [K][out], h [K][in]) of each; X fp16 [tokens][in]; go: the gradient of attention's
    result.  Returns that result and, per projection, the gradients of its weight, its g and its h."""
    first, t, dim = _starts(lens), X.shape[0], weights[0].shape[0] // heads
    cores = [rb.rb_couple(W, g, h) for W, (g, h) in zip(weights, scales)]
    layers = [rb.Layer(native, g, h, g.shape[0], *W.shape) for (_, native, _), W, (g, h) in zip(cores, weights, scales)]
    q, k, v = (rb.rb_linear_gemm(layer, X).view(t, n, dim) for layer, n in zip(layers, (heads, kv_heads, kv_heads)))
    o, lse = rb.rb_attn_prompt(q, k, v, first, want_lse=True)
    grads = []
    for d, (packed, _, _), (g, h) in zip(rb.rb_attn_prompt_grad(go, q, k, v, o, lse, first), cores, scales):
        G = rb.rb_weight_grad(d.view(t, -1), X)
        grads.append((G, *rb.rb_scale_grads(G, packed, g, h)))
    return o, grads


def main():
    torch.manual_seed(0)
    heads, kv_heads, dim = 32, 8, 128
    model = Blocks(blocks=2, heads=heads, kv_heads=kv_heads, dim=dim, ffn=11008, pages=64, page_tokens=16, positions=512)
    inputs = [torch.randn(n, heads * dim, device="cuda").half() for n in (180, 33, 97)]
    # two prompts at once; the third in two chunks beside the others' next tokens; then single tokens
    chunks = [(170, 23, 0), (1, 1, 60), (1, 1, 29)] + [(1, 1, 1)] * 8
    out = serve(model, inputs, chunks)
    torch.cuda.synchronize()
    print("served", [tuple(o.shape) for o in out], "rms", [round(float(o.float().square().mean().sqrt()), 3) for o in out])

    model = Blocks(blocks=2, heads=heads, kv_heads=kv_heads, dim=dim, ffn=11008, pages=64, page_tokens=16, positions=512, in_8_bits=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    embedding = torch.randn(32000, heads * dim, device="cuda", generator=gen).half()
    head, norm = random_layer(gen, 32000, heads * dim, rms=4.0), torch.ones(heads * dim, device="cuda").half()
    prompts = [torch.randint(32000, (n,), device="cuda", generator=gen) for n in (180, 33, 97)]
    each = lambda *x: torch.tensor(x, device="cuda")
    tokens = generate(model, embedding, norm, head, prompts, 16, torch.rand((16, 3), device="cuda", generator=gen), temperature=each(0.0, 0.8, 1.0),
                      top_k=each(0, 50, 0).int(), top_p=each(1.0, 0.95, 0.9), min_p=each(0.0, 0.0, 0.05))
    torch.cuda.synchronize()
    print("generated", tokens.t().tolist())

    lens, inn = (300, 77), 1024
    X = torch.randn(sum(lens), inn, device="cuda").half()
    weights = [torch.randn(n * 64, inn, device="cuda") * 0.02 for n in (8, 2, 2)]
    scales = [(torch.full((2, W.shape[0]), 0.126, device="cuda").half(), torch.full((2, inn), 0.126, device="cuda").half()) for W in weights]
    go = (0.01 * torch.randn(sum(lens), 8, 64, device="cuda")).half()
    o, grads = train_step(weights, scales, X, go, lens, 8, 2)
    torch.cuda.synchronize()
    print("trained", tuple(o.shape), "gradients", [tuple(G.shape) for G, _, _ in grads])


if __name__ == "__main__":
    main()
