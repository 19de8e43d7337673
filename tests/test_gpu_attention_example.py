"""The example: decoder blocks over a shared cache give the same whichever way the tokens come in, and the training step's
gradients are those of 64-bit automatic differentiation through the effective weights."""
import importlib.util
import os

import pytest
import torch

import paper_2602_05367_amd as rb

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("attention_example", os.path.join(ROOT, "examples", "attention.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_serving_does_not_depend_on_how_tokens_come_in():
    ex = _example()
    torch.manual_seed(1)
    make = lambda: ex.Blocks(blocks=2, heads=8, kv_heads=2, dim=64, ffn=1376, pages=40, page_tokens=16, positions=256, seed=3)
    inputs = [torch.randn(n, 512, device="cuda").half() for n in (90, 17, 141)]
    whole = ex.serve(make(), inputs, [(90, 17, 141)])
    parts = ex.serve(make(), inputs, [(60, 0, 1), (1, 9, 100), (20, 1, 0), (1, 1, 33)] + [(1, 1, 1)] * 6 + [(2, 0, 1)])
    for a, b in zip(whole, parts):
        # every op of a block rounds its fp16 result (2^-11 each, some twenty of them); other kernels for other numbers of tokens round elsewhere
        rel = float((a.double() - b.double()).norm() / a.double().norm())
        assert a.shape == b.shape and torch.isfinite(a).all() and rel < 20 * 2.0 ** -11, rel


def test_training_step_against_automatic_differentiation():
    ex = _example()
    torch.manual_seed(2)
    lens, inn, heads, kv, dim = (130, 45), 256, 4, 2, 64
    t = sum(lens)
    X = torch.randn(t, inn, device="cuda").half()
    weights = [torch.randn(n * dim, inn, device="cuda") * 0.06 for n in (heads, kv, kv)]
    scales = [((0.22 + 0.01 * torch.randn(2, W.shape[0], device="cuda")).half(), (0.22 + 0.01 * torch.randn(2, inn, device="cuda")).half()) for W in weights]
    go = torch.randn(t, heads, dim, device="cuda").half()
    o, grads = ex.train_step(weights, scales, X, go, lens, heads, kv)
    torch.cuda.synchronize()
    # the same in 64 bits on the CPU: effective weights, attention per sequence and head, gradients of sum(go * o)
    effective = []
    for W, (g, h) in zip(weights, scales):
        packed = rb.rb_couple(W, g, h)[0].cpu()
        bits = (packed[..., None] >> torch.arange(32)) & 1
        signs = 1.0 - 2.0 * bits.reshape(2, W.shape[0], inn).double()
        effective.append((g.double().cpu()[:, :, None] * signs * h.double().cpu()[:, None, :]).sum(0).requires_grad_())
    x = X.double().cpu()
    q, k, v = ((x @ W.t()).view(t, -1, dim) for W in effective)
    parts, begin = [], 0
    for n in lens:
        s = slice(begin, begin + n)
        begin += n
        K, V = (y[s].repeat_interleave(heads // kv, 1).transpose(0, 1) for y in (k, v))
        w = (q[s].transpose(0, 1) @ K.transpose(1, 2)) * dim ** -0.5
        w = w.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), float("-inf")).softmax(-1)
        parts.append((w @ V).transpose(0, 1))
    ref = torch.cat(parts)
    (ref * go.double().cpu()).sum().backward()
    assert float((o.double().cpu() - ref.detach()).norm() / ref.detach().norm()) < 2e-3
    for (G, _, _), W in zip(grads, effective):
        # q, k, v, dq, dk and dv are fp16, each rounded once (2^-11), weights and score gradients once more
        assert float((G.double().cpu() - W.grad).norm() / W.grad.norm()) < 8 * 2.0 ** -11
