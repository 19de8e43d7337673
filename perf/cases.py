"""The work that this library is used for, as cases to time: single calls of a layer, prepared stacks
and decoder blocks, a prompt through decoder blocks, one training step of a layer and its
initialisation, each through the public entry points of the package.

Sizes are those of the paper's models as the repository's workloads use them (`synth.LLAMA_SHAPES`,
`synth.prefill_shapes`), next to ragged ones; `draw` covers the ranges in between.  Layers are what
training leaves behind: the paths are derived on the device from a Gaussian weight
(`rb_couple`), so the second path is the binarised residual of the first and padding is as the library
writes it; the scales are those that the derivation gives for N(0, 0.02^2) weights, with a constant
folded into g that brings outputs of RMS-1 inputs to RMS 1.  Activations of single layers are N(0, 1) with one channel in a hundred
times 20.
"""
import math

import torch

import paper_2602_05367_amd as rb
import synth

DEVICE = "cuda"
PATH_SCALES = (0.0160, 0.0097, 0.0058)     # g_k h_k of the paths of a N(0, 0.02^2) weight
KEPT = {2: 0.7585, 3: 0.837}               # |W_hat|^2 / |W|^2 of such layers, measured on long chains
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
DTYPES = {"f16": F16, "bf16": BF16, "f32": F32}


# ------------------------------------------------------------------ cases ---
def listed():
    d7, f7, n7 = synth.LLAMA_SHAPES["7b"]
    d13, f13, _ = synth.LLAMA_SHAPES["13b"]
    return [
        # one token through one small layer, nothing prepared: launches and host work
        {"name": "gemv 2048x2048", "kind": "linear", "K": 2, "out": 2048, "inn": 2048, "T": 1, "act": "f16", "res": "f16"},
        # a handful of tokens (a small serving batch, a speculative draft) through one ragged layer
        {"name": "linear 10999x4128 T7", "kind": "linear", "K": 2, "out": 10999, "inn": 4128, "T": 7, "act": "bf16", "res": "f32"},
        # the three-path variant, a batch of 16
        {"name": "linear K3 4096x11008 T16", "kind": "linear", "K": 3, "out": 4096, "inn": 11008, "T": 16, "act": "f16", "res": "f16"},
        # prefill of a long prompt, the largest matrix
        {"name": "linear 28672x8192 T2048", "kind": "linear", "K": 2, "out": 28672, "inn": 8192, "T": 2048, "act": "bf16", "res": "f16"},
        # single-stream decoding, the whole stack prepared once: the headline workload
        {"name": "chain 7b T1", "kind": "chain", "K": 2, "d": d7, "f": f7, "blocks": n7, "T": 1},
        # a serving batch of 16 in step through the same stack
        {"name": "chain 7b T16", "kind": "chain", "K": 2, "d": d7, "f": f7, "blocks": n7, "T": 16},
        # three paths, six sequences, wider layers
        {"name": "chain 13b K3 T6", "kind": "chain", "K": 3, "d": d13, "f": f13, "blocks": 8, "T": 6},
        # decoder blocks with their normalisations and residuals, three sequences in step
        {"name": "blocks 7b T3", "kind": "blocks", "K": 2, "d": d7, "f": f7, "blocks": n7, "T": 3},
        # a ragged prompt through decoder blocks, op by op
        {"name": "prompt 7b T333", "kind": "prompt", "K": 2, "d": d7, "f": f7, "blocks": 2, "T": 333},
        # one training step of a layer: derive the cores, forward, gradients
        {"name": "train 4096x11008 N512", "kind": "train", "K": 2, "out": 4096, "inn": 11008, "T": 512},
        # initialisation of the same layer, five sweeps
        {"name": "derive 4096x11008", "kind": "derive", "K": 2, "out": 4096, "inn": 11008, "sweeps": 5},
    ]


def draw(rng):
    def log_int(lo, hi, step=1):
        return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))) / step) * step))

    kind = rng.choice(("linear", "linear", "linear", "chain", "chain", "blocks", "prompt", "train", "derive"))
    K = rng.choice((2, 2, 3))
    if kind == "linear":
        T = rng.choice((1, log_int(2, 32), log_int(33, 2048), log_int(1, 2048)))
        c = {"kind": kind, "K": K, "out": log_int(256, 28672), "inn": log_int(256, 28672, 32), "T": T,
             "act": rng.choice(("f16", "bf16")), "res": rng.choice(("f16", "bf16", "f32"))}
        while c["out"] * c["inn"] * K > 2 * 28672 * 8192:
            c["out"] = c["out"] // 2 + 1
        return c
    if kind in ("chain", "blocks", "prompt"):
        d = log_int(1024, 5120, 64)
        f = int(d * rng.uniform(2.0, 4.0) / 64) * 64
        if kind == "blocks":
            T = rng.randint(1, 4) if K == 2 else 1
        elif kind == "chain":
            T = rng.choice((1, rng.randint(2, 16)))
        else:
            T = log_int(17, 1024)
        c = {"kind": kind, "K": K, "d": d, "f": f, "blocks": log_int(1, 32) if kind != "prompt" else rng.randint(1, 2), "T": T}
        while c["blocks"] > 1 and K * c["blocks"] * (4 * d * d + 3 * d * f) > 2 * 32 * (4 * 4096 ** 2 + 3 * 4096 * 11008):
            c["blocks"] -= 1
        return c
    c = {"kind": kind, "K": K, "out": log_int(512, 11008), "inn": log_int(512, 11008, 32)}
    while c["out"] * c["inn"] > 4096 * 11008:
        c["out"] = c["out"] // 2 + 1
    if kind == "train":
        c["T"] = log_int(33, 512)
    else:
        c["sweeps"] = rng.randint(1, 5) if K == 2 else rng.randint(1, 3)
    return c


# ----------------------------------------------------------------- inputs ---
def _randn(gen, *shape):
    return torch.randn(shape, device=DEVICE, generator=gen)


def _activations(gen, T, n, dtype=F16):
    x = _randn(gen, T, n)
    ch = torch.randperm(n, device=DEVICE, generator=gen)[: -(-n // 100)]
    x[:, ch] *= 20.0
    return x.to(dtype)


def _scales(gen, K, out, inn, gain):
    """fp16 g [K][out], h [K][inn]: nearly constant g_k h_k with 1 % jitter, `gain` folded into g."""
    a = torch.tensor(PATH_SCALES[:K], device=DEVICE).sqrt()[:, None]
    return (a * gain * (1 + 0.01 * _randn(gen, K, out))).half(), (a * (1 + 0.01 * _randn(gen, K, inn))).half()


def _layer(gen, K, out, inn, rms=1.0):
    W = _randn(gen, out, inn) * 0.02
    g, h = _scales(gen, K, out, inn, 1.0)
    _, native, _ = rb.rb_couple(W, g, h)
    # inputs of variance 1 give outputs of variance inn * E[W_hat^2]; a chain of a hundred ops stays
    # in fp16's range only if this is right to a percent
    c = rms / (0.02 * math.sqrt(inn * KEPT[K]))
    return rb.Layer(native, (g.float() * c).half(), h, K, out, inn)


def _arena(T, widths):
    """Buffers [T][width] as parts of one tensor, each at a multiple of 64 elements."""
    starts, n = [], 0
    for w in widths:
        starts.append(n)
        n += -(-T * w // 64) * 64
    whole = torch.zeros(n, dtype=F16, device=DEVICE)
    return whole, [whole[s:s + T * w].view(T, w) for s, w in zip(starts, widths)]


def _prepare_chain(case, gen):
    """q, k, v read x; o reads v; gate, up read o; down reads gate; the next block reads down."""
    T, K, d, f = case["T"], case["K"], case["d"], case["f"]
    layers, ops, widths, x = [], [], [], -1
    for _ in range(case["blocks"]):
        b = len(widths)
        for out, inn, src in ((d, d, x), (d, d, x), (d, d, x), (d, d, b + 2), (f, d, b + 3), (f, d, b + 3), (d, f, b + 4)):
            ops.append((len(layers), src + 1, len(widths) + 1))
            layers.append(_layer(gen, K, out, inn))
            widths.append(out)
        x = b + 6
    outputs, bufs = _arena(T, widths)
    x0 = (_randn(gen, T, d)).half()
    stack = rb.Stack(layers, ops, [x0] + bufs, T)
    stack.prepare()
    return {"stack": stack, "outputs": outputs}


def _prepare_blocks(case, gen):
    """The same layers with normalised inputs of q, k, v and gate, up, silu(gate) * up and both
    residual additions; every op writes a buffer of its own."""
    T, K, d, f = case["T"], case["K"], case["d"], case["f"]
    layers, norms, ops, widths, x = [], [], [], [], 0
    for _ in range(case["blocks"]):
        n1, b, l = len(norms), len(widths) + 1, len(layers)
        norms += [(1 + 0.1 * _randn(gen, d)).half() for _ in range(2)]
        for out, inn, rms in ((d, d, 1.0), (d, d, 1.0), (d, d, 1.0), (d, d, 1.0), (f, d, 1.0), (f, d, 1.0), (d, f, 2.0)):
            layers.append(_layer(gen, K, out, inn, rms))
        ops += [(l, x, b, n1, rb.RB_EPI_NONE, -1), (l + 1, x, b + 1, n1, rb.RB_EPI_NONE, -1),
                (l + 2, x, b + 2, n1, rb.RB_EPI_NONE, -1), (l + 3, b + 2, b + 3, -1, rb.RB_EPI_ADD, x),
                (l + 4, b + 3, b + 4, n1 + 1, rb.RB_EPI_SILU_MUL, l + 5), (l + 6, b + 4, b + 5, -1, rb.RB_EPI_ADD, b + 3)]
        widths += [d, d, d, d, f, d]
        x = b + 5
    outputs, bufs = _arena(T, widths)
    x0 = (_randn(gen, T, d)).half()
    block = rb.Block(layers, norms, 1e-5, ops, [x0] + bufs, T)
    block.prepare()
    return {"stack": block, "outputs": outputs}


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind, K = case["kind"], case["K"]
    if kind == "linear":
        X = _activations(gen, case["T"], case["inn"], DTYPES[case["act"]])
        state = {"layer": _layer(gen, K, case["out"], case["inn"]), "res": DTYPES[case["res"]]}
        state["X"] = X[0].clone() if _is_gemv(case) else X
    elif kind == "chain":
        state = _prepare_chain(case, gen)
    elif kind == "blocks":
        state = _prepare_blocks(case, gen)
    elif kind == "prompt":
        d, f = case["d"], case["f"]
        state = {"x": _randn(gen, case["T"], d).half(), "blocks": []}
        for _ in range(case["blocks"]):
            shapes = ((d, d, 1.0), (d, d, 1.0), (d, d, 1.0), (d, d, 1.0), (f, d, 1.0), (f, d, 1.0), (d, f, 2.0))
            state["blocks"].append(([_layer(gen, K, o, i, r) for o, i, r in shapes],
                                    [(1 + 0.1 * _randn(gen, d)).half() for _ in range(2)]))
    elif kind == "train":
        g, h = _scales(gen, K, case["out"], case["inn"], 1.0)
        state = {"W": _randn(gen, case["out"], case["inn"]) * 0.02, "g": g, "h": h,
                 "X": _activations(gen, case["T"], case["inn"]), "Delta": (_randn(gen, case["T"], case["out"]) * 0.01).half()}
    else:
        # channel statistics as the preconditioning uses them: positive, spread over a factor of a few
        row = torch.exp(-0.3 * _randn(gen, case["out"]).abs()).double()
        col = torch.exp(-0.3 * _randn(gen, case["inn"]).abs()).double()
        state = {"W": _randn(gen, case["out"], case["inn"]) * 0.02, "row": row, "col": col, "K": K, "sweeps": case["sweeps"]}
    state["kind"] = kind
    return state


def _is_gemv(case):
    return case["T"] == 1 and case["act"] == "f16" and case["res"] == "f16"


# -------------------------------------------------------------------- run ---
def run(state):
    kind = state["kind"]
    if kind == "linear":
        if state["X"].dim() == 1:
            return rb.rb_linear_gemv(state["layer"], state["X"])
        return rb.rb_linear_gemm(state["layer"], state["X"], out_dtype=state["res"])
    if kind in ("chain", "blocks"):
        state["stack"].run_prepared()
        return state["outputs"]
    if kind == "prompt":
        x, kv = state["x"], []
        for layers, norms in state["blocks"]:
            q, k, v, o, gate, up, down = layers
            n = rb.rb_rmsnorm(x, norms[0], 1e-5)
            kv += [rb.rb_linear_gemm(m, n) for m in (q, k, v)]      # the linear layers alone, without attention: o reads v
            x = rb.rb_add(rb.rb_linear_gemm(o, kv[-1]), x)
            n = rb.rb_rmsnorm(x, norms[1], 1e-5)
            a = rb.rb_silu_mul(rb.rb_linear_gemm(gate, n), rb.rb_linear_gemm(up, n))
            x = rb.rb_add(rb.rb_linear_gemm(down, a), x)
        return {"x": x, "qkv": kv}
    if kind == "train":
        W, g, h = state["W"], state["g"], state["h"]
        packed, native, _ = rb.rb_couple(W, g, h)
        Y = rb.rb_linear_gemm(rb.Layer(native, g, h, g.shape[0], *W.shape), state["X"])
        G = rb.rb_weight_grad(state["Delta"], state["X"])
        grad_g, grad_h = rb.rb_scale_grads(G, packed, g, h)
        return {"packed": packed, "Y": Y, "G": G, "grad_g": grad_g, "grad_h": grad_h}
    packed, g, h, err = rb.rb_derive_iterative(state["W"], state["K"], state["sweeps"], state["row"], state["col"])
    return {"packed": packed, "g": g, "h": h, "err": err}


# --------------------------------------------------------- work, tolerance ---
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def _layer_bytes(K, out, inn):
    return K * out * inn // 8 + 2 * K * (out + inn)


def work(case):
    kind, K = case["kind"], case["K"]
    if kind == "linear":
        out, inn, T = case["out"], case["inn"], case["T"]
        return {"bytes": _layer_bytes(K, out, inn) + T * (inn * _SIZE[case["act"]] + out * _SIZE[case["res"]]),
                "flops": 2 * out * inn * T}
    if kind in ("chain", "blocks", "prompt"):
        d, f, T, n = case["d"], case["f"], case["T"], case["blocks"]
        weights = 4 * _layer_bytes(K, d, d) + 2 * _layer_bytes(K, f, d) + _layer_bytes(K, d, f)
        stored = {"chain": 5 * d + 2 * f, "blocks": 5 * d + f, "prompt": 3 * d}[kind]
        return {"bytes": n * (weights + 2 * T * stored) + 2 * T * d, "flops": 2 * n * T * (4 * d * d + 3 * d * f)}
    out, inn = case["out"], case["inn"]
    if kind == "train":
        T = case["T"]
        # W in, the cores and G out; X, Delta and Y once
        return {"bytes": 8 * out * inn + K * out * inn // 8 + 2 * T * (inn + 2 * out), "flops": 4 * out * inn * T}
    # W in and the cores out.  Every SVID step is a power iteration, two matrix-vector products at
    # least; their operations are not bounded below by anything this file could state
    return {"bytes": 4 * out * inn + K * out * inn // 8, "flops": case["sweeps"] * K * 4 * out * inn}


def tolerance(case):
    """About four times what the path differs by from the same computation in 64 bits (every stored
    fp16 value rounded where the library rounds it); errors of a chain grow with the root of its length."""
    kind = case["kind"]
    if kind == "linear":
        # fp16 results 2.1e-4 to 4.3e-4 (the larger: many tokens, effective weights in fp16), bf16 results 1.7e-3
        return {"rel": 7e-3, "max": 1.6e-2} if case["res"] == "bf16" else {"rel": 1.7e-3, "max": 8.5e-3}
    if kind == "train":
        return {"rel": 1.6e-3, "max": 8e-3, "differ": 0.0}      # Y in fp16; G and the gradients 4e-7
    if kind == "derive":
        return {"rel": 1e-9, "max": 1e-8, "differ": 1e-6}       # fp64, the iteration stops at changes of 1e-10
    depth = math.sqrt(case["blocks"])
    # measured: 2.3e-3 and 2.5e-3 over 32 blocks, 1.2e-3 over 2 blocks of the many-token kernel
    rel, most = {"chain": (1.6e-3, 1.25e-2), "blocks": (1.8e-3, 2.1e-2), "prompt": (3.5e-3, 1.8e-2)}[kind]
    return {"rel": rel * depth, "max": most * depth}
