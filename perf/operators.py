"""Weights in four bits and orthogonal updates, as cases for timing: plain forms, and the calls of ozimmu.

A weight matrix W (n x k) in four bits is cut like a slice tensor: every run of `group` elements of a row has one scale,
s = RN(RN32(max |w| / 7)) in the scales' type, and its elements are the integers c = RNE(w / s), clamped to [-8, 7]. Two of
them make a byte (c + 8, the even position in the low half); a row takes a multiple of 16 bytes. The operators:

  split   W -> codes and scales, and back to the weights s c that they stand for
  gemm    Y = X W^T     (t tokens: one while an answer is written, thousands while a prompt is read)
  grad    dX = dY W     (the gradient that goes on to the layer below)
  orth    X_0 = G / (|G| + eps), X_{i+1} = a X_i + (b A + c A^2) X_i with A = X_i X_i^T: the update of a weight matrix
          with its singular values brought near one; the iteration runs on the shorter side
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
EPS = 1e-7


def listed():
    return [
        # a small layer with rows that end inside a group: single-precision weights, cut after a training step
        dict(name="split_ragged", op="split", n=500, k=1000, group=32, type="f32", scales="bf16"),
        # a large layer as it is loaded
        dict(name="split_8192", op="split", n=8192, k=8192, group=128, type="bf16", scales="bf16"),
        # one token through a small layer: latency
        dict(name="token_2048", op="gemm", t=1, n=2048, k=2048, group=64, type="bf16"),
        # one token through a wide layer: the bytes of its weights
        dict(name="token_16384", op="gemm", t=1, n=16384, k=8192, group=128, type="bf16"),
        # a few answers written side by side, odd sizes, the finest groups
        dict(name="tokens_ragged", op="gemm", t=13, n=4095, k=5000, group=32, type="f16"),
        # a short prompt in single precision
        dict(name="prompt_f32", op="gemm", t=300, n=1500, k=1000, group=64, type="f32"),
        # long prompts
        dict(name="prompt_4096", op="gemm", t=4096, n=8192, k=4096, group=128, type="bf16"),
        # the gradient through a layer of odd sizes
        dict(name="grad_ragged", op="grad", t=777, n=1500, k=2000, group=32, type="f16"),
        # the gradient of a training step through a large layer
        dict(name="grad_4096", op="grad", t=4096, n=8192, k=4096, group=128, type="bf16"),
        # the update of a small square matrix: latency
        dict(name="orth_64", op="orth", batch=1, m=64, n=64, type="f32"),
        # the updates of several layers of one shape, taller than wide, odd
        dict(name="orth_batch", op="orth", batch=6, m=1000, n=520, type="f16"),
        # the update of a large square layer
        dict(name="orth_4096", op="orth", batch=1, m=4096, n=4096, type="bf16"),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def _orth_flops(c):
    r, l = sorted((c["m"], c["n"]))
    return c["batch"] * STEPS * (3.0 * r * r * l + 1.0 * r * r * r)   # the two symmetric products by half


def draw(rng):
    op = rng.choice(("split", "gemm", "gemm", "grad", "orth"))
    kind = rng.choice(("f32", "bf16", "f16"))
    while True:
        if op == "split":
            c = dict(op=op, n=_log(rng, 32, 16384), k=_log(rng, 32, 16384), group=rng.choice((32, 64, 128)), type=kind,
                     scales=rng.choice(("f32", "bf16", "f16")))
            fits = c["n"] * c["k"] <= 8192 * 8192
        elif op == "orth":
            c = dict(op=op, batch=_log(rng, 1, 16), m=_log(rng, 16, 4096), n=_log(rng, 16, 4096), type=kind)
            fits = _orth_flops(c) <= _orth_flops(dict(batch=1, m=4096, n=4096))
        else:
            t = _log(rng, 1, 64) if rng.random() < 0.5 and op == "gemm" else _log(rng, 16, 4096)
            c = dict(op=op, t=t, n=_log(rng, 64, 16384), k=_log(rng, 64, 16384), group=rng.choice((32, 64, 128)), type=kind)
            fits = c["t"] * c["n"] * c["k"] * (3 if kind == "f32" else 1) <= 4096 * 8192 * 4096 and c["n"] * c["k"] <= 16384 * 8192
        if fits:
            return c


def _cut(W, group, kind):
    """codes (n x row bytes, uint8) and scales (n x groups) of a weight matrix."""
    n, k = W.shape
    groups = -(-k // group)
    w = torch.nn.functional.pad(W.float(), (0, groups * group - k)).view(n, groups, group)
    top = w.abs().amax(dim=2)
    s = (top / torch.full_like(top, 7.0)).to(kind)   # (by a tensor: a quotient, not a product with a rounded 1/7)
    wide = torch.where(s == 0, torch.ones_like(s), s).double().unsqueeze(2)
    c = torch.round(w.double() / wide).clamp_(-8, 7).to(torch.int32).view(n, -1)   # (in 64 bits: a quotient next to a border)
    c = torch.nn.functional.pad(c[:, :k], (0, -k % 32)) + 8
    return (c[:, 0::2] | (c[:, 1::2] << 4)).to(torch.uint8), s


def _weights(codes, scales, group, k):
    """The weights s c in 32 bits."""
    c = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1)[:, :k].float() - 8.0
    return c * scales.float().repeat_interleave(group, dim=1)[:, :k]


def _normal(shape, seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=device)


def _weight_matrix(n, k, seed):
    """Normal weights; rows differ in size by a factor of a few."""
    return _normal((n, k), seed) / math.sqrt(k) * torch.exp(0.5 * _normal((n, 1), seed + 1))


def prepare(case, seed):
    op, kind = case["op"], TYPES[case["type"]]
    seed = 10 * seed
    state = dict(case)
    if op == "split":
        state["W"] = _weight_matrix(case["n"], case["k"], seed).to(kind)
    elif op == "orth":
        # a gradient: a few strong directions above noise
        b, m, n = case["batch"], case["m"], case["n"]
        r = min(16, m, n)
        state["G"] = (torch.bmm(_normal((b, m, r), seed), _normal((b, r, n), seed + 1)) / math.sqrt(r) + 0.3 * _normal((b, m, n), seed + 2)).to(kind)
    else:
        t, n, k, group = case["t"], case["n"], case["k"], case["group"]
        state["codes"], state["scales"] = _cut(_weight_matrix(n, k, seed), group, kind)
        # activations and their gradients: normal, with a few columns that stand out
        cols = k if op == "gemm" else n
        state["V"] = (_normal((t, cols), seed + 2) * torch.exp(_normal((1, cols), seed + 3))).to(kind)
    if own:   # what a program keeps between calls: the outputs' memory and the workspace
        from paper_2306_11975_amd import ozimmu

        if op == "split":
            n, k, group = case["n"], case["k"], case["group"]
            state["codes"] = torch.empty((n, ozimmu.q4_row_bytes(k)), dtype=torch.uint8, device="cuda")
            state["scales"] = torch.empty((n, -(-k // group)), dtype=TYPES[case["scales"]], device="cuda")
            state["out"] = torch.empty((n, k), dtype=TYPES[case["scales"]], device="cuda")
        elif op == "orth":
            state["out"] = torch.empty_like(state["G"])
            state["workspace"] = ozimmu.alloc_orthogonalize_workspace(case["batch"], case["m"], case["n"], kind)
        else:
            state["out"] = torch.empty((case["t"], case["n"] if op == "gemm" else case["k"]), dtype=kind, device="cuda")
            state["workspace"] = ozimmu.alloc_q4_workspace(case["t"], case["n"], case["k"], case["group"], kind, gradient=op == "grad")
    return state


def _orthogonalize(G):
    a, b, c = COEFFICIENTS
    X = G.float()
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2).contiguous()
    X = X / (X.double().square().sum(dim=(1, 2), keepdim=True).sqrt().float() + EPS)
    for _ in range(STEPS):
        A = torch.bmm(X, X.transpose(1, 2).contiguous())
        X = a * X + torch.bmm(b * A + c * torch.bmm(A, A), X)
    return (X.transpose(1, 2) if tall else X).to(G.dtype).contiguous()


def run(state):
    op = state["op"]
    if own:
        from paper_2306_11975_amd import ozimmu

        if op == "split":
            ozimmu.q4_split(state["W"], state["group"], state["codes"], state["scales"])
            ozimmu.q4_expand(state["codes"], state["scales"], state["group"], state["out"])
            return {"scales": state["scales"], "weights": state["out"]}
        if op == "orth":
            ozimmu.orthogonalize(state["G"], state["out"], state["workspace"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
        elif op == "gemm":
            ozimmu.q4_gemm(state["V"], state["codes"], state["scales"], state["group"], state["out"], state["workspace"])
        else:
            ozimmu.q4_gemm_grad(state["V"], state["codes"], state["scales"], state["group"], state["out"], state["workspace"])
        return state["out"]
    if op == "split":
        codes, scales = _cut(state["W"], state["group"], TYPES[state["scales"]])
        return {"scales": scales, "weights": _weights(codes, scales, state["group"], state["k"]).to(scales.dtype)}
    if op == "orth":
        return _orthogonalize(state["G"])
    W = _weights(state["codes"], state["scales"], state["group"], state["k"])
    V = state["V"]
    return torch.matmul(V.float(), W.t() if op == "gemm" else W).to(V.dtype)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "split":
        W, group, kind = state["W"], case["group"], TYPES[case["scales"]]
        n, k = W.shape
        scales, weights = [], torch.empty((n, k), dtype=torch.float64, device=W.device)
        for k0 in range(0, k, group):   # group by group, in 64 bits but for the two roundings of the definition
            w = W[:, k0:k0 + group].double()
            top = w.abs().max(dim=1).values
            s = (top / torch.full_like(top, 7.0)).float().to(kind).double()
            q = torch.where(s[:, None] > 0, w / s[:, None], torch.zeros_like(w))
            low = torch.floor(q)
            up = (q - low > 0.5) | ((q - low == 0.5) & (low.remainder(2) == 1))
            weights[:, k0:k0 + group] = torch.clamp(low + up.double(), -8, 7) * s[:, None]
            scales.append(s)
        return {"scales": torch.stack(scales, dim=1), "weights": weights}
    if op == "orth":
        a, b, c = COEFFICIENTS
        outs = []
        for G in state["G"].double():
            X = G.t().contiguous() if G.shape[0] > G.shape[1] else G
            X = X / (torch.linalg.vector_norm(X) + EPS)
            for _ in range(STEPS):
                A = X @ X.t()
                X = (A @ A * c + A * b) @ X + a * X
            outs.append(X.t().contiguous() if G.shape[0] > G.shape[1] else X)
        return torch.stack(outs)
    n, k, group = case["n"], case["k"], case["group"]
    W = torch.empty((n, k), dtype=torch.float64, device="cuda")
    W[:, 0::2] = (state["codes"] % 16).double()[:, :(k + 1) // 2]
    W[:, 1::2] = torch.div(state["codes"], 16, rounding_mode="floor").double()[:, :k // 2]
    for g in range(state["scales"].shape[1]):
        W[:, g * group:(g + 1) * group] = (W[:, g * group:(g + 1) * group] - 8) * state["scales"][:, g:g + 1].double()
    V = state["V"].double()
    return V @ W.t() if op == "gemm" else V @ W


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    op = case["op"]
    if op == "orth":
        return {"bytes": 2.0 * case["batch"] * case["m"] * case["n"] * size[case["type"]], "flops": _orth_flops(case)}
    n, k = case["n"], case["k"]
    groups = -(-k // case["group"])
    if op == "split":   # the weights in, codes and scales and what they stand for out
        return {"bytes": n * k * (size[case["type"]] + 0.5 + size[case["scales"]]) + n * groups * size[case["scales"]], "flops": 3.0 * n * k}
    return {"bytes": n * k * 0.5 + (n * groups + case["t"] * (n + k)) * size[case["type"]], "flops": 2.0 * case["t"] * n * k}
