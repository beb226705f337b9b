"""Products in 8-bit floating point and mixtures of experts, as cases for timing: plain forms, and the calls of ozimmu.

A matrix in eight bits: every block of 1 x 128 (tokens) or 128 x 128 (weights) elements has a scale 2^e, e the least integer from -127 on
with max |x| <= 448 2^e, and its elements are codes RNE(x / 2^e) of four significand bits (e4m3: the largest is 448, the least 2^-9). The
operators:

  cut      X -> codes and scales, and back to the values that they stand for
  gemm     Y = cut(X) W^T           (t tokens through a layer whose weights are held in eight bits)
  grad     dX = cut(dY) W and dW = cut(dY^T) cut(X^T)^T   (the runs of 128 of the second product lie along the tokens)
  experts, experts_grad             the same over experts: rows offsets[e] to offsets[e + 1] meet the weights of expert e; row r of the
                                    tokens is X[source[r]]; runs along the tokens start anew with every expert
  route    scores of a token's logits, the best experts under a bias and by groups, their weights; the order of the (token, choice) pairs
           by expert; the gradient of the logits
  combine  Y[t] = sum_j w[t, j] O[place[t, j]], and the gradients of O and w
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-20      # beside the sum of sigmoid scores


def listed():
    return [
        # activations of a small layer, odd sizes, single precision
        dict(name="cut_ragged", op="cut", n=500, k=1000, rows=1, type="f32"),
        # the weights of a large layer, after a training step
        dict(name="cut_8192", op="cut", n=8192, k=8192, rows=128, type="bf16"),
        # one token through a small layer: latency
        dict(name="token_2048", op="gemm", t=1, n=2048, k=2048, type="bf16"),
        # a long prompt through a large layer
        dict(name="prompt_4096", op="gemm", t=4096, n=8192, k=4096, type="bf16"),
        # both gradients of a training step through a large layer
        dict(name="grad_4096", op="grad", t=4096, n=8192, k=4096, type="bf16"),
        # sixteen answers written side by side, eight experts to a token: the bytes of the experts' weights
        dict(name="experts_decode", op="experts", t=16, top=8, experts=64, n=2048, k=2048, type="bf16"),
        # a prompt through the same experts
        dict(name="experts_prompt", op="experts", t=4096, top=8, experts=64, n=2048, k=2048, type="bf16"),
        # both gradients through a few experts of odd sizes
        dict(name="experts_grad_ragged", op="experts_grad", t=1001, top=2, experts=8, n=1000, k=520, type="f16"),
        # the choice for a few answers among few experts: latency
        dict(name="route_small", op="route", t=16, experts=8, top=2, score="softmax", bias=False, groups=1, top_groups=1, type="f32"),
        # the choice for a long batch among many experts, in groups
        dict(name="route_16384", op="route", t=16384, experts=256, top=8, score="sigmoid", bias=True, groups=8, top_groups=4, type="bf16"),
        # results of a short prompt, odd sizes, single precision
        dict(name="combine_ragged", op="combine", t=333, top=3, n=1001, type="f32"),
        # results of a long batch
        dict(name="combine_8192", op="combine", t=8192, top=8, n=4096, type="bf16"),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(("cut", "gemm", "gemm", "grad", "experts", "experts", "experts_grad", "route", "route", "combine"))
    kind = rng.choice(("f32", "bf16", "f16"))
    while True:
        if op == "cut":
            c = dict(op=op, n=_log(rng, 1, 16384), k=_log(rng, 32, 16384), rows=rng.choice((1, 128)), type=kind)
            fits = c["n"] * c["k"] <= (8192 * 8192 if kind != "f32" else 8192 * 4096)
        elif op == "gemm":
            t = _log(rng, 1, 64) if rng.random() < 0.5 else _log(rng, 16, 8192)
            c = dict(op=op, t=t, n=_log(rng, 64, 16384), k=_log(rng, 64, 16384), type=kind)
            fits = c["t"] * c["n"] * c["k"] <= 4096 * 8192 * 4096 and c["n"] * c["k"] <= 8192 * 16384
        elif op == "grad":
            c = dict(op=op, t=_log(rng, 16, 8192), n=_log(rng, 64, 16384), k=_log(rng, 64, 16384), type=kind)
            fits = c["t"] * c["n"] * c["k"] <= 4096 * 8192 * 4096 and c["n"] * c["k"] <= 8192 * 8192
        elif op in ("experts", "experts_grad"):
            t = _log(rng, 1, 64) if rng.random() < 0.4 and op == "experts" else _log(rng, 16, 8192)
            experts = _log(rng, 2, 256)
            c = dict(op=op, t=t, top=rng.randint(1, min(8, experts)), experts=experts, n=_log(rng, 64, 8192), k=_log(rng, 64, 8192), type=kind)
            fits = c["t"] * c["top"] * c["n"] * c["k"] <= 32768 * 2048 * 2048 and experts * c["n"] * c["k"] <= 64 * 2048 * 2048
        elif op == "route":
            experts = _log(rng, 2, 512)
            groups = rng.choice([g for g in (1, 1, 2, 4, 8) if experts % g == 0 and experts // g >= 2 or g == 1])
            top_groups = rng.randint(1, groups)
            c = dict(op=op, t=_log(rng, 1, 32768), experts=experts, top=rng.randint(1, min(8, experts // groups * top_groups)),
                     score=rng.choice(("softmax", "sigmoid")), bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, type=kind)
            fits = c["t"] * experts <= 16384 * 256
        else:
            c = dict(op=op, t=_log(rng, 1, 16384), top=rng.randint(1, 8), n=_log(rng, 64, 8192), type=kind)
            fits = c["t"] * c["top"] * c["n"] * SIZE[kind] <= 8192 * 8 * 4096 * 2
        if fits:
            return c


# ---- the plain forms

def _blocks(X, rows):
    """X padded with zeros to whole blocks, as (row blocks, rows, column blocks, 128)."""
    n, k = X.shape
    X = torch.nn.functional.pad(X, (0, -k % 128, 0, -n % rows))
    return X.view(X.shape[0] // rows, rows, X.shape[1] // 128, 128)


def _exponents(X, rows):
    """The exponents e of the blocks (int32)."""
    m, q = torch.frexp(_blocks(X.float(), rows).abs().amax(dim=(1, 3)))      # the largest is m 2^q, 448 is 0.875 2^9
    return torch.where(m == 0, torch.full_like(q, -127), (q - 9 + (m > 0.875).int()).clamp(min=-127))


def _power(e):
    """2^e in 32 bits, by its bits: exp2 may be off by one."""
    return ((e + 127) << 23).view(torch.float32)


def _values(X, e, rows):
    """What codes under the exponents e stand for, in 32 bits. (Two factors for a scale: 2^-127 has no inverse that is one.)"""
    n, k = X.shape
    e = e[:, None, :, None]
    near, far = e // 2, e - e // 2
    y = (_blocks(X.float(), rows) * _power(-near) * _power(-far)).to(torch.float8_e4m3fn).float()
    return (y * _power(near) * _power(far)).reshape(-1, e.shape[2] * 128)[:n, :k]


def _cut(X, rows=1):
    return _values(X, _exponents(X, rows), rows)


def _weights(codes, scales, k):
    """The weights that codes (n x row bytes) and scales (a byte e + 127 for each block) stand for, in 32 bits."""
    n, groups = codes.shape[0], -(-k // 128)
    s = _power(scales[:, :groups].int() - 127).repeat_interleave(128, dim=0)[:n].repeat_interleave(128, dim=1)[:, :k]
    return codes[:, :k].view(torch.float8_e4m3fn).float() * s


def _codes(X, rows):
    """Codes and scales as they are kept: rows of 128 bytes for each run, and of four bytes for four runs."""
    n, k = X.shape
    e = _exponents(X, rows)
    y = _values(X, e, rows) * _power(-e).repeat_interleave(rows, dim=0)[:n].repeat_interleave(128, dim=1)[:, :k]
    codes = torch.nn.functional.pad(y, (0, -k % 128)).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 4))


def _choice(state):
    """Indices of the best experts, best first, and the scores in 64 bits. Ties go to the lowest index."""
    l = state["logits"].double()
    s = torch.softmax(l, dim=1) if state["score"] == "softmax" else 1.0 / (1.0 + torch.exp(-l))
    c = s if state["bias_values"] is None else s + state["bias_values"].double()
    t, experts = l.shape
    groups = state["groups"]
    if groups > 1:
        by_group = c.view(t, groups, -1)
        value = by_group.sort(dim=2, descending=True).values[:, :, :2].sum(dim=2)
        kept = value.sort(dim=1, descending=True, stable=True).indices[:, :state["top_groups"]]
        allowed = torch.zeros_like(value, dtype=torch.bool).scatter_(1, kept, True)
        c = torch.where(allowed[:, :, None], by_group, torch.full_like(by_group, -math.inf)).view(t, experts)
    return c.sort(dim=1, descending=True, stable=True).indices[:, :state["top"]], s


def _order(indices, experts):
    """offsets, source and place of the pairs sorted by expert, as they come within one."""
    t, top = indices.shape
    flat = indices.reshape(-1).long()
    order = flat.sort(stable=True).indices
    place = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=order.device))
    counts = (flat[None, :] == torch.arange(experts, device=flat.device)[:, None]).sum(dim=1)
    offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0))
    return offsets.int(), (order // top).int(), place.view(t, top).int()


def _route(state):
    chosen, s = _choice(state)
    s = s.float()
    p = s.gather(1, chosen)
    total = p.sum(dim=1, keepdim=True) + (EPS if state["score"] == "sigmoid" else 0.0)
    w = p / total
    dw = state["dweights"]
    inner = (dw - (dw * w).sum(dim=1, keepdim=True)) / total      # the gradient of the chosen scores
    if state["score"] == "softmax":
        dl = p * inner      # (the sum over all of the gradient times the score is zero)
    else:
        dl = inner * p * (1.0 - p)
    dlogits = torch.zeros_like(s).scatter_(1, chosen, dl)
    return {"indices": chosen.int(), "weights": w, "dlogits": dlogits.to(state["logits"].dtype)}


# ---- inputs

def _normal(shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


def _weight_matrix(n, k, seed):
    """Normal weights; rows differ in size by a factor of a few."""
    return _normal((n, k), seed) / math.sqrt(k) * torch.exp(0.5 * _normal((n, 1), seed + 1))


def _activations(t, k, seed, kind):
    """Normal, with a few columns that stand out."""
    return (_normal((t, k), seed) * torch.exp(_normal((1, k), seed + 1))).to(kind)


def prepare(case, seed):
    op, kind = case["op"], TYPES[case["type"]]
    seed = 10 * seed
    state = dict(case)
    if op == "cut":
        state["X"] = _weight_matrix(case["n"], case["k"], seed).to(kind) if case["rows"] == 128 else _activations(case["n"], case["k"], seed, kind)
    elif op == "route":
        # some experts are more popular than others
        state["logits"] = (_normal((case["t"], case["experts"]), seed) + 0.5 * _normal((1, case["experts"]), seed + 1)).to(kind)
        state["bias_values"] = 0.1 * _normal((case["experts"],), seed + 2) if case["bias"] else None
        state["dweights"] = _normal((case["t"], case["top"]), seed + 3)
    elif op == "combine":
        t, top, n = case["t"], case["top"], case["n"]
        state["O"] = _normal((t * top, n), seed).to(kind)
        state["place"] = _normal((t * top,), seed + 1).argsort().view(t, top).int()
        state["weights"] = torch.softmax(_normal((t, top), seed + 2), dim=1)
        state["dY"] = _normal((t, n), seed + 3).to(kind)
    else:
        t, n, k = case["t"], case["n"], case["k"]
        rows = t
        if "experts" in case:
            experts, top = case["experts"], case["top"]
            rows = t * top
            logits = _normal((t, experts), seed + 4) + 0.5 * _normal((1, experts), seed + 5)
            offsets, source, _ = _order(logits.sort(dim=1, descending=True, stable=True).indices[:, :top], experts)
            state["offsets"], state["source"], state["bounds"] = offsets, source, offsets.tolist()
            parts = [_codes(_weight_matrix(n, k, seed + 1000003 * (e + 1)), 128) for e in range(experts)]
            state["codes"], state["scales"] = torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])
        else:
            state["codes"], state["scales"] = _codes(_weight_matrix(n, k, seed), 128)
        state["X"] = _activations(t, k, seed + 2, kind)
        if op in ("grad", "experts_grad"):
            state["dY"] = (_normal((rows, n), seed + 6) * torch.exp(_normal((rows, 1), seed + 7)) / math.sqrt(n)).to(kind)
    if own:   # what a program keeps between calls: the outputs' memory and the workspace
        from paper_2306_11975_amd import ozimmu

        def empty(*shape, dtype=kind):
            return torch.empty(shape, dtype=dtype, device="cuda")

        if op == "cut":
            n, k = case["n"], case["k"]
            state["codes"] = empty(n, ozimmu.f8_row_bytes(k), dtype=torch.uint8)
            state["scales"] = empty(-(-n // case["rows"]), ozimmu.f8_scale_bytes(k), dtype=torch.uint8)
            state["out"] = empty(n, k)
        elif op == "route":
            t, top, experts = case["t"], case["top"], case["experts"]
            state["indices"], state["place"] = empty(t, top, dtype=torch.int32), empty(t, top, dtype=torch.int32)
            state["source"], state["offsets"] = empty(t * top, dtype=torch.int32), empty(experts + 1, dtype=torch.int32)
            state["weights"], state["dlogits"] = empty(t, top, dtype=torch.float32), empty(t, experts)
            state["workspace"] = ozimmu.alloc_expert_order_workspace(t, top, experts)
        elif op == "combine":
            state["Y"], state["dO"], state["dweights"] = empty(case["t"], case["n"]), empty(case["t"] * case["top"], case["n"]), empty(case["t"], case["top"], dtype=torch.float32)
        else:
            experts = case.get("experts", 0)
            if op in ("gemm", "experts"):
                state["Y"] = empty(rows, n)
                state["workspace"] = ozimmu.alloc_f8_workspace("gemm", t, n, k, kind, rows=rows, experts=experts)
            else:
                state["dX"], state["dW"] = empty(rows, k), empty(*((experts,) if experts else ()), n, k)
                state["workspace"] = ozimmu.alloc_f8_workspace("grad", rows, n, k, kind, rows=rows, experts=experts)
                state["workspace_w"] = ozimmu.alloc_f8_workspace("weight_grad", t, n, k, kind, rows=rows, experts=experts)
    return state


def _run_own(s):
    from paper_2306_11975_amd import ozimmu

    op = s["op"]
    if op == "cut":
        ozimmu.f8_split(s["X"], s["codes"], s["scales"], s["rows"])
        ozimmu.f8_expand(s["codes"], s["scales"], s["out"], s["rows"])
        return {"scales": s["scales"][:, :-(-s["k"] // 128)], "values": s["out"]}
    if op == "route":
        how = dict(score=s["score"], renormalize=True)
        ozimmu.route(s["logits"], s["indices"], s["weights"], bias=s["bias_values"], groups=s["groups"], top_groups=s["top_groups"], **how)
        ozimmu.expert_order(s["indices"], s["experts"], s["offsets"], s["source"], s["place"], s["workspace"])
        ozimmu.route_grad(s["logits"], s["indices"], s["dweights"], s["dlogits"], **how)
        return {x: s[x] for x in ("indices", "weights", "offsets", "source", "place", "dlogits")}
    if op == "combine":
        ozimmu.expert_combine(s["O"], s["place"], s["weights"], s["Y"])
        ozimmu.expert_combine_grad(s["dY"], s["O"], s["place"], s["weights"], s["dO"], s["dweights"])
        return {x: s[x] for x in ("Y", "dO", "dweights")}
    if op == "gemm":
        ozimmu.f8_gemm(s["X"], s["codes"], s["scales"], s["Y"], s["workspace"])
        return s["Y"]
    if op == "experts":
        ozimmu.f8_gemm(s["X"], s["codes"], s["scales"], s["Y"], s["workspace"], offsets=s["offsets"], source=s["source"])
        return s["Y"]
    if op == "grad":
        ozimmu.f8_gemm_grad(s["dY"], s["codes"], s["scales"], s["dX"], s["workspace"])
        ozimmu.f8_weight_grad(s["dY"], s["X"], s["dW"], s["workspace_w"])
    else:
        ozimmu.f8_gemm_grad(s["dY"], s["codes"], s["scales"], s["dX"], s["workspace"], offsets=s["offsets"])
        ozimmu.f8_weight_grad(s["dY"], s["X"], s["dW"], s["workspace_w"], offsets=s["offsets"], source=s["source"])
    return {"dX": s["dX"], "dW": s["dW"]}


def run(state):
    if own:
        return _run_own(state)
    op, kind = state["op"], TYPES[state["type"]]
    if op == "cut":
        e = _exponents(state["X"], state["rows"])
        return {"scales": (e + 127).to(torch.uint8), "values": _values(state["X"], e, state["rows"]).to(kind)}
    if op == "route":
        out = _route(state)
        out["offsets"], out["source"], out["place"] = _order(out["indices"], state["experts"])
        return {x: out[x] for x in ("indices", "weights", "offsets", "source", "place", "dlogits")}
    if op == "combine":
        w, dY = state["weights"], state["dY"].float()
        place = state["place"].long()
        rows = state["O"][place.view(-1)].view(*place.shape, -1).float()      # t x top x n
        dO = torch.empty_like(state["O"])
        dO[place.view(-1)] = (w[:, :, None] * dY[:, None, :]).to(kind).view(-1, dY.shape[1])
        return {"Y": (w[:, :, None] * rows).sum(dim=1).to(kind), "dO": dO, "dweights": (rows * dY[:, None, :]).sum(dim=2)}
    k = state["k"]
    if op == "gemm":
        return torch.matmul(_cut(state["X"]), _weights(state["codes"], state["scales"], k).t()).to(kind)
    if op == "grad":
        dX = torch.matmul(_cut(state["dY"]), _weights(state["codes"], state["scales"], k))
        dW = torch.matmul(_cut(state["dY"].t()), _cut(state["X"].t()).t())
        return {"dX": dX.to(kind), "dW": dW.to(kind)}
    bounds, source = state["bounds"], state["source"].long()
    if op == "experts":
        V, Y = _cut(state["X"]), torch.empty((len(source), state["n"]), dtype=kind, device="cuda")
        for e in range(state["experts"]):
            a, b = bounds[e], bounds[e + 1]
            if b > a:
                Y[a:b] = torch.matmul(V[source[a:b]], _weights(state["codes"][e], state["scales"][e], k).t()).to(kind)
        return Y
    dX, dW = torch.empty((len(source), k), dtype=kind, device="cuda"), torch.zeros((state["experts"], state["n"], k), dtype=kind, device="cuda")
    V = _cut(state["dY"])
    for e in range(state["experts"]):
        a, b = bounds[e], bounds[e + 1]
        if b > a:
            dX[a:b] = torch.matmul(V[a:b], _weights(state["codes"][e], state["scales"][e], k)).to(kind)
            dW[e] = torch.matmul(_cut(state["dY"][a:b].t()), _cut(state["X"][source[a:b]].t()).t()).to(kind)
    return {"dX": dX, "dW": dW}


# ---- the definitions in 64 bits

def _pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_cut(X, rows):
    """Exponents by trying, and values by the spacing of numbers of four significand bits, run by run of 128 columns."""
    n, k = X.shape
    X = X.double()
    exponents, values = [], torch.empty_like(X)
    for k0 in range(0, k, 128):
        x = X[:, k0:k0 + 128]
        top = x.abs().max(dim=1).values
        top = torch.nn.functional.pad(top, (0, -n % rows)).view(-1, rows).max(dim=1).values
        e = torch.clamp(torch.floor(torch.log2(torch.clamp(top, min=1e-300) / 448.0)) - 1.0, -127, 127).int()      # (one less than it may be, for the logarithm's rounding)
        for _ in range(3):
            e = torch.where(top > 448.0 * _pow2(e), e + 1, e)
        s = _pow2(e).repeat_interleave(rows)[:n, None]
        q = x / s
        step = _pow2(torch.clamp(torch.floor(torch.log2(torch.clamp(q.abs(), min=1e-9))), min=-6).int() - 3)
        step = torch.where(q.abs() >= 16.0 * step, 2.0 * step, step)      # (the logarithm's rounding again)
        step = torch.where((q.abs() < 8.0 * step) & (step > 2.0 ** -9), 0.5 * step, step)
        r = q / step
        low = torch.floor(r)
        up = (r - low > 0.5) | ((r - low == 0.5) & (low.remainder(2) == 1))
        values[:, k0:k0 + 128] = (low + up.double()) * step * s
        exponents.append(e)
    return torch.stack(exponents, dim=1), values


def _exact_weights(codes, scales, k):
    c = codes[:, :k].long()
    power, part = (c // 8) % 16, (c % 8).double()
    w = torch.where(power == 0, part * 2.0 ** -9, (8.0 + part) * _pow2((power - 10).int()))
    w = torch.where(c >= 128, -w, w)
    for g in range(-(-k // 128)):
        for r in range(scales.shape[0]):
            w[r * 128:(r + 1) * 128, g * 128:(g + 1) * 128] *= _pow2(scales[r, g].long() - 127)
    return w


def _exact_route(state):
    l = state["logits"].double()
    t, experts = l.shape
    if state["score"] == "softmax":
        s = torch.exp(l - torch.logsumexp(l, dim=1, keepdim=True))
    else:
        s = torch.sigmoid(l)
    c = s.clone() if state["bias_values"] is None else s + state["bias_values"].double()[None, :]
    per, line = experts // state["groups"], torch.arange(t, device=l.device)

    def best(v):
        """The place of each row's largest value, the lowest where several are."""
        return (v == v.max(dim=1, keepdim=True).values).int().argmax(dim=1)

    if state["groups"] > 1:
        value = torch.empty((t, state["groups"]), dtype=torch.float64, device=l.device)
        for g in range(state["groups"]):
            part = c[:, g * per:(g + 1) * per].clone()
            first = best(part)
            value[:, g] = part[line, first]
            if per > 1:
                part[line, first] = -math.inf
                value[:, g] += part.max(dim=1).values
        allowed = torch.zeros((t, state["groups"]), dtype=torch.bool, device=l.device)
        for _ in range(state["top_groups"]):
            g = best(value)
            allowed[line, g] = True
            value[line, g] = -math.inf
        c[~allowed.repeat_interleave(per, dim=1)] = -math.inf
    chosen = []
    for _ in range(state["top"]):
        chosen.append(best(c))
        c[line, chosen[-1]] = -math.inf
    chosen = torch.stack(chosen, dim=1)
    p = s.gather(1, chosen)
    total = p.sum(dim=1) + (EPS if state["score"] == "sigmoid" else 0.0)
    dw = state["dweights"].double()
    dlogits = torch.zeros_like(s)
    mean = (dw * p).sum(dim=1) / total
    slope = torch.ones_like(p) if state["score"] == "softmax" else 1.0 - p
    dlogits.scatter_(1, chosen, p * slope * (dw - mean[:, None]) / total[:, None])
    flat = chosen.reshape(-1)
    offsets = torch.tensor([0] + [int((flat <= e).sum()) for e in range(experts)], dtype=torch.int32)
    order = torch.cat([torch.nonzero(flat == e).view(-1) for e in range(experts)])
    place = torch.empty(t * state["top"], dtype=torch.int32, device=l.device)
    place[order] = torch.arange(t * state["top"], dtype=torch.int32, device=l.device)
    return {"indices": chosen.int(), "weights": p / total[:, None], "offsets": offsets.to(l.device),
            "source": torch.div(order, state["top"], rounding_mode="floor").int(), "place": place.view(t, -1), "dlogits": dlogits}


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "cut":
        e, values = _exact_cut(state["X"], case["rows"])
        return {"scales": (e + 127).to(torch.uint8), "values": values}
    if op == "route":
        return _exact_route(state)
    if op == "combine":
        place, w, dY = state["place"].long(), state["weights"].double(), state["dY"].double()
        Y, dO = torch.zeros_like(dY), torch.empty(state["O"].shape, dtype=torch.float64, device="cuda")
        dw = torch.empty_like(w)
        for j in range(case["top"]):
            rows = state["O"][place[:, j]].double()
            Y += w[:, j:j + 1] * rows
            dO[place[:, j]] = w[:, j:j + 1] * dY
            dw[:, j] = (rows * dY).sum(dim=1)
        return {"Y": Y, "dO": dO, "dweights": dw}
    k = case["k"]

    def cut(X):
        return _exact_cut(X, 1)[1]

    if op == "gemm":
        return cut(state["X"]) @ _exact_weights(state["codes"], state["scales"], k).t()
    if op == "grad":
        dX = cut(state["dY"]) @ _exact_weights(state["codes"], state["scales"], k)
        return {"dX": dX, "dW": cut(state["dY"].t().contiguous()) @ cut(state["X"].t().contiguous()).t()}
    bounds, source = state["bounds"], state["source"].long()
    parts, weights = [], []
    for e in range(case["experts"]):
        a, b = bounds[e], bounds[e + 1]
        W = _exact_weights(state["codes"][e], state["scales"][e], k) if b > a else None
        x = state["X"][source[a:b]]
        if op == "experts":
            if b > a:
                parts.append(cut(x) @ W.t())
        else:
            dy = state["dY"][a:b]
            if b > a:
                parts.append(cut(dy) @ W)
                weights.append(cut(dy.t().contiguous()) @ cut(x.t().contiguous()).t())
            else:
                weights.append(torch.zeros((case["n"], k), dtype=torch.float64, device="cuda"))
    return torch.cat(parts) if op == "experts" else {"dX": torch.cat(parts), "dW": torch.stack(weights)}


def work(case):
    size, op = SIZE[case["type"]], case["op"]
    if op == "cut":   # values in, codes and scales and what they stand for out
        n, k = case["n"], case["k"]
        return {"bytes": n * k * (2.0 * size + 1.0) + n * k / (128.0 * case["rows"]), "flops": 3.0 * n * k}
    if op == "route":   # logits, their gradient and the weights' in; choices, weights, order and gradient out
        t, experts, top = case["t"], case["experts"], case["top"]
        return {"bytes": 2.0 * t * experts * size + t * top * 20.0 + 4.0 * experts, "flops": 10.0 * t * experts}
    if op == "combine":
        t, top, n = case["t"], case["top"], case["n"]
        return {"bytes": 2.0 * t * n * size + 2.0 * t * top * n * size + t * top * 12.0, "flops": 5.0 * t * top * n}
    t, n, k = case["t"], case["n"], case["k"]
    rows, used = t, 1
    if "experts" in case:
        rows, used = t * case["top"], min(case["experts"], t * case["top"])
    if op in ("gemm", "experts"):
        return {"bytes": used * n * k * (1.0 + 1.0 / 16384) + (t * k + rows * n) * size, "flops": 2.0 * rows * n * k}
    written = case.get("experts", 1)
    return {"bytes": used * n * k * (1.0 + 1.0 / 16384) + written * n * k * size + (t * k + rows * n + rows * k) * size, "flops": 4.0 * rows * n * k}
