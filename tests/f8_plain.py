"""Plain 64-bit forms of the operators in 8-bit floating point and of those for mixtures of experts (CPU), shared by their tests."""
import math

import torch

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


def half_step(dt):
    return torch.finfo(dt).eps / 2


def round_to(x64, dt):
    """A 64-bit value that 32 bits hold, or nearly: rounded once to dt."""
    return x64.to(F32).to(dt) if dt != F32 else x64.to(F32)


def e4m3(q):
    """RNE to e4m3 of 64-bit values of at most 448, by the spacing of the format."""
    m, ex = torch.frexp(q)
    step = torch.ldexp(torch.ones_like(q), torch.clamp(ex - 1, min=-6) - 3)
    return torch.round(q / step) * step


def exponents(X, rows, along=1):
    """e of the blocks of `rows` x 128, over finite values."""
    X = X.double()
    a = torch.where(torch.isfinite(X), X.abs(), torch.zeros_like(X))
    n, k = a.shape
    a = torch.nn.functional.pad(a, (0, -k % 128, 0, -n % rows)).view(-(-n // rows), rows, -(-k // 128), 128).amax(dim=(1, 3))
    m, q = torch.frexp(a)
    return torch.where(a == 0, torch.full_like(q, -127), (q - 9 + (m > 0.875).int()).clamp(min=-127))


def spread(e, n, k, rows):
    return e.repeat_interleave(rows, dim=0)[:n].repeat_interleave(128, dim=1)[:, :k]


def cut(X, rows=1):
    """(exponents, codes' values, values) of a matrix."""
    n, k = X.shape
    e = exponents(X, rows)
    s = torch.ldexp(torch.ones(n, k, dtype=torch.float64), spread(e, n, k, rows))
    x = X.double()
    c = e4m3(torch.where(torch.isfinite(x), x / s, torch.full_like(x, math.nan)))
    return e, c, c * s


def cut_columns(X):
    """Values cut in runs of 128 along the rows."""
    return cut(X.t().contiguous())[2].t()


def decode(codes):
    return codes.cpu().view(torch.uint8).view(torch.float8_e4m3fn).to(F32).double()


def guarded(rows, cols, dt, extra=0, offset=0, fill=77.0, device="cuda"):
    """A (rows x cols) view inside a larger buffer (row stride cols + extra, `offset` values from its start), and the buffer."""
    ld = cols + extra
    buf = torch.full((rows * ld + offset + 64,), fill, dtype=dt, device=device)
    return buf[offset:offset + rows * ld].view(rows, ld)[:, :cols], buf


def untouched(buf, rows, cols, extra, offset, fill=77.0):
    ld = cols + extra
    inner = buf[offset:offset + rows * ld].view(rows, ld)
    return bool((buf[:offset] == fill).all() and (inner[:, cols:] == fill).all() and (buf[offset + rows * ld:] == fill).all())


def small_integers(shape, g, top=8):
    """Integers of at most four bits, times 1, 2 or 4 by rows: their cut is lossless and their products' sums are exact in 32 bits."""
    x = torch.randint(-top, top + 1, shape, generator=g).double()
    return x * torch.pow(2.0, torch.randint(0, 2, (shape[0], 1), generator=g).double())


# ---- choice of experts
def route64(logits, top, bias=None, score="softmax", groups=1, top_groups=1, renormalize=True, scale=1.0):
    l = logits.double().cpu()
    t, experts = l.shape
    indices, weights = torch.full((t, top), -1, dtype=torch.int32), torch.zeros(t, top, dtype=torch.float64)
    per = experts // groups
    for i in range(t):
        row = l[i]
        bad = bool(row.isnan().any()) or (score == "softmax" and bool((row == math.inf).any()))
        if score == "softmax":
            m = row.max()
            s = torch.zeros_like(row) if m == -math.inf else torch.exp(row - m) / torch.exp(row - m).sum()
        else:
            s = 1.0 / (1.0 + torch.exp(-row))
        c = s if bias is None else s + bias.double().cpu()
        c = torch.where(row == -math.inf, torch.full_like(c, -math.inf), c)
        bad = bad or bool(c.isnan().any())
        if bad:
            weights[i] = math.nan
            continue
        v = c.tolist()
        if groups > 1:
            value = []
            for g in range(groups):
                best = sorted((x for x in v[g * per:(g + 1) * per] if x > -math.inf), reverse=True)[:2]
                value.append(best[0] + best[1] if len(best) > 1 else best[0] if best else -math.inf)
            kept = [g for g in sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups] if value[g] > -math.inf]
            v = [x if e // per in kept else -math.inf for e, x in enumerate(v)]
        chosen = [e for e in sorted(range(experts), key=lambda e: (-v[e], e)) if v[e] > -math.inf][:top]
        if not chosen:
            continue
        p = s[chosen]
        if renormalize:
            if score == "softmax":
                x = torch.exp(row[chosen] - row[chosen].max())
                p = x / x.sum()
            else:
                p = p / (p.sum() + 1e-20)
        indices[i, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
        weights[i, :len(chosen)] = p * scale
    return indices, weights


def route_weights(l, indices, score, renormalize, scale):
    """The weights of a given choice as a differentiable function of 64-bit logits."""
    there = indices >= 0
    s = torch.softmax(l, dim=1) if score == "softmax" else torch.sigmoid(l)
    p = torch.where(there, s.gather(1, indices.clamp(min=0).long()), torch.zeros((), dtype=torch.float64))
    if renormalize:
        p = p / (p.sum(dim=1, keepdim=True) + (1e-20 if score == "sigmoid" else 0.0))
    return p * scale


def order64(indices, experts):
    t, top = indices.shape
    flat = indices.reshape(-1).tolist()
    rows = [p for e in range(experts) for p in range(t * top) if flat[p] == e]
    offsets = [0]
    for e in range(experts):
        offsets.append(offsets[-1] + flat.count(e))
    place = [-1] * (t * top)
    for r, p in enumerate(rows):
        place[p] = r
    source = [p // top for p in rows] + [-1] * (t * top - len(rows))
    return offsets, source, place
