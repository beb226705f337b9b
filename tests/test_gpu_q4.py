"""Weights in four bits against plain 64-bit implementations: the cut and its inverse exactly, products and gradients within bounds that count roundings."""
import math

import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
GUARD = 0x5A


def half_step(dt):
    return torch.finfo(dt).eps / 2


# ---------------------------------------------------------------- plain implementations (CPU, 64 bits)
def plain_cut(W, group, stype):
    """codes (int, n x k) and scales by the definition; quotients in 64 bits, where they cannot fall onto a border they only come near."""
    n, k = W.shape
    groups = -(-k // group)
    codes, scales = torch.zeros(n, k, dtype=torch.int64), torch.zeros(n, groups, dtype=stype)
    for g in range(groups):
        w = W[:, g * group:(g + 1) * group].double()
        top = w.abs().amax(dim=1)      # (NaN stays)
        s = (top.float() / torch.full((n,), 7.0)).to(stype)
        scales[:, g] = s
        usable = (s.double() > 0) & torch.isfinite(s.double())
        q = w / torch.where(usable, s.double(), torch.ones(n, dtype=torch.float64))[:, None]
        c = torch.round(torch.nan_to_num(q, nan=0.0, posinf=0.0, neginf=0.0)).clamp(-8, 7)
        codes[:, g * group:(g + 1) * group] = torch.where(usable[:, None], c, torch.zeros_like(c)).long()
    return codes, scales


def unpack(codes, k):
    c = codes.cpu().long()
    return torch.stack((c & 15, c >> 4), dim=2).view(c.shape[0], -1)[:, :k] - 8


def pack(c):
    c = torch.nn.functional.pad(c, (0, -c.shape[1] % 32)) + 8
    return (c[:, 0::2] | (c[:, 1::2] << 4)).to(torch.uint8)


def weights64(c, scales, group):
    return c.double() * scales.cpu().double().repeat_interleave(group, dim=1)[:, :c.shape[1]]


def padded(rows, cols, dt, extra, offset, fill=None, seed=None):
    """A (rows x cols) view on the GPU inside a larger buffer (row stride cols + extra, `offset` values from its start), and the buffer."""
    ld = cols + extra
    buf = torch.full((rows * ld + offset + 64,), fill if fill is not None else 77.0, dtype=dt, device=DEV)
    return buf[offset:offset + rows * ld].view(rows, ld)[:, :cols], buf


def random_weights(n, k, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n, k, generator=g) * torch.exp(torch.randn(n, 1, generator=g)) / math.sqrt(max(k, 1))


def device_cut(W, group, stype):
    n, k = W.shape
    codes = torch.zeros(n, oz.q4_row_bytes(k), dtype=torch.uint8, device=DEV)
    scales = torch.zeros(n, -(-k // group), dtype=stype, device=DEV)
    oz.q4_split(W, group, codes, scales)
    return codes, scales


# ---------------------------------------------------------------- the cut
SPLITS = [(1, 1, 32), (1, 31, 32), (3, 32, 32), (5, 33, 64), (17, 1000, 32), (64, 129, 128), (130, 257, 64), (9, 4096, 128), (2, 20000, 128), (1000, 96, 128)]


@pytest.mark.parametrize("stype", TYPES)
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("n,k,group", SPLITS)
def test_split_and_expand(n, k, group, dt, stype):
    W0 = random_weights(n, k, n * 31 + k).to(dt)
    for extra, offset in ((0, 0), (5, 3), (8, 8)):
        W, _ = padded(n, k, dt, extra, offset)
        W.copy_(W0)
        rb = oz.q4_row_bytes(k)
        codes = torch.full((n, rb + 16), GUARD, dtype=torch.uint8, device=DEV)
        groups = -(-k // group)
        scales, sbuf = padded(n, groups, stype, 2, 1)
        oz.q4_split(W, group, codes, scales)
        c, s = plain_cut(W0, group, stype)
        assert torch.equal(scales.cpu(), s)
        assert torch.equal(unpack(codes[:, :rb], k), c)
        assert (codes[:, rb:] == GUARD).all()                       # what lies between rows is left alone
        assert torch.equal(unpack(codes[:, :rb], rb * 2)[:, k:], torch.zeros(n, 2 * rb - k, dtype=torch.int64))
        assert (sbuf.view(-1)[:1] == 77).all() and (sbuf[1:1 + n * (groups + 2)].view(n, -1)[:, groups:] == 77).all()
        out, obuf = padded(n, k, stype, extra, offset)
        oz.q4_expand(codes, scales, group, out)
        # s c is exact in 64 bits; rounded once
        assert torch.equal(out.cpu(), weights64(c, s, group).to(torch.float32).to(stype) if stype != F32 else weights64(c, s, group).to(F32))
        assert (obuf[:offset] == 77).all() and (obuf[offset:offset + n * (k + extra)].view(n, -1)[:, k:] == 77).all()


@pytest.mark.parametrize("stype", TYPES)
def test_split_at_borders_and_extremes(stype):
    """Quotients on and next to a border, groups of zeros, scales that underflow or overflow their type, infinities and NaN."""
    group, rows = 32, []
    g = torch.Generator().manual_seed(5)
    for top in (7.0, 1.0, 3.3, 0.1, 1e-3, 2.0 ** -20, 2.0 ** -26, 1e-30, 1e-38, 1e-41, 2.0 ** -149, 3e38, 1e6, 5e5, 458745.0):
        s = float((torch.tensor([top], dtype=F32) / torch.tensor([7.0])).to(stype))
        row = torch.zeros(group, dtype=F32)
        row[0] = top
        for i in range(1, 16):     # (j + 1/2) s and its neighbours in 32 bits
            mid = torch.tensor((i % 8 - 0.5) * s * (-1 if i & 1 else 1), dtype=F32).clamp(-top, top)
            row[2 * i - 1] = mid
            row[2 * i] = torch.nextafter(mid, torch.tensor(0.0 if i & 2 else math.copysign(math.inf, float(mid) or 1.0))).clamp(-top, top)
        rows.append(row)
    rows.append(torch.zeros(group))
    rows.append(-torch.zeros(group))
    for bad in (math.inf, -math.inf, math.nan):
        row = torch.randn(group, generator=g)
        row[11] = bad
        rows.append(row)
    W = torch.stack(rows)
    W = torch.cat((W, torch.randn(W.shape, generator=g)), dim=1)     # the group beside it is what it would be anyway
    codes, scales = device_cut(W.to(DEV), group, stype)
    c, s = plain_cut(W, group, stype)
    assert torch.equal(scales.cpu().float().nan_to_num(nan=-1.0), s.float().nan_to_num(nan=-1.0))
    assert torch.equal(unpack(codes, 64), c)
    out = torch.empty(W.shape, dtype=stype, device=DEV)
    oz.q4_expand(codes, scales, group, out)
    assert out[-1].isnan()[:32].all() and out[-2].isnan()[:32].all() and not out[:, 32:].isnan().any()


# ---------------------------------------------------------------- products
def tokens(t, cols, dt, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(t, cols, generator=g) * torch.exp(torch.randn(1, cols, generator=g))).to(dt)


def check(got, V, W, dt, inner, rounded_weights):
    """|got - V W| against what roundings can do. One rounding of the result; weights rounded to a 16-bit type (products of more than 16 tokens may do that,
    gradients do); 32-bit values as two slices (each operand off by at most 2^-22 of itself or 2^-40 of its row's largest, a third product of 2^-22 left out); the sums in 32 bits,
    whose terms may carry the codes' offset (up to 24 + 16 for codes up to 8: five times the largest term)."""
    want = V.double() @ W
    terms = V.double().abs() @ W.abs()
    top = V.double().abs().amax(dim=1, keepdim=True) @ W.abs().amax(dim=0, keepdim=True)
    sums = (3 if dt == F32 else 1) * (inner + 8) * 2.0 ** -24      # (32 bits: three products to a term)
    if dt == F32:
        bound = 3 * 2.0 ** -22 * terms + 4 * inner * 2.0 ** -40 * top + sums * terms
    else:
        bound = (half_step(dt) if rounded_weights else 0.0) * terms + (inner + 8) * 2.0 ** -24 * 40 * top
    bound = bound + half_step(dt) * (want.abs() + bound) + torch.finfo(dt).tiny
    off = (got.cpu().double() - want).abs()
    assert (off <= bound).all(), f"off by up to {(off / bound).max():.3g} times what roundings can do"
    # and typical errors are far below the worst: in the norm, one rounding of the result and of the weights
    if want.numel() > 64:
        rel = float(off.norm() / want.norm())
        assert rel <= (2e-6 if dt == F32 else 1.5 * half_step(dt)), rel


GEMMS = [(1, 1, 1, 32), (1, 16, 128, 128), (1, 2048, 512, 64), (1, 9000, 200, 128), (2, 15, 33, 32), (3, 33, 1000, 64), (5, 100, 257, 128), (13, 4095, 500, 32),
         (16, 64, 4096, 128), (16, 8200, 130, 64), (17, 40, 100, 32), (40, 130, 64, 64), (64, 64, 1024, 128), (65, 333, 777, 32), (129, 257, 96, 64), (300, 150, 1000, 128),
         (1000, 700, 320, 64), (2100, 4200, 192, 128), (3800, 3700, 100, 32),
         (400, 2500, 2570, 32), (200, 6000, 1100, 64), (33, 17000, 260, 128), (16, 16500, 1000, 64), (400, 1700, 260, 64),
         # tiles of 64 and of 128 that end in every way, with k from eight on; many tokens of few and of many positions
         (300, 2000, 8, 32), (290, 2001, 9, 32), (310, 1987, 15, 64), (257, 2050, 63, 128), (1000, 1030, 129, 64), (64, 8200, 200, 32), (2000, 2100, 513, 64),
         # one token and two, the row's end in every part of a piece
         (1, 5, 513, 32), (1, 9, 4097, 128), (1, 2051, 1111, 32), (1, 8200, 600, 64), (1, 8193, 9000, 128), (1, 300, 20001, 64), (2, 6, 541, 32), (2, 1100, 5000, 64),
         (2, 2500, 1537, 128), (2, 9000, 1026, 32), (2, 4, 33000, 128),
         # every tile of the passes, with rows of tokens at odd places and an end inside a step
         (20, 100, 2500, 32), (5, 387, 10575, 64), (37, 300, 2049, 128), (60, 1500, 701, 128), (33, 2500, 129, 32), (100, 2500, 1001, 64), (64, 8200, 513, 128), (9, 9000, 127, 64), (20, 9000, 300, 32),
         (2000, 4130, 66, 32), (2500, 4097, 60, 128), (3000, 2100, 7, 32), (52000, 260, 7, 32), (2000, 2100, 2570, 32), (2048, 2048, 2560, 128)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k,group", GEMMS)
def test_gemm(t, n, k, group, dt):
    W0 = random_weights(n, k, 7 * n + k)
    c, s = plain_cut(W0, group, dt)
    codes, scales = pack(c).to(DEV), s.to(DEV)
    X0 = tokens(t, k, dt, t + k)
    W = weights64(c, s, group).t()
    ws = oz.alloc_q4_workspace(t, n, k, group, dt)
    ws.fill_(0xFF)     # NaN in every type: what is read has been written
    for extra, offset in ((0, 0), (3, 1), (16, 8)):
        X, _ = padded(t, k, dt, extra, offset, fill=float("nan"))
        X.copy_(X0)
        Y, ybuf = padded(t, n, dt, extra, offset)
        oz.q4_gemm(X, codes, scales, group, Y, ws)
        check(Y, X0, W, dt, k, t > 16)
        assert (ybuf[:offset] == 77).all() and (ybuf[offset:offset + t * (n + extra)].view(t, -1)[:, n:] == 77).all() and (ybuf[offset + t * (n + extra):] == 77).all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k,group", [(1, 1, 1, 32), (1, 500, 300, 64), (7, 64, 64, 32), (16, 100, 1000, 128), (100, 33, 257, 64), (129, 128, 96, 128), (333, 150, 1000, 32),
                                         (1000, 320, 700, 64), (2100, 192, 4200, 128), (3800, 100, 3700, 64)])
def test_gradient(t, n, k, group, dt):
    c, s = plain_cut(random_weights(n, k, 3 * n + k), group, dt)
    codes, scales = pack(c).to(DEV), s.to(DEV)
    D0 = tokens(t, n, dt, t + n)
    W = weights64(c, s, group)
    ws = oz.alloc_q4_workspace(t, n, k, group, dt, gradient=True)
    ws.fill_(0xFF)
    for extra, offset in ((0, 0), (3, 1), (16, 8)):
        D, _ = padded(t, n, dt, extra, offset, fill=float("nan"))
        D.copy_(D0)
        R, rbuf = padded(t, k, dt, extra, offset)
        oz.q4_gemm_grad(D, codes, scales, group, R, ws)
        check(R, D0, W, dt, n, True)
        assert (rbuf[:offset] == 77).all() and (rbuf[offset:offset + t * (k + extra)].view(t, -1)[:, k:] == 77).all() and (rbuf[offset + t * (k + extra):] == 77).all()


@pytest.mark.parametrize("t", [4, 50])
def test_gradient_against_differences(t):
    """<dY, Y(X + E) - Y(X)> = <dX, E>: the product is linear, so the difference has no higher terms. Each side is a sum of t n (t k) products that are off by at most what
    test_gemm allows; the norms below bound it."""
    n, k, group = 96, 160, 32
    c, s = plain_cut(random_weights(n, k, 1), group, F32)
    codes, scales = pack(c).to(DEV), s.to(DEV)
    X, E, D = (tokens(t, cols, F32, seed).to(DEV) for cols, seed in ((k, 1), (k, 2), (n, 3)))
    ws = oz.alloc_q4_workspace(t, n, k, group, F32, gradient=True)
    wf = oz.alloc_q4_workspace(t, n, k, group, F32)
    Y0, Y1, R = torch.empty(t, n, device=DEV), torch.empty(t, n, device=DEV), torch.empty(t, k, device=DEV)
    oz.q4_gemm(X, codes, scales, group, Y0, wf)
    oz.q4_gemm(X + E, codes, scales, group, Y1, wf)
    oz.q4_gemm_grad(D, codes, scales, group, R, ws)
    left = (D.double() * (Y1.double() - Y0.double())).sum()
    right = (R.double() * E.double()).sum()
    W = weights64(c, s, group).to(DEV).abs()
    size = (D.double().abs() * ((2 * X.double().abs() + E.double().abs()) @ W.t())).sum() + ((D.double().abs() @ W) * E.double().abs()).sum()
    assert abs(left - right) <= (max(n, k) + 16) * 2.0 ** -24 * size
    assert abs(left) > 1e3 * (max(n, k) + 16) * 2.0 ** -24       # (there is something to compare)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t", [3, 40])
def test_empty_inner_dimension_gives_zeros(t, dt):
    Y, buf = padded(t, 70, dt, 2, 1)
    oz.q4_gemm(torch.empty(t, 0, dtype=dt, device=DEV), torch.empty(70, 0, dtype=torch.uint8, device=DEV), torch.empty(70, 0, dtype=dt, device=DEV), 32, Y)
    assert (Y == 0).all() and int((buf == 0).sum()) == t * 70
    R, buf = padded(t, 70, dt, 2, 1)
    oz.q4_gemm_grad(torch.empty(t, 0, dtype=dt, device=DEV), torch.empty(0, 48, dtype=torch.uint8, device=DEV), torch.empty(0, 3, dtype=dt, device=DEV), 32, R, None)
    assert (R == 0).all() and int((buf == 0).sum()) == t * 70


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n", [(5, 100), (70, 100), (300, 2000)])
def test_a_row_that_is_not_finite_stays_alone(t, n, dt):
    k, group = 200, 64
    c, s = plain_cut(random_weights(n, k, 9), group, dt)
    codes, scales = pack(c).to(DEV), s.to(DEV)
    for grad in (False, True):
        V = tokens(t, n if grad else k, dt, 4).to(DEV)
        ws = oz.alloc_q4_workspace(t, n, k, group, dt, gradient=grad)
        f = oz.q4_gemm_grad if grad else oz.q4_gemm
        clean = torch.empty(t, k if grad else n, dtype=dt, device=DEV)
        f(V, codes, scales, group, clean, ws)
        bad = V.clone()
        bad[1, 17] = float("nan")
        bad[3, 0] = float("inf")
        out = torch.empty_like(clean)
        f(bad, codes, scales, group, out, ws)
        rest = [i for i in range(t) if i not in (1, 3)]
        assert torch.equal(out[rest], clean[rest]) and out[1].isnan().all() and not out[3].isfinite().any()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("n,k", [(30, 700), (2100, 600), (8200, 1025)])
def test_one_of_two_tokens_is_not_finite(n, k, dt):
    c, s = plain_cut(random_weights(n, k, 9), 32, dt)
    codes, scales = pack(c).to(DEV), s.to(DEV)
    V = tokens(2, k, dt, 4).to(DEV)
    clean, out = (torch.empty(2, n, dtype=dt, device=DEV) for _ in range(2))
    oz.q4_gemm(V, codes, scales, 32, clean)
    for at, value in ((0, "nan"), (k - 1, "nan"), (17, "inf")):
        bad = V.clone()
        bad[1, at] = float(value)
        oz.q4_gemm(bad, codes, scales, 32, out)
        # (an infinity times a code of zero is NaN, which the formula gives too)
        assert torch.equal(out[0], clean[0]) and (out[1].isnan().all() if value == "nan" else not out[1].isfinite().any())


@pytest.mark.parametrize("dt", [F32, BF16])
def test_large_and_small_values(dt):
    """Rows of tokens of very different size, up to the ends of the type's range: each keeps its relative precision."""
    t, n, k, group = 40, 64, 256, 32
    c, s = plain_cut(random_weights(n, k, 2), group, dt)
    X0 = tokens(t, k, F32, 8) / 64
    X0 = (X0 * torch.logspace(-30, 30, t)[:, None]).to(dt)
    Y = torch.empty(t, n, dtype=dt, device=DEV)
    oz.q4_gemm(X0.to(DEV), pack(c).to(DEV), s.to(DEV), group, Y, oz.alloc_q4_workspace(t, n, k, group, dt))
    check(Y, X0, weights64(c, s, group).t(), dt, k, True)
    R = torch.empty(t, k, dtype=dt, device=DEV)
    D0 = (tokens(t, n, F32, 3) / 64 * torch.logspace(-30, 30, t)[:, None]).to(dt)
    # columns of W of very different size: the exponent goes with the group
    s2 = (s.float() * torch.logspace(-4, 4, s.shape[1])).to(dt)
    oz.q4_gemm_grad(D0.to(DEV), pack(c).to(DEV), s2.to(DEV), group, R, oz.alloc_q4_workspace(t, n, k, group, dt, gradient=True))
    check(R, D0, weights64(c, s2, group), dt, n, True)


@pytest.mark.parametrize("t,n,k", [(3, 50, 300), (400, 2000, 300), (2100, 4200, 192), (2000, 2100, 2570)])
def test_subnormal_values_of_sixteen_bits(t, n, k):
    """Tokens below 2^-14 and weights below it too are not normal in fp16: their bits count all the same. (Results are exact multiples of 2^-48 near 2^-24 and come out as multiples of
    2^-24: the bound is half of that, and what check counts for normal values.)"""
    c, s = plain_cut(random_weights(n, k, 3) * 2.0 ** -9, 64, F16)
    X0 = (tokens(t, k, F32, 2) * 2.0 ** -10).to(F16)
    D0 = (tokens(t, n, F32, 3) * 2.0 ** -10).to(F16)
    assert (X0.abs() < 2.0 ** -14).any() and (s < 2.0 ** -14).any()
    W = weights64(c, s, 64)
    W16 = W.to(F16).double()     # (a weight that is not normal is off by up to half of 2^-24)
    for V, M, M16, grad in ((X0, W.t(), W16.t(), False), (D0, W, W16, True)):
        R = torch.empty(t, M.shape[1], dtype=F16, device=DEV)
        (oz.q4_gemm_grad if grad else oz.q4_gemm)(V.to(DEV), pack(c).to(DEV), s.to(DEV), 64, R, oz.alloc_q4_workspace(t, n, k, 64, F16, gradient=grad))
        want, terms = V.double() @ M, V.double().abs() @ M.abs()
        # weights rounded to 16 bits with many tokens (their own difference, exactly), sums in 32 bits with the codes' offset, one rounding
        near = V.double() @ M16 if grad or t > 16 else want
        bound = (M.shape[0] + 8) * 2.0 ** -24 * 6 * terms + 2.0 ** -25 + half_step(F16) * near.abs()
        assert ((R.cpu().double() - near).abs() <= bound * (1 + 1e-6)).all()


@pytest.mark.parametrize("dt", TYPES)
def test_other_stream_and_replayed_graph(dt):
    """One call on a stream of its own, and prompt, token, gradient and a new cut captured into one graph that shares a workspace, replayed with other inputs."""
    t, n, k, group = 70, 300, 500, 64
    W = random_weights(n, k, 1).to(dt).to(DEV)
    codes, scales = device_cut(W, group, dt)
    X, D = tokens(t, k, dt, 1).to(DEV), tokens(t, n, dt, 2).to(DEV)
    ws = oz.alloc_q4_workspace(t, n, k, group, dt, gradient=True)
    ws = torch.empty(max(ws.numel(), oz.q4_workspace_bytes(t, n, k, group, dt)), dtype=torch.uint8, device=DEV)
    Y, y1, R = torch.empty(t, n, dtype=dt, device=DEV), torch.empty(1, n, dtype=dt, device=DEV), torch.empty(t, k, dtype=dt, device=DEV)

    def work():
        oz.q4_split(W, group, codes, scales)
        oz.q4_gemm(X, codes, scales, group, Y, ws)
        oz.q4_gemm(X[:1], codes, scales, group, y1)
        oz.q4_gemm_grad(D, codes, scales, group, R, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    eager = [x.clone() for x in (codes, scales, Y, y1, R)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        work()
    first = [x.clone() for x in (W, X, D)]
    for round_ in range(3):
        for x, f in zip((W, X, D), first):
            x.copy_(f * (1 + round_))       # twice and three times: other inputs
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (codes, scales, Y, y1, R)]
        work()
        torch.cuda.synchronize()
        for a, b in zip(got, (codes, scales, Y, y1, R)):
            assert torch.equal(a, b)
        if round_ == 0:
            for a, b in zip(got, eager):
                assert torch.equal(a, b)


def test_repeated_calls_give_the_same_bits():
    t, n, k, group = 13, 1000, 3000, 32
    c, s = plain_cut(random_weights(n, k, 1), group, F16)
    X, Y = tokens(t, k, F16, 1).to(DEV), torch.empty(2, t, n, dtype=F16, device=DEV)
    for i in range(2):
        oz.q4_gemm(X, pack(c).to(DEV), s.to(DEV), group, Y[i])
    assert torch.equal(Y[0], Y[1])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k", [(17, 1, 40), (300, 257, 2500), (2000, 2100, 2570), (64, 70, 9000), (700, 520, 1000)])
def test_nothing_beyond_the_workspace_is_written(t, n, k, dt):
    c, s = plain_cut(random_weights(n, k, 5), 32, dt)
    codes, scales = pack(c).to(DEV), s.to(DEV)
    for grad in (False, True):
        need = oz.q4_workspace_bytes(t, n, k, 32, dt, gradient=grad)
        room = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
        V = tokens(t, n if grad else k, dt, 2)
        R = torch.empty(t, k if grad else n, dtype=dt, device=DEV)
        (oz.q4_gemm_grad if grad else oz.q4_gemm)(V.to(DEV), codes, scales, 32, R, room[:need] if need else None)
        assert (room[need:] == 0x5A).all()
        W = weights64(c, s, 32)
        check(R, V, W if grad else W.t(), dt, n if grad else k, True)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k,group", [(1, 40, 700, 32), (2, 2100, 600, 64), (9, 100, 333, 128), (30, 60, 2500, 32), (300, 2000, 100, 64), (1100, 1000, 500, 32), (2000, 2100, 2570, 64)])
def test_codes_and_scales_inside_larger_arrays(t, n, k, group, dt):
    """Rows of codes and scales further apart than they need be; what lies between them is not read for anything and not written."""
    W0 = random_weights(n, k, 11).to(dt)
    rb, groups = oz.q4_geometry(k, group)
    code_room = torch.full((n, rb + 48), 0x5A, dtype=torch.uint8, device=DEV)
    scale_room = torch.full((n, groups + 3), float("nan"), dtype=dt, device=DEV)
    codes, scales = code_room[:, 16:16 + rb], scale_room[:, 1:1 + groups]
    oz.q4_split(W0.to(DEV), group, codes, scales)
    tight_codes, tight_scales = device_cut(W0.to(DEV), group, dt)
    assert torch.equal(codes, tight_codes[:, :rb]) and torch.equal(scales, tight_scales)
    assert (code_room[:, :16] == 0x5A).all() and (code_room[:, 16 + rb:] == 0x5A).all() and scale_room[:, 0].isnan().all() and scale_room[:, 1 + groups:].isnan().all()
    back, tight_back = torch.empty(n, k, dtype=dt, device=DEV), torch.empty(n, k, dtype=dt, device=DEV)
    oz.q4_expand(codes, scales, group, back)
    oz.q4_expand(tight_codes, tight_scales, group, tight_back)
    assert torch.equal(back, tight_back)
    for grad in (False, True):
        V = tokens(t, n if grad else k, dt, 3).to(DEV)
        R = torch.empty(2, t, k if grad else n, dtype=dt, device=DEV)
        f, ws = oz.q4_gemm_grad if grad else oz.q4_gemm, oz.alloc_q4_workspace(t, n, k, group, dt, gradient=grad)
        f(V, codes, scales, group, R[0], ws)
        f(V, tight_codes, tight_scales, group, R[1], ws)
        assert R.isfinite().all() and torch.equal(R[0], R[1])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k", [(2, 50, 600), (16, 50, 200), (70, 300, 90), (140, 2500, 70), (130, 1100, 400)])
def test_rows_as_far_apart_as_allowed(t, n, k, dt):
    """Tokens and results 2^24 values apart: the last rows lie beyond 32-bit offsets."""
    ld = 1 << 24
    c, s = plain_cut(random_weights(n, k, 5), 32, dt)
    codes, scales = pack(c).to(DEV), s.to(DEV)
    for grad in (False, True):
        rows, cols = (n, k) if grad else (k, n)
        V0 = tokens(t, rows, dt, 7)
        room = torch.empty((t - 1) * ld + max(rows, cols), dtype=dt, device=DEV)
        V, tight, R = room.as_strided((t, rows), (ld, 1)), V0.to(DEV), torch.empty(t, cols, dtype=dt, device=DEV)
        V.copy_(V0)
        f, ws = oz.q4_gemm_grad if grad else oz.q4_gemm, oz.alloc_q4_workspace(t, n, k, 32, dt, gradient=grad)
        f(tight, codes, scales, 32, R, ws)
        far = torch.empty_like(R)
        f(V, codes, scales, 32, far, ws)
        assert torch.equal(far, R)
        out = room.as_strided((t, cols), (ld, 1))
        f(tight, codes, scales, 32, out, ws)
        assert torch.equal(out, R)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k", [(1, 90, 100), (1, 90, 700), (2, 90, 700), (5, 90, 333), (40, 90, 2300), (300, 2000, 100), (2000, 2100, 2570)])
def test_weights_that_are_not_finite(t, n, k, dt):
    """The weights of a group with an infinity or a NaN are NaN: so are their output and, on the way back, their group's positions; everything else is what it was."""
    W = random_weights(n, k, 13).to(dt)
    bad = W.clone()
    bad[3, 10], bad[7, k - 1] = float("inf"), float("nan")
    clean, broken = device_cut(W.to(DEV), 32, dt), device_cut(bad.to(DEV), 32, dt)
    for grad in (False, True):
        V = tokens(t, n if grad else k, dt, 3).to(DEV)
        R = torch.empty(2, t, k if grad else n, dtype=dt, device=DEV)
        for (codes, scales), out in zip((clean, broken), R):
            (oz.q4_gemm_grad if grad else oz.q4_gemm)(V, codes, scales, 32, out, oz.alloc_q4_workspace(t, n, k, 32, dt, gradient=grad))
        hit = torch.zeros(R.shape[2], dtype=torch.bool, device=DEV)
        if grad:
            hit[:32] = hit[(k - 1) // 32 * 32:] = True
        else:
            hit[3] = hit[7] = True
        assert R[0].isfinite().all() and R[1][:, hit].isnan().all() and torch.equal(R[1][:, ~hit], R[0][:, ~hit])
