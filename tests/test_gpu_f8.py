"""Products in 8-bit floating point against plain 64-bit forms: the cut and its inverse exactly, products of small integers exactly, others within
bounds that count what is dropped."""
import math

import pytest
import torch

from f8_plain import BF16, F16, F32, TYPES, cut, cut_columns, decode, e4m3, exponents, guarded, half_step, round_to, small_integers, spread, untouched
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def weights(n, k, seed):
    g = gen(seed)
    return torch.randn(n, k, generator=g) * torch.exp(torch.randn(n, 1, generator=g)) / math.sqrt(k)


def device_cut(W, block_rows=128):
    n, k = W.shape
    codes = torch.full((n, oz.f8_row_bytes(k)), 0x5A, dtype=torch.uint8, device=DEV)
    scales = torch.full((-(-n // block_rows), oz.f8_scale_bytes(k)), 0x5A, dtype=torch.uint8, device=DEV)
    oz.f8_split(W.to(DEV), codes, scales, block_rows)
    return codes, scales


# ---------------------------------------------------------------- the cut
SPLITS = [(1, 1), (1, 127), (3, 128), (5, 129), (17, 1000), (129, 513), (128, 512), (300, 257), (9, 4096), (2, 20000)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("n,k", SPLITS)
def test_split_and_expand(n, k, block_rows, dt):
    W0 = weights(n, k, n * 31 + k).to(dt)
    e, c, v = cut(W0, block_rows)
    for extra, offset in ((0, 0), (5, 3), (8, 8)):
        W, _ = guarded(n, k, dt, extra, offset)
        W.copy_(W0)
        rb, sb, rows = oz.f8_row_bytes(k), oz.f8_scale_bytes(k), -(-n // block_rows)
        codes = torch.full((n, rb + 16), 0x5A, dtype=torch.uint8, device=DEV)
        scales = torch.full((rows, sb + 4), 0x5A, dtype=torch.uint8, device=DEV)
        oz.f8_split(W, codes, scales, block_rows)
        assert torch.equal(scales[:, :e.shape[1]].cpu().int() - 127, e)
        assert not scales[:, e.shape[1]:sb].any() and (scales[:, sb:] == 0x5A).all()
        assert torch.equal(decode(codes[:, :k].contiguous()), c)
        assert not codes[:, k:rb].any() and (codes[:, rb:] == 0x5A).all()
        for out_dt in TYPES:
            out, buf = guarded(n, k, out_dt, extra, offset)
            oz.f8_expand(codes, scales, out, block_rows)
            assert torch.equal(out.cpu(), round_to(v, out_dt))      # (32 bits hold every value)
            assert untouched(buf, n, k, extra, offset)


@pytest.mark.parametrize("dt", TYPES)
def test_split_at_borders_and_extremes(dt):
    """Ties and their neighbours, largest values on and next to 448 2^e, zeros, subnormal values, infinities and NaN."""
    rows = []
    g = gen(5)
    finfo = torch.finfo(dt)
    for top in (448.0, 449.0, 447.0, 1.0, 1.75, 1.7500001, 2.0 ** -20, 2.0 ** -127, 2.0 ** -140, 2.0 ** -149, finfo.max, finfo.tiny, finfo.smallest_normal * 3, 0.0):
        row = torch.randn(128, generator=g) * top / 8
        e = exponents(torch.tensor([[float(torch.tensor(top).to(dt))]]), 1)[0, 0]
        for i in range(60):      # midpoints between codes, and what is next to them
            a = e4m3(torch.tensor([2.0 ** (i / 4 - 10)], dtype=torch.float64))[0]
            step = 2.0 ** (max(math.floor(math.log2(float(a))) if a > 0 else -6, -6) - 3)
            mid = torch.ldexp(torch.tensor(float(a) + step / 2, dtype=torch.float64), e).to(F32)
            row[2 * i] = mid.clamp(-top, top)
            row[2 * i + 1] = torch.nextafter(mid, torch.tensor(math.inf if i & 1 else 0.0)).clamp(-top, top)
        row[127] = -top
        rows.append(row)
    for bad in (math.inf, -math.inf, math.nan):
        row = torch.randn(128, generator=g)
        row[11] = bad
        rows.append(row)
    W = torch.stack(rows).to(dt)
    for block_rows, part in ((1, W), (128, W[:-3]), (128, W)):
        codes, scales = device_cut(part, block_rows)
        e, c, v = cut(part, block_rows)
        assert torch.equal(scales[:, :1].cpu().int() - 127, e)
        assert torch.equal(decode(codes).nan_to_num(nan=1e9), c.nan_to_num(nan=1e9))
        out = torch.empty(part.shape, dtype=F32, device=DEV)
        oz.f8_expand(codes, scales, out, block_rows)
        assert torch.equal(out.cpu().nan_to_num(nan=1e9), round_to(v, F32).nan_to_num(nan=1e9))


def test_types_of_eight_bits_and_wide_scales():
    """torch's own types for codes and scales; 32-bit scales made elsewhere, subnormal, negative and not finite ones among them."""
    n, k = 200, 300
    W = weights(n, k, 3)
    codes, scales = device_cut(W)
    codes8, scales8 = torch.zeros_like(codes).view(torch.float8_e4m3fn), torch.zeros_like(scales).view(torch.float8_e8m0fnu)
    oz.f8_split(W.to(DEV), codes8, scales8)
    assert torch.equal(codes8.view(torch.uint8), codes) and torch.equal(scales8.view(torch.uint8), scales)
    assert torch.equal(codes8.float()[:, :k].cpu().double(), cut(W, 128)[1])
    wide = torch.tensor([[0.3, -1.7, 2.0 ** -130], [math.inf, 3e38, math.nan]], device=DEV)
    out = torch.empty(n, k, device=DEV)
    oz.f8_expand(codes8, wide, out)
    want = (decode(codes)[:, :k].to(F32) * wide.cpu().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k])
    got = out.cpu()
    bad = ~torch.isfinite(wide.cpu()).repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    assert got[bad].isnan().all()
    assert torch.equal(got[~bad], want[~bad])
    bytes_ = scales.clone()
    bytes_[0, 1] = 255
    oz.f8_expand(codes, bytes_, out)
    assert out[:128, 128:256].isnan().all() and not out[:, :128].isnan().any()


# ---------------------------------------------------------------- products
SIZES = [(1, 1, 1), (1, 17, 128), (3, 130, 129), (16, 64, 512), (17, 100, 513), (33, 256, 640), (130, 129, 1000), (257, 300, 384), (64, 1000, 2048), (300, 70, 5000), (513, 515, 130)]


def exact_products(t, n, k, dt, out_dt, seed, extra=0, offset=0, wide=False):
    """Y = X W^T of small integers: every sum is exact, so the result is one rounding."""
    g = gen(seed)
    X0, W0 = small_integers((t, k), g), small_integers((n, k), g)
    X, _ = guarded(t, k, dt, extra, offset)
    X.copy_(X0)
    codes, scales = device_cut(W0.to(F32))
    e = scales[:, :-(-k // 128)].cpu().int() - 127
    W1 = W0
    if wide:      # scales that are no powers of two: integers up to 3
        m = torch.randint(1, 4, e.shape, generator=g) * torch.where(torch.rand(e.shape, generator=g) < 0.3, -1, 1)
        scales = (torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e) * m).to(F32).to(DEV)
        W1 = W0 * spread(m, n, k, 128)
    Y, buf = guarded(t, n, out_dt, extra, offset)
    ws = oz.alloc_f8_workspace("gemm", t, n, k, dt)
    oz.f8_gemm(X, codes, scales, Y, ws)
    assert torch.equal(Y.cpu(), round_to(X0 @ W1.t(), out_dt))
    assert untouched(buf, t, n, extra, offset)
    # the gradient
    dY0 = small_integers((t, n), g)
    dY, _ = guarded(t, n, dt, extra, offset)
    dY.copy_(dY0)
    dX, buf = guarded(t, k, out_dt, extra, offset)
    oz.f8_gemm_grad(dY, codes, scales, dX, oz.alloc_f8_workspace("grad", t, n, k, dt))
    assert torch.equal(dX.cpu(), round_to(dY0 @ W1, out_dt))
    assert untouched(buf, t, k, extra, offset)
    # that of the weights
    dW, buf = guarded(n, k, out_dt, extra, offset)
    oz.f8_weight_grad(dY, X, dW, oz.alloc_f8_workspace("weight_grad", t, n, k, dt))
    assert torch.equal(dW.cpu(), round_to(dY0.t() @ X0, out_dt))
    assert untouched(buf, n, k, extra, offset)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k", SIZES)
def test_products_of_integers(t, n, k, dt):
    exact_products(t, n, k, dt, dt, t * 7 + n + k)
    exact_products(t, n, k, dt, dt, t * 7 + n + k + 1, extra=3, offset=1)


@pytest.mark.parametrize("out_dt", TYPES)
@pytest.mark.parametrize("t,n,k", [(5, 130, 300), (200, 300, 700)])
def test_products_of_integers_wide_scales_and_other_results(t, n, k, out_dt):
    exact_products(t, n, k, BF16, out_dt, 11, wide=True)
    exact_products(t, n, k, F32, out_dt, 12, extra=4, offset=4)


def bound(A, B, inner, out, exact):
    """Half a step of the result; every addition of the sums may lose a unit of 32 bits of the magnitudes' sum; the matrix cores' 8-bit products drop
    less than 2^-13 of the largest of eight for each of them."""
    magnitude = A.abs() @ B.abs().t()
    return magnitude * ((inner + 8) * 2.0 ** -23 + (0.0 if exact else 2.0 ** -12))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k", [(1, 300, 1000), (16, 130, 4000), (40, 200, 777), (300, 400, 1500)])
def test_products_of_reals(t, n, k, dt):
    g = gen(t + n)
    X = (torch.randn(t, k, generator=g) * torch.exp(2 * torch.randn(1, k, generator=g))).to(dt)
    W = weights(n, k, k)
    dY = (torch.randn(t, n, generator=g) * torch.exp(torch.randn(t, 1, generator=g))).to(dt)
    codes, scales = device_cut(W)
    V, U = cut(W, 128)[2], cut(X)[2]
    D = cut(dY)[2]
    exact = dt == F32
    for got, A, B, sure in (
            (product("gemm", X, codes, scales, (t, n), dt), U, V, exact or t <= 16),
            (product("grad", dY, codes, scales, (t, k), dt), D, V.t(), exact or t <= 16),
            (weight_product(dY, X, dt), cut_columns(dY).t(), cut_columns(X).t(), exact)):
        want = A @ B.t()
        allowed = bound(A, B, A.shape[1], dt, sure) + want.abs() * half_step(dt) + torch.finfo(dt).smallest_normal * half_step(dt)
        # what rounds to an infinity is one (fp16: from 65520 on), and may be one where the bound reaches that far
        got, edge = got.double().cpu(), torch.finfo(dt).max * (1 + half_step(dt))
        infinite = got.isinf() & (got.sign() == want.sign())
        assert infinite[want.abs() - allowed >= edge].all() and (want.abs() + allowed >= edge)[infinite].all()
        assert ((got - want).abs() <= allowed * (1 + 2.0 ** -10))[~infinite].all()


def product(op, V, codes, scales, shape, dt, **more):
    out = torch.full(shape, 77.0, dtype=dt, device=DEV)
    k = shape[1] if op == "grad" else V.shape[1]
    n = V.shape[1] if op == "grad" else shape[1]
    experts = more["offsets"].numel() - 1 if more.get("offsets") is not None else 0
    ws = oz.alloc_f8_workspace(op, V.shape[0], n, k, V.dtype, rows=shape[0], experts=experts)
    (oz.f8_gemm_grad if op == "grad" else oz.f8_gemm)(V.to(DEV), codes, scales, out, ws, **more)
    return out


def weight_product(dY, X, dt, experts=0, **more):
    n, k = dY.shape[1], X.shape[1]
    dW = torch.full((experts, n, k) if experts else (n, k), 77.0, dtype=dt, device=DEV)
    oz.f8_weight_grad(dY.to(DEV), X.to(DEV), dW, oz.alloc_f8_workspace("weight_grad", X.shape[0], n, k, X.dtype, rows=dY.shape[0], experts=experts), **more)
    return dW


@pytest.mark.parametrize("t", [4, 150])
def test_codes_given_equal_codes_made(t):
    """Tokens that the program has cut itself give the same bits; so do equal calls."""
    n, k = 300, 700
    g = gen(t)
    X = torch.randn(t, k, generator=g, device="cpu").to(BF16)
    codes, scales = device_cut(weights(n, k, 1))
    xc, xs = device_cut(X, 1)
    for dt in (BF16, F32):
        a = product("gemm", X, codes, scales, (t, n), dt)
        b = torch.empty_like(a)
        oz.f8_gemm(xc, codes, scales, b, x_scales=xs)
        assert torch.equal(a, b)
        oz.f8_gemm(xc.view(torch.float8_e4m3fn), codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), b, x_scales=xs.view(torch.float8_e8m0fnu))
        assert torch.equal(a, b)
        assert torch.equal(a, product("gemm", X, codes, scales, (t, n), dt))
    dY = torch.randn(t, n, generator=g).to(BF16)
    dc, ds = device_cut(dY, 1)
    a = product("grad", dY, codes, scales, (t, k), BF16)
    b = torch.empty_like(a)
    oz.f8_gemm_grad(dc, codes, scales, b, oz.alloc_f8_workspace("grad", t, n, k, torch.uint8), dy_scales=ds)
    assert torch.equal(a, b)


@pytest.mark.parametrize("t", [5, 150])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_nan_stays_in_its_row(t, dt):
    n, k = 200, 500
    X, W = torch.randn(t, k, generator=gen(1)).to(dt), weights(n, k, 2)
    codes, scales = device_cut(W)
    clean = product("gemm", X, codes, scales, (t, n), dt)
    for bad in (math.nan, math.inf):
        X2 = X.clone()
        X2[3, 200] = bad
        # beside it everything is what it would be with another finite value there that leaves the scale alone
        X3 = X.clone()
        X3[3, 200] = 0
        got = product("gemm", X2, codes, scales, (t, n), dt)
        assert got[3].isnan().all()
        rest = [i for i in range(t) if i != 3]
        assert torch.equal(got[rest], clean[rest])
        W2 = W.clone()
        W2[7, 10] = bad
        c2, s2 = device_cut(W2)
        got = product("gemm", X, c2, s2, (t, n), dt)
        assert got[:, 7].isnan().all() and not got[:, :7].isnan().any() and not got[:, 8:].isnan().any()
    s2 = scales.clone()
    s2[1, 2] = 255
    got = product("gemm", X, codes, s2, (t, n), dt)
    assert got[:, 128:].isnan().all() and torch.equal(got[:, :128], clean[:, :128])


@pytest.mark.parametrize("t", [5, 150, 2100])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_nan_scale_of_a_token(t, dt):
    """A byte of 255 among the scales of given codes is a NaN for its row, whatever the other scale is."""
    n, k = 2300, 700
    codes, scales = device_cut(weights(n, k, 2))
    xc, xs = device_cut(torch.randn(t, k, generator=gen(1)), 1)
    clean, got = torch.empty(t, n, dtype=dt, device=DEV), torch.empty(t, n, dtype=dt, device=DEV)
    ws = oz.alloc_f8_workspace("gemm", t, n, k, torch.uint8)
    oz.f8_gemm(xc, codes, scales, clean, ws, x_scales=xs)
    xs[2, 4], scales[0, 4] = 255, 0
    xs[3, 4] = 254
    oz.f8_gemm(xc, codes, scales, got, ws, x_scales=xs)
    assert got[2].isnan().all() and not got[[i for i in range(t) if i != 2]].isnan().any()
    rest = [i for i in range(t) if i not in (2, 3)]
    assert torch.equal(got[rest][:, 128:], clean[rest][:, 128:])


@pytest.mark.parametrize("t", [5, 150])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_scales_far_apart(t, dt):
    """Tokens and weights whose scales meet only in their product; zero codes under scales whose product overflows."""
    n, k = 130, 256
    g = gen(9)
    X0, W0 = small_integers((t, k), g), small_integers((n, k), g)
    for down in (-100, -60, 60, 100):
        X, W = torch.ldexp(X0, torch.tensor(down)).to(dt), torch.ldexp(W0, torch.tensor(-down)).to(F32)
        codes, scales = device_cut(W)
        assert torch.equal(product("gemm", X, codes, scales, (t, n), dt).cpu(), round_to(X0 @ W0.t(), dt))
    X, W = X0.clone(), W0.clone()
    X[:, 0], W[:, 0] = 2.0 ** 100, 0.0
    W[:, 1], X[:, 1] = 2.0 ** 100, 0.0
    X[:, 2:], W[:, 2:] = 0, 0      # 2^100 meets 0 only
    codes, scales = device_cut(W.to(F32))
    assert not product("gemm", X.to(dt), codes, scales, (t, n), dt).any()


def test_empty_inner_dimension_and_no_rows():
    codes, scales = torch.zeros(5, 0, dtype=torch.uint8, device=DEV), torch.zeros(1, 0, dtype=torch.uint8, device=DEV)
    for t in (3, 40):
        for dt in TYPES:
            Y = torch.full((t, 5), 77.0, dtype=dt, device=DEV)
            oz.f8_gemm(torch.empty(t, 0, dtype=dt, device=DEV), codes, scales, Y)
            assert not Y.any()
    dW = torch.full((7, 9), 77.0, device=DEV)
    oz.f8_weight_grad(torch.empty(0, 7, device=DEV), torch.empty(0, 9, device=DEV), dW, None)
    assert not dW.any()
    oz.f8_gemm(torch.empty(0, 128, device=DEV), torch.zeros(5, 128, dtype=torch.uint8, device=DEV), torch.zeros(1, 4, dtype=torch.uint8, device=DEV), torch.empty(0, 5, device=DEV))


# ---------------------------------------------------------------- over experts
def expert_case(counts, n, k, t, behind, seed, by_source=True):
    g = gen(seed)
    E, rows = len(counts), sum(counts) + behind
    offsets = torch.tensor([sum(counts[:e]) for e in range(E + 1)], dtype=torch.int32)
    source = torch.randint(0, t, (rows,), generator=g, dtype=torch.int32) if by_source else None
    X = small_integers((t if by_source else rows, k), g)
    W = torch.stack([small_integers((n, k), g) for _ in range(E)])
    cut_w = [device_cut(w.to(F32)) for w in W]
    codes, scales = torch.stack([c for c, _ in cut_w]), torch.stack([s for _, s in cut_w])
    dY = small_integers((rows, n), g)
    return offsets, source, X, W, codes, scales, dY


CASES = [([3, 0, 5, 1], 40, 130, 6, 0), ([0, 0, 0], 20, 128, 3, 4), ([1] * 70, 33, 200, 9, 2), ([200, 0, 17, 130, 1], 150, 300, 64, 11), ([300], 129, 128, 40, 0), ([0, 513, 2], 64, 513, 50, 3),
         ([2] * 300, 16, 128, 30, 1)]


@pytest.mark.parametrize("by_source", [True, False])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("counts,n,k,t,behind", CASES)
def test_experts(counts, n, k, t, behind, dt, by_source):
    offsets, source, X, W, codes, scales, dY = expert_case(counts, n, k, t, behind, len(counts) + n, by_source)
    E, rows, used = len(counts), sum(counts) + behind, sum(counts)
    if source is not None and rows > 2:
        source[1] = -1          # rows without a token
        source[rows - 1] = t
    o, s = offsets.to(DEV), None if source is None else source.to(DEV)
    Xr = X if source is None else torch.where(((source >= 0) & (source < t))[:, None], X[source.clamp(0, t - 1).long()], torch.zeros((), dtype=torch.float64))
    want = torch.full((rows, n), 77.0, dtype=torch.float64)
    wantx = torch.full((rows, k), 77.0, dtype=torch.float64)
    wantw = torch.zeros(E, n, k, dtype=torch.float64)
    for e in range(E):
        a, b = int(offsets[e]), int(offsets[e + 1])
        want[a:b], wantx[a:b] = Xr[a:b] @ W[e].t(), dY[a:b] @ W[e]
        wantw[e] = dY[a:b].t() @ Xr[a:b]
    assert torch.equal(product("gemm", X.to(dt), codes, scales, (rows, n), dt, offsets=o, source=s).cpu(), round_to(want, dt))
    assert torch.equal(product("grad", dY.to(dt), codes, scales, (rows, k), dt, offsets=o).cpu(), round_to(wantx, dt))
    assert torch.equal(weight_product(dY.to(dt), X.to(dt), dt, E, offsets=o, source=s).cpu(), round_to(wantw, dt))


@pytest.mark.parametrize("counts", [[5, 4, 3], [90, 4, 100]])
def test_experts_wide_scales(counts):
    n, k, t = 140, 300, 20
    offsets, source, X, W, codes, scales, dY = expert_case(counts, n, k, t, 2, 5)
    g = gen(3)
    m = torch.randint(1, 4, scales.shape, generator=g)
    wide = torch.ldexp(m.double(), scales.cpu().int() - 127).to(F32)[:, :, :3].contiguous().to(DEV)
    for dt in (BF16, F32):
        want, wantx = torch.full((sum(counts) + 2, n), 77.0, dtype=torch.float64), torch.full((sum(counts) + 2, k), 77.0, dtype=torch.float64)
        for e in range(3):
            a, b = int(offsets[e]), int(offsets[e + 1])
            We = W[e] * spread(m[e], n, k, 128)
            want[a:b], wantx[a:b] = X[source[a:b].long()] @ We.t(), dY[a:b] @ We
        assert torch.equal(product("gemm", X.to(dt), codes, wide, want.shape, dt, offsets=offsets.to(DEV), source=source.to(DEV)).cpu(), round_to(want, dt))
        assert torch.equal(product("grad", dY.to(dt), codes, wide, wantx.shape, dt, offsets=offsets.to(DEV)).cpu(), round_to(wantx, dt))


@pytest.mark.parametrize("few", [True, False])
def test_offsets_that_leave_their_range(few):
    """An offset is at least the largest before it, and within the rows; nothing outside the ranges is written."""
    n, k, t = 40, 128, 30 if few else 200
    n = n if few else 6000
    g = gen(2)
    X, W = small_integers((t, k), g), torch.stack([small_integers((n, k), g) for _ in range(4)])
    cut_w = [device_cut(w.to(F32)) for w in W]
    codes, scales = torch.stack([c for c, _ in cut_w]), torch.stack([s for _, s in cut_w])
    dY = small_integers((t, n), g)
    for given, taken in (([-5, 10, 7, 20, t + 1000], [0, 10, 10, 20, t]), ([3, 8, 2, 1, 9], [3, 8, 8, 8, 9]), ([t + 7, 5, 6, 7, 8], [t] * 5), ([-9, -8, -7, 4, -1], [0, 0, 0, 4, 4])):
        offsets = torch.tensor(given, dtype=torch.int32, device=DEV)
        want, wantx, wantw = torch.full((t, n), 77.0, dtype=torch.float64), torch.full((t, k), 77.0, dtype=torch.float64), torch.zeros(4, n, k, dtype=torch.float64)
        for e in range(4):
            a, b = taken[e], taken[e + 1]
            want[a:b], wantx[a:b], wantw[e] = X[a:b] @ W[e].t(), dY[a:b] @ W[e], dY[a:b].t() @ X[a:b]
        assert torch.equal(product("gemm", X.to(BF16), codes, scales, (t, n), BF16, offsets=offsets).cpu(), round_to(want, BF16))
        assert torch.equal(product("grad", dY.to(BF16), codes, scales, (t, k), BF16, offsets=offsets).cpu(), round_to(wantx, BF16))
        assert torch.equal(weight_product(dY.to(BF16), X.to(BF16), BF16, 4, offsets=offsets).cpu(), round_to(wantw, BF16))


def test_other_stream_and_graph():
    """A captured call, replayed with new inputs between the program's own work, and calls on a stream of their own."""
    n, k, E = 300, 700, 4
    t, rows = 40, 80
    g = gen(1)
    W = torch.stack([weights(n, k, i) for i in range(E)])
    cut_w = [device_cut(w) for w in W]
    codes, scales = torch.stack([c for c, _ in cut_w]), torch.stack([s for _, s in cut_w])
    X = torch.randn(t, k, generator=g).to(BF16).to(DEV)
    dY = torch.randn(rows, n, generator=g).to(BF16).to(DEV)
    offsets = torch.tensor([0, 30, 30, 71, 80], dtype=torch.int32, device=DEV)
    source = torch.randint(0, t, (rows,), generator=g, dtype=torch.int32).to(DEV)
    Y, dX, dW = torch.empty(rows, n, dtype=BF16, device=DEV), torch.empty(rows, k, dtype=BF16, device=DEV), torch.empty(E, n, k, dtype=BF16, device=DEV)
    wg, wd, ww = (oz.alloc_f8_workspace(op, t if op != "grad" else rows, n, k, BF16, rows=rows, experts=E) for op in ("gemm", "grad", "weight_grad"))

    def step():
        oz.f8_gemm(X, codes, scales, Y, wg, offsets=offsets, source=source)
        oz.f8_gemm_grad(dY, codes, scales, dX, wd, offsets=offsets)
        oz.f8_weight_grad(dY, X, dW, ww, offsets=offsets, source=source)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other = torch.cuda.Stream()
    for i in range(4):
        X.copy_(torch.randn(t, k, generator=g).to(BF16))
        dY.copy_(torch.randn(rows, n, generator=g).to(BF16))
        offsets.copy_(torch.tensor([0, 10 * i, 40, 40 + 5 * i, 80], dtype=torch.int32))
        step()
        want = [x.clone() for x in (Y, dX, dW)]
        for x in (Y, dX, dW):
            x.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((Y, dX, dW), want))
        for x in (Y, dX, dW):
            x.fill_(77)
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            step()
        torch.cuda.current_stream().wait_stream(other)
        assert all(torch.equal(a, b) for a, b in zip((Y, dX, dW), want))
