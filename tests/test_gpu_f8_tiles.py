"""Products in 8-bit floating point of more rows than the direct kernel takes, against 64-bit products of the same small integers (whose sums are exact): tiles of
every size, shared walks, over experts, along the tokens, with odd sizes and strides."""
import math

import pytest
import torch

from f8_plain import BF16, F16, F32, TYPES, guarded, small_integers, untouched
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rounded(x64, dt):
    return x64.to(F32).to(dt)      # (sums below 2^24: 32 bits hold them)


def cut_weights(W, wide):
    """Codes and scales of integer weights (experts x n x k), and the weights that they stand for."""
    E, n, k = W.shape
    codes = torch.empty(E, n, oz.f8_row_bytes(k), dtype=torch.uint8, device=DEV)
    scales = torch.empty(E, -(-n // 128), oz.f8_scale_bytes(k), dtype=torch.uint8, device=DEV)
    for e in range(E):
        oz.f8_split(W[e].float(), codes[e], scales[e])
    if not wide:
        return codes, scales, W
    m = torch.randint(1, 4, (E, scales.shape[1], -(-k // 128)), generator=gen(n)).to(DEV)
    values = torch.ldexp(m.double(), scales[:, :, :m.shape[2]].int() - 127).float()
    return codes, values, W * m.repeat_interleave(128, 1)[:, :n].repeat_interleave(128, 2)[:, :, :k]


# sizes, and the tile that the estimate gives them (16-bit results; 32-bit ones)
DENSE = [(4000, 4090, 4100),      # 256; 128
         (2040, 4090, 4100),      # 128
         (2040, 2050, 4100),      # 64 x 128; 64, a shared rest
         (700, 4030, 1100),       # 64
         (1100, 1030, 1150),      # 32 x 64
         (40, 8190, 8900),        # 64, shared walks
         (130, 2050, 5000)]       # 32 x 64, shared walks


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k", DENSE)
def test_dense(t, n, k, dt):
    for seed, wide, extra, offset in ((1, False, 0, 0), (2, True, 3, 1)):
        g = gen(seed)
        X0, W0, dY0 = small_integers((t, k), g, 3).to(DEV), small_integers((n, k), g, 3).to(DEV), small_integers((t, n), g, 3).to(DEV)
        codes, scales, W = cut_weights(W0[None], wide)
        codes, scales, W = codes[0], scales[0], W[0]
        X, _ = guarded(t, k, dt, extra, offset)
        dY, _ = guarded(t, n, dt, extra, offset)
        X.copy_(X0)
        dY.copy_(dY0)
        Y, ybuf = guarded(t, n, dt, extra, offset)
        oz.f8_gemm(X, codes, scales, Y, oz.alloc_f8_workspace("gemm", t, n, k, dt))
        assert torch.equal(Y, rounded(X0 @ W.t(), dt)) and untouched(ybuf, t, n, extra, offset)
        dX, xbuf = guarded(t, k, dt, extra, offset)
        oz.f8_gemm_grad(dY, codes, scales, dX, oz.alloc_f8_workspace("grad", t, n, k, dt))
        assert torch.equal(dX, rounded(dY0 @ W, dt)) and untouched(xbuf, t, k, extra, offset)


# tokens, n, k of weights' gradients
ALONG = [(4100, 4000, 4090),      # 256; 128
         (4100, 2040, 4090),      # 128
         (5000, 1000, 1500),      # 64
         (600, 130, 8190),        # 32 x 64
         (20000, 300, 200)]       # 64, shared walks


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,n,k", ALONG)
def test_weights_gradients(t, n, k, dt):
    for seed, extra, offset in ((1, 0, 0), (2, 3, 1)):
        g = gen(seed)
        X0, dY0 = torch.randint(-3, 4, (t, k), generator=g).double().to(DEV), torch.randint(-3, 4, (t, n), generator=g).double().to(DEV)
        X, _ = guarded(t, k, dt, extra, offset)
        dY, _ = guarded(t, n, dt, extra, offset)
        X.copy_(X0)
        dY.copy_(dY0)
        dW, buf = guarded(n, k, dt, extra, offset)
        oz.f8_weight_grad(dY, X, dW, oz.alloc_f8_workspace("weight_grad", t, n, k, dt))
        assert torch.equal(dW, rounded(dY0.t() @ X0, dt)) and untouched(buf, n, k, extra, offset)


# rows of each expert, n, k, rows behind the last
EXPERTS = [([4000, 0, 3300, 5000, 4000], 1030, 4200, 3),      # 256 throughout; 128
           ([1200, 3, 1500, 1300, 1000], 1030, 1100, 7),      # 64 x 128 and 64
           ([200] * 15 + [0], 3000, 1100, 0),                 # 64 x 128; 64
           ([14, 0, 30, 1] * 16, 2000, 2100, 5),              # 32 x 64
           ([0, 700, 0], 1100, 130, 1)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("counts,n,k,behind", EXPERTS)
def test_experts(counts, n, k, behind, dt):
    E, used = len(counts), sum(counts)
    rows, t = used + behind, max(3, used // 3)
    for wide, extra in ((False, 0), (True, 2)):
        g = gen(n + wide)
        X0 = torch.randint(-3, 4, (t, k), generator=g).double().to(DEV)
        W0 = torch.stack([torch.randint(-3, 4, (n, k), generator=g) for _ in range(E)]).double().to(DEV)
        dY0 = torch.randint(-3, 4, (rows, n), generator=g).double().to(DEV)
        codes, scales, W = cut_weights(W0, wide)
        source = torch.randint(0, t, (rows,), generator=g, dtype=torch.int32)
        source[2], source[used - 1] = -7, t + 5      # rows without a token
        there = (source >= 0) & (source < t)
        Xr = torch.where(there[:, None].to(DEV), X0[source.clamp(0, t - 1).long().to(DEV)], torch.zeros((), dtype=torch.float64, device=DEV))
        offsets = torch.tensor([sum(counts[:e]) for e in range(E + 1)], dtype=torch.int32, device=DEV)
        source = source.to(DEV)
        X, _ = guarded(t, k, dt, extra, extra)
        dY, _ = guarded(rows, n, dt, extra, extra)
        X.copy_(X0)
        dY.copy_(dY0)
        Y, ybuf = guarded(rows, n, dt, extra, extra)
        dX, xbuf = guarded(rows, k, dt, extra, extra)
        dW = torch.full((E, n, k + extra), 77.0, dtype=dt, device=DEV)[:, :, :k]
        oz.f8_gemm(X, codes, scales, Y, oz.alloc_f8_workspace("gemm", t, n, k, dt, rows=rows, experts=E), offsets=offsets, source=source)
        oz.f8_gemm_grad(dY, codes, scales, dX, oz.alloc_f8_workspace("grad", rows, n, k, dt, rows=rows, experts=E), offsets=offsets)
        oz.f8_weight_grad(dY, X, dW, oz.alloc_f8_workspace("weight_grad", t, n, k, dt, rows=rows, experts=E), offsets=offsets, source=source)
        for e in range(E):
            a, b = sum(counts[:e]), sum(counts[:e + 1])
            assert torch.equal(Y[a:b], rounded(Xr[a:b] @ W[e].t(), dt)), e
            assert torch.equal(dX[a:b], rounded(dY0[a:b] @ W[e], dt)), e
            assert torch.equal(dW[e], rounded(dY0[a:b].t() @ Xr[a:b], dt)), e
        assert (Y[used:] == 77).all() and (dX[used:] == 77).all()
        assert untouched(ybuf, rows, n, extra, extra) and untouched(xbuf, rows, k, extra, extra)


@pytest.mark.parametrize("dt", TYPES)
def test_one_workspace_serves_fewer_rows(dt):
    n, k = 1030, 1100
    g = gen(5)
    W0 = small_integers((n, k), g, 3).to(DEV)
    codes, scales, W = cut_weights(W0[None], False)
    ws = {op: oz.alloc_f8_workspace(op, 5000, n, k, dt) for op in ("gemm", "grad", "weight_grad")}
    for t in (5000, 3000, 1500, 700, 300, 64, 3, 1):
        X0, dY0 = torch.randint(-3, 4, (t, k), generator=g).double().to(DEV), torch.randint(-3, 4, (t, n), generator=g).double().to(DEV)
        X, dY = X0.to(dt), dY0.to(dt)
        Y, dX, dW = torch.empty(t, n, dtype=dt, device=DEV), torch.empty(t, k, dtype=dt, device=DEV), torch.empty(n, k, dtype=dt, device=DEV)
        oz.f8_gemm(X, codes[0], scales[0], Y, ws["gemm"])
        oz.f8_gemm_grad(dY, codes[0], scales[0], dX, ws["grad"])
        oz.f8_weight_grad(dY, X, dW, ws["weight_grad"])
        assert torch.equal(Y, rounded(X0 @ W[0].t(), dt)) and torch.equal(dX, rounded(dY0 @ W[0], dt)) and torch.equal(dW, rounded(dY0.t() @ X0, dt))


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("t", [700, 4100])
def test_nan_stays_in_its_row(t, dt):
    n, k = 4090, 1100
    g = gen(3)
    X, W = torch.randn(t, k, generator=g).to(dt).to(DEV), (torch.randn(n, k, generator=g) / math.sqrt(k)).to(DEV)
    codes = torch.empty(n, oz.f8_row_bytes(k), dtype=torch.uint8, device=DEV)
    scales = torch.empty(-(-n // 128), oz.f8_scale_bytes(k), dtype=torch.uint8, device=DEV)
    oz.f8_split(W, codes, scales)
    ws = oz.alloc_f8_workspace("gemm", t, n, k, dt)
    clean, got = torch.empty(t, n, dtype=dt, device=DEV), torch.empty(t, n, dtype=dt, device=DEV)
    oz.f8_gemm(X, codes, scales, clean, ws)
    X[t - 2, k - 1] = math.nan
    X[5, 0] = math.inf
    oz.f8_gemm(X, codes, scales, got, ws)
    assert got[[5, t - 2]].isnan().all()
    keep = torch.ones(t, dtype=torch.bool, device=DEV)
    keep[[5, t - 2]] = False
    assert torch.equal(got[keep], clean[keep])
    scales[1, 2] = 255
    oz.f8_gemm(X, codes, scales, got, ws)
    assert got[:, 128:256].isnan().all() and torch.equal(got[keep][:, :128], clean[keep][:, :128]) and torch.equal(got[keep][:, 256:], clean[keep][:, 256:])


def test_large_tiles_in_a_graph_and_on_two_streams():
    """Two captured graphs and eager calls, each with a workspace of its own, give the same bits."""
    t, n, k = 4100, 4090, 1100
    g = gen(1)
    W = (torch.randn(n, k, generator=g) / math.sqrt(k)).to(DEV)
    codes = torch.empty(n, oz.f8_row_bytes(k), dtype=torch.uint8, device=DEV)
    scales = torch.empty(-(-n // 128), oz.f8_scale_bytes(k), dtype=torch.uint8, device=DEV)
    oz.f8_split(W, codes, scales)
    X = torch.randn(t, k, generator=g).to(BF16).to(DEV)
    outs = [torch.empty(t, n, dtype=BF16, device=DEV) for _ in range(3)]
    ws = [oz.alloc_f8_workspace("gemm", t, n, k, BF16) for _ in range(3)]
    for i in range(3):
        oz.f8_gemm(X, codes, scales, outs[i], ws[i])
    torch.cuda.synchronize()
    graphs = []
    for i in (1, 2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            oz.f8_gemm(X, codes, scales, outs[i], ws[i])
    side = torch.cuda.Stream()
    for _ in range(3):
        X.copy_(torch.randn(t, k, generator=g).to(BF16))
        for o in outs:
            o.fill_(77)
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        oz.f8_gemm(X, codes, scales, outs[0], ws[0])
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
