"""The operators in 8-bit floating point and over experts on matrices whose rows lie so far apart that offsets pass 32 bits: the same bits as on compact ones, and nothing
written between the rows near them."""
import pytest
import torch

from f8_plain import BF16, F16, F32
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
SPAN = (1 << 32) + (1 << 28)


def far(rows, cols, dt, fill=None):
    """A matrix over more than 4 GiB (as far as the distance between rows allows); two columns behind the rows hold 77."""
    size = torch.empty(0, dtype=dt).element_size()
    ld = min(1 << 24, max(cols + 16, -(-SPAN // (rows * size)) + 15) // 16 * 16)
    buf = torch.empty(rows, ld, dtype=dt, device=DEV)
    buf[:, :cols + 2] = 77
    if fill is not None:
        buf[:, :cols] = fill
    return buf[:, :cols], buf


def near(rows, cols, dt, fill=None):
    return torch.full((rows, cols), 77, dtype=dt, device=DEV) if fill is None else fill.clone(), None


def kept(buf, cols):
    return buf is None or bool((buf[:, cols:cols + 2] == 77).all())


# (few rows, small tiles, tiles of 256)
@pytest.mark.parametrize("t,n,k", [(300, 300, 130), (600, 1500, 300), (4100, 4090, 400)])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_products(t, n, k, dt):
    g = torch.Generator().manual_seed(n)
    X0, W0, dY0 = (torch.randn(a, b, generator=g).to(dt).to(DEV) for a, b in ((t, k), (n, k), (t, n)))
    bytes_, sbytes = oz.f8_row_bytes(k), oz.f8_scale_bytes(k)
    results = []
    for make in (near, far):
        codes, cbuf = make(n, bytes_, torch.uint8)
        scales = torch.empty(-(-n // 128), sbytes, dtype=torch.uint8, device=DEV)
        W, X, dY = make(n, k, dt, W0)[0], make(t, k, dt, X0)[0], make(t, n, dt, dY0)[0]
        oz.f8_split(W, codes, scales)
        del W
        back, bbuf = make(n, k, F16)
        oz.f8_expand(codes, scales, back)
        xc, xbuf = make(t, bytes_, torch.uint8)
        xs = torch.empty(t, sbytes, dtype=torch.uint8, device=DEV)
        oz.f8_split(X, xc, xs, 1)
        out = [codes.clone(), scales, back.clone(), xc.clone(), xs]
        assert kept(cbuf, bytes_) and kept(bbuf, k) and kept(xbuf, bytes_)
        del back, bbuf
        Y, ybuf = make(t, n, dt)
        ws = oz.alloc_f8_workspace("gemm", t, n, k, dt)
        oz.f8_gemm(X, codes, scales, Y, ws)
        out.append(Y.clone())
        oz.f8_gemm(xc, codes, scales, Y, ws, x_scales=xs)
        out.append(Y.clone())
        assert kept(ybuf, n)
        del Y, ybuf, xc, xbuf
        dX, dbuf = make(t, k, dt)
        oz.f8_gemm_grad(dY, codes, scales, dX, oz.alloc_f8_workspace("grad", t, n, k, dt))
        out.append(dX.clone())
        assert kept(dbuf, k)
        del dX, dbuf, codes, cbuf
        dW, wbuf = make(n, k, dt)
        oz.f8_weight_grad(dY, X, dW, oz.alloc_f8_workspace("weight_grad", t, n, k, dt))
        out.append(dW.clone())
        assert kept(wbuf, k)
        results.append(out)
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_experts(dt):
    """Experts' weights beyond 4 GiB, each row by its expert; tokens, results and gradients as far apart."""
    E, top, t, n, k = 24, 2, 300, 200, 260
    g = torch.Generator().manual_seed(1)
    logits0 = torch.randn(t, E, generator=g).to(dt).to(DEV)
    X0, W0 = torch.randn(t, k, generator=g).to(dt).to(DEV), torch.randn(E * n, k, generator=g).to(DEV)
    dw0 = torch.randn(t, top, generator=g).to(DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    results = []
    for make in (near, far):
        logits, X = make(t, E, dt, logits0)[0], make(t, k, dt, X0)[0]
        indices, weights = torch.empty(t, top, **i32), torch.empty(t, top, device=DEV)
        offsets, source, place = torch.empty(E + 1, **i32), torch.empty(t * top, **i32), torch.empty(t, top, **i32)
        oz.route(logits, indices, weights)
        dl, lbuf = make(t, E, dt)
        oz.route_grad(logits, indices, dw0, dl)
        assert kept(lbuf, E)
        oz.expert_order(indices, E, offsets, source, place, oz.alloc_expert_order_workspace(t, top, E))
        out = [indices, weights, dl.clone()]
        del logits, dl, lbuf
        codes, cbuf = make(E * n, oz.f8_row_bytes(k), torch.uint8)
        codes = codes.view(E, n, -1) if make is near else codes.as_strided((E, n, codes.shape[1]), (n * codes.stride(0), codes.stride(0), 1))
        scales = torch.empty(E, -(-n // 128), oz.f8_scale_bytes(k), dtype=torch.uint8, device=DEV)
        for e in range(E):
            oz.f8_split(W0[e * n:e * n + n], codes[e], scales[e])
        O, obuf = make(t * top, n, dt)
        oz.f8_gemm(X, codes, scales, O, oz.alloc_f8_workspace("gemm", t, n, k, dt, rows=t * top, experts=E), offsets=offsets, source=source)
        assert kept(obuf, n)
        Y, ybuf = make(t, n, dt)
        oz.expert_combine(O, place, weights, Y)
        assert kept(ybuf, n)
        out += [O.clone(), Y.clone()]
        dO, gbuf = make(t * top, n, dt)
        dweights = torch.empty(t, top, device=DEV)
        oz.expert_combine_grad(Y, O, place, weights, dO, dweights)
        assert kept(gbuf, n)
        out += [dO.clone(), dweights]
        del O, obuf, Y, ybuf
        dX, xbuf = make(t * top, k, dt)
        oz.f8_gemm_grad(dO, codes, scales, dX, oz.alloc_f8_workspace("grad", t * top, n, k, dt, rows=t * top, experts=E), offsets=offsets)
        assert kept(xbuf, k)
        out.append(dX.clone())
        del dX, xbuf, codes, cbuf
        dW, wbuf = make(E * n, k, dt)
        dW = dW.view(E, n, k) if make is near else dW.as_strided((E, n, k), (n * dW.stride(0), dW.stride(0), 1))
        oz.f8_weight_grad(dO, X, dW, oz.alloc_f8_workspace("weight_grad", t, n, k, dt, rows=t * top, experts=E), offsets=offsets, source=source)
        assert kept(wbuf, k)
        out.append(dW.clone())
        results.append(out)
    for a, b in zip(*results):
        assert torch.equal(a, b)
