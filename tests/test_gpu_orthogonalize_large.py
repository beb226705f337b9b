"""Orthogonal updates of 16-bit types on every tile of the last product, against 64 bits: results are those of an iteration in 32 bits, rounded once, whatever the size."""
import math

import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
MUON = (3.4445, -4.7750, 2.0315)


def gradient(m, n, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = min(8, m, n)
    strong = torch.randn(m, r, generator=g, device=DEV) @ torch.randn(r, n, generator=g, device=DEV)
    return strong / math.sqrt(r) + 0.3 * torch.randn(m, n, generator=g, device=DEV)


def iterate(G, dt):
    """On the GPU: minutes on the CPU. (No batches, and right operands that lie in rows.)"""
    a, b, c = MUON
    X = G.double()
    X = (X / (X.norm() + 1e-7)).to(dt)
    tall = X.shape[0] > X.shape[1]
    X = X.t().contiguous() if tall else X
    for _ in range(5):
        A = X @ X.t().contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return (X.t() if tall else X).double()


def check(got, G):
    """Before the last rounding errors are up to four times those of the same iteration in 32 bits (two slices hold 22 bits, and a product has two operands), in the norm; an
    element's may be as large as all of its row's or column's errors taken together are in the mean, sqrt(longer side) times an element's mean. The rounding is half a step of the element."""
    want, plain = iterate(G, torch.float64), iterate(G, F32)
    m, n = want.shape
    before = 4 * float((plain - want).norm() / want.norm()) + 2.0 ** -22            # relative, in the norm
    mean = float(want.norm()) / math.sqrt(m * n)
    off = (got.double() - want).abs()
    bound = torch.finfo(got.dtype).eps / 2 * want.abs() + before * mean * math.sqrt(max(m, n)) + torch.finfo(got.dtype).tiny
    assert (off <= bound).all(), f"off by up to {float((off / bound).max()):.3g} times the bound"
    # and in the norm: the rounding alone, of the same values from the 64-bit iteration, and the errors before it
    rounded = float((want.to(got.dtype).double() - want).norm() / want.norm())
    rel = float(off.norm() / want.norm())
    assert rel <= 1.01 * rounded + before, (rel, rounded, before)


# last products of 64 x 64 tiles in both forms, of 128 and of 256, and of 64 and 128 with tiles that several workgroups share (2304 x 2304, 2048 x 4100);
# wide, tall and square; two matrices
SHAPES = [(1, 65, 300), (1, 300, 700), (1, 700, 300), (2, 520, 1000), (1, 1100, 1100), (1, 1100, 4352), (1, 4352, 1100), (1, 2304, 2304),
          (1, 2048, 4100), (1, 4100, 2048), (2, 1800, 1850), (1, 4096, 4096), (1, 130, 16000), (1, 16000, 130)]


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("batch,m,n", SHAPES)
def test_sixteen_bits(batch, m, n, dt):
    G = torch.stack([gradient(m, n, i + m) for i in range(batch)]).to(dt)
    X = torch.empty_like(G)
    ws = oz.alloc_orthogonalize_workspace(batch, m, n)
    ws.fill_(0xFF)
    oz.orthogonalize(G, X, ws)
    for i in range(batch):
        check(X[i], G[i])


@pytest.mark.parametrize("m,n", [(60, 256), (60, 1000), (60, 9000)])
@pytest.mark.parametrize("dt", [BF16, F16])
def test_sixteen_bits_of_narrow_matrices(m, n, dt):
    """One workgroup, panels, and the tiled products: one precision."""
    for G in (gradient(m, n, 1).to(dt), gradient(n, m, 2).to(dt)):
        X = torch.empty_like(G)
        oz.orthogonalize(G, X, oz.alloc_orthogonalize_workspace(1, *G.shape))
        check(X, G)
