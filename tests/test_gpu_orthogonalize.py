"""The orthogonal update against the same iteration in 64 bits, and a layer that is trained with it: four-bit product, gradient, update, new cut."""
import math

import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
MUON = (3.4445, -4.7750, 2.0315)


def iterate(G, steps, coefficients, eps, dt=torch.float64):
    a, b, c = coefficients
    X = G.double()
    X = (X / (X.norm() + eps) if float(X.norm()) + eps > 0 else X).to(dt)
    tall = X.shape[0] > X.shape[1]
    X = X.t() if tall else X
    for _ in range(steps):
        A = X @ X.t()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.t() if tall else X


def gradient(m, n, seed, noise=0.3):
    g = torch.Generator().manual_seed(seed)
    r = min(8, m, n)
    return torch.randn(m, r, generator=g) @ torch.randn(r, n, generator=g) / math.sqrt(r) + noise * torch.randn(m, n, generator=g)


def check(got, G, steps=5, coefficients=MUON, eps=1e-7):
    """A value held as two slices is off by at most 2^-23 of itself, one in 32 bits by 2^-24, and a product has two operands: errors up to four times those of the same
    iteration in 32 bits (measured on the same matrix, in the norm), and no less than a rounding of 2^-23 of everything. Then one rounding of the result."""
    want = iterate(G, steps, coefficients, eps)
    if want.norm() == 0:
        assert (got == 0).all()
        return
    plain = iterate(G, steps, coefficients, eps, F32).double()
    off = float((got.cpu().double() - want).norm() / want.norm())
    allowed = 4 * float((plain - want).norm() / want.norm()) + 2.0 ** -22
    if got.dtype != F32:
        allowed += torch.finfo(got.dtype).eps / 2
    assert off <= allowed, (off, allowed)


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (16, 16), (31, 33), (33, 31), (64, 64), (64, 48), (65, 64), (64, 256), (256, 63), (20, 257), (33, 100), (100, 300), (300, 100), (128, 128), (129, 520), (513, 200), (700, 700),
          (64, 1000), (1000, 64), (5, 8192), (8191, 33), (60, 8193), (1, 300)]


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("m,n", SHAPES)
def test_against_64_bits(m, n, dt):
    G0 = gradient(m, n, m * 100 + n).to(dt)
    ws = oz.alloc_orthogonalize_workspace(1, m, n)
    for extra, offset in ((0, 0), (5, 3)):
        ws.fill_(0xFF)
        ld = n + extra
        gbuf = torch.full((m * ld + offset + 8,), float("nan"), dtype=dt, device=DEV)
        xbuf = torch.full((m * ld + offset + 8,), 77.0, dtype=dt, device=DEV)
        G, X = (b[offset:offset + m * ld].view(m, ld)[:, :n] for b in (gbuf, xbuf))
        G.copy_(G0)
        oz.orthogonalize(G, X, ws)
        check(X, G0)
        assert (xbuf[:offset] == 77).all() and (xbuf[offset:offset + m * ld].view(m, ld)[:, n:] == 77).all() and (xbuf[offset + m * ld:] == 77).all()
    oz.orthogonalize(G, G, ws)      # in place
    assert torch.equal(G, X)


@pytest.mark.parametrize("batch,m,n", [(1, 2304, 2304), (1, 1100, 4352), (1, 4352, 1100), (2, 3600, 3650)])
def test_large(batch, m, n):
    G = torch.stack([gradient(m, n, i) for i in range(batch)]).to(DEV)
    X = torch.empty_like(G)
    oz.orthogonalize(G, X, oz.alloc_orthogonalize_workspace(batch, m, n))
    for i in range(batch):   # (64 bits on the GPU: minutes on the CPU)
        want = iterate(G[i], 5, MUON, 1e-7)
        plain = iterate(G[i], 5, MUON, 1e-7, F32).double()
        off = float((X[i].double() - want).norm() / want.norm())
        assert off <= 4 * float((plain - want).norm() / want.norm()) + 2.0 ** -22


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("batch,m,n", [(3, 40, 50), (5, 130, 64), (70, 20, 20), (2, 300, 700), (7, 30, 400), (3, 1100, 60)])
def test_batches(batch, m, n, dt):
    G0 = torch.stack([gradient(m, n, i) * 10.0 ** (i % 5 - 2) for i in range(batch)]).to(dt)
    G0[1] = 0
    G = torch.zeros(batch, m + 1, n + 3, dtype=dt, device=DEV)[:, :m, :n]
    G.copy_(G0)
    X = torch.empty(batch, m, n, dtype=dt, device=DEV)
    ws = oz.alloc_orthogonalize_workspace(batch, m, n)
    oz.orthogonalize(G, X, ws)
    for i in range(batch):
        check(X[i], G0[i])
    if batch > 2:
        clean = X.clone()
        G[0, m // 2, n // 2] = float("nan")
        oz.orthogonalize(G, X, ws)
        assert torch.equal(X[1:], clean[1:]) and X[0].isnan().any()
        G[0, m // 2, n // 2] = float("inf")
        oz.orthogonalize(G, X, ws)
        assert torch.equal(X[1:], clean[1:]) and X[0].isnan().any()


def test_one_matrix_for_a_whole_batch():
    """stride 0: a broadcast input."""
    G = gradient(50, 60, 1).to(DEV)
    X, X1 = torch.empty(4, 50, 60, device=DEV), torch.empty(50, 60, device=DEV)
    oz.orthogonalize(G.expand(4, 50, 60), X, oz.alloc_orthogonalize_workspace(4, 50, 60))
    oz.orthogonalize(G, X1, oz.alloc_orthogonalize_workspace(1, 50, 60))
    for i in range(4):
        assert torch.equal(X[i], X1)


@pytest.mark.parametrize("steps,coefficients,eps", [(1, MUON, 0.0), (1, (1.0, 0.0, 0.0), 0.5), (3, (2.0, -1.5, 0.5), 1e-7), (6, MUON, 1e-3),
                                                    (1, (30.0, -20.0, 10.0), 0.0)])
def test_other_polynomials(steps, coefficients, eps):
    for m, n in ((48, 80), (200, 150), (900, 50)):
        G = gradient(m, n, steps)
        X = torch.empty(m, n, device=DEV)
        oz.orthogonalize(G.to(DEV), X, oz.alloc_orthogonalize_workspace(1, m, n), steps=steps, coefficients=coefficients, eps=eps)
        check(X, G, steps, coefficients, eps)


@pytest.mark.parametrize("coefficients", [(0.0, 1.0, 0.0), (0.0, 0.0, 1.0), (0.9, 0.1, 0.0)])
def test_polynomials_that_shrink_small_values_are_refused(coefficients):
    """x^5 of x^5 leaves a matrix of 1e-10: below what slices under a common power of two hold of it."""
    G = gradient(48, 80, 2).to(DEV)
    with pytest.raises(oz.OzimmuError) as e:
        oz.orthogonalize(G, G, oz.alloc_orthogonalize_workspace(1, 48, 80), steps=2, coefficients=coefficients)
    assert e.value.code == oz.ERR_BAD_POLYNOMIAL


def test_the_plain_iteration_ends_at_the_nearest_orthogonal_matrix():
    m, n = 60, 90
    G = gradient(m, n, 3, noise=1.0)
    X = torch.empty(m, n, device=DEV)
    oz.orthogonalize(G.to(DEV), X, oz.alloc_orthogonalize_workspace(1, m, n), steps=40, coefficients=(1.5, -0.5, 0.0), eps=0.0)
    U, _, Vt = torch.linalg.svd(G.double(), full_matrices=False)
    X = X.cpu().double()
    # at the fixed point a step's roundings (2^-22 of the matrix, whose rows have norm one) are what is left; the derivative there is zero
    assert (X @ X.t() - torch.eye(m, dtype=torch.float64)).norm() <= 32 * 2.0 ** -22 * math.sqrt(m)
    # roundings on the way turn small singular directions: the gap of the smallest singular value carries them
    s = torch.linalg.svdvals(G.double())
    assert (X - U @ Vt).norm() <= 64 * 2.0 ** -22 * float(s[0] / s[-1]) * math.sqrt(m)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e15, 1e37])
def test_the_size_of_the_matrix_does_not_matter(scale):
    G = (gradient(70, 90, 5) / 8).to(DEV)
    X0, X1 = torch.empty_like(G), torch.empty_like(G)
    ws = oz.alloc_orthogonalize_workspace(1, 70, 90)
    oz.orthogonalize(G, X0, ws, eps=0.0)
    oz.orthogonalize(G * scale, X1, ws, eps=0.0)
    check(X1, (G * scale).cpu(), eps=0.0)
    assert (X0 - X1).norm() <= 1e-4 * X0.norm()


@pytest.mark.parametrize("batch,m,n", [(1, 65, 65), (3, 70, 1500), (1, 1500, 90), (2, 520, 1000), (1, 1100, 1100), (3, 40, 700), (1, 2000, 64)])
def test_nothing_beyond_the_workspace_is_written(batch, m, n):
    need = oz.orthogonalize_workspace_bytes(batch, m, n)
    room = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
    G0 = torch.stack([gradient(m, n, 3 + i) for i in range(batch)])
    X = torch.empty(batch, m, n, device=DEV)
    oz.orthogonalize(G0.to(DEV), X, room[:need])
    assert (room[need:] == 0x5A).all()
    for got, G in zip(X, G0):
        check(got, G)


@pytest.mark.parametrize("m,n", [(40, 50), (50, 900), (300, 200)])
def test_in_place(m, n):
    G = torch.stack([gradient(m, n, i) for i in range(2)]).to(DEV)
    X = torch.empty_like(G)
    ws = oz.alloc_orthogonalize_workspace(2, m, n)
    oz.orthogonalize(G, X, ws)
    oz.orthogonalize(G, G, ws)
    assert torch.equal(G, X)


@pytest.mark.parametrize("m,n", [(100, 140), (60, 700)])
def test_graph_shares_a_workspace_with_eager_calls(m, n):
    G = torch.stack([gradient(m, n, i) for i in range(2)]).to(DEV)
    X = torch.empty_like(G)
    ws = oz.alloc_orthogonalize_workspace(2, m, n)
    oz.orthogonalize(G, X, ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        oz.orthogonalize(G, X, ws)
    first = G.clone()
    for i in range(3):
        G.copy_(first + i * first.flip(0))
        g.replay()
        torch.cuda.synchronize()
        got = X.clone()
        oz.orthogonalize(G, X, ws)
        torch.cuda.synchronize()
        assert torch.equal(got, X)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_a_layer_trained_in_four_bits(dt):
    """The operators as they are used together: the master weights are cut, tokens go through the four-bit layer, the gradient comes back through it, the weights' gradient (straight
    through the cut) is orthogonalised, and the updated weights are cut again. Every result against 64 bits from the same inputs."""
    t, n, k, group = 96, 160, 224, 32
    g = torch.Generator().manual_seed(1)
    master = (torch.randn(n, k, generator=g) / math.sqrt(k)).to(DEV)
    codes = torch.empty(n, oz.q4_row_bytes(k), dtype=torch.uint8, device=DEV)
    scales = torch.empty(n, -(-k // group), dtype=dt, device=DEV)
    W = torch.empty(n, k, dtype=dt, device=DEV)
    Y, dX, U = torch.empty(t, n, dtype=dt, device=DEV), torch.empty(t, k, dtype=dt, device=DEV), torch.empty(n, k, device=DEV)
    wf, wg = oz.alloc_q4_workspace(t, n, k, group, dt), oz.alloc_q4_workspace(t, n, k, group, dt, gradient=True)
    wo = oz.alloc_orthogonalize_workspace(1, n, k)
    for step in range(3):
        X, T = torch.randn(t, k, generator=g).to(dt).to(DEV), torch.randn(t, n, generator=g).to(DEV)
        oz.q4_split(master, group, codes, scales)
        oz.q4_expand(codes, scales, group, W)
        oz.q4_gemm(X, codes, scales, group, Y, wf)
        dY = ((Y.float() - T) / t).to(dt)
        oz.q4_gemm_grad(dY, codes, scales, group, dX, wg)
        dW = dY.float().t().contiguous() @ X.float()
        oz.orthogonalize(dW, U, wo)
        half = torch.finfo(dt).eps / 2
        exact_w = (codes.long() & 15, codes.long() >> 4)
        exact_w = (torch.stack(exact_w, dim=2).view(n, -1)[:, :k] - 8).double() * scales.double().repeat_interleave(group, dim=1)[:, :k]
        assert (W.double() - exact_w).abs().max() <= half * exact_w.abs().max()
        # a cut is off by at most half a step of its scale, and by what the scale's rounding clips of the largest value (7 steps)
        steps = scales.double().repeat_interleave(group, dim=1)[:, :k]
        assert ((exact_w - master.double()).abs() <= (0.5 + 2.0 ** -23) * steps).all()
        for got, want, terms in ((Y, X.double() @ exact_w.t(), X.double().abs() @ exact_w.t().abs()), (dX, dY.double() @ exact_w, dY.double().abs() @ exact_w.abs())):
            assert ((got.double() - want).abs() <= half * (terms + want.abs()) * 1.01 + 2.0 ** -16 * terms).all()
        check(U, dW.cpu())
        master -= 0.02 * U
