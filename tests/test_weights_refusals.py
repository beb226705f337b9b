"""What the operators on weight matrices (four-bit weights, orthogonal update) refuse, on the host, before anything is launched, and their geometry. No GPU."""
import ctypes

import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

FAKE = ctypes.c_void_p(4096)     # never dereferenced: validation fails first
ODD = ctypes.c_void_p(4097)
BIG = 1 << 40
MAX = 1 << 22


def split(n=4, k=64, group=32, type_=0, W=FAKE, ldw=64, codes=FAKE, ldq=32, stype=0, scales=FAKE, lds=2):
    return oz.lib().ozimmu_q4_split(n, k, group, type_, W, ldw, codes, ldq, stype, scales, lds, None)


def expand(n=4, k=64, group=32, type_=0, codes=FAKE, ldq=32, scales=FAKE, lds=2, W=FAKE, ldw=64):
    return oz.lib().ozimmu_q4_expand(n, k, group, type_, codes, ldq, scales, lds, W, ldw, None)


LARGE = dict(n=4096, k=4096, ldv=4096, ldq=2048, lds=128, ldr=4096)      # a size that takes a workspace


def gemm(t=4000, n=8, k=64, group=32, type_=0, V=FAKE, ldv=64, codes=FAKE, ldq=32, scales=FAKE, lds=2, R=FAKE, ldr=64, ws=FAKE, size=BIG, grad=False):
    f = oz.lib().ozimmu_q4_gemm_grad if grad else oz.lib().ozimmu_q4_gemm
    return f(t, n, k, group, type_, V, ldv, codes, ldq, scales, lds, R, ldr, ws, size, None)


WIDE = dict(n=300, ldg=300, ldx=300)      # a size that takes a workspace


def orth(batch=1, m=8, n=16, type_=0, G=FAKE, ldg=16, sg=0, X=FAKE, ldx=16, sx=0, steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, ws=FAKE, size=BIG):
    return oz.lib().ozimmu_orthogonalize(batch, m, n, type_, G, ldg, sg, X, ldx, sx, steps, a, b, c, eps, ws, size, None)


def test_geometry():
    assert oz.q4_geometry(0, 32) == (0, 0)
    assert oz.q4_geometry(1, 128) == (16, 1)
    assert oz.q4_geometry(32, 32) == (16, 1)
    assert oz.q4_geometry(33, 32) == (32, 2)
    assert oz.q4_geometry(1000, 64) == (512, 16)
    assert oz.q4_row_bytes(4096) == 2048
    for k, group in ((-1, 32), (MAX + 1, 32), (64, 0), (64, 16), (64, 96), (64, 256)):
        with pytest.raises(oz.OzimmuError) as e:
            oz.q4_geometry(k, group)
        assert e.value.code == oz.ERR_BAD_DIM


def test_workspace_sizes():
    size = oz.q4_workspace_bytes
    assert size(1, 4096, 4096, 128, torch.bfloat16) == 0           # the codes themselves are multiplied
    assert size(0, 4096, 4096, 128, torch.bfloat16) == 0
    assert size(16, 4096, 4096, 128, torch.bfloat16, gradient=True) > 0
    assert size(3000, 4096, 4000, 128, torch.float16) >= 2 * 4000 * 4096
    assert size(300, 4096, 4000, 128, torch.float32) >= 4 * 4000 * 4096
    assert size(1 << 21, 1, 1, 32, torch.float32) > 0             # more tokens than a launch of passes takes
    # more tokens never ask for less: a workspace serves fewer tokens than it was made for
    for dt in (torch.float32, torch.bfloat16):
        for grad in (False, True):
            for n, k in ((1000, 3000), (4096, 4096), (16384, 8192), (100, 70)):
                sizes = [size(t, n, k, 64, dt, grad) for t in [*range(0, 1300, 3), 4096, 10 ** 5, 10 ** 6, 1 << 21]]
                assert sizes == sorted(sizes)
    with pytest.raises(ValueError):
        size(1, 1, 1, 32, torch.float64)
    out = ctypes.c_size_t()
    assert oz.lib().ozimmu_q4_workspace_bytes(1, 1, 1, 32, 3, 0, ctypes.byref(out)) == oz.ERR_BAD_TYPE
    assert oz.lib().ozimmu_q4_workspace_bytes(1, 1, 1, 32, 0, 0, None) == oz.ERR_NULL
    assert oz.lib().ozimmu_q4_workspace_bytes(-1, 1, 1, 32, 0, 0, ctypes.byref(out)) == oz.ERR_BAD_DIM
    assert oz.orthogonalize_workspace_bytes(0, 4, 4) == 0
    assert oz.orthogonalize_workspace_bytes(9, 64, 256) == oz.orthogonalize_workspace_bytes(9, 256, 64) == 0       # one workgroup per matrix
    assert oz.orthogonalize_workspace_bytes(9, 64, 257) > 0 and oz.orthogonalize_workspace_bytes(9, 65, 65) > 0
    assert oz.orthogonalize_workspace_bytes(3, 100, 200) >= 3 * 4 * (100 * 200 + 2 * 100 * 200 + 2 * 100 * 100)
    assert oz.lib().ozimmu_orthogonalize_workspace_bytes(1, 4, 4, None) == oz.ERR_NULL
    assert oz.lib().ozimmu_orthogonalize_workspace_bytes(65536, 4, 4, ctypes.byref(out)) == oz.ERR_BAD_DIM


@pytest.mark.parametrize("call,bad,code", [
    (split, dict(n=-1), oz.ERR_BAD_DIM), (split, dict(k=MAX + 1), oz.ERR_BAD_DIM), (split, dict(group=48), oz.ERR_BAD_DIM),
    (split, dict(type_=3), oz.ERR_BAD_TYPE), (split, dict(stype=-1), oz.ERR_BAD_TYPE), (split, dict(ldw=63), oz.ERR_BAD_LD),
    (split, dict(ldq=16), oz.ERR_BAD_LD), (split, dict(ldq=40), oz.ERR_BAD_LD), (split, dict(lds=1), oz.ERR_BAD_LD), (split, dict(W=None), oz.ERR_NULL),
    (split, dict(codes=None), oz.ERR_NULL), (split, dict(scales=None), oz.ERR_NULL), (split, dict(W=ODD), oz.ERR_MISALIGNED),
    (split, dict(codes=ctypes.c_void_p(4104)), oz.ERR_MISALIGNED), (split, dict(scales=ctypes.c_void_p(4098)), oz.ERR_MISALIGNED),
    (expand, dict(n=-1), oz.ERR_BAD_DIM), (expand, dict(group=0), oz.ERR_BAD_DIM), (expand, dict(type_=7), oz.ERR_BAD_TYPE),
    (expand, dict(ldw=10), oz.ERR_BAD_LD), (expand, dict(ldq=8), oz.ERR_BAD_LD), (expand, dict(W=None), oz.ERR_NULL), (expand, dict(W=ODD), oz.ERR_MISALIGNED),
    (expand, dict(codes=None), oz.ERR_NULL),
    (gemm, dict(t=-1), oz.ERR_BAD_DIM), (gemm, dict(n=MAX + 1), oz.ERR_BAD_DIM), (gemm, dict(group=31), oz.ERR_BAD_DIM), (gemm, dict(type_=9), oz.ERR_BAD_TYPE),
    (gemm, dict(ldv=63), oz.ERR_BAD_LD), (gemm, dict(ldr=7), oz.ERR_BAD_LD), (gemm, dict(ldq=0), oz.ERR_BAD_LD), (gemm, dict(lds=0), oz.ERR_BAD_LD),
    (gemm, dict(V=None), oz.ERR_NULL), (gemm, dict(R=None), oz.ERR_NULL), (gemm, dict(codes=None), oz.ERR_NULL), (gemm, dict(scales=None), oz.ERR_NULL),
    (gemm, dict(V=ODD), oz.ERR_MISALIGNED), (gemm, dict(R=ODD), oz.ERR_MISALIGNED), (gemm, dict(codes=ODD), oz.ERR_MISALIGNED),
    (gemm, dict(ws=None, **LARGE), oz.ERR_WORKSPACE), (gemm, dict(ws=ctypes.c_void_p(4224), **LARGE), oz.ERR_WORKSPACE), (gemm, dict(size=64, **LARGE), oz.ERR_WORKSPACE),
    (gemm, dict(ldv=(1 << 24) + 1), oz.ERR_BAD_LD), (gemm, dict(ldr=(1 << 24) + 1), oz.ERR_BAD_LD), (gemm, dict(ldq=(1 << 24) + 16), oz.ERR_BAD_LD), (gemm, dict(lds=(1 << 24) + 1), oz.ERR_BAD_LD),
    (split, dict(ldw=(1 << 24) + 1), oz.ERR_BAD_LD), (expand, dict(ldw=1 << 25), oz.ERR_BAD_LD),
    (gemm, dict(grad=True, ldv=7), oz.ERR_BAD_LD), (gemm, dict(grad=True, ldr=63), oz.ERR_BAD_LD), (gemm, dict(grad=True, ws=None), oz.ERR_WORKSPACE),
    (gemm, dict(grad=True, t=1, ws=None), oz.ERR_WORKSPACE), (gemm, dict(grad=True, type_=-1), oz.ERR_BAD_TYPE),
    (orth, dict(batch=-1), oz.ERR_BAD_DIM), (orth, dict(batch=65536), oz.ERR_BAD_DIM), (orth, dict(m=-1), oz.ERR_BAD_DIM), (orth, dict(n=MAX + 1), oz.ERR_BAD_DIM),
    (orth, dict(type_=3), oz.ERR_BAD_TYPE), (orth, dict(steps=0), oz.ERR_BAD_POLYNOMIAL), (orth, dict(steps=65), oz.ERR_BAD_POLYNOMIAL),
    (orth, dict(a=float("nan")), oz.ERR_BAD_POLYNOMIAL), (orth, dict(c=float("inf")), oz.ERR_BAD_POLYNOMIAL), (orth, dict(eps=-1e-9), oz.ERR_BAD_POLYNOMIAL),
    (orth, dict(eps=float("nan")), oz.ERR_BAD_POLYNOMIAL), (orth, dict(a=0.99), oz.ERR_BAD_POLYNOMIAL), (orth, dict(a=-3.4445, b=4.775, c=-2.0315), oz.ERR_BAD_POLYNOMIAL), (orth, dict(a=5000.0), oz.ERR_BAD_POLYNOMIAL), (orth, dict(a=3.0, b=4.0, c=5.0), oz.ERR_BAD_POLYNOMIAL),
    (orth, dict(ldg=15), oz.ERR_BAD_LD), (orth, dict(ldx=15), oz.ERR_BAD_LD), (orth, dict(batch=2, sg=128, sx=127), oz.ERR_BAD_LD),
    (orth, dict(batch=2, sg=-1, sx=128), oz.ERR_BAD_LD), (orth, dict(G=None), oz.ERR_NULL), (orth, dict(X=None), oz.ERR_NULL), (orth, dict(G=ODD), oz.ERR_MISALIGNED),
    (orth, dict(X=ODD, type_=1), oz.ERR_MISALIGNED), (orth, dict(ws=None, **WIDE), oz.ERR_WORKSPACE), (orth, dict(ws=ctypes.c_void_p(4352 + 16), **WIDE), oz.ERR_WORKSPACE),
    (orth, dict(size=1000, **WIDE), oz.ERR_WORKSPACE),
])
def test_refusals(call, bad, code):
    assert call(**bad) == code


def test_empty_calls_do_nothing():
    none = dict(W=None, codes=None, scales=None)
    assert split(n=0, **none) == oz.OK and split(k=0, **none) == oz.OK
    assert expand(n=0, **none) == oz.OK and expand(k=0, **none) == oz.OK
    empty = dict(V=None, codes=None, scales=None, R=None, ws=None, size=0)
    assert gemm(t=0, **empty) == oz.OK and gemm(n=0, **empty) == oz.OK and gemm(t=0, grad=True, **empty) == oz.OK and gemm(k=0, grad=True, **empty) == oz.OK
    for zero in ("batch", "m", "n"):
        assert orth(**{zero: 0}, G=None, X=None, ws=None, size=0) == oz.OK


def test_binding_checks():
    cpu = dict(dtype=torch.float32)
    W, codes, scales = torch.zeros(4, 64, **cpu), torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, **cpu)
    ok = (W, 32, codes, scales)
    with pytest.raises(ValueError, match="GPU"):
        oz.q4_split(*ok)
    for bad in ((W.double(), 32, codes, scales), (W, 32, codes.int(), scales), (W, 32, codes[:3], scales), (W, 32, codes[:, :16], scales),
                (W, 32, codes, scales[:, :1]), (W.t(), 32, codes, scales), (W, 64, codes, scales)):
        with pytest.raises(ValueError):
            oz.q4_split(*bad)
    X, Y = torch.zeros(3, 64, **cpu), torch.zeros(3, 4, **cpu)
    for bad in ((X, codes, scales, 32, Y[:2]), (X.half(), codes, scales, 32, Y), (X, codes, scales, 32, Y.half()), (X, codes, scales, 32, Y)):
        with pytest.raises(ValueError):
            oz.q4_gemm(*bad)
    with pytest.raises(ValueError):
        oz.q4_gemm_grad(Y, codes, scales, 32, X[:2], None)
    G = torch.zeros(2, 8, 8, **cpu)
    for bad in ((G, G[0]), (G, G.half()), (G[0, 0], G[0, 0]), (G.transpose(1, 2), G), (G, G)):
        with pytest.raises(ValueError):
            oz.orthogonalize(*bad, None)
