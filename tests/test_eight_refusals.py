"""What the operators in 8-bit floating point and those for mixtures of experts refuse, on the host, before anything is launched, and their geometry. No GPU."""
import ctypes

import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

FAKE = ctypes.c_void_p(4096)     # never dereferenced: validation fails first
ODD = ctypes.c_void_p(4097)
BIG = 1 << 40
MAX = 1 << 22
L = lambda name: getattr(oz.lib(), "ozimmu_" + name)


def split(n=4, k=64, block=128, type_=0, W=FAKE, ldw=64, codes=FAKE, ldq=128, scales=FAKE, lds=4):
    return L("f8_split")(n, k, block, type_, W, ldw, codes, ldq, scales, lds, None)


def expand(n=4, k=64, block=128, codes=FAKE, ldq=128, stype=4, scales=FAKE, lds=4, type_=0, W=FAKE, ldw=64):
    return L("f8_expand")(n, k, block, codes, ldq, stype, scales, lds, type_, W, ldw, None)


def gemm(t=40, rows=40, n=8, k=64, experts=0, type_=0, X=FAKE, ldx=64, xs=None, ldxs=0, codes=FAKE, ldq=128, stype=4, scales=FAKE, lds=4, offsets=None, source=None, out=0, Y=FAKE, ldy=8, ws=FAKE,
         size=BIG):
    return L("f8_gemm")(t, rows, n, k, experts, type_, X, ldx, xs, ldxs, codes, ldq, stype, scales, lds, offsets, source, out, Y, ldy, ws, size, None)


def grad(rows=40, n=8, k=64, experts=0, type_=0, dY=FAKE, lddy=8, ys=None, ldys=0, codes=FAKE, ldq=128, stype=4, scales=FAKE, lds=4, offsets=None, out=0, dX=FAKE, lddx=64, ws=FAKE, size=BIG):
    return L("f8_gemm_grad")(rows, n, k, experts, type_, dY, lddy, ys, ldys, codes, ldq, stype, scales, lds, offsets, out, dX, lddx, ws, size, None)


def wgrad(t=40, rows=40, n=8, k=64, experts=0, type_=0, dY=FAKE, lddy=8, X=FAKE, ldx=64, offsets=None, source=None, out=0, dW=FAKE, lddw=64, ws=FAKE, size=BIG):
    return L("f8_weight_grad")(t, rows, n, k, experts, type_, dY, lddy, X, ldx, offsets, source, out, dW, lddw, ws, size, None)


def route(t=4, experts=8, top=2, type_=0, logits=FAKE, ldl=8, bias=None, score=0, groups=1, top_groups=1, renorm=1, scale=1.0, indices=FAKE, weights=FAKE):
    return L("route")(t, experts, top, type_, logits, ldl, bias, score, groups, top_groups, renorm, scale, indices, weights, None)


def route_grad(t=4, experts=8, top=2, type_=0, logits=FAKE, ldl=8, indices=FAKE, dw=FAKE, score=0, renorm=1, scale=1.0, dl=FAKE, lddl=8):
    return L("route_grad")(t, experts, top, type_, logits, ldl, indices, dw, score, renorm, scale, dl, lddl, None)


def order(t=4000, top=2, experts=8, indices=FAKE, offsets=FAKE, source=FAKE, place=FAKE, ws=FAKE, size=BIG):
    return L("expert_order")(t, top, experts, indices, offsets, source, place, ws, size, None)


def combine(t=4, top=2, rows=8, n=16, type_=0, O=FAKE, ldo=16, place=FAKE, weights=None, Y=FAKE, ldy=16):
    return L("expert_combine")(t, top, rows, n, type_, O, ldo, place, weights, Y, ldy, None)


def combine_grad(t=4, top=2, rows=8, n=16, type_=0, dY=FAKE, lddy=16, O=FAKE, ldo=16, place=FAKE, weights=FAKE, dO=FAKE, lddo=16, dw=FAKE):
    return L("expert_combine_grad")(t, top, rows, n, type_, dY, lddy, O, ldo, place, weights, dO, lddo, dw, None)


def test_geometry():
    assert oz.f8_geometry(0) == (0, 0)
    assert oz.f8_geometry(1) == (128, 4)
    assert oz.f8_geometry(512) == (512, 4)
    assert oz.f8_geometry(513) == (640, 8)
    assert oz.f8_row_bytes(4096) == 4096 and oz.f8_scale_bytes(4096) == 32
    for k in (-1, MAX + 1):
        with pytest.raises(oz.OzimmuError) as e:
            oz.f8_geometry(k)
        assert e.value.code == oz.ERR_BAD_DIM
    assert oz.lib().ozimmu_f8_geometry(1, None, None) == oz.ERR_NULL


def test_workspace_sizes():
    size = oz.f8_workspace_bytes
    for op in ("gemm", "grad", "weight_grad"):
        assert size(op, 0, 4096, 4096, torch.bfloat16) == 0
        for n, k in ((1000, 3000), (4096, 4096), (100, 70)):
            sizes = [size(op, t, n, k, torch.float16) for t in [*range(0, 1300, 3), 4096, 10 ** 5, 10 ** 6, 1 << 21]]
            assert sizes == sorted(sizes)       # a workspace serves fewer tokens than it was made for
            sizes = [size(op, 500, n, k, torch.float16, rows=r, experts=37) for r in [*range(0, 1300, 3), 4096, 10 ** 5]]
            assert sizes == sorted(sizes)
    assert size("gemm", 16, 2048, 2048, torch.bfloat16) == size("gemm", 1, 8192, 4096, torch.float32) == 0      # cut on the way
    assert size("gemm", 300, 1000, 4000, torch.uint8) <= size("gemm", 300, 1000, 4000, torch.float32)
    assert size("gemm", 300, 1000, 4000, torch.float32) >= 300 * 4096
    assert size("grad", 300, 1000, 4000, torch.float8_e4m3fn) >= 4000 * 1024
    assert size("weight_grad", 300, 1000, 4000, torch.float32) >= (1000 + 4000) * 384
    out = ctypes.c_size_t()
    f = oz.lib().ozimmu_f8_workspace_bytes
    assert f(0, 1, 1, 1, 1, 0, 0, None) == oz.ERR_NULL
    assert f(3, 1, 1, 1, 1, 0, 0, ctypes.byref(out)) == f(-1, 1, 1, 1, 1, 0, 0, ctypes.byref(out)) == oz.ERR_BAD_DIM
    assert f(0, 1, 2, 1, 1, 0, 0, ctypes.byref(out)) == f(0, 1, 1, 1, 1, 1025, 0, ctypes.byref(out)) == oz.ERR_BAD_DIM
    assert f(2, 1, 1, 1, 1, 0, 3, ctypes.byref(out)) == f(0, 1, 1, 1, 1, 0, 4, ctypes.byref(out)) == oz.ERR_BAD_TYPE
    with pytest.raises(ValueError):
        size("gemm", 1, 1, 1, torch.float64)
    with pytest.raises(ValueError):
        size("product", 1, 1, 1, torch.float32)
    assert oz.expert_order_workspace_bytes(1, 8, 64) == 0
    sizes = [oz.expert_order_workspace_bytes(t, 8, 64) for t in [*range(0, 9000, 100), 32768, 32769, 40000, 10 ** 6]]
    assert sizes == sorted(sizes) and sizes[-1] > 0
    assert oz.lib().ozimmu_expert_order_workspace_bytes(1, 33, 4, ctypes.byref(out)) == oz.ERR_BAD_DIM
    assert oz.lib().ozimmu_expert_order_workspace_bytes(1, 1, 4, None) == oz.ERR_NULL


DIM, TYPE, LD, NULL, MIS, WS = oz.ERR_BAD_DIM, oz.ERR_BAD_TYPE, oz.ERR_BAD_LD, oz.ERR_NULL, oz.ERR_MISALIGNED, oz.ERR_WORKSPACE
OVER = dict(experts=3, offsets=FAKE)
LARGE = dict(n=8192, k=8192, ldq=8192, lds=64)      # weights that take a workspace with these rows


@pytest.mark.parametrize("call,bad,code", [
    (split, dict(n=-1), DIM), (split, dict(k=MAX + 1), DIM), (split, dict(block=64), DIM), (split, dict(type_=3), TYPE), (split, dict(ldw=63), LD), (split, dict(ldq=120), LD),
    (split, dict(ldq=136), LD), (split, dict(lds=3), LD), (split, dict(lds=6), LD), (split, dict(W=None), NULL), (split, dict(codes=None), NULL), (split, dict(scales=None), NULL),
    (split, dict(W=ODD), MIS), (split, dict(codes=ctypes.c_void_p(4104)), MIS), (split, dict(scales=ODD), MIS), (split, dict(ldw=1 << 25), LD),
    (expand, dict(n=-1), DIM), (expand, dict(block=0), DIM), (expand, dict(stype=1), TYPE), (expand, dict(type_=4), TYPE), (expand, dict(ldw=63), LD), (expand, dict(stype=0, lds=0), LD),
    (expand, dict(scales=ODD), MIS), (expand, dict(codes=None), NULL), (expand, dict(W=ODD), MIS),
    (gemm, dict(t=-1), DIM), (gemm, dict(t=3), DIM), (gemm, dict(n=MAX + 1), DIM), (gemm, dict(experts=-1), DIM), (gemm, dict(experts=1025, offsets=FAKE), DIM), (gemm, dict(offsets=FAKE), DIM),
    (gemm, dict(source=FAKE), DIM), (gemm, dict(experts=3), NULL), (gemm, dict(t=50, **OVER), DIM), (gemm, dict(experts=3, offsets=ODD), MIS), (gemm, dict(source=ODD, **OVER), MIS),
    (gemm, dict(type_=4), TYPE), (gemm, dict(stype=2), TYPE), (gemm, dict(out=3), TYPE), (gemm, dict(ldx=63), LD), (gemm, dict(ldy=7), LD), (gemm, dict(ldq=64), LD), (gemm, dict(lds=2), LD),
    (gemm, dict(X=None), NULL), (gemm, dict(Y=None), NULL), (gemm, dict(codes=None), NULL), (gemm, dict(scales=None), NULL), (gemm, dict(X=ODD), MIS), (gemm, dict(Y=ODD), MIS),
    (gemm, dict(ws=None, ldx=8192, ldy=8192, **LARGE), WS), (gemm, dict(size=100, ldx=8192, ldy=8192, **LARGE), WS), (gemm, dict(ws=ctypes.c_void_p(4096 + 16), ldx=8192, ldy=8192, **LARGE), WS), (gemm, dict(type_=3, ldx=128, xs=None, ldxs=4), NULL),
    (gemm, dict(type_=3, ldx=64, xs=FAKE, ldxs=4), LD), (gemm, dict(type_=3, ldx=128, xs=FAKE, ldxs=2), LD), (gemm, dict(type_=3, ldx=128, xs=ODD, ldxs=4), MIS),
    (gemm, dict(t=MAX, k=1024, ldx=1024, ldq=1024, source=FAKE, **OVER), LD), (gemm, dict(type_=3, t=MAX, ldx=1024, xs=FAKE, ldxs=4, source=FAKE, **OVER), LD),
    (grad, dict(rows=-1), DIM), (grad, dict(type_=5), TYPE), (grad, dict(stype=1), TYPE), (grad, dict(lddy=7), LD), (grad, dict(lddx=63), LD), (grad, dict(dY=None), NULL), (grad, dict(ws=None), WS),
    (grad, dict(size=1000), WS), (grad, dict(experts=2), NULL), (grad, dict(type_=3, lddy=128), LD), (grad, dict(codes=ODD), MIS),
    (wgrad, dict(t=-1), DIM), (wgrad, dict(t=3), DIM), (wgrad, dict(t=3, **OVER), DIM), (wgrad, dict(type_=3), TYPE), (wgrad, dict(out=4), TYPE), (wgrad, dict(lddy=7), LD), (wgrad, dict(ldx=63), LD),
    (wgrad, dict(lddw=63), LD), (wgrad, dict(dY=None), NULL), (wgrad, dict(X=None), NULL), (wgrad, dict(dW=None), NULL), (wgrad, dict(ws=None), WS), (wgrad, dict(size=1000), WS), (wgrad, dict(X=ODD), MIS),
    (wgrad, dict(experts=2), NULL),
    (route, dict(t=-1), DIM), (route, dict(experts=0), DIM), (route, dict(experts=1025, ldl=1025), DIM), (route, dict(top=0), DIM), (route, dict(top=9), DIM), (route, dict(top=33, experts=64, ldl=64), DIM),
    (route, dict(groups=3), DIM), (route, dict(groups=0), DIM), (route, dict(groups=4, top_groups=5), DIM), (route, dict(top_groups=0), DIM), (route, dict(scale=float("inf")), DIM),
    (route, dict(scale=float("nan")), DIM), (route, dict(scale=1e39), DIM), (route, dict(type_=3), TYPE), (route, dict(score=2), TYPE), (route, dict(ldl=7), LD), (route, dict(logits=None), NULL),
    (route, dict(indices=None), NULL), (route, dict(weights=None), NULL), (route, dict(bias=ODD), MIS), (route, dict(indices=ODD), MIS),
    (route_grad, dict(t=MAX + 1), DIM), (route_grad, dict(top=9), DIM), (route_grad, dict(score=-1), TYPE), (route_grad, dict(lddl=7), LD), (route_grad, dict(dl=None), NULL), (route_grad, dict(dw=None), NULL),
    (route_grad, dict(dw=ODD), MIS),
    (order, dict(t=-1), DIM), (order, dict(top=0), DIM), (order, dict(experts=0), DIM), (order, dict(experts=1025), DIM), (order, dict(indices=None), NULL), (order, dict(offsets=None), NULL),
    (order, dict(place=None), NULL), (order, dict(source=ODD), MIS), (order, dict(ws=None), WS), (order, dict(size=8), WS),
    (combine, dict(t=-1), DIM), (combine, dict(top=33), DIM), (combine, dict(rows=-1), DIM), (combine, dict(n=MAX + 1), DIM), (combine, dict(type_=4), TYPE), (combine, dict(ldo=15), LD),
    (combine, dict(ldy=15), LD), (combine, dict(O=None), NULL), (combine, dict(place=None), NULL), (combine, dict(Y=ODD), MIS), (combine, dict(weights=ODD), MIS),
    (combine_grad, dict(rows=1 << 31), DIM), (combine_grad, dict(lddo=15), LD), (combine_grad, dict(lddy=15), LD), (combine_grad, dict(weights=None), NULL), (combine_grad, dict(dw=None), NULL),
    (combine_grad, dict(dO=None), NULL), (combine_grad, dict(place=ODD), MIS), (combine_grad, dict(type_=3), TYPE)])
def test_refusals(call, bad, code):
    assert call(**bad) == code


def test_nothing_to_do():
    assert split(n=0, W=None) == split(k=0, codes=None) == expand(n=0, W=None) == oz.OK
    assert gemm(t=0, rows=0, X=None, ws=None, size=0) == gemm(n=0, Y=None, ldy=0) == oz.OK
    assert grad(rows=0, dY=None, ws=None, size=0) == grad(k=0, dX=None) == oz.OK
    assert wgrad(n=0, dW=None) == wgrad(k=0, dW=None) == oz.OK
    assert route(t=0, logits=None) == route_grad(t=0, dl=None) == combine(t=0, Y=None) == combine(n=0, Y=None) == combine_grad(t=0, dw=None) == oz.OK


def test_binding_refusals():
    """The binding's own checks, with tensors that need no GPU: wrong shapes and types never reach the library."""
    f32, u8, i32 = (dict(dtype=d) for d in (torch.float32, torch.uint8, torch.int32))
    W, codes, scales = torch.empty(200, 300), torch.empty(200, 384, **u8), torch.empty(2, 4, **u8)
    X, Y = torch.empty(5, 300), torch.empty(5, 200)
    E = torch.empty(3, 200, 384, **u8), torch.empty(3, 2, 4, **u8), torch.empty(4, **i32)
    wrong = [
        lambda: oz.f8_split(W, codes[:199], scales), lambda: oz.f8_split(W, codes[:, :383], scales), lambda: oz.f8_split(W, codes, scales[:1]), lambda: oz.f8_split(W, codes, scales, 1),
        lambda: oz.f8_split(W, codes, scales, 2), lambda: oz.f8_split(W, codes.int(), scales), lambda: oz.f8_split(W, codes, torch.empty(2, 3)), lambda: oz.f8_split(W.double(), codes, scales),
        lambda: oz.f8_split(W.t(), codes, scales), lambda: oz.f8_expand(codes, scales[:, :3], W), lambda: oz.f8_expand(codes, scales.short(), W),
        lambda: oz.f8_gemm(X, codes[:100], scales, Y), lambda: oz.f8_gemm(X, codes, scales[:1], Y), lambda: oz.f8_gemm(X[:4], codes, scales, Y), lambda: oz.f8_gemm(X.double(), codes, scales, Y),
        lambda: oz.f8_gemm(X, codes, scales, Y, x_scales=scales), lambda: oz.f8_gemm(X.byte(), codes, scales, Y), lambda: oz.f8_gemm(X, E[0], E[1], Y),
        lambda: oz.f8_gemm(X, E[0], E[1], Y, offsets=E[2][:3]), lambda: oz.f8_gemm(X, E[0], E[1], Y, offsets=E[2].long()), lambda: oz.f8_gemm(X, E[0], E[1][:2], Y, offsets=E[2]),
        lambda: oz.f8_gemm(X, E[0], E[1], Y, offsets=E[2], source=torch.empty(4, **i32)), lambda: oz.f8_gemm(X, E[0][:, :100], E[1], Y, offsets=E[2]), lambda: oz.f8_gemm(X, codes, scales, Y),
        lambda: oz.f8_gemm_grad(Y, codes, scales, X[:4], None), lambda: oz.f8_gemm_grad(Y, codes[:, :256], scales, X, None), lambda: oz.f8_weight_grad(Y, X[:4], W, None),
        lambda: oz.f8_weight_grad(Y, X.half(), W, None), lambda: oz.f8_weight_grad(Y, X, W[:, :299], None), lambda: oz.f8_weight_grad(Y, X, W, None, offsets=E[2]),
        lambda: oz.route(X, torch.empty(5, 2, **i32), torch.empty(5, 3)), lambda: oz.route(X, torch.empty(4, 2, **i32), torch.empty(4, 2)), lambda: oz.route(X, torch.empty(5, 2), torch.empty(5, 2)),
        lambda: oz.route(X, torch.empty(5, 2, **i32), torch.empty(5, 2), score="relu"), lambda: oz.route(X, torch.empty(5, 2, **i32), torch.empty(5, 2), bias=torch.empty(299)),
        lambda: oz.route(X, torch.empty(2, 5, **i32).t(), torch.empty(5, 2)), lambda: oz.route_grad(X, torch.empty(5, 2, **i32), torch.empty(5, 2), X.half()),
        lambda: oz.expert_order(torch.empty(5, 2, **i32), 3, torch.empty(3, **i32), torch.empty(10, **i32), torch.empty(5, 2, **i32)),
        lambda: oz.expert_order(torch.empty(10, **i32), 3, torch.empty(4, **i32), torch.empty(10, **i32), torch.empty(5, 2, **i32)),
        lambda: oz.expert_combine(X, torch.empty(5, 2, **i32), torch.empty(5, 2, **f32), Y), lambda: oz.expert_combine(X, torch.empty(4, 2, **i32), None, X),
        lambda: oz.expert_combine_grad(X, X, torch.empty(5, 2, **i32), torch.empty(5, 2), X[:4], torch.empty(5, 2)),
    ]
    for call in wrong:      # (the last kind: everything fits but the device)
        with pytest.raises(ValueError):
            call()


def test_binding_takes_tensors_and_numbers():
    """What is no tensor, no number or no such score is refused as such; a call's own module refuses another count of arguments."""
    W, codes, scales, i32 = torch.empty(200, 300), torch.empty(200, 384, dtype=torch.uint8), torch.empty(2, 4, dtype=torch.uint8), dict(dtype=torch.int32)
    l, i, w = torch.empty(5, 8), torch.empty(5, 2, **i32), torch.empty(5, 2)
    for call in (lambda: oz.f8_split(None, codes, scales), lambda: oz.f8_split(W, codes, [1]), lambda: oz.f8_gemm(W, codes, scales, W, workspace=3), lambda: oz.f8_split(W, codes, scales, "a"),
                 lambda: oz.route(l, i, w, groups=1.5), lambda: oz.route(l, i, w, scale="a"), lambda: oz.expert_order(i, None, i, i, i), lambda: oz._calls().route(l, i, w)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: oz.route(l[0], i, w), lambda: oz.route(l, i[0], w), lambda: oz.route(l, i, w, score=None), lambda: oz.expert_combine(l, i, w, l.to("meta")), lambda: oz.f8_split(W[None], codes, scales),
                 lambda: oz.f8_weight_grad(l, l, torch.empty(8, 8), torch.empty(8, 8).t())):
        with pytest.raises(ValueError):
            call()
