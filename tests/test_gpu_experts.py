"""The choice of experts, the order of rows by expert and the experts' results brought together, against plain 64-bit forms and differences; and a layer of
experts as a program runs it."""
import math

import pytest
import torch

from f8_plain import BF16, F16, F32, TYPES, cut, cut_columns, guarded, half_step, order64, route64, route_weights, untouched
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN, INF = math.nan, math.inf


def gen(seed):
    return torch.Generator().manual_seed(seed)


def device_route(logits, top, extra=0, **how):
    t, experts = logits.shape
    l, _ = guarded(t, experts, logits.dtype, extra, extra)
    l.copy_(logits)
    indices = torch.full((t + 1, top), 77, dtype=torch.int32, device=DEV)
    weights = torch.full((t + 1, top), 77.0, device=DEV)
    bias = how.pop("bias", None)
    oz.route(l, indices[:t], weights[:t], bias=None if bias is None else bias.to(DEV), **how)
    assert (indices[t] == 77).all() and (weights[t] == 77).all()
    return indices[:t].cpu(), weights[:t].cpu()


def check_weights(got, want):
    """Computed in 64 bits (or to as much) and rounded once: half a step, and a few units of 64 bits' exponentials; kept to four 32-bit roundings, which an
    exponential, a sum, a quotient and the scale take."""
    assert torch.equal(got.isnan(), want.isnan())
    w = want.nan_to_num()
    assert ((got.double().nan_to_num() - w).abs() <= w.abs() * 8 * half_step(F32) + 2.0 ** -126).all()


ROUTES = [  # t, experts, top, score, bias, groups, top_groups
    (1, 1, 1, "softmax", False, 1, 1), (5, 2, 2, "sigmoid", True, 1, 1), (16, 8, 2, "softmax", False, 1, 1), (33, 64, 8, "sigmoid", True, 8, 4), (17, 65, 3, "softmax", True, 5, 2),
    (9, 100, 6, "sigmoid", False, 10, 3), (40, 256, 8, "sigmoid", True, 8, 4), (7, 300, 32, "softmax", True, 100, 40), (3, 1000, 5, "softmax", False, 1, 1), (4, 1024, 32, "sigmoid", True, 1024, 33),
    (130, 16, 16, "softmax", False, 4, 4), (6, 513, 4, "softmax", True, 3, 1), (11, 128, 1, "sigmoid", False, 2, 1), (21, 96, 4, "softmax", False, 6, 2)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,experts,top,score,bias,groups,top_groups", ROUTES)
def test_route(t, experts, top, score, bias, groups, top_groups, dt):
    g = gen(t + experts)
    logits = (2 * torch.randn(t, experts, generator=g)).to(dt)
    b = 0.1 * torch.randn(experts, generator=g) if bias else None
    for renormalize, scale, extra in ((True, 1.0, 0), (False, 2.5, 3)):
        how = dict(score=score, groups=groups, top_groups=top_groups, renormalize=renormalize, scale=scale, bias=b)
        indices, weights = device_route(logits, top, extra, **how)
        want, w = route64(logits, top, **how)
        assert torch.equal(indices, want)
        check_weights(weights, w)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_ties_and_neighbours(score):
    """Ties go to the lowest index; choice values that differ by less than 32 bits show keep their order."""
    t, experts = 64, 96
    g = gen(1)
    logits = torch.randint(-2, 3, (t, experts), generator=g).float()
    for groups, top_groups in ((1, 1), (8, 3)):
        got, _ = device_route(logits, 10, score=score, groups=groups, top_groups=top_groups)
        want, _ = route64(logits, 10, score=score, groups=groups, top_groups=top_groups)
        assert torch.equal(got, want)
    # scores around 1/2 (sigmoid) a few units of 32 bits apart
    near = 1.0 + torch.randint(0, 40, (t, experts), generator=g) * 2.0 ** -23
    bias = torch.randint(-1, 2, (experts,), generator=g) * 2.0 ** -24
    for b in (None, bias):
        got, _ = device_route(near, 16, score=score, bias=b)
        want, _ = route64(near, 16, score=score, bias=b)
        assert torch.equal(got, want)
    got, _ = device_route(near, 8, score=score, groups=16, top_groups=5, bias=bias)
    want, _ = route64(near, 8, score=score, groups=16, top_groups=5, bias=bias)
    assert torch.equal(got, want)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top,groups,top_groups", [(16, 2, 1, 1), (64, 8, 1, 1), (256, 8, 8, 4), (256, 15, 1, 1), (512, 16, 1, 1), (1024, 32, 1, 1)])
def test_route_few_neighbours(experts, top, groups, top_groups, score):
    """Most of many tokens are clear; some have two or more experts too near for 32 bits among the chosen, at the border and just behind it."""
    t = 2000
    g = gen(experts + top)
    logits = torch.randn(t, experts, generator=g)
    bias = (torch.randn(experts, generator=g) * 0.1).bfloat16().float()
    for b in (None, bias):
        l = logits.clone()
        p = route64(l, experts if groups == 1 and experts <= 32 else min(32, experts), score=score, bias=b, groups=groups, top_groups=top_groups)[0].long()
        for first, count in ((0, 2), (top - 1, 2), (top - 2, 2), (top - 1, 3), (top - 2, 4), (0, min(32, experts))):
            rows = torch.arange(t)[first + 7 * count::61]
            chosen = p[rows][:, first:first + count]
            chosen = chosen[:, (chosen >= 0).all(dim=0)]
            if b is None:        # the same logit but for a few units
                at = l[rows, chosen[:, 0]][:, None]
                l[rows[:, None], chosen] = at * (1 + torch.randint(-3, 4, chosen.shape, generator=g) * 2.0 ** -23)
            elif score == "sigmoid":   # the same sum of score and bias but for what the rounding of the logit leaves
                value = torch.sigmoid(l[rows, chosen[:, 0]].double())[:, None] + b.double()[chosen[:, :1]]
                l[rows[:, None], chosen] = torch.logit((value - b.double()[chosen]).clamp(0.05, 0.95)).float()
        how = dict(score=score, bias=b, groups=groups, top_groups=top_groups)
        got, weights = device_route(l, top, **how)
        want, w = route64(l, top, **how)
        assert torch.equal(got, want)
        check_weights(weights, w)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,top_groups", [(64, 8, 4), (256, 8, 4), (256, 64, 1), (512, 4, 3), (1024, 8, 2)])
def test_route_few_near_groups(experts, groups, top_groups, score):
    """Some of many tokens have groups whose sums of two are too near for 32 bits, the two among several that are nearly as large; and biases that
    always or never choose an expert."""
    t, top, per = 1000, 4, experts // groups
    g = gen(experts)
    logits = torch.randn(t, experts, generator=g)
    bias = (torch.randn(experts, generator=g) * 0.1).bfloat16().float()
    never = bias.clone()
    never[::5], never[3::11] = -INF, INF
    for b in (None, bias, never):
        l = logits.clone()
        by_group, value = l.view(t, groups, per), torch.zeros(per) if b is None else b.view(groups, per)
        for i in range(0, t, 29):
            first, second = torch.randperm(groups, generator=g)[:2].tolist()
            order = by_group[i, first].topk(min(3, per)).values
            if b is None or score == "softmax":
                by_group[i, second, :len(order)] = order * (1 + torch.randint(-2, 3, order.shape, generator=g) * 2.0 ** -23)
            else:
                shift = (value[first] - value[second]).nan_to_num(0.0, 0.0, 0.0).double()
                by_group[i, second] = torch.logit((torch.sigmoid(by_group[i, first].double()) + shift).clamp(0.02, 0.98)).float()
            if i % 2:      # more than two in a group
                by_group[i, first, :3] = by_group[i, first].max() * (1 + torch.randint(-2, 3, by_group[i, first, :3].shape, generator=g) * 2.0 ** -23)
        how = dict(score=score, bias=b, groups=groups, top_groups=top_groups)
        got, weights = device_route(l, top, **how)
        want, w = route64(l, top, **how)
        assert torch.equal(got, want)
        check_weights(weights, w)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (4, 2)])
def test_route_masks(score, groups, top_groups, dt):
    """Masked experts, groups and rows; infinities and NaN; the type's lowest value, which masks nothing."""
    experts, top = 16, 3
    g = gen(4)
    logits = torch.randn(12, experts, generator=g)
    logits[0] = -INF                       # nothing is left
    logits[1, 2:] = -INF                   # two experts for three choices
    logits[2, 4:] = -INF                   # one group
    logits[3, ::2] = -INF
    logits[4, 5] = NAN
    logits[5, 5] = INF
    logits[6] = torch.finfo(dt).min        # all alike
    logits[7, 3:] = torch.finfo(dt).min
    logits[8, 1:] = -INF
    logits[9] = -INF
    logits[9, 7] = NAN
    logits[10] = torch.finfo(dt).max
    logits = logits.to(dt)
    for bias in (None, torch.where(torch.arange(experts) == 1, torch.tensor(-INF), torch.randn(experts, generator=g) * 0.1)):
        for renormalize in (True, False):
            how = dict(score=score, groups=groups, top_groups=top_groups, renormalize=renormalize, bias=bias)
            indices, weights = device_route(logits, top, **how)
            want, w = route64(logits, top, **how)
            assert torch.equal(indices, want)
            check_weights(weights, w)
            dl = device_grad(logits, indices, torch.randn(12, top, generator=g), score=score, renormalize=renormalize)
            assert torch.isfinite(dl[[0, 1, 2, 3, 6, 7, 8, 9, 10, 11]].float()).all()
            assert not dl[[0, 9]].any() and not dl[3, ::2].any()


def device_grad(logits, indices, dweights, **how):
    dl, buf = guarded(*logits.shape, logits.dtype, 3, 1)
    oz.route_grad(logits.to(DEV), indices.to(DEV), dweights.to(DEV), dl, **how)
    assert untouched(buf, *logits.shape, 3, 1)
    return dl.cpu()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("t,experts,top", [(1, 1, 1), (5, 3, 2), (30, 64, 8), (9, 70, 32), (4, 256, 8), (3, 1000, 5)])
def test_route_gradient(t, experts, top, renormalize, score, dt):
    """Against the formula by automatic differentiation in 64 bits, and against differences."""
    g = gen(experts)
    logits, dw, scale = torch.randn(t, experts, generator=g).to(dt), torch.randn(t, top, generator=g), 1.5
    indices, _ = route64(logits, top, score=score)
    if top > 2:
        indices[0, 1], indices[0, 2] = -1, indices[0, 0]      # a choice that is none, and one that stands twice
    l = logits.double().requires_grad_()
    (route_weights(l, indices, score, renormalize, scale) * dw.double()).sum().backward()
    got = device_grad(logits, indices, dw, score=score, renormalize=renormalize, scale=scale)
    # terms of the gradient before they cancel: |dw| scale times the slope, at most |dw| scale
    size = dw.double().abs().sum(dim=1, keepdim=True) * scale
    assert ((got.double() - l.grad).abs() <= l.grad.abs() * half_step(dt) + size * 16 * half_step(F32) + torch.finfo(dt).smallest_normal * half_step(dt)).all()
    for e in range(0, experts, max(1, experts // 5)):
        h = torch.zeros(t, experts, dtype=torch.float64)
        h[:, e] = 1e-5
        up, down = (route_weights(logits.double() + x, indices, score, renormalize, scale) for x in (h, -h))
        slope = ((up - down) * dw.double()).sum(dim=1) / 2e-5
        assert ((got[:, e].double() - slope).abs() <= slope.abs() * half_step(dt) + size[:, 0] * 1e-6 + torch.finfo(dt).smallest_normal * half_step(dt)).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_gradient_of_one_choice_is_zero(score):
    """One renormalised weight is 1 whatever the logits are."""
    logits = torch.randn(200, 24, generator=gen(1))
    indices, _ = route64(logits, 1, score=score)
    assert not device_grad(logits, indices, torch.randn(200, 1, generator=gen(2)), score=score).any()


# ---------------------------------------------------------------- order
def device_order(indices, experts):
    t, top = indices.shape
    offsets = torch.full((experts + 2,), 77, dtype=torch.int32, device=DEV)
    source, place = torch.full((t * top + 1,), 77, dtype=torch.int32, device=DEV), torch.full((t + 1, top), 77, dtype=torch.int32, device=DEV)
    oz.expert_order(indices.to(DEV), experts, offsets[:-1], source[:-1], place[:-1], oz.alloc_expert_order_workspace(t, top, experts))
    assert offsets[-1] == 77 and source[-1] == 77 and (place[-1] == 77).all()
    return offsets[:-1].cpu(), source[:-1].cpu(), place[:-1].cpu()


@pytest.mark.parametrize("t,top,experts", [(1, 1, 1), (7, 3, 5), (64, 8, 64), (1000, 4, 33), (513, 8, 256), (600, 7, 1024), (3000, 3, 2), (5000, 4, 100), (40000, 1, 1024), (16384, 8, 256), (70000, 4, 70), (150000, 8, 8)])
def test_order(t, top, experts):
    g = gen(t)
    indices = torch.randint(-1 if t % 2 else 0, experts, (t, top), generator=g, dtype=torch.int32)
    indices[0, 0] = experts + 3 if t > 100 else indices[0, 0]
    if experts > 10:
        indices[indices % 7 == 3] = 0      # experts without rows, and a crowded one
    flat = indices.reshape(-1).long()
    there = (flat >= 0) & (flat < experts)
    key = torch.where(there, flat, torch.full_like(flat, experts))
    rows = key.sort(stable=True).indices[:int(there.sum())]
    place = torch.full_like(flat, -1)
    place[rows] = torch.arange(len(rows))
    offsets = torch.nn.functional.pad(torch.bincount(key, minlength=experts + 1)[:experts].cumsum(0), (1, 0))
    got = device_order(indices, experts)
    assert torch.equal(got[0].long(), offsets)
    assert torch.equal(got[1][:len(rows)].long(), rows // top) and (got[1][len(rows):] == -1).all()
    assert torch.equal(got[2].view(-1).long(), place)
    if t * top <= 600:
        o, s, p = order64(torch.where((indices < experts), indices, -1), experts)
        assert got[0].tolist() == o and got[1].tolist() == s and got[2].view(-1).tolist() == p


def test_order_of_no_tokens():
    offsets = torch.full((4,), 77, dtype=torch.int32, device=DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    oz.expert_order(none.view(0, 2), 3, offsets, none, none.view(0, 2))
    assert not offsets.any()


# ---------------------------------------------------------------- combine
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("t,top,n,extra,offset", [(1, 1, 1, 0, 0), (5, 3, 7, 0, 0), (33, 8, 129, 3, 1), (9, 32, 1000, 8, 8), (300, 2, 64, 0, 0), (4, 5, 5000, 1, 3), (2, 4, 10001, 0, 0)])
def test_combine(t, top, n, extra, offset, dt):
    g = gen(n)
    rows = t * top + 5
    O0, dY0 = torch.randn(rows, n, generator=g).to(dt), torch.randn(t, n, generator=g).to(dt)
    place = torch.randperm(rows, generator=g)[:t * top].view(t, top).int()
    weights = torch.randn(t, top, generator=g)
    if t > 1:
        place[1, 0], place[0, top - 1] = -1, rows + 3      # pairs without a row
    there = (place >= 0) & (place < rows)
    picked = torch.where(there[:, :, None], O0.double()[place.clamp(0, rows - 1).long()], torch.zeros((), dtype=torch.float64))
    O, _ = guarded(rows, n, dt, extra, offset)
    O.copy_(O0)
    for w in (weights, None):
        Y, buf = guarded(t, n, dt, extra, offset)
        oz.expert_combine(O, place.to(DEV), None if w is None else w.to(DEV), Y)
        terms = picked if w is None else picked * w.double()[:, :, None]
        want = terms.sum(dim=1)
        allowed = want.abs() * half_step(dt) + terms.abs().sum(dim=1) * top * half_step(F32) + torch.finfo(dt).smallest_normal * half_step(dt)
        assert ((Y.double().cpu() - want).abs() <= allowed * (1 + 2.0 ** -10)).all()
        assert untouched(buf, t, n, extra, offset)
    dY, _ = guarded(t, n, dt, extra, offset)
    dY.copy_(dY0)
    dO, buf = guarded(rows, n, dt, extra, offset)
    dw = torch.full((t, top), 77.0, device=DEV)
    oz.expert_combine_grad(dY, O, place.to(DEV), weights.to(DEV), dO, dw)
    want = torch.full((rows, n), 77.0, dtype=torch.float64)
    want[place[there].long()] = (weights.double()[:, :, None] * dY0.double()[:, None, :])[there]
    # the product rounded to 32 bits and then to the type, or at once (0.85083008406: fp16 0.8510742 at once, 0.8505859 by 32 bits, which hold a tie)
    allowed = want.abs() * (half_step(dt) + half_step(F32) * (dt != F32)) + torch.finfo(dt).smallest_normal * half_step(dt)
    allowed[(want == 77.0)] = 0
    assert ((dO.double().cpu() - want).abs() <= allowed).all()
    assert untouched(buf, rows, n, extra, offset)
    dots, size = (picked * dY0.double()[:, None, :]).sum(dim=2), (picked * dY0.double()[:, None, :]).abs().sum(dim=2)
    assert ((dw.double().cpu() - dots).abs() <= size * (n + 64) * half_step(F32)).all()


def test_combine_of_values_that_are_not_finite():
    """A pair without a row is a row of zeros: its weight still tells a NaN; rows that are not finite reach their tokens alone."""
    O = torch.randn(4, 8, device=DEV)
    O[2, 3] = INF
    place = torch.tensor([[0, -1], [1, 2], [3, -1]], dtype=torch.int32, device=DEV)
    w = torch.tensor([[1.0, 2.0], [1.0, 0.5], [1.0, NAN]], device=DEV)
    Y = torch.empty(3, 8, device=DEV)
    oz.expert_combine(O, place, w, Y)
    assert torch.equal(Y[0], O[0]) and Y[2].isnan().all()
    assert Y[1, 3] == INF and torch.isfinite(Y[1, [0, 1, 2, 4, 5, 6, 7]]).all()


# ---------------------------------------------------------------- together
def layer(x, logits, bias, w1, w2, dy, top, dt, groups=1, top_groups=1, workspaces=None):
    """A layer of experts, forward and backward, from the operators: what a program calls."""
    t, k = x.shape
    E, n = w1[0].shape[:2]
    rows = t * top
    new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device=DEV)
    indices, weights, place = new(t, top, dtype=torch.int32), new(t, top, dtype=F32), new(t, top, dtype=torch.int32)
    offsets, source = new(E + 1, dtype=torch.int32), new(rows, dtype=torch.int32)
    oz.route(logits, indices, weights, bias=bias, score="sigmoid", groups=groups, top_groups=top_groups, scale=2.0)
    oz.expert_order(indices, E, offsets, source, place, workspaces["order"])
    h, o, y = new(rows, n).zero_(), new(rows, k).zero_(), new(t, k)
    oz.f8_gemm(x, *w1, h, workspaces["gemm1"], offsets=offsets, source=source)
    a = torch.relu(h)
    oz.f8_gemm(a, *w2, o, workspaces["gemm2"], offsets=offsets)
    oz.expert_combine(o, place, weights, y)
    do, dw, da, dh, dx_rows, dx = new(rows, k).zero_(), new(t, top, dtype=F32), new(rows, n).zero_(), new(rows, n), new(rows, k).zero_(), new(t, k)
    dw1, dw2, dl = new(E, n, k), new(E, k, n), torch.empty_like(logits)
    oz.expert_combine_grad(dy, o, place, weights, do, dw)
    oz.f8_gemm_grad(do, *w2, da, workspaces["grad2"], offsets=offsets)
    oz.f8_weight_grad(do, a, dw2, workspaces["wgrad2"], offsets=offsets)
    dh = torch.where(h > 0, da, torch.zeros((), dtype=dt, device=DEV))
    oz.f8_gemm_grad(dh, *w1, dx_rows, workspaces["grad1"], offsets=offsets)
    oz.f8_weight_grad(dh, x, dw1, workspaces["wgrad1"], offsets=offsets, source=source)
    oz.expert_combine(dx_rows, place, None, dx)
    oz.route_grad(logits, indices, dw, dl, score="sigmoid", scale=2.0)
    return dict(indices=indices, weights=weights, offsets=offsets, y=y, dx=dx, dw1=dw1, dw2=dw2, dl=dl, h=h, a=a, o=o, do=do, dh=dh)


def layer_case(t, k, n, E, top, dt, seed):
    g = gen(seed)
    x, dy = torch.randn(t, k, generator=g).to(dt), torch.randn(t, k, generator=g).to(dt)
    logits, bias = torch.randn(t, E, generator=g), 0.1 * torch.randn(E, generator=g)
    logits[0] = -INF                       # a padded token: it goes to no expert
    W1, W2 = torch.randn(E, n, k, generator=g) / math.sqrt(k), torch.randn(E, k, n, generator=g) / math.sqrt(n)

    def cut_all(W):
        parts = []
        for w in W:
            codes = torch.empty(w.shape[0], oz.f8_row_bytes(w.shape[1]), dtype=torch.uint8, device=DEV)
            scales = torch.empty(-(-w.shape[0] // 128), oz.f8_scale_bytes(w.shape[1]), dtype=torch.uint8, device=DEV)
            oz.f8_split(w.to(DEV), codes, scales)
            parts.append((codes, scales))
        return torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])

    rows = t * top
    alloc = oz.alloc_f8_workspace
    workspaces = {"order": oz.alloc_expert_order_workspace(t, top, E), "gemm1": alloc("gemm", t, n, k, dt, rows=rows, experts=E), "gemm2": alloc("gemm", rows, k, n, dt, rows=rows, experts=E),
                  "grad1": alloc("grad", rows, n, k, dt, rows=rows, experts=E), "grad2": alloc("grad", rows, k, n, dt, rows=rows, experts=E),
                  "wgrad1": alloc("weight_grad", t, n, k, dt, rows=rows, experts=E), "wgrad2": alloc("weight_grad", rows, k, n, dt, rows=rows, experts=E)}
    return x, dy, logits, bias, W1, W2, cut_all(W1), cut_all(W2), workspaces


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("t,k,n,E,top", [(3, 130, 100, 4, 2), (70, 260, 150, 8, 3)])
def test_layer(t, k, n, E, top, dt):
    """Each step against its 64-bit form on the inputs that it had, so that no step's rounding is counted in the next."""
    x, dy, logits, bias, W1, W2, w1, w2, workspaces = layer_case(t, k, n, E, top, dt, t)
    r = layer(x.to(DEV), logits.to(DEV), bias.to(DEV), w1, w2, dy.to(DEV), top, dt, workspaces=workspaces)
    r = {name: v.cpu() for name, v in r.items()}
    indices, weights = route64(logits, top, bias, "sigmoid", scale=2.0)
    assert torch.equal(r["indices"], indices) and (r["indices"][0] == -1).all()
    check_weights(r["weights"], weights)
    offsets, source, place = order64(indices, E)
    assert r["offsets"].tolist() == offsets
    used = offsets[-1]
    assert not r["y"][0].any() and not r["dx"][0].any() and not r["dl"][0].any()
    steps = 2.0 ** -12      # (see the bound of the products' tests)
    def near(got, terms, magnitude, inner):
        allowed = magnitude * ((inner + 8) * 2.0 ** -23 + steps) + terms.abs() * half_step(dt) + torch.finfo(dt).smallest_normal
        assert ((got.double() - terms).abs() <= allowed * (1 + 2.0 ** -10)).all()
    src = torch.tensor(source[:used])
    V1, V2 = [cut(w, 128)[2] for w in W1], [cut(w, 128)[2] for w in W2]
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        u = cut(x[src[a:b]])[2] if b > a else x[:0].double()
        if b > a:
            near(r["h"][a:b], u @ V1[e].t(), u.abs() @ V1[e].abs().t(), k)
            ua = cut(r["a"][a:b])[2]
            near(r["o"][a:b], ua @ V2[e].t(), ua.abs() @ V2[e].abs().t(), n)
            P, Q = cut_columns(r["dh"][a:b]).t(), cut_columns(x[src[a:b]])
            near(r["dw1"][e], P @ Q, P.abs() @ Q.abs(), b - a)
            P, Q = cut_columns(r["do"][a:b]).t(), cut_columns(r["a"][a:b])
            near(r["dw2"][e], P @ Q, P.abs() @ Q.abs(), b - a)
        else:
            assert not r["dw1"][e].any() and not r["dw2"][e].any()
    p = torch.tensor(place).view(t, top)
    picked = torch.where((p >= 0)[:, :, None], r["o"].double()[p.clamp(min=0)], torch.zeros((), dtype=torch.float64)) * r["weights"].double()[:, :, None]
    near(r["y"], picked.sum(dim=1), picked.abs().sum(dim=1), top)


def test_layer_in_a_graph():
    t, k, n, E, top, dt = 40, 260, 150, 8, 3, BF16
    x, dy, logits, bias, W1, W2, w1, w2, workspaces = layer_case(t, k, n, E, top, dt, 5)
    x, dy, logits, bias = x.to(DEV), dy.to(DEV), logits.to(DEV), bias.to(DEV)
    names = ("indices", "weights", "offsets", "y", "dx", "dw1", "dw2", "dl")
    run = lambda: layer(x, logits, bias, w1, w2, dy, top, dt, groups=4, top_groups=2, workspaces=workspaces)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    g = gen(8)
    for _ in range(4):
        x.copy_(torch.randn(t, k, generator=g).to(dt))
        logits.copy_(torch.randn(t, E, generator=g))
        want = {a: v.clone() for a, v in run().items() if a in names}
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[a], want[a]) for a in names)


def test_stream_as_an_argument():
    """Each call on a stream that is handed over gives what it gives on the current one."""
    t, experts, top, n, k = 300, 16, 3, 200, 260
    g = gen(5)
    logits, X = torch.randn(t, experts, generator=g).to(DEV), torch.randn(t, k, generator=g).to(BF16).to(DEV)
    W, dw = torch.randn(experts, n, k, generator=g).to(DEV), torch.randn(t, top, generator=g).to(DEV)
    dY = torch.randn(t * top, n, generator=g).to(BF16).to(DEV)

    def run(stream):
        with torch.cuda.stream(torch.cuda.Stream() if stream is None else torch.cuda.current_stream()):
            new = lambda *shape, dt=torch.int32: torch.zeros(*shape, dtype=dt, device=DEV)
            i, w, dl = new(t, top), new(t, top, dt=F32), new(t, experts, dt=F32)
            offsets, source, place = new(experts + 1), new(t * top), new(t, top)
            codes, scales = new(experts, n, oz.f8_row_bytes(k), dt=torch.uint8), new(experts, 2, oz.f8_scale_bytes(k), dt=torch.uint8)
            back, Y, dX = new(n, k, dt=BF16), new(t * top, n, dt=BF16), new(t * top, k, dt=BF16)
            dW, out, dO, dweights = new(experts, n, k, dt=F32), new(t, n, dt=BF16), new(t * top, n, dt=BF16), new(t, top, dt=F32)
            ws = {op: oz.alloc_f8_workspace(op, t, n, k, BF16, rows=t * top, experts=experts) for op in ("gemm", "grad", "weight_grad")}
            order = oz.alloc_expert_order_workspace(t, top, experts)
            torch.cuda.synchronize()
            oz.route(logits, i, w, stream=stream)
            oz.route_grad(logits, i, dw, dl, stream=stream)
            oz.expert_order(i, experts, offsets, source, place, order, stream=stream)
            for e in range(experts):
                oz.f8_split(W[e], codes[e], scales[e], stream=stream)
            oz.f8_expand(codes[1], scales[1], back, stream=stream)
            oz.f8_gemm(X, codes, scales, Y, ws["gemm"], offsets=offsets, source=source, stream=stream)
            oz.f8_gemm_grad(dY, codes, scales, dX, ws["grad"], offsets=offsets, stream=stream)
            oz.f8_weight_grad(dY, X, dW, ws["weight_grad"], offsets=offsets, source=source, stream=stream)
            oz.expert_combine(Y, place, w, out, stream=stream)
            oz.expert_combine_grad(out, Y, place, w, dO, dweights, stream=stream)
            torch.cuda.synchronize()
        return i, w, dl, offsets, source, place, codes, scales, back, Y, dX, dW, out, dO, dweights

    for a, b in zip(run(None), run(torch.cuda.Stream())):
        assert torch.equal(a, b) and a.any()
