"""The choice of experts where 32-bit values do not show which groups are best: those whose two largest values nearly cancel, or whose sum 32 bits do not
hold. Against the plain form in 64 bits."""
import math

import pytest
import torch

from f8_plain import F32, half_step, route64
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = math.inf
LOWEST = torch.finfo(F32).min


def gen(seed):
    return torch.Generator().manual_seed(seed)


def check(logits, top, **how):
    """Indices equal; weights within what test_gpu_experts.py allows."""
    t = logits.shape[0]
    indices, weights = torch.empty(t, top, dtype=torch.int32, device=DEV), torch.empty(t, top, device=DEV)
    bias = how.pop("bias", None)
    oz.route(logits.to(DEV), indices, weights, bias=None if bias is None else bias.to(DEV), **how)
    want, w = route64(logits, top, bias=bias, **how)
    assert torch.equal(indices.cpu(), want)
    assert ((weights.cpu().double() - w).abs() <= w.abs() * 8 * half_step(F32) + 2.0 ** -126).all()


GROUPS = [(16, 8, 4), (32, 4, 1), (256, 8, 4), (96, 6, 2), (512, 4, 2), (1024, 8, 3), (100, 10, 3)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [64.0, 1024.0, 2.0 ** 20])
@pytest.mark.parametrize("experts,groups,top_groups", GROUPS)
def test_groups_whose_values_nearly_cancel(experts, groups, top_groups, size, score):
    """Biases of opposite signs force one expert of a group on and push the others off: the two largest values nearly cancel, and each of them has been rounded by
    more than the groups are apart."""
    t, per = 400, experts // groups
    g = gen(experts)
    bias = torch.full((groups, per), -4.0 * size)
    bias[:, 0], bias[:, per - 1] = size, -size
    logits = torch.randn(t, groups, per, generator=g)
    s = torch.sigmoid(logits.double())
    for i in range(t if score == "sigmoid" else 0):      # sums of all groups within 2^-24 of the biases of each other
        total = (0.8 + 0.4 * torch.rand(1, generator=g).item()) + size * 2.0 ** -24 * torch.randn(groups, generator=g).double()
        logits[i, :, per - 1] = torch.logit((total - s[i, :, 0]).clamp(0.02, 0.98)).float()
    if score == "softmax":      # two groups alike in each token but for a few units
        for i in range(t):
            a, b = torch.randperm(groups, generator=g)[:2].tolist()
            logits[i, b] = logits[i, a] * (1 + 2.0 ** -20 * torch.randn(per, generator=g))
    logits = logits.view(t, experts)
    if groups > 2:      # the biases of some groups are another's
        bias[1] *= 0.5
        bias[2, 0] = bias[2, 0] + 1.0
    check(logits, 2, score=score, groups=groups, top_groups=top_groups, bias=bias.view(-1))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,top_groups", GROUPS)
def test_groups_under_the_lowest_bias(experts, groups, top_groups, score):
    """The lowest bias of 32 bits, or one next to it, is no -inf: where too few groups are without it, the sum of two of them still takes part."""
    t, per = 60, experts // groups
    g = gen(experts + 1)
    logits = torch.randn(t, experts, generator=g)
    top = min(2 * per, 15)
    for low in (LOWEST, -2e38, -1.8e38):
        for free in {0, 1, max(0, top_groups - 1), top_groups, min(groups, top_groups + 1)}:
            bias = torch.full((groups, per), low)
            for n, group in enumerate(torch.randperm(groups, generator=g)[:free].tolist()):
                bias[group] = 0.1 * torch.randn(per, generator=g)
                if n == 1:
                    bias[group, 1:] = low      # one of its experts is free
            check(logits, top, score=score, groups=groups, top_groups=top_groups, bias=bias.view(-1))
    bias = torch.where(torch.rand(experts, generator=g) < 0.3, torch.tensor(INF), 0.1 * torch.randn(experts, generator=g))
    bias[::7] = -INF
    check(logits, top, score=score, groups=groups, top_groups=top_groups, bias=bias)
    check(logits, top, score=score, groups=groups, top_groups=top_groups, bias=torch.where(torch.rand(experts, generator=g) < 0.5, 3e38, -3e38))
