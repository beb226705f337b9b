"""The choice of experts where logits do not show its order: sigmoid scores that are 0 in 64 bits. Against the plain form in 64 bits."""
import pytest
import torch

from f8_plain import F32, TYPES, half_step, route64
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


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


# ---------------------------------------------------------------- scores that are 0
def test_sigmoid_scores_of_zero_are_equal():
    """Fewer ordinary logits than choices: of the others, all of whose scores are 0 in 64 bits, the lowest index comes first."""
    row = torch.tensor([[-800.0, -750.0, -2e4, -900.0, 2.0, 1.0, -1000.0, -1e4]])
    for bias in (None, torch.zeros(8)):
        indices, weights = torch.empty(1, 4, dtype=torch.int32, device=DEV), torch.empty(1, 4, device=DEV)
        oz.route(row.to(DEV), indices, weights, bias=None if bias is None else bias.to(DEV), score="sigmoid")
        assert indices.tolist() == [[4, 5, 0, 1]] and weights[0, 2:].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top,groups,top_groups", [(8, 4, 1, 1), (40, 15, 1, 1), (256, 8, 1, 1), (256, 20, 1, 1), (300, 8, 1, 1), (1000, 32, 1, 1), (64, 8, 8, 4)])
def test_finite_masks(experts, top, groups, top_groups, score, dt):
    """Masks of finite numbers beside few ordinary logits, and logits about where a sigmoid score becomes subnormal and 0 (-708.4 to -709.8)."""
    g, t = gen(experts + top), 48
    l = torch.randn(t, experts, generator=g)
    ordinary = torch.rand(t, experts, generator=g).argsort(dim=1).argsort(dim=1) < torch.arange(t)[:, None] % (top + 2)
    far = -torch.exp(torch.rand(t, experts, generator=g) * 5 + 6.3)             # -545 to -8e4
    border = -705.0 - 10.0 * torch.rand(t, experts, generator=g)
    mask = torch.where((torch.arange(t) % 3 == 0)[:, None], border, far)
    mask[torch.arange(t) % 3 == 1] += -1e4
    logits = torch.where(ordinary, l, mask).clamp(min=torch.finfo(dt).min).to(dt)
    for bias in (None, torch.zeros(experts), torch.where(torch.arange(experts) % 5 == 0, 0.125, 0.0)):
        for renormalize in (True, False):
            check(logits, top, score=score, groups=groups, top_groups=top_groups, renormalize=renormalize, bias=bias)
