"""The choice of experts with equal logits and biases that differ by less than 32 bits show, zero among them."""
import pytest
import torch

from f8_plain import TYPES, route64
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


def chosen(logits, top, bias, **how):
    t = logits.shape[0]
    indices, weights = torch.empty(t, top, dtype=torch.int32, device=DEV), torch.empty(t, top, device=DEV)
    oz.route(logits.to(DEV), indices, weights, bias=bias.to(DEV), **how)
    return indices.cpu()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("low,high", [(-1.0, 0.0), (0.0, 1.0), (-1.0, 1.0), (1.0, 2.0)])
def test_two_equal_logits(low, high, score):
    logits = torch.tensor([[1.921875, -3.0, 1.921875, -2.0, -4.0]])
    bias = torch.tensor([low, 0.0, high, 0.0, 0.0]) * 2.0 ** -24
    assert chosen(logits, 2, bias, score=score).tolist() == [[2, 0]]
    assert chosen(logits, 1, bias, score=score).tolist() == [[2]]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top,groups,top_groups", [(6, 2, 1, 1), (85, 2, 1, 1), (256, 8, 1, 1), (256, 8, 8, 4), (300, 3, 1, 1), (1000, 32, 1, 1), (100, 9, 10, 3)])
def test_many_equal_logits(experts, top, groups, top_groups, score, dt):
    g, t = torch.Generator().manual_seed(experts + top), 300
    logits = (torch.randn(t, experts, generator=g) * 8).round() / 8
    bias = torch.randint(-1, 2, (experts,), generator=g) * 2.0 ** -24
    how = dict(score=score, groups=groups, top_groups=top_groups)
    assert torch.equal(chosen(logits.to(dt), top, bias, **how), route64(logits.to(dt), top, bias, **how)[0])
