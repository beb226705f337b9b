"""The choice of experts where different logits have one score in 64 bits, beside equal logits: the lowest index comes first among all of them."""
import pytest
import torch

from f8_plain import TYPES, route64
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


def chosen(logits, top, **how):
    t = logits.shape[0]
    indices, weights = torch.empty(t, top, dtype=torch.int32, device=DEV), torch.empty(t, top, device=DEV)
    oz.route(logits.to(DEV), indices, weights, **how)
    return indices.cpu()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_logits_before_a_smaller_one_with_their_score(score):
    row = torch.tensor([[1e-30, -1.0, 2e-30, 2e-30, -1.0]])
    for dt in (torch.bfloat16, torch.float32):
        assert chosen(row.to(dt), 1, score=score).tolist() == [[0]]
        assert chosen(row.to(dt), 2, score=score).tolist() == [[0, 2]]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top", [(3, 1), (8, 2), (40, 5), (256, 15), (256, 20), (700, 8)])
def test_few_values_about_zero(experts, top, score, dt):
    g, t = torch.Generator().manual_seed(experts), 150
    steps = torch.randint(-3, 4, (t, experts), generator=g).float()
    size = torch.tensor([1e-30, 1e-20, 1e-16, 1e-12, 1e-9, 1e-7, 1e-6, 1e-5, 1e-3])[torch.arange(t) % 9][:, None]
    logits = torch.where(torch.rand(t, experts, generator=g) < 0.2, torch.randn(t, experts, generator=g), steps * size)
    logits[::2] = (steps * size)[::2]
    logits[9] = 0
    logits = logits.to(dt)
    got = chosen(logits, top, score=score).long()
    if score == "sigmoid":
        assert torch.equal(got.int(), route64(logits, top, score=score)[0])
        return
    # Two exponentials that 64 bits tell apart by a unit or two, 2^-53 of them each, have quotients by the sum that are equal or not as the sum's last bits
    # have it: (1 - 2^-53) / 3 is 1 / 3 in 64 bits, whose unit is 2^-54 there, and the sum's order is nobody's definition. Logits 10^-16 apart reach that,
    # and either order is right. Exponentials that are equal have equal quotients whatever the sum is: there the index decides.
    e = torch.exp(logits.double() - logits.double().amax(dim=1, keepdim=True))
    place = torch.full((t, experts), top).scatter_(1, got, torch.arange(top).expand(t, top))      # (those not chosen come behind all that are)
    assert (place < top).sum() == t * top
    for i in range(t):
        first = place[i][:, None] < place[i][None, :]
        a, b = e[i][:, None], e[i][None, :]
        before = torch.arange(experts)[:, None] < torch.arange(experts)[None, :]
        assert torch.where(a == b, before, a >= b * (1 - 2.0 ** -52))[first].all()
