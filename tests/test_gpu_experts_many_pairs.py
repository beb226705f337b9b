"""More pairs than one dimension of a launch has threads for, a wavefront to each: 2^26 and up, within the 2^27 that the operators take."""
import pytest
import torch

from f8_plain import F16
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("t,top", [((1 << 22) - 3, 17), (1 << 22, 32)])
def test_combine_and_gradient(t, top):
    n, rows = 2, t * top
    assert rows > 1 << 26
    g = torch.Generator(device=DEV).manual_seed(top)
    O = torch.randint(-4, 5, (rows, n), generator=g, device=DEV, dtype=torch.int8).to(F16)
    dY = torch.randint(-4, 5, (t, n), generator=g, device=DEV, dtype=torch.int8).to(F16)
    weights = torch.randint(-2, 3, (t, top), generator=g, device=DEV, dtype=torch.int8).float()
    place = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device=DEV).view(t, top)
    dO, dw, Y = torch.full_like(O, 77.0), torch.full_like(weights, 77.0), torch.empty_like(dY)
    oz.expert_combine_grad(dY, O, place, weights, dO, dw)
    oz.expert_combine(O, place, weights, Y)
    picked, made = O.flip(0).view(t, top, n), dO.flip(0).view(t, top, n)
    for a in range(0, t, 1 << 19):      # small whole numbers: exact in every type here
        b = slice(a, min(t, a + (1 << 19)))
        assert torch.equal(made[b], weights[b][:, :, None].to(F16) * dY[b][:, None, :])
        assert torch.equal(dw[b], (picked[b].float() * dY[b].float()[:, None, :]).sum(dim=2))
        assert torch.equal(Y[b].float(), (picked[b].float() * weights[b][:, :, None]).sum(dim=1))


def test_order():
    t, top, experts = 1 << 22, 32, 60
    pairs = t * top
    g = torch.Generator(device=DEV).manual_seed(1)
    indices = torch.randint(-1, experts, (t, top), generator=g, device=DEV, dtype=torch.int32)
    offsets, source, place = torch.full((experts + 1,), 77, dtype=torch.int32, device=DEV), torch.full((pairs,), 77, dtype=torch.int32, device=DEV), torch.full_like(indices, 77)
    oz.expert_order(indices, experts, offsets, source, place, oz.alloc_expert_order_workspace(t, top, experts))
    key, row = indices.view(-1), place.view(-1)
    there = key >= 0
    assert (row[~there] == -1).all()
    used = int(there.sum())
    assert int(offsets[0]) == 0 and int(offsets[-1]) == used and (source[used:] == -1).all()
    pair = torch.full((used,), -1, dtype=torch.int32, device=DEV)
    pair[row[there].long()] = torch.arange(pairs, dtype=torch.int32, device=DEV)[there]
    assert (pair >= 0).all()      # every row has its pair
    assert torch.equal(source[:used], pair // top)
    of = key[pair.long()]
    assert ((of[1:] > of[:-1]) | ((of[1:] == of[:-1]) & (pair[1:] > pair[:-1]))).all()
    assert torch.equal(torch.bincount(of, minlength=experts).cumsum(0).int(), offsets[1:])
