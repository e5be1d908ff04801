"""The gradient of the weights alone: the experts' rows have none where they are frozen.

A sum of D products in fp32 in any order is off by at most D 2^-23 times the sum of the magnitudes.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,k,E,D,pad", [(1, 1, 1, 1, 0), (1, 2, 4, 768, 0), (300, 3, 7, 1001, 0), (77, 8, 16, 64, 5), (2049, 2, 16, 1152, 8)])
def test_gradient_of_the_weights_alone(M, T, k, E, D, pad, dtype):
    g = torch.Generator().manual_seed(T + D)
    ids = torch.randint(-1, E, (T, k), generator=g).to(torch.int32).cuda()
    plan = M.expert_sort(ids, E)
    dout, rows = (torch.randn(n, D + pad, generator=g).to(dtype).cuda()[:, :D] for n in (T, T * k))
    weights = torch.randn(T, k, generator=g).cuda()
    drows, dw = M.expert_combine_grad(dout, rows, plan, weights, drows=False)
    assert drows is None
    place = plan.place.long()
    terms = torch.where((place >= 0)[..., None], rows.double()[place.clamp(min=0)], 0.0) * dout.double()[:, None]
    assert bool(((dw.double() - terms.sum(-1)).abs() <= D * 2.0 ** -23 * terms.abs().sum(-1)).all())
    given = torch.full_like(dw, 3.0)
    assert M.expert_combine_grad(dout, rows, plan, weights, drows=False, dweights=given)[1] is given and torch.equal(given, dw)
    assert M.expert_combine_grad(dout, rows, plan, weights, drows=False, dweights=False) == (None, None)
    both = M.expert_combine_grad(dout, rows, plan, weights)
    assert both[0].shape == rows.shape and bool(((both[1].double() - terms.sum(-1)).abs() <= D * 2.0 ** -23 * terms.abs().sum(-1)).all())
