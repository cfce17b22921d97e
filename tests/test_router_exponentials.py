"""moe_router_topk with softmax scores of two experts: the exponential over its whole range, from the weights and from the gradient, against float64."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
STEP = 2.0 ** -23                                 # a step of fp32 is at most this much of the value


def differences():
    """Two logits of which one is 0: their difference x is exact.  Dense from 0 to 100, around multiples of ln 2, and tiny."""
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.linspace(0, 100, 400001), torch.rand(200000, generator=g) * 2, torch.arange(145) * 0.69314718, 2.0 ** torch.arange(-60.0, 7.0)]).float()
    return x.to(DEV)


def logits_of(x, E):
    """The two experts' columns are 1 and E - 2; the others are masked."""
    l = torch.full((len(x), E), -float("inf"), device=DEV)
    l[:, 1] = 0.0
    l[:, E - 2] = -x
    return l


@pytest.mark.parametrize("E", [4, 64, 100, 256, 300])
def test_gradient(lib, E):
    """d of the smaller one's weight w = e / (1 + e) is w (1 - w).  The exponential is off by 2 steps, which move w (1 - w) by up to 1 + w / (1 - w) times as much; beside it stand fewer than
    16 roundings of half a step.  Results below 2^-126 may be anything from zero to that."""
    x = differences()
    l = logits_of(x, E)
    ids = torch.full((len(x), 1), E - 2, dtype=torch.int32, device=DEV)
    d = lib.moe_router_topk_backward(torch.ones(len(x), 1, device=DEV), l, ids, "softmax", False).double()
    e = torch.exp(-x.double())
    w = e / (1 + e)
    want = w * (1 - w)
    tol = want * ((1 + w / (1 - w)) * 2 * STEP + 8 * STEP) + 2.0 ** -126
    assert (d[:, E - 2] - want).abs().le(tol).all(), float(((d[:, E - 2] - want).abs() / tol).max())
    assert (d[:, 1] + want).abs().le(tol).all(), float(((d[:, 1] + want).abs() / tol).max())
    rest = [c for c in range(E) if c not in (1, E - 2)]
    assert not d[:, rest].any()


@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("E,T", [(4, None), (64, None), (100, None), (256, None), (256, 3000), (300, None)])
def test_weights(lib, E, T, renormalise):
    """w = e / (1 + e) and 1 - w = 1 / (1 + e): 2 steps of the exponential and fewer than 16 roundings of half a step."""
    x = differences()
    x = x if T is None else x[torch.randperm(len(x), generator=torch.Generator().manual_seed(2))[:T].to(DEV)]
    ids, gates = lib.moe_router_topk(logits_of(x, E), 2, "softmax", renormalise)
    e = torch.exp(-x.double())
    want = torch.stack([1 / (1 + e), e / (1 + e)], 1)
    assert (ids[:, 0] == 1).all() and (ids[:, 1] == E - 2).all()          # the lower index where they are equal
    tol = want * 10 * STEP + 2.0 ** -126
    assert (gates.double() - want).abs().le(tol).all(), float(((gates.double() - want).abs() / tol).max())
