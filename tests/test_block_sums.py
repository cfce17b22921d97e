"""Gradients of the norms' weights, which are sums over the tokens: many rows of which some scattered ones have a gradient, so that the sum over all workgroups is that of few terms."""
import pytest
import torch

from test_block import CHAIN

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


def repeated(rows, T, d, dtype, seed):
    return torch.randn(rows, d, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV).repeat((T + rows - 1) // rows, 1)[:T]


# up to more than 2^31 elements
@pytest.mark.parametrize("T,d,dtype", [(524288 + 515, 4096, torch.bfloat16), (70001, 64, torch.float32), (33333, 2304, torch.float32), (9999, 7168, torch.bfloat16), (5001, 8200, torch.bfloat16)])
def test_weight_gradients_over_many_rows(lib, T, d, dtype):
    """A term is off by CHAIN of what it is made of (a row's sums and a handful of products), twice where it goes through both norms; adding n of them, and zeros, rounds n times."""
    z, out = repeated(1031, T, d, torch.bfloat16, 1), repeated(1033, T, d, dtype, 2)
    g = torch.Generator().manual_seed(3)
    pick = torch.unique(torch.cat([torch.randint(0, T, (150,), generator=g), torch.tensor([0, 1, T // 2, T - 1]), T - 1 - torch.randint(0, 300, (20,), generator=g)])).to(DEV)
    n = len(pick)
    d_next, d_out = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV), torch.zeros(T, d, dtype=dtype, device=DEV)
    d_next[pick] = torch.randn(n, d, generator=g).bfloat16().to(DEV)
    d_out[pick] = torch.randn(n, d, generator=g).to(dtype).to(DEV)
    w1, w2 = torch.linspace(0.5, 1.5, d, device=DEV), torch.linspace(-1.0, 1.0, d, device=DEV)
    gate = torch.rand(T, generator=g).to(DEV)
    join = lib.moe_block_join_backward(d_out, d_next, z, out, w1, gate, w2, 0.75, EPS)
    norm = lib.moe_block_norm_backward(d_next, out, w2, EPS)
    n1, n2 = (v / (v.square().mean(1, keepdim=True) + EPS).sqrt() for v in (z[pick].double(), out[pick].double()))
    r2 = 1 / (out[pick].double().square().mean(1, keepdim=True) + EPS).sqrt()
    dn, do, gt = d_next[pick].double(), d_out[pick].double(), gate[pick].double()[:, None]
    through = dn * w2.double()
    total = do + r2 * (through - n2 * (through * n2).mean(1, keepdim=True))
    size = do.abs() + r2 * (through.abs() + n2.abs() * (through * n2).abs().mean(1, keepdim=True))
    adds = (n + 32) * 2.0 ** -24
    for got, terms, parts, off in ((norm["d_weight"], dn * n2, (dn * n2).abs(), CHAIN), (join["d_next_weight"], dn * n2, (dn * n2).abs(), CHAIN),
                                   (join["d_post_weight"], gt * total * n1, gt * size * n1.abs(), 2 * CHAIN)):
        err, tol = (got.double() - terms.sum(0)).abs(), (off + adds) * parts.sum(0)
        assert (err <= tol).all(), float((err / tol).max())
        assert float((tol / terms.sum(0).abs().mean()).max()) < 1e-2      # (small beside the sums, so that a row that is lost shows)
