"""The backward passes of moe_block_norm and moe_block_join where a row's sum of squares passes the range of fp32: such a row counts as infinitely long, so that
nothing flows back through its norm, and the other rows and the sums over the tokens are what they are without it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LONG = 3                                          # rows 0 .. 2 of the five


def rows(T, d, dtype, seed):
    return torch.randn(T, d, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def with_long_rows(x, length):
    """Rows 0 and 1 of one sign and of both, row 2 long in one half; and the same rows as zeros, which add nothing to a sum over the tokens either."""
    a, b = x.clone(), x.clone()
    a[0] = length
    a[1] = length * torch.sign(x[1].float()).to(x.dtype)
    a[2, ::2] = -length
    b[:LONG] = 0
    return a, b


@pytest.mark.parametrize("length", [1e20, 1e36, 3e38])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 1000, 2048, 2304, 4096, 7168, 8200])
def test_norm_backward(lib, d, dtype, length):
    T = 5
    x, zeros = with_long_rows(rows(T, d, dtype, 1), length)
    # gradients of one sign make the product with the row as large as can be
    d_out, d_stream, w = rows(T, d, torch.bfloat16, 2).abs() * 8, rows(T, d, dtype, 3), torch.linspace(0.5, 4.0, d, device=DEV)
    assert not lib.moe_block_norm(x, w)[:LONG].any()
    got, other = lib.moe_block_norm_backward(d_out, x, w, d_stream=d_stream), lib.moe_block_norm_backward(d_out, zeros, w, d_stream=d_stream)
    assert torch.equal(got["d_x"][:LONG], d_stream[:LONG])
    assert torch.equal(got["d_x"][LONG:], other["d_x"][LONG:]) and torch.equal(got["d_weight"], other["d_weight"])


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("length", [1e20, 1e36, 3e38])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 1000, 2048, 2304, 4096, 7168, 8200])
def test_join_backward(lib, d, dtype, length, gated):
    T = 5
    z, z0 = with_long_rows(rows(T, d, torch.bfloat16, 1), length)
    out, out0 = with_long_rows(rows(T, d, dtype, 4), length)
    d_next, d_out, w = rows(T, d, torch.bfloat16, 2).abs() * 8, rows(T, d, dtype, 3).abs() * 8, torch.linspace(0.5, 4.0, d, device=DEV)
    gate = torch.rand(T, generator=torch.Generator().manual_seed(5)).to(DEV) if gated else None
    got, other = (lib.moe_block_join_backward(d_out, d_next, a, b, w, gate, w, 0.75) for a, b in ((z, out), (z0, out0)))
    assert torch.equal(got["d_stream"][:LONG], (0.75 * d_out[:LONG].float()).to(dtype)) and not got["d_z"][:LONG].any()
    for name in ("d_stream", "d_z") + (("d_gate",) if gated else ()):
        assert torch.equal(got[name][LONG:], other[name][LONG:]), name
    if gated:
        assert not got["d_gate"][:LONG].any()
    for name in ("d_post_weight", "d_next_weight"):
        assert torch.equal(got[name], other[name]), name
