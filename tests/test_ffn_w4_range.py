"""moe_expert_ffn_w4_sliced at the ends of its range: activations of one sign next to the largest finite value, in x and between the products."""
import numpy as np
import pytest
import torch

from test_ffn_w4 import check, offsets_of, run, weights

pytestmark = pytest.mark.gpu
LARGEST = torch.finfo(torch.bfloat16).max
# few rows and many: streaming and every tile, for both products
SHAPES = [(1, 1, 256, 128), (1, 16, 256, 4096), (1, 16, 4096, 128), (1, 300, 256, 128), (1, 700, 256, 2048), (2, 3000, 256, 128), (2, 2000, 256, 512), (2, 2000, 1024, 128)]


def with_codes(w, codes):
    """All codes and zero points as far apart as they can be, or as they are."""
    if codes != "random":
        q, z = (0xFF, 0) if codes == "largest" else (0x00, 15)
        for n in ("gate", "up", "down"):
            w["q_" + n].fill_(q)
            if w["z_" + n] is not None:
                w["z_" + n].fill_(z)
    return w


@pytest.mark.parametrize("codes", ["random", "largest", "smallest"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("E,M,d,f", SHAPES)
def test_largest_activations_of_one_sign(lib, E, M, d, f, group, zeros, codes):
    """Rows of the largest finite value, of the smallest, and of both halves; scales of 2^-126 make the sums small: no sum of products on the way leaves the range of fp32."""
    w = with_codes(weights(E, d, f, group, zeros, M), codes)
    for n in ("gate", "up"):
        w["s_" + n] = torch.full_like(w["s_" + n], 2.0 ** -126)
    x = torch.full((M, d), LARGEST, dtype=torch.bfloat16)
    x[1::3] = -LARGEST
    x[2::3, ::2] = -LARGEST
    off = offsets_of([M - M // E * (E - 1)] + [M // E] * (E - 1))
    check(run(lib, x, off, 1, E, w), x, off, E, w)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("E,M,d,f", SHAPES)
def test_largest_hidden_activations(lib, E, M, d, f, group, zeros):
    """g = u near 1.7e19, so that h = g u is 0.8 .. 0.9 of the largest finite value in every column; down scales of 2^-126."""
    w = with_codes(weights(E, d, f, group, zeros, M), "largest")
    s = (2.0 ** 52 if zeros else 2.0 ** 53) * 256 / d
    for n in ("gate", "up"):
        w["s_" + n] = torch.full_like(w["s_" + n], s)
    w["s_down"] = torch.full_like(w["s_down"], 2.0 ** -126)
    x = torch.ones((M, d), dtype=torch.bfloat16)
    if not zeros:
        x[:, -d // 32:] = 2.0                                             # 7 * 264 * 2^53 = 1.66e19
    x[1::2] = -x[1::2]                                                    # silu of -1.7e19: zero rows between them
    off = offsets_of([M - M // E * (E - 1)] + [M // E] * (E - 1))
    y = run(lib, x, off, 1, E, w)
    check(y, x, off, E, w)
    assert (y[::2] > 0).all() and not y[1::2].any()
