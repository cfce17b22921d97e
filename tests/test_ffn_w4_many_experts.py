"""moe_expert_ffn_w4_sliced with few rows on a rank that holds many experts: which kernels the call takes, and its results."""
import numpy as np
import pytest
import torch

from test_ffn_w4 import activations, check, offsets_of, weights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def few_experts_hold_rows(lib, E, M, d, f, group, zeros):
    """-> names of the kernels that a call takes whose rows lie with four of its E experts (the others' codes are zeros)"""
    some = sorted({0, E // 3, E // 2, E - 1})
    w = weights(len(some), d, f, group, zeros, E + M)
    c = {}
    for n, v in w.items():
        c[n] = None
        if v is not None:
            c[n] = torch.zeros((E,) + tuple(v.shape[1:]), dtype=v.dtype, device=DEV)
            c[n][torch.tensor(some, device=DEV)] = v.to(DEV)
    sizes = np.zeros(E, dtype=int)
    sizes[some] = np.random.default_rng(E + M).multinomial(M, np.full(len(some), 1.0 / len(some)))
    x = activations(M, d, M)
    lib.moe_kernel_timing_enable(True)
    try:
        y = lib.moe_expert_ffn_w4_sliced(x.to(DEV), torch.from_numpy(offsets_of(sizes)).to(DEV), 1, E, **c)
        names = set(lib.moe_kernel_timing_read())
    finally:
        lib.moe_kernel_timing_enable(False)
    check(y, x, offsets_of(sizes[some]), len(some), w)
    return names


@pytest.mark.parametrize("group,zeros", [(128, False), (32, True)])
@pytest.mark.parametrize("E,M,d,f", [(64, 1, 256, 2048), (64, 3, 2048, 256), (128, 3, 2048, 128), (128, 2, 256, 4096), (128, 4, 2048, 768)])
def test_idle_workgroups_are_counted(lib, E, M, d, f, group, zeros):
    """Streaming launches a row of workgroups for every expert; where hardly any expert has rows they would be nearly all of its time (128 experts of 2048 x 768: 4 rows 51 + 64 us
    against 15 + 15 in tiles)."""
    names = few_experts_hold_rows(lib, E, M, d, f, group, zeros)
    assert not any("stream" in n for n in names), names


def test_few_experts_still_stream(lib):
    assert "ffn_w4_stream1_kernel" in few_experts_hold_rows(lib, 4, 4, 4096, 128, 128, False)
