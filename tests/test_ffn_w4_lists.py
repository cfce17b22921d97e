"""moe_expert_ffn_w4_sliced where a launch ahead lists the rows by expert: both launches that can make the list, calls that take none, and offsets and maps that make no sense."""
import numpy as np
import pytest
import torch

from test_ffn_w4 import activations, check, offsets_of, run, weights
from test_ffn_w4_ways import check_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PLANS = {"ffn_small_plan_kernel", "ffn_plan_kernel"}


def kernels(lib, *args, **more):
    lib.moe_kernel_timing_enable(True)
    try:
        y = run(lib, *args, **more)
        return y, set(lib.moe_kernel_timing_read())
    finally:
        lib.moe_kernel_timing_enable(False)


# group, M of M + 3 rows, S, E, d, f, kernels: few groups and rows, whose list one workgroup makes, and a case that takes no list
SMALL_LIST = "ffn_small_plan_kernel"
SMALL = [(128, 1600, 1, 8, 256, 512, {SMALL_LIST, "ffn_w4_middle1_kernel", "ffn_w4_middle2_kernel"}), (32, 1000, 6, 4, 512, 512, {SMALL_LIST, "ffn_w4_middle1_kernel", "ffn_w4_middle2_kernel"}),
         (128, 1600, 6, 8, 256, 2048, {SMALL_LIST, "ffn_w4_large1_kernel", "ffn_w4_middle2_kernel"}), (64, 1600, 40, 8, 256, 1024, {"ffn_w4_middle1_kernel", "ffn_w4_small2_kernel"}),
         (64, 1600, 100, 8, 512, 1024, {SMALL_LIST, "ffn_w4_middle1_kernel", "ffn_w4_middle2_kernel"}), (128, 300, 3, 24, 2048, 1024, {SMALL_LIST, "ffn_w4_large1_kernel", "ffn_w4_large2_kernel"})]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group,M,S,E,d,f,expected", SMALL)
def test_small_list(lib, group, M, S, E, d, f, expected, zeros):
    rng = np.random.default_rng(M + E)
    off = offsets_of(rng.multinomial(M, rng.dirichlet(np.full(S * E, 0.5))))
    extra = 3
    x, w = activations(M + extra, d, M), weights(E, d, f, group, zeros, M + d)
    row_map, row_gate = rng.permutation(M + extra).astype(np.int32), rng.random(M + extra).astype(np.float32)
    y = torch.full((M + extra, d), 3.0, dtype=torch.bfloat16, device=DEV)
    _, names = kernels(lib, x, off, S, E, w, y=y, row_map=torch.from_numpy(row_map).to(DEV), row_gate=torch.from_numpy(row_gate).to(DEV))
    assert names == expected, names
    check_rows(y, x, off, E, w, row_map, row_gate)
    plain = run(lib, x, off, S, E, w)                                     # neither map nor weights
    check(plain, x, off, E, w)


@pytest.mark.parametrize("M,d,f,kernel", [(2000, 256, 512, "ffn_w4_large1_kernel"), (2000, 1024, 128, "ffn_w4_large2_kernel"), (3000, 256, 128, "ffn_w4_middle1_kernel"),
                                          (3000, 256, 128, "ffn_w4_middle2_kernel")])
def test_tiles_without_a_list(lib, M, d, f, kernel):
    E = 2
    off = offsets_of([M // 3, M - M // 3])
    x, w = activations(M, d, 1), weights(E, d, f, 128, True, 2)
    y, names = kernels(lib, x, off, 1, E, w)
    assert not names & PLANS and kernel in names, names
    check(y, x, off, E, w)


LISTED = [(1600, 8, 256, 512, "ffn_small_plan_kernel"), (3000, 8, 256, 512, "ffn_plan_kernel"), (3000, 8, 256, 2048, "ffn_plan_kernel")]


@pytest.mark.parametrize("M,E,d,f,plan", LISTED)
def test_malformed_offsets_stay_inside(lib, M, E, d, f, plan):
    """Boundaries that fall, pass M or are negative: nothing outside y is written, and with groups that do not overlap every row of theirs is right."""
    S, x, w = 2, activations(M, d, 1), weights(E, d, f, 128, True, 2)
    base = torch.full((M + 40, d), 5.0, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(M)
    anywhere = torch.from_numpy(rng.integers(-(1 << 31), 1 << 31, M).astype(np.int32)).to(DEV)
    for off in ([0, M] * (S * E // 2) + [0], [M - 64 * i for i in range(S * E + 1)], [-9, -3, 1 << 30] + [5] * (S * E - 2), list(rng.integers(-M, 2 * M, S * E + 1))):
        for more in ({}, dict(row_map=anywhere)):
            _, names = kernels(lib, x, np.array(off, dtype=np.int32), S, E, w, y=base[20:20 + M], **more)
            assert plan in names, names
            assert (base[:20] == 5).all() and (base[20 + M:] == 5).all()
    # a first boundary below 0 and a last one behind M count as 0 and M
    off = offsets_of(rng.multinomial(M, np.full(S * E, 1.0 / (S * E))))
    bent = off.copy()
    bent[0], bent[-1] = -77, M + 1000
    check(run(lib, x, bent, S, E, w), x, off, E, w)


@pytest.mark.parametrize("M,E,d,f,group,kernel", [(M, E, d, f, 128, plan) for M, E, d, f, plan in LISTED] + [(1600, 8, 256, 512, 64, "ffn_w4_small2_kernel"), (3000, 8, 256, 512, 64, "ffn_plan_kernel"),
                                                                                                     (3000, 8, 256, 2048, 64, "ffn_plan_kernel")])
def test_maps_out_of_range_name_row_0(lib, M, E, d, f, group, kernel):
    """Every fifth entry of the map lies outside [0, M); the others are right, and the rows that none names are left as they were."""
    S, x, w = 2, activations(M, d, 3), weights(E, d, f, group, False, 4)
    rng = np.random.default_rng(M + 1)
    off = offsets_of(rng.multinomial(M, np.full(S * E, 1.0 / (S * E))))
    row_map = rng.permutation(M).astype(np.int32)
    bad = (np.arange(M) % 5 == 2) | (row_map == 0)
    row_map[bad] = rng.choice(np.array([-1, M, M + 1, (1 << 31) - 1, -(1 << 31)]), bad.sum())
    y = torch.full((M, d), 3.0, dtype=torch.bfloat16, device=DEV)
    _, names = kernels(lib, x, off, S, E, w, y=y, row_map=torch.from_numpy(row_map).to(DEV))
    assert kernel in names, names
    got = y.cpu()
    left = np.setdiff1d(np.arange(1, M), row_map[~bad])
    assert (got[torch.from_numpy(left)] == 3).all()
    # the good entries as a schedule of their own
    sizes = [int((~bad[off[i]:off[i + 1]]).sum()) for i in range(S * E)]
    order = torch.from_numpy(row_map[~bad].astype(np.int64))
    check(got[order], x[order], offsets_of(sizes), E, w)
