"""moe_expert_ffn_w4_sliced: every kernel that its choice by sizes can take, named by the kernel timing, and rows far behind 2^31 bytes."""
import numpy as np
import pytest
import torch

from test_ffn_w4 import activations, check, offsets_of, run, weights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# group, M of M + 3 rows in the schedule, S, E, d, f: few rows and many, few experts and many, few slices and many
WAYS = [(32, 1, 1, 1, 256, 1024), (128, 1, 1, 8, 1024, 128), (128, 5, 1000, 2, 1024, 1024), (32, 16, 1, 1, 4096, 128), (128, 16, 1, 1, 256, 4096), (64, 33, 1, 2, 256, 4096),
        (32, 17, 1, 1, 256, 128), (128, 200, 1, 8, 256, 512), (32, 200, 1, 8, 256, 512), (128, 400, 1, 16, 256, 128), (128, 400, 1, 64, 256, 128), (128, 1000, 1, 16, 256, 512),
        (128, 2000, 3, 64, 256, 256), (32, 1, 2000, 1, 256, 128), (64, 700, 1200, 3, 256, 128), (128, 33, 1000, 64, 256, 512), (128, 200, 1000, 64, 1024, 128), (128, 3000, 1, 256, 256, 128),
        (64, 130, 1, 1, 512, 2048), (128, 2500, 1, 2, 512, 1024), (128, 100, 1, 4, 4096, 128), (128, 200, 1, 256, 256, 128), (128, 1, 1, 8, 256, 4096)]
ran = {}                                                                  # case -> its kernels


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group,M,S,E,d,f", WAYS)
def test_every_way(lib, group, M, S, E, d, f, zeros):
    rng = np.random.default_rng(M + S)
    sizes = rng.multinomial(M, rng.dirichlet(np.full(S * E, 0.3)))        # uneven, most groups empty
    off = offsets_of(sizes)
    extra = 3
    x, w = activations(M + extra, d, M), weights(E, d, f, group, zeros, M + d)
    row_map = rng.permutation(M + extra).astype(np.int32)                 # its first M entries are the schedule's
    row_gate = rng.random(M + extra).astype(np.float32)
    y = torch.full((M + extra, d), 3.0, dtype=torch.bfloat16, device=DEV)
    lib.moe_kernel_timing_enable(True)
    try:
        run(lib, x, off, S, E, w, y=y, row_map=torch.from_numpy(row_map).to(DEV), row_gate=torch.from_numpy(row_gate).to(DEV))
        names = set(lib.moe_kernel_timing_read())
    finally:
        lib.moe_kernel_timing_enable(False)
    print(names)
    ran[group, M, S, E, d, f, zeros] = names
    check_rows(y, x, off, E, w, row_map, row_gate)


def test_every_way_was_taken():
    """After the cases above: they have used every kernel for both products, and the list of rows and its absence."""
    if len(ran) < 2 * len(WAYS):
        pytest.skip("not all cases were run")
    names = set().union(*ran.values())
    assert names >= {"ffn_w4_%s%d_kernel" % (way, phase) for way in ("stream", "small", "middle", "large") for phase in (1, 2)} | {"ffn_plan_kernel"}, names
    assert any("ffn_plan_kernel" not in n and "ffn_w4_large1_kernel" in n for n in ran.values()) and any("ffn_plan_kernel" not in n and "ffn_w4_middle1_kernel" in n for n in ran.values())


def check_rows(y, x, off, E, w, row_map, row_gate):
    """test_ffn_w4.check for a map that names each row of x at most once and has as many entries as x has rows: the rows it leaves out keep their 3."""
    M = int(off[-1])
    order = torch.from_numpy(row_map[:M].astype(np.int64))
    got = y.cpu()[order]
    check(got, x[order], off, E, w, row_gate=row_gate[:M], kept=3.0)
    left = np.setdiff1d(np.arange(len(x)), row_map[:M])
    assert (y.cpu()[torch.from_numpy(left)].double() == 3.0).all()


@pytest.mark.parametrize("M,d,f,zeros", [(131000, 16384, 128, True), (131000, 256, 16384, False)])
def test_rows_behind_two_gib(lib, M, d, f, zeros):
    """Rows at the end of 4 GiB of x, y and intermediates: the last ones against the oracle, all others with an expert whose scales are zero."""
    E, S = 2, 1
    last = 70
    off = offsets_of([M - last, last])
    w = weights(E, d, f, 128, zeros, 5)
    for n in ("s_gate", "s_up", "s_down"):
        w[n][0] = 0.0
    tail = activations(last, d, 3)
    x = torch.ones(M, d, dtype=torch.bfloat16, device=DEV)
    x[M - last:] = tail.to(DEV)
    c = {k: (None if v is None else v.to(DEV)) for k, v in w.items()}
    y = lib.moe_expert_ffn_w4_sliced(x, torch.from_numpy(off).to(DEV), S, E, **c)
    assert not y[: M - last].any().item()
    one = {k: (None if v is None else v[1:]) for k, v in w.items()}
    check(y[M - last:], tail, offsets_of([last]), 1, one)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("E,M,e,S", [(8, 200, 3, 1), (64, 300, 63, 5), (8, 41, 0, 1), (4, 2000, 1, 2)])
def test_all_rows_with_one_expert(lib, E, M, e, S, group):
    """An expert with many times the average has more row blocks than its grid has: workgroups take another one."""
    sizes = np.zeros(S * E, dtype=int)
    sizes[e::E] = np.random.default_rng(M).multinomial(M, np.full(S, 1.0 / S))
    off = offsets_of(sizes)
    x, w = activations(M, 512, M), weights(E, 512, 512, group, True, M)
    check(run(lib, x, off, S, E, w), x, off, E, w)


def test_millions_of_rows(lib):
    """More row blocks than a grid's third dimension counts; the last rows against the oracle, the others with scales of zero."""
    M, d, f, last = 4194304 + 700, 256, 128, 70
    off = offsets_of([M - last, last])
    w = weights(2, d, f, 128, True, 9)
    for n in ("s_gate", "s_up", "s_down"):
        w[n][0] = 0.0
    tail = activations(last, d, 4)
    c = {k: v.to(DEV) for k, v in w.items()}
    x = torch.ones(M, d, dtype=torch.bfloat16, device=DEV)
    x[M - last:] = tail.to(DEV)
    y = lib.moe_expert_ffn_w4_sliced(x, torch.from_numpy(off).to(DEV), 1, 2, **c)
    assert not y[: M - last].any().item()
    check(y[M - last:], tail, offsets_of([last]), 1, {k: v[1:] for k, v in w.items()})
    # one expert, so that no list of the rows is made: the same rows in the same places
    y = lib.moe_expert_ffn_w4_sliced(x, torch.tensor([0, M], dtype=torch.int32, device=DEV), 1, 1, **{k: v[1:] for k, v in c.items()})
    check(y[M - last:], tail, offsets_of([last]), 1, {k: v[1:] for k, v in w.items()})
    assert torch.equal(y[: M - last], y[:1].expand(M - last, d))


@pytest.mark.parametrize("M", [5, 700])
def test_most_experts(lib, M):
    """65536 experts, all that the groups of a schedule allow: rows with the first, the last and some between."""
    E, d, f, G = 65536, 256, 128, 128
    some = [0, 1, 32768, 65534, 65535]
    w = weights(len(some), d, f, G, True, 3)
    c = {}
    for n, v in w.items():
        c[n] = torch.zeros((E,) + tuple(v.shape[1:]), dtype=v.dtype, device=DEV)
        c[n][torch.tensor(some, device=DEV)] = v.to(DEV)
    sizes = np.zeros(E, dtype=int)
    sizes[some] = np.random.default_rng(M).multinomial(M, np.full(len(some), 1.0 / len(some)))
    x = activations(M, d, M)
    y = lib.moe_expert_ffn_w4_sliced(x.to(DEV), torch.from_numpy(offsets_of(sizes)).to(DEV), 1, E, **c)
    check(y, x, offsets_of(sizes[some]), len(some), w)
