"""moe_combine_topk_sum_backward: the oracle against differences of the forward oracle, refusals on the host, and the kernels against the oracle."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import workloads

DEV = "cuda:0"


def test_oracle_matches_differences_of_the_forward_pass():
    rng = np.random.default_rng(4)
    R, d, T, k = 5, 3, 4, 2
    row_of = np.array([[2, 0], [1, 1], [3, -1], [0, 7]], dtype=np.int32)      # row 1 twice by one token, row 0 by two, row 4 by none
    gate = rng.random((T, k)).astype(np.float32)
    y = workloads.activations(R, d, seed=2)
    d_out = rng.normal(size=(T, d))
    d_y, d_gate = oracle.combine_topk_sum_backward(d_out, oracle.decode_bf16(y), row_of, gate.astype(np.float64))
    value = lambda yb, g: (d_out * oracle.combine_topk_sum(yb, row_of, g)).sum()           # noqa: E731
    base = value(y, gate)
    for r in range(R):
        for c in range(d):
            y2 = y.copy()
            y2[r, c] = workloads.f32_to_bf16_bits(np.float32(oracle.decode_bf16(y)[r, c] + 1.0)).item()
            step = oracle.decode_bf16(y2)[r, c] - oracle.decode_bf16(y)[r, c]
            assert abs((value(y2, gate) - base) / step - d_y[r, c]) < 1e-10
    for t in range(T):
        for j in range(k):
            g2 = gate.copy()
            g2[t, j] += np.float32(1.0)
            assert abs((value(y, g2) - base) / (float(g2[t, j]) - float(gate[t, j])) - d_gate[t, j]) < 1e-10


def test_refusals_need_no_gpu(hostlib):
    L = hostlib.load()
    p, odd = ctypes.c_void_p(4096), ctypes.c_void_p(4104)

    def f(do=p, y=p, ro=p, gate=p, T=2, k=2, d=64, R=4, dy=p, dg=p, ws=p, size=1 << 30):
        return L.moe_combine_topk_sum_backward(do, y, ro, gate, T, k, d, R, dy, dg, ws, size, None)
    assert f(T=-1) == -1 and f(k=0) == -1 and f(d=0) == -1 and f(R=-1) == -1 and f(d=12) == -2 and f(d=16392) == -2 and f(T=1 << 30, k=4) == -2
    for name in ("do", "y", "ro", "gate", "dy", "dg"):
        assert f(**{name: None}) == -1, name                              # a weight without its gradient, or the other way round
    for name in ("do", "y", "dy", "ws"):
        assert f(**{name: odd}) == -1, name
    assert f(ws=None) == -3 and f(size=15) == -3 and f(T=0, R=0, do=None, ro=None, y=None, dy=None, ws=None) == 0
    assert L.moe_combine_backward_workspace_bytes(-1) == 0 and L.moe_combine_backward_workspace_bytes(1000) >= 4000


def _case(T, k, d, R, seed, gated):
    rng = np.random.default_rng(seed)
    row_of = rng.permutation(max(R, T * k))[:T * k].reshape(T, k).astype(np.int32)           # some are past the last row
    row_of[rng.random((T, k)) < 0.05] = -1
    f = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).bfloat16()      # noqa: E731
    return f(T, d), f(R, d), row_of, rng.random((T, k)).astype(np.float32) if gated else None


def _check(lib, d_out, y, row_of, gate):
    dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)                      # noqa: E731
    got = lib.moe_combine_topk_sum_backward(d_out.to(DEV), y.to(DEV), dev(row_of), dev(gate))
    do, yy, g = d_out.double().numpy(), y.double().numpy(), None if gate is None else gate.astype(np.float64)
    d_y, d_gate = oracle.combine_topk_sum_backward(do, yy, row_of, g)
    # a row's terms are added in fp32 one after the other and rounded to bf16 once
    uses = np.zeros(y.shape[0])
    size = np.zeros_like(yy)
    for t, j in np.ndindex(row_of.shape):
        if 0 <= row_of[t, j] < y.shape[0]:
            uses[row_of[t, j]] += 1
            size[row_of[t, j]] += np.abs(do[t]) * (1.0 if g is None else g[t, j])
    err = np.abs(got["d_y"].double().cpu().numpy() - d_y)
    assert (err <= 2.0 ** -8 * np.abs(d_y) + 2.0 ** -24 * (uses[:, None] + 1) * size).all(), err.max()
    assert (got["d_gate"] is None) == (gate is None)
    if gate is not None:
        ok = (row_of >= 0) & (row_of < y.shape[0])
        # a chain of at most 16 values per thread and 11 levels over the threads, products included fewer than 64 roundings
        bound = 64 * 2.0 ** -24 * np.where(ok, (np.abs(do)[:, None, :] * np.abs(yy)[np.where(ok, row_of, 0)]).sum(2), 0.0)
        err = np.abs(got["d_gate"].double().cpu().numpy() - d_gate)
        assert (err <= bound).all(), err.max()
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("T,k,d,R", [(1, 1, 8, 1), (37, 2, 256, 80), (50, 3, 2056, 160), (19, 8, 4096, 140), (33, 5, 520, 165), (7, 4, 7168, 28), (3, 6, 16384, 20), (9, 1, 1024, 3), (21, 9, 72, 500), (5, 2, 8200, 10), (1, 8, 2048, 8)])
def test_gradients(lib, T, k, d, R, gated):
    _check(lib, *_case(T, k, d, R, T + d, gated))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 2304])
def test_rows_named_more_than_once(lib, d):
    """The same row by several slots, of one token and of many, adds up in the order of the assignments: the same bits on every run."""
    d_out, y, row_of, gate = _case(300, 3, d, 1000, 11, True)
    row_of[:, 1] = row_of[:, 0]
    row_of[17:290, 2] = 5
    a = _check(lib, d_out, y, row_of, gate)
    b = _check(lib, d_out, y, row_of, gate)
    assert torch.equal(a["d_y"], b["d_y"]) and torch.equal(a["d_gate"], b["d_gate"])


@pytest.mark.gpu
def test_edges_and_refused_tensors(lib):
    bf = dict(dtype=torch.bfloat16, device=DEV)
    got = lib.moe_combine_topk_sum_backward(torch.empty(0, 64, **bf), torch.ones(5, 64, **bf), torch.empty(0, 2, dtype=torch.int32, device=DEV), torch.empty(0, 2, device=DEV))
    assert not got["d_y"].any() and got["d_gate"].shape == (0, 2)          # no tokens: no row has a gradient
    got = lib.moe_combine_topk_sum_backward(torch.ones(3, 64, **bf), torch.empty(0, 64, **bf), torch.zeros(3, 2, dtype=torch.int32, device=DEV), torch.ones(3, 2, device=DEV))
    assert not got["d_gate"].any()                                        # no rows: every assignment is out of range
    x, y, r, g = torch.ones(3, 64, **bf), torch.ones(6, 64, **bf), torch.zeros(3, 2, dtype=torch.int32, device=DEV), torch.ones(3, 2, device=DEV)
    y[2] = float("nan")                                                   # of a row that nothing names
    r[0, 1] = -1
    got = lib.moe_combine_topk_sum_backward(x, y, r, g)
    assert torch.isfinite(got["d_gate"]).all() and torch.isfinite(got["d_y"]).all()
    for bad in (lambda: lib.moe_combine_topk_sum_backward(x[:, :32], y, r, g), lambda: lib.moe_combine_topk_sum_backward(x.float(), y, r, g),
                lambda: lib.moe_combine_topk_sum_backward(x, y, r.long(), g), lambda: lib.moe_combine_topk_sum_backward(x, y, r, g[:, :1]),
                lambda: lib.moe_combine_topk_sum_backward(x[:2], y, r, g)):
        with pytest.raises(lib.MoeError):
            bad()


@pytest.mark.gpu
@pytest.mark.parametrize("T,R", [(2000, 7000), (1366, 4096), (1365, 4097), (1365, 4096), (40, 9000)])
def test_many_rows_with_odd_ones(lib, T, R):
    """Both ways of counting the rows' uses, at their boundary too: rows that nothing names, rows named twice and rows named by many."""
    d_out, y, row_of, gate = _case(T, 3, 72, R, T + R, True)
    row_of[::7, 1] = row_of[::7, 0]
    row_of[5::11, 2] = R - 1
    row_of[3::13, 0] = -1
    _check(lib, d_out, y, row_of, gate)
    _check(lib, d_out, y, row_of, None)
