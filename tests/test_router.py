"""moe_router_topk and its backward pass: the oracle against differences, refusals on the host, and the kernels against the oracle."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import router

DEV = "cuda:0"
INF = float("inf")
MODES = [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)]
# exp of a difference x that is itself rounded: |x| 2^-24 and 2 steps; beyond |x| = 90 the value is below 2^-126 of the largest.  A sum over the experts is
# a chain of at most 64 values per lane and 6 levels, and a few products and quotients follow: fewer than 256 roundings.
REL, TINY = 256 * 2.0 ** -24, 2.0 ** -120


def test_oracle_gradient_matches_differences():
    rng = np.random.default_rng(2)
    for score, ren in MODES:
        l = rng.normal(size=(3, 7))
        l[1, 2] = l[0, 5] = -INF
        ids, _ = router.topk(l, 3, score, ren, 1.5)
        dg = rng.normal(size=(3, 3))
        ids[2, 1] = -1
        got = router.topk_backward(dg, l, ids, score, ren, 1.5)
        value = lambda l: sum((dg[t] * router.weights(l[t], ids[t], score, ren, 1.5)).sum() for t in range(3))      # noqa: E731
        for i in np.ndindex(l.shape):
            if np.isfinite(l[i]):
                a, b = l.copy(), l.copy()
                a[i] += 1e-5
                b[i] -= 1e-5
                assert abs((value(a) - value(b)) / 2e-5 - got[i]) < 1e-8, (score, ren, i)
            else:
                assert got[i] == 0


def test_oracle_choice_and_masks():
    ids, g = router.topk(np.array([[1.0, 3, 3, -INF], [-INF, -INF, -INF, -INF], [np.nan, 0, -INF, 0], [INF, 0, INF, 1]]), 3, "softmax", False)
    assert ids.tolist() == [[1, 2, 0], [-1, -1, -1], [1, 3, -1], [0, 2, 3]]
    assert np.allclose(g[3], [0.5, 0.5, 0]) and np.allclose(g[2], [0.5, 0.5, 0]) and not g[1].any()


def test_refusals_need_no_gpu(hostlib):
    L = hostlib.load()
    p, odd = ctypes.c_void_p(4096), ctypes.c_void_p(4097)

    def fwd(l=p, t=1, T=1, E=8, k=2, score=0, flags=0, scale=1.0, ids=p, gates=p):
        return L.moe_router_topk(l, t, T, E, k, score, flags, scale, ids, gates, None)

    def bwd(dg=p, l=p, t=1, ids=p, T=1, E=8, k=2, score=0, flags=0, scale=1.0, dl=p):
        return L.moe_router_topk_backward(dg, l, t, ids, T, E, k, score, flags, scale, dl, None)
    for f in (fwd, bwd):
        assert f(t=2) == -1 and f(T=-1) == -1 and f(E=0) == -1 and f(k=0) == -1 and f(k=9) == -1 and f(score=2) == -1 and f(flags=2) == -1
        assert f(scale=INF) == -1 and f(scale=float("nan")) == -1 and f(E=4097) == -2 and f(E=64, k=33) == -2 and f(l=None) == -1 and f(l=odd) == -1
        assert f(ids=None) == -1 and f(ids=odd) == -1 and f(T=0, l=None, ids=None) == 0
    assert fwd(gates=None) == -1 and fwd(gates=odd) == -1 and bwd(dg=None) == -1 and bwd(dl=None) == -1 and bwd(dl=odd) == -1 and bwd(dg=odd) == -1


def _logits(T, E, kind, seed, masked=True):
    rng = np.random.default_rng(seed)
    l = torch.from_numpy((2.0 * rng.normal(size=(T, E))).astype(np.float32))
    if masked:
        l[torch.from_numpy(rng.random((T, E)) < 0.15)] = -INF
        if T > 3:
            l[1], l[2] = -INF, 0.5                                        # nothing left; all equal
            l[3, : max(1, E // 2)] = float("nan")
    return l if kind == "f32" else l.bfloat16()


SHAPES = [(1, 1, 1), (5, 2, 2), (9, 3, 1), (33, 8, 2), (7, 16, 16), (17, 17, 5), (40, 60, 4), (70, 64, 6), (19, 100, 8), (11, 128, 32), (23, 160, 6), (300, 256, 8), (6, 257, 3),
          (5, 512, 32), (4, 515, 7), (5, 1024, 8), (3, 1025, 4), (4, 4096, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k", SHAPES)
@pytest.mark.parametrize("score,ren", MODES)
def test_topk(lib, T, E, k, kind, score, ren):
    l = _logits(T, E, kind, T + E)
    ids, gates = lib.moe_router_topk(l.to(DEV), k, score, ren, 1.25)
    ref_ids, ref = router.topk(l.double().numpy(), k, score, ren, 1.25)
    assert np.array_equal(ids.cpu().numpy(), ref_ids)
    assert (np.abs(gates.double().cpu().numpy() - ref) <= REL * np.abs(ref) + TINY).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k", [s for s in SHAPES if s[1] <= 1025])
@pytest.mark.parametrize("score,ren", MODES)
def test_topk_backward(lib, T, E, k, kind, score, ren):
    rng = np.random.default_rng(T * E)
    l = _logits(T, E, kind, T + E)
    ids = router.topk(l.double().numpy(), k, score, ren)[0]
    if T > 4 and k > 1:
        ids[4, 0], ids[0, 1] = -1, E                                      # dropped and out of range
        ids[2, 1] = ids[2, 0]                                             # the same expert twice
    dg = rng.normal(size=(T, k)).astype(np.float32)
    got = lib.moe_router_topk_backward(torch.from_numpy(dg).to(DEV), l.to(DEV), torch.from_numpy(ids).to(DEV), score, ren, 1.25).double().cpu().numpy()
    ref = router.topk_backward(dg.astype(np.float64), l.double().numpy(), ids, score, ren, 1.25)
    # every term of the sums is a product of scores with a gradient: |w| (|G| + sum |G w|), summed in fp32
    size = np.zeros((T, E))
    for t in range(T):
        w = np.abs(router.weights(l[t].double().numpy(), ids[t], score, ren, 1.0))
        G = 1.25 * np.abs(dg[t])
        for j in range(k):
            if 0 <= ids[t, j] < E:
                size[t, ids[t, j]] += w[j] * (G[j] + (G * w).sum())
        if score == "softmax" and not ren:
            size[t] += router._scores(l[t].double().numpy(), score) * (G * w).sum()
    # the oracle adds, in 64 bits, at most 2 k + 2 terms per expert that are each no larger than the token's gradients together (a score's derivative, and a score,
    # over the sum of the scores are at most 1); where they cancel, that leaves up to this much of nothing
    size64 = (2 * k + 2) * 4 * 2.0 ** -53 * 1.25 * np.abs(dg).sum(1, keepdims=True)
    bound = (REL + (2.0 ** -8 if kind == "bf16" else 0.0)) * np.abs(ref) + REL * size + size64 + TINY
    assert (np.abs(got - ref) <= bound).all(), np.abs(got - ref).max()


@pytest.mark.gpu
@pytest.mark.parametrize("score,ren", MODES)
def test_extreme_logits(lib, score, ren):
    l = torch.tensor([[INF, 1.0, INF, -3.0], [-200.0, -190.0, -201.0, -INF], [3e38, -3e38, 3e38, 0.0], [-3e38, -3e38, -3.1e38, -INF], [0.0, -0.0, 0.0, -0.0], [1e-45, 0.0, -1e-45, 1e-40]])
    ids, gates = lib.moe_router_topk(l.to(DEV), 3, score, ren)
    ref_ids, ref = router.topk(l.double().numpy(), 3, score, ren)
    if score == "sigmoid" and ren:
        ref[3] = [0.5, 0.5, 0.0]                                          # both scores are zero in 64 bits, their ratio is one
    assert np.array_equal(ids.cpu().numpy(), ref_ids)
    assert (np.abs(gates.double().cpu().numpy() - ref) <= REL * np.abs(ref) + TINY).all()
    d = lib.moe_router_topk_backward(torch.ones(6, 3, device=DEV), l.to(DEV), ids, score, ren)
    assert torch.isfinite(d).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("E", [64, 256])
def test_rows_that_start_anywhere(lib, kind, E):
    """Logits that do not start on 16 bytes give the same bits."""
    l = _logits(50, E, kind, 3)
    buf = torch.zeros(50 * E + 1, dtype=l.dtype, device=DEV)
    buf[1:] = l.flatten()
    a, b = lib.moe_router_topk(l.to(DEV), 4), lib.moe_router_topk(buf[1:].view(50, E), 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    dg = torch.randn(50, 4, device=DEV)
    for score, ren in MODES:
        assert torch.equal(lib.moe_router_topk_backward(dg, l.to(DEV), a[0], score, ren), lib.moe_router_topk_backward(dg, buf[1:].view(50, E), a[0], score, ren))


@pytest.mark.gpu
def test_many_tokens_and_refused_tensors(lib):
    T, E, k = 70001, 64, 2
    l = _logits(T, E, "bf16", 9)
    ids, gates = lib.moe_router_topk(l.to(DEV), k)
    v, i = torch.sort(torch.nan_to_num(l.float(), nan=-INF, posinf=INF, neginf=-INF), dim=1, descending=True, stable=True)
    assert torch.equal(ids.cpu(), torch.where(v[:, :k] == -INF, -1, i[:, :k]).int())
    traffic, counts = lib.moe_route_histogram(ids.view(1, T, k), E)       # a slot without expert is not counted
    assert int(traffic.sum()) == int((ids >= 0).sum())
    assert lib.moe_router_topk(torch.empty(0, E, device=DEV), k)[0].shape == (0, k)
    x = l[:8].to(DEV)
    for bad in (lambda: lib.moe_router_topk(x.t(), 2), lambda: lib.moe_router_topk(x.half(), 2), lambda: lib.moe_router_topk(x, 0), lambda: lib.moe_router_topk(x, 65),
                lambda: lib.moe_router_topk(x, 2, "max"), lambda: lib.moe_router_topk(x[:, ::2], 2), lambda: lib.moe_router_topk(x, 2, scale=INF),
                lambda: lib.moe_router_topk_backward(torch.ones(8, 3, device=DEV), x, ids[:8]), lambda: lib.moe_router_topk_backward(torch.ones(8, 2, device=DEV), x, ids[:8].long())):
        with pytest.raises(lib.MoeError):
            bad()


@pytest.mark.gpu
def test_refused_numbers_of_slots(lib):
    l = torch.zeros(3, 4, device=DEV)
    for k in (-1, 0, 5):
        with pytest.raises(lib.MoeError):
            lib.moe_router_topk(l, k)
    ids, gates = lib.moe_router_topk(l, 4)
    assert ids.tolist() == [[0, 1, 2, 3]] * 3 and gates.tolist() == [[0.25] * 4] * 3
