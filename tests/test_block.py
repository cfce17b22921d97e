"""moe_block_norm, moe_block_join and their backward passes: the float64 oracle against differences, refusals on the host, and the kernels against
the oracle on the same inputs."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from oracle import block

DEV = "cuda:0"
EPS = 1e-6
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
# One fp32 operation is off by 2^-24 of its result.  A sum over the columns of a row is a chain of at most 64 values per thread and a tree over the threads (10 levels),
# its root halves the relative error, and a handful of products follow: fewer than 128 operations in a row.
CHAIN = 128 * 2.0 ** -24


# ------------------------------------------------------------------------------------------------ oracle
def test_oracle_gradients_match_differences():
    rng = np.random.default_rng(1)
    T, d, scale = 3, 16, 0.75
    z, x, wp, wn, gate = rng.normal(size=(T, d)), rng.normal(size=(T, d)), rng.normal(size=d), rng.normal(size=d), rng.random(T)
    a, b = rng.normal(size=(T, d)), rng.normal(size=(T, d))

    def loss(z, x, wp, wn, gate):
        out, nxt = block.join(z, x, wp, gate, wn, scale, EPS)
        return (a * out).sum() + (b * nxt).sum()

    out, _ = block.join(z, x, wp, gate, wn, scale, EPS)
    g = block.join_backward(a, b, z, out, wp, gate, wn, scale, EPS)
    args = [z, x, wp, wn, gate]
    for k, name in enumerate(("d_z", "d_stream", "d_post_weight", "d_next_weight", "d_gate")):
        for i in np.ndindex(args[k].shape):
            h = 1e-5
            up, dn = [v.copy() for v in args], [v.copy() for v in args]
            up[k][i] += h
            dn[k][i] -= h
            assert abs((loss(*up) - loss(*dn)) / (2 * h) - g[name][i]) < 1e-6, (name, i)


def test_oracle_hand_example():
    # rms([3, 4, 0, 0]) = 2.5
    assert np.allclose(block.norm(np.array([[3.0, 4, 0, 0]]), np.array([1.0, 2, 1, 1]), 0.0), [[1.2, 3.2, 0, 0]])
    out, nxt = block.join(np.array([[3.0, 4, 0, 0]]), np.array([[1.0, 0, 2, 0]]), np.ones(4), np.array([2.0]), np.ones(4), 0.5, 0.0)
    assert np.allclose(out, [[2.9, 3.2, 1, 0]]) and np.allclose(nxt, out / np.sqrt((out ** 2).mean()))


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals_need_no_gpu(hostlib):
    L = hostlib.load()
    p, odd, inf = ctypes.c_void_p(4096), ctypes.c_void_p(4104), float("inf")
    norm = lambda x=p, t=0, w=p, eps=1e-6, T=1, d=64, out=p: L.moe_block_norm(x, t, w, eps, T, d, out, None)                       # noqa: E731
    assert norm(t=2) == -1 and norm(eps=0.0) == -1 and norm(eps=-1.0) == -1 and norm(eps=inf) == -1 and norm(eps=float("nan")) == -1
    assert norm(T=-1) == -1 and norm(d=0) == -1 and norm(d=12) == -2 and norm(d=16392) == -2
    assert norm(x=None) == -1 and norm(w=None) == -1 and norm(out=None) == -1 and norm(x=odd) == -1 and norm(w=odd) == -1 and norm(out=odd) == -1
    assert norm(x=None, w=None, out=None, T=0) == 0

    def join(z=p, x=p, wp=p, gate=p, wn=p, scale=1.0, T=1, d=64, out=p, nxt=p):
        return L.moe_block_join(z, x, 0, wp, gate, wn, scale, 1e-6, T, d, out, nxt, None)
    assert join(wn=None) == -1 and join(nxt=None) == -1                  # next and its weight come together
    assert join(z=None) == -1 and join(x=None) == -1 and join(out=None) == -1 and join(scale=inf) == -1 and join(scale=float("nan")) == -1
    for name in ("z", "x", "wp", "wn", "out", "nxt"):
        assert join(**{name: odd}) == -1, name
    assert join(T=0, z=None) == 0

    assert L.moe_block_backward_workspace_bytes(-1, 8) == 0 and L.moe_block_backward_workspace_bytes(5, 0) == 0
    sizes = [L.moe_block_backward_workspace_bytes(T, 4096) for T in (0, 1, 7, 1000, 1024, 5000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    big = 1 << 40

    def nb(d_out=p, x=p, w=p, ds=p, T=1, d=64, dx=p, dw=p, ws=p, size=big):
        return L.moe_block_norm_backward(d_out, x, 0, w, ds, 1e-6, T, d, dx, dw, ws, size, None)
    for name in ("d_out", "x", "w", "dx", "dw"):
        assert nb(**{name: None}) == -1 and nb(**{name: odd}) == -1, name
    assert nb(ds=odd) == -1 and nb(ws=None) == -3 and nb(size=64 * 8 - 1) == -3 and nb(d=12) == -2

    def jb(d_out=p, d_next=p, z=p, out=p, wp=p, gate=p, wn=p, T=1, d=64, dz=p, ds=p, dg=p, dwp=p, dwn=p, ws=p, size=big):
        return L.moe_block_join_backward(d_out, d_next, z, out, 0, wp, gate, wn, 1.0, 1e-6, T, d, dz, ds, dg, dwp, dwn, ws, size, None)
    for name in ("d_next", "z", "out", "wp", "gate", "wn", "dz", "ds", "dg", "dwp", "dwn"):
        assert jb(**{name: None}) == -1, name                             # an output without its input, or the other way round
    assert jb(d_out=None, d_next=None, wn=None, dwn=None) == -1          # no gradient at all
    assert jb(ws=None) == -3 and jb(size=64 * 8 - 1) == -3
    for name in ("d_out", "d_next", "z", "out", "wp", "wn", "dz", "ds", "dwp", "dwn", "ws"):
        assert jb(**{name: odd}) == -1, name


# ------------------------------------------------------------------------------------------------ kernels
def _case(T, d, stream, seed, post=True, gate=True, nxt=True):
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if stream == "f32" else torch.bfloat16
    r = lambda *s: torch.randn(s, generator=g)                                          # noqa: E731
    c = dict(z=r(T, d).bfloat16(), x=(2 * r(T, d)).to(dt), post_weight=1 + 0.3 * r(d) if post else None, gate=torch.rand(T, generator=g) if gate else None,
             next_weight=1 + 0.3 * r(d) if nxt else None, d_out=r(T, d).to(dt), d_next=r(T, d).bfloat16() if nxt else None)
    if T > 2:
        c["z"][1] = 0                                                     # a row without length
        c["x"][1] = 0
    return c


def _n(t):
    return None if t is None else t.double().numpy()


def _dev(t):
    return None if t is None else t.to(DEV)


def _within(got, ref, tol, what):
    got = got.double().cpu().numpy()
    over = np.abs(got - ref) - tol
    assert np.isfinite(got).all() and over.max(initial=-1.0) <= 0, (what, float(np.abs(got - ref).max()), np.unravel_index(over.argmax(), over.shape))


SHAPES = [(1, 8), (3, 64), (5, 520), (4, 1000), (7, 1024), (2, 1032), (9, 2048), (3, 2056), (6, 2880), (5, 4096), (3, 4104), (2, 7168), (3, 8200), (2, 16384), (1, 16376), (700, 256), (2600, 72)]


@pytest.mark.gpu
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_norm(lib, T, d, stream):
    c = _case(T, d, stream, T + d)
    got = lib.moe_block_norm(_dev(c["x"]), _dev(c["next_weight"]), EPS)
    ref = block.norm(_n(c["x"]), _n(c["next_weight"]), EPS)
    _within(got, ref, (ROUND["bf16"] + CHAIN) * np.abs(ref), (T, d))


@pytest.mark.gpu
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("post,gate,nxt", [(True, True, True), (False, False, True), (True, False, False), (False, True, True)])
def test_join(lib, T, d, stream, post, gate, nxt):
    c = _case(T, d, stream, 2 * T + d, post, gate, nxt)
    out, got = lib.moe_block_join(_dev(c["z"]), _dev(c["x"]), _dev(c["post_weight"]), _dev(c["gate"]), _dev(c["next_weight"]), 0.75, EPS)
    z, x, wp, wn, gt = (_n(c[k]) for k in ("z", "x", "post_weight", "next_weight", "gate"))
    ref, ref_next = block.join(z, x, wp, gt, wn, 0.75, EPS)
    u, _ = block.join(z, 0 * x, wp, gt, None, 0.75, EPS)
    size = np.abs(0.75 * x) + np.abs(u)                                   # what the fp32 sum of the two is off by is relative to this
    _within(out, ref, ROUND[stream] * np.abs(ref) + CHAIN * size, (T, d))
    assert (got is None) == (not nxt)
    if nxt:
        rms = np.sqrt((ref ** 2).mean(1, keepdims=True) + EPS)
        rel = CHAIN * np.sqrt((size ** 2).mean(1, keepdims=True)) / rms     # of the length of out
        _within(got, ref_next, (ROUND["bf16"] + CHAIN + rel) * np.abs(ref_next) + CHAIN * size / rms * np.abs(wn), (T, d))


@pytest.mark.gpu
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_norm_backward(lib, T, d, stream):
    c = _case(T, d, stream, 3 * T + d)
    for along in (True, False):
        got = lib.moe_block_norm_backward(_dev(c["d_next"]), _dev(c["x"]), _dev(c["next_weight"]), EPS, d_stream=_dev(c["d_out"]) if along else None)
        x, w, dn, ds = _n(c["x"]), _n(c["next_weight"]), _n(c["d_next"]), _n(c["d_out"]) if along else np.zeros((T, d))
        dx, dw = block.norm_gradient(dn, x, w, EPS)
        r = np.sqrt((x * x).mean(1, keepdims=True) + EPS)
        n = np.abs(x / r)
        size = (np.abs(dn * w) + n * (np.abs(dn * w) * n).mean(1, keepdims=True)) / r + np.abs(ds)
        _within(got["d_x"], dx + ds, ROUND[stream] * np.abs(dx + ds) + CHAIN * size, "d_x")
        # a thread adds up at most T rows, 1024 parts are added in 16 strides of 64 and these 16
        _within(got["d_weight"], dw, (CHAIN + T * 2.0 ** -24) * (np.abs(dn) * n).sum(0), "d_weight")


@pytest.mark.gpu
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("post,gate,nxt,along", [(True, True, True, True), (False, True, True, False), (True, False, False, True), (False, False, True, True)])
def test_join_backward(lib, T, d, stream, post, gate, nxt, along):
    c = _case(T, d, stream, 4 * T + d, post, gate, nxt)
    scale = 0.75
    z, x, wp, wn, gt = (_n(c[k]) for k in ("z", "x", "post_weight", "next_weight", "gate"))
    go, dn = _n(c["d_out"]) if along else None, _n(c["d_next"])
    got = lib.moe_block_join_backward(_dev(c["d_out"]) if along else None, _dev(c["d_next"]), _dev(c["z"]), _dev(c["x"]), _dev(c["post_weight"]), _dev(c["gate"]),
                                      _dev(c["next_weight"]), scale, EPS)
    ref = block.join_backward(go, dn, z, x, wp, gt, wn, scale, EPS)       # x stands for out: any row will do
    size = np.zeros((T, d)) if go is None else np.abs(go)
    if nxt:
        r2 = np.sqrt((x * x).mean(1, keepdims=True) + EPS)
        n2 = np.abs(x / r2)
        size = size + (np.abs(dn * wn) + n2 * (np.abs(dn * wn) * n2).mean(1, keepdims=True)) / r2
        _within(got["d_next_weight"], ref["d_next_weight"], (CHAIN + T * 2.0 ** -24) * (np.abs(dn) * n2).sum(0), "d_next_weight")
    e_total = CHAIN * size                                                # of the gradient of out, before any rounding
    _within(got["d_stream"], ref["d_stream"], ROUND[stream] * np.abs(ref["d_stream"]) + scale * e_total, "d_stream")
    total = ref["d_stream"] / scale
    g1 = np.ones((T, 1)) if gt is None else gt[:, None]
    r1 = np.sqrt((z * z).mean(1, keepdims=True) + EPS) if post else np.ones((T, 1))
    n1, w1 = np.abs(z / r1), np.abs(wp) if post else np.ones(d)
    if gate:
        _within(got["d_gate"], ref["d_gate"], (n1 * w1 * (e_total + CHAIN * np.abs(total))).sum(1), "d_gate")
    if post:
        _within(got["d_post_weight"], ref["d_post_weight"], (g1 * n1 * (e_total + (CHAIN + T * 2.0 ** -24) * np.abs(total))).sum(0), "d_post_weight")
    s, e_s = np.abs(total) * w1, (e_total + CHAIN * np.abs(total)) * w1
    back = n1 * (e_s * n1 + CHAIN * s * n1).mean(1, keepdims=True) if post else 0.0
    _within(got["d_z"], ref["d_z"], ROUND["bf16"] * np.abs(ref["d_z"]) + g1 / r1 * (e_s + back + CHAIN * (s + (n1 * (s * n1).mean(1, keepdims=True) if post else 0.0))), "d_z")
    assert [got[k] is None for k in ("d_gate", "d_post_weight", "d_next_weight")] == [not gate, not post, not nxt]


@pytest.mark.gpu
def test_no_tokens(lib):
    e = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device=DEV)              # noqa: E731
    w = torch.ones(64, device=DEV)
    assert lib.moe_block_norm(e(0, 64), w).shape == (0, 64)
    assert lib.moe_block_join(e(0, 64), e(0, 64), w, None, w)[1].shape == (0, 64)
    got = lib.moe_block_norm_backward(e(0, 64), e(0, 64), w)
    assert torch.equal(got["d_weight"], torch.zeros(64, device=DEV))
    got = lib.moe_block_join_backward(e(0, 64), e(0, 64), e(0, 64), e(0, 64), w, e(0, dt=torch.float32), w)
    assert torch.equal(got["d_post_weight"], torch.zeros(64, device=DEV)) and torch.equal(got["d_next_weight"], torch.zeros(64, device=DEV))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [256, 4096])
def test_in_place_and_the_same_bits(lib, d):
    """out over the stream, next over z, gradients over the ones that came in: the same bits as into other tensors, on every run, and alone as in a batch."""
    c = {k: _dev(v) for k, v in _case(37, d, "bf16", 5).items()}
    out, nxt = lib.moe_block_join(c["z"], c["x"], c["post_weight"], c["gate"], c["next_weight"], 0.75, EPS)
    x, z = c["x"].clone(), c["z"].clone()
    lib.moe_block_join(z, x, c["post_weight"], c["gate"], c["next_weight"], 0.75, EPS, out=x, next_out=z)
    assert torch.equal(x, out) and torch.equal(z, nxt)
    one = lib.moe_block_join(c["z"][5:6], c["x"][5:6], c["post_weight"], c["gate"][5:6], c["next_weight"], 0.75, EPS)
    assert torch.equal(one[0], out[5:6]) and torch.equal(one[1], nxt[5:6])
    args = (c["d_out"], c["d_next"], c["z"], out, c["post_weight"], c["gate"], c["next_weight"], 0.75, EPS)
    a, b = lib.moe_block_join_backward(*args), lib.moe_block_join_backward(*args)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    L, ds, dz = lib.load(), c["d_out"].clone(), c["d_next"].clone()
    ws = torch.empty(L.moe_block_backward_workspace_bytes(37, d), dtype=torch.uint8, device=DEV)
    P = lambda t: t.data_ptr()                                            # noqa: E731
    dg, dwp, dwn = (torch.empty_like(a[k]) for k in ("d_gate", "d_post_weight", "d_next_weight"))
    assert L.moe_block_join_backward(P(ds), P(dz), P(c["z"]), P(out), 0, P(c["post_weight"]), P(c["gate"]), P(c["next_weight"]), 0.75, EPS, 37, d, P(dz), P(ds), P(dg),
                                     P(dwp), P(dwn), P(ws), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(ds, a["d_stream"]) and torch.equal(dz, a["d_z"]) and torch.equal(dg, a["d_gate"]) and torch.equal(dwn, a["d_next_weight"])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [72, 2880, 7168])
def test_rows_keep_to_themselves(lib, d):
    """NaN and infinity in one row reach no other row, rows behind T stay as they were, and columns far apart in size do no harm."""
    c = {k: _dev(v) for k, v in _case(6, d, "f32", 7).items()}
    ref = lib.moe_block_join(c["z"], c["x"], c["post_weight"], c["gate"], c["next_weight"], 1.0, EPS)
    x = c["x"].clone()
    x[2, 3], x[4, 0] = float("nan"), float("inf")
    out = torch.full((8, d), 7.0, device=DEV)
    nxt = torch.full((8, d), 7.0, device=DEV, dtype=torch.bfloat16)
    lib.moe_block_join(c["z"], x, c["post_weight"], c["gate"], c["next_weight"], 1.0, EPS, out=out[:6], next_out=nxt[:6])
    for t in (0, 1, 3, 5):
        assert torch.equal(out[t], ref[0][t]) and torch.equal(nxt[t], ref[1][t])
    assert torch.isnan(nxt[2]).all() and (out[6:] == 7).all() and (nxt[6:] == 7).all()


@pytest.mark.gpu
def test_refused_tensors(lib):
    x, w = torch.ones(4, 64, device=DEV, dtype=torch.bfloat16), torch.ones(64, device=DEV)
    for bad in (lambda: lib.moe_block_norm(x.t(), w), lambda: lib.moe_block_norm(x, w.bfloat16()), lambda: lib.moe_block_norm(x, w[:32]), lambda: lib.moe_block_norm(x.half(), w),
                lambda: lib.moe_block_norm(x[:, ::2], w[:32]), lambda: lib.moe_block_norm(x.cpu(), w), lambda: lib.moe_block_norm(x, None),
                lambda: lib.moe_block_join(x, x[:3], w), lambda: lib.moe_block_join(x, x, w, gate=torch.ones(3, device=DEV)), lambda: lib.moe_block_norm(x, w, eps=0.0),
                lambda: lib.moe_block_join_backward(x, None, x, x, w, None, w), lambda: lib.moe_block_join_backward(None, None, x, x, w)):
        with pytest.raises(lib.MoeError):
            bad()
