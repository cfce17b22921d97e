"""The operators around the experts in a row, as a MoE layer uses them: serving with 4-bit experts over the slices of a schedule, eager, captured and on
another stream, and a training step whose gradients go back through all of them."""
import numpy as np
import pytest
import torch

import oracle
from oracle import block, ffn_w4, router
from test_ffn_w4 import check as check_ffn_w4
from test_ffn_w4 import weights as w4_weights

DEV = "cuda:0"
EPS = 1e-6
HALF = 2.0 ** -8                                  # a rounding to bf16, relative


def near(got, want, tol):
    got = got.detach().double().cpu().numpy()
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())


def f64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ serving
class Layer:
    """N ranks of T tokens each; every rank's part of the layer runs here, one after the other."""

    def __init__(self, N, T, E, k, d, f, group, seed):
        self.N, self.T, self.E, self.k, self.d, self.e_loc, self.kmax = N, T, E, k, d, E // N, 2 * N
        g = torch.Generator().manual_seed(seed)
        self.router = (torch.randn(E, d, generator=g) / d ** 0.5).to(DEV)
        self.pre, self.post, self.next = ((1 + 0.2 * torch.randn(d, generator=g)).to(DEV) for _ in range(3))
        self.host = [w4_weights(self.e_loc, d, f, group, True, seed + r) for r in range(N)]
        self.experts = [{n: v.to(DEV) for n, v in w.items()} for w in self.host]

    def run(self, lib, stream, sizes=None):
        """stream float32 [N * T][d] -> everything made on the way; sizes: rows of the ranks (read from the traffic if None; a constant bound for a capture)"""
        o = {}
        o["h"] = lib.moe_block_norm(stream, self.pre, EPS)
        o["logits"] = o["h"].float() @ self.router.t()
        o["ids"], o["gates"] = lib.moe_router_topk(o["logits"], self.k, "sigmoid", True, 2.5)
        ids = o["ids"].view(self.N, self.T, self.k)
        o["traffic"], _ = lib.moe_route_histogram(ids, self.E)
        o["sched"] = lib.moe_decompose_greedy(o["traffic"].unsqueeze(0), self.kmax, zero_diag=True)
        n = self.N * self.T * self.k
        row_of = torch.full((n + 1,), -1, dtype=torch.int32, device=DEV)
        o["parts"], first = [], 0
        if sizes is None:
            sizes = o["traffic"].sum(0).tolist()
        Y = torch.zeros((sum(sizes), self.d), dtype=torch.bfloat16, device=DEV)
        for r, M in enumerate(sizes):
            off, _, asg = lib.moe_slice_table_rows(ids, self.E, r, o["traffic"], o["sched"]["perms"][0], o["sched"]["durations"][0], o["sched"]["counts"], self.kmax, M)
            x = o["h"][(asg.clamp(min=0) // self.k).long()]
            lib.moe_expert_ffn_w4_sliced(x, off, self.kmax + 2, self.e_loc, y=Y[first:first + M], **self.experts[r])
            row_of.scatter_(0, torch.where(asg < 0, n, asg).long(), torch.arange(first, first + M, dtype=torch.int32, device=DEV))
            o["parts"].append((off, asg, x, Y[first:first + M]))
            first += M
        o["Y"], o["row_of"] = Y, row_of[:n].view(self.N * self.T, self.k)
        o["z"] = lib.moe_combine_topk_sum(Y, o["row_of"], o["gates"])
        o["out"], o["next"] = lib.moe_block_join(o["z"], stream, self.post, None, self.next, 1.0, EPS)
        return o


def small_stream(N, T, d, seed):
    x = torch.randn(N * T, d, generator=torch.Generator().manual_seed(seed)) * 2
    x[1] = 0.0                                                            # a token without length: all of its logits are equal
    return x.to(DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("N,T,E,k,d,f,group", [(2, 1, 4, 2, 256, 128, 32), (1, 7, 4, 4, 512, 256, 64), (2, 37, 8, 2, 512, 256, 128), (4, 300, 32, 4, 256, 256, 32)])
def test_serving(lib, N, T, E, k, d, f, group):
    L = Layer(N, T, E, k, d, f, group, N + T)
    stream = small_stream(N, T, d, T)
    o = L.run(lib, stream)
    torch.cuda.synchronize()
    s = f64(stream)
    near(o["h"], block.norm(s, f64(L.pre), EPS), HALF * np.abs(block.norm(s, f64(L.pre), EPS)) * 1.001 + 1e-30)
    ids, gates = router.topk(f64(o["logits"]), k, "sigmoid", True, 2.5)
    assert np.array_equal(o["ids"].cpu().numpy(), ids)
    near(o["gates"], gates, 2.0 ** -18 * gates)
    # the schedule covers every assignment once, and its row holds the token's hidden values
    row_of = o["row_of"].cpu().numpy()
    assert sorted(row_of.ravel()) == list(range(N * T * k))
    X = torch.cat([p[2] for p in o["parts"]])
    assert torch.equal(X[o["row_of"].long()], o["h"][:, None].expand(-1, k, -1))
    for r, (off, asg, x, y) in enumerate(o["parts"]):
        off = off.cpu().numpy()
        assert off[-1] == len(x)
        experts = np.concatenate([np.full(off[i + 1] - off[i], i % L.e_loc) for i in range(len(off) - 1)])
        assert (experts + r * L.e_loc == ids.ravel()[asg.cpu().numpy()]).all()
        if len(x):
            check_ffn_w4(y, x.cpu(), off, L.e_loc, L.host[r])
    y = f64(o["Y"])
    z = (f64(o["gates"])[:, :, None] * y[row_of]).sum(1)
    near(o["z"], z, HALF * np.abs(z) + 2.0 ** -20 * (f64(o["gates"])[:, :, None] * np.abs(y[row_of])).sum(1))
    out, nxt = block.join(f64(o["z"]), s, f64(L.post), None, f64(L.next), 1.0, EPS)
    u = block.norm(f64(o["z"]), f64(L.post), EPS)
    near(o["out"], out, 2.0 ** -20 * (np.abs(s) + np.abs(u)))
    # (next comes from out before its rounding; the root of its mean square is off by far less than a step of bf16)
    near(o["next"], nxt, (HALF + 2.0 ** -18) * np.abs(nxt) + 2.0 ** -18 * (np.abs(s) + np.abs(u)) / block._rms(out, EPS) * np.abs(f64(L.next)))


@pytest.mark.gpu
def test_serving_captured_twice_and_on_another_stream(lib):
    """Two captured layers, replayed in turn with eager work between them, give what the eager calls give, bit by bit; so does another stream."""
    N, T, E, k, d, f, group = 2, 24, 8, 2, 256, 256, 64
    layers = [Layer(N, T, E, k, d, f, group, s) for s in (1, 2)]
    sizes = [N * T * k] * N                                               # the most rows a rank can be sent
    inputs = [small_stream(N, T, d, s) for s in (3, 4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for L, x in zip(layers, inputs):
            L.run(lib, x, sizes)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs, captured = [], []
    for L, x in zip(layers, inputs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            captured.append(L.run(lib, x, sizes))
        graphs.append(g)
    for step in range(5):
        for i in (0, 1, 0):
            inputs[i].copy_(small_stream(N, T, d, 10 * step + i))
            if step % 2:
                with torch.cuda.stream(side):
                    side.wait_stream(torch.cuda.default_stream())
                    want = layers[i].run(lib, inputs[i])
                torch.cuda.current_stream().wait_stream(side)
            else:
                want = layers[i].run(lib, inputs[i])
            torch.cuda.synchronize()
            graphs[i].replay()
            graphs[1 - i].replay()                                        # (on its older input; it shares nothing with the other)
            torch.cuda.synchronize()
            for name in ("h", "ids", "gates", "traffic", "z", "out", "next"):
                assert torch.equal(captured[i][name], want[name]), (step, i, name)


# ------------------------------------------------------------------------------------------------ training
def plain_step(p, ids, c1, c2, scale):
    """Loss sum(c1 * out) + sum(c2 * next) of one layer and its gradients, float64, from the oracle's formulas; ids are given (the choice has no gradient)."""
    T, E = p["x"].shape[0], p["wr"].shape[0]
    h = block.norm(p["x"], p["pre"], EPS)
    logits = h @ p["wr"].T
    gates = np.stack([router.weights(logits[t], ids[t], "softmax", False, 1.0) for t in range(T)])
    z = np.zeros_like(h)
    kept = []
    for e in range(E):
        t, j = np.nonzero(ids == e)
        g, u = h[t] @ p["wg"][e].T, h[t] @ p["wu"][e].T
        sig = 1 / (1 + np.exp(-g))
        y = (g * sig * u) @ p["wd"][e].T
        np.add.at(z, t, gates[t, j][:, None] * y)
        kept.append((t, j, g, u, sig, y))
    out, nxt = block.join(z, p["x"], p["post"], None, p["next"], scale, EPS)
    loss = (c1 * out).sum() + (c2 * nxt).sum()
    J = block.join_backward(c1, c2, z, out, p["post"], None, p["next"], scale, EPS)
    dh, dgates = np.zeros_like(h), np.zeros_like(gates)
    grads = {n: np.zeros_like(p[n]) for n in ("wg", "wu", "wd")}
    for e, (t, j, g, u, sig, y) in enumerate(kept):
        dgates[t, j] = (J["d_z"][t] * y).sum(1)
        dy = gates[t, j][:, None] * J["d_z"][t]
        dm = dy @ p["wd"][e]
        du, dg = dm * g * sig, dm * u * sig * (1 + g * (1 - sig))
        np.add.at(dh, t, dg @ p["wg"][e] + du @ p["wu"][e])
        grads["wd"][e], grads["wg"][e], grads["wu"][e] = dy.T @ (g * sig * u), dg.T @ h[t], du.T @ h[t]
    dl = router.topk_backward(dgates, logits, ids, "softmax", False, 1.0)
    grads["wr"] = dl.T @ h
    # A gate's gradient is the inner product of d_z and y, and d_z is orthogonal to z (the norm of z does not see its length): with one expert per token nothing is left
    # of it, with more it is a difference.  Its terms' sizes, and what they make of the gradients behind it, are what its roundings are relative to.
    agates, asize = np.zeros_like(gates), dict.fromkeys(grads, 0.0)
    for t, j, _, _, _, y in kept:
        agates[t, j] = (np.abs(J["d_z"][t]) * np.abs(y)).sum(1)
    prob = np.stack([router._scores(l, "softmax") for l in logits])
    adl = prob * (agates * gates).sum(1, keepdims=True)
    for j in range(ids.shape[1]):
        there = np.flatnonzero(ids[:, j] >= 0)
        adl[there, ids[there, j]] += agates[there, j] * gates[there, j]
    ah = adl @ np.abs(p["wr"])
    asize.update(wr=np.linalg.norm(adl.T @ np.abs(h)), pre=np.linalg.norm((ah * np.abs(h / p["pre"])).sum(0)), x=np.linalg.norm(2 * ah * np.abs(p["pre"]) / block._rms(p["x"], EPS)))
    dx, grads["pre"] = block.norm_gradient(dh + dl @ p["wr"], p["x"], p["pre"], EPS)
    grads.update(x=dx + J["d_stream"], post=J["d_post_weight"], next=J["d_next_weight"])
    return loss, grads, asize


def training_case(T, E, k, d, f, seed):
    g = np.random.default_rng(seed)
    bf = lambda a: torch.from_numpy(a).bfloat16().double().numpy()                          # noqa: E731
    f32 = lambda a: a.astype(np.float32).astype(np.float64)                                 # noqa: E731
    p = dict(x=f32(g.normal(size=(T, d))), pre=f32(1 + 0.2 * g.normal(size=d)), wr=f32(g.normal(size=(E, d)) / d ** 0.5), wg=bf(g.normal(size=(E, f, d)) / d ** 0.5),
             wu=bf(g.normal(size=(E, f, d)) / d ** 0.5), wd=bf(g.normal(size=(E, d, f)) / f ** 0.5), post=f32(1 + 0.2 * g.normal(size=d)), next=f32(1 + 0.2 * g.normal(size=d)))
    return p, f32(g.normal(size=(T, d))), bf(g.normal(size=(T, d)))


def test_plain_step_matches_differences():
    T, E, k, d, f = 5, 4, 2, 16, 8
    p, c1, c2 = training_case(T, E, k, d, f, 0)
    ids = np.stack([np.random.default_rng(t).permutation(E)[:k] for t in range(T)])
    ids[3, 1] = -1
    _, grads, _ = plain_step(p, ids, c1, c2, 0.75)
    rng = np.random.default_rng(1)
    for name in p:
        v = rng.normal(size=p[name].shape)
        step = 1e-5
        up, down = (plain_step(dict(p, **{name: p[name] + s * v}), ids, c1, c2, 0.75)[0] for s in (step, -step))
        # the third derivative times step^2 is some 1e-10 of the slope's size, the differences of sums near 50 in 1e-16 by 1e-5 some 1e-9
        slope, want = (up - down) / (2 * step), (grads[name] * v).sum()
        assert abs(slope - want) <= 1e-6 * (np.abs(grads[name] * v).sum() + 1), (name, slope, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k,d,f", [(1, 2, 1, 256, 256), (45, 4, 2, 256, 256), (203, 8, 3, 512, 256)])
def test_training(lib, T, E, k, d, f):
    p, c1, c2 = training_case(T, E, k, d, f, T)
    scale = 0.75
    up = lambda a, t: torch.from_numpy(a).to(t).to(DEV)                                     # noqa: E731
    q = {n: up(a, torch.bfloat16 if n in ("wg", "wu", "wd") else torch.float32) for n, a in p.items()}
    h = lib.moe_block_norm(q["x"], q["pre"], EPS)
    logits = h.float() @ q["wr"].t()
    ids, gates = lib.moe_router_topk(logits, k, "softmax", False)
    traffic, _ = lib.moe_route_histogram(ids.view(1, T, k), E)
    sched = lib.moe_decompose_greedy(traffic.unsqueeze(0), 2)
    M = T * k
    off, _, asg = lib.moe_slice_table_rows(ids.view(1, T, k), E, 0, traffic, sched["perms"][0], sched["durations"][0], sched["counts"], 2, M)
    X = h[(asg // k).long()]
    experts = (q["wg"], q["wu"], q["wd"])
    y = lib.moe_expert_ffn_sliced(X, off, 4, E, *experts)
    row_of = torch.empty(M, dtype=torch.int32, device=DEV)
    row_of[asg.long()] = torch.arange(M, dtype=torch.int32, device=DEV)
    row_of = row_of.view(T, k)
    z = lib.moe_combine_topk_sum(y, row_of, gates)
    out, nxt = lib.moe_block_join(z, q["x"], q["post"], None, q["next"], scale, EPS)
    # back
    J = lib.moe_block_join_backward(up(c1, torch.float32), up(c2, torch.bfloat16), z, out, q["post"], None, q["next"], scale, EPS)
    C = lib.moe_combine_topk_sum_backward(J["d_z"], y, row_of, gates)
    F = lib.moe_expert_ffn_backward_sliced(X, C["d_y"], off, 4, E, *experts)
    d_h = lib.moe_combine_topk_sum(F["dx"], row_of)                       # the gather's gradient is the sum over a token's rows
    d_logits = lib.moe_router_topk_backward(C["d_gate"], logits, ids, "softmax", False)
    d_h = (d_h.float() + d_logits @ q["wr"]).bfloat16()
    B = lib.moe_block_norm_backward(d_h, q["x"], q["pre"], EPS, d_stream=J["d_stream"])
    got = dict(x=B["d_x"], pre=B["d_weight"], post=J["d_post_weight"], next=J["d_next_weight"], wg=F["dw_gate"], wu=F["dw_up"], wd=F["dw_down"], wr=d_logits.t() @ h.float())
    # The way through the router's weights, whose gradients are small differences, step by step: each from what the one before returned
    i64, s, w = ids.cpu().numpy().astype(np.int64), np.stack([router._scores(l, "softmax") for l in f64(logits)]), f64(gates)
    terms = f64(J["d_z"])[:, None, :] * f64(y)[row_of.cpu().numpy()]
    near(C["d_gate"], terms.sum(2), 64 * 2.0 ** -24 * np.abs(terms).sum(2))
    dg = f64(C["d_gate"])
    size = s * (np.abs(dg) * w).sum(1, keepdims=True)
    np.add.at(size, (np.arange(T)[:, None], i64), np.abs(dg) * w)
    near(d_logits, router.topk_backward(dg, f64(logits), i64, "softmax", False), 2.0 ** -16 * size)
    _, want, sizes = plain_step(p, ids.cpu().numpy().astype(np.int64), c1, c2, scale)
    # Between x and a gradient lie the roundings to bf16 of h, the experts' inner values, y, z, next, d_z, d_y, the inner gradients (3), dx, d_h (2) and the
    # gradient itself: 13 of at most 2^-8 relative each, of which each may grow by two through the products and the norms' Jacobians: 13 * 2 * 2^-8 = 0.10.
    # A term that is missing or taken twice is off by its whole size.  (The gates' gradients: relative to their terms, see plain_step.  T 1, k 1: the true gradient of
    # wr is zero but for eps, the terms' is 1e3 times the difference that the two roundings of d_z and y leave.)
    for name, ref in want.items():
        err = np.linalg.norm(f64(got[name]) - ref) / max(np.linalg.norm(ref) + sizes.get(name, 0.0), 1e-300)
        assert err <= 0.10, (name, err)
        print(name, "%.4f" % err)


# ------------------------------------------------------------------------------------------------ a backward pass captured
@pytest.mark.gpu
def test_backward_captured(lib):
    T, d, E, k = 130, 1032, 64, 4
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(s, generator=g).to(DEV)                                      # noqa: E731
    static = dict(z=r(T, d).bfloat16(), x=r(T, d), d_out=r(T, d), d_next=r(T, d).bfloat16(), gate=r(T).abs(), wp=r(d), wn=r(d), logits=r(T, E), gates=r(T, k), dg=r(T, k))
    row_of = torch.randperm(T * k, generator=g).to(DEV).int().view(T, k)
    row_of[3, 1], row_of[5, 0] = -1, row_of[6, 0]                         # unnamed rows and one named twice
    y = r(T * k, d).bfloat16()

    def step():
        s = static
        out, nxt = lib.moe_block_join(s["z"], s["x"], s["wp"], s["gate"], s["wn"], 0.5, EPS)
        J = lib.moe_block_join_backward(s["d_out"], s["d_next"], s["z"], out, s["wp"], s["gate"], s["wn"], 0.5, EPS)
        C = lib.moe_combine_topk_sum_backward(J["d_z"], y, row_of, s["gates"])
        ids, gates = lib.moe_router_topk(s["logits"], k)
        dl = lib.moe_router_topk_backward(s["dg"], s["logits"], ids)
        B = lib.moe_block_norm_backward(s["d_next"], s["x"], s["wn"], EPS, d_stream=J["d_stream"])
        return [out, nxt, *[v for v in J.values() if v is not None], C["d_y"], C["d_gate"], ids, gates, dl, B["d_x"], B["d_weight"]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        for name, t in static.items():
            t.copy_(r(*t.shape).abs() if name == "gate" else r(*t.shape))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(captured, want)):
            assert torch.equal(a, b), (i, n)


# ------------------------------------------------------------------------------------------------ more than 2^31 elements
def repeated(rows, T, dtype, seed, d=4096):
    part = torch.randn(rows, d, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)
    return part, part.repeat((T + rows - 1) // rows, 1)[:T]


@pytest.mark.gpu
def test_block_of_many_rows(lib):
    """Rows behind element 2^31 get what the same rows get in a small call."""
    T, d, rows = 524288 + 515, 4096, 1031
    tail = T % rows
    x, X = repeated(rows, T, torch.bfloat16, 1)
    z, Z = repeated(rows, T, torch.bfloat16, 2)
    w = torch.linspace(0.5, 1.5, d, device=DEV)
    small, large = lib.moe_block_join(z, x, w, None, w, 0.5), lib.moe_block_join(Z, X, w, None, w, 0.5)
    for a, b in zip(small, large):
        assert torch.equal(b[-tail:], a[:tail]) and torch.equal(b[:rows], a)
    assert torch.equal(lib.moe_block_norm(X, w)[-tail:], lib.moe_block_norm(x, w)[:tail])
    # gradients: all but the last rows have none of their own, so that the weights' gradients are the last rows' alone
    D = torch.zeros_like(X)
    D[-tail:] = z[:tail]
    J, j = (lib.moe_block_join_backward(a, b, c, e, w, None, w, 0.5) for a, b, c, e in ((D, D, Z, large[0], ), (z[:tail], z[:tail], z[:tail], small[0][:tail])))
    for name in ("d_z", "d_stream"):
        assert torch.equal(J[name][-tail:], j[name]) and not J[name][:-tail].any().item()
    for name in ("d_post_weight", "d_next_weight"):
        # the same terms in another order: at most 2 * rows roundings of 2^-24 of their absolute sum; the terms reach about 8 each, 1e-3 is far above
        assert (J[name] - j[name]).abs().max().item() <= 2 * rows * 2.0 ** -24 * rows * 8
    del J, j
    B, b = lib.moe_block_norm_backward(D, X, w, d_stream=D), lib.moe_block_norm_backward(z[:tail], x[:tail], w, d_stream=z[:tail])
    assert torch.equal(B["d_x"][-tail:], b["d_x"]) and (B["d_weight"] - b["d_weight"]).abs().max().item() <= 2 * rows * 2.0 ** -24 * rows * 8


@pytest.mark.gpu
def test_combine_and_router_of_many_rows(lib):
    T, k, d, rows = 262144 + 77, 2, 4096, 509
    g, G = repeated(rows, T, torch.bfloat16, 3)
    y = torch.randn(1024, d, generator=torch.Generator().manual_seed(4)).bfloat16().to(DEV)
    Y = y.repeat((T * k + 1023) // 1024, 1)[:T * k]
    row_of = torch.arange(T * k, dtype=torch.int32, device=DEV).flip(0).view(T, k).contiguous()
    gate = torch.rand(T, k, generator=torch.Generator().manual_seed(5)).to(DEV)
    o = lib.moe_combine_topk_sum_backward(G, Y, row_of, gate)
    for t in (0, 1, T // 2, T - 1):                                       # token t names rows T k - 1 - 2 t and the one before
        for j in (0, 1):
            row = T * k - 1 - (k * t + j)
            assert torch.equal(o["d_y"][row], (gate[t, j] * G[t].float()).bfloat16())
            # 4096 products: a chain of 16 per thread and the threads' tree, fewer than 64 roundings
            prod = G[t].double() * Y[row].double()
            assert abs(o["d_gate"][t, j].item() - prod.sum().item()) <= 64 * 2.0 ** -24 * prod.abs().sum().item()
    del o, G, Y
    T, E, rows = 8388608 + 777, 256, 4099
    l, L = repeated(rows, T, torch.float32, 6, E)
    tail = T % rows
    small, large = lib.moe_router_topk(l, 8), lib.moe_router_topk(L, 8)
    for a, b in zip(small, large):
        assert torch.equal(b[-tail:], a[:tail])
    dg = torch.randn(rows, 8, generator=torch.Generator().manual_seed(7)).to(DEV)
    DG = dg.repeat((T + rows - 1) // rows, 1)[:T]
    assert torch.equal(lib.moe_router_topk_backward(DG, L, large[0], renormalise=False)[-tail:], lib.moe_router_topk_backward(dg, l, small[0], renormalise=False)[:tail])


@pytest.mark.gpu
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("kind,E,k,T", [("f32", 4096, 32, 5), ("bf16", 4096, 1, 3), ("f32", 2049, 17, 6), ("bf16", 250, 32, 9)])
def test_router_gradients_of_many_experts(lib, kind, E, k, T, renormalise):
    rng = np.random.default_rng(E)
    l = torch.from_numpy(rng.normal(size=(T, E)).astype(np.float32))
    l = l if kind == "f32" else l.bfloat16()
    dg = rng.normal(size=(T, k)).astype(np.float32)
    ids, _ = lib.moe_router_topk(l.to(DEV), k, "softmax", renormalise)
    if k > 1:
        ids[1, 0] = ids[1, 1]                                             # one expert twice
    got = lib.moe_router_topk_backward(torch.from_numpy(dg).to(DEV), l.to(DEV), ids, "softmax", renormalise)
    ref = router.topk_backward(dg.astype(np.float64), f64(l), ids.cpu().numpy(), "softmax", renormalise)
    s = np.stack([router._scores(row, "softmax") for row in f64(l)])
    w = np.abs(np.stack([router.weights(f64(l)[t], ids.cpu().numpy()[t], "softmax", renormalise) for t in range(T)]))
    size = np.zeros((T, E))
    for t in range(T):
        mean = (np.abs(dg[t]) * w[t]).sum()
        np.add.at(size[t], ids.cpu().numpy()[t], (np.abs(dg[t]) + mean) * (w[t] if renormalise else s[t][ids.cpu().numpy()[t]]))
        if not renormalise:
            size[t] += s[t] * mean
        else:
            # an expert that was not chosen gets nothing; in the oracle its terms -dg w_j s_e and +dg w_j sum(w) s_e cancel but for their own roundings, of 2^-53 each
            # in sums of at most 33 terms: below 2^-47 of their sizes, of which 2^-16 is taken below
            size[t] += 2.0 ** -31 * 2 * s[t] * mean
    # d = p (G - mean): p and the weights to 2^-18 (exponent, sum over E in chains of at most E / 64 and 6 levels), the differences of what is left of it, one rounding at the end
    near(got, ref, 2.0 ** -16 * size + (HALF if kind == "bf16" else 2.0 ** -24) * np.abs(ref) + 1e-30)


@pytest.mark.gpu
def test_more_rows_than_a_launch(lib):
    """Calls that take several launches: the rows of the later ones get what the same rows get in a small call."""
    d, rows = 64, 1000
    T = (1 << 21) + 5
    x, X = repeated(rows, T, torch.bfloat16, 8, d)
    z, Z = repeated(rows, T, torch.bfloat16, 9, d)
    w = torch.linspace(0.5, 1.5, d, device=DEV)
    tail = T % rows
    for a, b in zip(lib.moe_block_join(z, x, w, None, w), lib.moe_block_join(Z, X, w, None, w)):
        assert torch.equal(b[-tail:], a[:tail]) and torch.equal(b[:rows], a)
    row_of = torch.arange(T, dtype=torch.int32, device=DEV).flip(0).view(T, 1).contiguous()
    row_of[7] = -1
    o = lib.moe_combine_topk_sum_backward(Z, X, row_of)
    want = Z.flip(0)
    want[T - 8] = 0
    assert o["d_gate"] is None and torch.equal(o["d_y"], want)
    T, E = (1 << 24) + 9, 8
    l, L = repeated(rows, T, torch.float32, 10, E)
    tail = T % rows
    small, large = lib.moe_router_topk(l, 2), lib.moe_router_topk(L, 2)
    assert all(torch.equal(b[-tail:], a[:tail]) for a, b in zip(small, large))
    dg, DG = repeated(rows, T, torch.float32, 11, 2)
    for ren in (False, True):
        assert torch.equal(lib.moe_router_topk_backward(DG, L, large[0], renormalise=ren)[-tail:], lib.moe_router_topk_backward(dg, l, small[0], renormalise=ren)[:tail])
