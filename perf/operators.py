"""Cases of the operators around the experts: what the rank that owns the tokens does before and after them, and the experts themselves
with weights of 4 bits.

A MoE block is: norm, router, experts, weighted sum of their results (combine), then the join with the residual stream, which also makes the next
block's normalised input.  Kinds "norm" and "join" (forward and "_backward"), "router" (and "router_backward"), "combine_backward"
and "ffn_w4".

  listed()  the cases            draw(rng)  one more case of the same ranges
  prepare(case, seed)            what the program holds before the call
  run(state)                     one pass: the plain form, or with `own` the library's calls
  exact(case, seed)              the definition in 64 bits            work(case)  what a pass cannot do without
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-6
ZIPF = 1.2


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # decoding one token: the join between two blocks, a launch of a few kilobytes
        dict(name="join_decode", kind="join", T=1, d=4096, stream="bf16", post=True, gate=False, next=True, scale=1.0),
        # a long prompt of a wide model: post-norm, token gate, residual scale and the next norm in one pass
        dict(name="join_prefill", kind="join", T=16381, d=7168, stream="bf16", post=True, gate=True, next=True, scale=0.75),
        # training with the residual stream in float32: all gradients of the join
        dict(name="join_backward", kind="join_backward", T=8192, d=4096, stream="f32", post=True, gate=True, next=True, scale=0.75),
        # training: the norm before the block, its gradient added to the one that came along the stream
        dict(name="norm_backward", kind="norm_backward", T=16384, d=2048, stream="bf16"),
        # a decoding batch through the router of a layer of 256 experts, top-8 of sigmoid scores
        dict(name="router_decode", kind="router", T=64, E=256, topk=8, logits="f32", score="sigmoid", renormalise=True, masked=False),
        # a prompt's routes; some tokens are padding and masked altogether, logits in bf16 with their many ties
        dict(name="router_prefill", kind="router", T=32771, E=64, topk=2, logits="bf16", score="softmax", renormalise=False, masked=True),
        # training: the gradient of every logit through the probabilities
        dict(name="router_backward", kind="router_backward", T=16384, E=256, topk=8, logits="f32", score="softmax", renormalise=False, masked=False),
        # training on few tokens: two experts per token, odd number of tokens, some assignments dropped
        dict(name="combine_backward", kind="combine_backward", T=777, topk=2, d=2048),
        # training, the wide layer with eight experts per token
        dict(name="combine_backward_top8", kind="combine_backward", T=8192, topk=8, d=4096),
        # decoding one token on a rank that holds one large expert: the weights' way from memory
        dict(name="ffn_w4_one_row", kind="ffn_w4", E_loc=1, S=1, d=4096, f=14336, M=1, group=128, zeros=False, mapped=False),
        # a decoding batch over four experts in the slices of a schedule, groups of 32 with zero points, gather and scatter fused
        dict(name="ffn_w4_decode", kind="ffn_w4", E_loc=4, S=18, d=7168, f=2048, M=203, group=32, zeros=True, mapped=True),
        # a prompt: thousands of ragged rows, where the products count and not the weights
        dict(name="ffn_w4_prefill", kind="ffn_w4", E_loc=4, S=10, d=2048, f=1408, M=8191, group=128, zeros=False, mapped=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


W4_MOST = 6.0 * 2048 * 1408 * 8191               # products of the largest listed case of 4-bit weights
ROWS_MOST = 16381 * 7168                         # values of the largest listed stream


def draw(rng):
    kind = rng.choice(["join", "join", "join_backward", "norm", "norm_backward", "router", "router", "router_backward",
                       "combine_backward", "combine_backward", "ffn_w4", "ffn_w4", "ffn_w4", "ffn_w4"])
    if kind in ("join", "join_backward", "norm", "norm_backward"):
        d = rng.choice([256, 1280, 2048, 2880, 4096, 5120, 7168, 8192, 8 * rng.randint(1, 1024)])
        c = dict(kind=kind, T=min(_log(rng, 1, 32768), ROWS_MOST // (2 * d)), d=d, stream=rng.choice(["bf16", "f32"]))
        if kind.startswith("join"):
            c.update(post=rng.random() < 0.7, gate=rng.random() < 0.5, next=rng.random() < 0.8, scale=rng.choice([1.0, 0.75, 1.5]))
        return c
    if kind.startswith("router"):
        E = rng.choice([4, 8, 16, 60, 64, 128, 160, 256, 256, rng.randint(2, 256)])
        topk = min(E, rng.choice([1, 2, 2, 4, 6, 8, 8, 3]))
        return dict(kind=kind, T=_log(rng, 1, 32768), E=E, topk=topk, logits=rng.choice(["f32", "bf16"]), score=rng.choice(["softmax", "sigmoid"]),
                    renormalise=topk > 1 and rng.random() < 0.5, masked=rng.random() < 0.4)
    if kind == "combine_backward":
        topk, d = rng.choice([1, 2, 2, 3, 4, 6, 8]), rng.choice([256, 1280, 2048, 2880, 4096, 7168, 8 * rng.randint(1, 896)])
        return dict(kind=kind, T=min(_log(rng, 1, 16384), 8192 * 8 * 4096 // (topk * d)), topk=topk, d=d)
    d, f = rng.choice([(256, 512), (2048, 1408), (4096, 14336), (7168, 2048), (256 * rng.randint(1, 20), 128 * rng.randint(2, 40))])
    E_loc = rng.choice([1, 2, 4, 8])
    while E_loc > 1 and E_loc * d * f > 1.2e8:
        E_loc //= 2
    return dict(kind=kind, E_loc=E_loc, S=rng.choice([1, 1, 6, 18, 50]), d=d, f=f, M=min(_log(rng, 1, 8191), int(W4_MOST / (6.0 * d * f))),
                group=rng.choice([32, 64, 128, 128]), zeros=rng.random() < 0.5, mapped=rng.random() < 0.4)


# ------------------------------------------------------------------------------------------------ inputs
def _randn(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device=DEV) * std


def _rows(T, d, g, dtype):
    """Activations of T tokens: their sizes differ from token to token, and a few columns stand out."""
    size = torch.exp(_randn((T, 1), g, 0.5))
    columns = torch.exp(_randn((1, d), g, 0.5))
    return (_randn((T, d), g) * size * columns).to(dtype)


def _popularity(E, rng):
    p = (rng.permutation(E) + 1.0) ** -ZIPF
    return p / p.sum()


def _w4(E, n, k, group, zeros, g):
    """N(0, 0.02) weights in 4 bits: codes two to a byte (even input in the low half), one scale and, with `zeros`, one zero point per group."""
    w = (_randn((E, n, k), g, 0.02)).view(E, n, k // group, group)
    if zeros:
        lo, hi = w.amin(3), w.amax(3)
        s = ((hi - lo) / 15.0).to(torch.bfloat16)
        z = (-lo / s.float()).round().clamp_(0, 15)
    else:
        s = (w.abs().amax(3) / 7.0).to(torch.bfloat16)
        z = torch.full_like(w[..., 0], 8.0)
    q = (w / s.float()[..., None] + z[..., None]).round_().clamp_(0, 15).to(torch.uint8).view(E, n, k)
    codes = (q[..., 0::2] | (q[..., 1::2] << 4)).contiguous()
    return codes, s.transpose(1, 2).contiguous(), z.to(torch.uint8).transpose(1, 2).contiguous() if zeros else None


def _group_sizes(S, E_loc, M, rng):
    """Rows per (slice, local expert): slice 0 local, matchings of falling size of which some bring nothing."""
    w = rng.uniform(0.5, 1.5, S) * (1.0 - 0.6 * np.arange(S) / S) * (rng.random(S) >= 0.08)
    w[0] = 1.0
    return rng.multinomial(M, np.outer(w / w.sum(), _popularity(E_loc, rng)).ravel())


def prepare(case, seed):
    c = case
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(c)
    kind = c["kind"]
    if kind in ("join", "join_backward", "norm", "norm_backward"):
        T, d = c["T"], c["d"]
        dtype = torch.float32 if c["stream"] == "f32" else torch.bfloat16
        weight = lambda: 1.0 + _randn((d,), g, 0.2)                                        # noqa: E731
        if kind.startswith("norm"):
            s["x"], s["weight"] = _rows(T, d, g, dtype), weight()
            if kind == "norm_backward":
                s["d_out"], s["d_stream"] = _rows(T, d, g, torch.bfloat16), _rows(T, d, g, dtype)
            return s
        s["z"] = _rows(T, d, g, torch.bfloat16)
        s["post_weight"] = weight() if c["post"] else None
        s["next_weight"] = weight() if c["next"] else None
        s["token_gate"] = torch.sigmoid(_randn((T,), g)) if c["gate"] else None
        if kind == "join":
            s["x"] = _rows(T, d, g, dtype)
        else:
            s["out"], s["d_out"] = _rows(T, d, g, dtype), _rows(T, d, g, dtype)
            s["d_next"] = _rows(T, d, g, torch.bfloat16) if c["next"] else None
        return s
    if kind in ("router", "router_backward"):
        T, E = c["T"], c["E"]
        logits = _randn((T, E), g, 1.5) + torch.from_numpy(np.log(_popularity(E, rng))).float().to(DEV)
        if c["masked"]:                                          # experts out of order for some tokens, and padding that has none
            logits[torch.rand((T, E), generator=g, device=DEV) < 0.1] = -math.inf
            logits[torch.rand((T,), generator=g, device=DEV) < 0.02] = -math.inf
        s["x"] = logits.to(torch.float32 if c["logits"] == "f32" else torch.bfloat16)
        if kind == "router_backward":
            s["ids"] = _select(s["x"], c["topk"])[0]
            s["d_gates"] = _randn((T, c["topk"]), g)
        return s
    if kind == "combine_backward":
        T, topk, d = c["T"], c["topk"], c["d"]
        R = T * topk
        s["y"] = torch.empty((R, d), dtype=torch.bfloat16, device=DEV)
        for at in range(0, R, 32768):
            s["y"][at:at + 32768] = _randn((min(32768, R - at), d), g).to(torch.bfloat16)
        row_of = torch.randperm(R, generator=g, device=DEV).int()
        row_of[torch.rand((R,), generator=g, device=DEV) < 0.01] = -1                    # dropped assignments
        s["row_of"] = row_of.view(T, topk)
        s["route_gate"] = torch.softmax(_randn((T, topk), g), dim=1)
        s["d_out"] = _rows(T, d, g, torch.bfloat16)
        return s
    E, S, M, d, f = c["E_loc"], c["S"], c["M"], c["d"], c["f"]
    sizes = _group_sizes(S, E, M, rng)
    s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)).to(DEV)
    s["most"] = int(sizes.reshape(S, E).sum(0).max())                                      # rows of the most popular expert
    s["x"] = _randn((M, d), g).to(torch.bfloat16)
    for name, n, k in (("gate", f, d), ("up", f, d), ("down", d, f)):
        s["q_" + name], s["s_" + name], s["z_" + name] = _w4(E, n, k, c["group"], c["zeros"], g)
    s["row_map"] = torch.randperm(M, generator=g, device=DEV).int() if c["mapped"] else None
    s["row_gate"] = torch.rand((M,), generator=g, device=DEV) if c["mapped"] else None
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _normed(v):
    return v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)


def _norm_gradient(dn, v):
    """The gradient of v from that of v * rsqrt(mean(v^2) + eps)."""
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    n = v * r
    return r * (dn - n * (dn * n).mean(1, keepdim=True))


def _plain_join(s):
    z, x = s["z"].float(), s["x"].float()
    u = _normed(z) * s["post_weight"] if s["post"] else z
    if s["gate"]:
        u = u * s["token_gate"][:, None]
    out = s["scale"] * x + u
    return out.to(s["x"].dtype), (_normed(out) * s["next_weight"]).to(torch.bfloat16) if s["next"] else None


def _plain_join_backward(s):
    z, out, total = s["z"].float(), s["out"].float(), s["d_out"].float()
    g = dict(d_gate=None, d_post_weight=None, d_next_weight=None)
    if s["next"]:
        dn = s["d_next"].float()
        g["d_next_weight"] = (dn * _normed(out)).sum(0)
        total = total + _norm_gradient(dn * s["next_weight"], out)
    g["d_stream"] = (s["scale"] * total).to(s["out"].dtype)
    u = _normed(z) * s["post_weight"] if s["post"] else z
    du = total
    if s["gate"]:
        g["d_gate"] = (total * u).sum(1)
        du = total * s["token_gate"][:, None]
    if s["post"]:
        g["d_post_weight"] = (du * _normed(z)).sum(0)
        du = _norm_gradient(du * s["post_weight"], z)
    g["d_z"] = du.to(torch.bfloat16)
    return g


def _select(logits, topk):
    """The topk largest logits of each row, the lower index first where they are equal; masked ones are not taken (-1)."""
    v, i = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    v, i = v[:, :topk], i[:, :topk]
    return torch.where(v == -math.inf, -1, i).int(), v


def _shares(s, logits, chosen):
    """Scores of all experts and of the chosen ones, before they are made to sum to one; a masked expert's is zero."""
    if s["score"] == "sigmoid":
        p = torch.sigmoid(logits)
    else:
        top = logits.amax(1, keepdim=True)
        e = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
        p = e / e.sum(1, keepdim=True).clamp_min(1e-30)
    return p, torch.gather(p, 1, chosen.clamp_min(0).long()) * (chosen >= 0)


def _plain_router(s):
    ids, _ = _select(s["x"], s["topk"])
    w = _shares(s, s["x"].float(), ids)[1]
    if s["renormalise"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-30)
    return ids, w


def _plain_router_backward(s):
    logits, dg = s["x"].float(), s["d_gates"] * (s["ids"] >= 0)
    p, w = _shares(s, logits, s["ids"])
    if s["renormalise"]:
        total = w.sum(1, keepdim=True).clamp_min(1e-30)
        dg = (dg - (dg * w).sum(1, keepdim=True) / total) / total
    dp = torch.zeros_like(logits).scatter_add_(1, s["ids"].clamp_min(0).long(), dg * (s["ids"] >= 0))
    dl = dp * p * (1.0 - p) if s["score"] == "sigmoid" else p * (dp - (dp * p).sum(1, keepdim=True))
    return dl.to(s["x"].dtype)


def _plain_combine_backward(s):
    rows = s["row_of"].flatten()
    live = rows >= 0
    at = rows.clamp_min(0).long()
    do = s["d_out"].float().repeat_interleave(s["topk"], dim=0)
    d_gate = (do * s["y"][at].float()).sum(1) * live
    d_y = torch.zeros(s["y"].shape, dtype=torch.float32, device=DEV)
    d_y.index_add_(0, at, do * (s["route_gate"].flatten() * live)[:, None])
    return dict(d_y=d_y.to(torch.bfloat16), d_gate=d_gate.view_as(s["route_gate"]))


def _unpacked(q, scale, zero, group):
    codes = torch.stack((q & 15, q >> 4), dim=3).flatten(2)
    E, n, k = codes.shape
    z = 8.0 if zero is None else zero.transpose(1, 2)[..., None].float()
    return ((codes.view(E, n, k // group, group).float() - z) * scale.transpose(1, 2)[..., None].float()).view(E, n, k)


def _plain_ffn_w4(s):
    M, E = s["M"], s["E_loc"]
    w_gate, w_up, w_down = (_unpacked(s["q_" + n], s["s_" + n], s["z_" + n], s["group"]) for n in ("gate", "up", "down"))
    m = torch.arange(M, device=DEV, dtype=torch.int32)
    expert = (torch.searchsorted(s["offsets"], m, right=True) - 1) % E
    order = torch.argsort(expert, stable=True)
    count = (expert[:, None] == torch.arange(E, device=DEV)).sum(0)
    place = expert[order] * s["most"] + m - (count.cumsum(0) - count)[expert[order]]         # each expert's rows behind each other, padded to the most
    row = order if s["row_map"] is None else s["row_map"][order].long()
    x = torch.zeros((E * s["most"], s["d"]), device=DEV)
    x[place] = s["x"][row].float()
    x = x.view(E, s["most"], s["d"])
    g, u = torch.bmm(x, w_gate.transpose(1, 2)), torch.bmm(x, w_up.transpose(1, 2))
    out = torch.bmm(g * torch.sigmoid(g) * u, w_down.transpose(1, 2)).flatten(0, 1)[place]
    if s["row_gate"] is not None:
        out = out * s["row_gate"][order][:, None]
    y = torch.empty_like(s["x"])
    y[row] = out.to(torch.bfloat16)
    return y


def run(s):
    kind = s["kind"]
    if own:
        import paper_2605_26845_amd as moe
        if kind == "norm":
            return moe.moe_block_norm(s["x"], s["weight"], EPS)
        if kind == "norm_backward":
            return moe.moe_block_norm_backward(s["d_out"], s["x"], s["weight"], EPS, d_stream=s["d_stream"])
        if kind == "join":
            return moe.moe_block_join(s["z"], s["x"], s["post_weight"], s["token_gate"], s["next_weight"], s["scale"], EPS)
        if kind == "join_backward":
            return moe.moe_block_join_backward(s["d_out"], s["d_next"], s["z"], s["out"], s["post_weight"], s["token_gate"], s["next_weight"],
                                               s["scale"], EPS)
        if kind == "router":
            return moe.moe_router_topk(s["x"], s["topk"], s["score"], s["renormalise"])
        if kind == "router_backward":
            return moe.moe_router_topk_backward(s["d_gates"], s["x"], s["ids"], s["score"], s["renormalise"])
        if kind == "combine_backward":
            return moe.moe_combine_topk_sum_backward(s["d_out"], s["y"], s["row_of"], s["route_gate"])
        return moe.moe_expert_ffn_w4_sliced(s["x"], s["offsets"], s["S"], s["E_loc"], s["q_gate"], s["q_up"], s["q_down"], s["s_gate"], s["s_up"],
                                            s["s_down"], s["z_gate"], s["z_up"], s["z_down"], s["row_map"], s["row_gate"])
    if kind == "norm":
        return (_normed(s["x"].float()) * s["weight"]).to(torch.bfloat16)
    if kind == "norm_backward":
        x, dn = s["x"].float(), s["d_out"].float()
        return dict(d_x=(s["d_stream"].float() + _norm_gradient(dn * s["weight"], x)).to(s["x"].dtype), d_weight=(dn * _normed(x)).sum(0))
    return {"join": _plain_join, "join_backward": _plain_join_backward, "router": _plain_router, "router_backward": _plain_router_backward,
            "combine_backward": _plain_combine_backward, "ffn_w4": _plain_ffn_w4}[kind](s)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _rms64(v):
    return (v.square().sum(1) / v.shape[1] + EPS).sqrt()[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    D = lambda t: t.double()                                                               # noqa: E731
    kind = case["kind"]
    if kind == "norm":
        return D(s["x"]) / _rms64(D(s["x"])) * D(s["weight"])
    if kind in ("join", "join_backward", "norm_backward"):
        # gradients by differentiating the definition
        if kind == "norm_backward":
            x, w = D(s["x"]).requires_grad_(), D(s["weight"]).requires_grad_()
            dx, dw = torch.autograd.grad(x / _rms64(x) * w, (x, w), D(s["d_out"]))
            return dict(d_x=dx + D(s["d_stream"]), d_weight=dw)
        wp, wn, gate = (None if s[n] is None else D(s[n]).requires_grad_() for n in ("post_weight", "next_weight", "token_gate"))
        z = D(s["z"]).requires_grad_()
        u = z if wp is None else z / _rms64(z) * wp
        u = u if gate is None else gate[:, None] * u
        if kind == "join":
            out = s["scale"] * D(s["x"]) + u
            return out.detach(), None if wn is None else (out / _rms64(out) * wn).detach()
        out = D(s["out"]).requires_grad_()
        total, d_wn = D(s["d_out"]), None
        if wn is not None:
            through, d_wn = torch.autograd.grad(out / _rms64(out) * wn, (out, wn), D(s["d_next"]))
            total = total + through
        wanted = [v for v in (z, wp, gate) if v is not None]
        got = dict(zip([id(v) for v in wanted], torch.autograd.grad(u, wanted, total)))
        return dict(d_stream=s["scale"] * total, d_z=got[id(z)], d_post_weight=got.get(id(wp)) if wp is not None else None,
                    d_gate=got.get(id(gate)) if gate is not None else None, d_next_weight=d_wn)
    if kind in ("router", "router_backward"):
        # a masked expert has the score zero; the others' scores from the chosen columns one slot at a time
        logits = D(s["x"])
        there = logits > -math.inf
        safe = torch.where(there, logits, 0.0).requires_grad_()
        if case["score"] == "sigmoid":
            score = there / (1.0 + torch.exp(-safe))
        else:
            top = torch.where(there, logits, -1e30).amax(1, keepdim=True)
            e = there * torch.exp(torch.where(there, safe - top, 0.0))
            score = e / torch.where(there.any(1, keepdim=True), e.sum(1, keepdim=True), 1.0)
        if kind == "router":
            left, ids = torch.where(there, logits, -math.inf), []
            column = torch.arange(case["E"], device=DEV)
            for _ in range(case["topk"]):
                best = left.amax(1, keepdim=True)
                first = torch.where((left == best) & (best > -math.inf), column, case["E"]).amin(1)
                ids.append(torch.where(first < case["E"], first, -1))
                left = torch.where(column == first[:, None], -math.inf, left)
            ids = torch.stack(ids, 1)
        else:
            ids = s["ids"].long()
        gates = [torch.where(ids[:, j] >= 0, score.gather(1, ids[:, j:j + 1].clamp_min(0))[:, 0], 0.0) for j in range(case["topk"])]
        if case["renormalise"]:
            total = sum(gates)
            gates = [v / torch.where(total > 0, total, 1.0) for v in gates]
        gates = torch.stack(gates, 1)
        if kind == "router":
            return ids.int(), gates.detach()
        return torch.autograd.grad(gates, safe, D(s["d_gates"]))[0]
    if kind == "combine_backward":
        d_y, d_gate = torch.zeros_like(s["y"], dtype=torch.float64), torch.zeros_like(s["route_gate"], dtype=torch.float64)
        do = D(s["d_out"])
        for j in range(case["topk"]):
            t = (s["row_of"][:, j] >= 0).nonzero()[:, 0]
            r = s["row_of"][t, j].long()
            d_y[r] = do[t] * D(s["route_gate"][t, j])[:, None]
            d_gate[t, j] = (do[t] * D(s["y"][r])).sum(1)
        return dict(d_y=d_y, d_gate=d_gate)
    E, S, M = case["E_loc"], case["S"], case["M"]
    off = s["offsets"].tolist()
    y = torch.zeros((M, case["d"]), dtype=torch.float64, device=DEV)
    for e in range(E):
        rows = torch.cat([torch.arange(off[i * E + e], off[i * E + e + 1], device=DEV) for i in range(S)])
        w = []
        for name in ("gate", "up", "down"):
            q, scale, zero = s["q_" + name][e], D(s["s_" + name][e]).t(), s["z_" + name]
            code = torch.empty((q.shape[0], 2 * q.shape[1]), dtype=torch.float64, device=DEV)
            code[:, 0::2], code[:, 1::2] = D(q % 16), D(q // 16)
            zero = torch.full_like(scale, 8.0) if zero is None else D(zero[e]).t()
            w.append((code - zero.repeat_interleave(case["group"], 1)) * scale.repeat_interleave(case["group"], 1))
        at = rows if s["row_map"] is None else s["row_map"][rows].long()
        x = D(s["x"][at])
        g = x @ w[0].t()
        out = (g / (1.0 + torch.exp(-g)) * (x @ w[1].t())) @ w[2].t()
        y[at] = out if s["row_gate"] is None else out * D(s["row_gate"][rows])[:, None]
    return y


# ------------------------------------------------------------------------------------------------ work
def work(case):
    c, kind = case, case["kind"]
    if kind in ("join", "join_backward", "norm", "norm_backward"):
        T, d, stream = c["T"], c["d"], 4 if c["stream"] == "f32" else 2
        if kind == "norm":
            return dict(bytes=T * d * (stream + 2) + 4 * d, flops=4 * T * d)
        if kind == "norm_backward":                              # d_out, x, d_stream -> d_x
            return dict(bytes=T * d * (2 + 3 * stream) + 8 * d, flops=11 * T * d)
        vectors = 4 * d * (c["post"] + c["next"]) + 4 * T * c["gate"]
        if kind == "join":                                       # z, stream -> out, next
            return dict(bytes=T * d * (2 + 2 * stream + 2 * c["next"]) + vectors, flops=T * d * (3 + 4 * c["post"] + 4 * c["next"]))
        return dict(bytes=T * d * (4 + 2 * stream + (2 + stream) * c["next"]) + 2 * vectors, flops=T * d * (3 + 9 * c["post"] + 9 * c["next"]))
    if kind in ("router", "router_backward"):
        T, E, k, size = c["T"], c["E"], c["topk"], 4 if c["logits"] == "f32" else 2
        if kind == "router":
            return dict(bytes=T * (E * size + 8 * k), flops=4 * T * E)
        return dict(bytes=T * (2 * E * size + 8 * k), flops=5 * T * E)
    if kind == "combine_backward":
        T, k, d = c["T"], c["topk"], c["d"]
        return dict(bytes=T * (2 * d * (1 + 2 * k) + 12 * k), flops=3 * T * k * d)
    E, d, f = c["E_loc"], c["d"], c["f"]
    held = min(E, c["M"])                                        # experts that hold rows, at most
    scales = 3 * d * f // c["group"] * (3 if c["zeros"] else 2)
    return dict(bytes=held * (3 * d * f // 2 + scales) + 4 * c["M"] * d, flops=6.0 * c["M"] * d * f)
