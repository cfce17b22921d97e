"""moe_expert_ffn_w4_sliced: the oracle's unpacking, refusals on the host, and the kernels against the float64 oracle."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ffn_w4

DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------ inputs and oracle
def weights(E, d, f, group, zeros, seed):
    """Codes, scales and zero points as the library takes them (torch tensors on the host), with zero points at both ends."""
    g = torch.Generator().manual_seed(seed)
    out = {}
    for name, n, k in (("gate", f, d), ("up", f, d), ("down", d, f)):
        out["q_" + name] = torch.randint(0, 256, (E, n, k // 2), generator=g, dtype=torch.uint8)
        out["s_" + name] = ((0.5 + torch.rand(E, k // group, n, generator=g)) * 0.2 / k ** 0.5).bfloat16()
        out["z_" + name] = torch.randint(0, 16, (E, k // group, n), generator=g, dtype=torch.uint8) if zeros else None
    return out


def unpacked(w, e):
    z = lambda n: None if w["z_" + n] is None else w["z_" + n][e].numpy()                   # noqa: E731
    return tuple(ffn_w4.unpack(w["q_" + n][e].numpy(), w["s_" + n][e].double().numpy(), z(n)) for n in ("gate", "up", "down"))


def expert_of_rows(offsets, E, M):
    e = np.full(M, -1)
    for i in range(len(offsets) - 1):
        e[offsets[i]:offsets[i + 1]] = i % E
    return e


def check(y, x, offsets, E, w, row_map=None, row_gate=None, kept=None):
    """Every row of y against the oracle.  With a = sum |x| 55 |scale| (a code counts as 16 .. 31 and 16 + zero is taken off again) the fp32 sums g and u are off by
    at most 2^-16 a: fewer than 256 roundings.  h is off by that through silu and the product, and by 2^-8 |h| from its rounding; y by what this makes of
    the second product, its own sum, and 2^-8 |y|."""
    M, d = x.shape
    yy = y.double().cpu().numpy()
    expert = expert_of_rows(offsets, E, M)
    read = np.arange(M) if row_map is None else np.concatenate([row_map, np.arange(len(row_map), M)])[:M]
    xx = x.double().numpy()[read]
    full = [unpacked(w, e) for e in range(E)]
    ref, parts = ffn_w4.expert_ffn(xx, expert, full)
    gate = np.ones(M) if row_gate is None else np.concatenate([row_gate.astype(np.float64), np.ones(M - len(row_gate))])[:M]
    worst = 0.0
    for e, part in enumerate(parts):
        if part is None:
            continue
        sel, g, u, h = part
        s = [np.repeat(np.abs(w["s_" + n][e].double().numpy()), (f if n == "down" else d) // w["s_" + n].shape[1], axis=0) for n in ("gate", "up", "down") for f in [w["q_gate"].shape[1]]]
        ax = np.abs(xx[sel])
        eg, eu = 2.0 ** -16 * 55 * (ax @ s[0]), 2.0 ** -16 * 55 * (ax @ s[1])
        with np.errstate(over="ignore"):
            silu = g / (1.0 + np.exp(-g))
        eh = 1.1 * eg * np.abs(u) + np.abs(silu) * eu + 1.1 * eg * eu + (2.0 ** -8 + 2.0 ** -20) * np.abs(h)
        ey = eh @ np.abs(full[e][2]).T + 2.0 ** -16 * 55 * (np.abs(h) @ s[2])
        want = ref[sel] * gate[sel, None]
        err = np.abs(yy[read[sel]] - want)
        bound = np.abs(gate[sel, None]) * ey * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want)
        assert np.isfinite(yy[read[sel]]).all() and (err <= bound).all(), (e, float((err / bound).max()))
        scale = np.abs(want).max() if want.size else 0.0
        if scale > 0:
            worst = max(worst, float(err.max() / scale))
    # beside the worst case: two roundings to bf16 of sums whose terms partly cancel put an expert's largest error at 3e-3 .. 5e-3 of its largest output
    assert worst <= 1e-2, worst
    if kept is not None:
        untouched = np.setdiff1d(np.arange(M), read[expert >= 0])
        assert (yy[untouched] == kept).all()


def offsets_of(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


def run(lib, x, offsets, S, E, w, **more):
    c = {k: (None if v is None else v.to(DEV)) for k, v in w.items()}
    return lib.moe_expert_ffn_w4_sliced(x.to(DEV), torch.from_numpy(offsets).to(DEV), S, E, **c, **more)


def activations(M, d, seed):
    return torch.randn(M, d, generator=torch.Generator().manual_seed(seed)).bfloat16()


# ------------------------------------------------------------------------------------------------ host
def test_oracle_unpacks_by_hand():
    q = np.zeros((2, 16), dtype=np.uint8)
    q[0, 0], q[1, 15] = 0x2F, 0xA0                                        # row 0: inputs 0 and 1 are 15 and 2; row 1: inputs 30 and 31 are 0 and 10
    w = ffn_w4.unpack(q, np.array([[0.5, 2.0]]))
    assert w[0, :3].tolist() == [3.5, -3.0, -4.0] and w[1, 30:].tolist() == [-16.0, 4.0]
    w = ffn_w4.unpack(q, np.array([[0.5, 2.0], [1.0, 4.0]]), np.array([[15, 0], [1, 2]], dtype=np.uint8))
    assert w[0, :3].tolist() == [0.0, -6.5, -7.5] and w[0, 16] == -1.0 and w[1, 30:].tolist() == [-8.0, 32.0]


def test_refusals_need_no_gpu(hostlib):
    L = hostlib.load()
    p, odd, one = ctypes.c_void_p(4096), ctypes.c_void_p(4104), ctypes.c_void_p(4097)

    def f(x=p, off=p, M=4, S=1, E=1, d=256, ff=128, G=128, qg=p, qu=p, qd=p, sg=p, su=p, sd=p, zg=p, zu=p, zd=p, rm=None, rg=None, y=p, ws=p, size=1 << 40):
        return L.moe_expert_ffn_w4_sliced(x, off, M, S, E, d, ff, G, qg, qu, qd, sg, su, sd, zg, zu, zd, rm, rg, y, ws, size, None)
    assert f(M=-1) == -1 and f(S=-1) == -1 and f(E=0) == -1 and f(d=0) == -1 and f(ff=0) == -1
    for name in ("x", "off", "qg", "qu", "qd", "sg", "su", "sd", "y", "zg", "zu", "zd"):
        assert f(**{name: None}) == -1, name
    for name in ("x", "y", "qg", "qu", "qd", "ws"):
        assert f(**{name: odd}) == -1, name
    for name in ("sg", "su", "sd", "zg", "zu", "zd", "rm", "rg", "off"):
        assert f(**{name: one}) == -1, name
    for G in (0, 16, 48, 256, -32):
        assert f(G=G) == -2
    assert f(d=128) == -2 and f(ff=64) == -2 and f(S=70000) == -2 and f(d=1 << 16, ff=1 << 15) == -2 and f(M=(1 << 31) - 1, d=4096) == -2
    assert f(ws=None) == -3 and f(size=1) == -3 and f(M=0, x=None, y=None, ws=None) == 0 and f(S=0, x=None, y=None, ws=None) == 0
    sizes = [L.moe_ffn_w4_workspace_bytes(M, 2048, 1408) for M in (0, 1, 16, 17, 100, 1000, 4096, 4097, 100000)]
    assert sizes == sorted(sizes) and L.moe_ffn_w4_workspace_bytes(-1, 256, 128) == 0


# ------------------------------------------------------------------------------------------------ kernels
@pytest.mark.gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("E,d,f,M", [(1, 256, 128, 1), (1, 512, 384, 16), (2, 256, 256, 17), (1, 768, 640, 33), (3, 256, 128, 70), (2, 512, 1408, 200), (1, 2048, 128, 5), (1, 256, 2176, 130)])
def test_ffn(lib, E, d, f, M, group, zeros):
    rng = np.random.default_rng(M)
    S = 3
    off = offsets_of(rng.multinomial(M, np.full(S * E, 1.0 / (S * E))))
    x, w = activations(M, d, M), weights(E, d, f, group, zeros, M + d)
    y = run(lib, x, off, S, E, w)
    check(y, x, off, E, w)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,S,E", [([0, 3, 0, 0], 2, 2), ([1] * 40, 40, 1), ([500, 0, 1, 63], 1, 4), ([0] * 299 + [9], 300, 1), ([64, 65, 63, 128, 129, 127], 2, 3), ([256], 1, 1), ([1000, 3], 1, 2)])
def test_ffn_ragged(lib, sizes, S, E):
    d, f = 512, 256
    off = offsets_of(sizes)
    M = int(off[-1])
    x, w = activations(M + 5, d, S), weights(E, d, f, 64, True, E)
    y = torch.full((M + 5, d), 3.0, dtype=torch.bfloat16, device=DEV)
    run(lib, x, off, S, E, w, y=y)
    check(y, x, off, E, w, kept=3.0)                                      # rows behind the last group stay as they were


@pytest.mark.gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,extra", [(9, 0), (40, 7), (333, 3)])
def test_ffn_mapped(lib, M, extra, zeros):
    rng = np.random.default_rng(M)
    E, S, d, f = 2, 4, 256, 384
    off = offsets_of(rng.multinomial(M, np.full(S * E, 1.0 / (S * E))))
    x, w = activations(M + extra, d, M), weights(E, d, f, 32, zeros, 8)
    row_map = np.concatenate([rng.permutation(M), np.full(extra, 1 << 30)]).astype(np.int32)      # entries behind the last row are not read
    gate = np.concatenate([rng.normal(size=M), np.full(extra, np.nan)]).astype(np.float32)
    y = torch.full((M + extra, d), -2.0, dtype=torch.bfloat16, device=DEV)
    run(lib, x, off, S, E, w, y=y, row_map=torch.from_numpy(row_map).to(DEV), row_gate=torch.from_numpy(gate).to(DEV))
    check(y, x, off, E, w, row_map[:M], gate[:M], kept=-2.0)
    y = run(lib, x, off, S, E, w, row_gate=torch.from_numpy(gate).to(DEV))
    check(y, x, off, E, w, None, gate[:M])


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 150])
def test_ffn_first_group_later_and_rows_alone(lib, M):
    """Offsets that start behind 0, and a row's result that does not depend on the rows it is computed with beyond the order of its sums."""
    E, d, f = 2, 512, 256
    x, w = activations(M + 9, d, 1), weights(E, d, f, 128, True, 2)
    off = np.array([4, 4 + M // 2, 4 + M], dtype=np.int32)
    y = torch.full((M + 9, d), 1.0, dtype=torch.bfloat16, device=DEV)
    run(lib, x, off, 1, E, w, y=y)
    check(y, x, off, E, w, kept=1.0)
    again = torch.full((M + 9, d), 1.0, dtype=torch.bfloat16, device=DEV)
    run(lib, x, off, 1, E, w, y=again)
    assert torch.equal(y, again)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 16, 300])
@pytest.mark.parametrize("zeros", [False, True])
def test_ffn_large_activations_stay_finite(lib, M, zeros):
    """Activations up to the largest finite ones with scales that make the result finite: no sum on the way overflows."""
    d, f = 256, 128
    w = weights(1, d, f, 128, zeros, 3)
    for n in ("gate", "up"):
        w["s_" + n] = torch.full_like(w["s_" + n], 2.0 ** -126)
    x = (torch.sign(activations(M, d, 4).float()) * 3.3e38).bfloat16()
    off = np.array([0, M], dtype=np.int32)
    y = run(lib, x, off, 1, 1, w)
    assert torch.isfinite(y.float()).all() and (y != 0).any()
    xx = x.double().numpy()
    ref, _ = ffn_w4.expert_ffn(xx, np.zeros(M, dtype=int), [unpacked(w, 0)])
    assert np.abs(y.double().cpu().numpy() - ref).max() <= 2e-2 * np.abs(ref).max()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [20, 400])
def test_ffn_rows_keep_to_themselves(lib, M):
    d, f = 256, 256
    x, w, off = activations(M, d, 6), weights(1, d, f, 64, True, 7), np.array([0, M], dtype=np.int32)
    ref = run(lib, x, off, 1, 1, w)
    x2 = x.clone()
    x2[3, 5], x2[M - 2, 0] = float("nan"), float("inf")
    y = run(lib, x2, off, 1, 1, w)
    keep = [m for m in range(M) if m not in (3, M - 2)]
    assert torch.equal(y[keep], ref[keep]) and torch.isnan(y[3].float()).all() and not torch.isfinite(y[M - 2].float()).all()


@pytest.mark.gpu
def test_ffn_malformed_offsets_and_map_stay_inside(lib):
    """Boundaries that fall, pass M or are negative, and a map that points anywhere: nothing outside y is written."""
    M, d, f, E, S = 50, 256, 128, 2, 3
    x, w = activations(M, d, 1), weights(E, d, f, 128, False, 2)
    base = torch.full((M + 40, d), 5.0, dtype=torch.bfloat16, device=DEV)
    for off in ([0, 70, 20, -5, 90, 3, 50], [-9, -3, 1000, 5, 5, 2, 1 << 30], [50, 40, 30, 20, 10, 0, 0]):
        y = base[20:20 + M]
        run(lib, x, np.array(off, dtype=np.int32), S, E, w, y=y, row_map=torch.randint(-(1 << 31), (1 << 31) - 1, (M,), dtype=torch.int32, device=DEV))
        assert (base[:20] == 5).all() and (base[20 + M:] == 5).all()


@pytest.mark.gpu
def test_refused_tensors(lib):
    d, f, E, M = 256, 128, 1, 4
    x, off, w = activations(M, d, 1).to(DEV), torch.tensor([0, M], dtype=torch.int32, device=DEV), {k: None if v is None else v.to(DEV) for k, v in weights(E, d, f, 64, True, 1).items()}
    ok = lib.moe_expert_ffn_w4_sliced(x, off, 1, E, **w)
    assert ok.shape == (M, d)
    for change in (dict(q_up=w["q_up"][:, :64]), dict(s_gate=w["s_gate"].float()), dict(s_down=w["s_gate"]), dict(z_up=None), dict(z_gate=w["z_gate"].int()), dict(q_gate=w["q_gate"].int()),
                   dict(row_map=torch.zeros(3, dtype=torch.int32, device=DEV)), dict(row_gate=torch.zeros(M, device=DEV, dtype=torch.float64)), dict(y=x[:2]),
                   dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV)), dict(s_gate=w["s_gate"][:, :3])):
        with pytest.raises(lib.MoeError):
            lib.moe_expert_ffn_w4_sliced(x, off, 1, E, **{**w, **change})
    with pytest.raises(lib.MoeError):
        lib.moe_expert_ffn_w4_sliced(x, off, 2, E, **w)
