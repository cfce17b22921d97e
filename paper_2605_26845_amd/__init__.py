"""Python binding of libmoecircuit (MI355X / gfx950).

Argument marshalling only: every step of the path runs in the HIP kernels behind the C ABI
declared in include/moe_circuit.h.  torch is used for device memory and streams.  There is no
CPU fallback: if the shared library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import glob
import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
_CSRC = os.path.join(_HERE, "csrc")
_LIB_PATH = os.path.join(_HERE, "libmoecircuit.so")
_INCLUDE = os.path.join(os.path.dirname(_HERE), "include")

MOE_DECOMP_ZERO_DIAGONAL = 1
MOE_DECOMP_RESIDUAL_I32 = 2
MOE_DECOMP_RESIDUAL_U16 = 4
MOE_DECOMP_CLEAR_TAIL = 8
MOE_W_BF16 = 0
MOE_W_FP8_E4M3_B128 = 1
MOE_MAX_RANKS = 128
MOE_T_BF16 = 0
MOE_T_F32 = 1
MOE_ROUTER_SOFTMAX = 0
MOE_ROUTER_SIGMOID = 1
MOE_ROUTER_RENORMALISE = 1
MOE_ROUTER_MAX_TOPK = 32

_STATUS = {0: "MOE_OK", -1: "MOE_ERR_INVALID_ARG", -2: "MOE_ERR_UNSUPPORTED_SHAPE", -3: "MOE_ERR_WORKSPACE",
           -4: "MOE_ERR_HIP"}

EXPORTS = [
    "moe_route_histogram", "moe_decompose_greedy", "moe_decompose_bvn", "moe_slice_table_workspace_bytes",
    "moe_slice_table", "moe_ffn_workspace_bytes", "moe_ffn_expanded_weights_bytes", "moe_expert_ffn_sliced", "moe_kernel_timing_enable",
    "moe_kernel_timing_read", "moe_kernel_timing_select", "moe_last_hip_error", "moe_makespan_model", "moe_order_matchings", "moe_decompose_sinkhorn_bvn", "moe_slice_table_rows_workspace_bytes",
    "moe_slice_table_rows", "moe_expert_ffn_sliced_mapped", "moe_ffn_tile_override",
    "moe_slice_table_static", "moe_decompose_profile", "moe_combine_topk_sum",
    "moe_ffn_backward_workspace_bytes", "moe_expert_ffn_backward_sliced", "moe_probe_mfma_bf16",
    "moe_combine_backward_workspace_bytes", "moe_combine_topk_sum_backward", "moe_router_topk", "moe_router_topk_backward",
    "moe_block_backward_workspace_bytes", "moe_block_norm", "moe_block_norm_backward", "moe_block_join", "moe_block_join_backward",
    "moe_ffn_w4_workspace_bytes", "moe_expert_ffn_w4_sliced",
]

_lib = None
_torch = None                                                             # set by load()


class MoeError(RuntimeError):
    pass


class CostModel(ctypes.Structure):
    """struct moe_cost_model of moe_circuit.h."""
    _fields_ = [("bytes_per_row", ctypes.c_double), ("bandwidth", ctypes.c_double), ("reconf_s", ctypes.c_double),
                ("kind", ctypes.c_int), ("fixed_s", ctypes.c_double), ("per_row_s", ctypes.c_double),
                ("table_rows", ctypes.POINTER(ctypes.c_double)), ("table_seconds", ctypes.POINTER(ctypes.c_double)),
                ("table_len", ctypes.c_int)]


def build(verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 into libmoecircuit.so (in-tree)."""
    srcs = sorted(glob.glob(os.path.join(_CSRC, "*.hip")))
    cmd = ["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", _INCLUDE, "-o", _LIB_PATH] + srcs
    if verbose:
        print(" ".join(cmd))
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise MoeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err)
    return _LIB_PATH


def load():
    """Load the shared library (built beforehand by build()); fails loudly if it is absent."""
    global _lib, _torch
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise MoeError("libmoecircuit.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
    # torch ships its own HIP runtime (soname libamdhip64.so.7); importing it first makes the
    # library bind to that one instead of bringing a second runtime into the process
    import torch
    _torch = torch
    L = ctypes.CDLL(_LIB_PATH)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    L.moe_route_histogram.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, vp]
    L.moe_route_histogram.restype = ci
    L.moe_decompose_greedy.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp]
    L.moe_decompose_greedy.restype = ci
    L.moe_decompose_profile.argtypes = [vp, ci]
    L.moe_decompose_profile.restype = ci
    L.moe_decompose_bvn.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp]
    L.moe_decompose_bvn.restype = ci
    L.moe_decompose_sinkhorn_bvn.argtypes = [vp, ci, ci, ci, ci, ci, ctypes.c_double, vp, vp, vp, vp, vp, vp, vp]
    L.moe_decompose_sinkhorn_bvn.restype = ci
    L.moe_slice_table_workspace_bytes.argtypes = [ci, ci, ci]
    L.moe_slice_table_workspace_bytes.restype = sz
    L.moe_slice_table.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, vp, vp, ci, vp, vp, sz, vp]
    L.moe_slice_table.restype = ci
    L.moe_slice_table_static.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, vp, vp, ci, vp, vp]
    L.moe_slice_table_static.restype = ci
    L.moe_slice_table_rows_workspace_bytes.argtypes = [ci, ci, ci]
    L.moe_slice_table_rows_workspace_bytes.restype = sz
    L.moe_slice_table_rows.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, vp, vp, ci, vp, vp, vp, vp, sz, vp]
    L.moe_slice_table_rows.restype = ci
    L.moe_expert_ffn_sliced_mapped.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.moe_expert_ffn_sliced_mapped.restype = ci
    L.moe_ffn_workspace_bytes.argtypes = [ci, ci, ci]
    L.moe_ffn_workspace_bytes.restype = sz
    L.moe_ffn_expanded_weights_bytes.argtypes = [ci, ci, ci]
    L.moe_ffn_expanded_weights_bytes.restype = sz
    L.moe_expert_ffn_sliced.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.moe_expert_ffn_sliced.restype = ci
    L.moe_ffn_backward_workspace_bytes.argtypes = [ci, ci, ci, ci]
    L.moe_ffn_backward_workspace_bytes.restype = sz
    L.moe_expert_ffn_backward_sliced.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.moe_expert_ffn_backward_sliced.restype = ci
    L.moe_combine_topk_sum.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, vp]
    L.moe_combine_topk_sum.restype = ci
    cf = ctypes.c_float
    L.moe_combine_backward_workspace_bytes.argtypes = [ci]
    L.moe_combine_backward_workspace_bytes.restype = sz
    L.moe_combine_topk_sum_backward.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, sz, vp]
    L.moe_combine_topk_sum_backward.restype = ci
    L.moe_router_topk.argtypes = [vp, ci, ci, ci, ci, ci, ci, cf, vp, vp, vp]
    L.moe_router_topk.restype = ci
    L.moe_router_topk_backward.argtypes = [vp, vp, ci, vp, ci, ci, ci, ci, ci, cf, vp, vp]
    L.moe_router_topk_backward.restype = ci
    L.moe_block_backward_workspace_bytes.argtypes = [ci, ci]
    L.moe_block_backward_workspace_bytes.restype = sz
    L.moe_block_norm.argtypes = [vp, ci, vp, cf, ci, ci, vp, vp]
    L.moe_block_norm.restype = ci
    L.moe_block_norm_backward.argtypes = [vp, vp, ci, vp, vp, cf, ci, ci, vp, vp, vp, sz, vp]
    L.moe_block_norm_backward.restype = ci
    L.moe_block_join.argtypes = [vp, vp, ci, vp, vp, vp, cf, cf, ci, ci, vp, vp, vp]
    L.moe_block_join.restype = ci
    L.moe_block_join_backward.argtypes = [vp, vp, vp, vp, ci, vp, vp, vp, cf, cf, ci, ci, vp, vp, vp, vp, vp, vp, sz, vp]
    L.moe_block_join_backward.restype = ci
    L.moe_ffn_w4_workspace_bytes.argtypes = [ci, ci, ci]
    L.moe_ffn_w4_workspace_bytes.restype = sz
    L.moe_expert_ffn_w4_sliced.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci] + [vp] * 13 + [sz, vp]
    L.moe_expert_ffn_w4_sliced.restype = ci
    L.moe_probe_mfma_bf16.argtypes = [ci, ci, ci, vp, vp]
    L.moe_probe_mfma_bf16.restype = ci
    L.moe_ffn_tile_override.argtypes = [ci, ci, ci]
    L.moe_ffn_tile_override.restype = ci
    L.moe_kernel_timing_enable.argtypes = [ci]
    L.moe_kernel_timing_enable.restype = ci
    L.moe_kernel_timing_select.argtypes = [ctypes.c_char_p]
    L.moe_kernel_timing_select.restype = ci
    L.moe_kernel_timing_read.argtypes = [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_float),
                                         ctypes.POINTER(ctypes.c_int), ci]
    L.moe_kernel_timing_read.restype = ci
    L.moe_last_hip_error.argtypes = []
    L.moe_last_hip_error.restype = ctypes.c_char_p
    L.moe_makespan_model.argtypes = [vp, ci, vp, vp, ci, vp, ctypes.POINTER(CostModel), ctypes.POINTER(ctypes.c_double)]
    L.moe_makespan_model.restype = ci
    L.moe_order_matchings.argtypes = [vp, ci, vp, vp, ci, ctypes.POINTER(CostModel), vp]
    L.moe_order_matchings.restype = ci
    _lib = L
    return L


def _check(rc: int, what: str):
    if rc != 0:
        detail = ""
        if rc == -4:
            detail = ": " + (load().moe_last_hip_error() or b"").decode()
        raise MoeError("%s -> %s%s" % (what, _STATUS.get(rc, str(rc)), detail))


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev_check(t, dtype, name):
    import torch
    if t is None:
        return
    if not t.is_cuda or not t.is_contiguous() or t.dtype != dtype:
        raise MoeError("%s must be a contiguous CUDA tensor of dtype %s" % (name, dtype))


# ---------------------------------------------------------------------------------------------
def moe_route_histogram(ids, E: int, traffic=None, expert_counts=None, want_counts: bool = True):
    """ids int32 [N][T][topk] or [L][N][T][topk] -> (traffic [..][N][N], expert_counts [..][N][E] or None)."""
    import torch
    _dev_check(ids, torch.int32, "ids")
    batched = ids.dim() == 4
    L = ids.shape[0] if batched else 1
    N, T, topk = ids.shape[-3:]
    shp = (L, N) if batched else (N,)
    if traffic is None:
        traffic = torch.empty(shp + (N,), dtype=torch.int32, device=ids.device)
    if expert_counts is None and want_counts:
        expert_counts = torch.empty(shp + (E,), dtype=torch.int32, device=ids.device)
    _dev_check(traffic, torch.int32, "traffic")
    _dev_check(expert_counts, torch.int32, "expert_counts")
    _check(load().moe_route_histogram(_ptr(ids), L, N, T, topk, E, _ptr(traffic), _ptr(expert_counts), _stream()),
           "moe_route_histogram")
    return traffic, expert_counts


def _decomp_buffers(mats, kmax, want_perms, want_residual, want_hashes, out):
    import torch
    B, N, _ = mats.shape
    dev = mats.device
    out = dict(out or {})
    # what lies behind the last matching is zero in tensors that are made here, and untouched in the caller's: the kernel clears both
    # or none (three fills were a tenth of a small layer's time)
    clear = "perms" not in out and "durations" not in out
    fresh = torch.empty if clear else torch.zeros
    if "perms" not in out:
        out["perms"] = fresh((B, kmax, N), dtype=torch.uint8, device=dev) if want_perms else None
    if "durations" not in out:
        out["durations"] = fresh((B, kmax), dtype=torch.int32, device=dev)
    if "counts" not in out:
        out["counts"] = torch.empty((B,), dtype=torch.int32, device=dev)
    if "residual" not in out:
        out["residual"] = torch.empty((B, N, N), dtype=torch.int32, device=dev) if want_residual else None
    if "hashes" not in out:
        out["hashes"] = torch.empty((B,), dtype=torch.int64, device=dev) if want_hashes else None
    return out, MOE_DECOMP_CLEAR_TAIL if clear else 0


def moe_decompose_profile(counters=None):
    """Measurement hook: counters = device int64 tensor [capacity][4] that the following greedy / BvN calls fill per
    matrix with (shader cycles, 100 MHz ticks, search steps, searches); None switches recording off."""
    import torch
    if counters is None:
        _check(load().moe_decompose_profile(None, 0), "moe_decompose_profile")
        return
    _dev_check(counters, torch.int64, "counters")
    _check(load().moe_decompose_profile(_ptr(counters), counters.numel() // 4), "moe_decompose_profile")


def moe_decompose_greedy(mats, kmax: int, zero_diag: bool = False, want_perms=True, want_residual=True,
                         want_hashes=False, out=None, residual_bits: int = 0):
    """mats int32 [B][N][N] -> dict(perms, durations, counts, residual, hashes) of device tensors.
    residual_bits: 0 = the library decides how the residual is held on chip, 32 / 16 pin it (same results)."""
    import torch
    _dev_check(mats, torch.int32, "mats")
    B, N, _ = mats.shape
    o, clear = _decomp_buffers(mats, kmax, want_perms, want_residual, want_hashes, out)
    _check(load().moe_decompose_greedy(_ptr(mats), B, N, kmax,
                                       (MOE_DECOMP_ZERO_DIAGONAL if zero_diag else 0) | clear
                                       | {0: 0, 32: MOE_DECOMP_RESIDUAL_I32, 16: MOE_DECOMP_RESIDUAL_U16}[residual_bits],
                                       _ptr(o["perms"]), _ptr(o["durations"]), _ptr(o["counts"]), _ptr(o["residual"]),
                                       _ptr(o["hashes"]), _stream()), "moe_decompose_greedy")
    return o


def moe_decompose_bvn(mats, kmax: int, zero_diag: bool = False, want_perms=True, want_residual=True,
                      want_hashes=False, out=None):
    """As moe_decompose_greedy, plus pad_total int32 [B]."""
    import torch
    _dev_check(mats, torch.int32, "mats")
    B, N, _ = mats.shape
    o, clear = _decomp_buffers(mats, kmax, want_perms, want_residual, want_hashes, out)
    if "pad_total" not in o:
        o["pad_total"] = torch.empty((B,), dtype=torch.int32, device=mats.device)
    _check(load().moe_decompose_bvn(_ptr(mats), B, N, kmax, (MOE_DECOMP_ZERO_DIAGONAL if zero_diag else 0) | clear,
                                    _ptr(o["perms"]), _ptr(o["durations"]), _ptr(o["counts"]), _ptr(o["residual"]),
                                    _ptr(o["pad_total"]), _ptr(o["hashes"]), _stream()), "moe_decompose_bvn")
    return o


def moe_decompose_sinkhorn_bvn(mats, kmax: int, zero_diag: bool = False, sweeps: int = 100, eps: float = 1e-12,
                               want_perms=True, want_scaled=True, want_residual=True):
    """mats int32 [B][N][N] -> dict(perms uint8 [B][kmax][N], coeffs float64 [B][kmax], counts, scaled, residual, deviation)."""
    import torch
    _dev_check(mats, torch.int32, "mats")
    B, N, _ = mats.shape
    dev = mats.device
    o = dict(perms=torch.zeros((B, kmax, N), dtype=torch.uint8, device=dev) if want_perms else None,
             coeffs=torch.zeros((B, kmax), dtype=torch.float64, device=dev),
             counts=torch.zeros((B,), dtype=torch.int32, device=dev),
             scaled=torch.empty((B, N, N), dtype=torch.float64, device=dev) if want_scaled else None,
             residual=torch.empty((B, N, N), dtype=torch.float64, device=dev) if want_residual else None,
             deviation=torch.zeros((B,), dtype=torch.float64, device=dev))
    _check(load().moe_decompose_sinkhorn_bvn(_ptr(mats), B, N, kmax, MOE_DECOMP_ZERO_DIAGONAL if zero_diag else 0,
                                             int(sweeps), float(eps), _ptr(o["perms"]), _ptr(o["coeffs"]), _ptr(o["counts"]),
                                             _ptr(o["scaled"]), _ptr(o["residual"]), _ptr(o["deviation"]), _stream()),
           "moe_decompose_sinkhorn_bvn")
    return o


def moe_slice_table(ids, E: int, r: int, traffic, perms, durations, count, kmax: int, offsets=None, workspace=None):
    """ids [N][T][topk], traffic [N][N], perms uint8 [kmax][N], durations [kmax], count [1] -> offsets."""
    import torch
    _dev_check(ids, torch.int32, "ids")
    _dev_check(traffic, torch.int32, "traffic")
    _dev_check(perms, torch.uint8, "perms")
    _dev_check(durations, torch.int32, "durations")
    _dev_check(count, torch.int32, "count")
    N, T, topk = ids.shape
    e_loc = E // N
    if offsets is None:
        offsets = torch.empty(((kmax + 2) * e_loc + 1,), dtype=torch.int32, device=ids.device)
    need = load().moe_slice_table_workspace_bytes(N, kmax, E)
    if workspace is None:
        workspace = torch.empty((max(need, 1),), dtype=torch.uint8, device=ids.device)
    _check(load().moe_slice_table(_ptr(ids), N, T, topk, E, r, _ptr(traffic), _ptr(perms), _ptr(durations), _ptr(count),
                                  kmax, _ptr(offsets), _ptr(workspace), workspace.numel(), _stream()), "moe_slice_table")
    return offsets


def moe_slice_table_static(ids, E: int, r: int, traffic, perms, durations, count, kmax: int, offsets):
    """moe_slice_table on the library's built-in work area; `offsets` int32 [(kmax+2)*E_loc+1] is the caller's.
    Nothing is allocated here or in the library."""
    N, T, topk = ids.shape
    _check(load().moe_slice_table_static(_ptr(ids), N, T, topk, E, r, _ptr(traffic), _ptr(perms), _ptr(durations), _ptr(count),
                                         kmax, _ptr(offsets), _stream()), "moe_slice_table_static")
    return offsets


def moe_slice_table_rows(ids, E: int, r: int, traffic, perms, durations, count, kmax: int, M: int, offsets=None,
                         want_arrival=True, want_assignment=True, workspace=None):
    """moe_slice_table plus the row map: -> (offsets, row_arrival int32 [M] or None, row_assignment int32 [M] or None);
    M = number of assignments destined to r (column sum of traffic)."""
    import torch
    _dev_check(ids, torch.int32, "ids")
    _dev_check(traffic, torch.int32, "traffic")
    _dev_check(perms, torch.uint8, "perms")
    _dev_check(durations, torch.int32, "durations")
    _dev_check(count, torch.int32, "count")
    N, T, topk = ids.shape
    e_loc = E // N
    if offsets is None:
        offsets = torch.empty(((kmax + 2) * e_loc + 1,), dtype=torch.int32, device=ids.device)
    arr = torch.full((M,), -1, dtype=torch.int32, device=ids.device) if want_arrival else None
    asg = torch.full((M,), -1, dtype=torch.int32, device=ids.device) if want_assignment else None
    need = load().moe_slice_table_rows_workspace_bytes(N, kmax, E)
    if workspace is None:
        workspace = torch.empty((max(need, 1),), dtype=torch.uint8, device=ids.device)
    _check(load().moe_slice_table_rows(_ptr(ids), N, T, topk, E, r, _ptr(traffic), _ptr(perms), _ptr(durations), _ptr(count),
                                       kmax, _ptr(offsets), _ptr(arr), _ptr(asg), _ptr(workspace), workspace.numel(),
                                       _stream()), "moe_slice_table_rows")
    return offsets, arr, asg


def moe_ffn_workspace_bytes(M: int, d: int, f: int) -> int:
    return int(load().moe_ffn_workspace_bytes(M, d, f))


def moe_ffn_expanded_weights_bytes(E_loc: int, d: int, f: int) -> int:
    """Extra workspace that lets a call with fp8 weights and many rows expand them to bf16 once."""
    return int(load().moe_ffn_expanded_weights_bytes(E_loc, d, f))


def moe_expert_ffn_sliced_mapped(x, offsets, S: int, E_loc: int, w_gate, w_up, w_down, row_map, row_gate=None,
                                 s_gate=None, s_up=None, s_down=None, y=None, workspace=None):
    """As moe_expert_ffn_sliced with x and y in arrival order: schedule row m is row row_map[m] of both, and its
    result is scaled by row_gate[m]."""
    import torch
    _dev_check(row_map, torch.int32, "row_map")
    _dev_check(row_gate, torch.float32, "row_gate")
    return moe_expert_ffn_sliced(x, offsets, S, E_loc, w_gate, w_up, w_down, s_gate, s_up, s_down, y, workspace,
                                 _row_map=row_map, _row_gate=row_gate)


def moe_expert_ffn_sliced(x, offsets, S: int, E_loc: int, w_gate, w_up, w_down, s_gate=None, s_up=None, s_down=None,
                          y=None, workspace=None, _row_map=None, _row_gate=None):
    """x bf16 [M][d]; offsets int32 [S*E_loc+1]; bf16 weights (w_gate,w_up [E_loc][f][d], w_down [E_loc][d][f]) or
    uint8 E4M3 codes with float32 block scales -> y bf16 [M][d]."""
    import torch
    _dev_check(x, torch.bfloat16, "x")
    _dev_check(offsets, torch.int32, "offsets")
    M, d = x.shape
    f = w_gate.shape[1]
    fp8 = w_gate.dtype == torch.uint8
    wdt = torch.uint8 if fp8 else torch.bfloat16
    for name, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _dev_check(w, wdt, name)
    for name, sc in (("s_gate", s_gate), ("s_up", s_up), ("s_down", s_down)):
        _dev_check(sc, torch.float32, name)
    if tuple(w_gate.shape) != (E_loc, f, d) or tuple(w_up.shape) != (E_loc, f, d) or tuple(w_down.shape) != (E_loc, d, f):
        raise MoeError("weight shapes must be w_gate/w_up [E_loc][f][d], w_down [E_loc][d][f]")
    if offsets.numel() != S * E_loc + 1:
        raise MoeError("offsets must have S*E_loc+1 entries")
    if y is None:
        y = torch.empty_like(x)
    _dev_check(y, torch.bfloat16, "y")
    need = moe_ffn_workspace_bytes(M, d, f)
    if workspace is None:
        if fp8 and M >= 2048 * E_loc:
            need += moe_ffn_expanded_weights_bytes(E_loc, d, f)
        workspace = torch.empty((max(need, 1),), dtype=torch.uint8, device=x.device)
    if _row_map is not None or _row_gate is not None:
        _check(load().moe_expert_ffn_sliced_mapped(_ptr(x), _ptr(offsets), M, S, E_loc, d, f,
                                                   MOE_W_FP8_E4M3_B128 if fp8 else MOE_W_BF16, _ptr(w_gate), _ptr(w_up),
                                                   _ptr(w_down), _ptr(s_gate), _ptr(s_up), _ptr(s_down), _ptr(_row_map),
                                                   _ptr(_row_gate), _ptr(y), _ptr(workspace), workspace.numel(), _stream()),
               "moe_expert_ffn_sliced_mapped")
        return y
    _check(load().moe_expert_ffn_sliced(_ptr(x), _ptr(offsets), M, S, E_loc, d, f,
                                        MOE_W_FP8_E4M3_B128 if fp8 else MOE_W_BF16, _ptr(w_gate), _ptr(w_up),
                                        _ptr(w_down), _ptr(s_gate), _ptr(s_up), _ptr(s_down), _ptr(y), _ptr(workspace),
                                        workspace.numel(), _stream()), "moe_expert_ffn_sliced")
    return y


def moe_expert_ffn_backward_sliced(x, dy, offsets, S: int, E_loc: int, w_gate, w_up, w_down, workspace=None):
    """x, dy bf16 [M][d]; bf16 weights -> dict(dx [M][d], dw_gate, dw_up [E_loc][f][d], dw_down [E_loc][d][f])."""
    import torch
    for name, t in (("x", x), ("dy", dy), ("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _dev_check(t, torch.bfloat16, name)
    _dev_check(offsets, torch.int32, "offsets")
    M, d = x.shape
    f = w_gate.shape[1]
    if tuple(dy.shape) != (M, d) or tuple(w_gate.shape) != (E_loc, f, d) or tuple(w_up.shape) != (E_loc, f, d) or tuple(w_down.shape) != (E_loc, d, f):
        raise MoeError("shapes must be x, dy [M][d]; w_gate, w_up [E_loc][f][d]; w_down [E_loc][d][f]")
    if offsets.numel() != S * E_loc + 1:
        raise MoeError("offsets must have S*E_loc+1 entries")
    out = dict(dx=torch.empty_like(x), dw_gate=torch.empty_like(w_gate), dw_up=torch.empty_like(w_up), dw_down=torch.empty_like(w_down))
    need = int(load().moe_ffn_backward_workspace_bytes(M, E_loc, d, f))
    if workspace is None:
        workspace = torch.empty((max(need, 1),), dtype=torch.uint8, device=x.device)
    _check(load().moe_expert_ffn_backward_sliced(_ptr(x), _ptr(dy), _ptr(offsets), M, S, E_loc, d, f, _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                                 _ptr(out["dx"]), _ptr(out["dw_gate"]), _ptr(out["dw_up"]), _ptr(out["dw_down"]),
                                                 _ptr(workspace), workspace.numel(), _stream()), "moe_expert_ffn_backward_sliced")
    return out


def moe_combine_topk_sum(y, row_of, gate=None, out=None):
    """y bf16 [R][d], row_of int32 [T][topk], gate float32 [T][topk] or None -> out bf16 [T][d]."""
    import torch
    _dev_check(y, torch.bfloat16, "y")
    _dev_check(row_of, torch.int32, "row_of")
    _dev_check(gate, torch.float32, "gate")
    R, d = y.shape
    T, topk = row_of.shape
    if gate is not None and tuple(gate.shape) != (T, topk):
        raise MoeError("gate must have the shape of row_of")
    if out is None:
        out = torch.empty((T, d), dtype=torch.bfloat16, device=y.device)
    _dev_check(out, torch.bfloat16, "out")
    _check(load().moe_combine_topk_sum(_ptr(y), _ptr(row_of), _ptr(gate), T, topk, d, R, _ptr(out), _stream()),
           "moe_combine_topk_sum")
    return out


# --------------------------------------------------------------------------------------------- around the experts
def _operands(what, wanted):
    """wanted: (name, tensor or None, dtype or allowed dtypes, shape).  All tensors contiguous, of that type and shape, and on one GPU, whose number is
    returned."""
    device = -1
    for name, t, dtype, shape in wanted:
        if t is None:
            continue
        at = t.get_device()
        if at < 0 or t.shape != shape or not t.is_contiguous() or (t.dtype is not dtype and (type(dtype) is not tuple or t.dtype not in dtype)):
            raise MoeError("%s: %s must be a contiguous CUDA tensor of dtype %s and shape %s" % (what, name, dtype, list(shape)))
        if at != device:
            if device >= 0:
                raise MoeError("%s: %s is on another device" % (what, name))
            device = at
    return device


def _on(device, what, call, *args):
    """call(*args, stream) on the current stream of `device`, which is made current for it."""
    C = _torch._C                                                          # (the operands are on a GPU: torch has set it up)
    if device == C._cuda_getDevice():
        rc = call(*args, C._cuda_getCurrentRawStream(device))
    else:
        with _torch.cuda.device(device):
            rc = call(*args, C._cuda_getCurrentRawStream(device))
    if rc:
        _check(rc, what)


def _two(t, what, name):
    if t is None or t.dim() != 2:
        raise MoeError("%s: %s must be a tensor of two dimensions" % (what, name))
    return t.shape


def _at(t):
    return None if t is None else t.data_ptr()


def _bytes(need, workspace, device_of, what):
    if workspace is None:
        return device_of.new_empty((need or 1,), dtype=_torch.uint8)
    if not workspace.is_cuda or not workspace.is_contiguous() or workspace.dtype != _torch.uint8 or workspace.get_device() != device_of.get_device():
        raise MoeError("%s: workspace must be a contiguous uint8 tensor on the device of the operands" % what)
    return workspace


def moe_block_norm(x, weight, eps: float = 1e-6, out=None):
    """x bf16 or float32 [T][d], weight float32 [d] -> out bf16 [T][d] = x / rms(x) * weight."""
    L, torch, what = load(), _torch, "moe_block_norm"
    T, d = _two(x, what, "x")
    if out is None:
        out = torch.empty_like(x, dtype=torch.bfloat16)
    dev = _operands(what, (("x", x, (torch.bfloat16, torch.float32), (T, d)), ("weight", weight, torch.float32, (d,)), ("out", out, torch.bfloat16, (T, d))))
    _on(dev, what, L.moe_block_norm, x.data_ptr(), int(x.dtype == torch.float32), _at(weight), eps, T, d, out.data_ptr())
    return out


def moe_block_norm_backward(d_out, x, weight, eps: float = 1e-6, d_stream=None, workspace=None):
    """d_out bf16 [T][d], x and d_stream (or None) bf16 or float32 [T][d], weight float32 [d] -> dict(d_x like x = d_stream + the norm's gradient, d_weight)."""
    L, torch, what = load(), _torch, "moe_block_norm_backward"
    T, d = _two(x, what, "x")
    dev = _operands(what, (("d_out", d_out, torch.bfloat16, (T, d)), ("x", x, (torch.bfloat16, torch.float32), (T, d)), ("weight", weight, torch.float32, (d,)),
                           ("d_stream", d_stream, x.dtype, (T, d))))
    o = dict(d_x=torch.empty_like(x), d_weight=torch.empty_like(weight))
    workspace = _bytes(L.moe_block_backward_workspace_bytes(T, d), workspace, x, what)
    _on(dev, what, L.moe_block_norm_backward, _at(d_out), x.data_ptr(), int(x.dtype == torch.float32), _at(weight), _at(d_stream), eps, T, d,
        o["d_x"].data_ptr(), o["d_weight"].data_ptr(), workspace.data_ptr(), workspace.numel())
    return o


def moe_block_join(z, stream, post_weight=None, gate=None, next_weight=None, scale: float = 1.0, eps: float = 1e-6, out=None, next_out=None):
    """z bf16 [T][d] (the block's result), stream bf16 or float32 [T][d], weights float32 [d], gate float32 [T] ->
    (out like stream = scale * stream + gate * norm(z), next bf16 = norm(out) or None without next_weight)."""
    L, torch, what = load(), _torch, "moe_block_join"
    T, d = _two(z, what, "z")
    _two(stream, what, "stream")
    if out is None:
        out = torch.empty_like(stream)
    if next_out is None and next_weight is not None:
        next_out = torch.empty_like(z)
    stream_types = (torch.bfloat16, torch.float32)
    dev = _operands(what, (("z", z, torch.bfloat16, (T, d)), ("stream", stream, stream_types, (T, d)), ("post_weight", post_weight, torch.float32, (d,)),
                           ("gate", gate, torch.float32, (T,)), ("next_weight", next_weight, torch.float32, (d,)), ("out", out, stream.dtype, (T, d)),
                           ("next_out", next_out, torch.bfloat16, (T, d))))
    _on(dev, what, L.moe_block_join, z.data_ptr(), stream.data_ptr(), int(stream.dtype == torch.float32), _at(post_weight), _at(gate),
        _at(next_weight), scale, eps, T, d, out.data_ptr(), _at(next_out))
    return out, next_out


def moe_block_join_backward(d_out, d_next, z, out, post_weight=None, gate=None, next_weight=None, scale: float = 1.0, eps: float = 1e-6,
                            workspace=None):
    """d_out (like out, or None), d_next (bf16, with next_weight), z bf16 and out [T][d] as the forward call took and returned them ->
    dict(d_z, d_stream, d_gate, d_post_weight, d_next_weight); the last three are None where their input is."""
    L, torch, what = load(), _torch, "moe_block_join_backward"
    T, d = _two(z, what, "z")
    stream_types = (torch.bfloat16, torch.float32)
    if out is None:
        raise MoeError("%s: out is required" % what)
    dev = _operands(what, (("d_out", d_out, out.dtype, (T, d)), ("d_next", d_next, torch.bfloat16, (T, d)), ("z", z, torch.bfloat16, (T, d)),
                           ("out", out, stream_types, (T, d)), ("post_weight", post_weight, torch.float32, (d,)), ("gate", gate, torch.float32, (T,)),
                           ("next_weight", next_weight, torch.float32, (d,))))
    like = lambda t: None if t is None else torch.empty_like(t)                              # noqa: E731
    o = dict(d_z=torch.empty_like(z), d_stream=torch.empty_like(out), d_gate=like(gate), d_post_weight=like(post_weight), d_next_weight=like(next_weight))
    workspace = _bytes(L.moe_block_backward_workspace_bytes(T, d), workspace, z, what)
    _on(dev, what, L.moe_block_join_backward, _at(d_out), _at(d_next), z.data_ptr(), out.data_ptr(), int(out.dtype == torch.float32),
        _at(post_weight), _at(gate), _at(next_weight), scale, eps, T, d, o["d_z"].data_ptr(), o["d_stream"].data_ptr(), _at(o["d_gate"]),
        _at(o["d_post_weight"]), _at(o["d_next_weight"]), workspace.data_ptr(), workspace.numel())
    return o


_SCORES = {"softmax": MOE_ROUTER_SOFTMAX, "sigmoid": MOE_ROUTER_SIGMOID}


def _score(score, what):
    if score not in _SCORES:
        raise MoeError("%s: score must be 'softmax' or 'sigmoid'" % what)
    return _SCORES[score]


def moe_router_topk(logits, topk: int, score: str = "softmax", renormalise: bool = True, scale: float = 1.0, ids=None, gates=None):
    """logits bf16 or float32 [T][E] -> (ids int32 [T][topk], gates float32 [T][topk]); -inf masks an expert, a slot without expert is (-1, 0)."""
    L, torch, what = load(), _torch, "moe_router_topk"
    T, E = _two(logits, what, "logits")
    if not 1 <= topk <= E:
        raise MoeError("%s: topk must be between 1 and the number of experts" % what)
    if ids is None:
        ids = logits.new_empty((T, topk), dtype=torch.int32)
    if gates is None:
        gates = logits.new_empty((T, topk), dtype=torch.float32)
    dev = _operands(what, (("logits", logits, (torch.bfloat16, torch.float32), (T, E)), ("ids", ids, torch.int32, (T, topk)), ("gates", gates, torch.float32, (T, topk))))
    sc = _score(score, what)
    _on(dev, what, L.moe_router_topk, logits.data_ptr(), int(logits.dtype == torch.float32), T, E, topk, sc,
        MOE_ROUTER_RENORMALISE if renormalise else 0, scale, ids.data_ptr(), gates.data_ptr())
    return ids, gates


def moe_router_topk_backward(d_gates, logits, ids, score: str = "softmax", renormalise: bool = True, scale: float = 1.0, d_logits=None):
    """d_gates float32 [T][topk], logits and ids as the forward call took and returned them -> d_logits [T][E] in the type of the logits."""
    L, torch, what = load(), _torch, "moe_router_topk_backward"
    T, E = _two(logits, what, "logits")
    topk = _two(ids, what, "ids")[1]
    if d_logits is None:
        d_logits = torch.empty_like(logits)
    dev = _operands(what, (("d_gates", d_gates, torch.float32, (T, topk)), ("logits", logits, (torch.bfloat16, torch.float32), (T, E)), ("ids", ids, torch.int32, (T, topk)),
                           ("d_logits", d_logits, logits.dtype, (T, E))))
    sc = _score(score, what)
    _on(dev, what, L.moe_router_topk_backward, d_gates.data_ptr(), logits.data_ptr(), int(logits.dtype == torch.float32), ids.data_ptr(), T,
        E, topk, sc, MOE_ROUTER_RENORMALISE if renormalise else 0, scale, d_logits.data_ptr())
    return d_logits


def moe_combine_topk_sum_backward(d_out, y, row_of, gate=None, workspace=None):
    """d_out bf16 [T][d], y bf16 [R][d], row_of int32 [T][topk], gate float32 [T][topk] or None -> dict(d_y [R][d], d_gate [T][topk] or None)."""
    L, torch, what = load(), _torch, "moe_combine_topk_sum_backward"
    T, topk = _two(row_of, what, "row_of")
    R, d = _two(y, what, "y")
    dev = _operands(what, (("d_out", d_out, torch.bfloat16, (T, d)), ("y", y, torch.bfloat16, (R, d)), ("row_of", row_of, torch.int32, (T, topk)),
                           ("gate", gate, torch.float32, (T, topk))))
    o = dict(d_y=torch.empty_like(y), d_gate=None if gate is None else torch.empty_like(gate))
    workspace = _bytes(L.moe_combine_backward_workspace_bytes(R), workspace, y, what)
    _on(dev, what, L.moe_combine_topk_sum_backward, _at(d_out), y.data_ptr(), row_of.data_ptr(), _at(gate), T, topk, d, R,
        o["d_y"].data_ptr(), _at(o["d_gate"]), workspace.data_ptr(), workspace.numel())
    return o


def moe_ffn_w4_workspace_bytes(M: int, d: int, f: int) -> int:
    return int(load().moe_ffn_w4_workspace_bytes(M, d, f))


def moe_expert_ffn_w4_sliced(x, offsets, S: int, E_loc: int, q_gate, q_up, q_down, s_gate, s_up, s_down, z_gate=None, z_up=None, z_down=None,
                             row_map=None, row_gate=None, y=None, workspace=None):
    """x bf16 [M][d]; offsets int32 [S*E_loc+1]; codes uint8 q_gate, q_up [E_loc][f][d/2], q_down [E_loc][d][f/2] (even input in the low four bits); scales bf16
    [E_loc][d/group][f] and [E_loc][f/group][d]; zero points uint8 like the scales, or None (= 8); row_map int32 [M] and row_gate float32 [M]
    (entries behind the schedule's last row are not read) -> y bf16 [M][d]."""
    L, torch, what = load(), _torch, "moe_expert_ffn_w4_sliced"
    M, d = _two(x, what, "x")
    if s_gate is None or s_gate.dim() != 3 or q_gate is None or q_gate.dim() != 3 or s_gate.shape[1] < 1:
        raise MoeError("%s: codes and scales must be tensors of three dimensions" % what)
    f, group = q_gate.shape[1], d // s_gate.shape[1]
    if group not in (32, 64, 128) or d % group or f % group:
        raise MoeError("%s: scales must be one per group of 32, 64 or 128 inputs" % what)
    if (z_gate is None) != (z_up is None) or (z_gate is None) != (z_down is None):
        raise MoeError("%s: zero points are given for all three weights or for none" % what)
    if y is None:
        y = torch.empty_like(x)
    up, down = (E_loc, d // group, f), (E_loc, f // group, d)
    dev = _operands(what, (("x", x, torch.bfloat16, (M, d)), ("offsets", offsets, torch.int32, (S * E_loc + 1,)), ("y", y, torch.bfloat16, (M, d)),
                           ("q_gate", q_gate, torch.uint8, (E_loc, f, d // 2)), ("q_up", q_up, torch.uint8, (E_loc, f, d // 2)),
                           ("q_down", q_down, torch.uint8, (E_loc, d, f // 2)), ("s_gate", s_gate, torch.bfloat16, up), ("s_up", s_up, torch.bfloat16, up),
                           ("s_down", s_down, torch.bfloat16, down), ("z_gate", z_gate, torch.uint8, up), ("z_up", z_up, torch.uint8, up),
                           ("z_down", z_down, torch.uint8, down), ("row_map", row_map, torch.int32, (M,)), ("row_gate", row_gate, torch.float32, (M,))))
    workspace = _bytes(moe_ffn_w4_workspace_bytes(M, d, f), workspace, x, what)
    _on(dev, what, L.moe_expert_ffn_w4_sliced, x.data_ptr(), offsets.data_ptr(), M, S, E_loc, d, f, group, q_gate.data_ptr(), q_up.data_ptr(),
        q_down.data_ptr(), s_gate.data_ptr(), s_up.data_ptr(), s_down.data_ptr(), _at(z_gate), _at(z_up), _at(z_down), _at(row_map), _at(row_gate),
        y.data_ptr(), workspace.data_ptr(), workspace.numel())
    return y


def moe_probe_mfma_bf16(data: int, iters: int, workgroups: int, sink=None):
    """Measurement aid: one launch of the register-only MFMA loop (workgroups * 4 * iters * 16 * 32768 flop); returns
    the sink tensor (float32 [workgroups * 256])."""
    import torch
    if sink is None:
        sink = torch.empty((int(workgroups) * 256,), dtype=torch.float32, device="cuda")
    _dev_check(sink, torch.float32, "sink")
    if sink.numel() < int(workgroups) * 256:
        raise MoeError("sink must hold workgroups * 256 floats")
    _check(load().moe_probe_mfma_bf16(int(data), int(iters), int(workgroups), _ptr(sink), _stream()), "moe_probe_mfma_bf16")
    return sink


def moe_ffn_tile_override(tile_rows: int = 0, kernels: int = 0, panel_groups: int = 0):
    """Test / measurement hook: pin the row-block height (64, 128, 256; 0 = automatic), the kernel family (1 = tiles of
    128 columns instead of 256 x 256, 2 = 256 x 256 tiles with one launch per phase) and / or the panel width of the tile walk for the following
    FFN calls of this process.  Call with no arguments to restore the defaults."""
    _check(load().moe_ffn_tile_override(int(tile_rows), int(kernels), int(panel_groups)), "moe_ffn_tile_override")


def moe_kernel_timing_enable(on: bool):
    _check(load().moe_kernel_timing_enable(1 if on else 0), "moe_kernel_timing_enable")


def moe_kernel_timing_select(kernel_name=None):
    """Time only the launches of one kernel (None = all)."""
    _check(load().moe_kernel_timing_select(None if kernel_name is None else kernel_name.encode()), "moe_kernel_timing_select")


def moe_kernel_timing_read(cap: int = 32):
    """-> {kernel name: (total_ms, launches)}; synchronises the recorded events and resets the table."""
    names = (ctypes.c_char_p * cap)()
    ms = (ctypes.c_float * cap)()
    n_l = (ctypes.c_int * cap)()
    n = load().moe_kernel_timing_read(names, ms, n_l, cap)
    if n < 0:
        _check(n, "moe_kernel_timing_read")
    return {names[i].decode(): (float(ms[i]), int(n_l[i])) for i in range(n)}


# --------------------------------------------------------------------------------------------- host-side model
def _cost_struct(bytes_per_row, bandwidth, reconf_s, model):
    """model: dict(kind="linear", fixed=..., per_row=...) or dict(kind="table", rows=[...], seconds=[...])."""
    import numpy as np
    c = CostModel()
    c.bytes_per_row, c.bandwidth, c.reconf_s = float(bytes_per_row), float(bandwidth), float(reconf_s)
    keep = []
    if model["kind"] == "linear":
        c.kind, c.fixed_s, c.per_row_s, c.table_len = 0, float(model["fixed"]), float(model["per_row"]), 0
    else:
        xs = np.ascontiguousarray(model["rows"], dtype=np.float64)
        ys = np.ascontiguousarray(model["seconds"], dtype=np.float64)
        keep = [xs, ys]
        c.kind, c.table_len = 1, len(xs)
        c.table_rows = xs.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
        c.table_seconds = ys.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
    return c, keep


def _host_schedule(traffic, perms, durations):
    import numpy as np
    A = np.ascontiguousarray(traffic, dtype=np.int32)
    P = np.ascontiguousarray(perms, dtype=np.uint8).reshape(-1, A.shape[0])
    D = np.ascontiguousarray(durations, dtype=np.int32)
    if P.shape[0] != D.shape[0]:
        raise MoeError("perms and durations disagree on the number of matchings")
    return A, P, D


def moe_makespan_model(traffic, perms, durations, bytes_per_row, bandwidth, reconf_s, model, order=None):
    """Host arrays (numpy) -> dict(sequential, overlap, ideal, comm, compute) in seconds."""
    import numpy as np
    A, P, D = _host_schedule(traffic, perms, durations)
    c, keep = _cost_struct(bytes_per_row, bandwidth, reconf_s, model)
    O = None if order is None else np.ascontiguousarray(order, dtype=np.int32)
    out = (ctypes.c_double * 5)()
    vp = ctypes.c_void_p
    _check(load().moe_makespan_model(vp(A.ctypes.data), A.shape[0], vp(P.ctypes.data), vp(D.ctypes.data), P.shape[0],
                                     None if O is None else vp(O.ctypes.data), ctypes.byref(c), out), "moe_makespan_model")
    del keep
    return dict(zip(("sequential", "overlap", "ideal", "comm", "compute"), [float(v) for v in out]))


def moe_order_matchings(traffic, perms, durations, bytes_per_row, bandwidth, reconf_s, model):
    """Host arrays (numpy) -> int32 [K] play order by Johnson's rule."""
    import numpy as np
    A, P, D = _host_schedule(traffic, perms, durations)
    c, keep = _cost_struct(bytes_per_row, bandwidth, reconf_s, model)
    order = np.zeros((P.shape[0],), dtype=np.int32)
    vp = ctypes.c_void_p
    _check(load().moe_order_matchings(vp(A.ctypes.data), A.shape[0], vp(P.ctypes.data), vp(D.ctypes.data), P.shape[0],
                                      ctypes.byref(c), vp(order.ctypes.data)), "moe_order_matchings")
    del keep
    return order
