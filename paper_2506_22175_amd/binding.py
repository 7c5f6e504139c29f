"""Thin ctypes binding of libmoe_hip.so: argument marshalling only.

Every function has the name and the argument order of its C entry point in
include/moe.h; tensors are torch tensors on the GPU (used here only as device
memory), streams are torch.cuda.Stream objects or raw integers.  A non-zero
status raises MoEError.  There is no CPU fallback: if the HIP library is not
built, importing this module's functions raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe_hip.so")

MOE_F32, MOE_BF16, MOE_E4M3 = 0, 1, 2
MOE_SOFTMAX, MOE_SIGMOID = 0, 1
MOE_ACT_NONE, MOE_ACT_GELU, MOE_ACT_SILU = 0, 1, 2
MOE_REUSE_NONE, MOE_REUSE_BUFFERS, MOE_REUSE_RECOMPUTE = 0, 1, 2
MOE_REUSE_S1, MOE_REUSE_S2, MOE_REUSE_S3 = 3, 4, 5

EXPORTS = [
    "moe_capacity", "moe_workspace_bytes", "moe_route", "moe_assign_slots", "moe_assign_slots_static", "moe_slot_scratch_bytes",
    "moe_dispatch", "moe_expert_ffn_fwd", "moe_expert_ffn_bwd", "moe_dw_parts", "moe_combine",
    "moe_slot_rows", "moe_expert_ffn_fwd_gather",
    "moe_gate_bwd", "moe_gate_scratch_bytes", "moe_gate_weight_grad", "moe_dispatch_bwd", "moe_layer_step",
    "moe_layer_forward", "moe_layer_backward", "moe_launch_counts", "moe_status_string",
    "moe_last_error", "moe_profile_enable", "moe_profile_read",
    "moe_gran_create", "moe_gran_destroy", "moe_gran_lookup", "moe_gran_record", "moe_gran_ranges",
    "moe_search_best_gran", "moe_gran_get", "moe_strategy_cost", "moe_select_strategy",
    "moe_offload_bytes", "moe_layer_step_offload", "moe_layer_streams",
    "moe_gemm_tile",
    "moe_norm_fwd", "moe_norm_bwd", "moe_norm_scratch_bytes", "moe_router_fwd", "moe_router_bwd",
    "moe_w4_product", "moe_w4_scratch_bytes", "moe_w4_quantize",
    "moe_few_forward", "moe_few_scratch_bytes", "moe_linear_fwd", "moe_act_bwd", "moe_linear_bwd", "moe_linear_scratch_bytes",
    "moe_linear_tile",
    "moe_grad_bytes", "moe_grad_table", "moe_grad_norm", "moe_grad_scale", "moe_grad_clip",
]


# Calls that take nothing but pointers (the configuration's and the stream's among them): they are handed over as numbers,
# a microsecond less per call than as objects, and a decoding step makes these calls one after the other.
_POINTERS = {"moe_norm_fwd": 9, "moe_norm_bwd": 10, "moe_router_fwd": 7, "moe_router_bwd": 6, "moe_w4_product": 10,
             "moe_few_forward": 13, "moe_linear_fwd": 9, "moe_act_bwd": 7, "moe_linear_bwd": 9, "moe_grad_norm": 4}


class MoEError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = lib().moe_last_error().decode() if status == 5 else ""
        super().__init__(f"{where}: status {status} ({status_string(status)}) {detail}")


class MoEConfig(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("M", ctypes.c_int32), ("H", ctypes.c_int32), ("E", ctypes.c_int32),
                ("k", ctypes.c_int32), ("capacity_factor", ctypes.c_float), ("n_partitions", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("reuse", ctypes.c_int32), ("grad_overwrite", ctypes.c_int32), ("gate_renormalize", ctypes.c_int32),
                ("fuse_gather", ctypes.c_int32), ("wgrad_group", ctypes.c_int32), ("gemm_free_cus", ctypes.c_int32),
                ("fuse_combine", ctypes.c_int32)]


def make_config(T, M, H, E, k, capacity_factor, n_partitions=1, dtype=MOE_BF16, reuse=MOE_REUSE_NONE,
                grad_overwrite=0, gate_renormalize=0, fuse_gather=0, wgrad_group=0, gemm_free_cus=0, fuse_combine=0) -> MoEConfig:
    return MoEConfig(int(T), int(M), int(H), int(E), int(k), float(capacity_factor), int(n_partitions),
                     int(dtype), int(reuse), int(grad_overwrite), int(gate_renormalize), int(fuse_gather),
                     int(wgrad_group), int(gemm_free_cus), int(fuse_combine))


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2506_22175_amd.build` "
                               "(there is no fallback path)")
        _lib = ctypes.CDLL(LIB_PATH)
        for name in EXPORTS:
            fn = getattr(_lib, name)
            fn.restype = ctypes.c_char_p if name in ("moe_status_string", "moe_last_error") else ctypes.c_int
        for name, pointers in _POINTERS.items():
            getattr(_lib, name).argtypes = [ctypes.c_void_p] * pointers
    return _lib


def status_string(status: int) -> str:
    return lib().moe_status_string(ctypes.c_int(status)).decode()


def _p(t) -> ctypes.c_void_p:
    """Device (or host) pointer of a tensor, an int, or None."""
    if t is None:
        return ctypes.c_void_p(0)
    if isinstance(t, int):
        return ctypes.c_void_p(t)
    return ctypes.c_void_p(t.data_ptr())


def _s(stream) -> ctypes.c_void_p:
    return ctypes.c_void_p(_h(stream))


_now = None      # once torch uses the GPU: what gives the current stream's handle, and the current device


def _h(stream):
    """Handle of a stream, an int, or the current stream's."""
    global _now
    if stream is None:
        if _now is not None:                # the handle alone: a Stream object takes 2.8 us to make, more than many a kernel
            return _now[0](_now[1]())
        import torch
        stream = torch.cuda.current_stream()
        if torch.cuda.is_initialized():
            _now = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    return stream if isinstance(stream, int) else stream.cuda_stream


def _a(t):
    """Address of a tensor's first element, an int, or None."""
    return t if t is None or isinstance(t, int) else t.data_ptr()


def _check(status: int, where: str):
    if status != 0:
        raise MoEError(status, where)


def _cfg(cfg: MoEConfig):
    return ctypes.byref(cfg)


# ---- host-only queries -----------------------------------------------------------

def moe_capacity(cfg: MoEConfig) -> int:
    out = ctypes.c_int32(0)
    _check(lib().moe_capacity(_cfg(cfg), ctypes.byref(out)), "moe_capacity")
    return out.value


def moe_workspace_bytes(cfg: MoEConfig):
    """(total, saved, temp, routing) bytes."""
    v = [ctypes.c_size_t(0) for _ in range(4)]
    _check(lib().moe_workspace_bytes(_cfg(cfg), *[ctypes.byref(x) for x in v]), "moe_workspace_bytes")
    return tuple(x.value for x in v)


def moe_slot_scratch_bytes(cfg: MoEConfig) -> int:
    v = ctypes.c_size_t(0)
    _check(lib().moe_slot_scratch_bytes(_cfg(cfg), ctypes.byref(v)), "moe_slot_scratch_bytes")
    return v.value


def moe_gate_scratch_bytes(cfg: MoEConfig) -> int:
    v = ctypes.c_size_t(0)
    _check(lib().moe_gate_scratch_bytes(_cfg(cfg), ctypes.byref(v)), "moe_gate_scratch_bytes")
    return v.value


def moe_dw_parts(cfg: MoEConfig) -> int:
    v = ctypes.c_int32(0)
    _check(lib().moe_dw_parts(_cfg(cfg), ctypes.byref(v)), "moe_dw_parts")
    return v.value


def moe_layer_streams(cfg: MoEConfig) -> int:
    v = ctypes.c_int32(0)
    _check(lib().moe_layer_streams(_cfg(cfg), ctypes.byref(v)), "moe_layer_streams")
    return v.value


GEMMS = ("first", "second", "recompute", "dgelu", "dgrad", "dW2", "dW1")


def moe_gemm_tile(cfg: MoEConfig, part: int, gemm: str):
    """(rows, columns) of the output tiles of one of GEMMS for partition `part`."""
    r, c = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().moe_gemm_tile(_cfg(cfg), ctypes.c_int32(part), ctypes.c_int32(GEMMS.index(gemm)), ctypes.byref(r),
                               ctypes.byref(c)), "moe_gemm_tile")
    return r.value, c.value


def moe_launch_counts(reset: bool = False):
    arr = (ctypes.c_int64 * 3)()
    _check(lib().moe_launch_counts(arr, ctypes.c_int32(1 if reset else 0)), "moe_launch_counts")
    return tuple(arr)


PROFILE_KINDS = ["gemm_fwd1_gelu", "gemm_nn_store", "gemm_dgelu", "gemm_dgrad", "gemm_wgrad", "dispatch",
                 "combine", "dispatch_bwd", "route", "slots", "gate_bwd", "norm", "norm_bwd", "router", "router_bwd", "w4",
                 "few", "linear", "act_bwd", "grads"]


def moe_profile_enable(on: bool):
    _check(lib().moe_profile_enable(ctypes.c_int32(1 if on else 0)), "moe_profile_enable")


def moe_profile_read():
    """{kind: (launches, total_ms)} of the kernels timed since moe_profile_enable(True)."""
    n = len(PROFILE_KINDS)
    launches = (ctypes.c_int64 * n)()
    ms = (ctypes.c_double * n)()
    _check(lib().moe_profile_read(ctypes.c_int32(n), launches, ms), "moe_profile_read")
    return {PROFILE_KINDS[i]: (int(launches[i]), float(ms[i])) for i in range(n)}


# ---- device calls ----------------------------------------------------------------

def moe_route(cfg, x, Wg, gate_bias, logits, topk_idx, topk_w, stream=None):
    _check(lib().moe_route(_cfg(cfg), _p(x), _p(Wg), _p(gate_bias), _p(logits), _p(topk_idx), _p(topk_w),
                           _s(stream)), "moe_route")


def moe_assign_slots(cfg, topk_idx, topk_w, slot, counts, slot_w, scratch, stream=None):
    _check(lib().moe_assign_slots(_cfg(cfg), _p(topk_idx), _p(topk_w), _p(slot), _p(counts), _p(slot_w),
                                  _p(scratch), _s(stream)), "moe_assign_slots")


def moe_assign_slots_static(cfg, topk_idx, topk_w, slot, counts, slot_w, stream=None):
    _check(lib().moe_assign_slots_static(_cfg(cfg), _p(topk_idx), _p(topk_w), _p(slot), _p(counts), _p(slot_w),
                                         _s(stream)), "moe_assign_slots_static")


def moe_dispatch(cfg, part, src, slot, DI, dO_saved=None, dw=None, stream=None):
    _check(lib().moe_dispatch(_cfg(cfg), ctypes.c_int32(part), _p(src), _p(slot), _p(DI), _p(dO_saved), _p(dw),
                              _s(stream)), "moe_dispatch")


def moe_slot_rows(cfg, slot, rows, stream=None):
    _check(lib().moe_slot_rows(_cfg(cfg), _p(slot), _p(rows), _s(stream)), "moe_slot_rows")


def moe_expert_ffn_fwd_gather(cfg, part, x, rows, counts, W1, W2, Z, A, DO, stream=None):
    _check(lib().moe_expert_ffn_fwd_gather(_cfg(cfg), ctypes.c_int32(part), _p(x), _p(rows), _p(counts), _p(W1),
                                           _p(W2), _p(Z), _p(A), _p(DO), _s(stream)), "moe_expert_ffn_fwd_gather")


def moe_expert_ffn_fwd(cfg, part, DI, counts, W1, W2, Z, A, DO, stream=None):
    _check(lib().moe_expert_ffn_fwd(_cfg(cfg), ctypes.c_int32(part), _p(DI), _p(counts), _p(W1), _p(W2),
                                    _p(Z), _p(A), _p(DO), _s(stream)), "moe_expert_ffn_fwd")


def moe_expert_ffn_bwd(cfg, part, recompute, DI, Z, dDO, counts, slot_w, W1, W2, dZ, dDI, dW1, dW2, dw_part,
                       stream=None):
    _check(lib().moe_expert_ffn_bwd(_cfg(cfg), ctypes.c_int32(part), ctypes.c_int32(int(recompute)), _p(DI),
                                    _p(Z), _p(dDO), _p(counts), _p(slot_w), _p(W1), _p(W2), _p(dZ), _p(dDI),
                                    _p(dW1), _p(dW2), _p(dw_part), _s(stream)), "moe_expert_ffn_bwd")


def moe_combine(cfg, part, DO, slot, topk_w, y, stream=None):
    _check(lib().moe_combine(_cfg(cfg), ctypes.c_int32(part), _p(DO), _p(slot), _p(topk_w), _p(y), _s(stream)),
           "moe_combine")


def moe_gate_bwd(cfg, part, x, logits, topk_idx, slot, dw, dw_part, dL, dWg, scratch, stream=None):
    _check(lib().moe_gate_bwd(_cfg(cfg), ctypes.c_int32(part), _p(x), _p(logits), _p(topk_idx), _p(slot),
                              _p(dw), _p(dw_part), _p(dL), _p(dWg), _p(scratch), _s(stream)), "moe_gate_bwd")


def moe_gate_weight_grad(cfg, part, x, dL, dWg, scratch, stream=None):
    _check(lib().moe_gate_weight_grad(_cfg(cfg), ctypes.c_int32(part), _p(x), _p(dL), _p(dWg), _p(scratch), _s(stream)),
           "moe_gate_weight_grad")


def moe_dispatch_bwd(cfg, part, dDI, slot, dL, Wg, dx, stream=None):
    _check(lib().moe_dispatch_bwd(_cfg(cfg), ctypes.c_int32(part), _p(dDI), _p(slot), _p(dL), _p(Wg), _p(dx),
                                  _s(stream)), "moe_dispatch_bwd")


def _streams(streams: Optional[Sequence]):
    import torch
    if streams is None:
        cur = torch.cuda.current_stream()
        streams = [cur, cur]
    arr = (ctypes.c_void_p * len(streams))(*[_s(s).value for s in streams])
    return arr, ctypes.c_int32(len(streams))


def moe_layer_step(cfg, x, dy, Wg, gate_bias, W1, W2, y, dx, dWg, dW1, dW2, logits, topk_idx, topk_w, slot,
                   counts, workspace, streams=None):
    arr, n = _streams(streams)
    _check(lib().moe_layer_step(_cfg(cfg), _p(x), _p(dy), _p(Wg), _p(gate_bias), _p(W1), _p(W2), _p(y), _p(dx),
                                _p(dWg), _p(dW1), _p(dW2), _p(logits), _p(topk_idx), _p(topk_w), _p(slot),
                                _p(counts), _p(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                arr, n), "moe_layer_step")


def moe_layer_forward(cfg, x, Wg, gate_bias, W1, W2, y, logits, topk_idx, topk_w, slot, counts, workspace,
                      streams=None):
    arr, n = _streams(streams)
    _check(lib().moe_layer_forward(_cfg(cfg), _p(x), _p(Wg), _p(gate_bias), _p(W1), _p(W2), _p(y), _p(logits),
                                   _p(topk_idx), _p(topk_w), _p(slot), _p(counts), _p(workspace),
                                   ctypes.c_size_t(workspace.numel() * workspace.element_size()), arr, n),
           "moe_layer_forward")


def moe_layer_backward(cfg, x, dy, Wg, W1, W2, dx, dWg, dW1, dW2, logits, topk_idx, topk_w, slot, counts,
                       workspace, streams=None):
    arr, n = _streams(streams)
    _check(lib().moe_layer_backward(_cfg(cfg), _p(x), _p(dy), _p(Wg), _p(W1), _p(W2), _p(dx), _p(dWg), _p(dW1),
                                    _p(dW2), _p(logits), _p(topk_idx), _p(topk_w), _p(slot), _p(counts),
                                    _p(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                    arr, n), "moe_layer_backward")


# ---- adaptive pipeline granularity ---------------------------------------------------

class GranHandle:
    """Owner of a moe_gran handle (the table and the range set of the granularity search)."""

    def __init__(self):
        self._h = ctypes.c_void_p(0)
        _check(lib().moe_gran_create(ctypes.byref(self._h)), "moe_gran_create")

    def close(self):
        if self._h:
            lib().moe_gran_destroy(self._h)
            self._h = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def moe_gran_lookup(g: GranHandle, B: int) -> int:
    n = ctypes.c_int32(0)
    _check(lib().moe_gran_lookup(g._h, ctypes.c_int64(B), ctypes.byref(n)), "moe_gran_lookup")
    return n.value


def moe_gran_record(g: GranHandle, B: int, n: int):
    _check(lib().moe_gran_record(g._h, ctypes.c_int64(B), ctypes.c_int32(n)), "moe_gran_record")


def moe_gran_ranges(g: GranHandle):
    """[(lower, upper, n), ...] ordered by lower bound."""
    count = ctypes.c_int32(0)
    _check(lib().moe_gran_ranges(g._h, ctypes.c_int32(0), None, None, None, ctypes.byref(count)), "moe_gran_ranges")
    c = count.value
    lo, up, nn = (ctypes.c_int64 * max(c, 1))(), (ctypes.c_int64 * max(c, 1))(), (ctypes.c_int32 * max(c, 1))()
    _check(lib().moe_gran_ranges(g._h, ctypes.c_int32(c), lo, up, nn, ctypes.byref(count)), "moe_gran_ranges")
    return [(int(lo[i]), int(up[i]), int(nn[i])) for i in range(c)]


def _layer_args(cfg, x, dy, Wg, gate_bias, W1, W2, y, dx, dWg, dW1, dW2, logits, topk_idx, topk_w, slot, counts,
                workspace, streams):
    arr, n = _streams(streams)
    return (_cfg(cfg), _p(x), _p(dy), _p(Wg), _p(gate_bias), _p(W1), _p(W2), _p(y), _p(dx), _p(dWg), _p(dW1),
            _p(dW2), _p(logits), _p(topk_idx), _p(topk_w), _p(slot), _p(counts), _p(workspace),
            ctypes.c_size_t(workspace.numel() * workspace.element_size()), arr, n), arr


def moe_search_best_gran(cfg, x, dy, Wg, gate_bias, W1, W2, y, dx, dWg, dW1, dW2, logits, topk_idx, topk_w, slot,
                         counts, workspace, streams, candidates, warmup=1, iters=3):
    """(best n, [ms per step per candidate, -1 = skipped])."""
    args, keep = _layer_args(cfg, x, dy, Wg, gate_bias, W1, W2, y, dx, dWg, dW1, dW2, logits, topk_idx, topk_w,
                             slot, counts, workspace, streams)
    cand = (ctypes.c_int32 * len(candidates))(*candidates)
    ms = (ctypes.c_float * len(candidates))()
    best = ctypes.c_int32(0)
    _check(lib().moe_search_best_gran(*args, cand, ctypes.c_int32(len(candidates)), ctypes.c_int32(warmup),
                                      ctypes.c_int32(iters), ctypes.byref(best), ms), "moe_search_best_gran")
    return best.value, [float(v) for v in ms]


def moe_gran_get(g: GranHandle, cfg, x, dy, Wg, gate_bias, W1, W2, y, dx, dWg, dW1, dW2, logits, topk_idx, topk_w,
                 slot, counts, workspace, streams, candidates, warmup=1, iters=3):
    """(n, searched) for B = cfg.T."""
    args, keep = _layer_args(cfg, x, dy, Wg, gate_bias, W1, W2, y, dx, dWg, dW1, dW2, logits, topk_idx, topk_w,
                             slot, counts, workspace, streams)
    cand = (ctypes.c_int32 * len(candidates))(*candidates)
    n = ctypes.c_int32(0)
    searched = ctypes.c_int32(0)
    _check(lib().moe_gran_get(g._h, *args, cand, ctypes.c_int32(len(candidates)), ctypes.c_int32(warmup),
                              ctypes.c_int32(iters), ctypes.byref(n), ctypes.byref(searched)), "moe_gran_get")
    return n.value, bool(searched.value)


# ---- performance model of the reuse strategies -----------------------------------------

class MoESpeeds(ctypes.Structure):
    _fields_ = [("W_comp", ctypes.c_double), ("W_comm", ctypes.c_double), ("W_mem", ctypes.c_double),
                ("sigma", ctypes.c_double), ("mu_comp", ctypes.c_double), ("mu_all", ctypes.c_double),
                ("eta_all", ctypes.c_double)]


STRATEGIES = ("none", "S1", "S2", "S3", "S4")


def moe_strategy_cost(strategy: int, b: int, M: int, H: int, speeds: MoESpeeds):
    """(forward, backward) seconds per micro-batch."""
    fw, bw = ctypes.c_double(0), ctypes.c_double(0)
    _check(lib().moe_strategy_cost(ctypes.c_int32(strategy), ctypes.c_int64(b), ctypes.c_int64(M), ctypes.c_int64(H),
                                   ctypes.byref(speeds), ctypes.byref(fw), ctypes.byref(bw)), "moe_strategy_cost")
    return fw.value, bw.value


def moe_select_strategy(allowed_mask: int, b: int, M: int, H: int, speeds: MoESpeeds):
    """(strategy number, forward + backward seconds)."""
    best, cost = ctypes.c_int32(0), ctypes.c_double(0)
    _check(lib().moe_select_strategy(ctypes.c_uint32(allowed_mask), ctypes.c_int64(b), ctypes.c_int64(M),
                                     ctypes.c_int64(H), ctypes.byref(speeds), ctypes.byref(best), ctypes.byref(cost)),
           "moe_select_strategy")
    return best.value, cost.value


# ---- offloading strategies ---------------------------------------------------------------

def moe_offload_bytes(cfg: MoEConfig) -> int:
    v = ctypes.c_size_t(0)
    _check(lib().moe_offload_bytes(_cfg(cfg), ctypes.byref(v)), "moe_offload_bytes")
    return v.value


def moe_layer_step_offload(cfg, x, dy, Wg, gate_bias, W1, W2, y, dx, dWg, dW1, dW2, logits, topk_idx, topk_w, slot,
                           counts, workspace, host_buffer, streams):
    """host_buffer: pinned host tensor (uint8); streams: three streams."""
    arr, n = _streams(streams)
    _check(lib().moe_layer_step_offload(_cfg(cfg), _p(x), _p(dy), _p(Wg), _p(gate_bias), _p(W1), _p(W2), _p(y),
                                        _p(dx), _p(dWg), _p(dW1), _p(dW2), _p(logits), _p(topk_idx), _p(topk_w),
                                        _p(slot), _p(counts), _p(workspace),
                                        ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                        _p(host_buffer), ctypes.c_size_t(host_buffer.numel() * host_buffer.element_size()),
                                        arr, n), "moe_layer_step_offload")


# ---- the operators around the layer --------------------------------------------------------

class MoENormConfig(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("M", ctypes.c_int32), ("eps", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("out", ctypes.c_int32), ("group", ctypes.c_int32), ("grad_overwrite", ctypes.c_int32),
                ("ldx", ctypes.c_int64), ("ldr", ctypes.c_int64), ("ldh", ctypes.c_int64), ("ldy", ctypes.c_int64)]


def make_norm_config(T, M, eps=1e-6, dtype=MOE_BF16, out=None, group=0, grad_overwrite=0, ldx=0, ldr=0, ldh=0,
                     ldy=0) -> MoENormConfig:
    return MoENormConfig(int(T), int(M), float(eps), int(dtype), int(dtype if out is None else out), int(group),
                         int(grad_overwrite), int(ldx), int(ldr), int(ldh), int(ldy))


def moe_norm_scratch_bytes(cfg: MoENormConfig) -> int:
    v = ctypes.c_size_t(0)
    _check(lib().moe_norm_scratch_bytes(_cfg(cfg), ctypes.byref(v)), "moe_norm_scratch_bytes")
    return v.value


def moe_norm_fwd(cfg, x, residual, gain, h, y, scales=None, rstd=None, stream=None):
    _check(lib().moe_norm_fwd(_cfg(cfg), _a(x), _a(residual), _a(gain), _a(h), _a(y), _a(scales), _a(rstd),
                              _h(stream)), "moe_norm_fwd")


def moe_norm_bwd(cfg, dy, h, gain, rstd, dh, dx, dgain, scratch, stream=None):
    _check(lib().moe_norm_bwd(_cfg(cfg), _a(dy), _a(h), _a(gain), _a(rstd), _a(dh), _a(dx), _a(dgain), _a(scratch),
                              _h(stream)), "moe_norm_bwd")


class MoERouterConfig(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("E", ctypes.c_int32), ("k", ctypes.c_int32), ("scores", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("group_k", ctypes.c_int32), ("group_top", ctypes.c_int32),
                ("renormalize", ctypes.c_int32), ("scale", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("ld", ctypes.c_int64)]


def make_router_config(T, E, k, scores=MOE_SOFTMAX, groups=1, group_k=1, group_top=2, renormalize=0, scale=1.0,
                       dtype=MOE_F32, ld=0) -> MoERouterConfig:
    return MoERouterConfig(int(T), int(E), int(k), int(scores), int(groups), int(group_k), int(group_top),
                           int(renormalize), float(scale), int(dtype), int(ld))


def moe_router_fwd(cfg, logits, bias, topk_idx, topk_w, load=None, stream=None):
    _check(lib().moe_router_fwd(_cfg(cfg), _a(logits), _a(bias), _a(topk_idx), _a(topk_w), _a(load), _h(stream)),
           "moe_router_fwd")


def moe_router_bwd(cfg, logits, topk_idx, dw, dlogits, stream=None):
    _check(lib().moe_router_bwd(_cfg(cfg), _a(logits), _a(topk_idx), _a(dw), _a(dlogits), _h(stream)), "moe_router_bwd")


class MoEW4Config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("k", ctypes.c_int32), ("E", ctypes.c_int32), ("K", ctypes.c_int32),
                ("N", ctypes.c_int32), ("dtype", ctypes.c_int32), ("out", ctypes.c_int32), ("group", ctypes.c_int32),
                ("per_choice", ctypes.c_int32), ("combine", ctypes.c_int32), ("gelu", ctypes.c_int32),
                ("ldx", ctypes.c_int64), ("ldy", ctypes.c_int64)]


def make_w4_config(T, k, E, K, N, dtype=MOE_BF16, out=MOE_BF16, group=0, per_choice=0, combine=0, gelu=0, ldx=0,
                   ldy=0) -> MoEW4Config:
    return MoEW4Config(int(T), int(k), int(E), int(K), int(N), int(dtype), int(out), int(group), int(per_choice),
                       int(combine), int(gelu), int(ldx), int(ldy))


def moe_w4_scratch_bytes(cfg: MoEW4Config) -> int:
    v = ctypes.c_size_t(0)
    _check(lib().moe_w4_scratch_bytes(_cfg(cfg), ctypes.byref(v)), "moe_w4_scratch_bytes")
    return v.value


def moe_w4_product(cfg, x, x_scales, topk_idx, topk_w, Wq, Ws, y, scratch=None, stream=None):
    _check(lib().moe_w4_product(_cfg(cfg), _a(x), _a(x_scales), _a(topk_idx), _a(topk_w), _a(Wq), _a(Ws), _a(y),
                                _a(scratch), _h(stream)), "moe_w4_product")


def moe_w4_quantize(E, K, N, dtype, W, Wq, Ws, stream=None):
    _check(lib().moe_w4_quantize(ctypes.c_int32(E), ctypes.c_int32(K), ctypes.c_int32(N), ctypes.c_int32(dtype), _p(W),
                                 _p(Wq), _p(Ws), _s(stream)), "moe_w4_quantize")


# ---- more operators around the layer ---------------------------------------------------------

class MoEFewConfig(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("M", ctypes.c_int32), ("H", ctypes.c_int32), ("E", ctypes.c_int32),
                ("k", ctypes.c_int32), ("scores", ctypes.c_int32), ("groups", ctypes.c_int32), ("group_k", ctypes.c_int32),
                ("group_top", ctypes.c_int32), ("renormalize", ctypes.c_int32), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("ldx", ctypes.c_int64), ("ldy", ctypes.c_int64)]


def make_few_config(T, M, H, E, k, dtype=MOE_BF16, scores=MOE_SOFTMAX, groups=1, group_k=1, group_top=2, renormalize=0,
                    scale=1.0, ldx=0, ldy=0) -> MoEFewConfig:
    return MoEFewConfig(int(T), int(M), int(H), int(E), int(k), int(scores), int(groups), int(group_k), int(group_top),
                        int(renormalize), float(scale), int(dtype), int(ldx), int(ldy))


def moe_few_scratch_bytes(cfg: MoEFewConfig) -> int:
    v = ctypes.c_size_t(0)
    _check(lib().moe_few_scratch_bytes(_cfg(cfg), ctypes.byref(v)), "moe_few_scratch_bytes")
    return v.value


def moe_few_forward(cfg, x, Wg, gate_bias, bias, W1, W2, y, logits, topk_idx, topk_w, scratch, stream=None):
    _check(lib().moe_few_forward(_cfg(cfg), _a(x), _a(Wg), _a(gate_bias), _a(bias), _a(W1), _a(W2), _a(y), _a(logits),
                                 _a(topk_idx), _a(topk_w), _a(scratch), _h(stream)), "moe_few_forward")


class MoELinearConfig(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("K", ctypes.c_int32), ("N", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("act", ctypes.c_int32), ("grad_overwrite", ctypes.c_int32), ("ldx", ctypes.c_int64), ("ldy", ctypes.c_int64),
                ("ldr", ctypes.c_int64), ("ldz", ctypes.c_int64)]


def make_linear_config(T, K, N, dtype=MOE_BF16, act=MOE_ACT_NONE, grad_overwrite=0, ldx=0, ldy=0, ldr=0, ldz=0) -> MoELinearConfig:
    return MoELinearConfig(int(T), int(K), int(N), int(dtype), int(act), int(grad_overwrite), int(ldx), int(ldy), int(ldr),
                           int(ldz))


def moe_linear_scratch_bytes(cfg: MoELinearConfig) -> int:
    v = ctypes.c_size_t(0)
    _check(lib().moe_linear_scratch_bytes(_cfg(cfg), ctypes.byref(v)), "moe_linear_scratch_bytes")
    return v.value


def moe_linear_fwd(cfg, x, W, bias, residual, z, y, scratch, stream=None):
    _check(lib().moe_linear_fwd(_cfg(cfg), _a(x), _a(W), _a(bias), _a(residual), _a(z), _a(y), _a(scratch), _h(stream)),
           "moe_linear_fwd")


def moe_act_bwd(cfg, dy, z, dz, dbias, scratch, stream=None):
    _check(lib().moe_act_bwd(_cfg(cfg), _a(dy), _a(z), _a(dz), _a(dbias), _a(scratch), _h(stream)), "moe_act_bwd")


def moe_linear_bwd(cfg, dz, x, W, dx, dW, scratch, add=None, stream=None):
    _check(lib().moe_linear_bwd(_cfg(cfg), _a(dz), _a(x), _a(W), _a(add), _a(dx), _a(dW), _a(scratch), _h(stream)), "moe_linear_bwd")


LINEAR_GEMMS = ("fwd", "dx", "dW")


def moe_linear_tile(cfg, gemm: str):
    """(rows, columns, partial sums) of one of LINEAR_GEMMS."""
    v = [ctypes.c_int32(0) for _ in range(3)]
    _check(lib().moe_linear_tile(_cfg(cfg), ctypes.c_int32(LINEAR_GEMMS.index(gemm)), *(ctypes.byref(n) for n in v)), "moe_linear_tile")
    return tuple(n.value for n in v)


class MoEGradTensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class MoEGradList(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("chunks", ctypes.c_int64), ("tensors", ctypes.c_int32), ("outs", ctypes.c_int32)]


def moe_grad_bytes(tensors) -> tuple:
    """(table, scratch) bytes for an array of MoEGradTensor."""
    t, s = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().moe_grad_bytes(tensors, ctypes.c_int32(len(tensors)), ctypes.byref(t), ctypes.byref(s)), "moe_grad_bytes")
    return t.value, s.value


def moe_grad_table(tensors, table, stream=None) -> MoEGradList:
    out = MoEGradList()
    _check(lib().moe_grad_table(tensors, ctypes.c_int32(len(tensors)), _p(table), ctypes.byref(out), _s(stream)), "moe_grad_table")
    return out


def make_grad_list(grads, outs=None, stream=None) -> MoEGradList:
    """A list of gradient tensors (contiguous, float32 or bfloat16) with its table, which the returned object keeps alive; the
    tensors are the caller's to keep.  It takes some 5 us a tensor on the host, and a launch for every 64: a list is for gradients that stay at
    their addresses, and made once.  outs: where the clipped ones go (the gradients themselves for clipping in place), or None."""
    import torch
    code = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}
    outs = [None] * len(grads) if outs is None else outs
    if len(outs) != len(grads):
        raise ValueError(f"{len(grads)} gradients, {len(outs)} outputs")
    tensors = (MoEGradTensor * len(grads))()
    for t, g, o in zip(tensors, grads, outs):
        if g.dtype not in code or not g.is_contiguous():
            raise ValueError("gradients are contiguous tensors of float32 or bfloat16")
        if o is not None and (o.dtype != g.dtype or o.numel() != g.numel() or not o.is_contiguous() or o.device != g.device):
            raise ValueError("an output has its gradient's type, size and device, and is contiguous")
        t.grad, t.out, t.n, t.dtype = g.data_ptr(), None if o is None else o.data_ptr(), g.numel(), code[g.dtype]
    need, scratch = moe_grad_bytes(tensors)
    device = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
    if any(g.device != device for g in grads):
        raise ValueError("gradients of one list are on one device")
    with torch.cuda.device(device):
        if stream is None:
            stream = torch.cuda.current_stream()
        elif isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream)
        with torch.cuda.stream(stream):          # (memory of the stream that writes it: another's may still be in use there)
            table = torch.empty(need, dtype=torch.uint8, device=device)
            out = moe_grad_table(tensors, table, stream)
    out.memory, out.scratch = table, scratch
    return out


def moe_grad_scratch_bytes(grads: MoEGradList) -> int:
    """Of a list that make_grad_list made."""
    return grads.scratch


def moe_grad_norm(grads, norm, scratch, stream=None):
    _check(lib().moe_grad_norm(_cfg(grads), _a(norm), _a(scratch), _h(stream)), "moe_grad_norm")


def moe_grad_scale(grads, most, norm, stream=None):
    _check(lib().moe_grad_scale(_cfg(grads), ctypes.c_float(most), _p(norm), _s(stream)), "moe_grad_scale")


def moe_grad_clip(grads, most, norm, scratch, stream=None):
    _check(lib().moe_grad_clip(_cfg(grads), ctypes.c_float(most), _p(norm), _p(scratch), _s(stream)), "moe_grad_clip")
