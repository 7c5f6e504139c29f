"""A whole feed-forward block of a model around the expert layer, from the calls of include/moe.h: the residual's addition and
the norm, the gate's logits, the router, the experts, the weighted sum; and the same block serving, its experts in 4 bits.

    h = x + residual;  y = h / sqrt(mean(h^2) + eps) * gain;  logits = y Wg;  idx, w = router(logits, bias)
    out[t] = sum over j of w[t,j] * gelu(y[t] W1[idx[t,j]]) W2[idx[t,j]]  [+ gelu(y[t] V1 + b1) V2 + b2]

out and h are what the next block adds up; V1, b1, V2, b2 are a shared expert that every token goes through, if there is one.
Training (`Block`) has a capacity per expert and drops what is beyond, and ends with the gradients clipped by their norm; serving
drops nothing: from 4-bit weights (`Served`), or a few tokens at a time from the trained weights as they are (`Few`).  All buffers are
made once, so that each pass may be captured into a HIP graph after it has run once.

    python -m paper_2506_22175_amd.block          # times both on the GPU
"""
from __future__ import annotations

import time

import torch

from . import binding as B

_TORCH = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16}


def _code(name, W):
    for code, dtype in _TORCH.items():
        if W.dtype == dtype:
            return code
    raise ValueError(f"{name} is {W.dtype}: weights are float32 or bfloat16")


def _check_weights(device, *weights):
    """The library is handed addresses: what another type, size or order of the elements would make it read or write is refused here,
    before anything is allocated.  weights: (name, tensor or None, type, shape); of a vector its elements count."""
    device = torch.device(device)
    for name, W, dtype, shape in weights:
        if W is None:
            continue
        fits = W.numel() == shape[0] if len(shape) == 1 else W.shape == shape
        if W.dtype != dtype or not fits or not W.is_contiguous():
            raise ValueError(f"{name} has to be contiguous {dtype} {tuple(shape)}; it is {W.dtype} {tuple(W.shape)}, strides {W.stride()}")
        if W.device.type != device.type or (device.index is not None and W.device.index != device.index):
            raise ValueError(f"{name} is on {W.device}, the block on {device}")


class Shared:
    """The shared expert's two products for T rows of M: weights V1 [M,N], V2 [N,M], both float32 or both bfloat16 as the rows are, biases
    float32 or None.  With `training` its gradients dV1, dV2, db1, db2 (float) are overwritten by backward.  rows: width and type of the
    rows that it is to meet, refused where the weights have others."""

    def __init__(self, T, V1, V2, b1=None, b2=None, training=False, device="cuda:0", rows=None):
        (M, N), dtype = V1.shape, _code("V1", V1)
        if rows is not None and rows != (M, dtype):
            raise ValueError(f"V1 is {V1.dtype} {tuple(V1.shape)}: the block's rows are {_TORCH[rows[1]]} and {rows[0]} wide")
        _check_weights(device, ("V1", V1, V1.dtype, (M, N)), ("V2", V2, V1.dtype, (N, M)), ("b1", b1, torch.float32, (N,)),
                       ("b2", b2, torch.float32, (M,)))
        self.V1, self.V2, self.b1, self.b2 = V1, V2, b1, b2
        self.first = B.make_linear_config(T, M, N, dtype, B.MOE_ACT_GELU, 1)
        self.second = B.make_linear_config(T, N, M, dtype, B.MOE_ACT_NONE, 1)
        self.a = torch.empty((T, N), dtype=V1.dtype, device=device)
        self.z = self.da = None
        if training:
            self.z, self.da = torch.empty_like(self.a), torch.empty_like(self.a)
            self.dV1, self.dV2 = (torch.empty(V.shape, dtype=torch.float32, device=device) for V in (V1, V2))
            self.db1, self.db2 = (None if b is None else torch.empty(b.numel(), dtype=torch.float32, device=device) for b in (b1, b2))
        need = max(B.moe_linear_scratch_bytes(c) for c in (self.first, self.second))
        self.scratch = torch.empty(max(need, 16), dtype=torch.uint8, device=device)

    def forward(self, y, out):
        """out += the expert's rows for y."""
        B.moe_linear_fwd(self.first, y, self.V1, self.b1, None, self.z, self.a, self.scratch)
        B.moe_linear_fwd(self.second, self.a, self.V2, self.b2, out, None, out, self.scratch)

    def backward(self, y, dout, dy):
        """dy += the gradient of y."""
        if self.b2 is not None:
            B.moe_act_bwd(self.second, dout, None, None, self.db2, self.scratch)
        B.moe_linear_bwd(self.second, dout, self.a, self.V2, self.da, self.dV2, self.scratch)
        B.moe_act_bwd(self.first, self.da, self.z, self.da, self.db1, self.scratch)
        B.moe_linear_bwd(self.first, self.da, y, self.V1, dy, self.dV1, self.scratch, add=dy)

    def gradients(self):
        return [g for g in (self.dV1, self.db1, self.dV2, self.db2) if g is not None]


class Block:
    """Training.  Weights: gain [M] float, Wg [M,E], W1 [E,M,H], W2 [E,H,M] of `dtype`; bias [E] float or None moves the
    router's choice and not its weights (its gradient is none: it is set from `load`, the tokens counted per expert).
    shared: (V1, V2, b1, b2) of a shared expert, biases or None, or None."""

    def __init__(self, T, M, H, E, k, gain, Wg, W1, W2, bias=None, capacity_factor=1.25, dtype=B.MOE_BF16, eps=1e-6,
                 scores=B.MOE_SOFTMAX, renormalize=0, groups=1, group_k=1, scale=1.0, device="cuda:0", shared=None):
        f32, i32 = torch.float32, torch.int32
        _check_weights(device, ("gain", gain, f32, (M,)), ("Wg", Wg, _TORCH[dtype], (M, E)), ("W1", W1, _TORCH[dtype], (E, M, H)),
                       ("W2", W2, _TORCH[dtype], (E, H, M)), ("bias", bias, f32, (E,)))
        self.shared = None if shared is None else Shared(T, *shared, training=True, device=device, rows=(M, dtype))
        self.gain, self.Wg, self.W1, self.W2, self.bias = gain, Wg, W1, W2, bias
        self.layer = B.make_config(T, M, H, E, k, capacity_factor, 1, dtype, 0, 1)
        self.norm = B.make_norm_config(T, M, eps, dtype, grad_overwrite=1)
        self.router = B.make_router_config(T, E, k, scores, groups, group_k, 2, renormalize, scale, B.MOE_F32)
        rows = B.moe_capacity(self.layer) * E

        def new(*shape, dtype=_TORCH[dtype]):
            return torch.empty(shape, dtype=dtype, device=device)

        self.h, self.y, self.out, self.dy, self.dx = (new(T, M) for _ in range(5))
        self.rstd, self.logits, self.dlogits = new(T, dtype=f32), new(T, E, dtype=f32), new(T, E, dtype=f32)
        self.topk_idx, self.slot, self.counts = new(T, k, dtype=i32), new(T, k, dtype=i32), new(1, E, dtype=i32)
        self.topk_w, self.dw, self.slot_w = new(T, k, dtype=f32), new(T, k, dtype=f32), new(rows, dtype=f32)
        self.load = torch.zeros(E, dtype=i32, device=device)
        self.di, self.do, self.ddo, self.ddi = (new(rows, M) for _ in range(4))
        self.z, self.a, self.dz = (new(rows, H) for _ in range(3))
        self.dgain, self.dWg = new(M, dtype=f32), new(M, E, dtype=f32)
        self.dW1, self.dW2 = new(E, M, H, dtype=f32), new(E, H, M, dtype=f32)
        self.slot_scratch = new(B.moe_slot_scratch_bytes(self.layer), dtype=torch.uint8)
        self.gate_scratch = new(B.moe_gate_scratch_bytes(self.layer), dtype=torch.uint8)
        self.norm_scratch = new(B.moe_norm_scratch_bytes(self.norm), dtype=torch.uint8)
        # the gradients' list is laid out once: backward writes to the same memory every time
        self.gradients = [self.dgain, self.dWg, self.dW1, self.dW2] + ([] if shared is None else self.shared.gradients())
        self.grad_list = B.make_grad_list(self.gradients, self.gradients)
        self.grad_norm = new(1, dtype=f32)
        self.grad_scratch = new(B.moe_grad_scratch_bytes(self.grad_list), dtype=torch.uint8)

    def forward(self, x, residual=None):
        """(out, h); `load` counts on."""
        B.moe_norm_fwd(self.norm, x, residual, self.gain, self.h, self.y, None, self.rstd)
        # the layer's own gate makes the logits; its choice is replaced by the router's
        B.moe_route(self.layer, self.y, self.Wg, None, self.logits, self.topk_idx, self.topk_w)
        B.moe_router_fwd(self.router, self.logits, self.bias, self.topk_idx, self.topk_w, self.load)
        B.moe_assign_slots(self.layer, self.topk_idx, self.topk_w, self.slot, self.counts, self.slot_w, self.slot_scratch)
        B.moe_dispatch(self.layer, 0, self.y, self.slot, self.di)
        B.moe_expert_ffn_fwd(self.layer, 0, self.di, self.counts, self.W1, self.W2, self.z, self.a, self.do)
        B.moe_combine(self.layer, 0, self.do, self.slot, self.topk_w, self.out)
        if self.shared:
            self.shared.forward(self.y, self.out)
        return self.out, self.h

    def backward(self, dout, dh=None):
        """From the gradients of out and h that of x (and of residual alike); `gradients` are overwritten.  Once per forward: what forward kept of the experts' inner rows is used up."""
        B.moe_dispatch(self.layer, 0, dout, self.slot, self.ddo, self.do, self.dw)
        B.moe_expert_ffn_bwd(self.layer, 0, False, self.di, self.z, self.ddo, self.counts, self.slot_w, self.W1, self.W2,
                             self.dz, self.ddi, self.dW1, self.dW2, None)
        B.moe_router_bwd(self.router, self.logits, self.topk_idx, self.dw, self.dlogits)
        B.moe_gate_weight_grad(self.layer, 0, self.y, self.dlogits, self.dWg, self.gate_scratch)
        B.moe_dispatch_bwd(self.layer, 0, self.ddi, self.slot, self.dlogits, self.Wg, self.dy)
        if self.shared:
            self.shared.backward(self.y, dout, self.dy)
        B.moe_norm_bwd(self.norm, self.dy, self.h, self.gain, self.rstd, dh, self.dx, self.dgain, self.norm_scratch)
        return self.dx

    def clip(self, most):
        """Scales all gradients together so that their norm is at most `most`; the norm they had, a float on the GPU."""
        B.moe_grad_clip(self.grad_list, most, self.grad_norm, self.grad_scratch)
        return self.grad_norm


class Packed:
    """The experts' weights of a trained block in 4 bits, laid out once."""

    def __init__(self, W1, W2):
        (self.E, self.M, self.H), dtype = W1.shape, _code("W1", W1)
        _check_weights(W1.device, ("W1", W1, W1.dtype, W1.shape), ("W2", W2, W1.dtype, (self.E, self.H, self.M)))

        def pack(W, K, N):
            q = torch.empty((self.E, N, K // 2), dtype=torch.uint8, device=W.device)
            s = torch.empty((self.E, N, K // 32), dtype=torch.uint8, device=W.device)
            B.moe_w4_quantize(self.E, K, N, dtype, W, q, s)
            return q, s

        self.first, self.second = pack(W1, self.M, self.H), pack(W2, self.H, self.M)


class Served:
    """Serving T tokens at a time (1 for a single sequence) from `Packed` weights.  With `eight_bits` the experts' first product
    takes e4m3 rows with a scale per 128 columns, written by a second norm of the sum; the gate always reads `dtype`."""

    def __init__(self, T, k, gain, Wg, packed, bias=None, dtype=B.MOE_BF16, eps=1e-6, scores=B.MOE_SOFTMAX, renormalize=0,
                 groups=1, group_k=1, scale=1.0, eight_bits=False, device="cuda:0"):
        p, M, H, E = packed, packed.M, packed.H, packed.E
        _check_weights(device, ("gain", gain, torch.float32, (M,)), ("Wg", Wg, _TORCH[dtype], (M, E)), ("bias", bias, torch.float32, (E,)))
        self.gain, self.Wg, self.bias, self.packed, self.eight_bits = gain, Wg, bias, p, eight_bits
        self.layer = B.make_config(T, M, H, E, k, 1.0, 1, dtype)
        self.norm = B.make_norm_config(T, M, eps, dtype)
        self.norm8 = B.make_norm_config(T, M, eps, dtype, B.MOE_E4M3, 128)
        self.router = B.make_router_config(T, E, k, scores, groups, group_k, 2, renormalize, scale, B.MOE_F32)
        self.first = B.make_w4_config(T, k, E, M, H, B.MOE_E4M3 if eight_bits else dtype, dtype, 128 if eight_bits else 0,
                                      gelu=1)
        self.second = B.make_w4_config(T, k, E, H, M, dtype, dtype, per_choice=1, combine=1)

        def new(*shape, dtype=_TORCH[dtype]):
            return torch.empty(shape, dtype=dtype, device=device)

        f32 = torch.float32
        self.h, self.y, self.out, self.a = new(T, M), new(T, M), new(T, M), new(T, k, H)
        self.y8, self.scales = new(T, M, dtype=torch.float8_e4m3fn), new(T, (M + 127) // 128, dtype=f32)
        self.logits, self.topk_w = new(T, E, dtype=f32), new(T, k, dtype=f32)
        self.topk_idx = new(T, k, dtype=torch.int32)
        # the two products follow each other on one stream and may share their scratch
        self.scratch = new(max(B.moe_w4_scratch_bytes(self.first), B.moe_w4_scratch_bytes(self.second), 16), dtype=torch.uint8)

    def forward(self, x, residual=None):
        """(out, h)."""
        B.moe_norm_fwd(self.norm, x, residual, self.gain, self.h, self.y)
        rows, scales = self.y, None
        if self.eight_bits:
            rows, scales = self.y8, self.scales
            B.moe_norm_fwd(self.norm8, x, residual, self.gain, None, rows, scales)
        B.moe_route(self.layer, self.y, self.Wg, None, self.logits, self.topk_idx, self.topk_w)
        B.moe_router_fwd(self.router, self.logits, self.bias, self.topk_idx, self.topk_w)
        B.moe_w4_product(self.first, rows, scales, self.topk_idx, None, *self.packed.first, self.a, self.scratch)
        B.moe_w4_product(self.second, self.a, None, self.topk_idx, self.topk_w, *self.packed.second, self.out, self.scratch)
        return self.out, self.h


class Few:
    """Serving up to 256 tokens at a time from the trained weights as they are (`Block`'s); `shared` as there."""

    def __init__(self, T, k, gain, Wg, W1, W2, bias=None, eps=1e-6, scores=B.MOE_SOFTMAX, renormalize=0, groups=1, group_k=1,
                 scale=1.0, device="cuda:0", shared=None):
        (E, M, H), dtype = W1.shape, _code("W1", W1)
        _check_weights(device, ("gain", gain, torch.float32, (M,)), ("Wg", Wg, W1.dtype, (M, E)), ("W1", W1, W1.dtype, (E, M, H)),
                       ("W2", W2, W1.dtype, (E, H, M)), ("bias", bias, torch.float32, (E,)))
        self.shared = None if shared is None else Shared(T, *shared, device=device, rows=(M, dtype))
        self.gain, self.Wg, self.W1, self.W2, self.bias = gain, Wg, W1, W2, bias
        self.norm = B.make_norm_config(T, M, eps, dtype)
        self.layer = B.make_few_config(T, M, H, E, k, dtype, scores, groups, group_k, 2, renormalize, scale)
        self.h, self.y, self.out = (torch.empty((T, M), dtype=W1.dtype, device=device) for _ in range(3))
        self.logits, self.topk_w = (torch.empty((T, n), dtype=torch.float32, device=device) for n in (E, k))
        self.topk_idx = torch.empty((T, k), dtype=torch.int32, device=device)
        self.scratch = torch.empty(B.moe_few_scratch_bytes(self.layer), dtype=torch.uint8, device=device)

    def forward(self, x, residual=None):
        """(out, h)."""
        B.moe_norm_fwd(self.norm, x, residual, self.gain, self.h, self.y)
        B.moe_few_forward(self.layer, self.y, self.Wg, None, self.bias, self.W1, self.W2, self.out, self.logits, self.topk_idx,
                          self.topk_w, self.scratch)
        if self.shared:
            self.shared.forward(self.y, self.out)
        return self.out, self.h


def _timed(f, passes):
    f()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(passes):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - t0) / passes * 1e6


def main():
    g = torch.Generator(device="cuda:0").manual_seed(0)
    M, H, E, k = 1024, 4096, 16, 2

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda:0") * std).to(dtype)

    weights = (torch.ones(M, device="cuda:0"), normal(M, E, std=0.02), normal(E, M, H, std=0.02), normal(E, H, M, std=0.02))
    shared = (normal(M, H, std=0.02), normal(H, M, std=0.02), torch.zeros(H, device="cuda:0"), torch.zeros(M, device="cuda:0"))
    T = 4096
    x, residual, dout, dh = (normal(T, M) for _ in range(4))
    for beside in (None, shared):
        block = Block(T, M, H, E, k, *weights, renormalize=1, shared=beside)

        def step():
            block.forward(x, residual)
            block.backward(dout, dh)

        def clipped():
            step()
            block.clip(1.0)

        print(f"training, {T} tokens of {M}/{H}, {E} experts{', a shared one' if beside else ''}, {k} choices: {_timed(step, 20):.0f} us "
              f"per step, {_timed(clipped, 20):.0f} us with its gradients clipped", flush=True)
    packed = Packed(block.W1, block.W2)
    for T in (1, 16):
        x, residual = normal(T, M), normal(T, M)
        passes = [(f"4-bit weights, {'e4m3' if eight else 'bf16'} rows", Served(T, k, weights[0], weights[1], packed, renormalize=1, eight_bits=eight))
                  for eight in (False, True)]
        passes += [(f"bf16 weights{', a shared expert' if beside else ''}", Few(T, k, *weights, renormalize=1, shared=beside)) for beside in (None, shared)]
        for name, served in passes:
            eager = _timed(lambda: served.forward(x, residual), 200)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                served.forward(x, residual)
            print(f"serving, {T} tokens, {name}: {eager:.1f} us, as a graph {_timed(graph.replay, 200):.1f} us", flush=True)


if __name__ == "__main__":
    main()
