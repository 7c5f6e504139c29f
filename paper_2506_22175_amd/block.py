"""A whole feed-forward block of a model around the expert layer, from the calls of include/moe.h: the residual's addition and
the norm, the gate's logits, the router, the experts, the weighted sum; and the same block serving, its experts in 4 bits.

    h = x + residual;  y = h / sqrt(mean(h^2) + eps) * gain;  logits = y Wg;  idx, w = router(logits, bias)
    out[t] = sum over j of w[t,j] * gelu(y[t] W1[idx[t,j]]) W2[idx[t,j]]

out and h are what the next block adds up.  Training (`Block`) has a capacity per expert and drops what is beyond; serving
(`Served`) drops nothing.  All buffers are made once, so that each pass may be captured into a HIP graph after it has run once.

    python -m paper_2506_22175_amd.block          # times both on the GPU
"""
from __future__ import annotations

import time

import torch

from . import binding as B

_TORCH = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16}


class Block:
    """Training.  Weights: gain [M] float, Wg [M,E], W1 [E,M,H], W2 [E,H,M] of `dtype`; bias [E] float or None moves the
    router's choice and not its weights (its gradient is none: it is set from `load`, the tokens counted per expert)."""

    def __init__(self, T, M, H, E, k, gain, Wg, W1, W2, bias=None, capacity_factor=1.25, dtype=B.MOE_BF16, eps=1e-6,
                 scores=B.MOE_SOFTMAX, renormalize=0, groups=1, group_k=1, scale=1.0, device="cuda:0"):
        self.gain, self.Wg, self.W1, self.W2, self.bias = gain, Wg, W1, W2, bias
        self.layer = B.make_config(T, M, H, E, k, capacity_factor, 1, dtype, 0, 1)
        self.norm = B.make_norm_config(T, M, eps, dtype, grad_overwrite=1)
        self.router = B.make_router_config(T, E, k, scores, groups, group_k, 2, renormalize, scale, B.MOE_F32)
        rows = B.moe_capacity(self.layer) * E

        def new(*shape, dtype=_TORCH[dtype]):
            return torch.empty(shape, dtype=dtype, device=device)

        f32, i32 = torch.float32, torch.int32
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
        return self.out, self.h

    def backward(self, dout, dh=None):
        """From the gradients of out and h that of x (and of residual alike); dgain, dWg, dW1, dW2 are overwritten.  Once
        per forward: what forward kept of the experts' inner rows is used up."""
        B.moe_dispatch(self.layer, 0, dout, self.slot, self.ddo, self.do, self.dw)
        B.moe_expert_ffn_bwd(self.layer, 0, False, self.di, self.z, self.ddo, self.counts, self.slot_w, self.W1, self.W2,
                             self.dz, self.ddi, self.dW1, self.dW2, None)
        B.moe_router_bwd(self.router, self.logits, self.topk_idx, self.dw, self.dlogits)
        B.moe_gate_weight_grad(self.layer, 0, self.y, self.dlogits, self.dWg, self.gate_scratch)
        B.moe_dispatch_bwd(self.layer, 0, self.ddi, self.slot, self.dlogits, self.Wg, self.dy)
        B.moe_norm_bwd(self.norm, self.dy, self.h, self.gain, self.rstd, dh, self.dx, self.dgain, self.norm_scratch)
        return self.dx


class Packed:
    """The experts' weights of a trained block in 4 bits, laid out once."""

    def __init__(self, W1, W2):
        self.E, self.M, self.H = W1.shape
        dtype = B.MOE_F32 if W1.dtype == torch.float32 else B.MOE_BF16

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
    T = 4096
    block, x, residual = Block(T, M, H, E, k, *weights, renormalize=1), normal(T, M), normal(T, M)
    dout, dh = normal(T, M), normal(T, M)

    def step():
        block.forward(x, residual)
        block.backward(dout, dh)

    print(f"training, {T} tokens of {M}/{H}, {E} experts, {k} choices: {_timed(step, 20):.0f} us per step", flush=True)
    packed = Packed(block.W1, block.W2)
    for T in (1, 16):
        for eight_bits in (False, True):
            served = Served(T, k, weights[0], weights[1], packed, renormalize=1, eight_bits=eight_bits)
            x, residual = normal(T, M), normal(T, M)
            eager = _timed(lambda: served.forward(x, residual), 200)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                served.forward(x, residual)
            print(f"serving, {T} tokens, {'e4m3' if eight_bits else 'bf16'} rows: {eager:.1f} us, as a graph "
                  f"{_timed(graph.replay, 200):.1f} us", flush=True)


if __name__ == "__main__":
    main()
