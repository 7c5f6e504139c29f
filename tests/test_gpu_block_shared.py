"""The block with a shared expert, its gradients clipped, and served a few tokens at a time from the weights as they are: the new
operators in a run together, against 64 bits."""
import math

import pytest
import torch

from paper_2506_22175_amd import binding as B
from paper_2506_22175_amd.block import Block, Few, Packed, Served

pytestmark = pytest.mark.gpu
D = "cuda:0"
DT = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16}
# of a tensor's largest entry, as the layer's own tests allow: some ten roundings to bf16 of 2^-8 each, or of 2^-24 after
# sums of some hundred terms
TOL = {B.MOE_F32: 1e-4, B.MOE_BF16: 4e-2}


def _weights(M, H, E, N, dtype, biases, seed=0):
    g = torch.Generator().manual_seed(seed)
    Wg, W1, W2, V1, V2 = ((torch.randn(s, generator=g) * 0.1).to(DT[dtype]) for s in ((M, E), (E, M, H), (E, H, M), (M, N), (N, M)))
    b1, b2 = (torch.randn(n, generator=g) * 0.3 if biases else None for n in (N, M))
    return torch.rand(M, generator=g) + 0.5, Wg, W1, W2, (V1, V2, b1, b2)


def _rows(T, M, dtype, n, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((T, M), generator=g).to(DT[dtype]) for _ in range(n)]


def _gpu(ts):
    return tuple(None if t is None else t.to(D) for t in ts)


def _gelu(z):
    return z * torch.special.ndtr(z)


def _close(got, want, tol, what):
    got, want = got.cpu().double(), want.detach()
    assert (got - want).abs().max() <= tol * want.abs().max(), what


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("biases", [False, True])
@pytest.mark.parametrize("T", [24, 203])
def test_training_with_a_shared_expert_and_clipping(T, biases, dtype):
    M, H, E, k, N = 72, 104, 8, 3, 136
    gain, Wg, W1, W2, shared = _weights(M, H, E, N, dtype, biases)
    x, r, dout, dh = _rows(T, M, dtype, 4)
    block = Block(T, M, H, E, k, *_gpu((gain, Wg, W1, W2)), capacity_factor=0.9, dtype=dtype, renormalize=1, shared=_gpu(shared))
    for t in block.gradients + [block.out, block.dx]:
        t.fill_(float("nan"))
    out, h = block.forward(x.to(D), r.to(D))
    dx = block.backward(dout.to(D), dh.to(D))
    idx, kept = block.topk_idx.cpu().long(), block.slot.cpu() >= 0

    leaves = [None if t is None else t.double().requires_grad_() for t in (x, r, gain, Wg, W1, W2, *shared)]
    X, R, G, Vg, U1, U2, V1, V2, b1, b2 = leaves
    Hh = X + R
    Y = Hh * torch.rsqrt((Hh * Hh).mean(1, keepdim=True) + 1e-6) * G
    w = torch.softmax(Y @ Vg, 1).gather(1, idx)
    w = w / w.sum(1, keepdim=True)
    z = Y @ V1
    a = _gelu(z if b1 is None else z + b1)
    O = a @ V2 if b2 is None else a @ V2 + b2
    for e in range(E):
        t, j = ((idx == e) & kept).nonzero(as_tuple=True)
        O = O.index_add(0, t, _gelu(Y[t] @ U1[e]) @ U2[e] * w[t, j, None])
    ((O * dout.double()).sum() + (Hh * dh.double()).sum()).backward()
    pairs = [(block.dgain, G), (block.dWg, Vg), (block.dW1, U1), (block.dW2, U2), (block.shared.dV1, V1), (block.shared.db1, b1),
             (block.shared.dV2, V2), (block.shared.db2, b2)]
    pairs = [(got, leaf.grad) for got, leaf in pairs if got is not None]
    tol = TOL[dtype]
    for got, want, what in [(out, O, "out"), (h, Hh, "h"), (dx, X.grad, "dx")] + [(g, w, i) for i, (g, w) in enumerate(pairs)]:
        _close(got, want, tol, what)
    assert len(block.gradients) == len(pairs)

    before = [g.clone() for g in block.gradients]
    norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in before))
    assert abs(float(block.clip(2 * norm)) - norm) <= norm * 2.0 ** -23 and all(torch.equal(a, b) for a, b in zip(before, block.gradients))
    got = float(block.clip(0.25 * norm))
    for now, was in zip(block.gradients, before):
        want = was.double() * (float(torch.tensor(0.25 * norm)) / got)
        assert ((now.double() - want).abs() <= 2.0 ** -23 * want.abs() + 1e-45).all()


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("beside", [False, True])
@pytest.mark.parametrize("T", [1, 5, 70])
def test_serving_from_the_weights_as_they_are(T, beside, dtype):
    M, H, E, k, N = 96, 160, 8, 3, 200
    kw = dict(scores=B.MOE_SIGMOID, groups=4, group_k=2, renormalize=1, scale=2.5)
    gain, Wg, W1, W2, shared = _weights(M, H, E, N, dtype, True)
    x, r = _rows(T, M, dtype, 2)
    few = Few(T, k, *_gpu((gain, Wg, W1, W2)), shared=_gpu(shared) if beside else None, **kw)
    out, h = few.forward(x.to(D), r.to(D))
    idx = few.topk_idx.cpu().long()
    Hh = x.double() + r.double()
    Y = Hh * torch.rsqrt((Hh * Hh).mean(1, keepdim=True) + 1e-6) * gain.double()
    w = torch.sigmoid(few.logits.cpu().double()).gather(1, idx)
    w = w / w.sum(1, keepdim=True) * 2.5
    want = torch.zeros(T, M, dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            want[t] += _gelu(Y[t] @ W1[idx[t, j]].double()) @ W2[idx[t, j]].double() * w[t, j]
    if beside:
        V1, V2, b1, b2 = (t.double() for t in shared)
        want += _gelu(Y @ V1 + b1) @ V2 + b2
    _close(h, Hh, TOL[dtype], "h")
    _close(out, want, TOL[dtype], "out")

    first, X, R = out.clone(), x.to(D), r.to(D)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        few.forward(X, R)
    for _ in range(3):
        few.out.fill_(float("nan"))
        graph.replay()
        assert torch.equal(few.out, first)
        few.forward(X, R)
        torch.cuda.synchronize()
        assert torch.equal(few.out, first)


def test_the_router_chooses_as_for_4_bit_weights():
    """The layer's logits are float sums, the few tokens' 64-bit sums rounded to float: the same choices but for logits that lie closer than that."""
    T, M, H, E, k = 64, 256, 128, 16, 2
    gain, Wg, W1, W2, _ = _weights(M, H, E, 8, B.MOE_BF16, False)
    x, r = _rows(T, M, B.MOE_BF16, 2)
    few = Few(T, k, *_gpu((gain, Wg, W1, W2)))
    served = Served(T, k, gain.to(D), Wg.to(D), Packed(W1.to(D), W2.to(D)))
    few.forward(x.to(D), r.to(D))
    served.forward(x.to(D), r.to(D))
    assert (few.logits - served.logits).abs().max() <= M * 2.0 ** -24 * served.logits.abs().max()
    top = few.logits.sort(1, descending=True)[0]
    clear = ((top[:, 0] - top[:, 1]).abs() > 1e-4) & ((top[:, 1] - top[:, 2]).abs() > 1e-4)
    assert clear.sum() > T // 2 and torch.equal(few.topk_idx[clear], served.topk_idx[clear])
