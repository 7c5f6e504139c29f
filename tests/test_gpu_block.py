"""The block around the expert layer (norm, gate, router, experts) against 64 bits, training and serving."""
import pytest
import torch

from paper_2506_22175_amd import binding as B
from paper_2506_22175_amd.block import Block, Packed, Served

pytestmark = pytest.mark.gpu
D = "cuda:0"
DT = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16}
# of a tensor's largest entry, as the layer's own tests allow: some ten roundings to bf16 of 2^-8 each, or of 2^-24 after
# sums of some hundred terms
TOL = {B.MOE_F32: 1e-4, B.MOE_BF16: 4e-2}


def _weights(M, H, E, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    gain = torch.rand(M, generator=g) + 0.5
    Wg, W1, W2 = ((torch.randn(s, generator=g) * 0.1).to(DT[dtype]) for s in ((M, E), (E, M, H), (E, H, M)))
    return gain, Wg, W1, W2


def _rows(T, M, dtype, n, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((T, M), generator=g).to(DT[dtype]) for _ in range(n)]


def _gelu(z):
    return 0.5 * z * (1 + torch.erf(z / 2 ** 0.5))


def _close(got, want, tol, what):
    got, want = got.cpu().double(), want.detach()
    assert (got - want).abs().max() <= tol * want.abs().max(), what


ROUTERS = {
    "softmax": dict(),
    "renormalized": dict(renormalize=1, scale=1.5),
    "sigmoid, groups": dict(scores=B.MOE_SIGMOID, groups=4, group_k=2, renormalize=1, scale=2.5),
    "fewer experts than choices": dict(bias=[-float("inf"), 0.0, 0.1] + [-float("inf")] * 5),
}


def _scores(logits, idx, kw):
    """The chosen experts' weights; logits in 64 bits, choices that are none get 0."""
    s = torch.sigmoid(logits) if kw.get("scores") == B.MOE_SIGMOID else torch.softmax(logits, 1)
    w = s.gather(1, idx.clamp(min=0)) * (idx >= 0)
    if kw.get("renormalize"):
        w = w / w.sum(1, keepdim=True)
    return w * kw.get("scale", 1.0)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("router", list(ROUTERS))
@pytest.mark.parametrize("capacity", [0.6, 4.0])
def test_training(router, dtype, capacity):
    T, M, H, E, k = 203, 72, 104, 8, 3
    kw = dict(ROUTERS[router])
    bias = torch.tensor(kw.pop("bias"), device=D) if "bias" in kw else None
    gain, Wg, W1, W2 = _weights(M, H, E, dtype)
    x, r, dout, dh = _rows(T, M, dtype, 4)
    block = Block(T, M, H, E, k, *(t.to(D) for t in (gain, Wg, W1, W2)), bias=bias, capacity_factor=capacity, dtype=dtype, **kw)
    for t in (block.out, block.h, block.dx, block.dgain, block.dWg, block.dW1, block.dW2):
        t.fill_(float("nan"))
    out, h = block.forward(x.to(D), r.to(D))
    dx = block.backward(dout.to(D), dh.to(D))
    idx, kept = block.topk_idx.cpu().long(), block.slot.cpu() >= 0
    if bias is not None:
        assert (idx[:, :2] >= 0).all() and (idx[:, 2] == -1).all() and not kept[:, 2].any()
    assert kept.sum() == block.counts.sum() and (capacity > 1 or not kept[idx >= 0].all())
    assert torch.equal(block.load.cpu(), torch.bincount(idx[idx >= 0], minlength=E).int())

    X, R, G, Vg, V1, V2 = (t.double().requires_grad_() for t in (x, r, gain, Wg, W1, W2))
    Hh = X + R
    Y = Hh * torch.rsqrt((Hh * Hh).mean(1, keepdim=True) + 1e-6) * G
    W = _scores(Y @ Vg, idx, kw)
    O = torch.zeros(T, M, dtype=torch.float64)
    for e in range(E):
        t, j = ((idx == e) & kept).nonzero(as_tuple=True)
        O = O.index_add(0, t, _gelu(Y[t] @ V1[e]) @ V2[e] * W[t, j, None])
    ((O * dout.double()).sum() + (Hh * dh.double()).sum()).backward()
    tol = TOL[dtype]
    for got, want, what in ((out, O, "out"), (h, Hh, "h"), (dx, X.grad, "dx"), (block.dgain, G.grad, "dgain"),
                            (block.dWg, Vg.grad, "dWg"), (block.dW1, V1.grad, "dW1"), (block.dW2, V2.grad, "dW2")):
        _close(got, want, tol, what)


def _unpack(q, s):
    value = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    value = torch.cat([value, -value])
    q, s = q.cpu().long(), s.cpu().double()
    return torch.stack([value[q & 15], value[q >> 4]], -1).flatten(-2) * (2.0 ** (s - 127)).repeat_interleave(32, -1)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("eight_bits", [False, True])
@pytest.mark.parametrize("T", [1, 5, 70])
def test_serving(T, eight_bits, dtype):
    M, H, E, k = 96, 160, 8, 3
    kw = ROUTERS["sigmoid, groups"]
    gain, Wg, W1, W2 = _weights(M, H, E, dtype)
    x, r = _rows(T, M, dtype, 2)
    packed = Packed(W1.to(D), W2.to(D))
    served = Served(T, k, gain.to(D), Wg.to(D), packed, dtype=dtype, eight_bits=eight_bits, **kw)
    out, h = served.forward(x.to(D), r.to(D))
    idx = served.topk_idx.cpu().long()
    assert (idx >= 0).all()
    Hh = x.double() + r.double()
    Y = Hh * torch.rsqrt((Hh * Hh).mean(1, keepdim=True) + 1e-6) * gain.double()
    _close(h, Hh, TOL[dtype], "h")
    _close(served.y, Y, TOL[dtype], "y")
    W = _scores(served.logits.cpu().double(), idx, kw)
    _close(served.topk_w, W, 1e-5, "weights")
    rows = Y
    if eight_bits:          # the product's own input: half a step of 2^-4 from the norm's
        rows = served.y8.cpu().double() * served.scales.cpu().double().repeat_interleave(128, 1)[:, :M]
        _close(rows, Y, 2.0 ** -4 + TOL[dtype], "rows of 8 bits")
    V1, V2 = _unpack(*packed.first), _unpack(*packed.second)
    want = torch.zeros(T, M, dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            e = idx[t, j]
            want[t] += V2[e] @ _gelu(V1[e] @ rows[t]) * W[t, j]
    _close(out, want, TOL[dtype], "out")

    # the same pass as a graph, replayed between eager passes
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    X, R = x.to(D), r.to(D)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        served.forward(X, R)
    for _ in range(3):
        served.out.fill_(float("nan"))
        graph.replay()
        assert torch.equal(served.out, first)
        served.forward(X, R)
        torch.cuda.synchronize()
        assert torch.equal(served.out, first)
