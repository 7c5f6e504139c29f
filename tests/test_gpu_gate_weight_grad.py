"""The gate's weight gradient from a dL that is there already, against 64 bits: dWg (+)= x^T dL.

At most T additions of float; bfloat16 storage carries dL as two bfloat16 terms, 2^-17 of its size."""
import pytest
import torch

from paper_2506_22175_amd import binding as B
from paper_2506_22175_amd.block import Block

pytestmark = pytest.mark.gpu
D = "cuda:0"
DT = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16}


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T,n,M,E", [(1, 1, 8, 1), (63, 1, 24, 3), (64, 1, 64, 16), (65, 1, 72, 17), (200, 2, 136, 33), (1000, 1, 512, 64),
                                     (4096, 4, 256, 8), (130, 1, 2048, 47)])
def test_against_64_bits(T, n, M, E, dtype):
    g = torch.Generator().manual_seed(T + E)
    x, dL = torch.randn((T, M), generator=g).to(DT[dtype]), torch.randn((T, E), generator=g)
    dL[torch.rand((T, E), generator=g) < 0.5] = 0.0
    for overwrite in (1, 0):
        cfg = B.make_config(T, M, 8, E, 1, 1.0, n, dtype, 0, overwrite)
        need = B.moe_gate_scratch_bytes(cfg)
        scratch = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=D)
        dWg = torch.full((M, E), float("nan") if overwrite else 3.0, device=D)
        for part in range(n):
            B.moe_gate_weight_grad(cfg, part, x.to(D), dL.to(D), dWg, scratch)
        old = 0.0 if overwrite else 3.0
        want, size = x.double().t() @ dL.double() + old, x.double().abs().t() @ dL.double().abs() + old
        unit = (T + n + 64) * 2.0 ** -24 + (2.0 ** -17 if dtype == B.MOE_BF16 else 0.0)
        assert ((dWg.cpu().double() - want).abs() <= unit * size).all()
        assert (scratch[need:] == 0xFF).all()


def test_a_training_step_of_the_block_allocates_nothing():
    """Its buffers are made once, and the gate's weight gradient is a kernel of the library's."""
    T, M, H, E, k = 300, 64, 128, 8, 2
    g = torch.Generator().manual_seed(0)
    gain, Wg, W1, W2 = torch.ones(M), *((torch.randn(s, generator=g) * 0.1).bfloat16() for s in ((M, E), (E, M, H), (E, H, M)))
    x, r, dout, dh = (torch.randn((T, M), generator=g).bfloat16().to(D) for _ in range(4))
    block = Block(T, M, H, E, k, *(t.to(D) for t in (gain, Wg, W1, W2)), renormalize=1)
    block.forward(x, r)
    block.backward(dout, dh)
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    block.forward(x, r)
    block.backward(dout, dh)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
def test_a_training_step_of_the_block_in_a_graph(dtype):
    T, M, H, E, k = 300, 64, 128, 8, 2
    g = torch.Generator().manual_seed(0)
    gain, Wg, W1, W2 = torch.ones(M), *((torch.randn(s, generator=g) * 0.1).to(DT[dtype]) for s in ((M, E), (E, M, H), (E, H, M)))
    x, r, dout, dh = (torch.randn((T, M), generator=g).to(DT[dtype]).to(D) for _ in range(4))
    block = Block(T, M, H, E, k, *(t.to(D) for t in (gain, Wg, W1, W2)), renormalize=1, dtype=dtype)
    out = (block.out, block.h, block.dx, block.dgain, block.dWg, block.dW1, block.dW2)

    def step():
        block.forward(x, r)
        block.backward(dout, dh)

    step()
    torch.cuda.synchronize()
    first = [o.clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for o in out:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, first))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, first))
