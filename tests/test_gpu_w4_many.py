"""4-bit products of more assignments than the workgroups look through by themselves: listed by expert first."""
import pytest
import torch

from paper_2506_22175_amd import binding as B
from test_gpu_operator_paths import BF16, DEV, E4M3, F32, choices, product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,group", [(F32, 0), (BF16, 0), (E4M3, 128)])
@pytest.mark.parametrize("T,k,E,K,N", [(1024, 2, 64, 64, 40), (1025, 2, 4, 96, 40), (4097, 1, 1, 64, 20), (3000, 4, 600, 160, 33),
                                       (1100, 8, 40, 288, 70), (1000, 64, 4096, 32, 20)])
def test_many_assignments(T, k, E, K, N, dtype, group):
    g = torch.Generator().manual_seed(T + k)
    product(g, T, k, E, K, N, dtype, choices(g, T, k, E, 0.1), F32, group)
    product(g, T, k, E, K, N, dtype, choices(g, T, k, E, 0.1), BF16, group, combine=1, per_choice=1, gelu=1)


@pytest.mark.parametrize("E", [8, 512])
def test_many_assignments_of_uneven_experts(E):
    """One expert has every token, most have none; all choices missing; and the last expert alone."""
    g = torch.Generator().manual_seed(E)
    T, k = 3000, 2
    idx = torch.full((T, k), E - 1, dtype=torch.int32)
    idx[:, 1] = torch.arange(T) % 3
    idx[::7, 1] = -1
    product(g, T, k, E, 64, 40, BF16, idx)
    product(g, T, k, E, 64, 40, BF16, idx, combine=1)
    idx.fill_(E)
    product(g, T, k, E, 64, 40, BF16, idx)
    idx.fill_(E - 1)
    product(g, T, k, E, 64, 40, BF16, idx, per_choice=1)


def test_many_rows_of_one_expert_need_no_list():
    T, K, N = 5000, 64, 40
    g = torch.Generator().manual_seed(1)
    Wq, Ws = torch.randint(0, 256, (1, N, K // 2), generator=g, dtype=torch.uint8).to(DEV), torch.full((1, N, K // 32), 127, dtype=torch.uint8, device=DEV)
    x = torch.randn((T, K), generator=g).to(torch.bfloat16).to(DEV)
    cfg = B.make_w4_config(T, 1, 1, K, N, BF16, F32)
    alone, listed = torch.empty((T, N), device=DEV), torch.empty((T, N), device=DEV)
    B.moe_w4_product(cfg, x, None, None, None, Wq, Ws, alone, None)
    scratch = torch.empty(B.moe_w4_scratch_bytes(cfg), dtype=torch.uint8, device=DEV)
    B.moe_w4_product(cfg, x, None, torch.zeros((T, 1), dtype=torch.int32, device=DEV), None, Wq, Ws, listed, scratch)
    assert torch.equal(alone, listed)


def test_the_list_in_a_graph_and_on_another_stream():
    T, k, E, K, N = 3000, 2, 8, 96, 40
    g = torch.Generator().manual_seed(2)
    Wq = torch.randint(0, 256, (E, N, K // 2), generator=g, dtype=torch.uint8).to(DEV)
    Ws = torch.randint(121, 133, (E, N, K // 32), generator=g, dtype=torch.uint8).to(DEV)
    x, w = torch.randn((T, K), generator=g).to(torch.bfloat16).to(DEV), torch.rand((T, k), generator=g).to(DEV)
    idx = choices(g, T, k, E, 0.1).to(DEV)
    cfg = B.make_w4_config(T, k, E, K, N, BF16, BF16, combine=1)
    y, scratch = torch.empty((T, N), device=DEV, dtype=torch.bfloat16), torch.empty(B.moe_w4_scratch_bytes(cfg), dtype=torch.uint8, device=DEV)
    call = lambda s=None: B.moe_w4_product(cfg, x, None, idx, w, Wq, Ws, y, scratch, s)  # noqa: E731
    call()
    torch.cuda.synchronize()
    first = y.clone()
    side = torch.cuda.Stream()
    y.zero_()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert torch.equal(y, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        y.zero_(), scratch.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, first)
        call()
        torch.cuda.synchronize()
        assert torch.equal(y, first)
