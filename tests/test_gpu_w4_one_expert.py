"""4-bit products without topk_idx: all rows have expert 0, whatever the number of experts."""
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T,k,combine", [(8, 1, 0), (6, 2, 1), (16, 1, 0), (2, 1, 0), (40, 1, 1)])
def test_the_number_of_experts_does_not_matter(T, k, combine):
    """The same bits as with one expert: the same kernel, which reads the matrix once for all tokens where that pays.  Planned as
    if the tokens chose among 16 experts, eight of them went through the matrix one by one."""
    E, K, N = 16, 2048, 8192
    g = torch.Generator(device=DEV).manual_seed(T)
    Wq = torch.randint(0, 256, (E, N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    Ws = torch.randint(121, 133, (E, N, K // 32), generator=g, device=DEV, dtype=torch.uint8)
    x = torch.randn((T, K), generator=g, device=DEV).to(torch.bfloat16)
    out = []
    for experts in (k, E):                                  # (k <= E)
        cfg = B.make_w4_config(T, k, experts, K, N, B.MOE_BF16, B.MOE_F32, combine=combine)
        y = torch.empty((T if combine else T * k, N), device=DEV)
        scratch = torch.empty(B.moe_w4_scratch_bytes(cfg) + 16, dtype=torch.uint8, device=DEV)
        B.moe_w4_product(cfg, x, None, None, None, Wq, Ws, y, scratch)
        out.append(y)
    assert torch.equal(*out)
