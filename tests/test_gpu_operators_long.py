"""More rows than one launch has threads for."""
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_norm_of_more_rows_than_a_launch():
    """Rows of one wavefront, 2^26 of them and some: the pattern of the first 4099 rows over and over."""
    part, times, M = 4099, 16373, 8
    T = part * times
    assert T > 1 << 26
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.randn((part, M), generator=g, device=DEV).to(torch.bfloat16)
    want, rstd = torch.empty_like(x), torch.empty(part, device=DEV)
    B.moe_norm_fwd(B.make_norm_config(part, M), x, None, None, None, want, None, rstd)
    y, all_rstd = torch.zeros((T, M), dtype=torch.bfloat16, device=DEV), torch.zeros(T, device=DEV)
    B.moe_norm_fwd(B.make_norm_config(T, M), x.repeat(times, 1), None, None, None, y, None, all_rstd)
    values, factors = torch.equal(y.view(times, part, M), want.expand(times, part, M)), torch.equal(all_rstd.view(times, part), rstd.expand(times, part))
    assert values and factors


def test_norm_of_wide_rows_in_several_launches():
    """Sixteen wavefronts to a row: 2^21 rows to a launch."""
    T, M = (1 << 21) + 37, 4097
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((64, M), generator=g, device=DEV).to(torch.bfloat16).repeat(-(-T // 64), 1)[:T]
    rstd, few = torch.zeros(T, device=DEV), torch.empty(64, device=DEV)
    y = torch.empty((T, M), dtype=torch.bfloat16, device=DEV)
    B.moe_norm_fwd(B.make_norm_config(64, M), x, None, None, None, y, None, few)
    first = y[:64].clone()
    B.moe_norm_fwd(B.make_norm_config(T, M), x, None, None, None, y, None, rstd)
    factors = torch.equal(rstd, few.repeat(-(-T // 64))[:T])
    assert factors
    for at in (0, (1 << 21) - 64, 1 << 21):
        n = min(64, T - at)
        assert torch.equal(y[at:at + n].view(torch.int16), first[:n].view(torch.int16))


def test_router_of_more_tokens_than_a_launch():
    part, times = 16411, 16381
    T = part * times
    assert T > 1 << 28
    l = torch.randn((part, 1), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(torch.bfloat16)
    all_l = l.repeat(times, 1)
    kw = dict(scores=B.MOE_SIGMOID, dtype=B.MOE_BF16)
    idx, w = torch.full((T,), -9, dtype=torch.int32, device=DEV), torch.zeros(T, device=DEV)
    load = torch.zeros(1, dtype=torch.int32, device=DEV)
    few_idx, few_w = torch.empty(part, dtype=torch.int32, device=DEV), torch.empty(part, device=DEV)
    B.moe_router_fwd(B.make_router_config(part, 1, 1, **kw), l, None, few_idx, few_w)
    B.moe_router_fwd(B.make_router_config(T, 1, 1, **kw), all_l, None, idx, w, load)
    # (outside the asserts: a failing one would go through the tensors element by element)
    chosen, weights = bool((idx == 0).all()), torch.equal(w.view(times, part), few_w.expand(times, part))
    assert chosen and weights and load.item() == T
    dw, dl, few_dl = torch.ones(T, device=DEV), torch.zeros_like(all_l), torch.empty_like(l)
    B.moe_router_bwd(B.make_router_config(part, 1, 1, **kw), l, few_idx, dw, few_dl)
    B.moe_router_bwd(B.make_router_config(T, 1, 1, **kw), all_l, idx, dw, dl)
    gradients = torch.equal(dl.view(times, part), few_dl[:, 0].expand(times, part))
    assert gradients and (few_dl != 0).any()
