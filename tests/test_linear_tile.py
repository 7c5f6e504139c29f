"""Which tile a dense product has, asked on the host."""
import ctypes

import pytest

from paper_2506_22175_amd import binding as B


def test_refusals():
    v = [ctypes.c_int32(7) for _ in range(3)]
    at = [ctypes.byref(n) for n in v]
    ask = B.lib().moe_linear_tile
    cfg = B.make_linear_config(64, 64, 64)
    assert ask(None, 0, *at) == 1
    for missing in range(3):
        assert ask(ctypes.byref(cfg), 0, *[None if i == missing else a for i, a in enumerate(at)]) == 1
    for gemm in (-1, 3):
        assert ask(ctypes.byref(cfg), gemm, *at) == 2
    assert ask(ctypes.byref(B.make_linear_config(64, 60, 64)), 0, *at) == 3
    assert [n.value for n in v] == [7, 7, 7]
    assert all(B.moe_linear_tile(B.make_linear_config(0, 64, 64), gemm) == (0, 0, 0) for gemm in B.LINEAR_GEMMS)


@pytest.mark.parametrize("dtype,cols", [(B.MOE_F32, 64), (B.MOE_BF16, 128)])
def test_few_rows(dtype, cols):
    for T in (1, 16, 17, 32):
        assert B.moe_linear_tile(B.make_linear_config(T, 520, 1000, dtype), "fwd") == (16 if T <= 16 else 32, cols, 1)
        assert B.moe_linear_tile(B.make_linear_config(T, 8192, 2048, dtype), "fwd")[2] > 1


def test_the_scratch_holds_every_partial_sum():
    for T, K, N in ((1, 8192, 2048), (64, 8192, 2048), (30011, 520, 1000), (40, 72, 8192), (130, 4104, 520), (1000, 64, 64), (8192, 2048, 8192)):
        for dtype in (B.MOE_F32, B.MOE_BF16):
            cfg = B.make_linear_config(T, K, N, dtype)
            for gemm, size in (("fwd", T * N), ("dx", T * K), ("dW", K * N)):
                sums = B.moe_linear_tile(cfg, gemm)[2]
                assert sums >= 1 and (sums == 1 or 4 * sums * size <= B.moe_linear_scratch_bytes(cfg))


@pytest.mark.parametrize("act", [B.MOE_ACT_NONE, B.MOE_ACT_GELU])
@pytest.mark.parametrize("T,K,N", [(909, 1328, 80), (1664, 5584, 432), (42, 1256, 72), (1172, 4680, 568), (171, 1592, 816), (84, 2976, 5600), (911, 2848, 400)])
def test_long_sums_of_few_tiles_go_in_slices(T, K, N, act):
    """Weighed against the launch there would be without slices, and not one in tiles that the epilogue does not have (11.5 us against 9.3
    with slices, 36.5 and 28.1, 11.7 and 8.7, 33.4 and 26.5, 14.3 and 10.9, 22.7 and 16.1, 21.4 and 15.5)."""
    assert B.moe_linear_tile(B.make_linear_config(T, K, N, B.MOE_BF16, act), "fwd")[2] > 1
