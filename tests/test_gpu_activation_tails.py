"""The dense product's activations where their results are small: relative bounds, down to the smallest normal numbers.

A result is rounded once to its type, half a step, on top of what the float computation is off by, relative to the result:
  GeLU, bfloat16   9.7e-5 of the fit; the exponent's argument, at most 128 ln 2, has three roundings of 2^-24 and the exponential, the
                   reciprocal and six more operations a step or two each: 89 * 3 * 2^-24 + 12 * 2^-23, below 2e-5
  GeLU, float      Phi(-a) by erfc at 0.7071 a, whose two roundings count a^2 times: (a^2 + 16) 2^-22"""
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
D = "cuda:0"
DT = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16}
HALF = {B.MOE_F32: 2.0 ** -24, B.MOE_BF16: 2.0 ** -8}
TINY = 2.0 ** -126


def _grid(T, lo, hi, dtype):
    """T rows of 64 values from lo to hi, as the type has them."""
    return torch.linspace(lo, hi, T * 64, dtype=torch.float64).reshape(T, 64).to(DT[dtype]).to(D)


def _forward(z, dtype, act):
    cfg = B.make_linear_config(z.shape[0], 64, 64, dtype, act)
    eye, y = torch.eye(64, device=D).to(z.dtype), torch.empty_like(z)
    scratch = torch.empty(B.moe_linear_scratch_bytes(cfg), dtype=torch.uint8, device=D)
    B.moe_linear_fwd(cfg, z, eye, None, None, None, y, scratch)
    return y.double()


def _check(got, want, off, dtype):
    """off: of the computation, relative"""
    normal = want.abs() > TINY
    err = (off + HALF[dtype] * (1 + off)) * want.abs()
    assert normal.sum() > normal.numel() // 2
    assert ((got - want).abs() <= err)[normal].all(), float(((got - want).abs() / want.abs() / err * want.abs())[normal].max())


# (rows: the few-row form, then the grouped GEMM's)
@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [17, 800])
def test_gelu_far_on_the_negative_side(T, dtype):
    z = _grid(T, -13.0, 0.0, dtype)
    Z = z.double()
    want = Z * torch.exp(torch.special.log_ndtr(Z))
    off = 1.2e-4 if dtype == B.MOE_BF16 else (Z * Z + 16) * 2.0 ** -22
    _check(_forward(z, dtype, B.MOE_ACT_GELU), want, off, dtype)
