"""The dense product's activations where their results are small: relative bounds, down to the smallest normal numbers.

A result is rounded once to its type, half a step, on top of what the float computation is off by, relative to the result:
  GeLU, bfloat16   9.7e-5 of the fit; the exponent's argument, at most 128 ln 2, has three roundings of 2^-24 and the exponential, the
                   reciprocal and six more operations a step or two each: 89 * 3 * 2^-24 + 12 * 2^-23, below 2e-5
  GeLU, float      Phi(-a) by erfc at 0.7071 a, whose two roundings count a^2 times: (a^2 + 16) 2^-22
  SiLU             the exponential's argument z / 2 has two roundings, which its square doubles (float), and some ten operations a step of 2^-23
                   each: (|z| + 16) 2^-22
  GeLU's slope     Phi + z phi, of which Phi is at most 1 / z^2: the fit's 4 % of Phi at -13, 0.4 % at -6 and 4e-6 at -1.5 are below 3e-4;
                   the exponential as above, and a difference that is at least half of its larger part, below -1.5: (z^2 + 16) 2^-20
  SiLU's slope     s (1 + z (1 - s)), whose second factor is at least half of its larger term, below -2.5: (|z| + 16) 2^-21"""
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


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [17, 800])
def test_silu_far_on_the_negative_side(T, dtype):
    """Of bfloat16 down to 1e-36, and not further off than that where results are smaller."""
    for lo, hi in ((-92.0, -80.0), (-92.0, 0.0)):
        z = _grid(T, lo, hi, dtype)
        Z = z.double()
        got, want = _forward(z, dtype, B.MOE_ACT_SILU), Z * torch.sigmoid(Z)
        kept = want.abs() > (1e-36 if dtype == B.MOE_BF16 else 0.0)
        _check(got[kept], want[kept], ((Z.abs() + 16) * 2.0 ** -22)[kept], dtype)
        assert ((got - want).abs()[~kept] <= 1e-36).all()


# (rows: few, with the bias's gradient, go another way than many)
@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [17, 800])
@pytest.mark.parametrize("act,lo,hi", [(B.MOE_ACT_GELU, -13.4, -12.9), (B.MOE_ACT_GELU, -13.4, -1.5), (B.MOE_ACT_SILU, -92.0, -86.0), (B.MOE_ACT_SILU, -92.0, -2.5)])
def test_slopes_far_on_the_negative_side(act, lo, hi, T, dtype):
    z = _grid(T, lo, hi, dtype)
    Z = z.double()
    if act == B.MOE_ACT_GELU:
        want = torch.exp(torch.special.log_ndtr(Z)) + Z * torch.exp(-0.5 * Z * Z) / (2 * torch.pi) ** 0.5
        off = (Z * Z + 16) * 2.0 ** -20 + (3e-4 if dtype == B.MOE_BF16 else 0.0)
    else:
        s = torch.sigmoid(Z)
        want, off = s * (1 + Z * torch.sigmoid(-Z)), (Z.abs() + 16) * 2.0 ** -21
    cfg = B.make_linear_config(T, 64, 64, dtype, act, 1)
    scratch = torch.empty(B.moe_linear_scratch_bytes(cfg), dtype=torch.uint8, device=D)
    dz, db = torch.empty_like(z), torch.empty(64, device=D) if T < 64 else None
    B.moe_act_bwd(cfg, torch.ones_like(z), z, dz, db, scratch)
    _check(dz.double(), want, off, dtype)
