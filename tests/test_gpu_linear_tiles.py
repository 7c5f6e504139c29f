"""The dense product's epilogues, input gradients and weight gradients in every tile that a batch may choose, with rows and columns that end
inside the last one: against 64 bits, within the bounds that test_gpu_linear.py derives.  The library is asked which tile it is, so that
a change of the choice does not leave a tile without a test."""
import pytest
import torch

from paper_2506_22175_amd import binding as B
from test_gpu_linear import D, DT, HALF, U, _apart, _forward, _scratch, _untouched, test_activation_backward as _activation_backward

pytestmark = pytest.mark.gpu
NONE, GELU, SILU = B.MOE_ACT_NONE, B.MOE_ACT_GELU, B.MOE_ACT_SILU
BF16 = B.MOE_BF16


# (tile's rows, columns, partial sums), T, K, N, activations that choose it
FORWARD = [
    ((256, 256, 1), 2965, 200, 4112, (NONE, GELU, SILU)), ((256, 256, 1), 6761, 200, 1200, (NONE,)), ((256, 256, 1), 8192, 512, 2048, (SILU,)),
    ((256, 256, 1), 33064, 472, 136, (GELU,)), ((256, 128, 1), 16669, 840, 136, (NONE,)), ((256, 128, 1), 34058, 7648, 72, (GELU, SILU)),
    ((128, 128, 1), 9959, 360, 144, (NONE, GELU, SILU)), ((64, 128, 1), 299, 376, 88, (NONE, GELU, SILU)),
    ((64, 64, 10), 67, 3128, 80, (GELU,)), ((64, 128, 2), 72, 2032, 6480, (SILU,)), ((128, 128, 3), 65, 1816, 6896, (NONE,)),
]


@pytest.mark.parametrize("parts", ["", "b", "r", "z", "brz"])
@pytest.mark.parametrize("tile,T,K,N,act", [(t, T, K, N, a) for t, T, K, N, acts in FORWARD for a in acts])
def test_forward(tile, T, K, N, act, parts):
    for apart in (0, 8) if parts in ("", "brz") else (8,):
        cfg = B.make_linear_config(T, K, N, BF16, act, ldx=K + apart, ldr=N + 2 * apart, ldz=N + apart, ldy=N + 3 * apart)
        assert B.moe_linear_tile(cfg, "fwd") == tile
        _forward(T, K, N, BF16, act, "b" in parts, "r" in parts, "z" in parts, apart)


@pytest.mark.parametrize("tile,T,K,N,act", [(t, T, K, N, acts[-1]) for t, T, K, N, acts in FORWARD])
def test_the_residual_may_be_the_output(tile, T, K, N, act):
    g = torch.Generator(device=D).manual_seed(T)
    x, r = (torch.randn(s, generator=g, device=D).to(DT[BF16]) for s in ((T, K), (T, N)))
    W, b = (torch.randn((K, N), generator=g, device=D) * K ** -0.5).to(DT[BF16]), torch.randn(N, generator=g, device=D)
    cfg = B.make_linear_config(T, K, N, BF16, act)
    assert B.moe_linear_tile(cfg, "fwd") == tile
    apart, scratch = torch.empty_like(r), _scratch(cfg)
    B.moe_linear_fwd(cfg, x, W, b, r, None, apart, scratch)
    B.moe_linear_fwd(cfg, x, W, b, r, None, r, scratch)
    assert torch.equal(r, apart)


DX = [((256, 256, 1), 18999, 400, 200), ((256, 256, 1), 4096, 4096, 1024), ((256, 128, 1), 4100, 4104, 1024), ((256, 128, 1), 12529, 304, 200), ((128, 128, 1), 10053, 144, 208),
      ((64, 128, 1), 47, 200, 488), ((64, 128, 3), 189, 80, 1184), ((128, 128, 5), 2767, 136, 4384)]


@pytest.mark.parametrize("apart", [0, 8])
@pytest.mark.parametrize("tile,T,K,N", DX)
def test_input_gradient(tile, T, K, N, apart):
    """Alone, and with what reaches x past the product, in its place or another."""
    g = torch.Generator(device=D).manual_seed(T + K + N)
    dz, W = _apart(T, N, N + apart, DT[BF16], g, 9.0)[1], torch.randn((K, N), generator=g, device=D).to(DT[BF16])
    cfg = B.make_linear_config(T, K, N, BF16, ldx=K + apart, ldz=N + apart)
    assert B.moe_linear_tile(cfg, "dx") == tile
    scratch = _scratch(cfg)
    add = _apart(T, K, K + apart, DT[BF16], g, 9.0)[1]
    add.mul_(30.0)
    Z, V, A = dz.double(), W.double(), add.double()
    product, size = Z @ V.t(), Z.abs() @ V.abs().t()
    for more in (None, add):
        flat, dx = _apart(T, K, K + apart, DT[BF16], g, 7.0)
        dx.fill_(float("nan"))
        B.moe_linear_bwd(cfg, dz, None, W, dx, None, scratch, add=more)
        want, err = (product, 2 * (N + 20) * U * size) if more is None else (product + A, 2 * (N + 20) * U * (size + A.abs()))
        assert ((dx.double() - want).abs() <= err + HALF[BF16] * (want.abs() + err)).all()
        assert _untouched(flat, dx, 7.0) and (scratch[-64:] == 0xAB).all()
    B.moe_linear_bwd(cfg, dz, None, W, add, None, scratch, add=add)
    assert torch.equal(add, dx)


DW = [((256, 256, 1), 201, 1928, 6616), ((256, 128, 4), 5426, 136, 6568), ((256, 128, 4), 5362, 6544, 144),
      ((256, 128, 2), 4096, 1024, 4096), ((128, 128, 1), 183, 88, 152), ((128, 128, 3), 2100, 200, 8200)]


@pytest.mark.parametrize("overwrite", [0, 1])
@pytest.mark.parametrize("apart", [0, 8])
@pytest.mark.parametrize("tile,T,K,N", DW)
def test_weight_gradient(tile, T, K, N, apart, overwrite):
    g = torch.Generator(device=D).manual_seed(T + K + N)
    x, dz = _apart(T, K, K + apart, DT[BF16], g, 9.0)[1], _apart(T, N, N + apart, DT[BF16], g, 9.0)[1]
    cfg = B.make_linear_config(T, K, N, BF16, NONE, overwrite, ldx=K + apart, ldz=N + apart)
    assert B.moe_linear_tile(cfg, "dW") == tile
    scratch = _scratch(cfg)
    flat = torch.full((K * N + 32,), float("nan") if overwrite else 2.0, device=D)
    dW = flat[16:-16].view(K, N)
    flat[:16] = flat[-16:] = 7.0
    B.moe_linear_bwd(cfg, dz, x, None, None, dW, scratch)
    X, Z, old = x.double(), dz.double(), 0.0 if overwrite else 2.0
    assert ((dW.double() - old - X.t() @ Z).abs() <= 2 * (T + 20) * U * (X.abs().t() @ Z.abs() + old)).all()
    assert (flat[:16] == 7.0).all() and (flat[-16:] == 7.0).all() and (scratch[-64:] == 0xAB).all()


@pytest.mark.parametrize("dtype,T,N", [(B.MOE_BF16, 8201, 8200), (B.MOE_F32, 4105, 8200)])
@pytest.mark.parametrize("act", [NONE, GELU, SILU])
def test_activation_backward_past_the_caches(dtype, T, N, act):
    """dz of more than 128 MiB, in its own memory and in dy's or z's."""
    assert T * N * (2 if dtype == B.MOE_BF16 else 4) > 128 << 20
    _activation_backward(T, N, act, dtype)


@pytest.mark.parametrize("T,K,N", [(5, 136, 264), (20, 4104, 72), (299, 376, 88), (67, 3128, 80), (9959, 360, 144), (2965, 200, 4112)])
@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
def test_float_vectors_may_begin_anywhere(T, K, N, dtype):
    """The bias and its gradient, a float behind a multiple of 16 bytes, with guards about the gradient."""
    g = torch.Generator(device=D).manual_seed(T)
    x, dy = (torch.randn(s, generator=g, device=D).to(DT[dtype]) for s in ((T, K), (T, N)))
    W, b = (torch.randn((K, N), generator=g, device=D) * K ** -0.5).to(DT[dtype]), torch.randn(N + 1, generator=g, device=D)
    cfg = B.make_linear_config(T, K, N, dtype, SILU, 1)
    scratch, db = _scratch(cfg), torch.full((2, N + 2), 7.0, device=D)
    out = [[torch.empty((T, N), device=D, dtype=DT[dtype]) for _ in range(3)] for _ in range(2)]
    for (z, y, dz), bias, d in zip(out, (b[1:], b[1:].clone()), (db[0, 1:-1], db[1, :-2])):
        B.moe_linear_fwd(cfg, x, W, bias, None, z, y, scratch)
        B.moe_act_bwd(cfg, dy, z, dz, d, scratch)
    assert all(torch.equal(p, q) for p, q in zip(*out)) and torch.equal(db[0, 1:-1], db[1, :-2])
    assert db[0, 0] == 7.0 and (db[:, -1] == 7.0).all() and db[1, -2] == 7.0 and not torch.equal(out[0][0], torch.zeros_like(out[0][0]))
