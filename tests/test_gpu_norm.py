"""The norm and its backward pass against the formulas in 64 bits.

Tolerances count roundings.  A float result y = h * rstd * gain carries one each for the sum of the residual, the two
products, the mean, eps, root and quotient, and half of the relative error of the sum of squares, whose terms are positive:
at most 64 added in a row, 6 levels of lanes and 16 wavefronts, so 64 * 2^-24 covers all of it, relative to the value.  Storing it
adds eps / 2 of the type.  A gradient's terms have both signs, so its errors are relative to the sum of magnitudes."""
import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16, B.MOE_E4M3: torch.float8_e4m3fn}
FLOAT = 64 * 2.0 ** -24
F32, BF16, E4M3 = B.MOE_F32, B.MOE_BF16, B.MOE_E4M3


def half_step(dtype):
    return {F32: 2.0 ** -24, BF16: 2.0 ** -8}[dtype]


def rows(g, T, M, dtype, ld=None, offset=0):
    """[T, M] with row stride ld, `offset` elements into its memory."""
    ld = ld or M
    flat = torch.randn(offset + T * ld + M, generator=g).to(DT[dtype]).to(DEV)
    return torch.as_strided(flat, (T, M), (ld, 1), offset)


def empty_rows(T, M, dtype, ld=None, offset=0, fill=7.0):
    ld = ld or M
    flat = torch.full((offset + T * ld + M,), fill, device=DEV).to(DT[dtype])
    return flat, torch.as_strided(flat, (T, M), (ld, 1), offset)


def reference(x, r, gain, eps):
    h = x.double() + (r.double() if r is not None else 0.0)
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + eps)
    y = h * rstd[:, None] * (gain.double() if gain is not None else 1.0)
    return h, rstd, y


def check_e4m3(q, scales, y, group):
    M = y.shape[1]
    cols = group or M
    for c in range(0, M, cols):
        part = y[:, c:c + cols]
        want = torch.clamp(part.abs().amax(1) / 448.0, min=2.0 ** -126)
        got = scales[:, c // cols].double()
        assert ((got - want).abs() <= want * FLOAT).all()
        off = (q[:, c:c + cols].double() * got[:, None] - part).abs()
        # half a step of the value, or of the least normal number's values
        assert (off <= part.abs() * (2.0 ** -4 + 2 * FLOAT) + got[:, None] * 2.0 ** -10 * (1 + 2 * FLOAT)).all()


SIZES = [(1, 1), (1, 7), (3, 8), (5, 64), (4, 129), (2, 512), (7, 777), (1, 1024), (9, 1031), (3, 2048), (2, 2056), (5, 4040),
         (1, 4097), (2, 8192), (1, 8200), (2, 16385), (1, 32768), (300, 72)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,M", SIZES)
def test_forward(T, M, dtype):
    g = torch.Generator().manual_seed(T * 100003 + M)
    x, gain = rows(g, T, M, dtype), (1 + 0.3 * torch.randn(M, generator=g)).to(DEV)
    for residual, weights in ((True, True), (False, True), (True, False)):
        r = rows(g, T, M, dtype) if residual else None
        h = torch.empty_like(x)
        y, rstd = torch.empty_like(x), torch.empty(T, device=DEV)
        B.moe_norm_fwd(B.make_norm_config(T, M, 1e-5, dtype), x, r, gain if weights else None, h, y, None, rstd)
        H, R, Y = reference(x, r, gain if weights else None, float(np.float32(1e-5)))
        assert ((h.double() - H).abs() <= H.abs() * half_step(dtype)).all()
        assert ((rstd.double() - R).abs() <= R * FLOAT).all()
        assert ((y.double() - Y).abs() <= Y.abs() * (half_step(dtype) + FLOAT)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("T,M", [(1, 1), (1, 127), (3, 128), (5, 129), (4, 777), (2, 2048), (3, 4040), (1, 8192), (2, 20000)])
def test_forward_in_8_bits(T, M, group, dtype):
    g = torch.Generator().manual_seed(T + M)
    x, r, gain = rows(g, T, M, dtype), rows(g, T, M, dtype), (1 + 0.3 * torch.randn(M, generator=g)).to(DEV)
    x[:, ::97] *= 40.0                                             # columns far above the others
    flat, q = torch.full((T * M + 16,), 0x55, dtype=torch.uint8, device=DEV), None
    q = flat[:T * M].view(T, M)
    scales = torch.empty((T, -(-M // 128) if group else 1), device=DEV)
    B.moe_norm_fwd(B.make_norm_config(T, M, 1e-6, dtype, E4M3, group), x, r, gain, None, q, scales, None)
    check_e4m3(q.view(torch.float8_e4m3fn), scales, reference(x, r, gain, float(np.float32(1e-6)))[2], group)
    assert (flat[T * M:] == 0x55).all()


def test_rows_that_lie_apart_at_any_alignment_and_nothing_written_between_them():
    g = torch.Generator().manual_seed(3)
    T, M = 6, 203
    for dtype in (F32, BF16):
        x, r = rows(g, T, M, dtype, 211, 1), rows(g, T, M, dtype, 205, 3)
        hf, h = empty_rows(T, M, dtype, 220, 5)
        yf, y = empty_rows(T, M, dtype, 204, 1)
        B.moe_norm_fwd(B.make_norm_config(T, M, 1e-6, dtype, ldx=211, ldr=205, ldh=220, ldy=204), x, r, None, h, y)
        H, _, Y = reference(x, r, None, 1e-6)
        assert ((h.double() - H).abs() <= H.abs() * half_step(dtype)).all()
        assert ((y.double() - Y).abs() <= Y.abs() * (half_step(dtype) + FLOAT)).all()
        for flat, view in ((hf, h), (yf, y)):
            view.fill_(7.0)
            assert (flat == 7.0).all()


def test_h_in_place_of_either_input():
    g = torch.Generator().manual_seed(4)
    T, M = 37, 1500
    for which in (0, 1):
        x, r = rows(g, T, M, BF16), rows(g, T, M, BF16)
        H, _, Y = reference(x, r, None, 1e-6)
        y = torch.empty_like(x)
        B.moe_norm_fwd(B.make_norm_config(T, M), x, r, None, (x, r)[which], y)
        assert (((x, r)[which].double() - H).abs() <= H.abs() * 2.0 ** -8).all()
        assert ((y.double() - Y).abs() <= Y.abs() * (2.0 ** -8 + FLOAT)).all()


def test_zeros_infinities_and_nan_stay_in_their_rows():
    T, M = 6, 300
    x = torch.randn((T, M), generator=torch.Generator().manual_seed(5)).to(DEV)
    x[1] = 0.0
    x[2, 7] = float("inf")
    x[3, 299] = float("nan")
    y, rstd = torch.empty_like(x), torch.empty(T, device=DEV)
    B.moe_norm_fwd(B.make_norm_config(T, M, 0.0, F32), x, None, None, None, y, None, rstd)
    assert torch.isfinite(y[[0, 4, 5]]).all()
    assert rstd[1].isinf() and y[1].isnan().all()                   # eps = 0: 0 * inf, as the formula has it
    assert rstd[2] == 0 and y[2, 7].isnan() and (y[2, :7] == 0).all()
    assert y[3].isnan().all()
    B.moe_norm_fwd(B.make_norm_config(T, M, 1e-6, F32), x, None, None, None, y, None, rstd)
    assert (y[1] == 0).all()
    q, s = torch.empty((T, M), dtype=torch.uint8, device=DEV), torch.empty((T, 3), device=DEV)
    B.moe_norm_fwd(B.make_norm_config(T, M, 1e-6, F32, E4M3, 128), x, None, None, None, q, s)
    v = q.view(torch.float8_e4m3fn).float()
    assert (v[1] == 0).all() and (s[1] == 2.0 ** -126).all()        # a row of zeros has the least scale
    assert v[3].isnan().all() and s[3].isnan().all()
    assert s[2, 0].isnan() and v[2, :128].isnan().all() and (v[2, 128:] == 0).all()
    gain = torch.ones(M, device=DEV)
    gain[130] = float("nan")
    B.moe_norm_fwd(B.make_norm_config(T, M, 1e-6, F32, E4M3, 128), x, None, gain, None, q, s)
    v = q.view(torch.float8_e4m3fn).float()
    assert torch.isfinite(v[0, :128]).all() and v[0, 128:256].isnan().all() and torch.isfinite(v[0, 256:]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,M", SIZES + [(5000, 136)])
def test_backward(T, M, dtype):
    g = torch.Generator().manual_seed(T * 7 + M)
    h, dy, dh = (rows(g, T, M, dtype) for _ in range(3))
    gain = (1 + 0.3 * torch.randn(M, generator=g)).to(DEV)
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
    before = torch.randn(M, generator=g).to(DEV)
    for with_dh, weights, overwrite in ((True, True, 1), (False, True, 0), (True, False, 0)):
        cfg = B.make_norm_config(T, M, 1e-6, dtype, grad_overwrite=overwrite)
        need = B.moe_norm_scratch_bytes(cfg)
        scratch = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device=DEV)
        dx, dgain = torch.empty_like(h), before.clone()
        if overwrite:
            dgain.fill_(float("nan"))
        B.moe_norm_bwd(cfg, dy, h, gain if weights else None, rstd, dh if with_dh else None, dx, dgain, scratch)
        n, r = h.double() * rstd.double()[:, None], rstd.double()[:, None]
        up = dy.double() * (gain.double() if weights else 1.0)
        plus = dh.double() if with_dh else torch.zeros_like(n)
        want = plus + r * (up - n * (up * n).mean(1, keepdim=True))
        size = plus.abs() + r * (up.abs() + n.abs() * (up * n).abs().mean(1, keepdim=True))
        assert ((dx.double() - want).abs() <= want.abs() * half_step(dtype) + 2 * FLOAT * size).all()
        dg = (dy.double() * n).sum(0) + (0.0 if overwrite else before.double())
        size = (dy.double() * n).abs().sum(0) + (0.0 if overwrite else before.double().abs())
        # additions in a row: a wavefront's rows, a column's share of the partial sums, and the joins
        assert ((dgain.double() - dg).abs() <= (T / 1024 + 100) * 2.0 ** -24 * size).all()
        assert (scratch[need:] == 0xAB).all()


def test_backward_strides_in_place_and_without_gain_gradient():
    g = torch.Generator().manual_seed(9)
    T, M = 70, 301
    h, dy, dh = rows(g, T, M, BF16, 303, 1), rows(g, T, M, BF16, 310, 3), rows(g, T, M, BF16, 303, 5)
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
    flat, dx = empty_rows(T, M, BF16, 305, 1)
    cfg = B.make_norm_config(T, M, ldx=305, ldh=303, ldy=310)
    B.moe_norm_bwd(cfg, dy, h, None, rstd, dh, dx, None, None)
    again = dy.clone(memory_format=torch.preserve_format)
    same = torch.as_strided(torch.empty(T * 310 + M, dtype=torch.bfloat16, device=DEV), (T, M), (310, 1))
    same.copy_(again)
    B.moe_norm_bwd(B.make_norm_config(T, M, ldx=310, ldh=303, ldy=310), same, h, None, rstd, dh, same, None, None)
    assert torch.equal(same, dx)
    dx.fill_(7.0)
    assert (flat == 7.0).all()


def test_backward_of_no_tokens_stores_a_zero_gradient():
    for overwrite, left in ((1, 0.0), (0, 5.0)):
        dgain = torch.full((70,), 5.0, device=DEV)
        B.moe_norm_bwd(B.make_norm_config(0, 70, grad_overwrite=overwrite), None, None, None, None, None, None, dgain, None)
        assert (dgain == left).all()


def test_gradients_against_differences():
    g = torch.Generator().manual_seed(11)
    T, M, eps = 3, 40, 1e-3
    x, r, gain, up = (torch.randn(s, generator=g, dtype=torch.float64).float().double() for s in ((T, M), (T, M), (M,), (T, M)))

    def loss(x, gain):
        h = x + r
        return float((up * h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * gain).sum())

    f = lambda v: v.float().to(DEV)  # noqa: E731
    h, y, rstd = f(x).clone(), f(x).clone(), torch.empty(T, device=DEV)
    cfg = B.make_norm_config(T, M, eps, F32, grad_overwrite=1)
    B.moe_norm_fwd(cfg, f(x), f(r), f(gain), h, y, None, rstd)
    dx, dgain = torch.empty_like(h), torch.empty(M, device=DEV)
    scratch = torch.empty(B.moe_norm_scratch_bytes(cfg) + 4, dtype=torch.uint8, device=DEV)
    B.moe_norm_bwd(cfg, f(up), h, f(gain), rstd, None, dx, dgain, scratch)
    step = 1e-5                                                     # error step^2 / 6 of third derivatives of order one, plus 1e-16 / step
    for i in range(T):
        for c in range(0, M, 7):
            d = torch.zeros_like(x)
            d[i, c] = step
            num = (loss(x + d, gain) - loss(x - d, gain)) / (2 * step)
            assert abs(num - float(dx[i, c])) <= 1e-4
    for c in range(0, M, 5):
        d = torch.zeros_like(gain)
        d[c] = step
        assert abs((loss(x, gain + d) - loss(x, gain - d)) / (2 * step) - float(dgain[c])) <= 1e-4


def test_the_same_bits_every_time_on_another_stream_and_in_a_graph():
    g = torch.Generator().manual_seed(12)
    T, M = 3000, 640
    x, r, dy = (rows(g, T, M, BF16) for _ in range(3))
    gain = torch.randn(M, generator=g).to(DEV)
    cfg = B.make_norm_config(T, M, grad_overwrite=1)
    scratch = torch.empty(B.moe_norm_scratch_bytes(cfg), dtype=torch.uint8, device=DEV)
    out = [torch.empty_like(x), torch.empty_like(x), torch.empty(T, device=DEV), torch.empty_like(x), torch.empty(M, device=DEV)]

    def both(stream=None):
        B.moe_norm_fwd(cfg, x, r, gain, out[0], out[1], None, out[2], stream)
        B.moe_norm_bwd(cfg, dy, out[0], gain, out[2], None, out[3], out[4], scratch, stream)

    both()
    torch.cuda.synchronize()
    first = [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o in out:
        o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, first))
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, first))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,M", [(2, 64), (5, 513), (40, 260), (512, 1031), (300, 2048), (37, 9000), (513, 88)])
def test_backward_where_the_gradient_overwrites_dy(T, M, dtype):
    """The gain's gradient is of dy as it was, whether dx is dy or not, stored and accumulated."""
    g = torch.Generator().manual_seed(T + M)
    h, dy = rows(g, T, M, dtype), rows(g, T, M, dtype)
    gain = (1 + 0.3 * torch.randn(M, generator=g)).to(DEV)
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
    n = h.double() * rstd.double()[:, None]
    want, size = (dy.double() * n).sum(0), (dy.double() * n).abs().sum(0)
    tol = (T / 64 + 100) * 2.0 ** -24
    for overwrite in (1, 0):
        cfg = B.make_norm_config(T, M, 1e-6, dtype, grad_overwrite=overwrite)
        scratch = torch.empty(B.moe_norm_scratch_bytes(cfg) + 4, dtype=torch.uint8, device=DEV)
        old = 0.0 if overwrite else 3.0
        out, apart, same = torch.empty_like(h), torch.full((M,), 3.0, device=DEV), torch.full((M,), 3.0, device=DEV)
        B.moe_norm_bwd(cfg, dy, h, gain, rstd, None, out, apart, scratch)
        both = dy.clone()
        B.moe_norm_bwd(cfg, both, h, gain, rstd, None, both, same, scratch)
        assert torch.equal(both, out)
        for got in (apart, same):
            assert ((got.double() - old - want).abs() <= tol * (size + old)).all()
