"""The dense product with its epilogue, the activation's backward and the product's, against 64 bits.

u = 2^-24.  A float sum of n products is off by at most n roundings of 2 u of the sum of magnitudes (2: a matrix instruction may cut
where an addition would round); activations: the rational form of Phi is off by 1.5e-7 and its own roundings, 4e-7 |z| covers it; the
exponentials' arguments are rounded, 1e-6 |z| (1 + |z|)."""
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
D = "cuda:0"
DT = {B.MOE_F32: torch.float32, B.MOE_BF16: torch.bfloat16}
HALF = {B.MOE_F32: 2.0 ** -24, B.MOE_BF16: 2.0 ** -8}
U = 2.0 ** -24
ACTS = {B.MOE_ACT_NONE: lambda z: z, B.MOE_ACT_GELU: lambda z: z * torch.special.ndtr(z), B.MOE_ACT_SILU: lambda z: z * torch.sigmoid(z)}


def _act_error(z):
    return 1e-6 * z.abs() * (1 + z.abs())


def _apart(T, N, ld, dtype, g, pad):
    """Rows that lie `ld` apart in a buffer of `pad`, their values random; (buffer, rows)."""
    flat = torch.full((T * ld + 16,), pad, device=D).to(dtype)
    rows = torch.as_strided(flat, (T, N), (ld, 1), 8)
    rows.copy_(torch.randn((T, N), generator=g, device=D).to(dtype))
    return flat, rows


def _untouched(flat, rows, pad):
    keep = rows.clone()
    rows.fill_(pad)
    ok = bool((flat == pad).all())
    rows.copy_(keep)
    return ok


def _scratch(cfg):
    return torch.full((B.moe_linear_scratch_bytes(cfg) + 64,), 0xAB, dtype=torch.uint8, device=D)


def _forward(T, K, N, dtype, act, bias, residual, keep, apart=0):
    g = torch.Generator(device=D).manual_seed(T * 131 + K * 7 + N)
    dt = DT[dtype]
    W = (torch.randn((K, N), generator=g, device=D) * K ** -0.5).to(dt)
    x = _apart(T, K, K + apart, dt, g, 9.0)[1]
    b = torch.randn(N, generator=g, device=D) if bias else None
    r = _apart(T, N, N + 2 * apart, dt, g, 9.0)[1] if residual else None
    zf, z = _apart(T, N, N + apart, dt, g, 7.0) if keep else (None, None)
    yf, y = _apart(T, N, N + 3 * apart, dt, g, 7.0)
    cfg = B.make_linear_config(T, K, N, dtype, act, ldx=K + apart, ldr=N + 2 * apart, ldz=N + apart, ldy=N + 3 * apart)
    scratch = _scratch(cfg)
    B.moe_linear_fwd(cfg, x, W, b, r, z, y, scratch)
    X, V = x.double(), W.double()
    want = X @ V
    size = X.abs() @ V.abs()
    if bias:
        want, size = want + b.double(), size + b.double().abs()
    ez = 2 * (K + 20) * U * size
    out = ACTS[act](want)
    add = r.double() if residual else torch.zeros_like(out)
    err = 1.13 * ez + (_act_error(want) if act else 0) + 2 * U * (out.abs() + add.abs())
    assert ((y.double() - out - add).abs() <= err + HALF[dtype] * ((out + add).abs() + err)).all()
    if keep:
        assert ((z.double() - want).abs() <= ez + HALF[dtype] * (want.abs() + ez)).all()
        assert _untouched(zf, z, 7.0)
    assert _untouched(yf, y, 7.0)
    assert (scratch[-64:] == 0xAB).all()


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [1, 2, 8, 9, 16, 17, 31, 32, 33, 65, 200, 513])
@pytest.mark.parametrize("K,N", [(8, 8), (64, 64), (72, 136), (520, 1000), (1096, 264)])
def test_forward(T, K, N, dtype):
    i = (T + K) % 3
    _forward(T, K, N, dtype, (B.MOE_ACT_NONE, B.MOE_ACT_GELU, B.MOE_ACT_SILU)[i], bias=(T + N) % 2 == 0, residual=T % 3 != 1, keep=T % 2 == 1)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [1, 7, 20, 300])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("parts", ["", "b", "r", "z", "brz"])
def test_forward_epilogues_with_rows_that_lie_apart(T, act, parts, dtype):
    _forward(T, 200, 328, dtype, act, "b" in parts, "r" in parts, "z" in parts, apart=8)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T,K,N", [(1, 8192, 2048), (3, 2048, 8192), (32, 4096, 512), (1, 20000, 64), (1500, 512, 2048), (5000, 264, 520), (40, 8192, 264), (100, 5000, 72),
                                   (64, 2048, 2048), (130, 4104, 520)])
def test_forward_of_long_sums_and_many_rows(T, K, N, dtype):
    _forward(T, K, N, dtype, B.MOE_ACT_GELU, True, True, True)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [3, 300])
def test_the_residual_may_be_the_output(T, dtype):
    g = torch.Generator(device=D).manual_seed(T)
    K, N = 2048, 136
    x, W, r = (torch.randn(s, generator=g, device=D).to(DT[dtype]) for s in ((T, K), (K, N), (T, N)))
    cfg = B.make_linear_config(T, K, N, dtype)
    apart, scratch = torch.empty_like(r), _scratch(cfg)
    B.moe_linear_fwd(cfg, x, W, None, r, None, apart, scratch)
    B.moe_linear_fwd(cfg, x, W, None, r, None, r, scratch)
    assert torch.equal(r, apart)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [5, 100])
def test_infinities_and_nan_stay_in_their_rows_and_columns(T, dtype):
    K, N = 136, 200
    g = torch.Generator(device=D).manual_seed(T)
    x, W = torch.randn((T, K), generator=g, device=D).to(DT[dtype]), torch.randn((K, N), generator=g, device=D).to(DT[dtype])
    cfg, clean, y = B.make_linear_config(T, K, N, dtype, B.MOE_ACT_GELU), torch.empty((T, N), device=D, dtype=DT[dtype]), torch.empty((T, N), device=D, dtype=DT[dtype])
    scratch = _scratch(cfg)
    B.moe_linear_fwd(cfg, x, W, None, None, None, clean, scratch)
    x[1, 3], W[K - 1, 7], x[T - 1, K - 1] = float("nan"), float("inf"), float("inf")
    B.moe_linear_fwd(cfg, x, W, None, None, None, y, scratch)
    rows, cols = [t for t in range(T) if t not in (1, T - 1)], [n for n in range(N) if n != 7]
    assert torch.equal(y[rows][:, cols], clean[rows][:, cols])
    assert y[1].isnan().all() and not y[rows][:, 7].isfinite().logical_and(y[rows][:, 7].abs() > 1e-3).any()


def test_more_rows_than_32_bit_offsets_reach():
    T, K, N = 70000, 64, 16384
    g = torch.Generator(device=D).manual_seed(1)
    x, W = torch.randn((T, K), generator=g, device=D).to(torch.bfloat16), torch.randn((K, N), generator=g, device=D).to(torch.bfloat16)
    y = torch.full((T, N), float("nan"), device=D, dtype=torch.bfloat16)
    cfg = B.make_linear_config(T, K, N)
    scratch = _scratch(cfg)
    B.moe_linear_fwd(cfg, x, W, None, None, None, y, scratch)
    for t in (0, 1, 32767, 64255, 64256, 64511, 64512, 65535, 65536, 69999):
        want, size = x[t].double() @ W.double(), x[t].double().abs() @ W.double().abs()
        assert ((y[t].double() - want).abs() <= 2.0 ** -8 * want.abs() + 200 * U * size).all()
    assert y.isfinite().all()
    # back: y stands for dz
    dx, dW = torch.full((T, K), float("nan"), device=D, dtype=torch.bfloat16), torch.full((K, N), float("nan"), device=D)
    cfg = B.make_linear_config(T, K, N, grad_overwrite=1)
    B.moe_linear_bwd(cfg, y, x, W, dx, dW, scratch)
    for t in (0, 64255, 64256, 69999):
        want, size = W.double() @ y[t].double(), W.double().abs() @ y[t].double().abs()
        assert ((dx[t].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2 * N * U * size).all()
    cols = torch.tensor([0, 1, 8191, 16383], device=D)
    want, size = x.double().t() @ y[:, cols].double(), x.double().abs().t() @ y[:, cols].double().abs()
    assert ((dW[:, cols].double() - want).abs() <= 2 * T * U * size).all()


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
def test_more_rows_than_a_launch_of_floats_takes(dtype):
    T, K, N = 65535 // 4 * 256 + 70, 8, 16
    g = torch.Generator(device=D).manual_seed(2)
    x, dz = (torch.randn((T, n), generator=g, device=D).to(DT[dtype]) for n in (K, N))
    W = torch.randn((K, N), generator=g, device=D).to(DT[dtype])
    y, dx = torch.full((T, N), float("nan"), device=D, dtype=DT[dtype]), torch.full((T, K), float("nan"), device=D, dtype=DT[dtype])
    dW, db = torch.full((K, N), float("nan"), device=D), torch.full((N,), float("nan"), device=D)
    cfg = B.make_linear_config(T, K, N, dtype, grad_overwrite=1)
    scratch = _scratch(cfg)
    B.moe_linear_fwd(cfg, x, W, None, None, None, y, scratch)
    B.moe_linear_bwd(cfg, dz, x, W, dx, dW, scratch)
    B.moe_act_bwd(cfg, dz, None, None, db, scratch)
    X, Z, V = x.double(), dz.double(), W.double()
    for got, want, size in ((y, X @ V, X.abs() @ V.abs()), (dx, Z @ V.t(), Z.abs() @ V.t().abs())):
        err = 2 * (N + 20) * U * size
        assert ((got.double() - want).abs() <= err + HALF[dtype] * (want.abs() + err)).all()
    assert ((dW.double() - X.t() @ Z).abs() <= 2 * T * U * (X.abs().t() @ Z.abs())).all()
    assert ((db.double() - Z.sum(0)).abs() <= 2 * T * U * Z.abs().sum(0)).all()


# ---- gradients ---------------------------------------------------------------------------------

def _slope(act, z):
    with torch.enable_grad():
        v = z.clone().requires_grad_()
        return torch.autograd.grad(ACTS[act](v).sum(), v)[0]


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T,N", [(1, 8), (5, 64), (33, 520), (1000, 1032), (4097, 264)])
@pytest.mark.parametrize("act", list(ACTS))
def test_activation_backward(T, N, act, dtype):
    g = torch.Generator(device=D).manual_seed(T + N)
    for apart, overwrite, in_place in ((0, 1, None), (8, 0, None), (8, 1, "dy"), (8, 1, "z")):
        dy, z = _apart(T, N, N + apart, DT[dtype], g, 9.0)[1], _apart(T, N, N + apart, DT[dtype], g, 9.0)[1]
        z.mul_(3.0)
        G, Z = dy.double(), z.double()
        flat, dz = _apart(T, N, N + apart, DT[dtype], g, 7.0)
        if in_place:
            dz = dy if in_place == "dy" else z
        dbias = torch.full((N,), float("nan") if overwrite else 2.0, device=D)
        cfg = B.make_linear_config(T, 64, N, dtype, act, overwrite, ldy=N + apart, ldz=N + apart)
        scratch = _scratch(cfg)
        B.moe_act_bwd(cfg, dy, None if act == B.MOE_ACT_NONE else z, dz, dbias, scratch)
        want = G * _slope(act, Z)
        # the slope is of size one: its error is absolute, that of Phi and of z phi (z e^-z^2/2 is below 0.61), of the sigmoid alike
        err = 2e-6 * G.abs() if act else torch.zeros_like(G)
        assert ((dz.double() - want).abs() <= err + HALF[dtype] * (want.abs() + err) + 1e-44).all()
        old = 0.0 if overwrite else 2.0
        sums = (T + 30) * U * (want.abs().sum(0) + old) + err.sum(0)
        assert ((dbias.double() - old - want.sum(0)).abs() <= sums).all()
        if not in_place:
            assert _untouched(flat, dz, 7.0)
        assert (scratch[-64:] == 0xAB).all()
        alone = torch.full((N,), float("nan"), device=D)
        if not in_place and overwrite:
            B.moe_act_bwd(cfg, dy, z, None, alone, scratch)
            assert torch.equal(alone, dbias)
            B.moe_act_bwd(cfg, dy, z, dy, None, None)
            assert torch.equal(dy, dz)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T,N", [(31, 56), (64, 136), (65, 136), (256, 1032), (257, 72)])
@pytest.mark.parametrize("act", list(ACTS))
def test_activation_backward_of_few_rows(T, N, act, dtype):
    """About the numbers of rows up to which one workgroup has all of a column."""
    test_activation_backward(T, N, act, dtype)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T,K,N", [(1, 520, 1000), (32, 768, 136), (17, 776, 136), (32, 8, 8)])
def test_forward_about_one_slice(T, K, N, dtype):
    """About the sums that go in one slice, with a last step that is not full."""
    _forward(T, K, N, dtype, B.MOE_ACT_SILU, True, True, True, apart=8)


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("act", [B.MOE_ACT_GELU, B.MOE_ACT_SILU])
def test_activations_far_from_zero(act, dtype):
    """Exactly z or nothing far out, never NaN, whatever overflows on the way."""
    z = torch.tensor([[0.0, -0.0, 30.0, -30.0, 200.0, -200.0, 1e30, -1e30]], device=D).to(DT[dtype])
    cfg = B.make_linear_config(1, 8, 8, dtype, act, 1)
    eye, y, dz, scratch = torch.eye(8, device=D).to(DT[dtype]), torch.empty_like(z), torch.empty_like(z), _scratch(cfg)
    B.moe_linear_fwd(cfg, z, eye, None, None, None, y, scratch)
    B.moe_act_bwd(cfg, torch.ones_like(z), z, dz, None, None)
    Z = z[0].double()
    assert ((y[0].double() - ACTS[act](Z).nan_to_num(0.0)).abs() <= HALF[dtype] * Z.clamp(min=0) + 1e-10).all()
    assert ((dz[0].double() - torch.tensor([0.5, 0.5, 1, 0, 1, 0, 1, 0], device=D)).abs() <= 1e-10).all()


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T,K,N", [(1, 8, 8), (3, 64, 72), (40, 136, 64), (300, 520, 264), (1025, 64, 128), (5000, 72, 136), (2049, 1096, 72), (40, 72, 8192), (1, 264, 4104), (200, 64, 3000)])
def test_product_backward(T, K, N, dtype):
    g = torch.Generator(device=D).manual_seed(T + K + N)
    for apart, overwrite in ((0, 1), (8, 0)):
        x, dz = _apart(T, K, K + apart, DT[dtype], g, 9.0)[1], _apart(T, N, N + apart, DT[dtype], g, 9.0)[1]
        W = torch.randn((K, N), generator=g, device=D).to(DT[dtype])
        flat, dx = _apart(T, K, K + apart, DT[dtype], g, 7.0)
        dW = torch.full((K, N), float("nan") if overwrite else 2.0, device=D)
        cfg = B.make_linear_config(T, K, N, dtype, B.MOE_ACT_GELU, overwrite, ldx=K + apart, ldz=N + apart)
        scratch = _scratch(cfg)
        B.moe_linear_bwd(cfg, dz, x, W, dx, dW, scratch)
        X, Z, V = x.double(), dz.double(), W.double()
        want, err = Z @ V.t(), 2 * (N + 20) * U * (Z.abs() @ V.abs().t())
        assert ((dx.double() - want).abs() <= err + HALF[dtype] * (want.abs() + err)).all()
        old = 0.0 if overwrite else 2.0
        want = X.t() @ Z
        assert ((dW.double() - old - want).abs() <= 2 * (T + 20) * U * (X.abs().t() @ Z.abs() + old)).all()
        assert _untouched(flat, dx, 7.0) and (scratch[-64:] == 0xAB).all()
        # either alone: the same bits
        dx2, dW2 = torch.as_strided(torch.empty_like(flat), dx.shape, dx.stride(), 8), torch.full((K, N), old, device=D)
        B.moe_linear_bwd(cfg, dz, None, W, dx2, None, scratch)
        B.moe_linear_bwd(cfg, dz, x, None, None, dW2, scratch)
        assert torch.equal(dx2, dx) and torch.equal(dW2, dW)
        # with what reaches x past the product, in its place or another
        add = _apart(T, K, K + apart, DT[dtype], g, 9.0)[1]
        A = add.double()
        B.moe_linear_bwd(cfg, dz, None, W, dx2, None, scratch, add=add)
        want, err = Z @ V.t() + A, 2 * (N + 20) * U * (Z.abs() @ V.abs().t() + A.abs())
        assert ((dx2.double() - want).abs() <= err + HALF[dtype] * (want.abs() + err)).all()
        B.moe_linear_bwd(cfg, dz, None, W, add, None, scratch, add=add)
        assert torch.equal(add, dx2)


def test_no_rows_have_no_gradient():
    cfg, keep = B.make_linear_config(0, 64, 72, grad_overwrite=1), B.make_linear_config(0, 64, 72)
    dW, db = torch.full((64, 72), 3.0, device=D), torch.full((72,), 3.0, device=D)
    B.moe_linear_bwd(keep, None, None, None, None, dW, None)
    B.moe_act_bwd(keep, None, None, None, db, None)
    assert (dW == 3.0).all() and (db == 3.0).all()
    B.moe_linear_bwd(cfg, None, None, None, None, dW, None)
    B.moe_act_bwd(cfg, None, None, None, db, None)
    assert (dW == 0.0).all() and (db == 0.0).all()


@pytest.mark.parametrize("act", [B.MOE_ACT_GELU, B.MOE_ACT_SILU])
def test_gradients_against_differences(act):
    """Of L = sum(c * (act(x W + b) + r)), by central differences in 64 bits with h = 1e-5: off by h^2 and 1e-16 / h of L's terms."""
    T, K, N = 9, 16, 24
    g = torch.Generator(device=D).manual_seed(3)
    x, W, b, c = (torch.randn(s, generator=g, device=D) for s in ((T, K), (K, N), (N,), (T, N)))
    cfg = B.make_linear_config(T, K, N, B.MOE_F32, act, 1)
    scratch, z, y, dz = _scratch(cfg), torch.empty((T, N), device=D), torch.empty((T, N), device=D), torch.empty((T, N), device=D)
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
    B.moe_linear_fwd(cfg, x, W, b, None, z, y, scratch)
    B.moe_act_bwd(cfg, c, z, dz, db, scratch)
    B.moe_linear_bwd(cfg, dz, x, W, dx, dW, scratch)
    leaves = [t.double().cpu() for t in (x, W, b)]

    def loss(at):
        return float((c.double().cpu() * ACTS[act](at[0] @ at[1] + at[2])).sum())

    for n, (leaf, got) in enumerate(zip(leaves, (dx, dW, db))):
        for i in range(0, leaf.numel(), 7):
            v = []
            for h in (1e-5, -1e-5):
                at = [t.clone() for t in leaves]
                at[n].view(-1)[i] += h
                v.append(loss(at))
            assert abs((v[0] - v[1]) / 2e-5 - float(got.view(-1)[i])) <= 2e-4


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T", [4, 600])
def test_a_step_as_a_graph(T, dtype):
    """Forward and backward captured, replayed between eager ones, on another stream than the capture's."""
    K, N = 264, 1000
    g = torch.Generator(device=D).manual_seed(T)
    x, W, dy = (torch.randn(s, generator=g, device=D).to(DT[dtype]) for s in ((T, K), (K, N), (T, N)))
    b = torch.randn(N, generator=g, device=D)
    cfg = B.make_linear_config(T, K, N, dtype, B.MOE_ACT_SILU, 1)
    scratch = _scratch(cfg)
    out = {n: torch.empty(s, device=D, dtype=d) for n, s, d in (
        ("z", (T, N), DT[dtype]), ("y", (T, N), DT[dtype]), ("dz", (T, N), DT[dtype]), ("dx", (T, K), DT[dtype]),
        ("dW", (K, N), torch.float32), ("db", (N,), torch.float32))}

    def step():
        B.moe_linear_fwd(cfg, x, W, b, None, out["z"], out["y"], scratch)
        B.moe_act_bwd(cfg, dy, out["z"], out["dz"], out["db"], scratch)
        B.moe_linear_bwd(cfg, out["dz"], x, W, out["dx"], out["dW"], scratch)

    step()
    first = {n: t.clone() for n, t in out.items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for _ in range(3):
        for run in (graph.replay, step):
            for t in out.values():
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                run()
            torch.cuda.synchronize()
            for n, t in out.items():
                assert torch.equal(t, first[n]), n
