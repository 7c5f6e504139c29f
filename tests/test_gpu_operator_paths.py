"""The operators around the layer at the sizes where their launches differ from small ones: several rows after one another in a
workgroup, counts in a launch of their own, many rows to an expert, more choices than wavefronts.  References in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, E4M3 = B.MOE_F32, B.MOE_BF16, B.MOE_E4M3
DT = {F32: torch.float32, BF16: torch.bfloat16, E4M3: torch.float8_e4m3fn}
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,M", [(3003, 777), (2500, 1024), (2500, 2056), (2500, 4040), (1100, 9000), (600, 17000)])
def test_norm_backward_of_several_rows_to_a_workgroup(T, M, dtype):
    """Roundings: a row's sum has at most 32 terms in a row, 6 levels and 16 wavefronts, 64 with the factors; a column's sum the
    rows of a workgroup (of which there are 256 at least), 16 of the partial sums and 64 joined: T / 256 + 100."""
    g = torch.Generator(device=DEV).manual_seed(T + M)
    h, dy, dh = (torch.randn((T, M), generator=g, device=DEV).to(DT[dtype]) for _ in range(3))
    gain = 1 + 0.3 * torch.randn(M, generator=g, device=DEV)
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
    n, r = h.double() * rstd.double()[:, None], rstd.double()[:, None]
    up = dy.double() * gain.double()
    mean, size_mean = (up * n).mean(1, keepdim=True), (up * n).abs().mean(1, keepdim=True)
    dg, dg_size = (dy.double() * n).sum(0), (dy.double() * n).abs().sum(0)
    for with_dh, overwrite in ((True, 1), (False, 0)):
        cfg = B.make_norm_config(T, M, 1e-6, dtype, grad_overwrite=overwrite)
        need = B.moe_norm_scratch_bytes(cfg)
        scratch = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device=DEV)
        dx, dgain = torch.empty_like(h), torch.full((M,), float("nan") if overwrite else 3.0, device=DEV)
        B.moe_norm_bwd(cfg, dy, h, gain, rstd, dh if with_dh else None, dx, dgain, scratch)
        plus = dh.double() if with_dh else torch.zeros_like(n)
        want = plus + r * (up - n * mean)
        size = plus.abs() + r * (up.abs() + n.abs() * size_mean)
        assert ((dx.double() - want).abs() <= want.abs() * HALF[dtype] + 128 * 2.0 ** -24 * size).all()
        old = 0.0 if overwrite else 3.0
        assert ((dgain.double() - old - dg).abs() <= (T / 256 + 100) * 2.0 ** -24 * (dg_size + old)).all()
        assert (scratch[need:] == 0xAB).all()


@pytest.mark.parametrize("T,E,k", [(4096, 64, 2), (4097, 64, 3), (20000, 8, 1), (20001, 100, 7), (5000, 512, 16)])
def test_router_loads_of_many_tokens(T, E, k):
    rng = np.random.default_rng(T)
    l = (rng.standard_normal((T, E)) + 0.5 * rng.standard_normal(E)).astype(np.float32)
    l[rng.random(T) < 0.1] = -np.inf                              # padding
    l[rng.random((T, E)) < 0.2] = -np.inf
    order = np.argsort(-l, axis=1, kind="stable")[:, :k]
    want = np.where(np.take_along_axis(l, order, 1) > -np.inf, order, -1)
    assert (want == -1).any()
    before = rng.integers(0, 1000, E).astype(np.int32)
    idx, w = torch.empty((T, k), dtype=torch.int32, device=DEV), torch.empty((T, k), device=DEV)
    load = torch.from_numpy(before).to(DEV)
    B.moe_router_fwd(B.make_router_config(T, E, k), torch.from_numpy(l).to(DEV), None, idx, w, load)
    assert np.array_equal(idx.cpu().numpy(), want)
    assert np.array_equal(load.cpu().numpy(), before + np.bincount(want[want >= 0], minlength=E))


def test_router_backward_of_rows_that_lie_apart():
    """The same bits as of dense rows, and nothing written between the rows."""
    T, E, k, ld = 21, 50, 4, 53
    g = torch.Generator().manual_seed(1)
    for dtype in (F32, BF16):
        for kw in (dict(), dict(renormalize=1), dict(scores=B.MOE_SIGMOID)):
            l = torch.as_strided(torch.randn(T * ld + 60, generator=g).to(DT[dtype]).to(DEV), (T, E), (ld, 1), 3)
            idx = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).to(torch.int32).to(DEV)
            dw = torch.randn((T, k), generator=g).to(DEV)
            flat = torch.full((T * ld + 60,), 7.0, device=DEV).to(DT[dtype])
            dl, dense = torch.as_strided(flat, (T, E), (ld, 1), 5), torch.empty((T, E), device=DEV).to(DT[dtype])
            B.moe_router_bwd(B.make_router_config(T, E, k, dtype=dtype, ld=ld, **kw), l, idx, dw, dl)
            B.moe_router_bwd(B.make_router_config(T, E, k, dtype=dtype, **kw), l.contiguous(), idx, dw, dense)
            assert torch.equal(dl, dense) and (dense != 0).any()
            dl.fill_(7.0)
            assert (flat == 7.0).all()


def unpack(q, s):
    q, s = q.cpu(), s.cpu()
    codes = torch.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], -1).long()
    v = VALUES[codes & 7] * torch.where(codes >= 8, -1.0, 1.0)
    return v * torch.exp2(s.double() - 127.0).repeat_interleave(32, -1)


def product(g, T, k, E, K, N, dtype, idx, out=F32, group=0, per_choice=0, combine=0, gelu=0, weighted=True, scales=(121, 133), size=1.0,
            row_floor=0.0):
    """One product against 64 bits.  Additions: every matrix instruction adds 32 terms to a float sum, K / 128 of them in a row
    four times, in up to three parts, and at most 64 choices are joined: (K / 16 + 128) * 2^-24 of the sum of the terms'
    magnitudes.  GeLU passes an error on at most 1.13 times and adds that of erf; storing adds half a step.  row_floor: an
    absolute error of each of the rows' values."""
    Wq = torch.randint(0, 256, (E, N, K // 2), generator=g, dtype=torch.uint8)
    Ws = torch.randint(*scales, (E, N, K // 32), generator=g, dtype=torch.uint8)
    R = T * k if per_choice else T
    x = torch.randn((R, K), generator=g).mul_(size if dtype != E4M3 else 1.0).to(DT[dtype])
    cols = 128 if group else K
    xs = torch.rand((R, -(-K // cols)), generator=g).add_(0.5).mul_(size) if dtype == E4M3 else None
    w = torch.randn((T, k), generator=g) if weighted else None
    cfg = B.make_w4_config(T, k, E, K, N, dtype, out, group, per_choice, combine, gelu)
    need = B.moe_w4_scratch_bytes(cfg)
    scratch = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    rows = T if combine else T * k
    y = torch.full((rows + 1, N), 7.0, device=DEV).to(DT[out])
    up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    B.moe_w4_product(cfg, up(x), up(xs), up(idx), up(w), up(Wq), up(Ws), y, scratch)
    X = x.float().double()
    if xs is not None:
        X = X * xs.double().repeat_interleave(cols, 1)[:, :K]
    W, want, err = unpack(Wq, Ws), torch.zeros((T * k, N), dtype=torch.float64), torch.zeros((T * k, N), dtype=torch.float64)
    unit = (K / 16 + 128) * 2.0 ** -24
    flat = idx.reshape(-1).long()
    for e in range(E):
        at = (flat == e).nonzero()[:, 0]
        if len(at) == 0:
            continue
        xr = X[at if per_choice else at // k]
        z = xr @ W[e].t()
        er = (xr.abs() * unit + row_floor) @ W[e].abs().t()
        if gelu:
            z, er = 0.5 * z * (1 + torch.special.erf(z / math.sqrt(2))), 1.13 * er + z.abs() * 8 * 2.0 ** -24
        f = w.reshape(-1)[at, None].double() if weighted else torch.ones((len(at), 1), dtype=torch.float64)
        want[at], err[at] = f * z, f.abs() * (er + z.abs() * 2.0 ** -24)
    if combine:
        want, err = want.reshape(T, k, N), err.reshape(T, k, N)
        err = err.sum(1) + want.abs().sum(1) * k * 2.0 ** -24
        want = want.sum(1)
    got = y[:rows].cpu().double()
    assert torch.isfinite(want).all()
    assert ((got - want).abs() <= err + (want.abs() + err) * HALF[out]).all()
    assert (y[rows] == 7.0).all() and (scratch[need:] == 0xFF).all()


def choices(g, T, k, E, drop=0.0):
    idx = torch.rand((T, E), generator=g).argsort(1)[:, :k].to(torch.int32)
    gone = torch.rand((T, k), generator=g) < drop
    return torch.where(gone, torch.where(torch.rand((T, k), generator=g) < 0.3, E + 3, -1), idx).to(torch.int32).contiguous()


@pytest.mark.parametrize("dtype,group", [(F32, 0), (BF16, 0), (E4M3, 0), (E4M3, 128)])
def test_products_of_many_rows_with_wide_matrices(dtype, group):
    """75 rows to an expert, and columns for more workgroups than compute units."""
    g = torch.Generator().manual_seed(group + dtype)
    T, k, E, K, N = 300, 2, 8, 416, 2053
    product(g, T, k, E, K, N, dtype, choices(g, T, k, E, 0.1), F32, group)
    product(g, T, k, E, K, N, dtype, choices(g, T, k, E), BF16, group, gelu=1, weighted=False)
    product(g, T, k, E, K, N, dtype, choices(g, T, k, E, 0.1), BF16, group, per_choice=1, combine=1)


@pytest.mark.parametrize("dtype,group", [(F32, 0), (BF16, 0), (E4M3, 128)])
def test_products_where_one_expert_has_most_rows(dtype, group):
    """Every token's first choice is the same expert: four times the mean, more than its workgroups take in one pass."""
    g = torch.Generator().manual_seed(17)
    T, k, E, K, N = 300, 2, 8, 160, 2053
    idx = choices(g, T, k, E - 1)
    idx[:, 0] = E - 1
    product(g, T, k, E, K, N, dtype, idx, F32, group)
    product(g, T, k, E, 1184, 40, dtype, idx, F32, group, combine=1)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("T,k,K,N", [(1, 17, 96, 40), (1, 64, 608, 33), (2, 40, 1056, 17), (3, 20, 64, 16), (1, 33, 4128, 20)])
def test_products_of_more_choices_than_wavefronts(T, k, K, N, dtype):
    g = torch.Generator().manual_seed(k)
    for kw in (dict(combine=1), dict(combine=1, per_choice=1, gelu=1), dict(per_choice=1)):
        product(g, T, k, 64, K, N, dtype, choices(g, T, k, 64, 0.1), **kw)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("T,k,E,K,N", [(1, 2, 4, 160, 40), (20, 2, 8, 160, 40), (80, 2, 3, 160, 40), (300, 2, 8, 160, 2053)])
def test_the_least_scales(T, k, E, K, N, dtype):
    """Scale bytes 0, 1 and 2: weights below the normal numbers of the type that the matrix instructions take."""
    g = torch.Generator().manual_seed(T)
    product(g, T, k, E, K, N, dtype, choices(g, T, k, E), scales=(0, 3), size=2.0 ** 110)


@pytest.mark.parametrize("T,k,E,K,N", [(1, 2, 4, 160, 40), (20, 2, 8, 160, 40), (80, 2, 3, 160, 40)])
@pytest.mark.parametrize("power", [-100, -112, -120, -126])
def test_float_rows_near_the_least_float(T, k, E, K, N, power):
    """Rows whose parts fall below the normal numbers: what is below 2^-133, the least bfloat16, is cut off."""
    g = torch.Generator().manual_seed(T)
    product(g, T, k, E, K, N, F32, choices(g, T, k, E), scales=(225, 235), size=2.0 ** power, row_floor=2.0 ** -133)
