"""Products with 4-bit weights against 64 bits, and the packing of weights.

A product's terms are exact (4-bit weights times parts of the rows) or those of float.  Additions: every matrix instruction adds
32 terms to a float sum, K / 128 of them in a row in each of four wavefronts, in parts of up to three, and at most 64 choices are
joined: (K / 16 + 128) * 2^-24 of the sum of the terms' magnitudes covers them with each instruction's inner rounding counted
like a float addition of 8.  GeLU passes an error on at most 1.13 times and adds that of erf (4 units); storing adds eps / 2."""
import math

import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, E4M3 = B.MOE_F32, B.MOE_BF16, B.MOE_E4M3
DT = {F32: torch.float32, BF16: torch.bfloat16, E4M3: torch.float8_e4m3fn}
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def unpack(q, s):
    """[E, N, K] in 64 bits, on the host."""
    q, s = q.cpu(), s.cpu()
    codes = torch.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], -1).long()
    v = VALUES[codes & 7] * torch.where(codes >= 8, -1.0, 1.0)
    scale = torch.exp2(s.double() - 127.0)
    scale[s == 255] = float("nan")
    return v * scale.repeat_interleave(32, -1)


def weights(g, E, N, K, spread=6):
    q = torch.randint(0, 256, (E, N, K // 2), generator=g, dtype=torch.uint8)
    s = torch.randint(127 - spread, 127 + spread, (E, N, K // 32), generator=g, dtype=torch.uint8)
    return q.to(DEV), s.to(DEV)


def choices(g, T, k, E, drop=0.0):
    idx = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).to(torch.int32)
    if drop:
        gone = torch.rand((T, k), generator=g) < drop
        idx[gone] = -1
        idx[gone & (torch.rand((T, k), generator=g) < 0.3)] = E + 3
    return idx


def check(T, k, E, K, N, dtype=BF16, out=BF16, group=0, per_choice=0, combine=0, gelu=0, drop=0.0, dense=False, ldx=0, ldy=0,
          weighted=True, seed=0):
    g = torch.Generator().manual_seed(seed + T + K + N)
    Wq, Ws = weights(g, E, N, K)
    R = T * k if per_choice else T
    lx, ly = ldx or K, ldy or N
    xf = torch.randn((R, lx), generator=g).to(DT[dtype]).to(DEV)
    x = xf[:, :K]
    n_scales = -(-K // 128) if group else 1
    xs = torch.rand((R, n_scales), generator=g).add_(0.5).to(DEV) if dtype == E4M3 else None
    idx = None if dense else choices(g, T, k, E, drop)
    w = torch.randn((T, k), generator=g) if weighted else None
    cfg = B.make_w4_config(T, k, E, K, N, dtype, out, group, per_choice, combine, gelu, ldx, ldy)
    rows = T if combine else T * k
    yf = torch.full((rows + 1, ly), 7.0, device=DEV).to(DT[out])
    need = B.moe_w4_scratch_bytes(cfg)
    scratch = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    B.moe_w4_product(cfg, xf, xs, idx.to(DEV) if idx is not None else None, w.to(DEV) if weighted else None, Wq, Ws, yf, scratch)
    torch.cuda.synchronize()
    # 64 bits
    W = unpack(Wq, Ws)
    X = x.cpu().to(torch.float32).double()
    if xs is not None:
        X = X * xs.cpu().double().repeat_interleave(128 if group else K, 1)[:, :K]
    y = torch.zeros((T, k, N), dtype=torch.float64)
    err = torch.zeros((T, k, N), dtype=torch.float64)
    unit = (K / 16 + 128) * 2.0 ** -24
    for t in range(T):
        for j in range(k):
            e = 0 if idx is None else int(idx[t, j])
            if not 0 <= e < E:
                continue
            xr = X[t * k + j if per_choice else t]
            z, size = W[e] @ xr, W[e].abs() @ xr.abs()
            a, er = z, size * unit
            if gelu:
                a, er = 0.5 * z * (1 + torch.special.erf(z / math.sqrt(2))), 1.13 * er + z.abs() * 8 * 2.0 ** -24
            f = float(w[t, j]) if weighted else 1.0
            y[t, j], err[t, j] = f * a, abs(f) * (er + a.abs() * 2.0 ** -24)
    if combine:
        err = err.sum(1) + y.abs().sum(1) * k * 2.0 ** -24
        y = y.sum(1)
    y, err = y.reshape(rows, N), err.reshape(rows, N)
    got = yf[:rows, :N].cpu().double()
    assert ((got - y).abs() <= err + (y.abs() + err) * (2.0 ** -24 if out == F32 else 2.0 ** -8)).all()
    assert (yf[rows] == 7.0).all() and (yf[:, N:] == 7.0).all() and (scratch[need:] == 0xFF).all()


ROUTED = [(1, 1, 1, 32, 1), (1, 2, 8, 64, 16), (1, 4, 4, 96, 17), (2, 2, 16, 128, 33), (3, 2, 4, 160, 64), (5, 3, 6, 512, 65), (8, 8, 8, 1024, 40),
          (16, 2, 8, 256, 70), (17, 1, 1, 544, 31), (40, 4, 5, 288, 50), (70, 2, 2, 128, 24), (64, 1, 3, 2048, 16), (33, 8, 64, 416, 130)]


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("T,k,E,K,N", ROUTED)
def test_routed_rows(T, k, E, K, N, dtype):
    check(T, k, E, K, N, dtype, F32, gelu=0)
    check(T, k, E, K, N, dtype, BF16, group=128 if dtype == E4M3 else 0, gelu=1, drop=0.2, weighted=False)
    check(T, k, E, K, N, dtype, F32, group=128 if dtype == E4M3 else 0, per_choice=1, combine=1, drop=0.2)
    check(T, k, E, K, N, dtype, BF16, combine=1, gelu=1, weighted=False)
    check(T, k, E, K, N, dtype, BF16, per_choice=1)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("T", [1, 15, 16, 17, 33, 100, 300])
def test_one_expert_for_all(T, dtype):
    check(T, 1, 1, 320, 48, dtype, F32, dense=True, weighted=False)
    check(T, 1, 2, 320, 48, dtype, BF16, combine=1)


def test_rows_that_lie_apart():
    check(9, 2, 4, 96, 30, BF16, BF16, ldx=104, ldy=37)
    check(9, 2, 4, 96, 30, F32, F32, ldx=100, ldy=31, combine=1)
    check(9, 2, 4, 96, 30, E4M3, BF16, ldx=112, ldy=33)


def test_all_choices_missing_give_zeros():
    check(3, 2, 4, 64, 40, drop=1.1)
    check(3, 2, 4, 64, 40, drop=1.1, combine=1)
    check(30, 2, 4, 64, 40, E4M3, F32, drop=1.1, combine=1)
    check(30, 2, 4, 64, 40, drop=1.1)


def test_float_rows_keep_all_their_bits():
    """One weight of 1 per column: the product is the row's value itself."""
    K, N = 64, 64
    codes = torch.zeros((1, N, K), dtype=torch.uint8)
    codes[0, torch.arange(N), torch.arange(N)] = 2
    q = (codes[..., 0::2] | codes[..., 1::2] << 4).to(DEV)
    s = torch.full((1, N, 2), 127, dtype=torch.uint8, device=DEV)
    bits = np.random.default_rng(0).integers(0, 2 ** 32, (16, K), dtype=np.uint64).astype(np.uint32)
    x = torch.from_numpy(bits.view(np.float32).copy())
    x = torch.where(torch.isfinite(x) & (x.abs() > 1e-30), x, torch.tensor(1.2345678))
    y = torch.empty((16, N), device=DEV)
    B.moe_w4_product(B.make_w4_config(16, 1, 1, K, N, F32, F32), x.to(DEV), None, None, None, q, s, y)
    assert torch.equal(y.cpu(), x)


def test_infinities_and_nan_stay_in_their_rows_and_columns():
    g = torch.Generator().manual_seed(5)
    T, K, N = 20, 128, 40
    for dtype in (F32, BF16):
        x = torch.randn((T, K), generator=g).to(DT[dtype]).to(DEV)
        x[3, 5], x[4, 100], x[17, 0] = float("nan"), float("inf"), float("-inf")
        Wq, Ws = weights(g, 1, N, K)
        Ws[0, 11, 2] = 255
        y = torch.empty((T, N), device=DEV)
        B.moe_w4_product(B.make_w4_config(T, 1, 1, K, N, dtype, F32), x, None, None, None, Wq, Ws, y)
        y = y.cpu()
        ok = [t for t in range(T) if t not in (3, 4, 17)]
        assert y[3].isnan().all() and not torch.isfinite(y[4]).any() and not torch.isfinite(y[17]).any()
        assert y[:, 11].isnan().all()
        cols = [n for n in range(N) if n != 11]
        assert torch.isfinite(y[ok][:, cols]).all()


def test_weights_beyond_32_bit_offsets():
    """More than 2^31 packed bytes: the last experts are read, not what an offset cut to 32 bits points at."""
    E, K, N = 70, 8192, 8192                               # 2.3 GB
    Wq = torch.zeros((E, N, K // 2), dtype=torch.uint8, device=DEV)
    Ws = torch.full((E, N, K // 32), 127, dtype=torch.uint8, device=DEV)
    Wq[E - 1, :, 0] = 2                                    # column 0 of every weight row: 1
    Wq[E - 1, N - 1, K // 2 - 1] = 4 << 4                  # the last column of the last one: 2
    x = torch.ones((1, K), device=DEV, dtype=torch.bfloat16)
    y = torch.empty((1, 1, N), device=DEV, dtype=torch.float32)
    idx = torch.tensor([[E - 1]], dtype=torch.int32, device=DEV)
    B.moe_w4_product(B.make_w4_config(1, 1, E, K, N, BF16, F32), x, None, idx, None, Wq, Ws, y)
    want = torch.ones(N)
    want[N - 1] = 3
    assert torch.equal(y.cpu()[0, 0], want)


def test_the_same_bits_every_time_on_another_stream_and_in_a_graph():
    g = torch.Generator().manual_seed(6)
    T, k, E, K, N = 12, 2, 4, 512, 96
    Wq, Ws = weights(g, E, N, K)
    x, idx, w = torch.randn((T, K), generator=g).to(DEV), choices(g, T, k, E).to(DEV), torch.rand((T, k), generator=g).to(DEV)
    cfg = B.make_w4_config(T, k, E, K, N, F32, F32, combine=1)
    y, scratch = torch.empty((T, N), device=DEV), torch.empty(B.moe_w4_scratch_bytes(cfg) + 16, dtype=torch.uint8, device=DEV)
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
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, first)
        call()
        torch.cuda.synchronize()
        assert torch.equal(y, first)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E,K,N", [(1, 32, 1), (2, 64, 33), (3, 160, 300)])
def test_packing(E, K, N, dtype):
    """Bit for bit: the least shared power of two under which nothing exceeds 6, then the nearest value, ties to even codes."""
    g = torch.Generator().manual_seed(K + N)
    W = torch.randn((E, K, N), generator=g) * torch.exp2(torch.randint(-20, 20, (E, 1, N), generator=g).float())
    W[0, :32, 0] = 0.0
    W[0, 0, 0] = 6.0 * 2.0 ** 5                             # exactly 6: no larger scale
    if N > 4:
        W[0, :32, 1] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4) * 2.0 ** -3      # ties
        W[0, :32, 2] = -W[0, :32, 1]
        W[0, :32, 3] = 0.0
        W[0, :32, 4] = 2.0 ** -130                          # below the least scale
    W = W.to(DT[dtype])
    Wq = torch.full((E, N, K // 2), 0x77, dtype=torch.uint8, device=DEV)
    Ws = torch.full((E, N, K // 32), 0x77, dtype=torch.uint8, device=DEV)
    B.moe_w4_quantize(E, K, N, dtype, W.to(DEV), Wq, Ws)
    v = W.double().transpose(1, 2).reshape(E, N, K // 32, 32)
    most = v.abs().amax(-1)
    m, p = torch.frexp(most / 6.0)
    p = torch.where(m == 0.5, p - 1, p).double()            # ceil(log2(most / 6))
    p = torch.where(most == 0, torch.full_like(p, -126), p.clamp(min=-126))
    assert torch.equal(Ws.cpu().double(), p + 127)
    near = v.abs() / torch.exp2(p)[..., None]
    away = (near[..., None] - VALUES).abs()
    least = away.amin(-1, keepdim=True)
    code = torch.where(away == least, torch.tensor([0, 8, 1, 9, 2, 10, 3, 11]), 99).amin(-1)      # even codes before odd ones
    code = torch.tensor([0, 2, 4, 6, 0, 0, 0, 0, 1, 3, 5, 7])[code]
    code = (code + torch.where(torch.signbit(v), 8, 0)).reshape(E, N, K // 2, 2)
    assert torch.equal(Wq.cpu(), (code[..., 0] | code[..., 1] << 4).to(torch.uint8))


def test_packing_marks_blocks_that_are_not_finite():
    W = torch.ones((1, 96, 2))
    W[0, 3, 0], W[0, 40, 1] = float("inf"), float("nan")
    Wq, Ws = torch.empty((1, 2, 48), dtype=torch.uint8, device=DEV), torch.empty((1, 2, 3), dtype=torch.uint8, device=DEV)
    B.moe_w4_quantize(1, 96, 2, F32, W.to(DEV), Wq, Ws)
    assert (Ws.cpu() == 255).tolist() == [[[True, False, False], [False, True, False]]]


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
def test_loads_that_differ(dtype):
    """One expert with nearly all rows, in several passes and workgroups, beside experts with a row or none."""
    g = torch.Generator().manual_seed(8)
    T, k, E, K, N = 150, 2, 40, 288, 70
    Wq, Ws = weights(g, E, N, K)
    idx = torch.full((T, k), 7, dtype=torch.int32)
    idx[:, 1] = torch.arange(T) % 5 + 20
    idx[3, 0], idx[140, 1] = -1, 39
    x = torch.randn((T, K), generator=g).to(DT[dtype]).to(DEV)
    xs = torch.rand((T, 1), generator=g).to(DEV) if dtype == E4M3 else None
    y = torch.empty((T, k, N), device=DEV)
    B.moe_w4_product(B.make_w4_config(T, k, E, K, N, dtype, F32), x, xs, idx.to(DEV), None, Wq, Ws, y, None)
    X, W = x.cpu().float().double() * (xs.cpu().double() if xs is not None else 1.0), unpack(Wq, Ws)
    for t in range(T):
        for j in range(k):
            e = int(idx[t, j])
            want = W[e] @ X[t] if e >= 0 else torch.zeros(N, dtype=torch.float64)
            size = W[e].abs() @ X[t].abs() if e >= 0 else torch.zeros(N, dtype=torch.float64)
            assert ((y[t, j].cpu().double() - want).abs() <= (K / 16 + 129) * 2.0 ** -24 * size).all(), (t, j)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("T,k,E,K,N", [(17, 2, 16, 160, 65), (24, 4, 64, 1056, 70), (20, 1, 8, 512, 33), (18, 2, 64, 96, 24), (40, 2, 64, 2080, 40),
                                       (100, 8, 64, 544, 48), (16, 16, 16, 32, 7)])
def test_few_rows_to_an_expert(T, k, E, K, N, dtype):
    check(T, k, E, K, N, dtype, F32, group=128 if dtype == E4M3 else 0, drop=0.2)
    check(T, k, E, K, N, dtype, BF16, per_choice=1, combine=1)
    check(T, k, E, K, N, dtype, BF16, gelu=1, weighted=False)


def test_a_batch_that_reads_its_experts_weights_once():
    """Ten tokens whose choices share experts of a size where that counts."""
    check(10, 2, 4, 4096, 2048, BF16, F32, drop=0.2)
    check(10, 2, 4, 4096, 2048, BF16, BF16, per_choice=1, combine=1)
