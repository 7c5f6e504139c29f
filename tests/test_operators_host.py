"""Refusals of the norm, the router and the 4-bit products: every one is a status code before anything is launched, so no
GPU is needed and the pointers handed over are never read."""
import ctypes

import pytest

from paper_2506_22175_amd import binding as B

P = ctypes.c_void_p(4096)
NONE = ctypes.c_void_p(0)
NULL, SHAPE, UNSUPPORTED = 1, 2, 3
F32, BF16, E4M3 = B.MOE_F32, B.MOE_BF16, B.MOE_E4M3


def _norm_fwd(cfg, *args):
    return B.lib().moe_norm_fwd(ctypes.byref(cfg), *(args or (P,) * 7), None)


def _norm_bwd(cfg, *args):
    return B.lib().moe_norm_bwd(ctypes.byref(cfg), *(args or (P,) * 8), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1, M=64), SHAPE), (dict(T=1, M=0), SHAPE), (dict(T=1, M=64, eps=-1.0), SHAPE),
    (dict(T=1, M=64, eps=float("nan")), SHAPE), (dict(T=1, M=64, eps=float("inf")), SHAPE),
    (dict(T=1, M=64, ldx=63), SHAPE), (dict(T=1, M=64, ldr=1), SHAPE), (dict(T=1, M=64, ldh=-64), SHAPE),
    (dict(T=1, M=64, ldy=63), SHAPE),
    (dict(T=1, M=64, dtype=E4M3), UNSUPPORTED), (dict(T=1, M=64, dtype=7), UNSUPPORTED),
    (dict(T=1, M=64, dtype=F32, out=BF16), UNSUPPORTED), (dict(T=1, M=64, out=E4M3, group=64), UNSUPPORTED),
    (dict(T=1, M=64, out=BF16, group=128), UNSUPPORTED), (dict(T=1, M=32769), UNSUPPORTED),
    (dict(T=1, M=64, grad_overwrite=2), UNSUPPORTED),
])
def test_norm_refuses(kw, status):
    cfg = B.make_norm_config(**kw)
    assert _norm_fwd(cfg) == status and _norm_bwd(cfg) == status
    assert B.lib().moe_norm_scratch_bytes(ctypes.byref(cfg), ctypes.byref(ctypes.c_size_t())) == status


def test_norm_needs_its_pointers():
    cfg = B.make_norm_config(4, 64)
    for missing in (0, 4):                                       # x, y
        assert _norm_fwd(cfg, *[NONE if i == missing else P for i in range(7)]) == NULL
    assert _norm_fwd(B.make_norm_config(4, 64, out=E4M3), *[NONE if i == 5 else P for i in range(7)]) == NULL
    for missing in (0, 1, 3, 5):                                 # dy, h, rstd, dx
        assert _norm_bwd(cfg, *[NONE if i == missing else P for i in range(8)]) == NULL
    many = B.make_norm_config(100, 64)
    assert B.moe_norm_scratch_bytes(many) > 0
    assert _norm_bwd(many, *[NONE if i == 7 else P for i in range(8)]) == NULL
    assert _norm_bwd(B.make_norm_config(4, 64, out=E4M3)) == UNSUPPORTED     # no gradient of rounded rows
    assert B.lib().moe_norm_fwd(None, *(P,) * 7, None) == NULL


def test_norm_scratch_is_bounded():
    assert B.moe_norm_scratch_bytes(B.make_norm_config(0, 64)) == 0
    assert B.moe_norm_scratch_bytes(B.make_norm_config(1, 64)) == 0
    assert 0 < B.moe_norm_scratch_bytes(B.make_norm_config(1 << 30, 2048)) <= 2048 * 2048 * 4


def _router(cfg, fwd=(P,) * 5, bwd=(P,) * 4):
    return (B.lib().moe_router_fwd(ctypes.byref(cfg), *fwd, None), B.lib().moe_router_bwd(ctypes.byref(cfg), *bwd, None))


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1, E=8, k=2), SHAPE), (dict(T=1, E=0, k=1), SHAPE), (dict(T=1, E=8, k=0), SHAPE), (dict(T=1, E=8, k=9), SHAPE),
    (dict(T=1, E=8, k=2, groups=3), SHAPE), (dict(T=1, E=8, k=2, groups=0), SHAPE), (dict(T=1, E=8, k=2, group_k=0), SHAPE),
    (dict(T=1, E=8, k=2, groups=4, group_k=5), SHAPE), (dict(T=1, E=8, k=3, groups=4, group_k=1), SHAPE),
    (dict(T=1, E=8, k=2, scale=float("nan")), SHAPE), (dict(T=1, E=8, k=2, scale=float("inf")), SHAPE),
    (dict(T=1, E=8, k=2, ld=7), SHAPE), (dict(T=1, E=513, k=2), UNSUPPORTED), (dict(T=1, E=64, k=17), UNSUPPORTED),
    (dict(T=1, E=34, k=2, groups=17), UNSUPPORTED), (dict(T=1, E=8, k=2, scores=2), UNSUPPORTED),
    (dict(T=1, E=8, k=2, dtype=E4M3), UNSUPPORTED), (dict(T=1, E=8, k=2, renormalize=2), UNSUPPORTED),
    (dict(T=1, E=8, k=2, group_top=3), UNSUPPORTED), (dict(T=1, E=8, k=2, group_top=0), UNSUPPORTED),
])
def test_router_refuses(kw, status):
    assert _router(B.make_router_config(**kw)) == (status, status)


def test_router_needs_its_pointers():
    cfg = B.make_router_config(4, 8, 2)
    for missing in (0, 2, 3):
        assert _router(cfg, fwd=[NONE if i == missing else P for i in range(5)])[0] == NULL
    for missing in range(4):
        assert _router(cfg, bwd=[NONE if i == missing else P for i in range(4)])[1] == NULL
    assert B.lib().moe_router_fwd(None, *(P,) * 5, None) == NULL


def _w4(cfg, args=(P,) * 8):
    return B.lib().moe_w4_product(ctypes.byref(cfg), *args, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1, k=1, E=4, K=64, N=64), SHAPE), (dict(T=1, k=0, E=4, K=64, N=64), SHAPE), (dict(T=1, k=5, E=4, K=64, N=64), SHAPE),
    (dict(T=1, k=1, E=0, K=64, N=64), SHAPE), (dict(T=1, k=1, E=4, K=0, N=64), SHAPE), (dict(T=1, k=1, E=4, K=64, N=0), SHAPE),
    (dict(T=1, k=1, E=4, K=64, N=64, ldx=32), SHAPE), (dict(T=1, k=1, E=4, K=64, N=64, ldy=63), SHAPE),
    (dict(T=1, k=1, E=4, K=48, N=64), UNSUPPORTED), (dict(T=1, k=65, E=128, K=64, N=64), UNSUPPORTED),
    (dict(T=1, k=1, E=4097, K=64, N=64), UNSUPPORTED), (dict(T=1, k=1, E=4, K=64, N=64, dtype=9), UNSUPPORTED),
    (dict(T=1, k=1, E=4, K=64, N=64, out=E4M3), UNSUPPORTED), (dict(T=1, k=1, E=4, K=64, N=64, group=128), UNSUPPORTED),
    (dict(T=1, k=1, E=4, K=64, N=64, dtype=E4M3, group=64), UNSUPPORTED), (dict(T=1, k=1, E=4, K=64, N=64, gelu=2), UNSUPPORTED),
    (dict(T=1, k=1, E=4, K=64, N=64, combine=3), UNSUPPORTED), (dict(T=1, k=1, E=4, K=64, N=64, per_choice=-1), UNSUPPORTED),
    (dict(T=1, k=1, E=4, K=64, N=64, ldx=68), UNSUPPORTED), (dict(T=1, k=1, E=4, K=64, N=64, dtype=F32, ldx=66), UNSUPPORTED),
    (dict(T=1, k=1, E=4, K=64, N=64, dtype=E4M3, ldx=72), UNSUPPORTED), (dict(T=1 << 24, k=2, E=4, K=64, N=64), UNSUPPORTED),
    (dict(T=65536, k=1, E=4, K=64, N=64, combine=1), UNSUPPORTED),
])
def test_w4_refuses(kw, status):
    cfg = B.make_w4_config(**kw)
    assert _w4(cfg) == status
    assert B.lib().moe_w4_scratch_bytes(ctypes.byref(cfg), ctypes.byref(ctypes.c_size_t())) == status


def test_w4_needs_its_pointers_and_their_alignment():
    cfg = B.make_w4_config(4, 2, 4, 64, 64, combine=1)
    assert B.moe_w4_scratch_bytes(cfg) > 0
    for missing in (0, 4, 5, 6, 7):                              # x, Wq, Ws, y, scratch
        assert _w4(cfg, [NONE if i == missing else P for i in range(8)]) == NULL
    assert _w4(B.make_w4_config(4, 2, 4, 64, 64, dtype=E4M3), [NONE if i == 1 else P for i in range(8)]) == NULL
    for odd in (0, 4, 7):
        assert _w4(cfg, [ctypes.c_void_p(4104) if i == odd else P for i in range(8)]) == UNSUPPORTED
    q = B.lib().moe_w4_quantize
    assert q(4, 64, 64, BF16, None, P, P, None) == NULL and q(4, 64, 64, BF16, P, None, P, None) == NULL
    assert q(4, 64, 64, BF16, P, P, None, None) == NULL
    assert q(0, 64, 64, BF16, P, P, P, None) == SHAPE and q(4, 48, 64, BF16, P, P, P, None) == UNSUPPORTED
    assert q(4, 64, 64, E4M3, P, P, P, None) == UNSUPPORTED and q(5000, 64, 64, BF16, P, P, P, None) == UNSUPPORTED


def test_a_batch_without_tokens_is_no_error_and_launches_nothing():
    before = B.moe_launch_counts()
    assert _norm_fwd(B.make_norm_config(0, 64), *(NONE,) * 7) == 0
    assert _norm_bwd(B.make_norm_config(0, 64), *(NONE,) * 8) == 0
    assert _router(B.make_router_config(0, 8, 2), (NONE,) * 5, (NONE,) * 4) == (0, 0)
    assert _w4(B.make_w4_config(0, 1, 4, 64, 64), (NONE,) * 8) == 0
    assert B.moe_launch_counts() == before
