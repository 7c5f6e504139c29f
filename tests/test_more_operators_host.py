"""Refusals of the layer for a few tokens, the dense product and the gradients' norm: every one is a status code before
anything is launched, so no GPU is needed and the pointers handed over are never read."""
import ctypes

import pytest

from paper_2506_22175_amd import binding as B

P, NONE, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(0), ctypes.c_void_p(4104)
NULL, SHAPE, UNSUPPORTED = 1, 2, 3
F32, BF16, E4M3 = B.MOE_F32, B.MOE_BF16, B.MOE_E4M3


def _few(cfg, args=(P,) * 11):
    return B.lib().moe_few_forward(ctypes.byref(cfg), *args, None)


OK = dict(T=2, M=64, H=64, E=8, k=2)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), SHAPE), (dict(M=0), SHAPE), (dict(H=-8), SHAPE), (dict(E=0), SHAPE), (dict(k=0), SHAPE), (dict(k=9), SHAPE),
    (dict(groups=3), SHAPE), (dict(groups=4, group_k=5), SHAPE), (dict(k=3, groups=4, group_k=1), SHAPE),
    (dict(scale=float("nan")), SHAPE), (dict(ldx=56), SHAPE), (dict(ldy=63), SHAPE), (dict(ldx=-64), SHAPE),
    (dict(T=257), UNSUPPORTED), (dict(M=60), UNSUPPORTED), (dict(H=68), UNSUPPORTED), (dict(ldx=68), UNSUPPORTED),
    (dict(E=513), UNSUPPORTED), (dict(E=64, k=17), UNSUPPORTED), (dict(dtype=E4M3), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED),
    (dict(scores=2), UNSUPPORTED), (dict(renormalize=2), UNSUPPORTED), (dict(group_top=0), UNSUPPORTED),
    (dict(M=1 << 15, H=1 << 15), UNSUPPORTED), (dict(M=1 << 30), UNSUPPORTED), (dict(T=256, k=8, H=1 << 19), UNSUPPORTED),
    (dict(ldx=1 << 22), UNSUPPORTED),
])
def test_few_refuses(kw, status):
    cfg = B.make_few_config(**{**OK, **kw})
    assert _few(cfg) == status
    assert B.lib().moe_few_scratch_bytes(ctypes.byref(cfg), ctypes.byref(ctypes.c_size_t())) == status


def test_few_needs_its_pointers_and_their_alignment():
    cfg = B.make_few_config(**OK)
    for missing in (0, 1, 4, 5, 6, 7, 8, 9, 10):                 # all but the two biases
        assert _few(cfg, [NONE if i == missing else P for i in range(11)]) == NULL
    for odd in (0, 1, 4, 5, 10):                                 # x, Wg, W1, W2, scratch
        assert _few(cfg, [ODD if i == odd else P for i in range(11)]) == UNSUPPORTED
    assert B.lib().moe_few_forward(None, *(P,) * 11, None) == NULL
    assert B.moe_few_scratch_bytes(cfg) > 0


def _linear(cfg, fwd=(P,) * 7, act=(P,) * 5, bwd=(P,) * 7):
    c, lib = ctypes.byref(cfg), B.lib()
    return lib.moe_linear_fwd(c, *fwd, None), lib.moe_act_bwd(c, *act, None), lib.moe_linear_bwd(c, *bwd, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), SHAPE), (dict(K=0), SHAPE), (dict(N=-64), SHAPE), (dict(ldx=56), SHAPE), (dict(ldy=56), SHAPE),
    (dict(ldr=8), SHAPE), (dict(ldz=-64), SHAPE), (dict(K=60), UNSUPPORTED), (dict(N=68), UNSUPPORTED), (dict(ldx=68), UNSUPPORTED),
    (dict(ldz=70), UNSUPPORTED), (dict(dtype=E4M3), UNSUPPORTED), (dict(act=3), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
    (dict(grad_overwrite=2), UNSUPPORTED), (dict(N=40000), UNSUPPORTED), (dict(K=32768), UNSUPPORTED),
    (dict(ldy=1 << 22), UNSUPPORTED), (dict(ldx=1 << 40), UNSUPPORTED), (dict(T=1 << 30, K=2048, N=2048), UNSUPPORTED),
    (dict(T=(1 << 27) + 1, K=8, N=8), UNSUPPORTED), (dict(T=1 << 25, K=2048, N=8), UNSUPPORTED), (dict(ldr=(1 << 18) + 8), UNSUPPORTED),
])
def test_linear_refuses(kw, status):
    cfg = B.make_linear_config(**{**dict(T=4, K=64, N=64), **kw})
    assert _linear(cfg) == (status,) * 3
    assert B.lib().moe_linear_scratch_bytes(ctypes.byref(cfg), ctypes.byref(ctypes.c_size_t())) == status


def test_linear_needs_its_pointers_and_their_alignment():
    for T in (4, 400):
        cfg = B.make_linear_config(T, 64, 64, act=B.MOE_ACT_GELU)
        for missing in (0, 1, 5, 6):                             # x, W, y, scratch
            assert _linear(cfg, fwd=[NONE if i == missing else P for i in range(7)])[0] == NULL
        for missing in (0, 1):                                   # dy, z
            assert _linear(cfg, act=[NONE if i == missing else P for i in range(5)])[1] == NULL
        assert _linear(cfg, act=(P, P, NONE, NONE, P))[1] == NULL          # nothing to compute
        assert _linear(cfg, act=(P, P, P, P, NONE))[1] == NULL             # a bias gradient without scratch
        for missing in (0, 1, 2, 6):                             # dz, x, W, scratch
            assert _linear(cfg, bwd=[NONE if i == missing else P for i in range(7)])[2] == NULL
        assert _linear(cfg, bwd=(P, P, P, P, NONE, NONE, P))[2] == NULL
        for odd in (0, 1, 3, 4, 5, 6):                           # all but the bias
            assert _linear(cfg, fwd=[ODD if i == odd else P for i in range(7)])[0] == UNSUPPORTED
        for odd in (0, 1, 2, 4):
            assert _linear(cfg, act=[ODD if i == odd else P for i in range(5)])[1] == UNSUPPORTED
        for odd in range(7):
            assert _linear(cfg, bwd=[ODD if i == odd else P for i in range(7)])[2] == UNSUPPORTED
    lib = B.lib()
    assert lib.moe_linear_fwd(None, *(P,) * 7, None) == NULL and lib.moe_act_bwd(None, *(P,) * 5, None) == NULL
    assert lib.moe_linear_bwd(None, *(P,) * 7, None) == NULL


def _tensors(*entries):
    t = (B.MoEGradTensor * max(len(entries), 1))()
    for e, (grad, out, n, dtype) in zip(t, entries):
        e.grad, e.out, e.n, e.dtype = grad, out, n, dtype
    return t


def _table(*entries, table=P):
    return B.lib().moe_grad_table(_tensors(*entries), ctypes.c_int32(len(entries)), table, ctypes.byref(B.MoEGradList()), None)


@pytest.mark.parametrize("entry,status", [
    ((4096, None, -1, F32), SHAPE), ((4096, None, 8, E4M3), UNSUPPORTED), ((4096, None, 8, 9), UNSUPPORTED),
    ((None, None, 8, F32), NULL), ((4098, None, 8, F32), UNSUPPORTED), ((4097, None, 8, BF16), UNSUPPORTED),
    ((4096, 8194, 8, F32), UNSUPPORTED), ((4096, None, 1 << 50, F32), UNSUPPORTED),
])
def test_grad_lists_refuse(entry, status):
    t, s = ctypes.c_size_t(), ctypes.c_size_t()
    good = (1 << 20, None, 8, F32)
    for entries in ((entry,), (good, entry)):
        assert B.lib().moe_grad_bytes(_tensors(*entries), ctypes.c_int32(len(entries)), ctypes.byref(t), ctypes.byref(s)) == status
        assert _table(*entries) == status


def test_grad_lists_refuse_outputs_that_overlap():
    """An element that two workgroups scale, or that one scales while another still reads it."""
    a, n = 1 << 20, 100                                          # 400 bytes of float
    assert _table((a, a + 4, n, F32)) == SHAPE                   # partly its own input
    assert _table((a, a, n, F32), (a, a, n, F32)) == SHAPE       # in place, twice
    assert _table((a, a, n, F32), (a + 396, None, n, F32)) == SHAPE
    assert _table((a, None, n, F32), (1 << 22, a + 200, 10, BF16)) == SHAPE
    assert _table((a, 1 << 23, n, F32), (1 << 22, (1 << 23) + 399 - 3, 10, BF16)) == SHAPE
    assert _table((a, 1 << 23, 1000, F32), (1 << 22, 1 << 24, 10, F32), (1 << 25, (1 << 23) + 3996, 10, F32)) == SHAPE


def test_grad_calls_need_their_pointers():
    lib = B.lib()
    ok = B.MoEGradList(4096, 1, 1, 1)
    f = ctypes.c_float
    c = ctypes.byref(ok)
    assert lib.moe_grad_norm(c, None, P, None) == NULL and lib.moe_grad_norm(c, P, None, None) == NULL
    assert lib.moe_grad_norm(None, P, P, None) == NULL and lib.moe_grad_norm(ctypes.byref(B.MoEGradList(None, 1, 1, 1)), P, P, None) == NULL
    assert lib.moe_grad_norm(c, P, ctypes.c_void_p(4100), None) == UNSUPPORTED
    assert lib.moe_grad_norm(ctypes.byref(B.MoEGradList(4096, -1, 1, 1)), P, P, None) == SHAPE
    for most in (-1.0, float("nan"), float("inf")):
        assert lib.moe_grad_scale(c, f(most), P, None) == SHAPE and lib.moe_grad_clip(c, f(most), P, P, None) == SHAPE
    assert lib.moe_grad_scale(c, f(1.0), None, None) == NULL
    norms_only = ctypes.byref(B.MoEGradList(4096, 1, 1, 0))
    assert lib.moe_grad_scale(norms_only, f(1.0), P, None) == NULL and lib.moe_grad_clip(norms_only, f(1.0), P, P, None) == NULL
    assert lib.moe_grad_clip(c, f(1.0), P, None, None) == NULL and lib.moe_grad_clip(c, f(1.0), None, P, None) == NULL
    assert lib.moe_grad_table(None, ctypes.c_int32(1), P, ctypes.byref(ok), None) == NULL
    assert lib.moe_grad_table(None, ctypes.c_int32(-1), P, ctypes.byref(ok), None) == SHAPE
    t = _tensors((4096, None, 8, F32))
    assert lib.moe_grad_table(t, ctypes.c_int32(1), None, ctypes.byref(ok), None) == NULL
    assert lib.moe_grad_table(t, ctypes.c_int32(1), P, None, None) == NULL
    assert lib.moe_grad_table(t, ctypes.c_int32(1), ODD, ctypes.byref(ok), None) == UNSUPPORTED
    size = ctypes.c_size_t()
    assert lib.moe_grad_bytes(t, ctypes.c_int32(65537), ctypes.byref(size), ctypes.byref(size)) == UNSUPPORTED
    assert lib.moe_grad_bytes(t, ctypes.c_int32(1), None, ctypes.byref(size)) == NULL


def test_linear_takes_what_it_says():
    """The largest rows, dimensions and strides, and their scratch; a weight gradient has at most 64 partial sums."""
    for kw in (dict(T=1 << 27, K=8, N=8), dict(T=1 << 17, K=64, N=64, ldz=1 << 18), dict(T=1 << 20, K=31000, N=64), dict(T=5, K=8, N=31736)):
        for dtype in (F32, BF16):
            cfg = B.make_linear_config(dtype=dtype, **kw)
            assert 0 < B.moe_linear_scratch_bytes(cfg) <= 64 * 4 * max(kw["K"] * kw["N"], kw["T"] * kw["K"], kw["T"] * kw["N"], 1024 * kw["N"])


def test_grad_table_has_room_for_every_chunk():
    for n, dtype in ((0, F32), (1, BF16), (8192, F32), (8193, F32), (16384, BF16), (16385, BF16), (10 ** 9, F32)):
        table, scratch = B.moe_grad_bytes(_tensors((4096, None, n, dtype)))
        chunks = -(-n // (8192 if dtype == F32 else 16384))
        assert table >= 32 + 4 * chunks and scratch == 8 * min(max(chunks, 1), 2048)


def test_a_batch_without_tokens_is_no_error_and_launches_nothing():
    before = B.moe_launch_counts()
    assert _few(B.make_few_config(**{**OK, "T": 0}), (NONE,) * 11) == 0
    assert _linear(B.make_linear_config(0, 64, 64), (NONE,) * 7, (NONE,) * 5, (NONE,) * 7) == (0, 0, 0)
    assert B.moe_few_scratch_bytes(B.make_few_config(**{**OK, "T": 0})) == 0
    assert B.moe_linear_scratch_bytes(B.make_linear_config(0, 64, 64)) == 0
    assert B.moe_launch_counts() == before
