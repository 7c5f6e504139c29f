"""The block's weights are handed over as addresses: those of another type, shape or order are refused before anything is allocated,
so no GPU is needed."""
import pytest
import torch

from paper_2506_22175_amd import binding as B
from paper_2506_22175_amd.block import Block, Few, Packed, Served, Shared

T, M, H, E, k, N = 4, 64, 96, 8, 2, 32
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SHAPES = {"gain": (M,), "Wg": (M, E), "W1": (E, M, H), "W2": (E, H, M), "bias": (E,), "V1": (M, N), "V2": (N, M), "b1": (N,), "b2": (M,)}
VECTORS = ("gain", "bias", "b1", "b2")


def _weights(dtype):
    return {n: torch.zeros(s, dtype=F32 if n in VECTORS else dtype) for n, s in SHAPES.items()}


def _shared(w):
    return w["V1"], w["V2"], w["b1"], w["b2"]


class _Pack:
    E, M, H = E, M, H


MAKE = {
    "shared": lambda w, dtype: Shared(T, *_shared(w), device="cpu"),
    "trained": lambda w, dtype: Shared(T, *_shared(w), training=True, device="cpu"),
    "few": lambda w, dtype: Few(T, k, w["gain"], w["Wg"], w["W1"], w["W2"], w["bias"], device="cpu", shared=_shared(w)),
    "block": lambda w, dtype: Block(T, M, H, E, k, w["gain"], w["Wg"], w["W1"], w["W2"], w["bias"], device="cpu", shared=_shared(w),
                                    dtype=B.MOE_BF16 if dtype == BF16 else B.MOE_F32),
    "served": lambda w, dtype: Served(T, k, w["gain"], w["Wg"], _Pack, w["bias"], dtype=B.MOE_BF16 if dtype == BF16 else B.MOE_F32, device="cpu"),
    "packed": lambda w, dtype: Packed(w["W1"], w["W2"]),
}
TAKES = {"shared": ("V1", "V2", "b1", "b2"), "trained": ("V1", "V2", "b1", "b2"), "few": tuple(SHAPES), "block": tuple(SHAPES),
         "served": ("gain", "Wg", "bias"), "packed": ("W1", "W2")}
CASES = [(maker, name) for maker, names in TAKES.items() for name in names]


def _refused(maker, w, dtype):
    # (W1 and V1 say what the others have to be: where they are wrong themselves, another may be named)
    with pytest.raises(ValueError, match=r"^(%s) " % "|".join(SHAPES)):
        MAKE[maker](w, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("maker,name", CASES)
def test_other_types_are_refused(maker, name, dtype):
    for other in (F16, F32, BF16, torch.float64):
        w = _weights(dtype)
        if w[name].dtype != other:
            w[name] = w[name].to(other)
            _refused(maker, w, dtype)


@pytest.mark.parametrize("maker,name", CASES)
def test_other_shapes_and_orders_are_refused(maker, name):
    w = _weights(BF16)
    good = w[name]
    last = good.shape[-1]
    wrong = [torch.zeros(good.shape[:-1] + (n,), dtype=good.dtype) for n in (last - 8, last + 8) if n > 0]
    wrong.append(torch.zeros(good.shape[:-1] + (2 * last,), dtype=good.dtype)[..., ::2])       # the right shape, elements apart
    if good.dim() > 1:
        wrong.append(torch.zeros_like(good).transpose(-1, -2).contiguous())
        wrong.append(wrong[-1].transpose(-1, -2))                                             # the right shape, columns first
    for bad in wrong:
        w[name] = bad
        _refused(maker, w, BF16)


@pytest.mark.parametrize("of_rows,of_shared", [(BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("maker", ["few", "block"])
def test_a_shared_expert_of_another_type_or_width_is_refused(maker, of_rows, of_shared):
    w, other = _weights(of_rows), _weights(of_shared)
    w["V1"], w["V2"] = other["V1"], other["V2"]
    _refused(maker, w, of_rows)
    w = _weights(of_rows)
    w["V1"], w["V2"], w["b2"] = torch.zeros((2 * M, N), dtype=of_rows), torch.zeros((N, 2 * M), dtype=of_rows), torch.zeros(2 * M)
    _refused(maker, w, of_rows)


@pytest.mark.parametrize("maker", ["shared", "trained", "few", "block", "served"])
def test_weights_on_another_device_are_refused(maker):
    w = {n: torch.empty(s, dtype=F32 if n in VECTORS else BF16, device="meta") for n, s in SHAPES.items()}
    with pytest.raises(ValueError, match="is on meta"):
        MAKE[maker](w, BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_fits_is_taken(dtype):
    w = _weights(dtype)
    for b in (w["b1"], None):
        shared = Shared(T, w["V1"], w["V2"], b, w["b2"], training=True, device="cpu", rows=(M, B.MOE_BF16 if dtype == BF16 else B.MOE_F32))
        assert all(g.dtype == F32 for g in shared.gradients())
        assert [g.shape for g in shared.gradients()] == [(M, N)] + ([(N,)] if b is not None else []) + [(N, M), (M,)]
    few = MAKE["few"](w, dtype)
    assert few.out.dtype == dtype and few.shared.a.dtype == dtype
