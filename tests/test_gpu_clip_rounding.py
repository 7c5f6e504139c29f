"""Clipped bfloat16 gradients are products of 64 bits, rounded once: exactly, also where the product lies so near the middle of two
bfloat16 that its nearest float is that middle."""
import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
D = "cuda:0"
BF16 = torch.bfloat16


def _rounded(d):
    """float64 to bfloat16's 8 bits, ties to even; its numbers end at 2^-133."""
    unit = np.ldexp(1.0, np.maximum(np.frexp(d)[1] - 8, -133))
    return np.rint(d / unit) * unit


def _factors(seed, count):
    """Pairs of floats (most, norm) whose quotient takes some bfloat16 of [1,2) next to a middle."""
    rng = np.random.default_rng(seed)
    for _ in range(count):
        g, middle = 1 + rng.integers(128) / 128, (2 * (256 + rng.integers(256)) + 1) / 2 ** 10
        norm = np.float32(1 + rng.random())
        yield np.float32(float(norm) * min(middle / g / 2, 0.999)), norm


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("extra", [0, 1])                        # of an odd number the last is a value by itself
def test_products_next_to_the_middle_of_two(extra, in_place):
    sizes = [2.0 ** e for e in (0, 20, -20, -100, -118, -126, -130)]
    values = np.concatenate([[s * (1 + m / 128) * sign for m in range(128) for sign in (1, -1)] for s in sizes] + [np.full(extra, 1.5)])
    start = torch.from_numpy(values).to(BF16).to(D)
    g64 = start.double().cpu().numpy()
    grads = [start.clone()]
    outs = grads if in_place else [torch.empty_like(start)]
    lst = B.make_grad_list(grads, outs)
    through_float = 0
    for most, norm in _factors(extra, 200):
        grads[0].copy_(start)
        B.moe_grad_scale(lst, float(most), torch.tensor([norm], device=D))
        d = g64 * (float(most) / float(norm))
        want = _rounded(d)
        through_float += int((_rounded(d.astype(np.float32).astype(np.float64)) != want).sum())
        got = outs[0].double().cpu().numpy()
        assert (got == want).all(), (most, norm, np.flatnonzero(got != want)[:5])
    assert through_float > 20                                    # results that a second rounding would change


def test_what_has_no_rounding_is_kept():
    t = torch.tensor([0.0, -0.0, float("inf"), -float("inf"), float("nan"), 2.0 ** -133, 3.0 * 2.0 ** 100], device=D).to(BF16)
    out = torch.empty_like(t)
    lst = B.make_grad_list([t], [out])
    for most, norm, factor in ((0.5, 1.0, 0.5), (2.0, 1.0, 1.0), (1.0, float("nan"), 1.0), (1.0, float("inf"), 1.0)):
        B.moe_grad_scale(lst, most, torch.tensor([norm], device=D))
        want = [0.0, -0.0, float("inf"), -float("inf"), 0.0 if factor < 1 else 2.0 ** -133, 3.0 * 2.0 ** 100 * factor]
        got = out.double().tolist()
        assert got[4] != got[4] and got[:4] + got[5:] == want and str(got[1]) == "-0.0"
