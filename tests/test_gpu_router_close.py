"""The router where float scores do not say which of two experts, or groups, comes first: the choice is that of 64-bit scores.

The reference works on whole arrays.  Where the scores that decide are closer than 2^-44 of their size, 64 bits do not
decide either, and the token is not compared."""
import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NEG = -np.inf


def scores(l, bias, sigmoid):
    l = l.astype(np.float64)
    if sigmoid:
        s = 1.0 / (1.0 + np.exp(-l))
    else:
        s = np.exp(l - l.max(1, keepdims=True))
        s /= s.sum(1, keepdims=True)
    return np.where(l > NEG, s + bias.astype(np.float64), NEG)


def first_k(v, k):
    """The k largest per row, and whether each is further than rounding from the next."""
    idx = np.argsort(-v, axis=1, kind="stable")
    top = np.take_along_axis(v, idx[:, :k + 1], 1)
    with np.errstate(invalid="ignore"):
        clear = (top[:, :-1] - top[:, 1:] > 2.0 ** -44 * np.abs(top[:, :-1])).all(1)
    return np.where(top[:, :k] > NEG, idx[:, :k], -1), clear


def router(l, bias, k, **kw):
    T, E = l.shape
    idx, w = torch.empty((T, k), dtype=torch.int32, device=DEV), torch.empty((T, k), device=DEV)
    B.moe_router_fwd(B.make_router_config(T, E, k, **kw), torch.from_numpy(l).to(DEV),
                     None if bias is None else torch.from_numpy(bias).to(DEV), idx, w)
    return idx.cpu().numpy(), w.cpu().numpy()


@pytest.mark.parametrize("base", [0.6, 1.2, 2.2])
@pytest.mark.parametrize("E,values", [(16, 1), (32, 2), (64, 4), (128, 8), (256, 16), (512, 32)])
def test_two_scores_around_a_multiple_of_a_lanes_values(E, values, base):
    """Two experts within a unit of a float's last place of each other, one of the last in its lane and one of the first, on
    both sides of a score whose low bits are zero."""
    rng, T = np.random.default_rng(E), 40000
    bias = (base - 0.5 + 0.15 * (rng.random(E) - 0.5)).astype(np.float32)
    lane = np.stack([rng.permutation(16)[:2] for _ in range(T)])
    pair = np.stack([lane[:, 0] * values + values - 1, lane[:, 1] * values], 1)
    edge = ((base + 0.1 * rng.random((T, 1))).astype(np.float32).view(np.uint32) & np.uint32(2 ** 32 - values)).view(np.float32)
    p = edge + rng.normal(0, 0.6, (T, 2)) * np.spacing(edge) - bias[pair].astype(np.float64)
    l = np.full((T, E), NEG, np.float32)
    np.put_along_axis(l, pair, np.log(p / (1 - p)).astype(np.float32), 1)
    want, clear = first_k(scores(l, bias, True), 2)
    assert clear.mean() > 0.9
    for k in (1, 2):
        assert np.array_equal(router(l, bias, k, scores=B.MOE_SIGMOID)[0][clear], want[clear, :k])
