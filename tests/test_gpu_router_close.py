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


@pytest.mark.parametrize("E,groups,size", [(16, 8, 1e4), (16, 8, 1e2), (64, 8, 1e4), (256, 8, 1e3), (512, 16, 1e4), (48, 16, 1e3), (33, 11, 1e4)])
@pytest.mark.parametrize("sigmoid", [0, 1])
def test_groups_whose_two_best_nearly_cancel(E, groups, size, sigmoid):
    """Each group has one bias of + size and the others of - size: a group's score is some 1, and its parts are rounded as size."""
    rng, T, per, stay = np.random.default_rng(E + groups), 20000, E // groups, 3
    bias = np.full(E, -size, np.float32)
    bias[np.arange(groups) * per + rng.integers(0, per, groups)] = size
    l = (rng.standard_normal((T, E)) * 1.5).astype(np.float32)
    v = scores(l, bias, sigmoid)
    by_group = -np.sort(-v.reshape(T, groups, per), 2)[:, :, :2].sum(2)
    kept, _ = first_k(by_group, groups)
    ranked = np.take_along_axis(by_group, kept, 1)
    # sums of the parts in 64 bits: good to 2^-52 of `size`
    clear = ranked[:, stay - 1] - ranked[:, stay] > 2.0 ** -50 * size
    inside = (np.arange(E)[None, :] // per == kept[:, :stay, None]).any(1)
    # the one expert of each group with + size; the others are as far apart as rounding at `size` leaves them
    want = np.where(inside & (bias > 0), v, NEG)
    order, apart = first_k(want, stay)
    clear &= apart
    assert clear.mean() > 0.9
    idx = router(l, bias, stay, scores=sigmoid, groups=groups, group_k=stay, group_top=2)[0]
    assert np.array_equal(np.sort(idx[clear], 1), np.sort(order[clear], 1))


def test_a_wide_softmax_adds_its_small_terms():
    """Sixteen largest logits, each followed in its lane by terms of just under half a unit of 1: added to it one by one they
    would all be lost, 31 units of 2^-24 of the sum.  Each term passes through at most log2(32) + 4 additions; the quotient,
    a product and the smallest terms' own errors add three units more."""
    E, T = 512, 8
    l = np.full((T, E), np.log(0.9995 * 2.0 ** -24), np.float32)
    l[:, ::32] = 0.0
    idx, w = router(l, None, 16)
    s = scores(l, np.zeros(E, np.float32), 0)
    assert np.array_equal(idx, np.broadcast_to(np.arange(0, E, 32), (T, 16)))
    assert (np.abs(w - s[:, ::32]) <= 12 * 2.0 ** -24 * s[:, ::32]).all()


@pytest.mark.parametrize("E", [64, 128, 256, 512])
def test_softmax_parts_that_a_bias_brings_together(E):
    """A large part and one of nothing, whose bias makes up for it to some units of the sum's last place; many small terms."""
    rng, T, values = np.random.default_rng(E), 20000, max(1, E // 16)
    bias = np.zeros(E, np.float32)
    a, b = 0, E - 1
    l = (np.log(2.0 ** -24) - rng.random((T, E)) * 0.01).astype(np.float32)
    l[:, ::values] = 0.0
    l[:, b] = -60.0
    bias[:] = -8.0
    bias[a], bias[b] = -1.0 / 16, 0.0
    l[:, a] = (rng.normal(0, 2e-6, T)).astype(np.float32)
    v = scores(l, bias, 0)
    want, clear = first_k(v, 2)
    assert clear.mean() > 0.9 and 0.05 < (want[:, 0] == a).mean() < 0.95
    assert np.array_equal(router(l, bias, 2)[0][clear], want[clear])
