"""The router's weights and their gradients where logits lie far apart: their relative error does not grow with the distance.

Units of 2^-24, relative to a weight: the exponential 2, the difference's rest and its product 2, the sum 7 additions and 11 of its
terms' own exponentials (what 64 terms of any size can make), the quotient or reciprocal, products with it and with the
scale 4; the sum of a renormalised weight 5 additions and 5 of its terms.  32 covers them.  A gradient's terms are
products of two weights and their sum over the choices: 128 of the sum of their magnitudes."""
import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(span, E=64, T=2000):
    rng = np.random.default_rng(int(span))
    return (rng.uniform(-span, span, (T, E))).astype(np.float32), rng


@pytest.mark.parametrize("span", [1, 10, 30, 42])
@pytest.mark.parametrize("sigmoid,renorm", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_weights(span, sigmoid, renorm):
    l, rng = inputs(span)
    T, E = l.shape
    k = 16
    if sigmoid:
        l -= np.float32(span / 2)                            # down to where a sigmoid is all exponential
    bias = rng.permuted(np.linspace(-1e4, 1e4, E)).astype(np.float32)          # chooses whatever the logits are
    idx, w = torch.empty((T, k), dtype=torch.int32, device=DEV), torch.empty((T, k), device=DEV)
    B.moe_router_fwd(B.make_router_config(T, E, k, sigmoid, renormalize=renorm, scale=2.5), torch.from_numpy(l).to(DEV),
                     torch.from_numpy(bias).to(DEV), idx, w)
    want_idx = np.argsort(-bias, kind="stable")[:k]
    assert (idx.cpu().numpy() == want_idx).all()
    z = l.astype(np.float64)
    s = 1 / (1 + np.exp(-z)) if sigmoid else np.exp(z - z.max(1, keepdims=True))
    s = s if sigmoid else s / s.sum(1, keepdims=True)
    s = s[:, want_idx]
    want = (s / s.sum(1, keepdims=True) if renorm else s) * 2.5
    # (below the normal floats a value's last place is 2^-149; weights that small are not compared relatively)
    assert (np.abs(w.cpu().numpy() - want) <= 32 * 2.0 ** -24 * want + 2.0 ** -140).all()


@pytest.mark.parametrize("span", [1, 10, 30, 42])
@pytest.mark.parametrize("sigmoid", [0, 1])
def test_gradients_of_renormalised_weights(span, sigmoid):
    l, rng = inputs(span)
    T, E = l.shape
    k = 16
    idx = np.ascontiguousarray(rng.permuted(np.broadcast_to(np.arange(E), (T, E)), axis=1)[:, :k].astype(np.int32))
    dw = rng.standard_normal((T, k)).astype(np.float32)
    dl = torch.empty((T, E), device=DEV)
    B.moe_router_bwd(B.make_router_config(T, E, k, sigmoid, renormalize=1), torch.from_numpy(l).to(DEV), torch.from_numpy(idx).to(DEV),
                     torch.from_numpy(dw).to(DEV), dl)
    z = np.take_along_axis(l, idx, 1).astype(np.float64)
    a = 1 / (1 + np.exp(-z)) if sigmoid else np.exp(z - z.max(1, keepdims=True))
    w = a / a.sum(1, keepdims=True)
    d = dw.astype(np.float64)
    g, size = w * (d - (w * d).sum(1, keepdims=True)), w * (np.abs(d) + (w * np.abs(d)).sum(1, keepdims=True))
    if sigmoid:
        g, size = g / (1 + np.exp(z)), size / (1 + np.exp(z))
    got = np.take_along_axis(dl.cpu().numpy(), idx, 1)
    assert (np.abs(got - g) <= 128 * 2.0 ** -24 * size + 2.0 ** -140).all()
