"""Slots where a token has fewer choices than k: entries outside 0..E-1 take no position and get slot -1."""
import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
D = "cuda:0"


def _slots(idx, n, E, Cp):
    """Positions choice by choice, then in token order, inside each partition."""
    T, k = idx.shape
    slot, counts = np.full((T, k), -1, np.int32), np.zeros((n, E), np.int32)
    for p in range(n):
        for j in range(k):
            for t in range(p * (T // n), (p + 1) * (T // n)):
                e = idx[t, j]
                if 0 <= e < E and counts[p, e] < Cp:
                    slot[t, j] = e * Cp + counts[p, e]
                    counts[p, e] += 1
    return slot, counts


@pytest.mark.parametrize("T,n,E,k", [
    (1, 1, 1, 1), (40, 2, 5, 3), (130, 1, 64, 2), (1024, 1, 7, 3),      # counted by the ranking kernel itself
    (1025, 1, 3, 3), (4096, 2, 8, 2), (5000, 1, 64, 8),                 # counted by a launch of its own
])
@pytest.mark.parametrize("static", [False, True])
def test_entries_that_are_no_choice(T, n, E, k, static):
    rng = np.random.default_rng(T + E)
    idx = rng.integers(0, E, (T, k)).astype(np.int32)
    idx[rng.random((T, k)) < 0.3] = -1
    idx[T // 2:T // 2 + 70] = -1                        # more than a wavefront of tokens without any choice
    idx[0, k - 1] = E                                   # just outside
    w = rng.random((T, k), dtype=np.float32)
    cfg = B.make_config(T, 8, 8, E, k, 0.75, n, B.MOE_BF16, 0)
    Cp = B.moe_capacity(cfg)
    want, counts = _slots(idx, n, E, Cp)
    d_idx, d_w = torch.from_numpy(idx).to(D), torch.from_numpy(w).to(D)
    slot = torch.full((T, k), -9, dtype=torch.int32, device=D)
    c = torch.full((n, E), -9, dtype=torch.int32, device=D)
    slot_w = torch.full((n * E * Cp,), -1.0, device=D)
    if static:
        B.moe_assign_slots_static(cfg, d_idx, d_w, slot, c, slot_w)
    else:
        scratch = torch.full((B.moe_slot_scratch_bytes(cfg),), 0xFF, dtype=torch.uint8, device=D)
        B.moe_assign_slots(cfg, d_idx, d_w, slot, c, slot_w, scratch)
    assert np.array_equal(slot.cpu().numpy(), want) and np.array_equal(c.cpu().numpy(), counts)
    rows = np.full((n * E * Cp,), -1.0, np.float32)
    at = np.arange(T)[:, None] // (T // n) * (E * Cp) + want
    rows[at[want >= 0]] = w[want >= 0]
    assert np.array_equal(slot_w.cpu().numpy(), rows)
