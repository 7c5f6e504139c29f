"""The 4-bit products' scratch, without a GPU: every refusal is a status code before anything is launched."""
import ctypes

import pytest

from paper_2506_22175_amd import binding as B

P, NONE = ctypes.c_void_p(4096), ctypes.c_void_p(0)
NULL = 1


def test_many_assignments_have_a_list_in_the_scratch():
    """Workgroups that all look through the assignments for their rows read their number times the grid, which grows with them:
    T * k = 2^24 would take hours.  Beyond 2048 they are listed once, which needs 4 bytes each and some for each expert."""
    need = lambda T, k, **kw: B.moe_w4_scratch_bytes(B.make_w4_config(T, k, 16, 64, 64, **kw))  # noqa: E731
    assert need(1024, 2) == 0 and need(1, 1) == 0
    for T, k in ((1025, 2), (1 << 20, 4), (1 << 23, 2)):
        assert need(T, k) >= 4 * (T * k + 16)
    joined = [need(T, 2, combine=1) for T in (1, 2, 100, 1024, 1025, 1026, 65535)]
    assert joined == sorted(joined)
    assert joined[4] >= 1025 * 2 * (64 * 4 + 4)


@pytest.mark.parametrize("combine", [0, 1])
def test_the_list_needs_its_scratch(combine):
    cfg = B.make_w4_config(3000, 2, 16, 64, 64, combine=combine)
    args = [P] * 8
    args[7] = NONE
    assert B.lib().moe_w4_product(ctypes.byref(cfg), *args, None) == NULL


def test_more_columns_than_a_launch_has_workgroups_for():
    """2^26 columns with sixteen wavefronts for each 16 of them would be 2^32 threads, of which none would start."""
    P8 = [P] * 8
    most = (1 << 26) - 16
    for N, status in ((most + 1, 3), ((1 << 26) - 1, 3)):
        cfg = B.make_w4_config(1, 16, 16, 32, N, combine=1)
        assert B.lib().moe_w4_product(ctypes.byref(cfg), *P8, None) == status
    assert B.moe_w4_scratch_bytes(B.make_w4_config(1, 16, 16, 32, most, combine=1)) == 0
