"""Refusals of the gate's weight gradient: status codes before anything is launched, no GPU needed."""
import ctypes

from paper_2506_22175_amd import binding as B

P = ctypes.c_void_p(4096)


def test_refusals():
    call = lambda cfg, part=0, args=(P,) * 4: B.lib().moe_gate_weight_grad(ctypes.byref(cfg), part, *args, None)  # noqa: E731
    ok = B.make_config(256, 64, 128, 4, 1, 1.25, 2)
    for missing in range(4):                                     # x, dL, dWg, scratch
        assert call(ok, 0, [None if i == missing else P for i in range(4)]) == 1
    assert call(ok, 2) == 2 and call(ok, -1) == 2
    assert call(B.make_config(256, 64, 128, 4, 5, 1.25)) == 2
    assert call(B.make_config(256, 64, 128, 65, 1, 1.25)) == 3 and call(B.make_config(256, 60, 128, 4, 1, 1.25)) == 3
    assert B.lib().moe_gate_weight_grad(None, 0, P, P, P, P, None) == 1
