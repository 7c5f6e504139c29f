"""The norm of many tensors and clipping by it, against 64 bits."""
import math

import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
D = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def _scratch(lst):
    return torch.full((B.moe_grad_scratch_bytes(lst) + 64,), 0xAB, dtype=torch.uint8, device=D)


def _norm(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


def _run(grads, most, in_place=False):
    outs = grads if in_place else [torch.full_like(g, 7.0) for g in grads]
    lst = B.make_grad_list(grads, outs)
    norm, scratch = torch.full((3,), 5.0, device=D), _scratch(lst)
    want = [g.clone() for g in grads]
    B.moe_grad_clip(lst, most, norm[1:2], scratch)
    assert (scratch[-64:] == 0xAB).all() and norm[0] == 5.0 and norm[2] == 5.0
    return float(norm[1]), outs, want


def _expected(grads, most, norm):
    """One rounding of the product with the quotient, which is in 64 bits."""
    factor = float(torch.tensor(most)) / norm if norm > float(torch.tensor(most)) else 1.0
    return [(g.double() * factor) for g in grads], factor


SIZES = {
    "one element": [1], "ends of chunks": [8191, 8192, 8193, 16384, 16385], "nothing among them": [0, 5, 0, 4097, 0],
    "more than a launch lays out": [3 + 7 * i for i in range(150)], "many chunks": [20_000_003, 1001],
}


@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("types", ["f32", "bf16", "both"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_clipping(sizes, types, offset):
    g = torch.Generator(device=D).manual_seed(len(sizes) + offset)
    grads = []
    for j, n in enumerate(SIZES[sizes]):
        t = F32 if types == "f32" or (types == "both" and j % 2) else BF16
        grads.append((torch.randn(n + offset, generator=g, device=D) * 10.0 ** (j % 5 - 2)).to(t)[offset:])
    true = _norm(grads)
    for most, in_place in ((0.37 * true, False), (0.37 * true, True), (3 * true, False)):
        mine = [t.clone() if offset == 0 else torch.cat([t[:0].new_zeros(offset), t])[offset:] for t in grads]
        norm, outs, before = _run(mine, most, in_place)
        # sums of squares in 64 bits: their error is far below the rounding to float
        assert abs(norm - true) <= true * (2.0 ** -24 + 1e-12)
        want, factor = _expected(before, most, norm)
        for o, w, b in zip(outs, want, before):
            if factor == 1.0:
                assert torch.equal(o, b)
            else:
                # float: the product of 53 bits, rounded again; bfloat16: by way of float, half a step of each
                half = 2.0 ** -24 * (1 + 1e-6) if o.dtype == F32 else 2.0 ** -8 + 2.0 ** -23
                assert ((o.double() - w).abs() <= half * w.abs() + 1e-45).all()


def test_norm_only_and_the_factor_of_a_norm_from_elsewhere():
    g = [torch.randn(1000, device=D), torch.randn(77, device=D).to(BF16)]
    lst = B.make_grad_list(g)
    norm, scratch = torch.zeros(1, device=D), _scratch(lst)
    B.moe_grad_norm(lst, norm, scratch)
    true = _norm(g)
    assert abs(float(norm) - true) <= true * 2.0 ** -23
    with pytest.raises(B.MoEError):
        B.moe_grad_scale(lst, 1.0, norm)
    both = B.make_grad_list(g, g)
    want = [t.double() * (0.5 / 8.0) for t in g]
    B.moe_grad_scale(both, 0.5, torch.tensor([8.0], device=D))
    assert all(torch.equal(t.double(), w) for t, w in zip(g, want))          # a power of two


@pytest.mark.parametrize("size", [1e30, 1e-30, 1e38, 3e38, 1e-42])
def test_sizes_whose_squares_no_float_holds(size):
    g = [torch.tensor([3.0, 0.0], device=D) * size, torch.tensor([-4.0], device=D).mul_(size if size < 1e38 else size / 4)]
    true = _norm(g)
    norm, outs, before = _run(g, 1e-3 * size)
    if size == 3e38:                                             # 9e38 is an infinity among the elements already
        assert norm == float("inf") and all(torch.equal(o, b) for o, b in zip(outs, before))
        return
    assert abs(norm - true) <= max(true * 2.0 ** -23, 1e-45)
    want, _ = _expected(before, 1e-3 * size, norm)
    for o, w in zip(outs, want):
        assert ((o.double() - w).abs() <= 2.0 ** -23 * w.abs() + 1.5e-45).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norms_that_are_no_number_scale_nothing(bad, dtype):
    for at in (0, 12345, 40001):
        g = [torch.ones(40002, device=D).to(dtype), torch.ones(5, device=D)]
        g[0][at] = bad
        norm, outs, before = _run(g, 0.5)
        assert math.isnan(norm) if math.isnan(bad) else norm == float("inf")
        for o, b in zip(outs, before):
            assert torch.equal(o.nan_to_num(nan=9.0), b.nan_to_num(nan=9.0))


def test_limits_and_empty_lists():
    g = [torch.tensor([3.0, 4.0], device=D)]
    assert _run(g, 5.0)[1][0].tolist() == [3.0, 4.0]             # as large as allowed
    assert _run(g, 0.0)[1][0].tolist() == [0.0, 0.0]
    zeros = [torch.zeros(10, device=D)]
    norm, outs, _ = _run(zeros, 0.0)
    assert norm == 0.0 and outs[0].tolist() == [0.0] * 10
    for empty in ([], [torch.zeros(0, device=D)]):
        norm, _, _ = _run(empty, 1.0)
        assert norm == 0.0


def test_the_same_bits_every_time_and_from_graphs():
    """The last workgroup to finish adds the others' sums up, whichever it is; its count starts again by itself."""
    g = [torch.randn(3_000_001, device=D), torch.randn(100_000, device=D).to(BF16)]
    outs = [torch.empty_like(t) for t in g]
    lst = B.make_grad_list(g, outs)
    norm, scratch = torch.zeros(1, device=D), _scratch(lst)
    B.moe_grad_clip(lst, 1.0, norm, scratch)
    first = [norm.clone()] + [o.clone() for o in outs]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_grad_clip(lst, 1.0, norm, scratch)
    for _ in range(20):
        norm.fill_(-1.0)
        outs[0].fill_(-1.0)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(first, [norm] + outs))
        norm.fill_(-1.0)
        B.moe_grad_clip(lst, 1.0, norm, scratch)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, [norm] + outs))
    for t in g:                                                  # other values at the same addresses
        t.mul_(2.0)
    graph.replay()
    assert float(norm) == 2 * float(first[0])


def test_two_lists_on_two_streams():
    streams = [torch.cuda.Stream() for _ in range(2)]
    g = [[torch.randn(2_000_000 + 37 * i, device=D)] for i in range(2)]
    lists = [B.make_grad_list(t, t) for t in g]
    norms, scratch = [torch.zeros(1, device=D) for _ in g], [_scratch(lst) for lst in lists]
    true = [_norm(t) for t in g]
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            B.moe_grad_clip(lists[i], 1.0, norms[i], scratch[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert abs(float(norms[i]) - true[i]) <= true[i] * 2.0 ** -23
        assert abs(_norm(g[i]) - 1.0) <= 1e-6


def test_lists_refuse_what_they_cannot_hold():
    t = torch.zeros(8, device=D)
    for grads, outs in (([t.to(torch.float16)], None), ([t[::2]], None), ([t], [t, t]), ([t], [t[:4]]), ([t], [t.to(BF16)]), ([t], [t.cpu()])):
        with pytest.raises(ValueError):
            B.make_grad_list(grads, outs)
    with pytest.raises(B.MoEError) as e:
        B.make_grad_list([t, t], [t, t])
    assert e.value.status == 2
    B.make_grad_list([t, t])                                     # norms of the same tensor twice are no race


@pytest.mark.parametrize("handle", [False, True])
def test_the_table_belongs_to_the_stream_that_writes_it(handle):
    """Memory that the current stream still uses is not handed to another one."""
    grads = [torch.full((1000,), 2.0, device=D)]
    need = B.make_grad_list(grads).memory.numel()
    torch.cuda.synchronize()
    freed = [torch.empty(need, dtype=torch.uint8, device=D) for _ in range(4)]
    places = {t.data_ptr() for t in freed}
    freed.clear()
    side = torch.cuda.Stream()
    lst = B.make_grad_list(grads, stream=side.cuda_stream if handle else side)
    assert lst.memory.data_ptr() not in places
    norm, scratch = torch.zeros(1, device=D), _scratch(lst)
    side.wait_stream(torch.cuda.current_stream())
    B.moe_grad_norm(lst, norm, scratch, side)
    side.synchronize()
    assert float(norm) == float(torch.tensor(math.sqrt(4000.0)))
