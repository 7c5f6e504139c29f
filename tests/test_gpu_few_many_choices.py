"""The layer for a few tokens where a few have many choices: up to four tokens route inside the first product, and their assignments are 32 at
most, which the lanes have, or more, which go by way of LDS."""
import pytest

from paper_2506_22175_amd import binding as B
from test_gpu_few import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [B.MOE_F32, B.MOE_BF16])
@pytest.mark.parametrize("T,M,H,E,k", [(1, 64, 72, 16, 16), (2, 64, 72, 16, 16), (2, 1032, 264, 64, 16), (3, 72, 64, 20, 10), (3, 72, 64, 20, 11), (3, 520, 136, 64, 16),
                                       (4, 72, 64, 8, 8), (4, 520, 264, 33, 9), (4, 64, 1032, 64, 16), (5, 72, 64, 20, 6), (5, 72, 64, 20, 7), (8, 264, 72, 16, 4)])
def test_about_as_many_choices_as_lanes_have(T, M, H, E, k, dtype):
    for kw in (dict(renormalize=1), dict(scores=B.MOE_SIGMOID, scale=2.5)):
        layer = Layer(T, M, H, E, k, dtype, seed=T + E + k, **kw)
        layer.run()
        layer.check()
