"""The 8-bit norm's values are the quotients by the scale, rounded to the nearest: bit for bit where y is known exactly."""
import numpy as np
import pytest
import torch

from paper_2506_22175_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("M,group", [(256, 0), (777, 0), (4000, 0), (4000, 128), (20000, 0)])
def test_quotients_next_to_the_middle_of_two_values(M, group):
    """Rows of ones and eps = 0: y is the gain.  Gains are floats next to the scale times the middle of two neighbouring values
    of the type; a float quotient is rounded once, so the stored values are determined."""
    rng = np.random.default_rng(M)
    values = np.unique(np.abs(np.arange(127, dtype=np.uint8).view(np.uint8)))
    values = torch.from_numpy(values).view(torch.float8_e4m3fn).double().numpy()
    middles = (values[1:] + values[:-1]) / 2
    for _ in range(20):
        most = np.float32(rng.uniform(0.5, 2.0))
        scale = np.float32(most / np.float32(448))
        gain = (rng.choice(middles, M) * np.float64(scale)).astype(np.float32)
        gain = np.where(rng.random(M) < 0.5, gain, np.nextafter(gain, np.float32(rng.choice([0.0, 9.0])))) * rng.choice(np.float32([-1, 1]), M)
        gain = gain.astype(np.float32)
        gain[::128] = most
        want = torch.from_numpy(gain / scale).to(torch.float8_e4m3fn).view(torch.uint8)
        x = torch.ones((2, M), device=DEV)
        q, s = torch.empty((2, M), dtype=torch.uint8, device=DEV), torch.empty((2, -(-M // 128) if group else 1), device=DEV)
        B.moe_norm_fwd(B.make_norm_config(2, M, 0.0, B.MOE_F32, B.MOE_E4M3, group), x, None, torch.from_numpy(gain).to(DEV), None, q, s)
        assert (s.cpu() == float(scale)).all()
        assert torch.equal(q[0].cpu(), want) and torch.equal(q[1].cpu(), want)
