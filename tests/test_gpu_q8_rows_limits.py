"""Rows to int8 whose squares or sums leave fp32's range."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B
from test_gpu_q8_rows import KINDS, TYPES, _check_rows, _g, _norm_in_64_bits, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("C", [16, 256, 1024, 2048, 16384])
def test_rows_of_any_size(dtype, kind, C):
    """Rows from 2^-130 to just below the largest number, beside ordinary ones."""
    g = _g(C + 1)
    ups = [0, 60, 63, 64, 70, 100, 120, 126, -38, -45, -50, -63, -70, -110, -130, 0]
    x = torch.rand((len(ups), C), generator=g, device="cuda") + 0.25       # (a mean far from zero: its sum overflows too)
    x[:, ::3] *= -0.5
    x = (x.double() * torch.exp2(torch.tensor(ups, device="cuda").double())[:, None]).to(dtype)
    weight = None if kind == B.NORM_NONE else _randn(g, C, dtype=dtype)
    for eps in (0.0, 1e-35, 2.0 ** -80, 1e-6):
        q, scale = B.k_norm_q8(x, weight=weight, kind=kind, eps=eps)
        y = _norm_in_64_bits(x, kind, weight, None, eps)
        some = y.abs().amax(1) >= 2.0 ** -118            # (below 2^-119: zeros)
        _check_rows(q[some], scale[some], y[some])
        assert eps > 1e-35 or kind == B.NORM_NONE or int(some.sum()) >= len(ups) - (eps > 0)
