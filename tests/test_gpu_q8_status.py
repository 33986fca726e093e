"""The int8 product called without a status word of the caller's."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B
from test_gpu_q8_linear import _case, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [0, 3, 700])
def test_without_a_status_word(M):
    a, as_, w, ws, x, st = _case(M, 264, 80)
    want, got, sums = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    B.k_linear_q8(a, as_, w, ws, (want,), status=st)
    B.k_linear_q8(a, as_, w, ws, (got,), residual=x, sum_out=sums)
    assert torch.equal(got, want) and torch.equal(got, _t(a, as_, w, ws)) and torch.equal(sums, x + want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got.zero_()
    side.wait_stream(torch.cuda.current_stream())
    B.k_linear_q8(a, as_, w, ws, (got,), stream=side)     # (it has waited for its own stream)
    assert torch.equal(got, want)
