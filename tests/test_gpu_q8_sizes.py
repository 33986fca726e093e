"""The 8-bit operators where indexes pass 2^31, and with more sequences than a grid's second dimension holds."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B
from test_gpu_q8_attention import _case, _g
from test_gpu_q8_limits import _check
from test_gpu_q8_linear import _t

pytestmark = pytest.mark.gpu


def _slices(rows, width):
    at = 2 ** 31 // width
    return (slice(0, 70), slice(at - 70, at + 70), slice(rows - 150, rows))


def test_products_of_more_than_2_31_results():
    M, N, K = 2 ** 21 + 130, 1032, 32
    g = _g(1)
    a = torch.randint(-127, 128, (M, K), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-127, 128, (N, K), generator=g, device="cuda").to(torch.int8)
    as_, ws = (torch.rand(n, generator=g, device="cuda") * 0.02 for n in (M, N))
    st = torch.zeros(16, dtype=torch.int32, device="cuda")
    t, s = (torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = torch.ones((M, N), dtype=torch.bfloat16, device="cuda")
    B.k_linear_q8(a, as_, w, ws, (t,), status=st)
    B.k_linear_q8(a, as_, w, ws, (), residual=x, sum_out=s, status=st)
    for rows in _slices(M, N):
        want = _t(a[rows], as_[rows], w, ws)
        assert torch.equal(t[rows], want) and torch.equal(s[rows], 1 + want)
    assert int(st[0]) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_more_than_2_31_elements(dtype):
    rows, C = 2 ** 21 + 130, 1040
    x = torch.randn((1000, C), generator=_g(2), device="cuda").to(dtype).repeat(rows // 1000 + 1, 1)[:rows].contiguous()
    total = torch.empty_like(x)
    q, scale = B.k_norm_q8(x, residual=x, sum_out=total)
    for part in _slices(rows, C):
        want = B.k_norm_q8(x[part], residual=x[part])
        assert torch.equal(q[part], want[0]) and torch.equal(scale[part], want[1]) and torch.equal(total[part], x[part] * 2)


@pytest.mark.parametrize("seqs,M,heads,kv,capacity", [(66000, 1, 2, 1, 16), (66000, 12, 1, 1, 16), (5000, 200, 1, 1, 400)])
def test_many_sequences(seqs, M, heads, kv, capacity):
    """A hundred sequences over and over: each as the first time, wherever it lies, and the first hundred as they should be."""
    q, cache = _case(100, M, heads, kv, capacity)
    again = lambda t: t.repeat(seqs // 100, *[1] * (t.dim() - 1))
    lens = torch.randint(0, capacity + 1, (100,), generator=_g(3), device="cuda", dtype=torch.int32)
    many = B.new_cache_q8(seqs, capacity, kv)
    k, v = B.k_load_q8(cache, capacity)
    B.k_store_q8(many, again(k), again(v))
    assert all(torch.equal(m, again(c)) for m, c in zip(many, cache))
    live = (torch.rand((100, capacity), generator=_g(4), device="cuda") < 0.7).to(torch.uint8)
    out = B.k_attention_q8(again(q), many, lens=again(lens), live=again(live)).view(seqs // 100, 100, M, -1)
    first = out[0].clone()
    assert bool((out == first).all())
    want = _check(q, cache, lens, live)
    # (the hundred alone are cut otherwise: both are within the tolerance, twice the result's rounding and that of its weights)
    assert float((first.double() - want.double()).abs().max()) <= 2.0 ** -6 * float(want.abs().max())
