"""Rows to int8 behind a residual and a norm; keys and values into and out of an 8-bit cache."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]
KINDS = [B.NORM_NONE, B.NORM_RMS, B.NORM_LAYER]


def _g(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _norm_in_64_bits(h, kind, weight, bias, eps):
    y = h.double()
    if kind == B.NORM_LAYER:
        y = y - y.mean(-1, keepdim=True)
    if kind != B.NORM_NONE:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        y = y if weight is None else y * weight.double()
        y = y if bias is None else y + bias.double()
    return y


def _check_rows(q, scale, y):
    # a thread adds at most 64 terms in a row and the rest is a tree: under 100 roundings of 2^-24, on the mean and on the squares, and a
    # few more until y: 2e-5.  The quotient is off by 127 times that, and its rounding by half.
    most = y.abs().amax(-1)
    torch.testing.assert_close(scale.double(), most / 127, rtol=2e-5, atol=0)
    off = (q.double() - y / (most / 127).clamp(min=1e-300)[..., None]).abs()
    assert float(off.max()) <= 0.5 + 127 * 3e-5
    assert int(q.abs().max()) <= 127


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,C", [(1, 16), (5, 240), (4, 256), (33, 272), (7, 512), (1, 1024), (718, 768), (3, 1040), (2, 2048), (5, 2064), (9, 4096),
                                    (2, 5008), (3, 8192), (2, 16384)])
def test_rows(dtype, kind, rows, C):
    g = _g(rows + C)
    x, r = _randn(g, rows, C, dtype=dtype), _randn(g, rows, C, dtype=dtype)
    weight, bias = (None, None) if kind == B.NORM_NONE else (_randn(g, C, dtype=dtype), _randn(g, C, dtype=dtype))
    total = torch.empty_like(x)
    q, scale = B.k_norm_q8(x, weight=weight, bias=bias, residual=r, kind=kind, sum_out=total)
    h = (x.float() + r.float()).to(dtype)
    assert torch.equal(total, h)
    _check_rows(q, scale, _norm_in_64_bits(h, kind, weight, bias, 1e-6))
    q, scale = B.k_norm_q8(x, kind=kind, eps=0.25)
    _check_rows(q, scale, _norm_in_64_bits(x, kind, None, None, 0.25))


@pytest.mark.parametrize("C", [256, 4096])
def test_sum_in_place_and_leading_dimensions(C):
    g = _g(3)
    x, r = _randn(g, 3, 5, C, dtype=torch.bfloat16), _randn(g, 3, 5, C, dtype=torch.bfloat16)
    want_sum = torch.empty_like(x)
    want = B.k_norm_q8(x, residual=r, sum_out=want_sum)
    for into in (x.clone(), r.clone()):
        a, b = (into, r) if torch.equal(into, x) else (x, into)
        q, scale = B.k_norm_q8(a, residual=b, sum_out=into)
        assert torch.equal(into, want_sum) and torch.equal(q, want[0]) and torch.equal(scale, want[1])
    assert want[1].shape == (3, 5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("C", [64, 2048])
def test_rows_of_zeros_and_rows_that_are_not_finite(dtype, kind, C):
    x = _randn(_g(C), 8, C, dtype=dtype)
    alone = B.k_norm_q8(x, kind=kind)
    x[1] = 0
    x[3, C - 1] = float("inf")
    x[5, 0] = float("nan")
    x[6] = 1e-37 if kind == B.NORM_NONE else 0
    q, scale = B.k_norm_q8(x, kind=kind)
    assert not bool(q[[1, 3, 5, 6]].any()) and bool((scale[[1, 6]] == 0).all()) and bool(scale[[3, 5]].isnan().all())
    for i in (0, 2, 4, 7):
        assert torch.equal(q[i], alone[0][i]) and torch.equal(scale[i], alone[1][i])


def test_ties_and_the_largest_value():
    x = torch.zeros((1, 16), device="cuda")
    x[0, :6] = torch.tensor([127.0, -127.0, 0.5, 1.5, 2.5, -2.5])
    q, scale = B.k_norm_q8(x, kind=B.NORM_NONE)
    assert q[0, :6].tolist() == [127, -127, 0, 2, 2, -2] and float(scale[0]) == 1.0
    assert B.k_norm_q8(x[:0], kind=B.NORM_NONE)[0].shape == (0, 16)


# ------------------------------------------------------------------ the cache

def _pow2(e):
    """2^e in fp64, exact (a library's power is off by a bit for some whole exponents)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _blocks(x):
    """What a cache holds of [..., 64] (fp64, finite): whole numbers and the exponent."""
    most = x.abs().amax(-1)
    e = torch.full_like(most, -120.0)
    for k in range(-120, 128):
        e = torch.where(most >= 2.0 ** k, float(k), e)
    q = torch.round(x * _pow2(6 - e)[..., None])
    return q.clamp(-127, 127), e


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("seqs,M,heads,capacity", [(1, 1, 1, 16), (3, 7, 5, 32), (4, 1, 16, 160), (2, 69, 4, 336), (1, 329, 12, 1008)])
def test_store_and_load(dtype, seqs, M, heads, capacity):
    g = _g(M)
    k, v = (_randn(g, seqs, M, heads * 64, dtype=dtype) * torch.exp2(torch.randint(-9, 9, (seqs, M, 1), generator=g, device="cuda").float()).to(dtype)
            for _ in range(2))
    cache = B.new_cache_q8(seqs, capacity, heads)
    before = [c.random_(0, 100, generator=g).clone() for c in cache]
    start = torch.randint(0, capacity - M + 1, (seqs,), generator=g, device="cuda", dtype=torch.int32)
    B.k_store_q8(cache, k, v, start=start)
    back = B.k_load_q8(cache, capacity, dtype=dtype)
    for x, q8, ex, was_q, was_x, read in ((k, cache[0], cache[1], before[0], before[1], back[0]), (v, cache[2], cache[3], before[2], before[3], back[1])):
        q, e = _blocks(x.double().view(seqs, M, heads, 64))
        for s in range(seqs):
            at = int(start[s])
            inside = torch.zeros(capacity, dtype=torch.bool, device="cuda")
            inside[at:at + M] = True
            assert torch.equal(q8[s][inside].double().view(M, heads, 64), q[s])
            assert torch.equal(ex[s][:, inside].double().T, e[s] + 127)
            assert torch.equal(q8[s][~inside], was_q[s][~inside]) and torch.equal(ex[s][:, ~inside], was_x[s][:, ~inside])
            want = (q[s] * _pow2(e[s] - 6)[..., None]).view(M, -1)
            assert torch.equal(read[s, at:at + M].double(), want)
    # writing what was read gives the same bytes; a part of the rows reads as the whole
    again = B.new_cache_q8(seqs, capacity, heads)
    B.k_store_q8(again, *back)
    twice = B.k_load_q8(again, capacity, dtype=dtype)
    n = capacity // 3
    part = B.k_load_q8(cache, n, first=capacity - n, dtype=dtype)
    for s in range(seqs):
        rows = slice(int(start[s]), int(start[s]) + M)
        assert torch.equal(again[0][s, rows], cache[0][s, rows]) and torch.equal(again[3][s, :, rows], cache[3][s, :, rows])
        assert torch.equal(twice[1][s, rows], back[1][s, rows])
    assert torch.equal(part[0], back[0][:, capacity - n:]) and torch.equal(part[1], back[1][:, capacity - n:])


@pytest.mark.parametrize("dtype", TYPES)
def test_blocks_at_their_limits(dtype):
    """Powers of two and their neighbours, ties, the smallest and largest exponents, zeros, blocks that are not finite."""
    x = torch.zeros((1, 12, 64), dtype=torch.float64)
    x[0, 0, :3] = torch.tensor([2.0, 1.9921875, -1.9921875])
    x[0, 1, :5] = torch.tensor([1.0, 1 / 128, 3 / 128, -3 / 128, 63.5 / 64])
    x[0, 2, :2] = torch.tensor([1.9921875, -1.9921875])             # 127.5: at most 127
    x[0, 3, 5] = 2.0 ** -120
    x[0, 4, 5:7] = torch.tensor([2.0 ** -121, 2.0 ** -127])
    x[0, 5, 7] = -float(torch.finfo(dtype).max)
    x[0, 7, 63] = float("inf")
    x[0, 8, 0], x[0, 8, 1] = float("nan"), 1.0
    x[0, 9, 0], x[0, 9, 1] = -float("inf"), float("nan")
    x[0, 10] = 2.0 ** -126
    k = x.to("cuda").to(dtype)
    cache = B.new_cache_q8(1, 16, 1)
    B.k_store_q8(cache, k, -k)
    odd = torch.zeros(12, dtype=torch.bool, device="cuda")
    odd[7:10] = True
    q, e = _blocks(k[0].double()[~odd])
    for c, s in ((cache[0], 1), (cache[2], -1)):
        assert torch.equal(c[0, :12][~odd].double(), s * q) and not bool(c[0, :12][odd].any())
    for c in (cache[1], cache[3]):
        assert torch.equal(c[0, 0, :12][~odd].double(), e + 127) and bool((c[0, 0, :12][odd] == 255).all())
    back = B.k_load_q8(cache, 12, dtype=dtype)[0][0]
    assert bool(back[odd].isnan().all())
    assert torch.equal(back[~odd].double(), q * _pow2(e - 6)[:, None])


def test_store_skips_sequences_and_rows():
    g = _g(1)
    k, v = _randn(g, 4, 3, 64), _randn(g, 4, 3, 64)
    cache = B.new_cache_q8(4, 16, 1)
    B.k_store_q8(cache, k, v, start=torch.tensor([-1, 14, 16, 0x7FFFFFFF], dtype=torch.int32, device="cuda"))
    got = B.k_load_q8(cache, 16, dtype=torch.float32)
    whole = B.new_cache_q8(4, 16, 1)
    B.k_store_q8(whole, k, v)
    want = B.k_load_q8(whole, 3, dtype=torch.float32)
    for a, b in zip(got, want):
        assert torch.equal(a[1, 14:], b[1, :2])
        a[1, 14:] = 0
        assert not bool(a.any())


def test_arguments():
    cache = B.new_cache_q8(2, 16, 2)
    k = torch.zeros((2, 3, 128), device="cuda")
    for bad in (k[:1], k[..., :64].contiguous(), k.half(), k[0]):
        with pytest.raises(AssertionError):
            B.k_store_q8(cache, bad, bad)
    with pytest.raises(AssertionError):
        B.k_store_q8(cache, k, k, start=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(AssertionError):
        B.k_store_q8(cache, k.transpose(0, 1).contiguous().transpose(0, 1), k)
    with pytest.raises(B.OvggtError):
        B.k_load_q8(cache, 17)
    with pytest.raises(AssertionError):
        B.k_load_q8(cache, 4, dtype=torch.float16)
    x = torch.zeros((2, 64), device="cuda")
    for kw in (dict(weight=torch.zeros(64, device="cuda").bfloat16()), dict(residual=x[:1]), dict(q=x), dict(scale=torch.zeros(3, device="cuda"))):
        with pytest.raises(AssertionError):
            B.k_norm_q8(x, **kw)
    with pytest.raises(B.OvggtError):
        B.k_norm_q8(x, sum_out=torch.empty_like(x))
    with pytest.raises(B.OvggtError):
        B.k_norm_q8(torch.zeros((2, 24), device="cuda"))
