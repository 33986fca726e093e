"""The int8 product: its sums are exact, so its bits are those of the formula in fp32, at every size and split."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B

pytestmark = pytest.mark.gpu

# rows, columns, K: one token to frames, partial tiles on each side, K that ends inside a tile
SHAPES = [(1, 8, 16), (1, 4096, 1024), (2, 24, 48), (5, 1024, 4096), (7, 72, 80), (8, 264, 528), (9, 136, 64), (16, 768, 1040), (17, 48, 112), (33, 512, 2048),
          (64, 1024, 1024), (65, 128, 256), (127, 72, 64), (128, 256, 128), (129, 264, 192), (333, 512, 2064), (718, 2304, 768), (1041, 1024, 4096),
          (1374, 4096, 1024), (2049, 40, 16), (4500, 1032, 272), (20000, 520, 144), (30001, 72, 48)]


def _case(M, N, K, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(M + N + K + seed)
    a = torch.randint(-127, 128, (M, K), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda").to(torch.int8)
    as_, ws = (torch.rand(n, generator=g, device="cuda") * 0.02 / K ** 0.5 for n in (M, N))
    x = torch.randn((M, N), generator=g, device="cuda").bfloat16()
    return a, as_, w, ws, x, torch.zeros(16, dtype=torch.int32, device="cuda")


def _t(a, as_, w, ws):
    # (products of whole numbers: exact in 64 bits; rounded to fp32, scaled by the token's and then the channel's, to bf16)
    return ((a.double() @ w.double().T).float() * as_[:, None] * ws).bfloat16()


def _check_gelu(t, x):
    """t against GELU of bf16 x in fp64: 1e-5 of the value from the polynomial and its fp32 evaluation, the result's own rounding (2^-8, down to
    bf16's smallest step), and 1e-17 where it is cut off, below -9."""
    ref = 0.5 * x.double() * torch.special.erfc(-x.double() / 2 ** 0.5)        # (not by ndtr, which cancels in the tail)
    assert bool(((t.double() - ref).abs() <= (2.0 ** -8 + 1e-5) * ref.abs() + 2.0 ** -134 + 1e-17 * (x < -9)).all())


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(M, N, K):
    a, as_, w, ws, x, st = _case(M, N, K)
    ws = ws * 400                                        # (products of about one: GELU's middle)
    ref = _t(a, as_, w, ws)
    t, s = torch.empty_like(x), torch.empty_like(x)
    B.k_linear_q8(a, as_, w, ws, (t,), residual=x, sum_out=s, status=st)
    assert torch.equal(t, ref) and torch.equal(s, x + ref)
    s.zero_()
    B.k_linear_q8(a, as_, w, ws, (), residual=x, sum_out=s, status=st)
    assert torch.equal(s, x + ref)
    B.k_linear_q8(a, as_, w, ws, (), residual=x, sum_out=x, status=st)
    assert torch.equal(s, x)                             # (the residual stream in place)
    B.k_linear_q8(a, as_, w, ws, (t,), gelu=True, status=st)
    _check_gelu(t, ref)
    for n in (2, 3):
        if N % (8 * n) == 0:
            parts = [torch.empty((M, N // n), dtype=torch.bfloat16, device="cuda") for _ in range(n)]
            B.k_linear_q8(a, as_, w, ws, parts, status=st)
            assert torch.equal(torch.cat(parts, 1), ref)
    assert int(st[0]) == 0


@pytest.mark.parametrize("tiles", [False, True])
def test_gelu_over_its_range(tiles):
    """Every bf16 value there is, as the scale of a product with one: few tokens and many."""
    v = torch.arange(-2 ** 15, 2 ** 15, device="cuda").to(torch.int16).view(torch.bfloat16)
    v = v[:, None] if not tiles else torch.cat([v, v[:40]])[:, None]
    for lo in range(0, len(v), 2 ** 14):
        x = v[lo:lo + 2 ** 14].contiguous() if tiles else v[lo:lo + 2 ** 14]
        scale = x.float().view(-1)
        one = torch.zeros((8, 16), dtype=torch.int8, device="cuda")
        one[:, 0] = 1
        st = torch.zeros(16, dtype=torch.int32, device="cuda")
        step = len(scale) if tiles else 32
        out = torch.empty((len(scale), 8), dtype=torch.bfloat16, device="cuda")
        for i in range(0, len(scale), step):
            n = min(step, len(scale) - i)
            B.k_linear_q8(one[:1].expand(n, 16).contiguous(), scale[i:i + n].contiguous(), one, torch.ones(8, device="cuda"), (out[i:i + n],), gelu=True, status=st)
        x = x.view(-1, 1).expand(-1, 8)
        fine = x.isfinite()
        _check_gelu(out[fine], x[fine])
        assert bool(out[x.isnan()].isnan().all()) and bool((out[x == float("inf")] == float("inf")).all()) and bool((out[x == -float("inf")].abs() <= 1e-17).all())


@pytest.mark.parametrize("M", [1, 40, 700])
def test_largest_sums(M):
    """The longest K: every product -128 x -128, and the sum stays within int32."""
    K = 131056
    a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((8, K), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(M, device="cuda")
    t = torch.empty((M, 8), dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(16, dtype=torch.int32, device="cuda")
    B.k_linear_q8(a, one, w, torch.ones(8, device="cuda"), (t,), status=st)
    assert torch.equal(t, torch.full_like(t, float(16384 * K)))


@pytest.mark.parametrize("M", [3, 300])
def test_scales_that_are_not_finite(M):
    a, as_, w, ws, x, st = _case(M, 64, 64)
    as_[1], ws[5] = float("nan"), float("inf")
    t = torch.empty((M, 64), dtype=torch.bfloat16, device="cuda")
    B.k_linear_q8(a, as_, w, ws, (t,), status=st)
    ref = _t(a, as_, w, ws)
    assert torch.equal(t.isnan(), ref.isnan()) and torch.equal(t.nan_to_num(), ref.nan_to_num())
    assert bool(t[1].isnan().all()) and not bool(t[0, :5].isnan().any())


@pytest.mark.parametrize("M", [5, 300])
def test_rows_behind_the_last_are_left_alone(M):
    a, as_, w, ws, _, st = _case(M, 72, 80)
    whole = torch.full((M + 200, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    B.k_linear_q8(a, as_, w, ws, (whole[:M],), status=st)
    assert torch.equal(whole[:M], _t(a, as_, w, ws)) and bool((whole[M:] == 7).all())


@pytest.mark.parametrize("M,N,parts,gelu", [(4499, 1032, 1, True), (2049, 2400, 3, False), (1375, 4096, 2, True), (20001, 264, 1, False)])
def test_wide_tiles_write_their_rows_and_columns_alone(M, N, parts, gelu):
    """Results that leave by bulk copies: nothing behind the last row of any of them, nothing of one in another."""
    a, as_, w, ws, _, st = _case(M, N, 144)
    whole = [torch.full((M + 130, N // parts), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(parts)]
    B.k_linear_q8(a, as_, w, ws, [o[:M] for o in whole], gelu=gelu, status=st)
    got, ref = torch.cat([o[:M] for o in whole], 1), _t(a, as_, w, ws)
    if gelu:
        _check_gelu(got, ref)
    else:
        assert torch.equal(got, ref)
    assert all(bool((o[M:] == 7).all()) for o in whole) and int(st[0]) == 0


def test_arguments():
    a, as_, w, ws, x, st = _case(16, 32, 64)
    t = torch.empty_like(x)
    ok = dict(a=a, a_scale=as_, w=w, w_scale=ws, outs=(t,), residual=x, sum_out=torch.empty_like(x), status=st)
    B.k_linear_q8(**ok)
    for over in (dict(a=a.float()), dict(w=w.float()), dict(a=a[:, :48].contiguous()), dict(a_scale=as_[:8]), dict(w_scale=ws.double()),
                 dict(outs=(t.float(),)), dict(outs=(t[:8],)), dict(residual=x[:8]), dict(sum_out=x.float()), dict(outs=(t,) * 4),
                 dict(w=w.T.contiguous().T)):
        with pytest.raises(AssertionError):
            B.k_linear_q8(**dict(ok, **over))
    with pytest.raises(B.OvggtError):
        B.k_linear_q8(**dict(ok, residual=None))


# (a product by tiles has more blocks of 16 channels and 32 tokens than can run at once)
@pytest.mark.parametrize("M,N,K", [(9601, 8, 16), (4800, 40, 80), (1700, 72, 528), (700, 264, 2064), (250, 1032, 1040), (40, 4104, 272), (17, 5000, 1040),
                                   (256, 592, 144), (257, 592, 144)])
def test_few_columns_by_tiles(M, N, K):
    test_linear(M, N, K)


@pytest.mark.parametrize("K", [16, 496, 528, 1536, 1552, 2032, 2064, 4112, 6160])
@pytest.mark.parametrize("M,N", [(1, 4736), (8, 4744), (16, 4736), (13, 4744), (31, 24), (200, 72)])
def test_lengths_of_few_tokens(M, N, K):
    """K that ends in each of a warp's steps, in CTAs that run all at once and in several waves."""
    a, as_, w, ws, x, st = _case(M, N, K)
    t, s = torch.empty_like(x), torch.empty_like(x)
    B.k_linear_q8(a, as_, w, ws, (t,), residual=x, sum_out=s, status=st)
    ref = _t(a, as_, w, ws)
    assert torch.equal(t, ref) and torch.equal(s, x + ref)


def test_largest_sums_by_tiles():
    M, N, K = 3200, 56, 131056
    a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    t = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(16, dtype=torch.int32, device="cuda")
    B.k_linear_q8(a, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), (t,), status=st)
    assert torch.equal(t, torch.full_like(t, float(16384 * K))) and int(st[0]) == 0


def test_scales_that_are_not_finite_by_tiles():
    test_scales_that_are_not_finite(3000)


def test_rows_behind_the_last_are_left_alone_by_tiles():
    test_rows_behind_the_last_are_left_alone(2400)
