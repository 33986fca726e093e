"""Attention over an 8-bit cache where its arithmetic has least room: outliers in a query, tiny and far-apart values, scores far from zero.
By 8, 16 and 32 rows of the streaming kernel and by planes."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B

pytestmark = pytest.mark.gpu

# (tokens, heads, key heads, cached rows): 1 and 8 rows of a key head, 12, 24 and by planes; one part and several
PATHS = [(1, 2, 2, 96), (2, 8, 2, 4112), (3, 4, 1, 160), (12, 1, 1, 4112), (24, 1, 1, 320), (6, 4, 1, 4112), (2300, 1, 1, 2608)]


def _g(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _check(q, cache, lens=None, live=None):
    """Against fp64 by what the cache stands for.  What may be off: a score by the fp32 sums of 64 exact products in four steps of 16, each of 17
    terms cut to 2^-22 of the largest, 2^-17 of the sum of magnitudes in all; a weight by 1e-5 (exponentials, fp32 sums), from 9 rows of a
    key head on also by its rounding to bf16, 2^-8, and up to 8 by half of 2^-28 of the largest weight times step, 127 of which a value has at most;
    the result by its own rounding."""
    out = B.k_attention_q8(q, cache, lens=lens, live=live)
    seqs, M, _ = q.shape
    capacity, kv = cache[0].shape[1], cache[0].shape[2] // 64
    H = q.shape[2] // 64
    few = M * H // kv <= 8
    k, v = (x.double().view(seqs, capacity, kv, 64) for x in B.k_load_q8(cache, capacity, dtype=torch.float32))
    worst = 0.0
    for s in range(seqs):
        keep = torch.arange(capacity, device="cuda") < (capacity if lens is None else int(lens[s]))
        if live is not None:
            keep &= live[s] != 0
        n = int(keep.sum())
        if n == 0:
            assert not bool(out[s].any())
            continue
        for h in range(H):
            qh, kh, vh = q[s, :, h * 64:h * 64 + 64].double(), k[s, :, h * kv // H][keep], v[s, :, h * kv // H][keep]
            p = torch.softmax(qh @ kh.T / 8, -1)
            ref, spread = p @ vh, p @ vh.abs()
            ds = (qh.abs() @ kh.abs().T).amax(-1, keepdim=True) / 8 * 2.0 ** -17
            tol = (torch.expm1(2 * ds) + 1e-5 + (0.0 if few else 2.0 ** -8)) * spread + 2.0 ** -8 * ref.abs() + 2.0 ** -133
            if few:
                tol += n * 2.0 ** -28 * (p * vh.abs().amax(-1)).amax(-1, keepdim=True)
            off = (out[s, :, h * 64:h * 64 + 64].double() - ref).abs()
            assert not bool(off.isnan().any())
            worst = max(worst, float((off / tol).max()))
    assert worst <= 1, worst
    return out


@pytest.mark.parametrize("M,heads,kv,n", PATHS)
@pytest.mark.parametrize("up", [0, 6, 10, 14, 20])
def test_one_large_column_of_a_query(M, heads, kv, n, up):
    """One column of every query 2^up times the others, where the keys are zero: the others decide."""
    g = _g(M + n + up)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    k = rnd(1, n, kv * 64) * 2
    k.view(1, n, kv, 64)[..., 5] = 0
    q = rnd(1, M, heads * 64)
    q.view(1, M, heads, 64)[..., 5] = 2.0 ** up * (1 + rnd(1, M, heads).abs())
    cache = B.new_cache_q8(1, n, kv)
    B.k_store_q8(cache, k, rnd(1, n, kv * 64))
    _check(q.bfloat16(), cache)


@pytest.mark.parametrize("M,heads,kv,n", PATHS)
@pytest.mark.parametrize("kind", ["level", "ranging", "hidden"])
@pytest.mark.parametrize("up", [-118, -60, 100])
def test_values_of_any_size(M, heads, kv, n, kind, up):
    """Values about 2^up: all alike; down to 2^-7 of that in turn; or behind one row of zeros that weighs 2^9 times any other's."""
    g = _g(M + n + up)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    v = rnd(1, n, kv * 64).double()
    k = rnd(1, n, kv * 64) * 0.25
    q = torch.ones((1, M, heads * 64), device="cuda") + 0.25 * rnd(1, M, heads * 64)
    if kind == "ranging":
        v *= torch.exp2(-(torch.arange(n, device="cuda") % 8).double())[None, :, None]
    if kind == "hidden":
        k[0, n // 3] = 9 * 0.6931 / 8
        v[0, n // 3] = 0
    cache = B.new_cache_q8(1, n, kv)
    B.k_store_q8(cache, k, (v * 2.0 ** up).float())
    _check(q.bfloat16(), cache)


@pytest.mark.parametrize("M,heads,kv,n", PATHS)
@pytest.mark.parametrize("size", [1e3, 1e6, 1e9, -1e3, -1e9, -1e33])
def test_scores_far_from_zero(M, heads, kv, n, size):
    """All keys alike, so that every score is the same large number: the result is the mean of the values."""
    if abs(size) > 2.0 ** 30 and M > 1000:
        return                                           # (more than what is promised; the streaming kernel does it)
    g = _g(M + n)
    cache = B.new_cache_q8(3, n, kv)
    k = torch.zeros((3, n, kv, 64), device="cuda")
    k[..., 0] = 2.0 ** 20 if abs(size) < 2.0 ** 60 else 2.0 ** 60
    v = torch.randn((3, n, kv * 64), generator=g, device="cuda")
    v *= torch.exp2(-(torch.arange(n, device="cuda") % 8).float())[None, :, None]
    B.k_store_q8(cache, k.view(3, n, -1), v)
    q = torch.zeros((3, M, heads, 64), device="cuda")
    q[..., 0] = size * 8 / float(k.max())
    lens = torch.tensor([n, 37, n // 2], dtype=torch.int32, device="cuda")
    out = B.k_attention_q8(q.view(3, M, -1).bfloat16(), cache, lens=lens).double().view(3, M, heads, 64)
    back = B.k_load_q8(cache, n, dtype=torch.float32)[1].double().view(3, n, kv, 64)
    for s in range(3):
        x = back[s, :int(lens[s])].repeat_interleave(heads // kv, 1)
        tol = 2.0 ** -8 * x.mean(0).abs() + (1e-5 + (0 if M * heads // kv <= 8 else 2.0 ** -8)) * x.abs().mean(0) + 2.0 ** -28 * n * x.abs().amax(0)
        assert bool(((out[s] - x.mean(0)).abs() <= tol).all())
