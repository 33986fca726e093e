"""Attention over an 8-bit cache against fp64: lengths, masks, shared heads, tiles that end anywhere, values that are not finite."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B

pytestmark = pytest.mark.gpu


def _g(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _case(seqs, M, heads, kv, capacity, seed=0, spread=1.0):
    g = _g(seed + seqs + M + heads + capacity)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    cache = B.new_cache_q8(seqs, capacity, kv)
    k, v = rnd(seqs, capacity, kv * 64), rnd(seqs, capacity, kv * 64)
    k *= spread * torch.exp2(torch.randint(-3, 2, (seqs, capacity, 1), generator=g, device="cuda").float())
    v *= torch.exp2(torch.randint(-6, 7, (seqs, capacity, 1), generator=g, device="cuda").float())
    B.k_store_q8(cache, k, v)
    return (rnd(seqs, M, heads * 64) * 1.5).bfloat16(), cache


def _reference(q, cache, lens, live):
    """(out, how far the kernel's may be off) in fp64, by what the cache stands for."""
    seqs, M, _ = q.shape
    capacity, kv = cache[0].shape[1], cache[0].shape[2] // 64
    H = q.shape[2] // 64
    k, v = (x.double().view(seqs, capacity, kv, 64) for x in B.k_load_q8(cache, capacity, dtype=torch.float32))
    out = torch.zeros((seqs, M, H, 64), dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    for s in range(seqs):
        keep = torch.arange(capacity, device="cuda") < (capacity if lens is None else int(lens[s]))
        if live is not None:
            keep &= live[s] != 0
        if not bool(keep.any()):
            continue
        for h in range(H):
            qh, kh, vh = q[s].double().view(M, H, 64)[:, h], k[s][keep][:, h * kv // H], v[s][keep][:, h * kv // H]
            p = torch.softmax(qh @ kh.T / 8, -1)
            out[s, :, h] = p @ vh
            # q as whole numbers: off by half a unit, 2^-14 of the row's largest, in each of 64 places; P, as one bf16 number: 2^-8;
            # exponentials and fp32 sums: 1e-5.  All three on weights that add up to one; then the result's own rounding.
            dq = (qh.abs().amax(-1, keepdim=True) * 2.0 ** -14 * kh.abs().sum(-1).max() / 8)
            # (both the weights and their sum move by at most e^dq)
            tol[s, :, h] = (torch.expm1(2 * dq) + 2.0 ** -8 + 1e-5) * (p @ vh.abs()) + 2.0 ** -8 * out[s, :, h].abs()
    return out.view(seqs, M, -1), tol.view(seqs, M, -1)


def _check(q, cache, lens=None, live=None):
    out = B.k_attention_q8(q, cache, lens=lens, live=live)
    ref, tol = _reference(q, cache, lens, live)
    off = (out.double() - ref).abs() - tol
    assert float(off.max()) <= 0, float(off.max())
    return out


# (sequences, tokens, heads, key heads, capacity): one row to several tiles of 8, 16, 32, 128 and 256 rows; caches of one row to many tiles
SHAPES = [(1, 1, 1, 1, 16), (3, 1, 4, 4, 160), (2, 2, 8, 2, 48), (1, 8, 2, 2, 1008), (4, 3, 12, 4, 336), (2, 5, 8, 2, 112), (1, 17, 3, 3, 320),
          (2, 33, 4, 1, 208), (1, 69, 4, 4, 336), (1, 128, 2, 2, 400), (2, 129, 2, 2, 592), (1, 300, 2, 1, 976), (3, 65, 6, 2, 80), (1, 1, 16, 16, 16400),
          (1, 257, 1, 1, 4112), (5, 1, 8, 1, 2064)]
# the same by way of bf16 planes: one tile of 128 rows and many, a ragged last one, shared heads, several sequences at once
PLANES = [(1, 1041, 2, 2, 2720), (3, 700, 2, 1, 1504), (1, 1374, 5, 5, 1376), (20, 300, 8, 2, 400), (2, 333, 3, 1, 4112), (2, 130, 16, 16, 5008)]


def _by_planes(seqs, M, heads, kv, capacity):
    """Whether a call of these sizes widens the cache into planes (the rule beside the kernels; their bytes are then part of its scratch memory)."""
    rows, x = M * heads // kv, seqs * kv * capacity
    rule = 5e6 + 45 * x * -(-rows // 32) > 11e6 + x * (118 + 25 * ((rows - 1) // 128))
    scratch = B.lib().ovggt_k_attention_q8_scratch_bytes(seqs, M, heads, kv, capacity)
    assert not rule or scratch >= min(seqs, 8) * capacity * kv * 64 * 4
    return rule


def test_which_sizes_go_by_planes():
    assert all(_by_planes(*s) for s in PLANES) and not any(_by_planes(*s) for s in SHAPES)
    assert all(_by_planes(1, M, 1, 1, n) for M, n in ROWS_BY_PLANES)


# (tokens, capacity) of a single head and more
ROWS_BY_PLANES = [(2300, 2608)]


@pytest.mark.parametrize("seqs,M,heads,kv,capacity", SHAPES + PLANES)
def test_whole_caches(seqs, M, heads, kv, capacity):
    _check(*_case(seqs, M, heads, kv, capacity))


@pytest.mark.parametrize("seqs,M,heads,kv,capacity", SHAPES + PLANES)
def test_lengths_and_masks(seqs, M, heads, kv, capacity):
    q, cache = _case(seqs, M, heads, kv, capacity, seed=7)
    g = _g(capacity)
    lens = torch.randint(0, capacity + 1, (seqs,), generator=g, device="cuda", dtype=torch.int32)
    live = (torch.rand((seqs, capacity), generator=g, device="cuda") < 0.6).to(torch.uint8) * 3
    _check(q, cache, lens)
    _check(q, cache, None, live)
    _check(q, cache, lens, live)


@pytest.mark.parametrize("seqs,M,heads,kv,capacity", [(300, 1, 2, 2, 96), (40, 1, 4, 4, 1536), (10, 1, 8, 8, 4096), (3, 1, 8, 8, 2048), (160, 3, 4, 2, 256), (300, 12, 1, 1, 96),
                                                      (60, 12, 4, 4, 800), (5, 16, 16, 16, 2048), (2, 12, 4, 4, 2048), (300, 30, 1, 1, 96), (90, 20, 4, 4, 512), (7, 25, 16, 16, 1024)])
def test_more_heads_than_multiprocessors(seqs, M, heads, kv, capacity):
    """... and a half, and a third of them: an SM's warps in one CTA or in several, the cached rows in one part or in many."""
    q, cache = _case(seqs, M, heads, kv, capacity, seed=3)
    g = _g(seqs)
    lens = torch.randint(0, capacity + 1, (seqs,), generator=g, device="cuda", dtype=torch.int32)
    live = (torch.rand((seqs, capacity), generator=g, device="cuda") < 0.8).to(torch.uint8)
    _check(q, cache, lens)
    _check(q, cache, lens, live)


@pytest.mark.parametrize("M", [1, 2, 40, 200, 700])
def test_every_short_length(M):
    """Lengths 0 to 67 and around 192 at once: tiles that end anywhere, and none at all."""
    n = torch.cat([torch.arange(0, 68), torch.arange(189, 197)]).to(torch.int32).cuda()
    assert _by_planes(len(n), M, 2, 1, 208) == (M >= 200)
    q, cache = _case(len(n), M, 2, 1, 208)
    out = _check(q, cache, n)
    assert not bool(out[0].any())


@pytest.mark.parametrize("M,capacity", [(1, 48), (12, 48), (150, 48)] + ROWS_BY_PLANES)
def test_lengths_outside_the_cache(M, capacity):
    q, cache = _case(3, M, 2, 2, capacity)
    lens = torch.tensor([-5, capacity + 1, 0x7FFFFFFF], dtype=torch.int32, device="cuda")
    out = B.k_attention_q8(q, cache, lens=lens)
    assert not bool(out[0].any()) and torch.equal(out[1:], B.k_attention_q8(q, cache)[1:])


@pytest.mark.parametrize("M,capacity", [(1, 416), (16, 416), (30, 416), (260, 416)] + ROWS_BY_PLANES)
def test_one_live_row(M, capacity):
    """A single row, wherever it lies, is the result."""
    q, cache = _case(6, M, 2, 1, capacity)
    live = torch.zeros((6, capacity), dtype=torch.uint8, device="cuda")
    at = [0, 31, 32, 191, 192, capacity - 1]
    for s, j in enumerate(at):
        live[s, j] = 255
    out = _check(q, cache, None, live)
    v = B.k_load_q8(cache, capacity)[1]
    for s, j in enumerate(at):
        torch.testing.assert_close(out[s].view(M, 2, 64).double(), v[s, j].double().expand(M, 2, 64), rtol=2.0 ** -7, atol=0)


@pytest.mark.parametrize("M,capacity", [(1, 800), (24, 800), (140, 800)] + ROWS_BY_PLANES)
def test_peaked_scores_and_late_maxima(M, capacity):
    """Scores in the hundreds, their largest in the last rows: every tile moves the reference."""
    q, cache = _case(2, M, 2, 2, capacity, spread=12.0)
    k, v = B.k_load_q8(cache, capacity, dtype=torch.float32)
    ramp = torch.linspace(0.02, 1, capacity, device="cuda")[:, None]
    B.k_store_q8(cache, k * ramp, v)
    _check(q, cache)


@pytest.mark.parametrize("M", [1, 8, 24, 140, 3000])
def test_weights_that_grow_from_tile_to_tile(M):
    """Each tile of 32 rows outweighs those before it, by its scores, by its values or by both: the references move in every one."""
    g = _g(M)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    q = torch.ones((1, M, 64), device="cuda").bfloat16()
    n = 32 * 40
    tile = torch.arange(n, device="cuda")[None, :, None] // 32
    for up_k, up_v in ((12.0, 0), (0.0, 9), (7.0, 2), (20.0, -3)):
        cache = B.new_cache_q8(1, n, 1)
        k = rnd(1, n, 64) * 0.1 + up_k / 8 * (tile - 20)
        B.k_store_q8(cache, k, rnd(1, n, 64) * torch.exp2(up_v * 0.3 * (tile - 20)))
        _check(q, cache)


@pytest.mark.parametrize("M,capacity", [(1, 416), (8, 1008), (20, 416)] + ROWS_BY_PLANES)
def test_one_row_of_large_values(M, capacity):
    """One row's values are 2^14 times the others', in half the columns: the other half holds its zeros, and there the others are the result."""
    q, cache = _case(1, M, 1, 1, capacity)
    k, v = B.k_load_q8(cache, capacity, dtype=torch.float32)
    v = v.sign() * (1 + v.abs() % 1)
    v[0, capacity // 3] *= 2.0 ** 14
    v[0, capacity // 3, 1::2] = 0
    B.k_store_q8(cache, k, v)
    _check(q, cache)


@pytest.mark.parametrize("M,capacity", [(1, 224), (20, 224), (150, 224)] + ROWS_BY_PLANES)
def test_what_lies_in_masked_places(M, capacity):
    """NaN blocks and bytes that no store wrote, beyond the length and under the mask, change nothing."""
    q, cache = _case(2, M, 4, 2, capacity)
    lens = torch.tensor([capacity - 74, capacity], dtype=torch.int32, device="cuda")
    live = torch.ones((2, capacity), dtype=torch.uint8, device="cuda")
    live[1, 33:90] = 0
    want = B.k_attention_q8(q, cache, lens=lens, live=live)
    for c, fill in zip(cache, (-128, 255, -128, 255)):
        rows = c if c.dtype == torch.int8 else c.transpose(1, 2)
        rows[0, capacity - 74:] = fill
        rows[1, 33:90] = fill
    assert torch.equal(B.k_attention_q8(q, cache, lens=lens, live=live), want)


@pytest.mark.parametrize("M,capacity", [(1, 96), (9, 96), (21, 96), (150, 96)] + ROWS_BY_PLANES)
@pytest.mark.parametrize("side", [1, 3])
def test_a_live_block_that_is_not_finite(M, capacity, side):
    """... is NaN for the heads that read it, and for them alone."""
    q, cache = _case(2, M, 4, 2, capacity)
    want = B.k_attention_q8(q, cache)
    cache[side - 1][1, 40, 64:] = 0
    cache[side][1, 1, 40] = 255
    out = B.k_attention_q8(q, cache).view(2, M, 4, 64)
    want = want.view(2, M, 4, 64)
    assert bool(out[1, :, 2:].isnan().all())
    assert torch.equal(out[0], want[0]) and torch.equal(out[1, :, :2], want[1, :, :2])


@pytest.mark.parametrize("M,capacity", [(3, 96), (9, 96), (21, 96), (150, 96)] + ROWS_BY_PLANES)
def test_queries_that_are_not_finite(M, capacity):
    q, cache = _case(1, M, 2, 2, capacity)
    want = B.k_attention_q8(q, cache)
    q[0, 1, 3], q[0, 2, 64] = float("nan"), float("inf")
    out = B.k_attention_q8(q, cache)
    bad = torch.zeros_like(q, dtype=torch.bool)
    bad[0, 1, :64] = bad[0, 2, 64:] = True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], want[~bad])
    assert not bool(B.k_attention_q8(q, cache, lens=torch.zeros(1, dtype=torch.int32, device="cuda")).any())


@pytest.mark.parametrize("M,capacity", [(1, 64), (20, 64), (150, 64)] + ROWS_BY_PLANES)
def test_small_and_large_exponents(M, capacity):
    """Keys and values far from one: the powers of two meet without leaving fp32's range on the way."""
    g = _g(M)
    q = torch.randn((1, M, 64), generator=g, device="cuda")
    for up in (100, -100):
        cache = B.new_cache_q8(1, capacity, 1)
        k, v = torch.randn((1, capacity, 64), generator=g, device="cuda"), torch.randn((1, capacity, 64), generator=g, device="cuda")
        B.k_store_q8(cache, k * 2.0 ** up, v * 2.0 ** up)
        _check((q * 2.0 ** -up).bfloat16(), cache)


@pytest.mark.parametrize("M,live_rows", [(1, 3), (40, 40), (200, 64)])
def test_offsets_past_32_bits(M, live_rows):
    """A cache of more than 2^32 bytes a side: rows at its end."""
    capacity, heads = 2 ** 22 + 4096, 16
    cache = B.new_cache_q8(1, capacity, heads)
    g = _g(M)
    k, v = (torch.randn((1, live_rows, heads * 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    B.k_store_q8(cache, k, v, start=torch.tensor([capacity - live_rows], dtype=torch.int32, device="cuda"))
    back = B.k_load_q8(cache, live_rows, first=capacity - live_rows)
    small = B.new_cache_q8(1, live_rows, heads)
    B.k_store_q8(small, k, v)
    assert all(torch.equal(a, b) for a, b in zip(back, B.k_load_q8(small, live_rows)))
    live = torch.zeros((1, capacity), dtype=torch.uint8, device="cuda")
    live[0, capacity - live_rows:] = 1
    q = torch.randn((1, M, heads * 64), generator=g, device="cuda").bfloat16()
    out = B.k_attention_q8(q, cache, live=live)
    ref, tol = _reference(q, small, torch.tensor([live_rows], dtype=torch.int32), None)
    assert bool(((out.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("M,capacity", [(1, 608), (12, 608), (150, 608)] + ROWS_BY_PLANES)
def test_same_bits_again_and_beside_another_call(M, capacity):
    q, cache = _case(3, M, 4, 2, capacity)
    want = B.k_attention_q8(q, cache)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    outs, st = [], torch.zeros(16, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for i in range(6):
        o = torch.empty_like(q)
        B.k_attention_q8(q, cache, out=o, status=st, stream=other if i % 2 else None)
        outs.append(o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs) and int(st[0]) == 0


def test_arguments():
    q, cache = _case(2, 3, 4, 2, 32)
    for over in (dict(q=q.float()), dict(q=q[:1]), dict(q=q[..., :32].contiguous()), dict(lens=torch.zeros(2, dtype=torch.int64, device="cuda")),
                 dict(lens=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(live=torch.zeros((2, 16), dtype=torch.uint8, device="cuda")),
                 dict(live=torch.ones((2, 32), dtype=torch.bool, device="cuda")), dict(out=torch.empty_like(q).float()),
                 dict(cache=(cache[0], cache[1][:, :, :16].contiguous(), *cache[2:])), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(AssertionError):
            B.k_attention_q8(**dict(dict(q=q, cache=cache), **over))
    with pytest.raises(B.OvggtError):
        B.k_attention_q8(q[..., :192].contiguous(), cache)
