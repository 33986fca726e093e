"""Attention over an 8-bit cache, path by path: which one a call takes, by its launches; each at the precision that it promises; groups of
sequences that share their scratch memory; parts that hold nothing beside parts that are not numbers."""
import pytest
import torch

from paper_2603_05959_b200 import binding as B
from test_gpu_q8_attention import PLANES, ROWS_BY_PLANES, SHAPES, _case, _g
from test_gpu_q8_limits import PATHS, _check

pytestmark = pytest.mark.gpu


def _lens_and_mask(seqs, capacity, share=0.7):
    g = _g(seqs + capacity)
    return (torch.randint(0, capacity + 1, (seqs,), generator=g, device="cuda", dtype=torch.int32),
            (torch.rand((seqs, capacity), generator=g, device="cuda") < share).to(torch.uint8))


def _launches(q, cache, **kw):
    st = torch.zeros(16, dtype=torch.int32, device="cuda")
    before = B.kernel_launches()
    B.k_attention_q8(q, cache, status=st, **kw)
    return B.kernel_launches() - before


@pytest.mark.parametrize("seqs,M,heads,kv,capacity", SHAPES + PLANES + [(1, M, 1, 1, n) for M, n in ROWS_BY_PLANES])
def test_which_kernels_run(seqs, M, heads, kv, capacity):
    """By planes a mask takes a launch of its own; streaming, attention and perhaps a merge are all there is."""
    q, cache = _case(seqs, M, heads, kv, capacity)
    plain, masked = _launches(q, cache), _launches(q, cache, live=torch.ones((seqs, capacity), dtype=torch.uint8, device="cuda"))
    if (seqs, M, heads, kv, capacity) in SHAPES:
        assert plain == masked <= 2
    else:
        assert masked == plain + 1 and plain in (2, 3)


@pytest.mark.parametrize("seqs,M,heads,kv,capacity", SHAPES + PLANES)
def test_precision_of_each_path(seqs, M, heads, kv, capacity):
    q, cache = _case(seqs, M, heads, kv, capacity, seed=11)
    lens, live = _lens_and_mask(seqs, capacity)
    _check(q, cache)
    _check(q, cache, lens, live)


def test_groups_of_sequences():
    """More planes than are kept at once: two sequences, then one, in the same scratch memory."""
    seqs, M, heads, capacity = 3, 130, 16, 16000
    q, cache = _case(seqs, M, heads, heads, capacity)
    lens, live = _lens_and_mask(seqs, capacity)
    lens[0] = capacity
    one = B.lib().ovggt_k_attention_q8_scratch_bytes(1, M, heads, heads, capacity)
    assert B.lib().ovggt_k_attention_q8_scratch_bytes(seqs, M, heads, heads, capacity) < 3 * one
    assert _launches(q, cache, lens=lens, live=live) == 8 and _launches(q, cache, lens=lens) == 6          # (with a merge each)
    _check(q, cache)
    _check(q, cache, lens, live)
    lens[1] = 0                                          # (an empty one beside a full one, and a short one by itself)
    lens[2] = 5
    out = _check(q, cache, lens, live)
    assert not bool(out[1].any())


def test_groups_of_one_sequence():
    """A sequence whose planes fill what is kept at once goes alone."""
    seqs, M, heads, capacity = 3, 100, 16, 33024
    q, cache = _case(seqs, M, heads, heads, capacity)
    lens, live = _lens_and_mask(seqs, capacity)
    assert _launches(q, cache, lens=lens, live=live) == 12
    _check(q, cache, lens, live)


@pytest.mark.parametrize("M,heads,kv", [(1, 8, 8), (8, 4, 4), (12, 4, 4), (25, 4, 4), (2300, 1, 1)])
@pytest.mark.parametrize("side", [1, 3])
def test_parts_that_are_not_numbers(M, heads, kv, side):
    """A block that is not finite makes its heads' results none however the cached rows are cut, beside parts that hold nothing, and theirs alone."""
    capacity = 8192 if M < 100 else 2608
    q, cache = _case(3, M, heads, kv, capacity)
    assert _launches(q, cache) >= 2                      # (parts, and their merge)
    live = torch.zeros((3, capacity), dtype=torch.uint8, device="cuda")
    live[:, 700:760] = 1                                 # (all but one or two parts hold nothing)
    lens = torch.tensor([capacity, capacity, 740], dtype=torch.int32, device="cuda")
    want = [B.k_attention_q8(q, cache), B.k_attention_q8(q, cache, lens=lens, live=live)]
    assert not any(bool(w.isnan().any()) for w in want)
    cache[side - 1][1, 730, :64] = 0
    cache[side][1, 0, 730] = 255
    group = heads // kv * 64
    for w, kw in zip(want, ({}, dict(lens=lens, live=live))):
        out = B.k_attention_q8(q, cache, **kw)
        assert bool(out[1, :, :group].isnan().all())
        assert torch.equal(out[::2], w[::2]) and torch.equal(out[1, :, group:], w[1, :, group:])


@pytest.mark.parametrize("M,heads,kv,n", PATHS)
def test_weights_that_grow_on_every_path(M, heads, kv, n):
    """Each tile of 32 rows outweighs those before it, by its scores, by its values or by both: the references move in every one."""
    g = _g(M + n)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    q = torch.ones((1, M, heads * 64), device="cuda").bfloat16()
    tiles = n // 32
    tile = torch.arange(n, device="cuda")[None, :, None] // 32
    for up_k, up_v in ((12.0, 0.0), (0.0, 9.0), (7.0, 2.0), (20.0, -3.0)):
        cache = B.new_cache_q8(1, n, kv)
        k = rnd(1, n, kv * 64) * 0.1 + up_k / 8 * (tile - tiles // 2)
        B.k_store_q8(cache, k, rnd(1, n, kv * 64) * torch.exp2(up_v * 12 / tiles * (tile - tiles // 2)))
        _check(q, cache)
