"""CPU checks of the 8-bit entry points at the ends of their ranges: refused before a GPU is touched."""
from test_abi_q8 import ATTEND, BAD, LINEAR, MISALIGNED, NORM, P, UNSUPPORTED, _call, lib  # noqa: F401  (the fixture builds the library)


def test_rows_that_a_grid_cannot_count(lib):  # noqa: F811
    """Sixteen rows of up to 256 columns share a CTA: the count of CTAs, rounded up, would pass 32 bits."""
    for rows in (0x7FFFFFFF, 0x7FFFFFF1, 0x7FFFFF01):
        assert _call(lib.ovggt_k_norm_q8, list(NORM), NORM, rows=rows, C=16) == UNSUPPORTED


def test_a_status_word_that_cannot_be_written(lib):  # noqa: F811
    for by in (1, 2, 3):
        assert _call(lib.ovggt_k_linear_q8, list(LINEAR), LINEAR, status=P + by) == MISALIGNED


def test_sizes_without_a_scratch_size_are_unsupported(lib):  # noqa: F811
    """... also where the caller made its scratch memory of the 0 bytes it was told."""
    for over in (dict(capacity=40), dict(M=1 << 30), dict(n_seqs=1 << 20, capacity=1 << 12)):
        sizes = [dict(ATTEND, **over)[n] for n in ("n_seqs", "M", "n_heads", "n_kv_heads", "capacity")]
        assert lib.ovggt_k_attention_q8_scratch_bytes(*sizes) == 0
        assert _call(lib.ovggt_k_attention_q8, list(ATTEND), ATTEND, scratch=None, **over) == UNSUPPORTED, over
    assert _call(lib.ovggt_k_attention_q8, list(ATTEND), ATTEND, scratch=None) == BAD
