"""Which sizes the calls around the key/value cache take in one go, seen in the workspaces that they ask for. No kernel is launched."""
import pytest

from paper_2509_09090_b200 import binding as B
from test_lowbit_host import cache

PIECE = 2 * (64 * 4 + 8)                  # bytes of a row's piece: two heads of 64, maximum and denominator


def pieces(batch, max_q, max_len, max_group, max_prefix):
    """Pieces of a row of one group."""
    n = B.lib().sqap_kv_attention_shared_workspace_bytes(cache(), batch, max_q, max_len, 1, max_group, max_prefix, 2)
    assert n % (batch * max_q * PIECE) == 0
    return n // (batch * max_q * PIECE)


def test_own_tokens_behind_a_short_prefix_are_not_taken_together():
    """Of eight sequences, one tile of rows: max_prefix says nothing of how many own tokens a group with a shorter prefix has."""
    together = pieces(8, 1, 1 << 24, 8, 1024)
    assert pieces(8, 1, 1 << 24, 8, 1 << 24) == together
    for max_len in ((1 << 27) + 2048, 1 << 28, 1 << 30):
        for max_prefix in (1024, 1 << 27, max_len - 4096, max_len):
            assert pieces(8, 1, max_len, 8, min(max_prefix, max_len)) < together, (max_len, max_prefix)


def test_tiles_over_own_tokens_only_where_their_places_fit():
    """700 sequences behind a long prefix and 100 own tokens: tiles of rows take pieces of the own tokens, a sequence by itself joins the prefix's at once."""
    tiles, alone = pieces(700, 1, 1 << 20, 700, (1 << 20) - 100), pieces(700, 1, 1 << 28, 700, (1 << 28) - 100)
    assert alone < tiles and pieces(700, 1, 1 << 30, 700, (1 << 30) - 100) == alone


@pytest.mark.parametrize("rows", range(1, 17))
def test_all_sequences_that_a_tile_of_rows_meets_are_counted(rows):
    """Tiles of eight rows begin anywhere in a sequence of `rows` rows."""
    group = 24 // rows if rows <= 8 else 2                     # three tiles, or four
    met = max(min(8 * tile + 7, rows * group - 1) // rows - 8 * tile // rows + 1 for tile in range(-(-rows * group // 8)))
    together = pieces(group, rows, 1 << 24, group, 512)
    assert pieces(group, rows, (1 << 28) // met, group, 512) == together
    assert pieces(group, rows, (1 << 30) // met + 64, group, 512) != together         # one sequence of 2^30 + 64 tokens is refused
