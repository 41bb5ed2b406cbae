"""How fbsr_attend_kv cuts tables where the GPU holds all sequences, heads and tiles of rows once and not twice, as the workspace that it asks for
shows (runs without a GPU): two chunks up to a number of them that grows with the table, the line on which both choices cross."""
import pytest

from test_answer_refusals import b, desc    # noqa: F401 (b: a fixture)

ROW = 4 * 128 + 8                                # bytes of a row's sums in the workspace: dim numbers, maximum and sum


def chunks(b, batch, queries, tokens):
    """32 heads on 8, pages of 64: two tiles of 128 rows for more than 32 queries."""
    total = batch * queries
    need = b._L.fbsr_attend_workspace_bytes(desc(b, heads=8, page=64), batch, total, 32, queries, tokens // 64)
    assert need % (total * 32 * ROW) == 0
    return max(1, need // (total * 32 * ROW))


@pytest.mark.parametrize("tokens,two,one", [(1024, 4, 5), (2048, 5, 6), (4096, 6, 7), (8192, 7, 8), (16384, 8, 9)])
def test_two_chunks_up_to_where_one_takes_no_longer(b, tokens, two, one):
    for queries in (63, 40):
        assert chunks(b, two, queries, tokens) == 2 and chunks(b, one, queries, tokens) == 1
    for batch in range(10, 40):
        assert chunks(b, batch, 63, tokens) == 1


def test_fewer_than_half_the_places_take_what_fills_them(b):
    assert [chunks(b, batch, 63, 16384) for batch in (2, 3, 4)] == [4, 3, 2]
