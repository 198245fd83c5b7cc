"""Sizes of the attention whose products pass 64 bits: refused on the host (stand-in
device pointers are never dereferenced)."""
import pytest

pytest.importorskip("torch")

from paper_2609_02652_amd import _lib  # noqa: E402
from test_host_kv import FAKE, SHAPE, attend_args, cache, refused  # noqa: E402


@pytest.mark.parametrize("T,q_heads", [(1 << 60, 16), (1 << 62, 4), ((1 << 63) - 1, 2),
                                       ((1 << 31) // 4, 4)])
def test_more_rows_of_queries_than_32_bits_count(T, q_heads):
    """T · q_heads is 2^64 (0 in 64 bits), or more than 2^31 - 1."""
    refused(SHAPE, _lib.attend_workspace, cache(heads=2), attend_args(T=T, q_heads=q_heads))


@pytest.mark.parametrize("B,heads,group,split", [(1, 8, 1, True), (256, 8, 1, True),
                                                 (512, 8, 1, False), (1000, 8, 1, False),
                                                 (1000, 2, 1, True), (4096, 1, 1, False),
                                                 (1000, 8, 4, False)])
@pytest.mark.parametrize("starts", [None, FAKE])
def test_single_tokens_that_fill_the_card_are_not_split(B, heads, group, split, starts):
    """A sequence's one token is a tile of its own: what needs no split needs no
    workspace, whatever a tile could hold."""
    args = attend_args(T=B, B=B, q_heads=heads * group, q_start=starts, max_new=1, table_pages=4096)
    assert (_lib.attend_workspace(cache(heads=heads), args) > 0) == split
