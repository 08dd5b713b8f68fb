"""any4_attn_chunk with more requests than its first launch has places for, without a GPU: refused before anything touches the device."""
import pytest

from test_attention_host import lib  # noqa: F401
from test_rows_host import SHAPE, WORKSPACE, A, chunk

MOST = 1 << 29


@pytest.mark.parametrize("requests", (MOST + 1, 715827883, 1 << 30, (1 << 31) - 2048))
def test_more_requests_than_the_plan_has_places_for(lib, requests):  # noqa: F811
    """four words a request in 32-bit places; few rows, so that no other limit is met"""
    assert chunk(lib, n=requests) == chunk(lib, n=requests, ws=A, size=1 << 40) == SHAPE
    assert lib.any4_attn_chunk_workspace_bytes(requests, 5, 4, 2, 128, 64) == 0


def test_as_many_as_there_are_places_for(lib):  # noqa: F811
    assert 4 * MOST * 4 < lib.any4_attn_chunk_workspace_bytes(MOST, 5, 4, 2, 128, 64)
    assert chunk(lib, n=MOST) == WORKSPACE
