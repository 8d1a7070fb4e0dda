"""The paged cache's entry points: list lengths and sequence counts at their limits, refused before anything reaches the GPU.  CPU only."""
import pytest

from test_abi import E_UNSUP, lib  # noqa: F401
from test_pages_abi import calls, pool


@pytest.mark.parametrize("name", ["fork", "free"])
@pytest.mark.parametrize("n", [65536, 1 << 20, (1 << 24) - 1, (1 << 31) - 1])
def test_lists_longer_than_there_can_be_sequences(lib, name, n):  # noqa: F811
    """The work on a list grows with its square: 2^24 entries, which one launch can count, would keep the GPU for minutes."""
    assert calls(lib)[name](pool(), n=n) == E_UNSUP and b"65535" in lib.lookat_last_error()
