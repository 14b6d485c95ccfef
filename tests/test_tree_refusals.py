"""What tree attention refuses on the host beyond bad arguments: caches whose positions,
rounded up to whole tiles, pass 32 bits."""
import pytest

from test_kv_refusals import L, SHAPE, cache, tree  # noqa: F401


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 100, 2 ** 31 - 1024])
def test_positions_near_the_end_of_32_bits(L, bits, n):
    assert tree(L, c=cache(max_len=n, bits=bits, batch=1, n_kv=1)) == SHAPE
