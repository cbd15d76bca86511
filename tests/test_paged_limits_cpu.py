"""Paged cache, host side: the largest numbers that the calls take, and what lies just behind them."""
import numpy as np
import pytest

from tests.test_paged_cpu import lib  # noqa: F401 (a fixture)


@pytest.mark.parametrize("units,most,tiles", [(768, 774, 1 << 25), (1, 2, 1 << 25), (1000, 1001, 1 << 25), (896, 897, 9586981)])
def test_pieces_of_the_longest_sequences(lib, units, most, tiles):  # noqa: F811
    """Hardly more pieces than units, each of up to 2^25 tiles (2^30 slots): a piece's size is a number of more than
    32 bits there, of which the low ones alone would be 0, or little."""
    size = lib.t_size(units, units * tiles, most, 4)
    assert size >= 4
    n = lib.t_pieces(tiles, size)
    assert 1 <= n and units * n <= most
    assert lib.t_start(tiles, n, 0) == 0 and lib.t_start(tiles, n, n) == tiles


def test_pieces_fit_where_sizes_are_large(lib):  # noqa: F811
    rng = np.random.default_rng(1)
    for _ in range(2000):
        units = int(rng.integers(1, 4000))
        most = units + int(2.0 ** rng.uniform(0, 11))
        tiles = int(2.0 ** rng.uniform(18, 25))
        size = lib.t_size(units, units * tiles, most, 4)
        assert size >= 4 and units * lib.t_pieces(tiles, size) <= most
