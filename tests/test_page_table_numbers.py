"""Counts of tokens that a cache's offsets take, and those that they refuse, on the host."""
import numpy as np
import pytest

from paper_2607_01701_amd.page_table import PageTable


@pytest.mark.parametrize("tokens,cu", [
    ({2: 5, 0: 3}, [0, 3, 3, 8]), ([1, 2], [0, 1, 3, 3]), ({}, [0, 0, 0, 0]), ([], [0, 0, 0, 0]), (np.array([1, 0, 7]), [0, 1, 1, 8]),
    ({np.int64(1): np.int32(4)}, [0, 0, 4, 4]), (np.array([True, False, True]), [0, 1, 1, 2]), ([2.0, 0, 1], [0, 2, 2, 3]),
    ({0: 2 ** 31 - 1}, [0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1]),
])
def test_offsets(tokens, cu):
    got = PageTable(4, 16, 3, 4).offsets(tokens)
    assert got.dtype == np.int32 and got.tolist() == cu


@pytest.mark.parametrize("tokens", [{0: 1.5}, [1, 0.25, 1], {0.5: 1}, {0: float("nan")}, {0: float("inf")}, {0: -0.5}, {3: 1}, {-1: 1}, {0: -1}, [1, 1, 1, 1],
                                    {0: 2 ** 31}, {0: 2 ** 63}, {0: 2 ** 31 - 1, 1: 1}])
def test_offsets_of_no_number_of_tokens(tokens):
    with pytest.raises(ValueError, match="tokens"):
        PageTable(4, 16, 3, 4).offsets(tokens)


def test_a_fraction_of_a_token_is_not_dropped():
    """What a cache's own call does with it, without its GPU tensors."""
    from paper_2607_01701_amd import PagedCache
    cache = PagedCache.__new__(PagedCache)
    cache.host, cache._host, cache._to_device = PageTable(4, 16, 3, 4), lambda: cache.host, lambda x: x
    assert cache.offsets([1, 2]).tolist() == [0, 1, 3, 3]
    with pytest.raises(ValueError, match="tokens"):
        cache.offsets({0: 1.5})
