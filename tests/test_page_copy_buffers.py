"""Buffers of page copies that overlap are refused, on the CPU; those whose pages lie apart or between each other's are not."""
import ctypes
import random

import numpy as np
import pytest

from paper_2607_01701_amd import _lib

A = 1 << 40  # an address


def copy(buffers, pages, stride, size):
    b, one = (ctypes.c_void_p * len(buffers))(*buffers), [np.array([i], dtype=np.int32) for i in (0, 1)]
    L = _lib.lib()
    st = L.t2v_page_copy(b, len(b), pages, stride, size, *(x.ctypes.data for x in one), 1, None)
    return st == _lib.T2V_ERR_INVALID_ARG and "overlap" in _lib.t2v_last_error(L)


@pytest.fixture(autouse=True)
def _no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are no memory")


def test_views_of_one_cache():
    """Pages 0 .. 59 and 40 .. 99 of one buffer, and pages that begin inside others."""
    assert copy([A, A + 40 * 4096], 60, 4096, 4096)
    assert copy([A + 40 * 4096, A], 60, 4096, 4096)
    assert copy([A, A + 1024], 10, 4096, 2048)
    assert copy([A, A + 2560], 10, 4096, 2048)  # a page's end and the next page's begin
    assert copy([A, A + 2 ** 36, A + 2 ** 36 + 16], 10, 4096, 4096)
    assert not copy([A, A + 60 * 4096], 60, 4096, 4096)
    assert not copy([A, A + 2048], 60, 4096, 2048)
    assert not copy([A, A + 59 * 4096 + 2048], 60, 4096, 2048)
    assert not copy([A, A], 60, 4096, 4096)  # the same buffer twice
    assert not copy([A, A + 4096 + 2560], 2, 4096, 2048)  # behind the last page's bytes
    assert not copy([A + 1000 * 16 * i for i in range(150)], 20, 1000 * 16 * 150, 1000 * 16)
    assert copy([A + 1000 * 16 * i for i in range(151)], 20, 1000 * 16 * 150, 1000 * 16)


def test_against_every_byte():
    r = random.Random(1)
    seen = set()
    for _ in range(3000):
        pages, size = r.randint(2, 6), 16 * r.randint(1, 4)
        stride = size + 16 * r.randint(0, 6)
        at = [16 * r.randint(0, 60) for _ in range(r.randint(1, 5))]
        bytes_ = [{a // 16 + p * stride // 16 + b for p in range(pages) for b in range(size // 16)} for a in sorted(set(at))]
        meet = sum(map(len, bytes_)) != len(set().union(*bytes_))
        assert copy([A + x for x in at], pages, stride, size) == meet, (at, pages, stride, size)
        seen.add((meet, len(bytes_)))
    assert {(m, n) for m in (False, True) for n in (2, 3)} <= seen
