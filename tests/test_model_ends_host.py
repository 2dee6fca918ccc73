"""CPU-only checks of the C entries of the token model's two ends: workspaces they report, and arguments they refuse before touching a device."""

import pytest

from paper_2110_01595_b200 import binding, build

BAD = binding.ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


def test_embedding_refusals(lib):
    at = 4096                                   # an aligned address that no refused call reads
    f = lib.solon_embedding_forward
    assert f(at, 8, 1, at, 4, 8, 10, 1.0, at, 8, None) == BAD                      # no float64 here
    assert f(at, 7, 0, at, 4, 8, 10, 1.0, at, 8, None) == BAD                      # pitch
    assert f(at, 8, 0, at, 4, 8, 10, 1.0, at, 7, None) == BAD
    assert f(None, 8, 0, at, 4, 8, 10, 1.0, at, 8, None) == BAD
    assert f(at + 2, 8, 0, at, 4, 8, 10, 1.0, at, 8, None) == BAD                  # alignment
    assert f(at, 8, 0, at + 4, 4, 8, 10, 1.0, at, 8, None) == BAD
    assert f(at, 8, 0, None, 4, 8, 10, 1.0, at, 8, None) == BAD
    assert f(at, 8, 0, at, -1, 8, 10, 1.0, at, 8, None) == BAD
    assert f(at, 8, 0, at, 4, 8, 0, 1.0, at, 8, None) == BAD
    assert f(at, 1 << 23, 0, at, 4, 1 << 23, 10, 1.0, at, 1 << 23, None) == BAD
    assert f(None, 8, 0, None, 0, 8, 10, 1.0, None, 8, None) == 0                  # no rows: nothing to do
    w = lib.solon_embedding_backward_workspace
    assert w(0, 8, 3) >= 0 and w(4096, 1000, 4) >= 4096 * 16
    assert w(10, 8, 3) == BAD and w(10, 8, 0) == BAD and w(-1, 8, 1) == BAD and w(10, 0, 1) == BAD and w(2050, 4, 1025) == BAD
    assert w(1 << 31, 8, 1) == BAD
    b = lib.solon_embedding_backward
    big = 1 << 30
    assert b(at, 8, 1, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at, big, None) == BAD       # type of dy
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 3, 0, at, big, None) == BAD       # type of the gradient
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 79, 0, 0, at, big, None) == BAD       # its pitch
    assert b(at, 8, 0, at, 4, 8, 10, 3, 1.0, at, 80, 0, 0, at, big, None) == BAD       # partitions that do not divide the rows
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, None, big, None) == BAD     # no workspace
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at + 8, big, None) == BAD   # off its alignment
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at, w(4, 8, 2) - 1, None) == BAD
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, None, 80, 0, 0, at, big, None) == BAD
    assert b(None, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at, big, None) == BAD
    assert b(at, 8, 0, at, 4, 8, 1 << 45, 2, 1.0, at, 1 << 48, 0, 0, at, big, None) == BAD
