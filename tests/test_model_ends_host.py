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
    assert w(0, 8, 10, 3) >= 0 and w(4096, 1000, 10, 4) >= 4096 * 16
    assert w(10, 8, 10, 3) == BAD and w(10, 8, 10, 0) == BAD and w(-1, 8, 10, 1) == BAD and w(10, 0, 10, 1) == BAD and w(2050, 4, 10, 1025) == BAD
    assert w(1 << 31, 8, 10, 1) == BAD and w(10, 8, 0, 1) == BAD
    b = lib.solon_embedding_backward
    big = 1 << 30
    assert b(at, 8, 1, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at, big, None) == BAD       # type of dy
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 3, 0, at, big, None) == BAD       # type of the gradient
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 79, 0, 0, at, big, None) == BAD       # its pitch
    assert b(at, 8, 0, at, 4, 8, 10, 3, 1.0, at, 80, 0, 0, at, big, None) == BAD       # partitions that do not divide the rows
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, None, big, None) == BAD     # no workspace
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at + 8, big, None) == BAD   # off its alignment
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at, w(4, 8, 10, 2) - 1, None) == BAD
    assert b(at, 8, 0, at, 4, 8, 10, 2, 1.0, None, 80, 0, 0, at, big, None) == BAD
    assert b(None, 8, 0, at, 4, 8, 10, 2, 1.0, at, 80, 0, 0, at, big, None) == BAD
    assert b(at, 8, 0, at, 4, 8, 1 << 45, 2, 1.0, at, 1 << 48, 0, 0, at, big, None) == BAD


def test_head_refusals(lib):
    at, big = 4096, 1 << 40
    w = lib.solon_head_logprobs_workspace
    assert w(0, 8, 10, 0, 1) == 0 and w(1, 8, 10, 0, 1) > 0 and w(1000, 64, 1000, 2, 0) > w(1000, 64, 1000, 2, 1)
    assert w(4, 8, 10, 1, 1) == BAD and w(-1, 8, 10, 0, 1) == BAD and w(4, 0, 10, 0, 1) == BAD and w(4, 8, 0, 0, 1) == BAD and w(4, 1 << 23, 10, 0, 1) == BAD
    f = lib.solon_head_logprobs
    assert f(at, 8, at, 8, 1, at, 4, 8, 10, at, at, at, at, at, big, None) == BAD            # type
    assert f(at, 7, at, 8, 0, at, 4, 8, 10, at, at, at, at, at, big, None) == BAD            # pitches
    assert f(at, 8, at, 7, 0, at, 4, 8, 10, at, at, at, at, at, big, None) == BAD
    assert f(at + 2, 8, at, 8, 0, at, 4, 8, 10, at, at, at, at, at, big, None) == BAD        # alignment
    assert f(at, 8, at, 8, 0, at + 4, 4, 8, 10, at, at, at, at, at, big, None) == BAD
    assert f(at, 8, at, 8, 0, None, 4, 8, 10, at, at, at, at, at, big, None) == BAD          # logp without targets
    assert f(at, 8, at, 8, 0, at, 4, 8, 10, at, at, at, at, None, big, None) == BAD          # no workspace
    assert f(at, 8, at, 8, 0, at, 4, 8, 10, at, at, at, at, at + 16, big, None) == BAD
    assert f(at, 8, at, 8, 0, at, 4, 8, 10, at, at, at, at, at, w(4, 8, 10, 0, 1) - 1, None) == BAD
    assert f(None, 8, None, 8, 0, None, 0, 8, 10, None, None, None, None, None, 0, None) == 0
    v = lib.solon_head_logprobs_backward_workspace
    assert v(0, 8, 10, 1, 0, 0, 1) == 0 and v(4, 8, 10, 1, 0, 3, 1) == BAD and v(4, 8, 10, 1, 1, 0, 1) == BAD and v(4, 8, 10, 3, 0, 0, 1) == BAD
    assert v(100_000, 64, 50_000, 1, 2, 0, 1) < (1 << 29) + 100_000 * 128 * 4 + 4096                # dlogits comes in pieces
    b = lib.solon_head_logprobs_backward

    def call(h=at + 256, hp=8, m=at + 512, mp=8, dtype=0, t=at, rows=4, cols=8, vocab=10, parts=2, peak=at, ls=at, ent=None, g=at, gh=None, dh=at, dhp=8, dw=at, dwp=80, gt=0, ws=at, n=big):
        return b(h, hp, m, mp, dtype, t, rows, cols, vocab, parts, peak, ls, ent, g, gh, dh, dhp, dw, dwp, gt, ws, n, None)

    assert call(dtype=1) == BAD and call(hp=7) == BAD and call(mp=7) == BAD and call(h=None) == BAD and call(m=at + 1) == BAD and call(dh=at + 256) == BAD and call(dw=at + 512) == BAD and call(dh=at + 512) == BAD
    assert call(parts=3) == BAD and call(parts=0) == BAD and call(peak=None) == BAD and call(ls=None) == BAD and call(t=None) == BAD
    assert call(gh=at) == BAD and call(dhp=7) == BAD and call(dwp=79) == BAD and call(gt=3) == BAD and call(ws=None) == BAD and call(ws=at + 128) == BAD
    assert call(n=v(4, 8, 10, 2, 0, 0, 1) - 1) == BAD and call(cols=1 << 23) == BAD
    assert call(dh=None, dw=None) == 0                                                          # nothing wanted
