"""Outputs of the token model's two ends that share memory with inputs or with one another are refused, wherever they begin; views that lie between one
another's rows are not.  The refusals need no device: the addresses are never read."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build

BAD = binding.ERR_INVALID_ARG
BASE = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


def _embed(lib, out, weight=BASE, tokens=BASE << 4, rows=4, cols=8, vocab=10, out_pitch=8):
    return lib.solon_embedding_forward(weight, 8, 0, tokens, rows, cols, vocab, 1.0, out, out_pitch, None)


def test_embedding(lib):
    size = 10 * 8 * 4
    for out in (BASE, BASE + 4, BASE + size - 4, BASE - 4 * 8 * 4 + 4, (BASE << 4) - 4, (BASE << 4) + 4 * 8 - 4):
        assert _embed(lib, out) == BAD
    b = lib.solon_embedding_backward

    def back(dw, dy=BASE, tokens=BASE << 4, workspace=BASE << 8):
        return b(dy, 8, 0, tokens, 4, 8, 10, 2, 1.0, dw, 100, 0, 0, workspace, 1 << 30, None)

    whole = (100 + 80) * 4
    for dw in (BASE, BASE + 4, BASE + 4 * 8 * 4 - 4, BASE - whole + 4, (BASE << 4) - 4, (BASE << 4) + 28):
        assert back(dw) == BAD


def _back(lib, dh=BASE << 1, dw=BASE << 2, h=BASE << 3, w=BASE << 4, t=BASE << 5, peak=BASE << 6, log_sum=BASE << 7, ent=BASE << 8, g=BASE << 9, gh=BASE << 10, dhp=8, hp=8,
          workspace=BASE << 12):
    return lib.solon_head_logprobs_backward(h, hp, w, 8, 0, t, 4, 8, 10, 2, peak, log_sum, ent, g, gh, dh, dhp, dw, 100, 0, workspace, 1 << 40, None)


def test_head(lib):
    matrix, vocabulary, gradient = 4 * 8 * 4, 10 * 8 * 4, (100 + 80) * 4
    for at, size in ((BASE << 3, matrix), (BASE << 4, vocabulary), (BASE << 5, 32), (BASE << 6, 16), (BASE << 7, 16), (BASE << 8, 16), (BASE << 9, 16), (BASE << 10, 16)):
        for out, own in (("dh", matrix), ("dw", gradient)):
            for begin in (at, at + size - 4, at - own + 4):
                assert _back(lib, **{out: begin}) == BAD, (out, at, begin)
    for begin in ((BASE << 2) - matrix + 4, BASE << 2, (BASE << 2) + 80 * 4 - 4, (BASE << 2) + gradient - 4):
        assert _back(lib, dh=begin) == BAD                        # the two outputs
    f = lib.solon_head_logprobs
    for out in (BASE << 5, (BASE << 5) + 28, (BASE << 3) + matrix - 4, (BASE << 4) - 12):
        assert f(BASE << 3, 8, BASE << 4, 8, 0, BASE << 5, 4, 8, 10, out, BASE << 6, BASE << 7, BASE << 8, BASE << 12, 1 << 40, None) == BAD


@pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would be launched")
def test_what_lies_between_is_not_refused(lib):
    """(Without a device an accepted call ends with the runtime's error.)"""
    size = 10 * 8 * 4
    assert _embed(lib, BASE + size) not in (BAD, 0) and _embed(lib, BASE - 4 * 8 * 4) not in (BAD, 0)
    assert _embed(lib, BASE + 32, out_pitch=16, weight=BASE + (1 << 12)) not in (BAD, 0)
    assert _back(lib) not in (BAD, 0)
    h = BASE << 3
    assert _back(lib, h=h, hp=16, dh=h + 32, dhp=16) not in (BAD, 0)                     # columns of one buffer
    assert _back(lib, h=h + 32, hp=24, dh=h, dhp=24) not in (BAD, 0)
    assert _back(lib, h=h, hp=16, dh=h + 28, dhp=16) == BAD and _back(lib, h=h, hp=16, dh=h + 36, dhp=16) == BAD
    assert _back(lib, h=h, hp=16, dh=h + 32, dhp=24) == BAD                              # pitches that drift into one another
    assert _back(lib, dh=(BASE << 2) + 80 * 4, dhp=100 - 60) == BAD                      # in the gap of the gradient's rows, but too long for it
    assert _back(lib, dh=(BASE << 2) + 80 * 4, dhp=8) == BAD


@pytest.mark.gpu
def test_columns_of_one_buffer():
    """hidden, dhidden and what lies beside them in the same rows."""
    rows, cols, vocab = 40, 64, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    both = torch.randn((rows, 2 * cols), device="cuda", generator=g)
    h, dh = both[:, :cols], both[:, cols:]
    w = torch.randn((vocab, cols), device="cuda", generator=g) * 0.2
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    r = binding.solon_head_logprobs(h, w, t)
    factor = torch.full((rows,), -1.0, device="cuda")
    want, want_dw = binding.solon_head_logprobs_backward(h.contiguous(), w, t, r.peak, r.log_sum, factor)
    got, dw = binding.solon_head_logprobs_backward(h, w, t, r.peak, r.log_sum, factor, dhidden=dh)
    assert torch.equal(got, want) and torch.equal(dw, want_dw)
    for shifted in (both[:, 1:cols + 1], both[:, cols - 1:-1]):
        with pytest.raises(binding.SolonError):
            binding.solon_head_logprobs_backward(h, w, t, r.peak, r.log_sum, factor, dhidden=shifted)
    flat = torch.cat([w.flatten(), w.flatten()])
    with pytest.raises(binding.SolonError):
        binding.solon_head_logprobs_backward(h, flat[:vocab * cols].view(vocab, cols), t, r.peak, r.log_sum, factor, dweight=flat[64:64 + vocab * cols][None])
    with pytest.raises(binding.SolonError):
        binding.solon_embedding_forward(w, t, out=w[5:5 + rows])
    with pytest.raises(binding.SolonError):
        binding.solon_embedding_backward(flat[:rows * cols].view(rows, cols), t, vocab, dweight=flat[:vocab * cols][None])
