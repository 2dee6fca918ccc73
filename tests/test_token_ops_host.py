"""CPU-only checks of the token-model operators' C entries: sizes they report, and arguments they refuse before touching a device."""

import ctypes

import pytest

from paper_2110_01595_b200 import binding, build

BAD = binding.ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


def test_state_blocks(lib):
    def blocks(*sizes):
        return lib.solon_adamw_state_blocks(len(sizes), (ctypes.c_int64 * max(1, len(sizes)))(*sizes))

    assert blocks(1) == 1 and blocks(256) == 1 and blocks(257, 0, 5) == 3 and blocks(0) == 0
    assert blocks() == BAD and blocks(-1) == BAD and blocks(1 << 41) == BAD
    assert blocks(1 << 36) == 1 << 28 and blocks(1 << 36, 1) == BAD and blocks(*[1 << 35] * 3) == BAD
    assert lib.solon_adamw_state_blocks(1, None) == BAD


def test_backward_workspace(lib):
    f = lib.solon_layernorm_backward_workspace
    assert f(0, 8, 3) == 0 and f(1, 100, 1) == 0
    for rows, cols, parts in ((4096, 1024, 1), (4500, 333, 45), (100, 20_000, 2)):
        need = f(rows, cols, parts)
        assert need > 0 and need % (parts * 2 * cols * 4) == 0
        assert need // (parts * 2 * cols * 4) <= rows // parts
    assert f(10, 8, 3) == BAD and f(10, 8, 0) == BAD and f(-1, 8, 1) == BAD and f(10, 0, 1) == BAD and f(10, 1 << 25, 1) == BAD and f(2050, 4, 1025) == BAD


def test_refused_arguments(lib):
    at = 4096                                   # an aligned address that no refused call reads
    assert lib.solon_layernorm_forward(at, 8, 9, None, None, 0, 4, 8, 1e-5, at, 8, None, None, None) == BAD        # element type
    assert lib.solon_layernorm_forward(at, 8, 1, None, None, 0, 4, 8, 1e-5, at, 8, None, None, None) == BAD        # no float64 here
    assert lib.solon_layernorm_forward(None, 8, 0, None, None, 0, 4, 8, 1e-5, at, 8, None, None, None) == BAD
    assert lib.solon_layernorm_forward(at + 2, 8, 0, None, None, 0, 4, 8, 1e-5, at, 8, None, None, None) == BAD    # alignment
    assert lib.solon_layernorm_forward(at, 7, 0, None, None, 0, 4, 8, 1e-5, at, 8, None, None, None) == BAD        # pitch
    assert lib.solon_layernorm_forward(at, 8, 0, None, None, 0, 0, 8, 1e-5, None, 8, None, None, None) == 0        # no rows: nothing to do
    back = lib.solon_layernorm_backward
    assert back(at, 64, at, 64, 0, None, 0, at, at, 4096, 64, 1, at, 64, at, at, 64, 0, None, 0, None) == BAD      # workspace missing
    assert back(at, 64, at, 64, 0, None, 0, at, at, 4096, 64, 1, at, 64, at, at, 64, 0, at, 16, None) == BAD       # workspace too small
    assert back(at, 64, at, 64, 0, None, 0, at, at, 4, 64, 2, at, 64, at, at, 63, 0, None, 0, None) == BAD         # gradient pitch
    assert back(at, 64, at, 64, 0, None, 0, at, at, 4, 64, 2, at, 64, at, at, 64, 2, None, 0, None) == BAD         # gradient type
    assert back(at, 64, at, 64, 0, None, 0, None, at, 4, 64, 2, at, 64, at, at, 64, 0, None, 0, None) == BAD       # no mean
    assert back(at, 64, at, 64, 0, None, 0, at, at, 4, 64, 2, None, 64, None, None, 64, 0, None, 0, None) == 0     # nothing wanted
    fwd = lib.solon_token_logprobs
    assert fwd(at, 8, 0, at, 4, 8, 9, at, at, at, at, at, at, None) == BAD and fwd(at, 99, 0, at, 4, 99, 33, at, at, at, at, at, at, None) == BAD
    assert fwd(at, 8, 0, None, 4, 8, 0, at, at, at, at, None, None, None) == BAD                                       # logp without targets
    assert fwd(at, 8, 0, at, 4, 8, 2, at, at, at, at, None, at, None) == BAD and fwd(at, 8, 0, at + 4, 4, 8, 0, at, at, at, at, None, None, None) == BAD
    assert fwd(None, 8, 0, None, 0, 8, 0, None, None, None, None, None, None, None) == 0
    bwd = lib.solon_token_logprobs_backward
    assert bwd(at, 8, 0, None, 4, 8, at, at, None, at, None, at, 8, None) == BAD                                       # gradient of logp without targets
    assert bwd(at, 8, 0, at, 4, 8, at, at, None, None, at, at, 8, None) == BAD                                         # gradient of the entropy without it
    assert bwd(at, 8, 0, at, 4, 8, at, None, None, at, None, at, 8, None) == BAD
    assert bwd(at, 8, 0, at, 4, 8, at, at, None, at, None, at, 9, None) == BAD                                         # in place with another pitch
    for call in (lib.solon_adamw_destroy, lambda h: lib.solon_adamw_set_step(h, 1), lambda h: lib.solon_adamw_get_steps(h, None, None),
                 lambda h: lib.solon_adamw_bind_grads(h, None, 0), lambda h: lib.solon_adamw_moments(h, at, at, None),
                 lambda h: lib.solon_adamw_step(h, at, 0, 1.0, 1.0, 0.0, None, None, None)):
        assert call(None) == BAD


def test_plans_refuse_the_types_of_the_token_operators(lib):
    plan = ctypes.c_void_p()
    for dtype in (binding.BF16, binding.F16, 4, -1):
        assert lib.solon_plan_create_ex(8, 1, 2, 4, 64, 1, dtype, ctypes.byref(plan)) == BAD and plan.value is None


def test_refused_handles(lib):
    at, handle = 4096, ctypes.c_void_p()
    n = (ctypes.c_int64 * 2)(10, 20)
    p = (ctypes.c_void_p * 2)(at, at)

    def create(count=2, numel=n, params=p, copies=None, decay=None, bits=32, m=at, v=at, base=None, b1=0.9, b2=0.99, eps=1e-8, out=ctypes.byref(handle)):
        return lib.solon_adamw_create(count, numel, params, copies, decay, bits, m, v, base, b1, b2, eps, 0, out)

    assert create(count=0) == BAD and create(numel=None) == BAD and create(params=None) == BAD and create(bits=16) == BAD and create(bits=8) == BAD
    assert create(m=None) == BAD and create(v=at + 4) == BAD and create(bits=8, base=at + 2) == BAD and create(out=None) == BAD
    assert create(b1=1.0) == BAD and create(b2=float("nan")) == BAD and create(eps=0.0) == BAD and create(eps=1e-60) == BAD
    assert create(params=(ctypes.c_void_p * 2)(at, None)) == BAD and create(params=(ctypes.c_void_p * 2)(at, at + 2)) == BAD
    assert create(copies=(ctypes.c_void_p * 2)(None, at + 1)) == BAD and create(decay=(ctypes.c_float * 2)(0.0, -0.1)) == BAD
    assert handle.value is None
