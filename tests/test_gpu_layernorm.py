"""Layer norm, forward and backward, against the formulas in float64 and against differences.

Tolerances (u = 2^-24, the rounding unit of float32; t that of the element type, doubled for the float32 value it rounds).
A row's sums run over 16 elements in a thread and a tree of at most 10 levels: 32 roundings cover them, so a mean is off by at
most 32 u max|x| and rstd by a relative 32 u + the mean's share.  y then is off by 64 u (rstd max|x| + |xh|) |w| + 2 u (|y| + |b|);
dx, whose mean and rstd are inputs, by 64 u rstd (|a| + mean|a| + |xh| mean|a xh|).  Sums over a partition's n rows: rounding
errors of independent sign grow as the root of their number: (16 + 2 sqrt n) u sum|terms|."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": (torch.float32, 2.0 ** -23), "bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -10)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, dtype, seed, scale=1.0, shift=0.0):
    return (torch.randn(shape, device="cuda", generator=_gen(seed)) * scale + shift).to(dtype)


def _strided(t, pitch, offset):
    """The same values in rows `pitch` elements apart, starting `offset` elements into a buffer."""
    buf = torch.full((offset + t.shape[0] * pitch,), 7.0, dtype=t.dtype, device="cuda")
    view = buf[offset:].view(t.shape[0], pitch)[:, :t.shape[1]]
    view.copy_(t)
    return view


def _forward_ref(x, w, b, eps):
    x = x.double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    rstd = (var + eps).rsqrt()
    xh = (x - mean[:, None]) * rstd[:, None]
    w = torch.ones_like(x[0]) if w is None else w.double()
    b = torch.zeros_like(x[0]) if b is None else b.double()
    return xh * w + b, mean, rstd, xh, w, b


def _check_forward(x, w, b, eps, y, mean, rstd, t):
    want, mean_w, rstd_w, xh, w, b = _forward_ref(x, w, b, eps)
    big = x.double().abs().amax(dim=1)
    assert ((mean.double() - mean_w).abs() <= 32 * U * big).all()
    assert ((rstd.double() - rstd_w).abs() <= rstd_w * (64 * U + 64 * U * (rstd_w * big))).all()
    # the statistics' error of the mean enters xh through the mean and, squared and first order, through rstd
    tol = 64 * U * ((rstd_w * big)[:, None] * (1 + xh.abs()) + xh.abs()) * w.abs() + 2 * U * (want.abs() + b.abs()) + t * want.abs() + (2.0 ** -24 if t == 2.0 ** -10 else 0)
    assert ((y.double() - want).abs() <= tol).all(), float(((y.double() - want).abs() / tol).max())


SHAPES = [(1, 1), (3, 2), (1, 2048), (7, 5), (33, 31), (64, 64), (9, 127), (130, 512), (65, 513), (40, 1000), (37, 1001), (300, 1024), (19, 2047),
          (50, 4096), (11, 4100), (6, 8192), (5, 9001), (9, 16384), (3, 16385), (4, 20000), (6, 1002), (5, 4102), (4, 10002), (9, 98)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_forward(rows, cols, dtype):
    dt, t = TYPES[dtype]
    x = _randn((rows, cols), dt, rows + cols, 2.0, 0.7)
    w, b = _randn(cols, torch.float32, 1), _randn(cols, torch.float32, 2)
    y, mean, rstd = binding.solon_layernorm_forward(x, w, b, eps=1e-5)
    _check_forward(x, w, b, 1e-5, y, mean, rstd, t)
    y, mean, rstd = binding.solon_layernorm_forward(x, w.to(dt), None, eps=1e-3)        # parameters in x's type; no bias
    _check_forward(x, w.to(dt), None, 1e-3, y, mean, rstd, t)
    y, mean, rstd = binding.solon_layernorm_forward(x)
    _check_forward(x, None, None, 1e-5, y, mean, rstd, t)


@pytest.mark.parametrize("cols,pitch,offset", [(64, 64, 1), (1000, 1003, 0), (1000, 1008, 8), (1000, 1004, 4), (129, 140, 3), (17000, 17001, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_strides_and_alignment(cols, pitch, offset, dtype):
    dt, t = TYPES[dtype]
    x = _strided(_randn((21, cols), dt, 3), pitch, offset)
    y = _strided(torch.zeros((21, cols), dtype=dt, device="cuda"), pitch + 3, offset)
    w, b = _randn(cols + 1, torch.float32, 1)[1:], _randn(cols + 1, torch.float32, 2)[1:]
    out, mean, rstd = binding.solon_layernorm_forward(x, w, b, y=y)
    assert out.data_ptr() == y.data_ptr()
    _check_forward(x, w, b, 1e-5, y, mean, rstd, t)
    before = y._base
    assert (before[:offset] == 7).all() and (before[offset:].view(21, pitch + 3)[:, cols:] == 7).all()      # nothing beside the rows
    before = x.clone()
    inplace, mean, rstd = binding.solon_layernorm_forward(x, w, b, y=x)
    assert inplace.data_ptr() == x.data_ptr()
    _check_forward(before, w, b, 1e-5, inplace, mean, rstd, t)


def test_forward_rows_that_are_constant_large_or_not_finite():
    x = torch.randn((6, 300), device="cuda", generator=_gen(4))
    x[0] = 3.0                       # no variance: y = b
    x[1] = 0.0
    x[2] += 1e4                      # a mean far above the deviations
    x[3, 17] = float("nan")
    x[4, 200] = float("inf")
    w, b = _randn(300, torch.float32, 1), _randn(300, torch.float32, 2)
    y, mean, rstd = binding.solon_layernorm_forward(x, w, b)
    for r in (0, 1, 2, 5):
        _check_forward(x[r:r + 1], w, b, 1e-5, y[r:r + 1], mean[r:r + 1], rstd[r:r + 1], 2.0 ** -23)
    assert y[3].isnan().all() and y[4].isnan().any() and torch.equal(y[1], b)


def _backward_ref(dy, x, mean, rstd, w, parts):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    w = torch.ones_like(x[:1]) if w is None else w.double()
    xh = (x - mean) * rstd
    a = dy * w
    dx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    tol = 64 * U * rstd * (a.abs() + a.abs().mean(1, keepdim=True) + xh.abs() * (a * xh).abs().mean(1, keepdim=True))
    n, cols = x.shape[0] // parts, x.shape[1]
    per = lambda z: z.view(parts, n, cols).sum(1)  # noqa: E731
    k = (16 + 2 * n ** 0.5) * U
    return dx, tol, per(dy * xh), k * per((dy * xh).abs()), per(dy), k * per(dy.abs())


def _check_backward(dy, x, mean, rstd, w, parts, got, t):
    dx_w, dx_t, dw_w, dw_t, db_w, db_t = _backward_ref(dy, x, mean, rstd, w, parts)
    dx, dw, db = got
    floor = 2.0 ** -24 if t == 2.0 ** -10 else 0
    assert ((dx.double() - dx_w).abs() <= dx_t + t * dx_w.abs() + floor).all(), float(((dx.double() - dx_w).abs() / (dx_t + t * dx_w.abs())).max())
    assert ((dw.double() - dw_w).abs() <= dw_t).all(), float(((dw.double() - dw_w).abs() / dw_t).max())
    assert ((db.double() - db_w).abs() <= db_t + 1e-300).all()


@pytest.mark.parametrize("parts,n,cols", [(1, 1, 1), (1, 1, 2048), (2, 3, 7), (15, 4, 64), (45, 7, 1001), (1, 700, 129), (4, 100, 513), (3, 33, 1000), (1, 2000, 256),
                                          (7, 40, 2048), (2, 50, 4096), (5, 9, 4097), (3, 20, 8192), (2, 9, 12345), (4, 8, 16384), (2, 5, 16387), (1, 40, 20000),
                                          (1000, 2, 40), (400, 1, 33), (3, 20, 1002), (2, 7, 5002),
                                          (3, 10, 6152), (2, 3, 10008), (5, 30, 98)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_backward_by_partitions(parts, n, cols, dtype):
    dt, t = TYPES[dtype]
    rows = parts * n
    x, dy = _randn((rows, cols), dt, rows + cols, 1.5, -0.4), _randn((rows, cols), dt, cols)
    w = _randn(cols, torch.float32, 5)
    _, mean, rstd = binding.solon_layernorm_forward(x, w)
    got = binding.solon_layernorm_backward(dy, x, mean, rstd, w, partitions=parts)
    _check_backward(dy, x, mean, rstd, w, parts, got, t)
    again = binding.solon_layernorm_backward(dy, x, mean, rstd, w, partitions=parts)
    assert all(torch.equal(p, q) for p, q in zip(got, again))                          # the order of the sums is fixed
    only_dx = binding.solon_layernorm_backward(dy, x, mean, rstd, w, partitions=parts, param_grads=False)
    assert torch.equal(only_dx[0], got[0])


@pytest.mark.parametrize("grad", [torch.float32, torch.float64])
@pytest.mark.parametrize("cols", [96, 1001, 17001])
def test_backward_writes_into_the_gradient_matrix(cols, grad):
    """Weight and bias gradients go to their columns of a P x d matrix with odd pitch; everything else in it stays."""
    parts, n, d = 6, 5, 2 * cols + 35
    x, dy = _strided(_randn((parts * n, cols), torch.float32, 1), cols + 5, 3), _strided(_randn((parts * n, cols), torch.float32, 2), cols + 1, 2)
    w = _randn(cols, torch.float32, 5)
    _, mean, rstd = binding.solon_layernorm_forward(x, w)
    grads = torch.full((parts, d), -3.0, dtype=grad, device="cuda")
    dx = _strided(torch.zeros((parts * n, cols), device="cuda"), cols + 2, 1)
    got = binding.solon_layernorm_backward(dy, x, mean, rstd, w, partitions=parts, dx=dx, dweight=grads[:, 11:11 + cols], dbias=grads[:, 20 + cols:20 + 2 * cols])
    _check_backward(dy, x, mean, rstd, w, parts, got, 2.0 ** -23)
    keep = torch.ones(d, dtype=torch.bool, device="cuda")
    keep[11:11 + cols] = False
    keep[20 + cols:20 + 2 * cols] = False
    assert (grads[:, keep] == -3).all() and (dx._base[1:].view(parts * n, cols + 2)[:, cols:] == 7).all() and dx._base[0] == 7
    for target in (dy, x):                                                            # dx over one of its inputs
        xc, dyc = x.clone(), dy.clone()
        over = dyc if target is dy else xc
        dw = torch.empty((parts, cols), device="cuda")
        got2 = binding.solon_layernorm_backward(dyc, xc, mean, rstd, w, partitions=parts, dx=over, dweight=dw, dbias=torch.empty_like(dw))
        assert got2[0].data_ptr() == over.data_ptr()
        _check_backward(dy, x, mean, rstd, w, parts, got2, 2.0 ** -23)


@pytest.mark.parametrize("parts,n,cols", [(1, 900, 8200), (1, 700, 16384), (45, 12, 8194), (2, 300, 8201), (149, 3, 9000), (1, 1, 16000), (20, 40, 8192), (50, 30, 5001),
                                          (1, 1300, 2048), (37, 9, 770)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_backward_of_rows_that_take_turns(parts, n, cols, dtype):
    """CTAs of one to many rows, shares of a partition that are not alike, on both sides of the widths where the kernel changes;
    dx over dy, over x, or not wanted; no weight."""
    dt, t = TYPES[dtype]
    rows = parts * n
    x, dy = _strided(_randn((rows, cols), dt, rows + cols, 1.5, -0.4), cols + 8, 0), _strided(_randn((rows, cols), dt, cols), cols + 16, 8)
    _, mean, rstd = binding.solon_layernorm_forward(x, None)
    got = binding.solon_layernorm_backward(dy, x, mean, rstd, None, partitions=parts)
    _check_backward(dy, x, mean, rstd, None, parts, got, t)
    w = _randn(cols, torch.float32, 5)
    want = binding.solon_layernorm_backward(dy, x, mean, rstd, w, partitions=parts)
    _check_backward(dy, x, mean, rstd, w, parts, want, t)
    over = dy.clone()                                                                  # (dense: the same elements, other pitches)
    dw = torch.empty((parts, cols), device="cuda")
    got = binding.solon_layernorm_backward(over, x, mean, rstd, w, partitions=parts, dx=over, dweight=dw, dbias=torch.empty_like(dw))
    assert got[0].data_ptr() == over.data_ptr()
    _check_backward(dy, x, mean, rstd, w, parts, got, t)
    over = x.clone()
    got = binding.solon_layernorm_backward(dy, over, mean, rstd, w, partitions=parts, dx=over, param_grads=False)
    _check_backward(dy, x, mean, rstd, w, parts, (got[0], *want[1:]), t)


def test_backward_agrees_with_differences():
    """Directional derivatives of sum c y by central differences of the forward kernel.  h = 2^-6 along a direction of unit
    entries: the second-order error is below h^2 relative, rounding (u |y| per output, independent) below sqrt(N) u / h of the
    direction's share; 2e-3 of the gradient's norm covers both."""
    rows, cols, parts = 12, 200, 3
    x, c = _randn((rows, cols), torch.float32, 1), _randn((rows, cols), torch.float32, 2)
    w, b = 1 + 0.3 * _randn(cols, torch.float32, 3), _randn(cols, torch.float32, 4)
    _, mean, rstd = binding.solon_layernorm_forward(x, w, b)
    dx, dw, db = binding.solon_layernorm_backward(c, x, mean, rstd, w, partitions=parts)
    h = 2.0 ** -6

    def f(x_, w_, b_):
        return (binding.solon_layernorm_forward(x_, w_, b_)[0].double() * c.double()).view(parts, -1).sum(1)

    for seed in range(5):
        ex, ew = _randn((rows, cols), torch.float32, 10 + seed).sign(), _randn(cols, torch.float32, 20 + seed).sign()
        got = (f(x + h * ex, w, b) - f(x - h * ex, w, b)) / (2 * h)
        assert ((got - (dx.double() * ex).view(parts, -1).sum(1)).abs() <= 2e-3 * dx.double().view(parts, -1).norm(dim=1) * 3).all()
        got = (f(x, w + h * ew, b) - f(x, w - h * ew, b)) / (2 * h)
        assert ((got - (dw.double() * ew).sum(1)).abs() <= 2e-3 * dw.double().norm(dim=1)).all()
        got = (f(x, w, b + h * ew) - f(x, w, b - h * ew)) / (2 * h)
        assert ((got - (db.double() * ew).sum(1)).abs() <= 2e-3 * db.double().norm(dim=1)).all()


def test_empty_and_other_streams():
    x = torch.empty((0, 40), device="cuda")
    y, mean, rstd = binding.solon_layernorm_forward(x)
    assert y.shape == (0, 40)
    dw = torch.full((3, 40), 5.0, device="cuda")
    dx, dw, db = binding.solon_layernorm_backward(x, x, mean, rstd, partitions=3, dweight=dw)
    assert (dw == 0).all() and (db == 0).all() and dx.shape == (0, 40)
    x = _randn((600, 777), torch.float32, 1)
    want = binding.solon_layernorm_forward(x)
    want_b = binding.solon_layernorm_backward(x, x, want[1], want[2], partitions=2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = binding.solon_layernorm_forward(x)
        got_b = binding.solon_layernorm_backward(x, x, got[1], got[2], partitions=2)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want + want_b, got + got_b))


def test_offsets_beyond_32_bits():
    """A matrix of more than 2^32 bytes and 2^31 elements: its last rows, and the last partition's sums, as those of a copy."""
    rows, cols, tail = 540_000, 4000, 1000
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[:-tail] = 1.0
    x[-tail:] = _randn((tail, cols), torch.bfloat16, 1)
    w = _randn(cols, torch.float32, 2)
    y, mean, rstd = binding.solon_layernorm_forward(x, w, w)
    part = binding.solon_layernorm_forward(x[-tail:].clone(), w, w)
    assert torch.equal(y[-tail:], part[0]) and torch.equal(mean[-tail:], part[1]) and torch.equal(rstd[-tail:], part[2])
    parts = rows // tail
    dx, dw, db = binding.solon_layernorm_backward(x, x, mean, rstd, w, partitions=parts, dx=y)
    got = binding.solon_layernorm_backward(x[-tail:].clone(), x[-tail:].clone(), part[1], part[2], w)
    assert torch.equal(dx[-tail:], got[0])
    assert float((dw[-1] - got[1][0]).abs().max()) <= 1e-4 * float(got[1].abs().max()) and float((db[-1] - got[2][0]).abs().max()) <= 1e-4 * float(got[2].abs().max())


def test_refusals():
    x = torch.zeros((6, 8), device="cuda")
    m = torch.zeros(6, device="cuda")
    bad = [lambda: binding.solon_layernorm_forward(x.cpu()), lambda: binding.solon_layernorm_forward(x > 0), lambda: binding.solon_layernorm_forward(x[0]),
           lambda: binding.solon_layernorm_forward(x.t()), lambda: binding.solon_layernorm_forward(x, torch.zeros(7, device="cuda")),
           lambda: binding.solon_layernorm_forward(x, torch.zeros(8, device="cuda", dtype=torch.bfloat16), torch.zeros(8, device="cuda")),
           lambda: binding.solon_layernorm_forward(x, y=torch.zeros((6, 9), device="cuda")),
           lambda: binding.solon_layernorm_backward(x, x, m[:5], m), lambda: binding.solon_layernorm_backward(x.bfloat16(), x, m, m),
           lambda: binding.solon_layernorm_backward(x, x, m, m, partitions=2, dweight=torch.zeros((3, 8), device="cuda")),
           lambda: binding.solon_layernorm_backward(x, x, m, m, dweight=torch.zeros((1, 8), device="cuda", dtype=torch.float16))]
    for call in bad[:-1]:
        with pytest.raises(ValueError):
            call()
    refused = [bad[-1], lambda: binding.solon_layernorm_forward(x.double()), lambda: binding.solon_layernorm_forward(x, eps=0.0), lambda: binding.solon_layernorm_forward(x, eps=float("nan")),
               lambda: binding.solon_layernorm_forward(x, torch.zeros(8, device="cuda", dtype=torch.bfloat16)),
               lambda: binding.solon_layernorm_backward(x, x, m, m, partitions=4), lambda: binding.solon_layernorm_backward(x, x, m, m, partitions=0),
               lambda: binding.solon_layernorm_forward(torch.zeros((2, 0), device="cuda"))]
    for call in refused:
        with pytest.raises(binding.SolonError) as err:
            call()
        assert err.value.status == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("parts,n,cols,pitch,offset", [(1, 3, 16_385, 16_385, 0), (3, 2, 16_387, 16_390, 1), (2, 60, 20_000, 20_001, 3), (1, 1, 65_537, 65_537, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_that_pass_registers(parts, n, cols, pitch, offset, dtype):
    """Rows of the streaming kernels, one CTA a row: every row's sums by all its warps, several rows to a CTA, in place."""
    dt, t = TYPES[dtype]
    x, dy = (_strided(_randn((parts * n, cols), dt, q, 1.5, 0.4), pitch, offset) for q in (5, 6))
    w, b = _randn(cols, torch.float32, 7), _randn(cols, torch.float32, 8)
    y, mean, rstd = binding.solon_layernorm_forward(x, w, b)
    _check_forward(x, w, b, 1e-5, y, mean, rstd, t)
    got = binding.solon_layernorm_backward(dy, x, mean, rstd, w, partitions=parts)
    _check_backward(dy, x, mean, rstd, w, parts, got, t)
    out = dy.clone()
    inplace = binding.solon_layernorm_backward(out, x, mean, rstd, w, partitions=parts, dx=out)
    assert inplace[0].data_ptr() == out.data_ptr() and all(torch.equal(p, q) for p, q in zip(inplace, got))
