"""Log probabilities straight from hidden states and output matrix, and their gradient, against the formulas in float64 and against differences.

Tolerances (u = 2^-24, s_iv = sum_c |h_ic w_vc|).  Products of 16-bit elements are exact in float32; the tensor cores add 16 of them to an accumulator
and cut off what lies below its last bit, less than 2 u of what it holds a step, and after 32 steps (64 u s at most) the sum is added to another in
float32, u s at most each time: a logit is off by at most z_tol = (64 + cols / 256) u s.  float32 elements are two float16 pieces: 2^-22 of each factor, the
product of the second pieces left out (2^-22) and 2^-40 of each tensor's largest element: 2^-20 s + cols 2^-39 max|h| max|w| more.
(Few rows: ordinary sums, (cols / 32 + 8) u s, which is below that.)
From there the statistics are those of solon_token_logprobs: with t = max z_tol over the row, k = vocab / 256 + 72 additions and D = E|z - M| + 4
under the softmax, log S is off by (k + 2 D) u + 2 t, logp by 2 u (|z_t - M| + |log S|) + 2 t more, the entropy by
(2 k + 4 D) u (1 + |log S| + E|z - M| + E|z - M|^2) + 2 t (1 + E|log p + H|).
Gradient: p is off by a relative r = (4 |log p| + 8) u + z_tol; so dz = -p (g + g_H (log p + H)) by p |g + g_H (log p + H)| (r + 4 u) + p |g_H| (z_tol + 4 u (|log p| + H));
a product with dz is off by what that gives, by the sum's c u times its absolute terms (c = 64 + n / 256 as above; 1040 + n / 4096 where the
result has 16 bits, as 256 steps are cut off before the sum is added to another), by dz's own rounding (half a step: 2^-8 for bfloat16, 2^-11 for
float16 with 2^-40 of the largest bound below; float16's squared where there are two pieces, which are float16 ones for float32 gradients of any
states, and 2^-40 of the largest bfloat16 state) and by half a step of the result's type.  A bfloat16 gradient
of float32 states takes the first float16 piece of both factors alone, so h's rounding of half a float16 step, 2^-11 of each term, joins dz's.
The tensor cores line a step's products up by the factors' exponents, and a float16 element below 2^-14 has the exponent of 2^-14 with zeros in front: what is
cut off is relative to that, so such an element counts as 2^-14 in the terms of 64 u s and c u (with 2^-20 at 2e-6, six bits less are kept: 64 u becomes 2^-12)."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f64": torch.float64}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _framed(rows, cols, dtype, pitch=None, offset=0, fill=99.0):
    pitch = cols if pitch is None else pitch
    buf = torch.full((offset + rows * pitch + 64,), fill, dtype=TYPES[dtype], device="cuda")
    return buf, buf[offset:offset + rows * pitch].view(rows, pitch)[:, :cols]


def _untouched(buf, view, fill=99.0):
    mark = torch.ones_like(buf, dtype=torch.bool)
    mark.as_strided(view.shape, view.stride(), view.storage_offset())[...] = False
    return bool((buf[mark] == fill).all())


def _inputs(rows, cols, vocab, dtype, seed, layout=(0, 0), scale=1.5):
    g = _gen(seed)
    offset, more = layout
    _, h = _framed(rows, cols, dtype, cols + more, offset)
    _, w = _framed(vocab, cols, dtype, cols + more, offset)
    w.copy_(torch.randn((vocab, cols), device="cuda", generator=g) * (scale * cols ** -0.5))
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    h.copy_(torch.randn((rows, cols), device="cuda", generator=g) + 2 * w[t].float())
    return h, w, t


def _logits(h, w):
    """Exact logits and what each may be off by."""
    a, b = h.double(), w.double()
    z, s = a @ b.t(), _size(h) @ _size(w).t()
    tol = (64 + h.shape[1] / 256 + h.shape[1] / 32 + 8) * U * s
    if h.dtype == torch.float32:
        tol = tol + 2.0 ** -20 * s + h.shape[1] * 2.0 ** -39 * a.abs().max() * b.abs().max()
    return z, tol


def _size(x):
    """Magnitudes as they count in what a sum cuts off."""
    return x.double().abs().clamp(min=2.0 ** -14) if x.dtype == torch.float16 else x.double().abs()


def _close(x, y, tol, what):
    x = x.double()
    same = (x == y) | ((x - y).abs() <= tol) | (x.isnan() & y.isnan())
    assert same.all(), (what, x[~same][:4], y[~same][:4], tol[~same][:4] if tol.dim() else tol)


def _check_forward(h, w, t, got):
    z, zt = _logits(h, w)
    vocab = z.shape[1]
    big = z.amax(1)
    tz = zt.amax(1)
    c = z - big[:, None]
    log_s = c.exp().sum(1).log()
    lp = c - log_s[:, None]
    p = lp.exp()
    ent = -(p * lp).sum(1)
    e1, e2 = (p * c.abs()).sum(1), (p * c * c).sum(1)
    k, d = vocab / 256 + 72, e1 + 4
    _close(got.peak, big, tz + U * big.abs(), "peak")
    tol = (k + 2 * d) * U + 2 * U * log_s.abs() + 2 * tz
    _close(got.log_sum, log_s, tol, "log_sum")
    _close(got.entropy, ent, (2 * k + 4 * d) * U * (1 + log_s.abs() + e1 + e2) + 2 * tz * (1 + (p * (lp + ent[:, None]).abs()).sum(1)), "entropy")
    if t is not None:
        ct = c.gather(1, t.clamp(min=0)[:, None])[:, 0]
        _close(got.logp, torch.where(t < 0, 0.0, ct - log_s), tol + 2 * U * (ct.abs() + log_s.abs()) + 2 * tz, "logp")
    else:
        assert got.logp is None
    assert got.top_ids is None and got.top_logp is None


SHAPES = [(1, 1, 1), (1, 64, 3), (2, 7, 50), (3, 100, 257), (5, 2048, 1000), (8, 333, 5001), (9, 64, 256), (13, 40, 300), (16, 1001, 700), (17, 24, 1025), (1, 9000, 333),
          (16, 9000, 70), (128, 128, 512), (129, 72, 513), (256, 256, 256), (257, 520, 1111), (600, 1001, 2003), (2050, 64, 3000), (40, 4096, 5000), (1, 512, 131_072), (300, 48, 50_001),
          (5, 40, 19_001), (8, 520, 18_944), (9, 2049, 19_000), (16, 333, 20_003), (23, 100, 19_500), (32, 65, 30_000)]


@pytest.mark.parametrize("rows,cols,vocab", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_forward(rows, cols, vocab, dtype):
    h, w, t = _inputs(rows, cols, vocab, dtype, rows + cols)
    if rows > 2:
        t[1] = -1
    _check_forward(h, w, t, binding.solon_head_logprobs(h, w, t))
    _check_forward(h, w, None, binding.solon_head_logprobs(h, w))


@pytest.mark.parametrize("rows,cols,vocab", [(3, 100, 300), (12, 65, 301), (300, 130, 700), (70, 1000, 300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", [(1, 0), (0, 1), (2, 2), (4, 4), (8, 8), (3, 5)])
def test_forward_strides_and_alignment(rows, cols, vocab, dtype, layout):
    h, w, t = _inputs(rows, cols, vocab, dtype, 3, layout)             # (the 99s beside the rows count nowhere)
    _check_forward(h, w, t, binding.solon_head_logprobs(h, w, t))


def _check_backward(h, w, t, peak, log_sum, g, entropy, gh, parts, dh, dw):
    rows, cols = h.shape
    vocab = w.shape[0]
    n = rows // parts
    z, zt = _logits(h, w)
    lp = z - peak.double()[:, None] - log_sum.double()[:, None]
    p = lp.exp()
    ga = torch.zeros(rows, dtype=torch.float64, device="cuda") if g is None else torch.where(t >= 0, g.double(), 0.0)
    gha = torch.zeros_like(ga) if gh is None else gh.double()
    ent = torch.zeros_like(ga) if gh is None else entropy.double()
    inner = ga[:, None] + gha[:, None] * (lp + ent[:, None])
    dz = -p * inner
    if g is not None:
        dz.scatter_add_(1, t.clamp(min=0)[:, None], ga[:, None])
    r = (4 * lp.abs() + 8) * U + zt
    dzt = p * inner.abs() * (r + 4 * U) + p * gha.abs()[:, None] * (zt + 4 * U * (lp.abs() + ent.abs()[:, None])) + 2 * U * dz.abs()
    dzt = dzt * 1.01 + 2.0 ** -125 * (ga.abs() + gha.abs())[:, None]
    half = torch.finfo(torch.bfloat16 if h.dtype == torch.bfloat16 else torch.float16).eps / 2
    bound = float((ga.abs() + gha.abs() * (ent.abs() + 1)).max())
    least = 0.0 if h.dtype == torch.bfloat16 else 2.0 ** -39 * bound

    def sums(result, a, atol, factor, pieces, inner_size, what):
        b = factor.double()
        x = a @ b
        size = a.abs() @ b.abs()
        step = torch.finfo(result.dtype).eps / 2
        c = 1040 + inner_size / 4096 if result.element_size() == 2 else 64 + inner_size / 256
        fine = pieces == 2 and h.dtype == torch.bfloat16          # bfloat16 states: dz in float16 pieces, the states as float16 elements
        rounding = (2.0 ** -21 if pieces == 2 else half) * size + (2.0 ** -39 * bound if fine else least) * b.abs().sum(-2, keepdim=True)
        if fine:
            rounding = rounding + 2.0 ** -39 * b.abs().max() * a.abs().sum(-1, keepdim=True)
        tol = atol @ b.abs() + rounding + c * U * (a.abs() @ _size(factor)) + step * x.abs()
        if h.dtype == torch.float32:                              # the other factor's pieces
            tol = tol + (2.0 ** -11 if pieces == 1 else 2.0 ** -20) * size + 2.0 ** -39 * b.abs().max() * a.abs().sum(-1, keepdim=True)
        if result.dtype == torch.float16:
            tol = tol + 2.0 ** -25                                # half a step of its smallest numbers
        _close(result, x, tol, what)

    if dh is not None:
        sums(dh, dz, dzt, w, 2 if h.dtype == torch.float32 else 1, vocab, "dhidden")
    if dw is not None:
        full = dw.as_strided((parts, vocab, cols), (dw.stride(0), cols, 1), dw.storage_offset())
        coarse = dw.dtype == torch.bfloat16
        for k in range(parts):
            q = slice(k * n, (k + 1) * n)
            sums(full[k], dz[q].t(), dzt[q].t(), h[q], 1 if coarse else 2, n, f"dweight {k}")


def _stats(h, w):
    z, _ = _logits(h, w)
    big = z.amax(1)
    lp = torch.log_softmax(z, 1)
    return big.float(), (torch.logsumexp(z, 1) - big).float(), (-(lp.exp() * lp).sum(1)).float()


# rows of a partition, partitions, columns, vocabulary
BACK = [(1, 1, 1, 1), (1, 3, 8, 40), (4, 2, 24, 130), (64, 5, 333, 700), (63, 3, 64, 257), (65, 2, 128, 256), (200, 1, 129, 1000), (300, 2, 520, 999), (1, 7, 1000, 300), (2000, 1, 72, 511),
        (512, 1, 1024, 512), (130, 1, 40, 20_000), (1, 1, 520, 19_000), (4, 4, 72, 19_003), (16, 1, 333, 19_100), (1, 7, 1001, 19_001), (2, 3, 40, 20_000)]


@pytest.mark.parametrize("n,parts,cols,vocab", BACK)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_backward(n, parts, cols, vocab, dtype):
    rows = n * parts
    for layout, (at, after), grad, with_g, with_h in (((0, 0), (0, 0), "f32", True, False), ((1, 3), (5, 3), "f32", True, True), ((8, 8), (16, 16), "bf16", True, False),
                                                      ((0, 0), (3, 1), "f64", False, True), ((0, 0), (1, 0), "bf16", True, True)):
        h, w, t = _inputs(rows, cols, vocab, dtype, n + cols, layout)
        g = _gen(7)
        if rows > 3:
            t[::5] = -1
        peak, log_sum, entropy = _stats(h, w)
        grad_logp = -torch.rand(rows, device="cuda", generator=g) / n if with_g else None
        grad_entropy = torch.randn(rows, device="cuda", generator=g) / n if with_h else None
        buf, dw = _framed(parts, vocab * cols, grad, vocab * cols + after, at)
        buf_h, dh = _framed(rows, cols, dtype, cols + layout[1], layout[0])
        a, b = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, grad_logp, entropy, grad_entropy, partitions=parts, dhidden=dh, dweight=dw)
        assert a is dh and b is dw and _untouched(buf, dw) and _untouched(buf_h, dh)
        _check_backward(h, w, t, peak, log_sum, grad_logp, entropy, grad_entropy, parts, dh, dw)
        only_h, none = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, grad_logp, entropy, grad_entropy, partitions=parts, weight_grad=False)
        assert none is None
        only_w = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, grad_logp, entropy, grad_entropy, partitions=parts, hidden_grad=False,
                                                      dweight=torch.empty_like(dw).contiguous())[1]
        assert torch.equal(only_w, dw)                            # the same bits again
        _check_backward(h, w, t, peak, log_sum, grad_logp, entropy, grad_entropy, parts, only_h, None)


@pytest.mark.parametrize("dtype,grad,rows", [("bf16", "f32", 24_000), ("f32", "f32", 32_000), ("f16", "bf16", 48_000), ("bf16", "bf16", 80_000)])
def test_backward_in_pieces_of_the_vocabulary(dtype, grad, rows):
    """So many rows that dlogits comes in pieces (at most 512 MB of them at a time), the last one ragged, targets in every piece."""
    cols, vocab, parts = 72, 7001, 2
    h, w, t = _inputs(rows, cols, vocab, dtype, 2)
    t[::7] = -1
    peak, log_sum, entropy = _stats(h, w)
    g = -torch.rand(rows, device="cuda", generator=_gen(1)) / rows
    dw = torch.empty((parts, vocab * cols), dtype=TYPES[grad], device="cuda")
    dh, _ = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, partitions=parts, dweight=dw)
    _check_backward(h, w, t, peak, log_sum, g, None, None, parts, dh, dw)


@pytest.mark.parametrize("rows", [4, 300])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_edges(rows, dtype):
    """Targets outside the vocabulary, equal logits, rows without a share in the loss, what is not finite."""
    vocab, cols = 517, 96
    h, w, t = _inputs(rows, cols, vocab, dtype, 5)
    t[0], t[1] = vocab, -(1 << 40)
    h[2] = 0.0                                                    # all logits equal
    got = binding.solon_head_logprobs(h, w, t)
    assert got.logp[0].isnan() and got.logp[1] == 0.0 and torch.isfinite(got.log_sum).all()
    assert abs(float(got.entropy[2]) - torch.log(torch.tensor(517.0)).item()) < 1e-5 and got.peak[2] == 0.0
    peak, log_sum, _ = _stats(h, w)
    g = torch.full((rows,), -0.25, device="cuda")
    dh, dw = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g)
    assert (dh[1] == 0).all()                                     # no target
    assert torch.isfinite(dh[2:]).all() and torch.isfinite(dw).all()
    zero = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, torch.zeros_like(g))
    assert (zero[0] == 0).all() and (zero[1] == 0).all()
    minus = peak.clone()
    minus[3] = -INF                                               # a row of which nothing is left
    assert (binding.solon_head_logprobs_backward(h, w, t, minus, log_sum, g)[0][3] == 0).all()
    # a NaN in the hidden states stays in its row, one in the output matrix in its token, as far as a softmax allows
    h[0, 5] = NAN
    got = binding.solon_head_logprobs(h, w, t)
    assert got.peak[0].isnan() and got.log_sum[0].isnan() and got.entropy[0].isnan() and torch.isfinite(got.log_sum[1:]).all()
    h[0, 5] = 1.0
    w[vocab - 1, 3] = NAN
    got = binding.solon_head_logprobs(h, w, t)
    assert got.peak.isnan().all() and got.log_sum.isnan().all() and got.logp[1] == 0.0
    w[vocab - 1, 3] = 0.0
    h[3], w[7], w[8] = 1.0, INF, -INF
    got = binding.solon_head_logprobs(h[3:4].contiguous() if rows == 4 else h, w, None)
    at = 0 if rows == 4 else 3
    if dtype == "f32" and rows > 16:                              # two pieces of an element: their products with infinity have no sum
        assert got.peak[at].isnan() and got.log_sum[at].isnan()
        return
    assert got.peak[at] == INF and got.log_sum[at].isnan()
    w[7] = 0.0                                                    # one token masked out by -infinity: p = 0 for it
    row = binding.solon_head_logprobs(h[3:4].contiguous() if rows == 4 else h, w, None)
    kept = torch.cat([w[:8], w[9:]]).contiguous()
    want = binding.solon_head_logprobs(h[3:4].contiguous() if rows == 4 else h, kept, None)
    for x, y in ((row.peak, want.peak), (row.log_sum, want.log_sum), (row.entropy, want.entropy)):
        assert abs(float(x[at]) - float(y[at])) <= 1e-5 * max(1.0, abs(float(y[at])))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_scales(dtype):
    """Tensors of very small or very large elements, and tiny gradients: pieces and dlogits carry powers of two."""
    for hs, ws, gs in ((1e-3, 1e3, 1e-6), (2e-6, 4e4, 1.0), (1e3, 1e-3, 1e-12), (3e4, 1e-4, 100.0)) if dtype == "f16" else \
            ((1e-20, 1e20, 1e-12), (1e15, 1e-15, 1e10), (1.0, 1.0, 1e-30)):
        h, w, t = _inputs(200, 64, 300, "f32", 8)
        h, w = (h * hs).to(TYPES[dtype]), (w * ws).to(TYPES[dtype])
        got = binding.solon_head_logprobs(h, w, t)
        _check_forward(h, w, t, got)
        peak, log_sum, entropy = _stats(h, w)
        g = -torch.rand(200, device="cuda", generator=_gen(3)) * gs
        dh, dw = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, partitions=2)
        if dtype == "f16" and not torch.isfinite(dh).all():
            continue                                              # beyond float16's range
        _check_backward(h, w, t, peak, log_sum, g, None, None, 2, dh, dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_agrees_with_the_logits_in_memory(dtype):
    """The same as the two calls with the logits between them, to what those are rounded to."""
    rows, cols, vocab = 400, 256, 3000
    h, w, t = _inputs(rows, cols, vocab, dtype, 4)
    z = (h.double() @ w.double().t()).float()
    want = binding.solon_token_logprobs(z, t)
    got = binding.solon_head_logprobs(h, w, t)
    for x, y in zip(got[:4], want[:4]):
        assert float((x - y).abs().max()) <= 2e-5
    g = -torch.rand(rows, device="cuda", generator=_gen(2)) / rows
    dz = binding.solon_token_logprobs_backward(z, t, want.peak, want.log_sum, g).double()
    dh, dw = binding.solon_head_logprobs_backward(h, w, t, got.peak, got.log_sum, g)
    limit = 2e-5 if dtype == "f32" else 2.0 ** -7
    for x, y, lim in ((dh, dz @ w.double(), limit), (dw.view(vocab, cols), dz.t() @ h.double(), 2e-5)):
        assert float((x.double() - y).norm()) <= lim * float(y.norm())


def test_differences():
    """The gradient against central differences of the value, in float32 elements: an element moved by +-e changes sum(g logp + g_H entropy) by
    2 e times its gradient, up to e^3 / 3 of a third derivative of order 1 and the values' rounding, 1e-5 / e here."""
    h, w, t = _inputs(20, 24, 60, "f32", 6)
    g, gh = torch.randn(20, device="cuda", generator=_gen(1)), torch.randn(20, device="cuda", generator=_gen(2)) * 0.3
    got = binding.solon_head_logprobs(h, w, t)
    dh, dw = binding.solon_head_logprobs_backward(h, w, t, got.peak, got.log_sum, g, got.entropy, gh)
    e = 2.0 ** -6

    def value():
        r = binding.solon_head_logprobs(h, w, t)
        return float((g.double() * r.logp.double() + gh.double() * r.entropy.double()).sum())

    for x, grad, at in ((h, dh, (3, 5)), (h, dh, (19, 23)), (w, dw.view(60, 24), (int(t[0]), 2)), (w, dw.view(60, 24), (59, 0))):
        was = float(x[at])
        x[at] = was + e
        up = value()
        x[at] = was - e
        down = value()
        x[at] = was
        assert abs((up - down) / (2 * e) - float(grad[at])) <= 3e-3 * (1 + abs(float(grad[at])))


def test_on_a_stream_and_in_graphs():
    for dtype, rows in (("bf16", 300), ("f32", 300), ("bf16", 2)):
        h, w, t = _inputs(rows, 96, 700, dtype, 9)
        g = torch.full((rows,), -1.0 / rows, device="cuda")
        want = binding.solon_head_logprobs(h, w, t)
        want_dh, want_dw = binding.solon_head_logprobs_backward(h, w, t, want.peak, want.log_sum, g)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = binding.solon_head_logprobs(h, w, t)
            dh, dw = binding.solon_head_logprobs_backward(h, w, t, got.peak, got.log_sum, g)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got.logp, want.logp) and torch.equal(dh, want_dh) and torch.equal(dw, want_dw)
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                r = binding.solon_head_logprobs(h, w, t)
                out = binding.solon_head_logprobs_backward(h, w, t, r.peak, r.log_sum, g)
            graphs.append((graph, r, out))
        h.copy_(h.flip(0))
        t.copy_(t.flip(0))
        want = binding.solon_head_logprobs(h, w, t)
        want_dh, want_dw = binding.solon_head_logprobs_backward(h, w, t, want.peak, want.log_sum, g)
        for graph, r, out in graphs + graphs[::-1]:
            graph.replay()
            assert torch.equal(r.logp, want.logp) and torch.equal(out[0], want_dh) and torch.equal(out[1], want_dw)


def test_two_calls_at_once():
    """Products that each want every SM, on two streams: they may run one after the other or side by side."""
    h, w, t = _inputs(2000, 256, 6000, "bf16", 1)
    g = torch.full((2000,), -1.0 / 2000, device="cuda")
    want = binding.solon_head_logprobs(h, w, t)
    want_dh, want_dw = binding.solon_head_logprobs_backward(h, w, t, want.peak, want.log_sum, g, partitions=4)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                r = binding.solon_head_logprobs(h, w, t)
                got.append((r, *binding.solon_head_logprobs_backward(h, w, t, r.peak, r.log_sum, g, partitions=4)))
    torch.cuda.synchronize()
    for r, dh, dw in got:
        assert torch.equal(r.logp, want.logp) and torch.equal(dh, want_dh) and torch.equal(dw, want_dw)


def test_offsets_beyond_32_bits():
    """Gradient rows that start beyond 2^31 elements, an output matrix whose last rows do, too (in bytes)."""
    parts, n, cols, vocab = 3, 2, 8192, 140_000
    g = _gen(1)
    h = torch.randn((parts * n, cols), device="cuda", generator=g).bfloat16()
    w = torch.empty((vocab, cols), dtype=torch.bfloat16, device="cuda").normal_(0.0, cols ** -0.5, generator=g)
    t = torch.tensor([vocab - 1, 0, 5, vocab - 2, 70_000, -1], device="cuda")
    z = (h.float() @ w.float().t()).double()
    lp = torch.log_softmax(z, 1)
    got = binding.solon_head_logprobs(h, w, t)
    assert float((got.logp[:5].double() - lp[torch.arange(5), t[:5]]).abs().max()) <= 1e-4
    grad = torch.full((parts * n,), -1.0, device="cuda")
    dw = torch.full((parts, vocab * cols), 9.0, dtype=torch.bfloat16, device="cuda")
    binding.solon_head_logprobs_backward(h, w, t, got.peak, got.log_sum, grad, partitions=parts, hidden_grad=False, dweight=dw)
    dz = lp.exp()
    dz[torch.arange(5), t[:5]] -= 1.0
    dz[5] = 0.0
    for k in range(parts):
        at = torch.tensor([0, 5, 65_535, 65_536, 70_000, vocab - 2, vocab - 1], device="cuda")
        want = dz[k * n:(k + 1) * n, at].t() @ h[k * n:(k + 1) * n].double()
        size = dz[k * n:(k + 1) * n, at].abs().t() @ h[k * n:(k + 1) * n].double().abs()
        # half a bfloat16 step of each dlogit and of the result, and a logit's 1e-4 in p
        assert ((dw[k].view(vocab, cols)[at].double() - want).abs() <= (2.0 ** -8 + 2e-4) * size + 2.0 ** -8 * want.abs()).all()
        assert float((dw[k] == 9.0).float().mean()) < 1e-3


def test_refusals():
    h, w = torch.zeros((4, 8), device="cuda"), torch.zeros((10, 8), device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    v = torch.zeros(4, device="cuda")
    with pytest.raises(ValueError):
        binding.solon_head_logprobs(h, w.bfloat16(), t)
    with pytest.raises(ValueError):
        binding.solon_head_logprobs(h, w[:, :7], t)
    with pytest.raises(binding.SolonError):
        binding.solon_head_logprobs(h.double(), w.double(), t)
    with pytest.raises(ValueError):
        binding.solon_head_logprobs(h, w, t.int())
    with pytest.raises(ValueError):
        binding.solon_head_logprobs_backward(h, w, t, v, v[:3], v)
    with pytest.raises(binding.SolonError):
        binding.solon_head_logprobs_backward(h, w, None, v, v, v)
    with pytest.raises(binding.SolonError):
        binding.solon_head_logprobs_backward(h, w, t, v, v, v, None, v)
    with pytest.raises(binding.SolonError):
        binding.solon_head_logprobs_backward(h, w, t, v, v, v, partitions=3)
    with pytest.raises(ValueError):
        binding.solon_head_logprobs_backward(h, w, t, v, v, v, partitions=2, dweight=torch.zeros((1, 80), device="cuda"))
    with pytest.raises(binding.SolonError):
        binding.solon_head_logprobs_backward(h, w, t, v, v, v, dweight=torch.zeros((1, 80), dtype=torch.float16, device="cuda"))
    empty = binding.solon_head_logprobs(h[:0], w, t[:0])
    assert empty.logp.shape == (0,)
    dh, dw = binding.solon_head_logprobs_backward(h[:0], w, t[:0], v[:0], v[:0], v[:0], partitions=2)
    assert dh.shape == (0, 8) and (dw == 0).all()
