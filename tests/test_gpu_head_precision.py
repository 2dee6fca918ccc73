"""What the head's results may be off by, element by element, where 16-bit results, ranges of magnitudes and neighbouring rows test it.

Tolerances as in test_gpu_head.py (u = 2^-24, s_iv = sum_c |h_ic w_vc|, a logit's z_tol, the gradient's dz_tol from it), with what dlogits and float32 elements are held in:
one float16 piece is off by half a step, 2^-11 of a value, two by half a step of what the first leaves, 2^-22."""

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


def _leaning(rows, cols, vocab, dtype, seed, lean=6.0):
    """Hidden states that lean to their targets, more or less so: of some rows a few tokens carry dlogits."""
    g = _gen(seed)
    w = torch.randn((vocab, cols), device="cuda", generator=g) * (1.5 * cols ** -0.5)
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    h = torch.randn((rows, cols), device="cuda", generator=g) + w[t] * (torch.rand((rows, 1), device="cuda", generator=g) * lean)
    return h.to(TYPES[dtype]), w.to(TYPES[dtype]), t


def _size(x):
    return x.double().abs().clamp(min=2.0 ** -14) if x.dtype == torch.float16 else x.double().abs()


def _logits(h, w):
    z, s = h.double() @ w.double().t(), _size(h) @ _size(w).t()
    return z, (64 + h.shape[1] / 256 + h.shape[1] / 32 + 8) * U * s + (2.0 ** -20 * s if h.dtype == torch.float32 else 0.0)


def _stats(h, w):
    z = h.double() @ w.double().t()
    big = z.amax(1)
    lp = torch.log_softmax(z, 1)
    return big.float(), (torch.logsumexp(z, 1) - big).float(), (-torch.special.xlogy(lp.exp(), lp.exp()).sum(1)).float()


def _dlogits(h, w, t, peak, log_sum, g, entropy=None, gh=None):
    """dlogits and what they may be off by before any rounding to pieces."""
    z, zt = _logits(h, w)
    lp = z - peak.double()[:, None] - log_sum.double()[:, None]
    p = lp.exp()
    ga = torch.where(t >= 0, g.double(), 0.0)
    gha = torch.zeros_like(ga) if gh is None else gh.double()
    ent = torch.zeros_like(ga) if gh is None else entropy.double()
    inner = ga[:, None] + gha[:, None] * (lp + ent[:, None])
    dz = (-p * inner).scatter_add(1, t.clamp(min=0)[:, None], ga[:, None])
    r = (4 * lp.abs() + 8) * U + zt
    tol = p * inner.abs() * (r + 4 * U) + p * gha.abs()[:, None] * (zt + 4 * U * (lp.abs() + ent.abs()[:, None])) + 2 * U * dz.abs()
    return dz, tol * 1.01 + 2.0 ** -125 * (ga.abs() + gha.abs())[:, None]


def _close(x, y, tol, what):
    x = x.double()
    off = (x - y).abs()
    bad = ~((x == y) | (off <= tol))
    assert not bad.any(), (what, int(bad.sum()), float((off / tol.clamp(min=1e-300))[bad].max()), x[bad][:4], y[bad][:4])


@pytest.mark.parametrize("dtype,grad", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,parts,cols,vocab", [(300, 2, 128, 400), (2, 1, 72, 1000), (512, 4, 65, 700), (1000, 1, 333, 517)])
def test_sixteen_bit_results_are_off_by_little_more_than_their_own_rounding(rows, parts, cols, vocab, dtype, grad):
    """Half a step of the result, and what dlogits are held in: one float16 piece for dh of bfloat16 states and for bfloat16 gradients (2^-11 of a term, and as
    much again for float32 states, of which these take one piece too), two elsewhere (2^-22); 2^-39 of the largest for what float16 does not reach, of dlogits and of
    bfloat16 states and weights as float16."""
    n = rows // parts
    for entropies in (False, True):
        h, w, t = _leaning(rows, cols, vocab, dtype, rows + cols)
        t[::7] = -1
        peak, log_sum, entropy = _stats(h, w)
        g = -torch.rand(rows, device="cuda", generator=_gen(1)) / n
        gh = torch.randn(rows, device="cuda", generator=_gen(2)) / (4 * n) if entropies else None
        dw = torch.empty((parts, vocab * cols), dtype=TYPES[grad], device="cuda")
        dh, _ = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, entropy, gh, partitions=parts, dweight=dw)
        dz, dzt = _dlogits(h, w, t, peak, log_sum, g, entropy, gh)
        bound = float((g.abs() + (gh.abs() * (entropy + 1) if entropies else 0.0)).max())

        def check(result, a, atol, factor, held, inner, what):
            b = factor.double()
            x, size = a @ b, a.abs() @ b.abs()
            c = 1040 + inner / 4096 if result.element_size() == 2 else 64 + inner / 256
            tol = atol @ b.abs() + held * size + c * U * (a.abs() @ _size(factor)) + 2.0 ** -39 * (bound * b.abs().sum(0) + b.abs().max() * a.abs().sum(1)[:, None])
            tol = tol + torch.finfo(result.dtype).eps / 2 * x.abs() + (2.0 ** -25 if result.dtype == torch.float16 else 0.0)
            _close(result, x, tol, what)

        pair = 2.0 ** -22 if dtype != "f32" else 2.0 ** -20
        check(dh, dz, dzt, w, 2.0 ** -11 if dtype == "bf16" else pair, vocab, "dhidden")
        one = 2.0 ** -11 if dtype != "f32" else 2.0 ** -10
        for k in range(parts):
            q = slice(k * n, (k + 1) * n)
            check(dw[k].view(vocab, cols), dz[q].t(), dzt[q].t(), h[q], one if grad == "bf16" else pair, n, f"dweight {k}")


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f32", "bf16"), ("f16", "f32"), ("bf16", "f32"), ("bf16", "f64"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows", [8, 300])
def test_rows_without_a_share_say_nothing_about_the_others(rows, dtype, grad):
    """What stands in grad_logp of a row without target, or in either factor of a row of which nothing is left, counts nowhere: the same bits as with zeros there."""
    cols, vocab, parts = 72, 19_000 if rows == 8 else 700, 2
    h, w, t = _leaning(rows, cols, vocab, dtype, 3)
    t[1::5] = -1
    peak, log_sum, entropy = _stats(h, w)
    peak[2::9] = -INF
    g, gh = -torch.rand(rows, device="cuda", generator=_gen(1)), torch.randn(rows, device="cuda", generator=_gen(2)) / 8
    g[1::5], g[2::9], gh[2::9] = 0.0, 0.0, 0.0

    def call():
        dw = torch.empty((parts, vocab * cols), dtype=TYPES[grad], device="cuda")
        return binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, entropy, gh, partitions=parts, dweight=dw)

    want = call()
    assert float(want[0].abs().max()) > 0
    g[1::5], g[2::9], gh[2::9] = 1e12, -3e20, 1e30
    got = call()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g[1::5], g[2::9], gh[2::9] = NAN, INF, NAN
    got = call()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rows", [3, 20, 100, 300])
def test_float32_elements_far_below_the_largest_of_their_row(rows):
    """A row whose largest element meets zeros in the output matrix: its other elements, 2^-26 of that, keep their 22 bits (and 2^-50 of the
    largest: 2^-24 of a weight each)."""
    cols, vocab = 80, 500
    h, w, t = _leaning(rows, cols, vocab, "f32", 4, 1.0)
    h[:, 1:] *= 2.0 ** -26
    h[:, 0] = 1.0
    w[:, 1:] *= 2.0 ** 26
    w[:, 0] = 0.0
    z, tol = _logits(h, w)
    floor = 2.0 ** -50 * float(w.abs().sum(1).max())
    got = binding.solon_head_logprobs(h, w, t)
    _close(got.peak, z.amax(1), tol.amax(1) + floor, "peak")
    # a token of its own in every row, so that log p says what a single logit is
    lp = torch.log_softmax(z, 1).gather(1, t[:, None])[:, 0]
    _close(got.logp, lp, 2 * (tol.amax(1) + floor) + 100 * U * (1 + lp.abs()), "logp")


@pytest.mark.parametrize("rows", [5, 300, 513])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradients_of_rare_tokens_keep_their_bits(dtype, rows):
    """Logits that fall from token to token down to p = 2^-36: dW of each is -g p h, two pieces 2^-22 of it and 2^-50 of g h at most, next to what p is off by."""
    cols, vocab = 64, 512
    g = _gen(6)
    h = torch.randn((rows, cols), device="cuda", generator=g) * 0.25
    h[:, 0] = 1.0
    w = torch.zeros((vocab, cols), device="cuda")
    w[:, 0] = -torch.arange(vocab, device="cuda") * (25.0 / vocab)
    h, w = h.to(TYPES[dtype]), w.to(TYPES[dtype])
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    peak, log_sum, _ = _stats(h, w)
    gl = -torch.rand(rows, device="cuda", generator=g)
    _, dw = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, gl, hidden_grad=False)
    dz, dzt = _dlogits(h, w, t, peak, log_sum, gl)
    b = h.double()
    size = dz.abs().t() @ b.abs()
    tol = dzt.t() @ b.abs() + (2.0 ** -20 + 66 * U) * size + 2.0 ** -49 * float(gl.abs().max()) * b.abs().sum(0)
    if dtype == "f16":
        tol = tol + 64 * U * (dz.abs().t() @ _size(h))
    _close(dw.view(vocab, cols), dz.t() @ b, tol, "dweight")


@pytest.mark.parametrize("rows,vocab", [(3, 700), (12, 700), (24, 19_000), (40, 700), (300, 700), (512, 701), (513, 701), (700, 300)])
def test_a_large_row_or_token_leaves_the_others_alone(rows, vocab):
    """Every logit is off by what its own row's and token's elements come to, whatever the size of their neighbours."""
    cols = 64
    h, w, t = _leaning(rows, cols, vocab, "f32", 9, 2.0)
    w[:, 0] = 0.0
    h[:, 0] = -1.0
    t = t.clamp(min=6)
    for what in ("row", "token"):
        a, b = h.clone(), w.clone()
        if what == "row":
            a[1] *= 1e12
        else:
            b[5, 0] = 1e12                                        # a logit of -1e12 in every row
        others = torch.arange(rows, device="cuda") != (1 if what == "row" else -1)
        z, tol = _logits(a, b)
        tokens = torch.arange(vocab, device="cuda") != (-1 if what == "row" else 5)
        most = tol[:, tokens].amax(1)[others]
        got = binding.solon_head_logprobs(a, b, t)
        _close(got.peak[others], z.amax(1)[others], most + U * z.amax(1)[others].abs(), "peak")
        lp = torch.log_softmax(z, 1).gather(1, t[:, None])[:, 0][others]
        _close(got.logp[others], lp, 2 * most + 200 * U * (1 + lp.abs()), "logp")
        # and in the backward pass
        peak, log_sum, _ = _stats(a, b)
        g = -torch.rand(rows, device="cuda", generator=_gen(1))
        dh, _ = binding.solon_head_logprobs_backward(a, b, t, peak, log_sum, g, weight_grad=False)
        dz, dzt = _dlogits(a, b, t, peak, log_sum, g)
        wd = b.double()
        size = dz.abs() @ wd.abs()
        dtol = dzt @ wd.abs() + (2.0 ** -20 + (64 + vocab / 256) * U) * size + 2.0 ** -49 * (g.double().abs()[:, None] * wd.abs().sum(0) + wd.abs().max() * dz.abs().sum(1)[:, None])
        _close(dh[others], (dz @ wd)[others], dtol[others], "dhidden")


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f16", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n", [4, 150])
def test_partitions_are_independent(n, dtype, grad):
    """Hidden states and factors of one partition, however large, change no bit of what the others get; nor does a row's factor change another row's dh."""
    parts, cols, vocab = 3, 72, 19_000 if n == 4 else 500
    rows = n * parts
    h, w, t = _leaning(rows, cols, vocab, dtype, 2)
    peak, log_sum, _ = _stats(h, w)
    g = -torch.rand(rows, device="cuda", generator=_gen(1))

    def call():
        dw = torch.empty((parts, vocab * cols), dtype=TYPES[grad], device="cuda")
        return binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, partitions=parts, dweight=dw)

    dh, dw = call()
    h[n:2 * n] *= 1e3 if dtype == "f16" else 1e10
    g[n:2 * n] *= 1e9
    peak[n:2 * n], log_sum[n:2 * n] = (s[n:2 * n] for s in _stats(h, w)[:2])
    other_dh, other_dw = call()
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[n:2 * n] = False
    assert torch.equal(other_dh[keep], dh[keep]) and torch.equal(other_dw[0], dw[0]) and torch.equal(other_dw[2], dw[2])
    g[0] *= 1e9
    last = call()[0]
    keep[0] = False
    assert torch.equal(last[keep], dh[keep])


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f16", "f64"), ("bf16", "f32"), ("bf16", "bf16")])
def test_rows_of_zeros_and_partitions_without_a_share(dtype, grad):
    """Hidden states of zeros beside tiny and large factors, a partition of such rows alone, one without a target: zeros, and the others as they are."""
    n, parts, cols, vocab = 40, 4, 64, 300
    rows = n * parts
    h, w, t = _leaning(rows, cols, vocab, dtype, 7, 2.0)
    h[3] = 0.0
    h[n:2 * n] = 0.0
    t[2 * n:3 * n] = -1
    g = -torch.rand(rows, device="cuda", generator=_gen(1))
    g[3] = 1e-36
    g[n:2 * n:2] = 1e-30
    g[0] = -1e6
    h[1] *= 2.0 ** -10
    peak, log_sum, _ = _stats(h, w)
    dw = torch.full((parts, vocab * cols), 7.0, dtype=TYPES[grad], device="cuda")
    dh, _ = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, partitions=parts, dweight=dw)
    assert torch.isfinite(dw).all()
    assert (dw[1:3] == 0).all() and (dh[2 * n:3 * n] == 0).all()
    dz, _ = _dlogits(h, w, t, peak, log_sum, g)
    for k in (0, 3):
        want = (dz[k * n:(k + 1) * n].t() @ h[k * n:(k + 1) * n].double()).reshape(-1)
        assert float((dw[k].double() - want).norm()) <= (2.0 ** -8 if grad == "bf16" else 1e-5) * float(want.norm())
    want = dz @ w.double()
    # the factor of 1e6 brings row 0 of dh to 1e6 |w| of some 2e5: beyond float16 (65504), where infinity is the nearest
    most = torch.finfo(dh.dtype).max
    assert torch.isfinite(dh)[want.abs() < most * (1 - 2.0 ** -8)].all()
    some = (want.abs().amax(1) > 0) & (want.abs().amax(1) < most * (1 - 2.0 ** -8))
    assert ((dh.double() - want).norm(dim=1)[some] <= (1e-5 if dtype == "f32" else 2.0 ** -8) * want.norm(dim=1)[some] + (2.0 ** -20 if dtype == "f16" else 0.0)).all()


@pytest.mark.parametrize("rows,vocab", [(1, 700), (3, 700), (20, 19_000), (40, 700), (300, 700)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_huge_finite_logits(rows, vocab, dtype):
    """Logits of -3e37 beside ordinary ones: tokens with p = 0, no NaN (their number times their distance is beyond float32)."""
    cols = 40
    h, w, t = _leaning(rows, cols, vocab, dtype, 5, 1.0)
    w[:, 0] = 0.0
    h[:, 0] = 1.0
    keep = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    keep[::300] = True                                            # tiles with and without an ordinary token
    w[~keep, 0] = -3e37
    got = binding.solon_head_logprobs(h, w, None)
    z, tol = _logits(h, w[keep])
    lp = torch.log_softmax(z, 1)
    most = tol.amax(1)
    _close(got.peak, z.amax(1), most + U * z.amax(1).abs(), "peak")
    _close(got.log_sum, torch.logsumexp(z, 1) - z.amax(1), 2 * most + 200 * U, "log_sum")
    _close(got.entropy, -(lp.exp() * lp).sum(1), 20 * most + 1000 * U, "entropy")
    # gradients: none from those tokens, with entropy factors too
    g, gh = torch.full((rows,), -0.5, device="cuda"), torch.full((rows,), 0.25, device="cuda")
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    t[-1] = 1                                                     # a target with p = 0
    _, dw = binding.solon_head_logprobs_backward(h, w, t, got.peak, got.log_sum, g, got.entropy, gh, hidden_grad=False)
    dw = dw.view(vocab, cols)
    assert torch.isfinite(dw).all()
    gone = ~keep
    gone[1] = False
    assert (dw[gone] == 0).all()
    _close(dw[1], -0.5 * h[-1].double(), 2.0 ** -20 * h[-1].double().abs(), "a target of p = 0")


@pytest.mark.parametrize("rows", [2, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_masked_token_as_the_target(rows, dtype):
    """A token masked by -infinity that is a row's target all the same: log p is -infinity, dz = g there."""
    cols, vocab = 64, 500
    h, w, t = _leaning(rows, cols, vocab, dtype, 8, 1.0)
    h[:] = h.abs() + 0.5
    w[7] = -INF
    t[:] = 7
    got = binding.solon_head_logprobs(h, w, t)
    assert (got.logp == -INF).all() and torch.isfinite(got.log_sum).all() and torch.isfinite(got.entropy).all()
    g = torch.full((rows,), -0.5, device="cuda")
    for entropy, gh in ((None, None), (got.entropy, torch.zeros(rows, device="cuda")), (got.entropy, torch.full((rows,), 0.125, device="cuda"))):
        _, dw = binding.solon_head_logprobs_backward(h, w, t, got.peak, got.log_sum, g, entropy, gh, hidden_grad=False)
        x = -0.5 * h.double().sum(0)
        _close(dw.view(vocab, cols)[7], x, 2.0 ** -18 * x.abs(), "dweight")
        assert torch.isfinite(dw).all()


def test_health():
    """No wait has run out in any call of this process (one that had would have left NaN where its results belong, and this said so)."""
    h, w, t = _leaning(300, 64, 700, "bf16", 1)
    r = binding.solon_head_logprobs(h, w, t)
    binding.solon_head_logprobs_backward(h, w, t, r.peak, r.log_sum, torch.full((300,), -1.0, device="cuda"))
    assert binding.solon_head_status() == binding.OK


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f32", "bf16"), ("f16", "f32"), ("bf16", "f64"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,vocab", [(8, 19_000), (16, 700), (300, 700)])
def test_hidden_states_of_rows_without_a_share_may_hold_anything(rows, vocab, dtype, grad):
    """NaN and infinity where padding stands: the same bits as with numbers there."""
    cols, parts = 72, 2
    h, w, t = _leaning(rows, cols, vocab, dtype, 3)
    t[1::4] = -1
    peak, log_sum, entropy = _stats(h, w)
    peak[2] = -INF
    g, gh = -torch.rand(rows, device="cuda", generator=_gen(1)), torch.randn(rows, device="cuda", generator=_gen(2)) / 8
    gh[1::4] = 0.0

    def call():
        dw = torch.empty((parts, vocab * cols), dtype=TYPES[grad], device="cuda")
        return binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, entropy, gh, partitions=parts, dweight=dw)

    want = call()
    h[1::4, ::3], h[1::4, 1::3], h[2] = NAN, INF, -INF
    log_sum[1::4], entropy[1::4], log_sum[2] = NAN, NAN, INF
    got = call()
    assert torch.isfinite(want[1]).all() and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rows,vocab,pieces", [(4, 5000, False), (5, 5000, True), (8, 5000, True), (8, 19_000, False), (32, 18_944, False), (33, 18_944, True)])
def test_where_infinity_in_float32_is_a_mask(rows, vocab, pieces):
    """Up to 4 rows, and up to 32 from 18,944 tokens on, elements are multiplied as they are: -infinity masks a token. In two pieces its products have no sum."""
    cols = 48
    h, w, t = _leaning(rows, cols, vocab, "f32", 8, 1.0)
    h[:] = h.abs() + 0.5
    w[7] = -INF
    t[:] = 8
    got = binding.solon_head_logprobs(h, w, t)
    if pieces:
        assert got.peak.isnan().all() and got.logp.isnan().all()
    else:
        want = torch.log_softmax((h.double() @ w.double().t()), 1)[:, 8]
        assert torch.isfinite(got.log_sum).all() and float((got.logp.double() - want).abs().max()) <= 1e-4


@pytest.mark.parametrize("dtype,rows,parts,cols,vocab", [("f32", 2880, 45, 333, 2003), ("f32", 16, 4, 768, 2134), ("f32", 332, 1, 163, 1536), ("bf16", 17, 1, 278, 4352),
                                                         ("bf16", 473, 43, 640, 18_048), ("f16", 92, 4, 128, 30_001)])
def test_float32_gradients_are_as_near_as_elementary_float32_operations(dtype, rows, parts, cols, vocab):
    """Of rows that lean to their targets the logits are 10 and more, so an error of theirs, a relative one of p, is what the gradient's is made of. Elementary
    operations round each sum at random; the tensor cores cut off towards 0, which adds up over the steps between two sums in registers, and two pieces leave
    2^-22 of an element. 2.5 times the error of elementary operations, by norms, holds both."""
    h, w, t = _leaning(rows, cols, vocab, dtype, 12, 4.0)
    peak, log_sum, entropy = _stats(h, w)
    n = rows // parts
    g, gh = -torch.rand(rows, device="cuda", generator=_gen(1)) / n, torch.randn(rows, device="cuda", generator=_gen(2)) / (8 * n)
    dh, dw = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, entropy, gh, partitions=parts)

    def plain(f):
        a, b = h.to(f), w.to(f)
        lp = a @ b.t() - peak.to(f)[:, None] - log_sum.to(f)[:, None]
        p = lp.exp()
        dz = -p * (g.to(f)[:, None] + gh.to(f)[:, None] * (lp + entropy.to(f)[:, None]))
        dz.scatter_add_(1, t[:, None], g.to(f)[:, None])
        return dz @ b, torch.bmm(dz.view(parts, n, vocab).transpose(1, 2), a.view(parts, n, cols)).view(parts, -1)

    exact, elementary = plain(torch.float64), plain(torch.float32)
    for x, y, e, name in ((dh, elementary[0], exact[0], "dhidden"), (dw, elementary[1], exact[1], "dweight")):
        if x.dtype == torch.float32:
            assert float((x.double() - e).norm()) <= 2.5 * float((y.double() - e).norm()), name


@pytest.mark.parametrize("rows", [40, 512, 513])
def test_weights_of_zeros_and_of_very_different_sizes(rows):
    """Tokens whose weights are zeros, 2^-60 and 2^60 of the others: float32 dh beside dW and alone, with the same bits."""
    cols, vocab = 72, 333                                         # (not a whole block of tokens)
    h, w, t = _leaning(rows, cols, vocab, "f32", 11, 1.0)
    h[:, 0] = -h[:, 0].abs() - 0.5
    w[3] = 0.0
    w[4] *= 2.0 ** -60
    w[vocab - 1] = 0.0
    w[5], w[5, 0] = 0.0, 2.0 ** 60                                # p = 0
    t[:4] = torch.tensor([3, 4, vocab - 1, 6], device="cuda")
    peak, log_sum, entropy = _stats(h, w)
    g, gh = -torch.rand(rows, device="cuda", generator=_gen(1)), torch.randn(rows, device="cuda", generator=_gen(2)) / 8
    dh, dw = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, entropy, gh)
    alone, _ = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, entropy, gh, weight_grad=False)
    _, dw_alone = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, entropy, gh, hidden_grad=False)
    assert torch.equal(alone, dh) and torch.equal(dw_alone, dw)
    dz, dzt = _dlogits(h, w, t, peak, log_sum, g, entropy, gh)
    dz[:, 5], dzt[:, 5] = 0.0, 0.0
    bound = (g.abs() + gh.abs() * (entropy + 1)).double()
    hd, wd = h.double(), w.double()
    size = dz.abs().t() @ hd.abs()
    tol = dzt.t() @ hd.abs() + (2.0 ** -20 + 66 * U) * size + 2.0 ** -49 * float((bound * hd.abs().amax(1)).max()) * rows
    _close(dw.view(vocab, cols), dz.t() @ hd, tol, "dweight")
    size = dz.abs() @ wd.abs()
    # of dz or the weights, whichever is below 2^-28 of its largest: an absolute 2^-50 of it; here of the weights of 2^60
    tol = dzt @ wd.abs() + (2.0 ** -20 + 66 * U) * size + 2.0 ** -49 * bound[:, None] * 2.0 ** 60 * 1.5
    _close(dh, dz @ wd, tol, "dhidden")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 40, 200, 600])
@pytest.mark.parametrize("hs,ws,gs", [(1e34, 1e-34, 1e3), (1e-34, 1e34, 1.0), (1e20, 1e-20, 1e33), (1.0, 1e-30, 1e37), (1.0, 1.0, 1e-34)])
def test_powers_of_two_near_the_ends_of_float32(hs, ws, gs, rows, dtype):
    """Products of ordinary size from factors of any: what undoes one factor's power of two alone would be infinite, or zero. By norms: 2^-20 for float32 and
    its gradients, half a bfloat16 step beside it for dh of bfloat16 states; ten times that where the logits' own error is part of it."""
    cols, vocab = 64, 300
    h, w, t = _leaning(rows, cols, vocab, "f32", 10, 1.0)
    h, w = (h * hs).to(TYPES[dtype]), (w * ws).to(TYPES[dtype])
    z = h.double() @ w.double().t()
    got = binding.solon_head_logprobs(h, w, t)
    assert float((got.peak.double() - z.amax(1)).abs().max()) <= 1e-5 * (1 + float(z.abs().max()))
    assert float((got.logp.double() - torch.log_softmax(z, 1).gather(1, t[:, None])[:, 0]).abs().max()) <= 2e-5 * (1 + float(z.abs().max()))
    peak, log_sum, _ = _stats(h, w)
    g = -torch.rand(rows, device="cuda", generator=_gen(3)) * gs
    dh, dw = binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g)
    dz, _ = _dlogits(h, w, t, peak, log_sum, g)
    most = torch.finfo(torch.float32).max
    for x, e, lim in ((dh, dz @ w.double(), 1e-5 if dtype == "f32" else 2.0 ** -8), (dw.view(vocab, cols), dz.t() @ h.double(), 1e-5)):
        if float(e.abs().max()) < most and float(e.abs().max()) > 2.0 ** -110:
            assert float((x.double() - e).norm()) <= lim * float(e.norm())


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f32", "bf16"), ("f16", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols,vocab", [(20, 8200, 130), (600, 9001, 70), (514, 64, 20_000)])
def test_wide_rows_and_a_graph_of_their_gradient(rows, cols, vocab, dtype, grad):
    """Rows that a whole CTA goes through; the backward pass captured and replayed on other inputs gives the bits of a call."""
    parts = 2
    h, w, t = _leaning(rows, cols, vocab, dtype, 13, 2.0)
    peak, log_sum, _ = _stats(h, w)
    g = -torch.rand(rows, device="cuda", generator=_gen(1)) / rows
    dw = torch.empty((parts, vocab * cols), dtype=TYPES[grad], device="cuda")

    def call():
        return binding.solon_head_logprobs_backward(h, w, t, peak, log_sum, g, partitions=parts, dweight=dw)

    dh = call()[0]
    n = rows // parts
    dz, _ = _dlogits(h, w, t, peak, log_sum, g)
    lim = {"f32": 1e-5, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
    e = dz @ w.double()
    assert float((dh.double() - e).norm()) <= (lim[dtype] + 1e-5) * float(e.norm()) + (2.0 ** -25 * e.numel() ** 0.5 if dtype == "f16" else 0.0)
    for k in range(parts):
        e = (dz[k * n:(k + 1) * n].t() @ h[k * n:(k + 1) * n].double()).reshape(-1)
        assert float((dw[k].double() - e).norm()) <= (1e-5 + (2.0 ** -8 if grad == "bf16" else 0.0)) * float(e.norm())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()[0]
    h.copy_(h.flip(0)), t.copy_(t.flip(0)), g.mul_(1e-6)
    g[0] = 3.0
    fresh = _stats(h, w)
    peak.copy_(fresh[0]), log_sum.copy_(fresh[1])
    for _ in range(2):
        graph.replay()
    got, got_w = out.clone(), dw.clone()
    assert torch.equal(got, call()[0]) and torch.equal(got_w, dw)
