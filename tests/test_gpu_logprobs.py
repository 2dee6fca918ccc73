"""Token log probabilities, entropy, likeliest tokens and the gradient, against the formulas in float64 and against differences.

Tolerances (u = 2^-24).  A term e^(z - M) carries a relative error of (2 |z - M| + 4) u; a thread adds at most cols / 256 + 32 of
them (where a warp has the row, cols / 64, whose rounding errors, of independent sign, stay below the same number) and the threads'
sums are joined over at most 40 more roundings.  With k = cols / 256 + 72 and D = E|z - M| + 4 under the softmax:
log S is off by (k + 2 D) u + 2 u |log S|, logp = (z_t - M) - log S by 2 u (|z_t - M| + |log S|) more, and the entropy, a difference of log S and A / S, by
(2 k + 4 D) u (1 + |log S| + E|z - M| + E|z - M|^2).  In the gradient, whose M, log S and entropy are inputs, p is off by a
relative (4 |log p| + 6) u, log p itself by 2 u (|z - M| + |log S|) and each product by 4 u more; then the element type's rounding."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": (torch.float32, 2.0 ** -23), "bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -10)}
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _logits(rows, cols, dtype, seed, scale=3.0, masked=0.0, pitch=None, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((rows, cols), device="cuda", generator=g) * scale
    if masked:
        z[torch.rand((rows, cols), device="cuda", generator=g) < masked] = -INF
    z = z.to(TYPES[dtype][0])
    if pitch is not None:
        buf = torch.full((offset + rows * pitch,), 99.0, dtype=z.dtype, device="cuda")
        view = buf[offset:].view(rows, pitch)[:, :cols]
        view.copy_(z)
        z = view
    targets = torch.randint(0, cols, (rows,), device="cuda", generator=g)
    return z, targets


def _top_ref(z, k):
    """Largest first, of equal ones the lower index first, NaN above all: a stable sort of the negated order."""
    z = z.float() + 0.0
    key = torch.where(z.isnan(), torch.full_like(z, INF), z).double()
    key = torch.where(z.isnan(), torch.full_like(key, 1e300), torch.where(key == INF, torch.full_like(key, 1e299), key))
    return torch.sort(key, dim=1, descending=True, stable=True).indices[:, :k]


def _check(z, targets, top_k, got):
    a = z.double()
    rows, cols = a.shape
    big = a.amax(dim=1)
    empty = big == -INF
    c = torch.where(empty[:, None], torch.full_like(a, -INF), a - big[:, None])
    log_s = torch.where(empty, torch.zeros_like(big), c.exp().sum(1).log())
    lp = c - log_s[:, None]
    p = lp.exp()
    d = torch.where(p > 0, c.abs(), torch.zeros_like(a))
    e1, e2 = (p * d).sum(1), (p * d * d).sum(1)
    k, dd = cols / 256 + 72, e1 + 4
    tol = (k + 2 * dd) * U + 2 * U * log_s

    def close(x, y, t, what):
        x = x.double()
        same = (x == y) | ((x - y).abs() <= t)
        assert same.all(), (what, x[~same][:4], y[~same][:4], t[~same][:4])

    assert torch.equal(got.peak.double(), big)
    close(got.log_sum, log_s, tol, "log_sum")
    want_h = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    close(got.entropy, want_h, (2 * k + 4 * dd) * U * (1 + log_s.abs() + e1 + e2), "entropy")

    def spread(x):
        return 2 * U * (torch.where(x == -INF, 0.0, x).abs() + log_s.view([-1] + [1] * (x.dim() - 1)))

    if targets is not None:
        ct = c.gather(1, targets.clamp(min=0)[:, None])[:, 0]
        close(got.logp, torch.where(targets < 0, torch.zeros_like(ct), ct - log_s), tol + spread(ct), "logp")
    if top_k:
        ids = _top_ref(z, top_k)
        assert torch.equal(got.top_ids, ids)
        ct = c.gather(1, ids)
        close(got.top_logp, ct - log_s[:, None], tol[:, None] + spread(ct), "top_logp")
    else:
        assert got.top_ids is None and got.top_logp is None


SHAPES = [(1, 1), (1, 2), (5, 7), (3, 33), (2, 255), (4, 256), (9, 1000), (1, 4096), (200, 1031), (2, 8193), (700, 2048), (1, 32768), (3, 50001), (1, 131072), (17, 65536),
          (150, 30001), (1, 200003), (400, 16384), (2000, 1), (1800, 37), (1999, 1031), (2400, 4096), (1777, 9001), (5000, 2000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_forward(rows, cols, dtype):
    z, targets = _logits(rows, cols, dtype, rows + cols)
    for k in (0, 1, 8, 32):
        k = min(k, cols)
        _check(z, targets, k, binding.solon_token_logprobs(z, targets, top_k=k))
    _check(z, None, 0, binding.solon_token_logprobs(z))


@pytest.mark.parametrize("cols,pitch,offset", [(64, 64, 1), (1000, 1003, 0), (1000, 1008, 8), (5000, 5004, 4), (129, 140, 3), (40001, 40008, 8), (40000, 40001, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 400, 1800])
def test_forward_strides_and_alignment(rows, cols, pitch, offset, dtype):
    z, targets = _logits(rows, cols, dtype, 5, pitch=pitch, offset=offset)
    _check(z, targets, 5, binding.solon_token_logprobs(z, targets, top_k=5))       # the 99s beside the rows are not read


@pytest.mark.parametrize("rows,cols", [(1, 50), (1, 3000), (1, 70001), (12, 50), (12, 3000), (12, 70001), (600, 50), (600, 3000), (600, 70001), (1800, 50), (1900, 9000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masks(rows, cols, dtype):
    """Rows with few tokens left, with one, with none, and masks of the type's lowest value instead of -infinity."""
    z, targets = _logits(rows, cols, dtype, 6, masked=0.9)
    lowest = torch.finfo(z.dtype).min
    z[0] = -INF
    if rows > 4:
        z[1] = -INF
        z[1, cols - 1] = 2.0
        z[2] = lowest                                        # every token equally masked: uniform
        z[3] = lowest
        z[3, cols // 2] = 1.0
        z[4] = -INF
        z[4, 3] = z[4, cols - 2] = lowest
        z[5] = -torch.finfo(z.dtype).min                     # all at the largest value
        z[6, 0], z[7, cols - 1] = lowest, -lowest
    for k in (0, 4, 32):
        _check(z, targets, k, binding.solon_token_logprobs(z, targets, top_k=k))


@pytest.mark.parametrize("rows,cols", [(1, 40), (1, 5000), (1, 100_000), (300, 40), (300, 5000), (300, 100_000), (1800, 40), (1800, 5000)])
def test_ties_orders_and_extremes_among_the_likeliest(rows, cols):
    """Constant rows, few distinct values, rising and falling rows, +0 and -0, the largest values packed into one stretch."""
    g = torch.Generator(device="cuda").manual_seed(3)
    patterns = [torch.full((cols,), 1.5, device="cuda"), torch.randint(0, 3, (cols,), device="cuda", generator=g).float(),
                torch.arange(cols, device="cuda").float() * (20.0 / cols), -torch.arange(cols, device="cuda").float() * (20.0 / cols),
                torch.where(torch.rand(cols, device="cuda", generator=g) < 0.5, -0.0, 0.0),
                torch.cat([torch.zeros(cols - 36, device="cuda"), 5 + torch.rand(36, device="cuda", generator=g)]),
                torch.cat([5 + torch.rand(36, device="cuda", generator=g), torch.zeros(cols - 36, device="cuda")])]
    for dtype in (torch.float32, torch.bfloat16):
        for pattern in patterns:
            z = pattern.to(dtype).expand(rows, cols).contiguous()
            targets = torch.zeros(rows, dtype=torch.long, device="cuda")
            for k in (1, 7, 32):
                _check(z, targets, k, binding.solon_token_logprobs(z, targets, top_k=k))


@pytest.mark.parametrize("rows,cols", [(2, 700), (2, 1500), (150, 1025), (3, 30_001), (900, 6000), (1790, 3001), (2000, 20_000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_likeliest(rows, cols, dtype):
    """Numbers of tokens on both sides of where the search for them changes; their values spread, in few columns, rising, tied."""
    z, targets = _logits(rows, cols, dtype, 9)
    spiked = z.clone()
    spiked[:, ::29] += 8.0
    near = z.clone()
    near[:, cols // 3:cols // 3 + 40] = 30.0                  # more equal ones than are wanted, in neighbouring columns
    few = torch.full_like(z, -1e4)                            # masked by a finite value, with fewer left than are wanted
    few[:, 11::cols // 9] = z[:, 11::cols // 9]
    for k in (8, 9, 16, 17, 24, 25, 31):
        for q in (z, spiked, near, few, z.sort(dim=1).values):
            _check(q, targets, k, binding.solon_token_logprobs(q, targets, top_k=k))


def test_wide_spread_of_values():
    """Logits over hundreds of units, each thread's and each CTA's maximum far from the row's."""
    for rows in (1, 3, 400, 1800):
        z = torch.linspace(-300, 300, 30_000, device="cuda").repeat(rows, 1)
        z = z[:, torch.randperm(30_000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))].contiguous()
        targets = torch.zeros(rows, dtype=torch.long, device="cuda")
        for order in (z, z.sort(dim=1).values, z.sort(dim=1, descending=True).values):
            _check(order, targets, 9, binding.solon_token_logprobs(order, targets, top_k=9))


@pytest.mark.parametrize("cols,copies", [(300, 1), (40_000, 1), (300, 400), (4000, 400)])
def test_targets_and_values_that_are_not_numbers(cols, copies):
    z, _ = _logits(6, cols, "f32", 8)
    targets = torch.tensor([0, -1, cols, cols - 1, 5, -100], device="cuda")
    z[4, 7] = float("nan")
    z[5, 9] = INF
    got = binding.solon_token_logprobs(z.repeat(copies, 1), targets.repeat(copies), top_k=3)
    got = binding.TokenLogprobs(*[x[-6:] for x in got])
    ok = [0, 1, 3]
    _check(z[ok], targets[ok], 3, binding.TokenLogprobs(*[t[ok] for t in got]))
    assert got.logp[2].isnan() and got.log_sum[2].isfinite()
    assert got.log_sum[4].isnan() and got.log_sum[5].isnan() and got.logp[4].isnan() and got.entropy[4].isnan() and got.entropy[5].isnan() and got.logp[5] == 0
    assert got.top_ids[4, 0] == 7 and got.top_ids[5, 0] == 9 and torch.equal(got.top_ids, _top_ref(z, 3))


def _grad_ref(z, targets, r, g, h, gh):
    a = z.double()
    lp = (a - r.peak.double()[:, None]) - r.log_sum.double()[:, None]
    p = lp.exp()
    g = torch.zeros_like(r.peak).double() if g is None else torch.where(targets >= 0, g.double(), 0.0)
    hit = torch.zeros_like(a)
    if targets is not None:
        hit.scatter_(1, targets.clamp(min=0)[:, None], 1.0)
    dz = g[:, None] * (hit - p)
    err = g.abs()[:, None] * (p * (4 * torch.where(p > 0, lp, 0.0).abs() + 10) + 2 * hit) * U
    if gh is not None:
        t = torch.where(p > 0, lp + h.double()[:, None], 0.0)
        dz = dz - gh.double()[:, None] * p * t
        bound = p * (torch.where(p > 0, lp, 0.0).abs() + h.double()[:, None].abs())
        err = err + gh.double().abs()[:, None] * bound * (4 * torch.where(p > 0, lp, 0.0).abs() + 10) * U
    none = r.peak == -INF
    dz[none] = 0
    err[none] = 0
    return dz, err


def _check_grad(z, targets, r, g, h, gh, got, t):
    want, err = _grad_ref(z, targets, r, g, h, gh)
    tol = err + t * want.abs() + (2.0 ** -24 if t == 2.0 ** -10 else 2.0 ** -126)      # (float16's subnormals; float32's below p = 2^-126)
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), (got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 1000), (70, 2049), (2, 70_001), (300, 4096)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_backward(rows, cols, dtype):
    z, targets = _logits(rows, cols, dtype, rows * cols, masked=0.2)
    g = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    gh = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    z[torch.arange(rows, device="cuda"), targets] = 1.0
    if rows > 4:
        z[3] = torch.finfo(z.dtype).min                  # everything masked alike: uniform
        z[4] = torch.finfo(z.dtype).min
        z[4, targets[4]] = 0.5
    if rows > 2:
        targets[1] = -1
        z[2] = -INF                                      # nothing left
        gh[0] = 0.0
    t = TYPES[dtype][1]
    r = binding.solon_token_logprobs(z, targets)
    for args in ((g, None, None), (g, r.entropy, gh), (None, r.entropy, gh)):
        got = binding.solon_token_logprobs_backward(z, targets, r.peak, r.log_sum, args[0], args[1], args[2])
        _check_grad(z, targets, r, *args, got, t)
    none = binding.solon_token_logprobs_backward(z, None, r.peak, r.log_sum, None, r.entropy, gh)
    assert torch.equal(none, got)
    want = binding.solon_token_logprobs_backward(z, targets, r.peak, r.log_sum, g)
    inplace = binding.solon_token_logprobs_backward(z, targets, r.peak, r.log_sum, g, out=z)
    assert inplace.data_ptr() == z.data_ptr() and torch.equal(inplace, want)


@pytest.mark.parametrize("cols,pitch,offset", [(1000, 1003, 3), (1000, 1008, 8), (129, 140, 1), (9000, 9004, 4)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_strides_and_alignment(cols, pitch, offset, dtype):
    z, targets = _logits(13, cols, dtype, 9, pitch=pitch, offset=offset)
    out, _ = _logits(13, cols, dtype, 9, pitch=pitch + 1, offset=2)
    g = torch.linspace(-1, 1, 13, device="cuda")
    r = binding.solon_token_logprobs(z, targets)
    binding.solon_token_logprobs_backward(z, targets, r.peak, r.log_sum, g, out=out)
    _check_grad(z, targets, r, g, None, None, out, TYPES[dtype][1])
    assert (out._base[:2] == 99).all() and (out._base[2:].view(13, pitch + 1)[:, cols:] == 99).all()
    assert (z._base[:offset] == 99).all() and (z._base[offset:].view(13, pitch)[:, cols:] == 99).all()


def test_backward_of_a_target_beyond_the_vocabulary_and_of_rows_without_gradient():
    z, targets = _logits(4, 500, "f32", 10)
    targets[1] = 500
    targets[2] = -7
    z[2, 5] = float("nan")
    r = binding.solon_token_logprobs(z, targets)
    g = torch.ones(4, device="cuda")
    g[3] = 0.0
    got = binding.solon_token_logprobs_backward(z, targets, r.peak, r.log_sum, g)
    assert got[1].isnan().all() and (got[2] == 0).all() and (got[3] == 0).all()
    _check_grad(z[:1], targets[:1], binding.TokenLogprobs(*[None if x is None else x[:1] for x in r]), g[:1], None, None, got[:1], 2.0 ** -23)


def test_backward_agrees_with_differences():
    """Directional derivatives of sum(g logp + gh H) by central differences of the forward kernel.  h = 2^-5 on directions of
    unit entries: the third derivatives of logp and H are below one per unit of p, so the truncation is h^2 of the weights' sum;
    rounding 64 u (|logp| + |H|) / h of it: 2e-3 sum(|g| + |gh|) covers both."""
    z, targets = _logits(10, 300, "f32", 11, scale=1.0)
    gen = torch.Generator(device="cuda").manual_seed(4)
    g, gh = torch.randn(10, device="cuda", generator=gen), torch.randn(10, device="cuda", generator=gen)
    r = binding.solon_token_logprobs(z, targets)
    dz = binding.solon_token_logprobs_backward(z, targets, r.peak, r.log_sum, g, r.entropy, gh).double()
    h = 2.0 ** -5

    def f(x):
        q = binding.solon_token_logprobs(x, targets)
        return float((g.double() * q.logp.double() + gh.double() * q.entropy.double()).sum())

    for _ in range(6):
        e = torch.randn(z.shape, device="cuda", generator=gen).sign()
        got = (f(z + h * e) - f(z - h * e)) / (2 * h)
        assert abs(got - float((dz * e.double()).sum())) <= 2e-3 * float((g.abs() + gh.abs()).sum())


def test_empty_other_streams_and_repeats():
    z = torch.empty((0, 40), device="cuda")
    r = binding.solon_token_logprobs(z, torch.empty(0, dtype=torch.long, device="cuda"), top_k=3)
    assert r.logp.shape == (0,) and r.top_ids.shape == (0, 3)
    assert binding.solon_token_logprobs_backward(z, None, r.peak, r.log_sum).shape == (0, 40)
    for rows in (2, 500, 2000):
        z, targets = _logits(rows, 20_000, "bf16", 12)
        want = binding.solon_token_logprobs(z, targets, top_k=6)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = binding.solon_token_logprobs(z, targets, top_k=6)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_offsets_beyond_32_bits():
    """A matrix of more than 2^32 bytes and 2^31 elements: its last rows as those of a copy, forward and backward in place."""
    rows, cols, tail = 70_000, 32_000, 2000
    z = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    z[-tail:], last = _logits(tail, cols, "bf16", 3)
    targets = torch.zeros(rows, dtype=torch.long, device="cuda")
    targets[-tail:] = last
    got = binding.solon_token_logprobs(z, targets, top_k=3)
    want = binding.solon_token_logprobs(z[-tail:].clone(), last, top_k=3)
    assert all(torch.equal(x[-tail:], y) for x, y in zip(got, want))
    g = torch.full((rows,), 0.5, device="cuda")
    want = binding.solon_token_logprobs_backward(z[-tail:].clone(), last, want.peak, want.log_sum, g[-tail:].clone())
    binding.solon_token_logprobs_backward(z, targets, got.peak, got.log_sum, g, out=z)
    assert torch.equal(z[-tail:], want)


def test_refusals():
    z = torch.zeros((6, 8), device="cuda")
    t = torch.zeros(6, dtype=torch.long, device="cuda")
    v = torch.zeros(6, device="cuda")
    for call in (lambda: binding.solon_token_logprobs(z.cpu()), lambda: binding.solon_token_logprobs(z.double() > 0), lambda: binding.solon_token_logprobs(z.t()),
                 lambda: binding.solon_token_logprobs(z, t.int()), lambda: binding.solon_token_logprobs(z, t[:5]),
                 lambda: binding.solon_token_logprobs_backward(z, t, v[:5], v, v), lambda: binding.solon_token_logprobs_backward(z, t, v, v, v, out=z.bfloat16())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.solon_token_logprobs(z.double()), lambda: binding.solon_token_logprobs(z, t, top_k=9),
                 lambda: binding.solon_token_logprobs(torch.zeros((6, 80), device="cuda"), t, top_k=33),
                 lambda: binding.solon_token_logprobs(z[:, :0], t), lambda: binding.solon_token_logprobs_backward(z, None, v, v, v),
                 lambda: binding.solon_token_logprobs_backward(z, t, v, v, v, None, v)):
        with pytest.raises(binding.SolonError) as err:
            call()
        assert err.value.status == binding.ERR_INVALID_ARG


HUGE = [1.2e7, 5e7, 1e9, 2e9, 3e9, 1e10, 1e12, 1e30, 1e38]


def _rows_with(value, cols, dtype):
    """Ordinary logits beside `value` and its neighbours (steps of 1 and of the type's spacing), a row a pattern."""
    g = torch.Generator(device="cuda").manual_seed(13)
    ordinary = torch.randn(cols, device="cuda", generator=g) * 3
    full = torch.full((cols,), value, device="cuda")
    at = torch.arange(cols, device="cuda")
    low = torch.full((cols,), -abs(value), device="cuda")
    step = max(1.0, abs(value) * torch.finfo(dtype).eps)
    near = full + torch.randint(-3, 4, (cols,), device="cuda", generator=g) * step
    far = torch.tensor([-1e38, -1e30, -1e10, -1e9, -1.2e7, -1e4, 0.0, 5.0], device="cuda")[at * 8 // cols]
    rows = [full, near, torch.where(at < cols * 3 // 4, low, ordinary), torch.where(at < cols // 3, ordinary, low),
            torch.where(at == cols - 1, ordinary, low), torch.where(at == cols // 2, ordinary, low), torch.where(at % 5 == 0, ordinary, near), far,
            torch.where(at == cols // 3, full, ordinary), near.sort().values]
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("rows,cols", [(10, 50), (10, 3000), (1, 70_001), (400, 16_384), (1800, 5000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [s * v for v in HUGE for s in (1, -1)] + [9.9e6, -9.9e6, -1e6])
def test_logits_of_large_magnitude(value, dtype, rows, cols):
    """Finite logits far from 0: masks other than the type's lowest value - throughout a row, over its first thousands of columns, all but
    one -, and rows whose values all lie there."""
    z = _rows_with(value, cols, TYPES[dtype][0])
    z = z.repeat(-(-rows // len(z)), 1)[:rows] if rows > 1 else z
    targets = torch.randint(0, cols, (len(z),), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    targets[::3] = cols // 3
    for part in z.split(1 if rows == 1 else rows):
        own = targets[:len(part)]
        for k in (0, 5, 32):
            _check(part, own, k, binding.solon_token_logprobs(part, own, top_k=k))


@pytest.mark.parametrize("rows,cols", [(4, 300), (4, 40_000), (1, 131_072), (400, 9000), (2400, 4000), (7, 1003), (7, 30_001), (1, 100_003), (2401, 2001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_peak_of_rows_that_hold_nan(rows, cols, dtype):
    """The largest logit as an elementary maximum has it: NaN where there is one, +infinity where there is that."""
    z, targets = _logits(rows, cols, dtype, 14, masked=0.3)
    for place in (0, cols // 2, cols - 1):
        for values, want in (([float("nan")], float("nan")), ([INF], INF), ([INF, float("nan")], float("nan")), ([-INF, float("nan")], float("nan"))):
            q = z.clone()
            if values[0] == -INF:
                q[::2] = -INF
            q[::2, place] = values[-1]
            if values[0] == INF:
                q[::2, cols // 3] = INF
            for k in (0, 3):
                got = binding.solon_token_logprobs(q, targets, top_k=k)
                assert torch.equal(got.peak.isnan(), q.float().amax(1).isnan()) and got.peak.isnan()[::2].all() == (want != want)
                assert torch.equal(got.peak.nan_to_num(nan=7.0, posinf=8.0), q.float().amax(1).nan_to_num(nan=7.0, posinf=8.0))
                assert got.log_sum[::2].isnan().all() and got.entropy[::2].isnan().all() and got.logp[::2].isnan().all()
                if rows > 1:
                    kept = [None if x is None else x[1::2] for x in got]
                    _check(q[1::2], targets[1::2], k, binding.TokenLogprobs(*kept))
