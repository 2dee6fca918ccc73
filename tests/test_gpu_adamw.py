"""The AdamW step against the formulas in float64: 32-bit and 8-bit states, flat and bound gradients, clipping, the guard of a
plan's decode, counting on the device, resuming.

Tolerances (u = 2^-24).  The scaled gradient carries 3 roundings (a clipped one the norm's relative 2^-20 more: squares and short
sums in float32, then float64), so m is off by 6 u (b1 |m| + (1 - b1) |g|) and v by 10 u v; the step's quotient then by 24 u relative to
(b1 |m| + (1 - b1) |g|) / denominator, and p by 3 u |p| more.  An 8-bit code is the window's rank of a value known to those bounds:
it has to lie between the codes of the bounds' ends for the slot's random bits."""

import math

import pytest
import torch

from paper_2110_01595_b200 import binding, build, synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8
SIZES = [1, 255, 256, 257, 0, 3, 2048, 2049, 10_000, 77]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(n, seed, scale=1.0):
    return torch.randn(n, device="cuda", generator=_gen(seed)) * scale


def _flat(blocked, sizes):
    """The elements of a blocks x 256 tensor in the tensors' order, and whether the padding is zero."""
    at, parts, padding = 0, [], []
    f = blocked.reshape(-1)
    for n in sizes:
        room = -(-n // 256) * 256
        parts.append(f[at:at + n])
        padding.append(f[at + n:at + room])
        at += room
    assert at == f.numel() and not torch.cat(padding).any()
    return torch.cat(parts)


def _slots(sizes):
    at, parts = 0, []
    for n in sizes:
        parts.append(torch.arange(at, at + n, device="cuda"))
        at += -(-n // 256) * 256
    return torch.cat(parts)


def _per_element(values, sizes):
    return torch.repeat_interleave(torch.tensor(values, dtype=torch.float64, device="cuda"), torch.tensor(sizes, device="cuda"))


def _mix(h):
    h = h ^ (h >> 16)
    h = (h * 0x85EBCA6B) & 0xFFFFFFFF
    h = h ^ (h >> 13)
    h = (h * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _random_bits(slots, seed, t):
    key = _mix((t * 0x9E3779B1 + (seed & 0xFFFFFFFF)) & 0xFFFFFFFF) ^ (seed >> 32)
    h = _mix(((slots * 0x9E3779B1) & 0xFFFFFFFF) ^ key)
    return (h & 0xFFFF) << 4, (h >> 16) << 4


class Ref:
    """One AdamW step in float64 with the bounds of the float32 one's errors."""

    def __init__(self, p, g, m, v, t, lr, decay, scale=1.0, max_norm=0.0):
        g = g.double() * scale
        self.norm = g.norm()
        rel = 6 * U
        if max_norm > 0:
            g = g * min(1.0, max_norm / (float(self.norm) + 1e-6))
            rel += 2.0 ** -20
        m, v, p = m.double(), v.double(), p.double()
        self.m, self.v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
        size = B1 * m.abs() + (1 - B1) * g.abs()
        self.m_tol, self.v_tol = rel * size, (2 * rel) * self.v + 2.0 ** -140
        den = (self.v / (1 - B2 ** t)).sqrt() + EPS
        step = lr / (1 - B1 ** t)
        self.p = p * (1 - lr * decay) - step * self.m / den
        self.p_tol = 3 * U * p.abs() + step * size / den * (24 * U + 4 * rel) + U * self.p.abs()


def _close(got, want, tol, what):
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4])


def _setup(sizes, seed, offset=0):
    """Parameters as views of one buffer (offset odd: off 16-byte boundaries), their flat form and a flat gradient."""
    d = sum(sizes)
    buf = _randn(d + offset, seed, 0.3)
    flat = buf[offset:]
    views, at = [], 0
    for n in sizes:
        views.append(flat[at:at + n])
        at += n
    return flat, views, _randn(d, seed + 1) * torch.exp(_randn(d, seed + 2))


@pytest.mark.parametrize("grad_type", [torch.float32, torch.float64, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("max_norm", [0.0, 0.7, 1e9])
def test_32_bit_states_over_several_steps(grad_type, offset, max_norm):
    flat, views, grad = _setup(SIZES, 1, offset)
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") if i % 2 else None for i, n in enumerate(SIZES)]
    with binding.AdamW(views, betas=(B1, B2), eps=EPS, weight_decay=decay, copies=copies) as opt:
        for t in range(1, 5):
            g = torch.roll(grad, t).to(grad_type)
            m, v = (_flat(x, SIZES).clone() for x in opt.moments())
            ref = Ref(flat.clone(), g, m, v, t, 1e-2, _per_element(decay, SIZES), 1 / 15, max_norm)
            norm = opt.step(g, lr=1e-2, grad_scale=1 / 15, max_norm=max_norm)
            assert (norm is None) == (max_norm == 0)
            if max_norm:
                assert abs(float(norm) - float(ref.norm)) <= 2.0 ** -20 * float(ref.norm)
            m, v = (_flat(x, SIZES) for x in opt.moments())
            _close(m, ref.m, ref.m_tol, "m")
            _close(v, ref.v, ref.v_tol, "v")
            _close(flat, ref.p, ref.p_tol, "p")
            for p, c in zip(views, copies):
                assert c is None or torch.equal(c, p.bfloat16())
        assert opt.steps() == (4, 0)


@pytest.mark.parametrize("grad_type", [torch.float32, torch.float64, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("max_norm", [0.0, 0.7, 1e9])
def test_moments_are_those_of_elementary_operations(grad_type, offset, max_norm):
    """Bit for bit those of float32 products and sums, one after the other, with the clip factor from the norm that is handed back."""
    flat, views, grad = _setup(SIZES, 21, offset)
    with binding.AdamW(views, betas=(B1, B2), eps=EPS) as opt:
        for t in range(1, 4):
            g = torch.roll(grad, t).to(grad_type)
            m, v = (_flat(x, SIZES).clone() for x in opt.moments())
            norm = opt.step(g, lr=1e-2, grad_scale=1 / 15, max_norm=max_norm)
            h = g.float() * (1 / 15)
            if max_norm:
                h = h * (max_norm * (norm + 1e-6).reciprocal()).clamp(max=1.0)
            got_m, got_v = (_flat(x, SIZES) for x in opt.moments())
            assert torch.equal(got_m, B1 * m + (1 - B1) * h) and torch.equal(got_v, B2 * v + (1 - B2) * h * h)


def test_clipping_by_a_norm_beyond_float32():
    flat, views, _ = _setup([4096], 22)
    grad = torch.full((4096,), 3e38, device="cuda")          # norm 1.92e40
    with binding.AdamW(views, betas=(B1, B2), eps=EPS) as opt:
        norm = opt.step(grad, lr=1e-2, max_norm=1.0)
        m, _ = (_flat(x, [4096]) for x in opt.moments())
        assert float(norm) == float("inf") and opt.steps() == (1, 0)
        assert ((m.double() * 10 * 64 - 1).abs() < 2.0 ** -20).all()     # g' = 1 / 64


def _codes(low, high, rand, base, levels):
    """The two ends' codes of magnitudes known to lie in [low, high] (float64), for given random bits and window bases."""
    out = []
    for x in (low, high):
        mant, exp = torch.frexp(x.clamp(min=2.0 ** -126))
        rank = (exp + 125).double() * 8 + 8 + (mant * 2 - 1) * 8 - 8 + 0          # bits / 2^20 of a normal float32, as a real number
        rank = torch.where(x < 2.0 ** -126, x / 2.0 ** -126 * 8, rank + 8)
        out.append((torch.floor(rank + rand.double() / 2 ** 20) - base).clamp(max=levels))
    return out


@pytest.mark.parametrize("offset,grad_type,max_norm", [(0, torch.float32, 0.0), (1, torch.float32, 0.5), (0, torch.float64, 0.0), (1, torch.bfloat16, 0.0)])
def test_8_bit_states_over_several_steps(offset, grad_type, max_norm):
    seed = 0x1234567890ABCDEF
    flat, views, grad = _setup(SIZES, 3, offset)
    grad[300:2400] *= 1e-7                        # blocks of small gradients, and blocks with both
    slots = _slots(SIZES)
    block = slots // 256
    with binding.AdamW(views, bits=8, betas=(B1, B2), eps=EPS, weight_decay=0.05, seed=seed) as opt:
        for t in range(1, 6):
            g = torch.roll(grad, 13 * t).to(grad_type)
            m, v = (_flat(x, SIZES).float() for x in opt.moments())
            ref = Ref(flat.clone(), g, m, v, t, 1e-2, torch.full((len(slots),), 0.05, device="cuda").double(), 1.0, max_norm)
            opt.step(g, lr=1e-2, max_norm=max_norm)
            _close(flat, ref.p, ref.p_tol, "p")
            mc, vc = (_flat(x, SIZES).long() for x in opt.state[:2])
            base = opt.state[2].long()
            for what, codes, levels, col, rand, x, tol in (("m", mc & 127, 127, 0, _random_bits(slots, seed, t)[0], ref.m.abs(), ref.m_tol),
                                                           ("v", vc, 255, 1, _random_bits(slots, seed, t)[1], ref.v, ref.v_tol)):
                low, high = (x - tol).clamp(min=0), x + tol
                # the window ends at the block's largest magnitude, rounded up to the grid
                for end, op in ((low, torch.le), (high, torch.ge)):
                    top = torch.zeros(base.shape[0], dtype=torch.float64, device="cuda").scatter_reduce(0, block, end, "amax")
                    rank = _codes(top, top, torch.full_like(top, 2 ** 20 - 1), 0.0, 1e9)[0]
                    assert op((rank - levels).clamp(min=0), base[:, col].double()).all(), what
                lo, hi = _codes(low, high, rand, base[block, col], levels)
                smallest = (x > 0).long() if what == "v" else torch.zeros_like(codes)
                assert ((codes >= lo.clamp(min=0)) & (codes <= torch.maximum(hi.clamp(min=0), smallest.double())) & (codes >= smallest)).all(), what
            assert ((mc >> 7 == 1) == ((ref.m < 0) & (mc & 127 > 0)))[ref.m.abs() > ref.m_tol].all()
            # what the codes stand for
            want = torch.where(vc > 0, (vc + base[block, 1]) << 20, 0).int().view(torch.float32)
            assert torch.equal(_flat(opt.moments()[1], SIZES).float(), want)
            want = torch.where(mc & 127 > 0, ((mc & 127) + base[block, 0]) << 20, 0).int().view(torch.float32)
            assert torch.equal(_flat(opt.moments()[0], SIZES).float(), want * (1 - 2 * (mc >> 7)))


def test_8_bit_rounding_is_unbiased():
    """Constant gradients from a zero state: m and v have closed forms.  A code is one of two neighbours 1/8 to 1/16 apart, chosen
    without bias, so over n = 20000 equal elements the mean state differs from the exact one by a relative
    0.0625 sqrt(sum of squared survivals) / sqrt(n) at one standard deviation: below 0.0625 * 3 / 141 for m, and for v, whose
    roundings of up to 60 steps survive, 0.0625 * sqrt(60) / 141; five of those are allowed."""
    n, steps = 20_000, 60
    p = torch.zeros(n, device="cuda")
    with binding.AdamW([p], bits=8, betas=(0.9, 0.99), seed=7) as opt:
        g = torch.full((n,), 0.37, device="cuda")
        for _ in range(steps):
            opt.step(g, lr=0.0)
        m, v = (_flat(x, [n]).double() for x in opt.moments())
    want_m, want_v = 0.37 * (1 - 0.9 ** steps), 0.37 ** 2 * (1 - 0.99 ** steps)
    assert abs(float(m.mean()) / want_m - 1) <= 5 * 0.0625 * 3 / math.sqrt(n)
    assert abs(float(v.mean()) / want_v - 1) <= 5 * 0.0625 * math.sqrt(steps) / math.sqrt(n)


def test_8_bit_training_follows_32_bit_training():
    """Least squares with noisy gradients: both widths bring the loss down by the same order."""
    d = 4096
    target = _randn(d, 5)
    losses = []
    for bits in (32, 8):
        p = torch.zeros(d, device="cuda")
        curvature = torch.exp(_randn(d, 6))
        with binding.AdamW([p[:1000], p[1000:]], bits=bits, betas=(0.9, 0.99)) as opt:
            for t in range(400):
                opt.step(curvature * (p - target) + 0.05 * _randn(d, 100 + t), lr=0.02)
        losses.append(float((p - target).square().mean()))
    assert losses[0] < 2e-3 and losses[1] < 2 * losses[0] + 1e-3, losses


def test_blocks_that_hold_values_that_are_not_finite():
    """An infinite or NaN gradient goes into its own weight; the other elements of its block keep their states."""
    for bits in (32, 8):
        p, q = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda")
        g = _randn(512, 9)
        bad = g.clone()
        bad[10], bad[300] = float("nan"), float("inf")
        a, b = binding.AdamW([p], bits=bits, seed=3), binding.AdamW([q], bits=bits, seed=3)
        for _ in range(3):
            a.step(bad, lr=1e-2)
            b.step(g, lr=1e-2)
        keep = torch.ones(512, dtype=torch.bool, device="cuda")
        keep[[10, 300]] = False
        assert p[10].isnan()
        if bits == 32:
            assert torch.equal(p[keep], q[keep])
        else:     # the two elements have no part in their block's window; where theirs was the largest the windows may differ
            assert p[keep].isfinite().all() and ((p - q)[keep].abs() <= 0.2 * 3e-2).all()


def test_clipping_to_a_norm_that_is_not_finite_skips_the_step():
    for value in (float("nan"), float("inf")):
        p = _randn(3000, 1)
        before = p.clone()
        g = torch.ones(3000, device="cuda")
        with binding.AdamW([p]) as opt:
            g[2999] = value
            opt.step(g, lr=1.0, max_norm=1.0)
            assert torch.equal(p, before) and opt.steps() == (0, 1) and not opt.state[0].any()
            g[2999] = 1.0
            opt.step(g, lr=1.0, max_norm=1.0)
            assert opt.steps() == (1, 1) and not torch.equal(p, before)


def test_bound_gradients_equal_the_flat_ones():
    for bits in (32, 8):
        flat, views, grad = _setup(SIZES, 5)
        other = [v.clone() for v in views]
        grads, at = [], 0
        for n in SIZES:
            grads.append(grad[at:at + n].clone())
            at += n
        a, b = binding.AdamW(views, bits=bits), binding.AdamW(other, bits=bits)
        with pytest.raises(binding.SolonError):
            b.step(None)
        b.bind_grads(grads)
        for clip in (0.0, 0.3):
            na, nb = a.step(grad, max_norm=clip), b.step(max_norm=clip)
            assert torch.equal(flat, torch.cat(other)) and (not clip or torch.equal(na, nb))
        assert all(torch.equal(x, y) for x, y in zip(a.state, b.state) if x is not None)


def test_guard_of_a_failed_decode():
    """A step whose plan could not decode changes nothing, whatever the aggregate holds; the next good decode's is applied."""
    wl = synth.small_variant(synth.WORKLOADS["tiny"], 5000)
    G = synth.make_grads(wl, "cuda")
    with binding.Plan(wl.P, wl.s, wl.m, wl.r, wl.d, seed=1) as plan:
        coded = plan.encode(G)
        p = _randn(wl.d, 1)
        before = p.clone()
        with binding.AdamW([p[:1], p[1:]], bits=8) as opt:
            received = coded.clone()
            received[[0, 1, 2]] = _randn(3 * plan.d_c, 2, 50.0).view(3, -1)          # three attackers where one is tolerated
            agg, _ = plan.decode(received)
            opt.step(agg, lr=1.0, max_norm=1.0, plan=plan)
            assert plan.decode_status() == binding.ERR_UNDECODABLE
            assert torch.equal(p, before) and opt.steps() == (0, 1)
            received, _ = synth.apply_attack(wl, coded)
            agg, _ = plan.decode(received)
            opt.step(agg, lr=1.0, plan=plan)
            assert plan.decode_status() == 0 and opt.steps() == (1, 1) and not torch.equal(p, before)
            side = torch.cuda.Stream()
            with torch.cuda.stream(side), pytest.raises(ValueError):
                opt.step(agg, plan=plan)


def test_step_from_the_aggregate_of_a_float64_plan():
    """The 8-byte wire format's aggregate goes into the step as it is; the same step from its float32 rounding is equal."""
    P, d = 8, 6001
    G = torch.randn((P, d), dtype=torch.float64, device="cuda", generator=_gen(3))
    with binding.Plan(P, 1, 2, 4, d, seed=1, dtype="f64") as plan:
        agg, mask = plan.decode(plan.encode(G))
        p, q = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
        a, b = binding.AdamW([p[:5], p[5:]], bits=8), binding.AdamW([q[:5], q[5:]], bits=8)
        a.step(agg, lr=1e-2, grad_scale=1 / P, plan=plan)
        b.step(agg.float(), lr=1e-2, grad_scale=1 / P, plan=plan)
        assert plan.decode_status() == 0 and not mask.any()
        assert torch.equal(p, q) and all(torch.equal(x, y) for x, y in zip(a.state, b.state))
        assert float((a.of_tensor(a.moments()[0], 1).float() - 0.1 * G.mean(0)[5:].float()).abs().max()) <= 0.13 * 0.1 * float(G.mean(0).abs().max())


def test_replayed_graph_counts_its_steps():
    for bits in (32, 8):
        flat, views, grad = _setup(SIZES, 7)
        flat2, views2, _ = _setup(SIZES, 7)
        a, b = binding.AdamW(views, bits=bits), binding.AdamW(views2, bits=bits)
        for _ in range(5):
            a.step(grad, lr=1e-2, max_norm=1.0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b.step(grad, lr=1e-2, max_norm=1.0)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.step(grad, lr=1e-2, max_norm=1.0)
        for _ in range(4):
            graph.replay()
        assert torch.equal(flat, flat2) and a.steps() == b.steps() == (5, 0)
        assert all(torch.equal(x, y) for x, y in zip(a.state, b.state) if x is not None)
        del graph


def test_resuming_from_a_saved_state():
    for bits in (32, 8):
        flat, views, grad = _setup(SIZES, 8)
        a = binding.AdamW(views, bits=bits, seed=5)
        for _ in range(3):
            a.step(grad)
        saved = tuple(None if t is None else t.clone() for t in a.state)
        p = flat.clone()
        resumed = binding.AdamW(list(p.split(SIZES)), bits=bits, seed=5, state=saved, step=a.steps()[0])
        a.step(grad)
        resumed.step(grad)
        assert torch.equal(p, flat) and resumed.steps() == (4, 0)
        assert torch.equal(a.of_tensor(a.state[0], 6), resumed.of_tensor(saved[0], 6)) and a.of_tensor(a.state[0], 6).numel() == SIZES[6]


def test_nothing_beside_the_tensors_is_written():
    for bits in (32, 8):
        for offset in (0, 1, 2, 3):
            n = 4097
            buf, cbuf = torch.full((n + 64,), 5.0, device="cuda"), torch.full((n + 64,), 5.0, device="cuda", dtype=torch.bfloat16)
            g = _randn(n + 8, 1)
            keep = g.clone()
            with binding.AdamW([buf[16 + offset:16 + offset + n]], bits=bits, copies=[cbuf[16 + offset:16 + offset + n]]) as opt:
                opt.step(g[offset:offset + n], lr=1.0, max_norm=1.0)
            for t in (buf, cbuf):
                assert (t[:16 + offset] == 5).all() and (t[16 + offset + n:] == 5).all() and (t[16 + offset:16 + offset + n] != 5).any()
            assert torch.equal(g, keep)


def test_offsets_beyond_32_bits():
    """More than 2^31 weights with 8-bit states: the last tensor's step as that of a handle of its own would be, but for the
    rounding's random bits (which go by the place in the state): parameters, whose step comes before the rounding, are equal."""
    n = 2_200_000_001
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-5000:], g[-5000:] = _randn(5000, 1), _randn(5000, 2).bfloat16()
    own, grad = p[-5000:].clone(), g[-5000:].clone()
    big, small = binding.AdamW([p[:-5000], p[-5000:]], bits=8), binding.AdamW([own], bits=8)
    a, b = big.step(g, lr=1e-2, max_norm=0.5), small.step(grad, lr=1e-2, max_norm=0.5)
    assert abs(float(a) - float(b)) <= 1e-6 * float(b) and float((p[-5000:] - own).abs().max()) <= 1e-6
    m, v = (big.of_tensor(t, 1).float() for t in big.moments())
    assert float((m - 0.1 * grad.float() * (0.5 / float(b))).abs().max()) <= 0.13 * 0.1 * float(grad.float().abs().max()) * 0.5 / float(b)
    assert (v > 0).all() and not big.state[0][:-20].any() and (p[:-5000] == 0).all()


def test_refusals():
    p = torch.zeros(100, device="cuda")
    g = torch.zeros(100, device="cuda")
    for call in (lambda: binding.AdamW([]), lambda: binding.AdamW([p.cpu()]), lambda: binding.AdamW([p.double()]), lambda: binding.AdamW([p[::2]]),
                 lambda: binding.AdamW([p], bits=16), lambda: binding.AdamW([p], weight_decay=[0.1, 0.2]), lambda: binding.AdamW([p], copies=[p]),
                 lambda: binding.AdamW([p], copies=[p.bfloat16()[:50]]), lambda: binding.AdamW([p], state=(g, g, None))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.AdamW([p], betas=(1.0, 0.9)), lambda: binding.AdamW([p], betas=(0.9, -0.1)), lambda: binding.AdamW([p], eps=0.0),
                 lambda: binding.AdamW([p], weight_decay=-1.0)):
        with pytest.raises(binding.SolonError) as err:
            call()
        assert err.value.status == binding.ERR_INVALID_ARG
    with binding.AdamW([p]) as opt:
        for call in (lambda: opt.step(g[:99]), lambda: opt.step(g.cpu()), lambda: opt.step(g.int()), lambda: opt.bind_grads([g, g]), lambda: opt.bind_grads([g[:5]])):
            with pytest.raises(ValueError):
                call()
        for call in (lambda: opt.step(g.half()), lambda: opt.step(g, lr=-1.0), lambda: opt.step(g, lr=float("nan")), lambda: opt.step(g, max_norm=float("inf")),
                     lambda: opt.step(g, grad_scale=float("nan")), lambda: opt.step(), lambda: opt.set_step(-1)):
            with pytest.raises(binding.SolonError) as err:
                call()
            assert err.value.status == binding.ERR_INVALID_ARG
        assert opt.steps() == (0, 0)


@pytest.mark.parametrize("bits", [32, 8])
def test_handles_made_bound_and_resumed_inside_another_stream(bits):
    """What the host uploads - chunk table, bound gradients, step count - has arrived before a step that is enqueued next on a stream
    that does not wait for the default one."""
    flat, views, grad = _setup(SIZES, 41, 1)
    flat2, views2, _ = _setup(SIZES, 41, 1)
    grads = list(grad.split(SIZES))
    other = [(-2 * g).clone() for g in grads]
    want = binding.AdamW(views, bits=bits, seed=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = binding.AdamW(views2, bits=bits, seed=3)
        for bound, count in ((grads, None), (other, None), (grads, 700), (other, 3), (grads, 0)):
            got.bind_grads(bound)
            if count is not None:
                got.set_step(count)
            got.step(None, lr=1e-2, max_norm=1.0)
    side.synchronize()
    for bound, count in ((grads, None), (other, None), (grads, 700), (other, 3), (grads, 0)):
        want.bind_grads(bound)
        if count is not None:
            want.set_step(count)
        want.step(None, lr=1e-2, max_norm=1.0)
    assert want.steps() == got.steps() == (1, 0) and torch.equal(flat, flat2)
    assert all(torch.equal(x, y) for x, y in zip(want.state, got.state) if x is not None)


def test_a_refused_binding_leaves_the_earlier_one():
    p, g = torch.zeros(3000, device="cuda"), _randn(3000, 51)
    with binding.AdamW([p]) as opt:
        with pytest.raises(binding.SolonError):
            opt.bind_grads([g.half()])
        with pytest.raises(binding.SolonError):
            opt.step()
        opt.bind_grads([g])
        for refused in (lambda: opt.bind_grads([g.half()]), lambda: opt.bind_grads([g[:7]]), lambda: opt.bind_grads([])):
            with pytest.raises((binding.SolonError, ValueError, IndexError)):
                refused()
        opt.step(lr=0.5)
        assert (p.sign() == -g.sign()).all() and opt.steps() == (1, 0)


@pytest.mark.parametrize("grad_type", [torch.float32, torch.float64, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_that_end_just_behind_a_block(bits, grad_type):
    """Sizes of 0 to 4 elements more than whole blocks and chunks, off 16-byte boundaries: as with tensors on them, bit for bit, and
    nothing beside them changes."""
    for whole in (256, 512, 2048, 4096):
        for extra in (0, 1, 2, 3, 4):
            n = whole + extra
            p, g = _randn(n, 61), _randn(n, 62).to(grad_type)
            own = p.clone()
            want = binding.AdamW([own], bits=bits, seed=9)
            for _ in range(2):
                want.step(g.clone(), lr=1e-2, max_norm=0.5)
            for offset in (1, 2, 3):
                buf, gbuf = torch.full((n + 16,), float("nan"), device="cuda"), torch.full((n + 16,), float("nan"), dtype=grad_type, device="cuda")
                view, grad = buf[4 + offset:4 + offset + n], gbuf[8 - offset:8 - offset + n]
                view.copy_(p)
                grad.copy_(g)
                with binding.AdamW([view], bits=bits, seed=9) as opt:
                    for _ in range(2):
                        opt.step(grad, lr=1e-2, max_norm=0.5)
                    assert torch.equal(view, own) and all(torch.equal(x, y) for x, y in zip(opt.state, want.state) if x is not None)
                assert buf.isnan().sum() == 16 and gbuf.isnan().sum() == 16


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-44, 1e-40, 1e-38, 1e-30, 1e30, 1e38, 3e38])
def test_eps_at_the_ends_of_its_range(eps, bits):
    """From a zero state the first step is lr g / (|g| + eps), whatever eps (4 u for the moments, 24 u for the quotient, as above);
    a weight that has had no gradient stays as it is."""
    p = torch.zeros(1024, device="cuda")
    g = _randn(1024, 31, 1e-3 if eps < 1 else 1e18)
    g[:100] = 0.0
    p[:100] = 3.0
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    with binding.AdamW([p], bits=bits, betas=(B1, B2), eps=eps) as opt:
        opt.step(g, lr=0.5)
    want = -0.5 * g.double() / (g.double().abs() + eps32)
    want[:100] = 3.0
    _close(p, want, 32 * U * want.abs() + 2.0 ** -126, "p")
