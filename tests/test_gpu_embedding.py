"""Embedding lookup and its gradient by sorted tokens, against indexing and sums in float64.

Tolerances (u = 2^-24).  The lookup with a factor is one float32 product and one rounding to the element type; without, the bits are copied.
A gradient is a float32 sum of at most t rows of one token in some order, so its error is at most t u times the sum of the absolute
values, (t + 2) u with the factor (rounded to float32, and the product); then half a step of the gradient's type, and one more of both
where the sum is added to what was there."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f64": torch.float64}
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _framed(rows, cols, dtype, pitch=None, offset=0, fill=99.0):
    """A matrix inside a larger buffer filled with a value that no result has."""
    pitch = cols if pitch is None else pitch
    buf = torch.full((offset + rows * pitch + 64,), fill, dtype=TYPES[dtype], device="cuda")
    return buf, buf[offset:offset + rows * pitch].view(rows, pitch)[:, :cols]


def _untouched(buf, view, fill=99.0):
    mark = torch.ones_like(buf, dtype=torch.bool)
    mark.as_strided(view.shape, view.stride(), view.storage_offset())[...] = False
    return bool((buf[mark] == fill).all())


@pytest.mark.parametrize("rows,cols,vocab", [(1, 1, 1), (1, 2048, 1000), (3, 7, 5), (1000, 1001, 301), (513, 64, 50_000), (700, 4096, 333), (5, 20_000, 17), (4097, 130, 9)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", [None, (0, 8), (1, 0), (8, 16), (3, 5), (2, 2), (4, 4)])      # (offset, additional pitch) in elements
def test_forward(rows, cols, vocab, dtype, layout):
    g = _gen(rows + cols)
    offset, more = layout or (0, 0)
    _, weight = _framed(vocab, cols, dtype, cols + more, offset)
    weight.copy_(torch.randn((vocab, cols), device="cuda", generator=g))
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    if rows > 2:
        tokens[1], tokens[2] = -1, vocab
    for scale in (1.0, 0.3):
        buf, out = _framed(rows, cols, dtype, cols + more, offset)
        got = binding.solon_embedding_forward(weight, tokens, scale=scale, out=out)
        assert got is out and _untouched(buf, out)
        want = weight[tokens.clamp(0, vocab - 1)]
        if scale != 1.0:
            want = (want.float() * torch.tensor(scale, device="cuda")).to(want.dtype)
        want[tokens < 0] = 0.0
        want[tokens >= vocab] = NAN
        assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(out.nan_to_num(5.0), want.nan_to_num(5.0))
    assert torch.equal(binding.solon_embedding_forward(weight, tokens[:1]), weight[tokens[:1]])


def _check(dy, tokens, vocab, parts, scale, got, before=None):
    rows, cols = dy.shape
    n = rows // parts
    got = got.view(parts, vocab, cols) if got.is_contiguous() else got.as_strided((parts, vocab, cols), (got.stride(0), cols, 1), got.storage_offset())
    step = torch.finfo(got.dtype).eps / 2
    keep = (tokens >= 0) & (tokens < vocab)
    for k in range(parts):
        r = slice(k * n, (k + 1) * n)
        t, x = tokens[r][keep[r]], dy[r][keep[r]].double() * scale
        want = torch.zeros((vocab, cols), dtype=torch.float64, device="cuda").index_add_(0, t, x)
        size = torch.zeros((vocab, cols), dtype=torch.float64, device="cuda").index_add_(0, t, x.abs())
        count = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, t, torch.ones(len(t), dtype=torch.float64, device="cuda"))
        if before is not None:
            want += before[k].double().view(vocab, cols)
        tol = (count[:, None] + 2) * U * size + (step + (U if before is not None else 0.0)) * want.abs()
        tol += 2.0 ** -140                                       # (products of a scale below float32's normal numbers)
        bad = (got[k].double() - want).abs() > tol * (1 + 1e-6)
        assert not bad.any(), (k, bad.nonzero()[:3], got[k][bad][:3], want[bad][:3], tol[bad][:3])
        if before is None:
            assert (got[k][count == 0] == 0).all()


# rows of a partition, partitions, columns, vocabulary
BACK = [(1, 1, 1, 1), (1, 3, 5, 7), (0, 4, 9, 30), (64, 45, 101, 203), (31, 2, 64, 3), (33, 2, 128, 1), (8, 1, 4096, 50), (100, 3, 1001, 1000), (2048, 4, 256, 513), (2049, 1, 40, 70_000),
        (5000, 2, 24, 100), (9000, 1, 33, 513), (20_000, 1, 16, 2), (40_000, 2, 8, 300_000), (70_001, 1, 3, 512), (1000, 1, 9000, 40), (300, 7, 66, 511)]


@pytest.mark.parametrize("n,parts,cols,vocab", BACK)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_backward(n, parts, cols, vocab, dtype):
    """Tokens as text has them, some that count nowhere, rows and gradient rows at any alignment; twice the same bits."""
    g = _gen(n + cols)
    rows = n * parts
    tokens = (torch.exp(torch.rand(rows, device="cuda", generator=g) * torch.log(torch.tensor(vocab + 1.0))).long() - 1).clamp(0, vocab - 1)
    if rows > 20:
        tokens[::17], tokens[5::19] = -1, vocab + 3
        tokens[7] = -(1 << 62)
        tokens[11] = (1 << 40) + 1
    for (offset, more), (at, after), grad, scale in (((0, 0), (0, 0), "f32", 1.0), ((1, 3), (5, 3), "f32", 2.5), ((8, 8), (16, 16), "bf16", 1.0),
                                                     ((4, 0), (2, 2), "f64", 1.0), ((2, 2), (3, 1), "bf16", 0.7)):
        _, dy = _framed(rows, cols, dtype, cols + more, offset)
        dy.copy_(torch.randn((rows, cols), device="cuda", generator=g))
        buf, dw = _framed(parts, vocab * cols, grad, vocab * cols + after, at)
        out = binding.solon_embedding_backward(dy, tokens, vocab, partitions=parts, scale=scale, dweight=dw)
        assert out is dw and _untouched(buf, dw)
        _check(dy, tokens, vocab, parts, float(torch.tensor(scale)), dw)
        again = binding.solon_embedding_backward(dy, tokens, vocab, partitions=parts, scale=scale, dweight=torch.empty_like(dw).contiguous())
        assert torch.equal(again, dw)


@pytest.mark.parametrize("n,parts,cols,vocab", [(64, 3, 33, 20), (2500, 2, 64, 300), (10_000, 1, 130, 4), (0, 2, 8, 5)])
@pytest.mark.parametrize("grad", ["f32", "bf16", "f64"])
def test_accumulate(n, parts, cols, vocab, grad):
    g = _gen(n)
    dy = torch.randn((n * parts, cols), device="cuda", generator=g)
    tokens = torch.randint(-1, vocab, (n * parts,), device="cuda", generator=g)
    before = torch.randn((parts, vocab * cols), device="cuda", generator=g).to(TYPES[grad])
    got = binding.solon_embedding_backward(dy, tokens, vocab, partitions=parts, scale=1.5, dweight=before.clone(), accumulate=True)
    _check(dy, tokens, vocab, parts, 1.5, got, before)


@pytest.mark.parametrize("n,cols", [(200, 40), (4096, 64), (33_000, 32), (65_536, 130)])
@pytest.mark.parametrize("case", ["one token", "two tokens", "rising", "falling", "none"])
def test_orders(n, cols, case):
    """All rows of one token (a run over every block), alternating tokens, sorted both ways, no row that counts; integers, so sums are exact."""
    vocab = n + 5
    i = torch.arange(n, device="cuda")
    tokens = {"one token": torch.full_like(i, 3), "two tokens": i % 2, "rising": i, "falling": n - i, "none": torch.full_like(i, -5)}[case]
    if cols * vocab > 1 << 22 and case in ("rising", "falling"):
        cols = 8
    dy = torch.randint(-8, 9, (n, cols), device="cuda", generator=_gen(n)).float()
    got = binding.solon_embedding_backward(dy, tokens, vocab)
    want = torch.zeros((vocab, cols), dtype=torch.float64, device="cuda")
    want.index_add_(0, tokens.clamp(min=0), torch.where(tokens[:, None] >= 0, dy, 0.0).double())
    assert torch.equal(got.view(vocab, cols).double(), want)


def test_not_finite():
    """What is not finite goes into its token's row and column alone; rows that count nowhere may hold anything."""
    dy = torch.ones((100, 9), device="cuda")
    tokens = torch.arange(100, device="cuda") % 10
    dy[3, 4], dy[15, 2] = NAN, float("inf")
    tokens[40] = -1
    dy[40] = NAN
    got = binding.solon_embedding_backward(dy, tokens, 10).view(10, 9)
    assert got[3, 4].isnan() and got[5, 2] == float("inf") and int((~torch.isfinite(got)).sum()) == 2
    assert (got[0, :] == 9).all()


def test_differences():
    """The gradient of sum(c * out) with respect to a weight is what a change of that weight does to it (exact: it is linear, and sums of
    these integers are)."""
    g = _gen(9)
    weight = torch.randint(-9, 10, (12, 6), device="cuda", generator=g).float()
    tokens = torch.randint(-1, 12, (50,), device="cuda", generator=g)
    c = torch.randint(-9, 10, (50, 6), device="cuda", generator=g).float()
    grad = binding.solon_embedding_backward(c, tokens, 12, scale=2.0).view(12, 6)

    def value(w):
        return float((c * binding.solon_embedding_forward(w, tokens, scale=2.0)).sum())

    for v, col in ((0, 0), (3, 5), (11, 2)):
        up = weight.clone()
        up[v, col] += 1
        assert value(up) - value(weight) == float(grad[v, col])


def test_offsets_beyond_32_bits():
    """Gradient rows that start beyond 2^31 elements (8.6 GB of bfloat16 gradients)."""
    vocab, cols, parts = 34_000, 32_768, 4
    dw = torch.full((parts, vocab * cols), 7.0, dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([vocab - 1, 0, 5, 33_999], device="cuda")
    dy = torch.arange(1, 5, device="cuda").float()[:, None].expand(4, cols).to(torch.bfloat16).contiguous()
    binding.solon_embedding_backward(dy, tokens, vocab, partitions=parts, dweight=dw)
    part = dw.view(parts, vocab, cols)
    for k in range(parts):
        assert (part[k, int(tokens[k])] == k + 1).all()
        assert int(part[k].count_nonzero()) == cols
    y = binding.solon_embedding_forward(part[3], tokens[3:])
    assert (y == 4).all()


def test_on_a_stream_and_in_a_graph():
    g = _gen(4)
    dy = torch.randn((3000, 72), device="cuda", generator=g)
    tokens = torch.randint(0, 50, (3000,), device="cuda", generator=g)
    weight = torch.randn((50, 72), device="cuda", generator=g)
    want = binding.solon_embedding_backward(dy, tokens, 50, partitions=3)
    rows = binding.solon_embedding_forward(weight, tokens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dw, out = torch.zeros_like(want), torch.zeros_like(rows)
    with torch.cuda.stream(side):
        binding.solon_embedding_backward(dy, tokens, 50, partitions=3, dweight=dw)
        binding.solon_embedding_forward(weight, tokens, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(dw, want) and torch.equal(out, rows)
    graphs = []
    for _ in range(2):                         # two graphs that may be replayed in any order
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.solon_embedding_backward(dy, tokens, 50, partitions=3, dweight=dw)
            binding.solon_embedding_forward(weight, tokens, out=out)
        graphs.append(graph)
    tokens.copy_(tokens.flip(0))
    dy.copy_(dy.flip(0) * 2)
    for graph in graphs + graphs[::-1]:
        dw.fill_(NAN)
        out.fill_(NAN)
        graph.replay()
        assert torch.equal(out, weight[tokens])
        assert torch.equal(dw, binding.solon_embedding_backward(dy, tokens, 50, partitions=3))


def test_refusals():
    weight = torch.zeros((5, 8), device="cuda")
    tokens = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        binding.solon_embedding_forward(weight.double(), tokens.int())
    with pytest.raises(binding.SolonError):
        binding.solon_embedding_forward(weight.double(), tokens)
    with pytest.raises(ValueError):
        binding.solon_embedding_forward(weight.t(), tokens)
    with pytest.raises(ValueError):
        binding.solon_embedding_forward(weight, tokens, out=torch.zeros((3, 9), device="cuda"))
    with pytest.raises(ValueError):
        binding.solon_embedding_forward(weight, tokens.cpu())
    dy = torch.zeros((3, 8), device="cuda")
    with pytest.raises(binding.SolonError):
        binding.solon_embedding_backward(dy, tokens, 5, partitions=2)
    with pytest.raises(ValueError):
        binding.solon_embedding_backward(dy, tokens, 5, dweight=torch.zeros((1, 39), device="cuda"))
    with pytest.raises(ValueError):
        binding.solon_embedding_backward(dy, tokens, 5, accumulate=True)
    with pytest.raises(ValueError):
        binding.solon_embedding_backward(dy, tokens[:2], 5)
    with pytest.raises(binding.SolonError):
        binding.solon_embedding_backward(dy, tokens, 5, dweight=torch.zeros((1, 40), dtype=torch.float16, device="cuda"))
    assert binding.solon_embedding_forward(weight, tokens[:0]).shape == (0, 8)
    assert (binding.solon_embedding_backward(dy[:0], tokens[:0], 5, partitions=2) == 0).all()
