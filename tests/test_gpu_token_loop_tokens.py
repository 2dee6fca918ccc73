"""What the token loop takes as tokens: integers of either width at any stride, and tokens outside the vocabulary."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build, lm

pytestmark = pytest.mark.gpu
P, S, M, R = 8, 1, 2, 4
V, C, N = 61, 24, 12


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.fixture(params=[False, True], ids=["logits", "fused"])
def loop(request):
    with binding.Plan(P, S, M, R, lm.parameter_count(V, C), seed=3) as plan:
        loop = lm.TokenLoop(plan, V, C, seed=1, fused_head=request.param)
        loop.weight.normal_(1.0, 0.2)
        loop.bias.normal_(0.0, 0.2)
        yield loop


def _batch():
    g = torch.Generator(device="cuda").manual_seed(5)
    return torch.randint(0, V, (P, N), device="cuda", generator=g), torch.randint(-1, V, (P, N), device="cuda", generator=g)


def test_widths_and_strides_of_tokens(loop):
    tokens, targets = _batch()
    logp = loop.partition_gradients(tokens, targets).clone()
    grads = loop.grads.clone()
    apart = torch.full((P, 2 * N), 7, dtype=torch.int64, device="cuda")
    apart[:, ::2] = tokens
    turned = tokens.t().contiguous().t()
    for x in (tokens.int(), apart[:, ::2], apart.int()[:, ::2], turned):
        loop.grads.fill_(3.0)
        assert torch.equal(loop.partition_gradients(x, targets), logp) and torch.equal(loop.grads, grads)
    apart_targets = torch.full((P, 2 * N), 7, dtype=torch.int64, device="cuda")
    apart_targets[:, ::2] = targets
    assert torch.equal(loop.partition_gradients(tokens, apart_targets[:, ::2]), logp)
    line = tokens[0].contiguous()
    want = loop.next_tokens(line, top_k=3)
    for x in (line.int(), apart[0, ::2], apart.int()[0, ::2], turned[0]):
        for a, b in zip(loop.next_tokens(x, top_k=3), want):
            assert torch.equal(a, b)
    one = loop.next_tokens(line[0], top_k=3)                      # a single token without an axis
    assert one[0].shape == (1, 3) and torch.equal(one[0], loop.next_tokens(line[:1], top_k=3)[0])


def test_refused_tokens(loop):
    tokens, targets = _batch()
    for x in (tokens.float(), tokens.bool()):
        with pytest.raises(ValueError):
            loop.partition_gradients(x, targets)
    with pytest.raises(ValueError):
        loop.partition_gradients(tokens, targets.int())
    with pytest.raises(ValueError):
        loop.next_tokens(tokens)                                  # a vector, not a batch of them


def test_tokens_outside_the_vocabulary(loop):
    """A negative token is a row of zeros: its target's gradient reaches head and layer norm, no embedding (1e-5 of a partition's norm as in the loop's
    other tests). One beyond the vocabulary is seen: NaN in its partition, in no other."""
    tokens, targets = _batch()
    tokens[:, ::5] = -3
    logp = loop.partition_gradients(tokens, targets)
    for k in range(P):
        w = [t.double().requires_grad_() for t in (loop.embed, loop.weight, loop.bias, loop.head)]
        x = torch.where(tokens[k][:, None] >= 0, w[0][tokens[k].clamp(min=0)], 0.0)
        y = torch.nn.functional.layer_norm(x, (C,), w[1], w[2], lm.LN_EPS)
        lp = torch.log_softmax(y @ w[3].t(), dim=1)
        picked = torch.where(targets[k] >= 0, lp.gather(1, targets[k].clamp(min=0)[:, None])[:, 0], 0.0)
        want = torch.cat([g.reshape(-1) for g in torch.autograd.grad(-picked.sum() / N, w)])
        assert float((loop.grads[k].double() - want).norm()) <= 1e-5 * float(want.norm())
        assert float((logp.view(P, N)[k].double() - picked.detach()).abs().max()) <= 1e-5
    clean = loop.grads.clone()
    tokens[2, 1] = V
    targets[2, 1] = 3
    logp = loop.partition_gradients(tokens, targets).view(P, N)
    keep = torch.arange(P, device="cuda") != 2
    assert logp[2, 1].isnan() and torch.isfinite(logp[keep]).all() and loop.grads[2].isnan().any()
    assert torch.equal(loop.grads[keep], clean[keep])
