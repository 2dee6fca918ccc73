"""The token model's closed loop with the loss straight from hidden states and output matrix: the embedding's lookup and gradient, the layer
norm, the head and AdamW run together as they are used, against automatic differentiation in float64 and against the loop with the logits in memory."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build, lm

pytestmark = pytest.mark.gpu
P, S, M, R = 8, 1, 2, 4


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _batch(step, V, n):
    g = torch.Generator(device="cuda").manual_seed(1000 + step)
    tokens = torch.randint(0, V, (P, n), device="cuda", generator=g)
    targets = (tokens * 7 + 3) % V
    return tokens, torch.where(torch.rand((P, n), device="cuda", generator=g) > 0.97, -1, targets)


@pytest.mark.parametrize("V,C,n", [(61, 24, 12), (61, 24, 2), (1003, 72, 40), (300, 33, 64)])
def test_partition_gradients_are_those_of_the_loss(V, C, n):
    """Every product and sum in the model runs over at most n, V or C terms; elements in two pieces keep 22 bits, so a term is off by 2^-20 at
    most and a partition's gradient, through the head, the layer norm and the embedding, by 1e-5 of its norm: ten times what five such
    steps of independent terms come to."""
    with binding.Plan(P, S, M, R, lm.parameter_count(V, C), seed=3) as plan:
        loop = lm.TokenLoop(plan, V, C, seed=1, fused_head=True)
        loop.weight.normal_(1.0, 0.2)
        loop.bias.normal_(0.0, 0.2)
        tokens, targets = _batch(0, V, n)
        logp = loop.partition_gradients(tokens, targets)
        for k in range(P):
            w = [t.double().requires_grad_() for t in (loop.embed, loop.weight, loop.bias, loop.head)]
            y = torch.nn.functional.layer_norm(w[0][tokens[k]], (C,), w[1], w[2], lm.LN_EPS)
            lp = torch.log_softmax(y @ w[3].t(), dim=1)
            picked = torch.where(targets[k] >= 0, lp.gather(1, targets[k].clamp(min=0)[:, None])[:, 0], 0.0)
            want = torch.cat([g.reshape(-1) for g in torch.autograd.grad(-picked.sum() / n, w)])
            assert float((loop.grads[k].double() - want).norm()) <= 1e-5 * float(want.norm())
            assert float((logp.view(P, n)[k].double() - picked.detach()).abs().max()) <= 1e-5


def test_a_run_with_attackers_equals_the_loop_with_logits():
    """Same model, same batches, attackers in one of the two: the decoded sums are the same to float32 rounding, so the losses follow each other."""
    V, C, n = 61, 24, 12
    d = lm.parameter_count(V, C)
    with binding.Plan(P, S, M, R, d, seed=3) as plan, binding.Plan(P, S, M, R, d, seed=3) as other:
        fused, plain = lm.TokenLoop(plan, V, C, seed=1, fused_head=True), lm.TokenLoop(other, V, C, seed=1)
        for t in range(30):
            tokens, targets = _batch(t, V, n)
            a = fused.step(tokens, targets, attackers=[t % 4, 4 + t % 3])
            b = plain.step(tokens, targets)
            assert abs(float(a.mean()) - float(b.mean())) <= 1e-3 * abs(float(b.mean()))
            assert plan.decode_status() == 0 and fused.mask.nonzero().flatten().tolist() == [t % 4, 4 + t % 3]
        assert fused.optimizer.steps() == (30, 0)
        ids, top_logp, entropy = fused.next_tokens(torch.arange(V, device="cuda"), top_k=2)
        assert ids.shape == (V, 2) and (top_logp[:, 0] >= top_logp[:, 1]).all() and (entropy > 0).all()


def test_tied_weights():
    """Embedding and output matrix in one: the embedding's gradient is added to the head's, in place, per partition."""
    V, C, n = 157, 40, 30
    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.randn((V, C), device="cuda", generator=g) * 0.3
    tokens = torch.randint(0, V, (P * n,), device="cuda", generator=g)
    targets = torch.randint(-1, V, (P * n,), device="cuda", generator=g)
    h = binding.solon_embedding_forward(w, tokens, scale=2.0)
    r = binding.solon_head_logprobs(h, w, targets)
    scale = torch.full((P * n,), -1.0 / n, device="cuda")
    grads = torch.full((P, V * C + 10), 7.0, device="cuda")
    dh, dw = binding.solon_head_logprobs_backward(h, w, targets, r.peak, r.log_sum, scale, partitions=P, dweight=grads[:, 5:-5])
    binding.solon_embedding_backward(dh, tokens, V, partitions=P, scale=2.0, dweight=dw, accumulate=True)
    assert (grads[:, :5] == 7).all() and (grads[:, -5:] == 7).all()
    for k in range(P):
        q = slice(k * n, (k + 1) * n)
        x = w.double().requires_grad_()
        lp = torch.log_softmax(2.0 * x[tokens[q]] @ x.t(), dim=1)
        picked = torch.where(targets[q] >= 0, lp.gather(1, targets[q].clamp(min=0)[:, None])[:, 0], 0.0)
        want, = torch.autograd.grad(-picked.sum() / n, x)
        assert float((dw[k].view(V, C).double() - want).norm()) <= 1e-5 * float(want.norm())
