"""The token model's closed loop: its partition gradients against automatic differentiation in float64, training with
attackers against training without, and what an undecodable step leaves behind."""

import pytest
import torch

from paper_2110_01595_b200 import binding, build, lm

pytestmark = pytest.mark.gpu
P, S, M, R = 8, 1, 2, 4
V, C, N = 61, 24, 12


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _plan(seed=3):
    return binding.Plan(P, S, M, R, lm.parameter_count(V, C), seed=seed)


def _batch(step, n=N):
    """A language with structure: the next token is a fixed permutation of the current one, with some noise."""
    g = torch.Generator(device="cuda").manual_seed(1000 + step)
    tokens = torch.randint(0, V, (P, n), device="cuda", generator=g)
    targets = (tokens * 7 + 3) % V
    noise = torch.rand((P, n), device="cuda", generator=g)
    targets = torch.where(noise < 0.05, torch.randint(0, V, (P, n), device="cuda", generator=g), targets)
    return tokens, torch.where(noise > 0.97, -1, targets)


def test_partition_gradients_are_those_of_the_loss():
    """Every product and sum in the model runs over at most n, V or C terms in float32: 1e-5 of a partition's gradient norm
    is ten times their rounding (sqrt(61) 2^-24 a product, five in a row)."""
    with _plan() as plan:
        loop = lm.TokenLoop(plan, V, C, seed=1)
        loop.weight.normal_(1.0, 0.2)
        loop.bias.normal_(0.0, 0.2)
        tokens, targets = _batch(0)
        logp = loop.partition_gradients(tokens, targets)
        for k in range(P):
            w = [t.double().requires_grad_() for t in (loop.embed, loop.weight, loop.bias, loop.head)]
            h = w[0][tokens[k]]
            y = torch.nn.functional.layer_norm(h, (C,), w[1], w[2], lm.LN_EPS)
            lp = torch.log_softmax(y @ w[3].t(), dim=1)
            keep = targets[k] >= 0
            picked = torch.where(keep, lp.gather(1, targets[k].clamp(min=0)[:, None])[:, 0], 0.0)
            want = torch.cat([g.reshape(-1) for g in torch.autograd.grad(-picked.sum() / N, w)])
            assert float((loop.grads[k].double() - want).norm()) <= 1e-5 * float(want.norm())
            assert float((logp.view(P, N)[k].double() - picked.detach()).abs().max()) <= 1e-5


def test_training_with_attackers_equals_training_without():
    """The decoded sum is exact to float32 rounding whatever the attackers send; AdamW's first steps, about lr times the sign of
    a gradient, turn that into up to lr per step only where a gradient is itself rounding noise, so the runs are compared by
    their losses and the bulk of their weights."""
    with _plan() as plan, _plan() as attacked_plan:
        clean, attacked = lm.TokenLoop(plan, V, C, seed=1), lm.TokenLoop(attacked_plan, V, C, seed=1)
        losses = []
        for t in range(40):
            tokens, targets = _batch(t)
            a = clean.step(tokens, targets)
            b = attacked.step(tokens, targets, attackers=[t % 4, 4 + (t * 3) % 4])
            losses.append((-float(a.mean()), -float(b.mean())))
            assert attacked_plan.decode_status() == 0
            assert attacked.mask.nonzero().flatten().tolist() == [t % 4, 4 + (t * 3) % 4]
        assert losses[-1][0] < 0.6 * losses[0][0]
        assert all(abs(x - y) <= 1e-3 * x for x, y in losses)
        assert float((clean.flat - attacked.flat).abs().median()) <= 1e-5
        assert clean.optimizer.steps() == attacked.optimizer.steps() == (40, 0)
        ids, top_logp, entropy = attacked.next_tokens(torch.arange(V, device="cuda"), top_k=3)
        assert float((ids[:, 0] == (torch.arange(V, device="cuda") * 7 + 3) % V).float().mean()) > 0.5
        assert (top_logp[:, 0] >= top_logp[:, 1]).all() and (entropy > 0).all()


def test_training_with_8_bit_states():
    with _plan() as plan:
        loop = lm.TokenLoop(plan, V, C, seed=1, bits=8)
        losses = [-float(loop.step(*_batch(t), attackers=[2]).mean()) for t in range(40)]
        assert losses[-1] < 0.65 * losses[0]


def test_a_failed_decode_leaves_the_model_as_it_is(monkeypatch):
    # (noise: three rows of a group that follow one rule, as the scaled ones do, would outvote the fourth)
    monkeypatch.setattr(lm, "attack_rows", lambda coded, idx, kind: torch.randn((len(idx), coded.shape[1]), device="cuda") * 50)
    with _plan() as plan:
        loop = lm.TokenLoop(plan, V, C, seed=1)
        before = loop.flat.clone()
        loop.step(*_batch(0), attackers=[0, 1, 2])              # three in one group, one is tolerated
        assert plan.decode_status() == binding.ERR_UNDECODABLE
        assert torch.equal(loop.flat, before) and loop.optimizer.steps() == (0, 1)
        loop.step(*_batch(0), attackers=[1])
        assert not torch.equal(loop.flat, before) and loop.optimizer.steps() == (1, 1)


def test_refusals():
    with binding.Plan(P, S, M, R, 1000, seed=1) as plan:
        with pytest.raises(ValueError):
            lm.TokenLoop(plan, V, C)
    with _plan() as plan:
        loop = lm.TokenLoop(plan, V, C)
        tokens, targets = _batch(0)
        with pytest.raises(ValueError):
            loop.step(tokens[:4], targets[:4])
