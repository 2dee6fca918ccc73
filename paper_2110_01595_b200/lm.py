"""Closed loop on a token model: every step's partition gradients of a next-token model go through Solon and AdamW.

Per step, for P partitions of n tokens each: embed -> layer norm (solon_layernorm_forward) -> logits -> log probabilities of
the next tokens (solon_token_logprobs) -> gradients, each partition's into its row of the P x d gradient matrix
(solon_token_logprobs_backward, solon_layernorm_backward by partitions) -> coded vectors (solon_encode) -> an adversary
overwrites some nodes' rows -> robust decode (solon_decode) -> AdamW on all parameters from the decoded sum
(solon_adamw_step), skipped on the device if the decode failed.

The model is the smallest that has every part: an embedding, one layer norm, one output matrix.  Products of matrices are plain
library ones, written straight into the gradient matrix.
"""

from __future__ import annotations

import torch

from . import binding
from .sgd import attack_rows

LN_EPS = 1e-5


def parameter_count(vocab: int, width: int) -> int:
    """d of the plan: embedding, layer norm's weight and bias, output matrix."""
    return 2 * vocab * width + 2 * width


class TokenLoop:
    """State of one run: parameters (views of one vector, in the order of the gradient), optimizer, buffers.

    bits: width of AdamW's state.  max_norm: clip of the mean gradient's norm (0: none)."""

    def __init__(self, plan: binding.Plan, vocab: int, width: int, seed: int = 0, bits: int = 32, lr: float = 1e-2, weight_decay: float = 0.0,
                 max_norm: float = 1.0, attack: str = "flip10"):
        if plan.d != parameter_count(vocab, width) or plan.dtype != "f32":
            raise ValueError(f"the plan must be float32 with d = {parameter_count(vocab, width)}")
        self.plan, self.vocab, self.width, self.lr, self.max_norm, self.attack = plan, vocab, width, float(lr), float(max_norm), attack
        plan.set_fresh_projections(True)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.flat = torch.zeros(plan.d, device="cuda")
        sizes = [vocab * width, width, width, vocab * width]
        embed, weight, bias, head = self.flat.split(sizes)
        embed.normal_(generator=g)
        weight.fill_(1.0)
        head.normal_(0.0, width ** -0.5, generator=g)
        self.embed, self.weight, self.bias, self.head = embed.view(vocab, width), weight, bias, head.view(vocab, width)
        self.optimizer = binding.AdamW([embed, weight, bias, head], bits=bits, weight_decay=[weight_decay, 0.0, 0.0, weight_decay], seed=seed)
        self.offsets = [0, sizes[0], sizes[0] + width, sizes[0] + 2 * width]
        self.grads = torch.empty((plan.P, plan.d), device="cuda")
        self.coded = torch.empty((plan.P, plan.d_c), device="cuda")
        self.agg = torch.empty(plan.d, device="cuda")
        self.mask = torch.empty(plan.P, dtype=torch.uint8, device="cuda")

    def _forward(self, tokens):
        hidden = self.embed.index_select(0, tokens)
        normed, mean, rstd = binding.solon_layernorm_forward(hidden, self.weight, self.bias, eps=LN_EPS)
        return hidden, normed, mean, rstd, normed @ self.head.t()

    def partition_gradients(self, tokens, targets):
        """Fills the gradient matrix with each partition's gradient of its mean loss -log p(target); returns the rows' log p.
        tokens, targets: P x n int64; a negative target counts in no gradient (n still divides)."""
        P, n = tokens.shape
        if P != self.plan.P or targets.shape != tokens.shape:
            raise ValueError("tokens and targets must be P x n")
        V, C = self.vocab, self.width
        flat_targets = targets.reshape(-1)
        hidden, normed, mean, rstd, logits = self._forward(tokens.reshape(-1))
        scored = binding.solon_token_logprobs(logits, flat_targets)
        g = torch.full((P * n,), -1.0 / n, device="cuda")
        dlogits = binding.solon_token_logprobs_backward(logits, flat_targets, scored.peak, scored.log_sum, g, out=logits)
        o = self.offsets
        part = self.grads.as_strided((P, V, C), (self.plan.d, C, 1), o[3])
        torch.bmm(dlogits.view(P, n, V).transpose(1, 2), normed.view(P, n, C), out=part)
        dhidden, _, _ = binding.solon_layernorm_backward(dlogits @ self.head, hidden, mean, rstd, self.weight, partitions=P,
                                                         dweight=self.grads[:, o[1]:o[2]], dbias=self.grads[:, o[2]:o[3]])
        part = self.grads.as_strided((P, V, C), (self.plan.d, C, 1), 0)
        part.zero_()
        rows = torch.arange(P, device="cuda").repeat_interleave(n)
        part.index_put_((rows, tokens.reshape(-1)), dhidden, accumulate=True)
        return scored.logp

    def step(self, tokens, targets, attackers=()):
        """One iteration; `attackers`: the nodes that send something else.  Returns the rows' log probabilities (before the step)."""
        logp = self.partition_gradients(tokens, targets)
        self.plan.encode(self.grads, self.coded)
        if len(attackers):
            idx = torch.tensor(list(attackers), dtype=torch.long, device="cuda")
            self.coded.index_copy_(0, idx, attack_rows(self.coded, idx, self.attack))
        self.plan.decode(self.coded, self.agg, self.mask)
        self.optimizer.step(self.agg, lr=self.lr, grad_scale=1.0 / self.plan.P, max_norm=self.max_norm, plan=self.plan)
        return logp

    def next_tokens(self, tokens, top_k: int = 5):
        """What the model expects after each token: (ids, log probabilities) of the top_k likeliest, and the entropy."""
        scored = binding.solon_token_logprobs(self._forward(tokens)[4], top_k=top_k)
        return scored.top_ids, scored.top_logp, scored.entropy
