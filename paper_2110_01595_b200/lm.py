"""Closed loop on a token model: every step's partition gradients of a next-token model go through Solon and AdamW.

Per step, for P partitions of n tokens each: embed (solon_embedding_forward) -> layer norm (solon_layernorm_forward) -> logits -> log probabilities of
the next tokens (solon_token_logprobs) -> gradients, each partition's into its row of the P x d gradient matrix
(solon_token_logprobs_backward, solon_layernorm_backward and solon_embedding_backward by partitions) -> coded vectors (solon_encode) -> an adversary
overwrites some nodes' rows -> robust decode (solon_decode) -> AdamW on all parameters from the decoded sum
(solon_adamw_step), skipped on the device if the decode failed.

The model is the smallest that has every part: an embedding, one layer norm, one output matrix.  Products of matrices are plain
library ones, written straight into the gradient matrix; with fused_head the logits are never in memory (solon_head_logprobs and its
gradient, which goes straight into the gradient matrix too).
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

    bits: width of AdamW's state.  max_norm: clip of the mean gradient's norm (0: none).  fused_head: loss and gradient straight
    from hidden states and output matrix: P n V logits less in memory, and in float32 less time (both passes on 2047 x 1001 over 50001 tokens
    2.3 ms against 10.5 with the library's float32 products, on 2880 x 333 over 2003 0.18 against 0.31)."""

    def __init__(self, plan: binding.Plan, vocab: int, width: int, seed: int = 0, bits: int = 32, lr: float = 1e-2, weight_decay: float = 0.0,
                 max_norm: float = 1.0, attack: str = "flip10", fused_head: bool = False):
        if plan.d != parameter_count(vocab, width) or plan.dtype != "f32":
            raise ValueError(f"the plan must be float32 with d = {parameter_count(vocab, width)}")
        self.plan, self.vocab, self.width, self.lr, self.max_norm, self.attack = plan, vocab, width, float(lr), float(max_norm), attack
        self.fused_head = fused_head
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
        if tokens.dtype not in (torch.int32, torch.int64) or tokens.dim() > 1:
            raise ValueError(f"tokens must be a vector of int32 or int64, got {tuple(tokens.shape)} {tokens.dtype}")
        tokens = tokens.reshape(-1).long().contiguous()
        hidden = binding.solon_embedding_forward(self.embed, tokens)
        return tokens, hidden, *binding.solon_layernorm_forward(hidden, self.weight, self.bias, eps=LN_EPS)

    def partition_gradients(self, tokens, targets):
        """Fills the gradient matrix with each partition's gradient of its mean loss -log p(target); returns the rows' log p.
        tokens: P x n int32 or int64, targets: P x n int64; a negative target counts in no gradient (n still divides).  A negative token
        (padding) is a row of zeros before the layer norm and has no embedding to learn; what its target says to the other parameters counts, so
        padded positions want negative targets too.  A token beyond the vocabulary makes its row, and its partition's gradient, NaN."""
        P, n = tokens.shape
        if P != self.plan.P or targets.shape != tokens.shape:
            raise ValueError("tokens and targets must be P x n")
        V, C = self.vocab, self.width
        flat_targets = targets.reshape(-1).contiguous()
        flat_tokens, hidden, normed, mean, rstd = self._forward(tokens.reshape(-1))
        g = torch.full((P * n,), -1.0 / n, device="cuda")
        o = self.offsets
        if self.fused_head:
            scored = binding.solon_head_logprobs(normed, self.head, flat_targets)
            dnormed, _ = binding.solon_head_logprobs_backward(normed, self.head, flat_targets, scored.peak, scored.log_sum, g, partitions=P,
                                                              dweight=self.grads[:, o[3]:])
        else:
            logits = normed @ self.head.t()
            scored = binding.solon_token_logprobs(logits, flat_targets)
            dlogits = binding.solon_token_logprobs_backward(logits, flat_targets, scored.peak, scored.log_sum, g, out=logits)
            part = self.grads.as_strided((P, V, C), (self.plan.d, C, 1), o[3])
            torch.bmm(dlogits.view(P, n, V).transpose(1, 2), normed.view(P, n, C), out=part)
            dnormed = dlogits @ self.head
        dhidden, _, _ = binding.solon_layernorm_backward(dnormed, hidden, mean, rstd, self.weight, partitions=P,
                                                         dweight=self.grads[:, o[1]:o[2]], dbias=self.grads[:, o[2]:o[3]])
        binding.solon_embedding_backward(dhidden, flat_tokens, V, partitions=P, dweight=self.grads[:, :o[1]])
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
        """What the model expects after each token: (ids, log probabilities) of the top_k likeliest, and the entropy.
        tokens: a vector of int32 or int64, as partition_gradients takes them."""
        scored = binding.solon_token_logprobs(self._forward(tokens)[2] @ self.head.t(), top_k=top_k)
        return scored.top_ids, scored.top_logp, scored.entropy
