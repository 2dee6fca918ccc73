"""What is timed of the two ends of a token model: the embedding lookup and its gradient, and the log probabilities of the next tokens
straight from hidden states and output matrix, without logits in memory, with their gradient.

Each case is one call of one operator as a training loop (or a server, for few rows) around the encode / decode path makes it.  With
``own`` false the operators are computed in their plain form by elementary torch operations in float32; with ``own`` true by the
library's entry points in ``paper_2110_01595_b200.binding``.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------------------------------ cases


def listed():
    return [
        # one new token of a served model: latency
        {"name": "emb_fwd_1x2048_bf16", "op": "emb_fwd", "rows": 1, "cols": 2048, "vocab": 131_072, "parts": 1, "dtype": "bf16", "grad": "f32", "scaled": False},
        # a training batch's tokens, rows scaled by the root of their width
        {"name": "emb_fwd_16384x4096_bf16", "op": "emb_fwd", "rows": 16_384, "cols": 4096, "vocab": 32_768, "parts": 1, "dtype": "bf16", "grad": "f32", "scaled": True},
        # 45 partitions of 64 tokens, odd width in float32, gradients into the rows of the gradient matrix (off 16-byte boundaries)
        {"name": "emb_bwd_45x64_2003x1001_f32", "op": "emb_bwd", "rows": 45 * 64, "cols": 1001, "vocab": 2003, "parts": 45, "dtype": "f32", "grad": "f32", "scaled": False},
        # 15 partitions of 2048 tokens: 2 GB of gradient matrix, most of it zeros
        {"name": "emb_bwd_15x2048_32768x1024_bf16", "op": "emb_bwd", "rows": 15 * 2048, "cols": 1024, "vocab": 32_768, "parts": 15, "dtype": "bf16", "grad": "f32", "scaled": True},
        # one large batch without partitions, gradients in bfloat16 for the optimizer, odd vocabulary
        {"name": "emb_bwd_32768_50001x2048_bf16", "op": "emb_bwd", "rows": 32_768, "cols": 2048, "vocab": 50_001, "parts": 1, "dtype": "bf16", "grad": "bf16", "scaled": False},
        # one served token over a large vocabulary: the output matrix is read once
        {"name": "head_fwd_1_131072x2048_bf16", "op": "head_fwd", "rows": 1, "cols": 2048, "vocab": 131_072, "parts": 1, "dtype": "bf16", "grad": "f32", "entropy": False},
        # scoring a served batch
        {"name": "head_fwd_96_131072x2048_bf16", "op": "head_fwd", "rows": 96, "cols": 2048, "vocab": 131_072, "parts": 1, "dtype": "bf16", "grad": "f32", "entropy": False},
        # a float32 model, odd sizes
        {"name": "head_fwd_2047_50001x1001_f32", "op": "head_fwd", "rows": 2047, "cols": 1001, "vocab": 50_001, "parts": 1, "dtype": "f32", "grad": "f32", "entropy": False},
        # the loss of a training batch
        {"name": "head_fwd_8192_32768x2048_bf16", "op": "head_fwd", "rows": 8192, "cols": 2048, "vocab": 32_768, "parts": 1, "dtype": "bf16", "grad": "f32", "entropy": False},
        # 45 partitions of 64 tokens of a small float32 model, odd sizes, with an entropy term
        {"name": "head_bwd_45x64_2003x333_f32", "op": "head_bwd", "rows": 45 * 64, "cols": 333, "vocab": 2003, "parts": 45, "dtype": "f32", "grad": "f32", "entropy": True},
        # 15 partitions of 512 tokens, gradients into the float32 gradient matrix
        {"name": "head_bwd_15x512_16384x1024_bf16", "op": "head_bwd", "rows": 15 * 512, "cols": 1024, "vocab": 16_384, "parts": 15, "dtype": "bf16", "grad": "f32", "entropy": False},
        # one large batch without partitions, gradients in bfloat16 for the optimizer
        {"name": "head_bwd_8192_32768x2048_bf16", "op": "head_bwd", "rows": 8192, "cols": 2048, "vocab": 32_768, "parts": 1, "dtype": "bf16", "grad": "bf16", "entropy": False},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def draw(rng):
    op = rng.choice(["emb_fwd", "emb_bwd", "emb_bwd", "head_fwd", "head_fwd", "head_bwd", "head_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    emb = op.startswith("emb")
    cols = _spread(rng, 60, 8_000 if emb else 4_096)
    if rng.random() < 0.6:
        cols = max(64, cols // 64 * 64)
    vocab = _spread(rng, 1_000, min(200_000, 400_000_000 // cols))
    if rng.random() < 0.5:
        vocab = max(1_024, vocab // 128 * 128)
    grad = "bf16" if dtype == "bf16" and rng.random() < 0.3 else "f32"
    parts = 1
    if op.endswith("bwd") and rng.random() < 0.6:
        parts = min(rng.choice([4, 15, 45]), max(1, 500_000_000 // (vocab * cols)))
    if emb:
        most = min(65_536, 67_000_000 // cols)
    else:
        most = min(16_384, 268_000_000 // vocab, 550_000_000_000 // (vocab * cols))
        if dtype == "f32":
            most = max(1, most // 2)
    rows = parts * max(1, _spread(rng, 1, most) // parts)
    case = {"op": op, "rows": rows, "cols": cols, "vocab": vocab, "parts": parts, "dtype": dtype, "grad": grad}
    return case | ({"scaled": rng.random() < 0.5} if emb else {"entropy": op == "head_bwd" and rng.random() < 0.4})


def work(case):
    op, size, gsize = case["op"], SIZES[case["dtype"]], SIZES[case["grad"]]
    rows, cols, vocab = case["rows"], case["cols"], case["vocab"]
    weights = case["parts"] * vocab * cols
    if op == "emb_fwd":
        return {"bytes": 2 * rows * cols * size + 8 * rows, "flops": rows * cols}
    if op == "emb_bwd":
        return {"bytes": rows * cols * size + 8 * rows + weights * gsize, "flops": rows * cols}
    if op == "head_fwd":
        return {"bytes": (rows + vocab) * cols * size + 24 * rows, "flops": 2 * rows * cols * vocab}
    return {"bytes": (2 * rows + vocab) * cols * size + weights * gsize + 24 * rows, "flops": 6 * rows * cols * vocab}


# ------------------------------------------------------------------------------------------ inputs


def _matrix(case):
    """The partition-gradient matrix: a row for each partition, this layer's weights behind a layer norm's weight and bias."""
    cols = case["cols"]
    return torch.zeros((case["parts"], 2 * cols + case["vocab"] * cols), device="cuda", dtype=DTYPES[case["grad"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, rows, cols, vocab, dt = case["op"], case["rows"], case["cols"], case["vocab"], DTYPES[case["dtype"]]
    if op in ("emb_fwd", "emb_bwd"):
        # tokens as text has them: the r-th likeliest with a probability of about 1 / r, likely ones spread over the vocabulary; some padding
        rank = torch.exp(torch.rand(rows, device="cuda", generator=g) * math.log(vocab)).long().clamp(max=vocab) - 1
        tokens = (rank * 7919 + 13) % vocab
        if rows > 8:
            tokens[torch.rand(rows, device="cuda", generator=g) < 0.03] = -1
        state = {"case": case, "tokens": tokens, "scale": math.sqrt(cols) if case["scaled"] else 1.0}
        if op == "emb_fwd":
            return state | {"weight": (torch.randn((vocab, cols), device="cuda", generator=g) * cols ** -0.5).to(dt)}
        return state | {"dy": (torch.randn((rows, cols), device="cuda", generator=g) / 64).to(dt), "matrix": _matrix(case)}
    weight = torch.randn((vocab, cols), device="cuda", generator=g) * (1.5 / math.sqrt(cols))
    targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    # normed hidden states that lean towards their targets, as a trained model's do
    hidden = torch.randn((rows, cols), device="cuda", generator=g) + weight[targets] * (torch.rand((rows, 1), device="cuda", generator=g) * 4)
    weight, hidden = weight.to(dt), hidden.to(dt)
    if rows > 8:
        targets[torch.rand(rows, device="cuda", generator=g) < 0.06] = -1
    state = {"case": case, "hidden": hidden, "weight": weight, "targets": targets}
    if op == "head_bwd":
        s = _plain_head_fwd(state)
        n = rows // case["parts"]
        state |= {"peak": s["peak"], "log_sum": s["log_sum"], "entropy": s["entropy"],
                  "g_logp": -torch.rand(rows, device="cuda", generator=g) / n,
                  "g_entropy": torch.randn(rows, device="cuda", generator=g) / (8 * n) if case["entropy"] else None, "matrix": _matrix(case)}
    return state


# ------------------------------------------------------------------------------------------ one pass


def _plain_emb_fwd(s):
    tokens = s["tokens"]
    y = s["weight"][tokens.clamp(min=0)].float() * s["scale"]
    return {"y": torch.where(tokens[:, None] >= 0, y, 0.0).to(s["weight"].dtype)}


def _plain_emb_bwd(s):
    case, tokens, dy = s["case"], s["tokens"], s["dy"]
    parts, vocab, cols = case["parts"], case["vocab"], case["cols"]
    dw = s["matrix"][:, 2 * cols:]
    keep = tokens >= 0
    rows = torch.where(keep[:, None], dy.float() * s["scale"], 0.0)
    part = torch.arange(parts, device="cuda").repeat_interleave(case["rows"] // parts)
    if dw.dtype == torch.float32:
        into = dw.as_strided((parts, vocab, cols), (dw.stride(0), cols, 1))
        into.zero_()
    else:
        into = torch.zeros((parts, vocab, cols), device="cuda")
    into.index_put_((part, tokens.clamp(min=0)), rows, accumulate=True)
    if dw.dtype != torch.float32:
        dw.copy_(into.view(parts, -1))
    return {"dw": dw}


def _plain_head_fwd(s):
    z, t = s["hidden"].float() @ s["weight"].float().t(), s["targets"]
    peak = z.amax(dim=1, keepdim=True)
    c = z - peak
    e = torch.exp(c)
    total = e.sum(dim=1)
    log_sum = torch.log(total)
    lp = c.gather(1, t.clamp(min=0)[:, None])[:, 0] - log_sum
    return {"logp": torch.where(t >= 0, lp, 0.0), "peak": peak[:, 0], "log_sum": log_sum, "entropy": log_sum - (e * c).sum(dim=1) / total}


def _plain_head_bwd(s):
    case, t = s["case"], s["targets"]
    parts, vocab, cols = case["parts"], case["vocab"], case["cols"]
    h, w = s["hidden"].float(), s["weight"].float()
    lp = h @ w.t() - s["peak"][:, None] - s["log_sum"][:, None]
    p = torch.exp(lp)
    dz = p * torch.where(t >= 0, -s["g_logp"], 0.0)[:, None]
    if s["g_entropy"] is not None:
        dz = dz - s["g_entropy"][:, None] * (p * (lp + s["entropy"][:, None]))
    dz.scatter_add_(1, t.clamp(min=0)[:, None], torch.where(t >= 0, s["g_logp"], 0.0)[:, None])
    dw = s["matrix"][:, 2 * cols:]
    dw.copy_((dz.view(parts, -1, vocab).transpose(1, 2) @ h.view(parts, -1, cols)).view(parts, -1))
    return {"dh": (dz @ w).to(s["hidden"].dtype), "dw": dw}


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"emb_fwd": _plain_emb_fwd, "emb_bwd": _plain_emb_bwd, "head_fwd": _plain_head_fwd, "head_bwd": _plain_head_bwd}[op](state)
    from paper_2110_01595_b200 import binding

    case = state["case"]
    if op == "emb_fwd":
        return {"y": binding.solon_embedding_forward(state["weight"], state["tokens"], scale=state["scale"])}
    if op == "emb_bwd":
        return {"dw": binding.solon_embedding_backward(state["dy"], state["tokens"], case["vocab"], partitions=case["parts"], scale=state["scale"],
                                                       dweight=state["matrix"][:, 2 * case["cols"]:])}
    if op == "head_fwd":
        r = binding.solon_head_logprobs(state["hidden"], state["weight"], state["targets"])
        return {"logp": r.logp, "peak": r.peak, "log_sum": r.log_sum, "entropy": r.entropy}
    dh, dw = binding.solon_head_logprobs_backward(state["hidden"], state["weight"], state["targets"], state["peak"], state["log_sum"],
                                                  state["g_logp"], state["entropy"], state["g_entropy"], partitions=case["parts"],
                                                  dweight=state["matrix"][:, 2 * case["cols"]:])
    return {"dh": dh, "dw": dw}


# ------------------------------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    f8, op, parts = torch.float64, case["op"], case["parts"]
    n = case["rows"] // parts
    if op == "emb_fwd":
        t = s["tokens"]
        y = torch.zeros((case["rows"], case["cols"]), dtype=f8, device="cuda")
        y[t >= 0] = s["weight"][t[t >= 0]].to(f8) * s["scale"]
        return {"y": y}
    if op == "emb_bwd":
        dw = torch.zeros((parts, case["vocab"], case["cols"]), dtype=f8, device="cuda")
        for k in range(parts):
            t, dy = s["tokens"][k * n:(k + 1) * n], s["dy"][k * n:(k + 1) * n]
            dw[k].index_add_(0, t[t >= 0], dy[t >= 0].to(f8), alpha=s["scale"])
        return {"dw": dw.view(parts, -1)}
    w = s["weight"].to(f8)
    if op == "head_fwd":
        found = {"logp": [], "peak": [], "log_sum": [], "entropy": []}
        for r in range(0, case["rows"], 1024):
            z, t = s["hidden"][r:r + 1024].to(f8) @ w.t(), s["targets"][r:r + 1024]
            lp = torch.log_softmax(z, dim=1)
            big = z.max(dim=1).values
            found["logp"].append(torch.where(t < 0, 0.0, lp[torch.arange(len(t), device="cuda"), t.clamp(min=0)]))
            found["peak"].append(big)
            found["log_sum"].append(torch.logsumexp(z, dim=1) - big)
            found["entropy"].append(-torch.special.xlogy(lp.exp(), lp.exp()).sum(dim=1))
        return {k: torch.cat(v) for k, v in found.items()}
    dh, dw = torch.zeros((case["rows"], case["cols"]), dtype=f8, device="cuda"), []
    for k in range(parts):
        part = torch.zeros((case["vocab"], case["cols"]), dtype=f8, device="cuda")
        for a in range(k * n, (k + 1) * n, 2048):
            r = slice(a, min(a + 2048, (k + 1) * n))
            h, t = s["hidden"][r].to(f8), s["targets"][r]
            lp = h @ w.t() - (s["peak"][r].to(f8) + s["log_sum"][r].to(f8))[:, None]
            g = s["g_logp"][r].to(f8) * (t >= 0)
            dz = -lp.exp() * g[:, None]
            dz[torch.arange(len(t), device="cuda"), t.clamp(min=0)] += g
            if s["g_entropy"] is not None:
                dz -= s["g_entropy"][r, None].to(f8) * lp.exp() * (lp + s["entropy"][r, None].to(f8))
            dh[r] = dz @ w
            part += dz.t() @ h
        dw.append(part.view(-1))
    return {"dh": dh, "dw": torch.stack(dw)}
