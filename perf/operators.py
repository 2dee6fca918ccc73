"""What is timed of the token-model operators: layer norm, token log probabilities and the AdamW step.

Each case is one call of one operator as a training loop (or a server, for single rows) around the encode / decode path makes it.  With
``own`` false the operators are computed in their plain form by elementary torch operations in float32; with ``own`` true by the
library's entry points in ``paper_2110_01595_b200.binding``.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256                      # elements that share one window of the 8-bit state
BETA1, BETA2, EPS, LR, SEED = 0.9, 0.999, 1e-8, 1e-3, 20211004
START = 1000                     # steps done before the timed ones: a state in the middle of a training run
LN_EPS = 1e-5


# ------------------------------------------------------------------------------------------ cases


def listed():
    return [
        # the least-squares loop's iterate: one small tensor, the whole call is launch latency
        {"name": "adamw32_100k", "op": "adamw", "d": 100_000, "tensors": 1, "bits": 32, "grad": "f32", "clip": False, "copy": False},
        # ResNet-18-sized model of 62 tensors of odd sizes updated from the decoded aggregate, with norm clipping
        {"name": "adamw32_resnet18_clip", "op": "adamw", "d": 11_173_962, "tensors": 62, "bits": 32, "grad": "f32", "clip": True, "copy": False},
        # VGG-13-sized model, states in 8 bits, the bfloat16 weights of the next forward pass written in the same step
        {"name": "adamw8_vgg13_copy", "op": "adamw", "d": 28_332_000, "tensors": 26, "bits": 8, "grad": "f32", "clip": False, "copy": True},
        # the sweep's largest gradient in the 8-byte wire format, 8-bit states, clipped
        {"name": "adamw8_50m_f64_clip", "op": "adamw", "d": 50_000_000, "tensors": 12, "bits": 8, "grad": "f64", "clip": True, "copy": False},
        # one new token of a served model: latency
        {"name": "ln_fwd_1x2048_bf16", "op": "ln_fwd", "rows": 1, "cols": 2048, "parts": 1, "dtype": "bf16"},
        # a training batch's activations
        {"name": "ln_fwd_16384x4096_bf16", "op": "ln_fwd", "rows": 16384, "cols": 4096, "parts": 1, "dtype": "bf16"},
        # 45 partitions of 64 tokens, odd width in float32, weight gradients into the gradient matrix (rows off 16-byte boundaries)
        {"name": "ln_bwd_45x64x1001_f32", "op": "ln_bwd", "rows": 45 * 64, "cols": 1001, "parts": 45, "dtype": "f32"},
        # 15 partitions of 2048 tokens
        {"name": "ln_bwd_15x2048x2048_bf16", "op": "ln_bwd", "rows": 15 * 2048, "cols": 2048, "parts": 15, "dtype": "bf16"},
        # one served token over a large vocabulary: log probability of the sampled token, entropy, eight alternatives
        {"name": "logp_1x131072_bf16_top8", "op": "logp", "rows": 1, "cols": 131_072, "top": 8, "dtype": "bf16"},
        # scoring a batch with 20 alternatives a token, odd vocabulary, float32 logits
        {"name": "logp_2047x50001_f32_top20", "op": "logp", "rows": 2047, "cols": 50_001, "top": 20, "dtype": "f32"},
        # the loss of a training batch
        {"name": "logp_8192x32768_bf16", "op": "logp", "rows": 8192, "cols": 32_768, "top": 0, "dtype": "bf16"},
        # its gradient, with an entropy term
        {"name": "logp_bwd_8192x32768_bf16", "op": "logp_bwd", "rows": 8192, "cols": 32_768, "entropy": True, "dtype": "bf16"},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["adamw", "ln_fwd", "ln_bwd", "logp", "logp_bwd"])
    if op == "adamw":
        bits = rng.choice([32, 8])
        d = _spread(rng, 1_000, 50_000_000 if bits == 8 else 33_000_000)
        return {"op": op, "d": d, "tensors": min(_spread(rng, 1, 200), d // 8), "bits": bits, "grad": rng.choice(["f32", "f32", "f64", "bf16"]),
                "clip": rng.random() < 0.5, "copy": rng.random() < 0.3}
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op in ("ln_fwd", "ln_bwd"):
        cols = _spread(rng, 60, 16_000)
        if rng.random() < 0.6:
            cols = max(64, cols // 128 * 128 + 64)
        parts = 1 if op == "ln_fwd" or rng.random() < 0.4 else rng.choice([4, 15, 45])
        rows = parts * max(1, _spread(rng, 1, min(32_768, 60_000_000 // cols)) // parts)
        return {"op": op, "rows": rows, "cols": cols, "parts": parts, "dtype": dtype}
    cols = _spread(rng, 1_000, 200_000)
    if rng.random() < 0.6:
        cols = max(1_024, cols // 64 * 64)
    rows = _spread(rng, 1, min(8_192, 100_000_000 // cols))
    if op == "logp":
        return {"op": op, "rows": rows, "cols": cols, "top": rng.choice([0, 1, 5, 8, 20, 32]), "dtype": dtype}
    return {"op": op, "rows": rows, "cols": cols, "entropy": rng.random() < 0.5, "dtype": dtype}


def work(case):
    op = case["op"]
    if op == "adamw":
        d = case["d"]
        each = 8 + {"f32": 4, "f64": 8, "bf16": 2}[case["grad"]] + (16 if case["bits"] == 32 else 4 + 4) + (2 if case["copy"] else 0)
        # (8 bits: the state read and written, one byte a moment, and the moments' values handed out as bfloat16)
        return {"bytes": d * each, "flops": d * (16 + (2 if case["clip"] else 0))}
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    rows, cols = case["rows"], case["cols"]
    if op == "ln_fwd":
        return {"bytes": 2 * rows * cols * size + 8 * cols + 8 * rows, "flops": 8 * rows * cols}
    if op == "ln_bwd":
        return {"bytes": 3 * rows * cols * size + 4 * cols + 8 * rows + 8 * case["parts"] * cols, "flops": 14 * rows * cols}
    if op == "logp":
        return {"bytes": rows * cols * size + rows * (20 + 12 * case["top"]), "flops": 5 * rows * cols}
    return {"bytes": 2 * rows * cols * size + rows * 24, "flops": (8 if case["entropy"] else 4) * rows * cols}


# ------------------------------------------------------------------------------------------ inputs


def _sizes(case):
    """Tensor sizes of a model of `d` weights: log-uniform over a factor 10^4, as layers and their biases are; one tensor, or odd sizes."""
    d, n = case["d"], case["tensors"]
    rng = random.Random(n)
    weights = [math.exp(rng.random() * math.log(1e4)) for _ in range(n)]
    sizes = [max(1, int(w / sum(weights) * d)) for w in weights]
    if n <= 32 and d % 1000 == 0:
        sizes = [max(8, s // 8 * 8) for s in sizes]     # models whose layers are all multiples of eight
    sizes[sizes.index(max(sizes))] += d - sum(sizes)
    return sizes


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _encode_nearest(x, levels):
    """Blocks of float32 magnitudes -> (codes, base): the 8-bit state's form, rounded to nearest, as a checkpoint holds it."""
    bits = x.view(torch.int32)
    base = ((bits.amax(dim=1, keepdim=True) + 0xFFFFF) >> 20).clamp(min=levels) - levels
    code = (((bits + 0x80000) >> 20) - base).clamp(min=0, max=levels)
    return code, base


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "adamw":
        sizes = _sizes(case)
        d = case["d"]
        starts = torch.tensor([0] + sizes, dtype=torch.long).cumsum(0)
        blocks = [-(-s // BLOCK) for s in sizes]
        first = torch.tensor([0] + blocks, dtype=torch.long).cumsum(0)
        n_blocks = int(first[-1])
        sizes_dev = torch.tensor(sizes, device="cuda")
        # where weight e of the concatenated vector lies in the blocked state (every tensor starts a block of its own)
        slot = torch.arange(d, device="cuda") + torch.repeat_interleave((first[:-1] * BLOCK - starts[:-1]).cuda(), sizes_dev, output_size=d)
        decay = [0.0 if s < 1000 and len(sizes) > 1 else 0.1 for s in sizes]         # biases and norms are not decayed
        scale = torch.exp(torch.empty(d, device="cuda").uniform_(-9.2, -2.3, generator=g)) if d < 1000 else torch.repeat_interleave(
            torch.exp(torch.empty(len(sizes), device="cuda").uniform_(-9.2, -2.3, generator=g)), sizes_dev, output_size=d)
        grad = (torch.randn(d, device="cuda", generator=g) * scale).to(DTYPES[case["grad"]])
        p = torch.randn(d, device="cuda", generator=g) * 0.05
        m = torch.zeros(n_blocks * BLOCK, device="cuda")
        v = torch.zeros(n_blocks * BLOCK, device="cuda")
        m[slot] = torch.randn(d, device="cuda", generator=g) * scale * 0.3
        v[slot] = (torch.randn(d, device="cuda", generator=g) * 0.2 + 1).square() * scale.square()
        state = {"case": case, "p": p, "grad": grad, "slot": slot, "sizes": sizes_dev, "decay": torch.tensor(decay, device="cuda"), "step": START,
                 "max_norm": 0.5 * float((grad.double() / 15).norm()) if case["clip"] else 0.0,
                 "copy": torch.zeros(d, dtype=torch.bfloat16, device="cuda") if case["copy"] else None}
        if case["bits"] == 32:
            state["m"], state["v"] = m.view(n_blocks, BLOCK), v.view(n_blocks, BLOCK)
        else:
            mc, mb = _encode_nearest(m.abs().view(n_blocks, BLOCK), 127)
            vc, vb = _encode_nearest(v.view(n_blocks, BLOCK), 255)
            state["m"] = (mc + 128 * (m.view(n_blocks, BLOCK) < 0) * (mc > 0)).to(torch.uint8)
            state["v"] = torch.where(v.view(n_blocks, BLOCK) > 0, vc.clamp(min=1), vc).to(torch.uint8)
            state["base"] = torch.cat([mb, vb], dim=1).to(torch.int16)
        if own:      # the handle that a program keeps: it takes the tensors above as they are
            from paper_2110_01595_b200 import binding

            def views(t):
                return [t[a:b] for a, b in zip(starts[:-1].tolist(), starts[1:].tolist())]

            state["opt"] = binding.AdamW(views(p), bits=case["bits"], betas=(BETA1, BETA2), eps=EPS, weight_decay=decay, seed=SEED, step=START,
                                         copies=views(state["copy"]) if case["copy"] else None,
                                         state=(state["m"], state["v"], state.get("base")))
        return state
    rows, cols, dt = case["rows"], case["cols"], DTYPES[case["dtype"]]
    if op in ("ln_fwd", "ln_bwd"):
        x = (torch.randn((rows, cols), device="cuda", generator=g) * 1.7 + 0.3).to(dt)
        w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=g)
        b = 0.1 * torch.randn(cols, device="cuda", generator=g)
        state = {"case": case, "x": x, "w": w, "b": b}
        if op == "ln_bwd":
            dy = torch.empty((rows, cols), device="cuda", dtype=dt)
            dy.copy_(torch.randn((rows, cols), device="cuda", generator=g))
            x32 = x.float()
            mean = x32.mean(dim=1)
            rstd = torch.rsqrt((x32 - mean[:, None]).square().mean(dim=1) + LN_EPS)
            # the partition-gradient matrix: a row for each partition, this layer's weight and bias somewhere inside it
            matrix = torch.zeros((case["parts"], 2 * cols + 38), device="cuda")
            state |= {"dy": dy, "mean": mean, "rstd": rstd, "matrix": matrix}
        return state
    # logits of a peaked distribution, some tokens masked out; in training some rows carry no target
    z = torch.randn((rows, cols), device="cuda", generator=g) * 2.5
    z[:, :: max(7, cols // 50)] += 6.0
    z[:, 3 :: 101] = float("-inf")
    z = z.to(dt)
    targets = torch.randint(4, cols, (rows,), device="cuda", generator=g)
    targets = targets - ((targets - 3) % 101 == 0).long()         # no target that is masked out
    if rows > 8:
        targets[torch.rand(rows, device="cuda", generator=g) < 0.06] = -1
    state = {"case": case, "z": z, "targets": targets}
    if op == "logp_bwd":
        z32 = z.float()
        peak = z32.amax(dim=1)
        log_sum = torch.log(torch.exp(z32 - peak[:, None]).sum(dim=1))
        lp = (z32 - peak[:, None]) - log_sum[:, None]
        state |= {"peak": peak, "log_sum": log_sum, "entropy": -(torch.exp(lp) * lp.clamp(min=-1e4)).sum(dim=1),
                  "g_logp": torch.randn(rows, device="cuda", generator=g) / 64,
                  "g_entropy": torch.randn(rows, device="cuda", generator=g) / 256 if case["entropy"] else None}
    return state


# ------------------------------------------------------------------------------------------ one pass


def _mix32(h):
    """MurmurHash3's 32-bit finaliser on int64 tensors or Python ints that hold 32-bit words."""
    h = h ^ (h >> 16)
    h = (h * 0x85EBCA6B) & 0xFFFFFFFF
    h = h ^ (h >> 13)
    h = (h * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _random_words(n, step):
    """The rounding's 32 random bits of slots 0 .. n - 1 in a step."""
    key = _mix32((step * 0x9E3779B1 + (SEED & 0xFFFFFFFF)) & 0xFFFFFFFF) ^ (SEED >> 32)
    return _mix32(((torch.arange(n, device="cuda") * 0x9E3779B1) & 0xFFFFFFFF) ^ key)


def _decode(code, base):
    """8-bit magnitudes and the blocks' bases -> float32."""
    return torch.where(code > 0, (code + base) << 20, 0).view(torch.float32)


def _encode(x, levels, rand):
    bits = x.view(torch.int32)
    base = ((bits.amax(dim=1, keepdim=True) + 0xFFFFF) >> 20).clamp(min=levels) - levels
    return (((bits + rand) >> 20) - base).clamp(min=0, max=levels), base


def _plain_adamw(s):
    case = s["case"]
    s["step"] += 1
    t = s["step"]
    g = s["grad"].float() * (1 / 15)
    norm = None
    if case["clip"]:
        norm = g.square().sum().sqrt()
        g = g * (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    m, v = s["m"], s["v"]
    if case["bits"] == 8:
        base = s["base"].int()
        mc = m.int()
        m32 = _decode(mc & 127, base[:, :1]) * (1 - 2 * (mc >> 7))
        v32 = _decode(v.int(), base[:, 1:])
    else:
        m32, v32 = m, v
    gb = torch.zeros(m.numel(), device="cuda")
    gb[s["slot"]] = g
    gb = gb.view(m.shape)
    m32 = BETA1 * m32 + (1 - BETA1) * gb
    v32 = BETA2 * v32 + (1 - BETA2) * gb * gb
    step = (LR / (1 - BETA1 ** t)) * m32 / (v32.sqrt() * (1 / math.sqrt(1 - BETA2 ** t)) + EPS)
    decay = torch.repeat_interleave(1 - LR * s["decay"], s["sizes"], output_size=case["d"])
    s["p"].mul_(decay).sub_(step.view(-1)[s["slot"]])
    out = {"p": s["p"], "norm": norm}
    if case["copy"]:
        s["copy"].copy_(s["p"])
        out["copy"] = s["copy"]
    if case["bits"] == 32:
        m.copy_(m32)
        v.copy_(v32)
        return out | {"m": m, "v": v}
    rand = _random_words(m.numel(), t).view(m.shape)
    mc, mb = _encode(m32.abs(), 127, ((rand & 0xFFFF) << 4).int())
    vc, vb = _encode(v32, 255, ((rand >> 16) << 4).int())
    vc = torch.where(v32 > 0, vc.clamp(min=1), vc)
    m.copy_(mc + 128 * ((m32 < 0) & (mc > 0)))
    v.copy_(vc)
    s["base"].copy_(torch.cat([mb, vb], dim=1))
    return out | {"m": (_decode(mc, mb) * torch.where(m32 < 0, -1.0, 1.0)).bfloat16(), "v": _decode(vc, vb).bfloat16()}


def _own_adamw(s):
    opt = s["opt"]
    norm = opt.step(s["grad"], lr=LR, grad_scale=1 / 15, max_norm=s["max_norm"])
    m, v = opt.moments()             # the state itself in 32 bits, what it stands for in 8
    return {"p": s["p"], "norm": norm, "copy": s["copy"], "m": m, "v": v}


def _plain_ln_fwd(s):
    x = s["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt(c.square().mean(dim=1, keepdim=True) + LN_EPS)
    return {"y": (c * rstd * s["w"] + s["b"]).to(s["x"].dtype), "mean": mean.view(-1), "rstd": rstd.view(-1)}


def _plain_ln_bwd(s):
    case = s["case"]
    parts, cols = case["parts"], case["cols"]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * rstd
    a = dy * s["w"]
    dx = rstd * (a - a.mean(dim=1, keepdim=True) - xh * (a * xh).mean(dim=1, keepdim=True))
    dw, db = s["matrix"][:, 7:7 + cols], s["matrix"][:, 7 + cols:7 + 2 * cols]
    dw.copy_((dy * xh).view(parts, -1, cols).sum(dim=1))
    db.copy_(dy.view(parts, -1, cols).sum(dim=1))
    return {"dx": dx.to(s["x"].dtype), "dw": dw, "db": db}


def _plain_logp(s):
    z, t, k = s["z"].float(), s["targets"], s["case"]["top"]
    big = z.amax(dim=1, keepdim=True)
    c = z - big
    e = torch.exp(c)
    total = e.sum(dim=1)
    log_total = torch.log(total)
    lp = c.gather(1, t.clamp(min=0)[:, None])[:, 0] - log_total
    out = {"logp": torch.where(t >= 0, lp, 0.0), "peak": big[:, 0], "log_sum": log_total,
           "entropy": log_total - torch.where(e > 0, e * c, 0.0).sum(dim=1) / total}
    if k:
        # the k largest, of equal ones the first: one 64-bit key of the value's order and the index
        b = (z + 0.0).view(torch.int32)
        order = torch.where(b >= 0, b, b ^ 0x7FFFFFFF).long()
        key = (order << 32) + (0xFFFFFFFF - torch.arange(z.shape[1], device="cuda"))
        ids = 0xFFFFFFFF - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)
        out |= {"top_ids": ids, "top_logp": c.gather(1, ids) - log_total[:, None]}
    return out


def _plain_logp_bwd(s):
    z, t = s["z"].float(), s["targets"]
    lp = (z - s["peak"][:, None]) - s["log_sum"][:, None]
    p = torch.exp(lp)
    g = torch.where(t >= 0, s["g_logp"], 0.0)[:, None]
    hit = t[:, None] == torch.arange(z.shape[1], device="cuda")
    dz = g * (hit.float() - p)
    if s["g_entropy"] is not None:
        dz = dz - s["g_entropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    return {"dz": dz.to(s["z"].dtype)}


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"adamw": _plain_adamw, "ln_fwd": _plain_ln_fwd, "ln_bwd": _plain_ln_bwd, "logp": _plain_logp, "logp_bwd": _plain_logp_bwd}[op](state)
    from paper_2110_01595_b200 import binding

    if op == "adamw":
        return _own_adamw(state)
    if op == "ln_fwd":
        y, mean, rstd = binding.solon_layernorm_forward(state["x"], state["w"], state["b"], eps=LN_EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "ln_bwd":
        cols = state["case"]["cols"]
        dw, db = state["matrix"][:, 7:7 + cols], state["matrix"][:, 7 + cols:7 + 2 * cols]
        dx, dw, db = binding.solon_layernorm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["w"],
                                                      partitions=state["case"]["parts"], dweight=dw, dbias=db)
        return {"dx": dx, "dw": dw, "db": db}
    if op == "logp":
        k = state["case"]["top"]
        r = binding.solon_token_logprobs(state["z"], state["targets"], top_k=k)
        out = {"logp": r.logp, "peak": r.peak, "log_sum": r.log_sum, "entropy": r.entropy}
        return out | {"top_ids": r.top_ids, "top_logp": r.top_logp} if k else out
    return {"dz": binding.solon_token_logprobs_backward(state["z"], state["targets"], state["peak"], state["log_sum"], state["g_logp"],
                                                        state["entropy"], state["g_entropy"])}


# ------------------------------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float64
    op = case["op"]
    if op == "adamw":
        t = START + 1
        d, slot = case["d"], s["slot"]
        g = s["grad"].to(f8) / 15
        out = {"norm": None, "copy": None}
        if case["clip"]:
            out["norm"] = torch.linalg.vector_norm(g)
            g = g * min(1.0, s["max_norm"] / (float(out["norm"]) + 1e-6))
        if case["bits"] == 32:
            m, v = s["m"].reshape(-1)[slot].to(f8), s["v"].reshape(-1)[slot].to(f8)
        else:
            block = slot // BLOCK
            mc, vc = s["m"].reshape(-1)[slot].long(), s["v"].reshape(-1)[slot].long()
            mq, vq = (mc % 128) + s["base"][block, 0].long(), vc + s["base"][block, 1].long()
            # a float32 of three mantissa bits by its rank q: (8 + q mod 8) 2^(q div 8 - 130), linear below the first binade
            val = lambda q: torch.where(q < 8, torch.ldexp(q.to(f8), torch.tensor(-129, device="cuda")), torch.ldexp((8 + q % 8).to(f8), q // 8 - 130))  # noqa: E731
            m = torch.where(mc % 128 > 0, val(mq), 0.0) * torch.where(mc > 127, -1.0, 1.0)
            v = torch.where(vc > 0, val(vq), 0.0)
        m = m * 0.9 + g * 0.1
        v = v * 0.999 + g ** 2 * 0.001
        p = s["p"].to(f8)
        tensor = torch.bucketize(torch.arange(d, device="cuda"), s["sizes"].cumsum(0), right=True)
        p = p - LR * s["decay"].to(f8)[tensor] * p - LR * (m / (1 - 0.9 ** t)) / ((v / (1 - 0.999 ** t)).sqrt() + EPS)
        out["p"] = p
        if case["copy"]:
            out["copy"] = p
        if case["bits"] == 32:
            out["m"], out["v"] = torch.zeros(s["m"].shape, dtype=f8, device="cuda"), torch.zeros(s["v"].shape, dtype=f8, device="cuda")
            out["m"].view(-1)[slot], out["v"].view(-1)[slot] = m, v
        else:
            out["m"] = out["v"] = None          # rounded at random: the values are compared with the plain form's alone
        return out
    if op == "ln_fwd":
        x = s["x"].to(f8)
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + LN_EPS) ** -0.5
        return {"y": (x - mean[:, None]) * (rstd[:, None] * s["w"].to(f8)) + s["b"].to(f8), "mean": mean, "rstd": rstd}
    if op == "ln_bwd":
        parts, n, cols = case["parts"], case["rows"] // case["parts"], case["cols"]
        dx, dw, db = [], [], []
        for k in range(parts):               # a partition at a time
            r = slice(k * n, (k + 1) * n)
            xh = (s["x"][r].to(f8) - s["mean"][r, None].to(f8)) * s["rstd"][r, None].to(f8)
            dy = s["dy"][r].to(f8)
            a = dy * s["w"].to(f8)
            dx.append((a - (a.sum(1, keepdim=True) + xh * (a * xh).sum(1, keepdim=True)) / cols) * s["rstd"][r, None].to(f8))
            dw.append(torch.einsum("rc,rc->c", dy, xh))
            db.append(dy.sum(0))
        return {"dx": torch.cat(dx), "dw": torch.stack(dw), "db": torch.stack(db)}
    z, t = s["z"], s["targets"]
    if op == "logp":
        logp, lse, peak, ent, top = [], [], [], [], []
        for r in range(0, z.shape[0], 512):
            a = z[r:r + 512].to(f8)
            l = torch.logsumexp(a, dim=1)
            p = torch.softmax(a, dim=1)
            ent.append(-torch.special.xlogy(p, p).sum(dim=1))
            peak.append(a.max(dim=1).values)
            lse.append(l - peak[-1])
            u = t[r:r + 512]
            logp.append(torch.where(u < 0, 0.0, a[torch.arange(len(u), device="cuda"), u.clamp(min=0)] - l))
            top.append(a.topk(max(1, case["top"]), dim=1).values - l[:, None])
        out = {"logp": torch.cat(logp), "peak": torch.cat(peak), "log_sum": torch.cat(lse), "entropy": torch.cat(ent)}
        return out | {"top_ids": None, "top_logp": torch.cat(top)} if case["top"] else out
    dz = []
    for r in range(0, z.shape[0], 512):
        a, u = z[r:r + 512].to(f8), t[r:r + 512]
        lp = a - (s["peak"][r:r + 512, None].to(f8) + s["log_sum"][r:r + 512, None].to(f8))
        p = lp.exp()
        g = s["g_logp"][r:r + 512].to(f8) * (u >= 0)
        part = -p * g[:, None]
        part[torch.arange(len(u), device="cuda"), u.clamp(min=0)] += g
        if s["g_entropy"] is not None:
            part -= s["g_entropy"][r:r + 512, None].to(f8) * (torch.special.xlogy(p, p) + p * s["entropy"][r:r + 512, None].to(f8))
        dz.append(part)
    return {"dz": torch.cat(dz)}
