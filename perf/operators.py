"""The operators at a model's vocabulary whose speed counts: what stands before and behind the sampling call in a
decoding step, and the loss and gradients of the step that trains the same matrices.

``rms_norm``: the final norm with the residual's addition, its output in bfloat16, float32 or 8-bit codes with a
scale a row, and its gradient.  ``linear_int8``: the head as a product of 8-bit integers with scales for each token and
channel; its output is the logits matrix that the sampling calls read.  ``embed``: lookup with scaling, and its gradient by
sorted tokens.  ``linear_xent``: the cross entropy of the head's logits without keeping them, alone (scoring given tokens) or with the
gradients of hidden states and weights.  Vocabularies are those of the repository's configurations and calls.

Where ``own`` is false, ``run`` computes the same by elementary operations in 32 bits.  Everything is made on the
GPU from the seed.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
BF16, F32 = torch.bfloat16, torch.float32
TYPES = {"bf16": BF16, "f32": F32}
MOST_NORM = 8192 * 4096          # values of the largest norm
MOST_EMBED = 128_256 * 4096      # values of the largest table
MOST_HEAD = 2048 * 128_256 * 4096   # products of the largest head
MOST_XENT = 8192 * 128_256 * 4096   # products of one of the largest loss's matrix products


def listed():
    return [
        # the final norm of a few interactive sequences, codes for the 8-bit head (latency)
        {"name": "norm_decode", "op": "norm8", "T": 8, "D": 4096, "dtype": "bf16", "residual": True},
        # the final norm of a long prefill or training batch
        {"name": "norm_prefill", "op": "norm", "T": 8192, "D": 4096, "dtype": "bf16", "residual": True},
        # the same batch's gradient, with the residual stream's own
        {"name": "norm_grad", "op": "norm_grad", "T": 8192, "D": 4096, "dtype": "bf16", "residual": True},
        # one sequence's logits: the head's bytes are read for one token
        {"name": "head_token", "op": "head", "T": 1, "V": 128_256, "K": 4096, "out": "f32"},
        # a decode batch
        {"name": "head_batch", "op": "head", "T": 256, "V": 151_936, "K": 2048, "out": "bf16"},
        # logits of every token of a few prompts
        {"name": "head_prompts", "op": "head", "T": 2048, "V": 128_256, "K": 4096, "out": "bf16"},
        # embedding of a prefill batch
        {"name": "embed_prefill", "op": "embed", "T": 8192, "V": 128_256, "D": 4096, "dtype": "bf16"},
        # the embedding's gradient of a training batch, frequent tokens as text has them
        {"name": "embed_grad", "op": "embed_grad", "T": 16_384, "V": 128_256, "D": 2048, "dtype": "bf16", "zipf": 1.1},
        # log-probabilities of the tokens that a few sequences drew
        {"name": "score_tokens", "op": "xent", "T": 16, "V": 128_256, "D": 4096, "grad": False},
        # scoring one prompt, nothing a multiple of anything
        {"name": "score_prompt", "op": "xent", "T": 777, "V": 50_001, "D": 1000, "grad": False},
        # loss and gradients of a small model's step
        {"name": "train_small", "op": "xent", "T": 2000, "V": 50_001, "D": 1024, "grad": True},
        # loss and gradients of a large model's step
        {"name": "train_large", "op": "xent", "T": 8192, "V": 128_256, "D": 4096, "grad": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A row's width: in half of the cases a multiple of 64, else any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.5 else max(lo, n // 64 * 64)


def draw(rng):
    """Another case of the same ranges: 1 to 16,384 tokens, rows of 64 to 8192 values, vocabularies of 1000 to 262,144."""
    op = rng.choice(["norm8", "norm", "norm_grad", "head", "head", "embed", "embed_grad", "xent", "xent"])
    if op in ("norm8", "norm", "norm_grad"):
        D = _width(rng, 64, 8192)
        T = min(_log_int(rng, 1, 16_384), MOST_NORM // D)
        return {"op": op, "T": T, "D": D, "dtype": "bf16" if T * D * 2 > MOST_NORM else rng.choice(["bf16", "f32"]), "residual": rng.random() < 0.7}
    if op == "head":
        K, V = _width(rng, 64, 8192), _log_int(rng, 1000, 262_144)
        return {"op": op, "T": max(1, min(_log_int(rng, 1, 4096), MOST_HEAD // (K * V))), "V": V, "K": K, "out": rng.choice(["bf16", "f32"])}
    if op in ("embed", "embed_grad"):
        V = _log_int(rng, 1000, 262_144)
        D = min(_width(rng, 64, 8192), MOST_EMBED // 2 // V)
        c = {"op": op, "T": min(_log_int(rng, 1, 16_384), MOST_NORM // 2 // D), "V": V, "D": D, "dtype": rng.choice(["bf16", "f32"])}
        return dict(c, zipf=round(rng.uniform(0.0, 1.4), 2)) if op == "embed_grad" else c
    V, D = _log_int(rng, 1000, 262_144), _width(rng, 64, 4096)
    return {"op": op, "T": max(1, min(_log_int(rng, 1, 8192), MOST_XENT // (V * D))), "V": V, "D": D, "grad": rng.random() < 0.6}


def work(case):
    op, T = case["op"], case["T"]
    if op in ("norm8", "norm", "norm_grad"):
        D, e = case["D"], 2 if case["dtype"] == "bf16" else 4
        r = 1 if case["residual"] else 0
        if op == "norm_grad":   # dy, h, the stream's gradient, dx; statistics, weight and its gradient
            return {"bytes": T * D * e * (3 + r) + 4 * T + D * (e + 4), "flops": 10 * T * D}
        # x, the stream in and out, the output (as values here: codes and scales, and what they stand for)
        return {"bytes": T * D * (e * (1 + 2 * r) + (4 if op == "norm8" else e)) + D * e, "flops": (7 if op == "norm8" else 5) * T * D}
    if op == "head":
        V, K = case["V"], case["K"]
        return {"bytes": (T + V) * (K + 4) + T * V * (2 if case["out"] == "bf16" else 4), "flops": 2 * T * V * K}
    V, D = case["V"], case["D"]
    if op in ("embed", "embed_grad"):
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 4 * T + T * D * e + (T * D * e if op == "embed" else V * D * e), "flops": T * D}
    if case["grad"]:
        return {"bytes": 2 * (T + V) * D * 2 + 16 * T, "flops": 8 * T * V * D}
    return {"bytes": (T + V) * D * 2 + 12 * T, "flops": 2 * T * V * D}


def _zipf_ids(T, V, s, gen):
    """T ids whose frequencies fall as rank^-s over a random permutation of the vocabulary."""
    p = torch.arange(1, V + 1, device=DEV, dtype=torch.float64) ** -s
    u = torch.rand(T, generator=gen, device=DEV, dtype=torch.float64) * p.sum()
    rank = torch.searchsorted(p.cumsum(0), u).clamp_(max=V - 1)
    return torch.randperm(V, generator=gen, device=DEV)[rank].to(torch.int32)


def _normal(shape, dtype, gen, sigma=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * sigma).to(dtype)


def _stream(T, D, dtype, gen):
    """Hidden states as a residual stream has them: rows of different size, a few channels far larger than the rest."""
    big = 1.0 + 20.0 * (torch.rand(D, generator=gen, device=DEV) < 0.01).float()
    rows = torch.exp(0.5 * torch.randn(T, 1, generator=gen, device=DEV))
    return (torch.randn(T, D, generator=gen, device=DEV) * big * rows).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, T = case["op"], case["T"]
    s = {"case": dict(case)}
    if op in ("norm8", "norm", "norm_grad"):
        D, dtype = case["D"], TYPES[case["dtype"]]
        s["weight"] = (1.0 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dtype)
        if op == "norm_grad":
            s["h"] = _stream(T, D, dtype, gen)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
            s["dy"] = _normal((T, D), dtype, gen, 0.01)
            s["dh"] = _normal((T, D), dtype, gen, 0.01) if case["residual"] else None
        else:
            s["x"] = _normal((T, D), dtype, gen)
            s["residual"] = _stream(T, D, dtype, gen) if case["residual"] else None
    elif op == "head":
        V, K = case["V"], case["K"]
        s["codes"] = (torch.randn(T, K, generator=gen, device=DEV) * 32).round().clamp_(-127, 127).to(torch.int8)
        s["scales"] = 0.02 + 0.02 * torch.rand(T, generator=gen, device=DEV)
        s["w_codes"] = (torch.randn(V, K, generator=gen, device=DEV) * 32).round().clamp_(-127, 127).to(torch.int8)
        s["w_scales"] = (0.02 + 0.02 * torch.rand(V, generator=gen, device=DEV)) * K ** -0.5
    elif op == "embed":
        s["table"] = _normal((case["V"], case["D"]), TYPES[case["dtype"]], gen)
        s["ids"] = _zipf_ids(T, case["V"], 1.1, gen)
    elif op == "embed_grad":
        s["ids"] = _zipf_ids(T, case["V"], case["zipf"], gen)
        s["dout"] = _normal((T, case["D"]), TYPES[case["dtype"]], gen, 0.01)
    else:
        V, D = case["V"], case["D"]
        s["weight"] = _normal((V, D), BF16, gen, 2.0 * D ** -0.5)
        s["targets"] = _zipf_ids(T, V, 1.1, gen)
        # states that lean towards their targets, from not at all to almost sure; a tenth of the tokens is masked
        lean = 3.0 * torch.rand(T, 1, generator=gen, device=DEV)
        s["hidden"] = (torch.randn(T, D, generator=gen, device=DEV) + lean * s["weight"][s["targets"].long()].float()).to(BF16)
        masked = torch.rand(T, generator=gen, device=DEV) < 0.1
        masked[0] = False
        s["targets"] = torch.where(masked, torch.full_like(s["targets"], -1), s["targets"])
        s["dloss"] = torch.where(masked, 0.0, 1.0 / (~masked).sum().float())
    if op in ("embed", "embed_grad"):
        s["scale"] = math.sqrt(case["D"])
    return s


def _plain_norm(x, residual, weight):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
    return h, rstd


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "norm8":
        h, rstd = _plain_norm(s["x"], s["residual"], s["weight"])
        u = h.float() * s["weight"].float()
        top = u.abs().amax(1)
        codes = torch.round(u * torch.div(torch.full_like(top, 127.0), top)[:, None])
        return {"h": h, "values": codes * (top * rstd / 127.0)[:, None]}
    if op == "norm":
        h, rstd = _plain_norm(s["x"], s["residual"], s["weight"])
        return {"h": h, "y": (h.float() * rstd[:, None] * s["weight"].float()).to(h.dtype)}
    if op == "norm_grad":
        h, dy, r = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
        g, n = dy * s["weight"].float(), h * r
        dx = r * (g - n * (g * n).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["h"].dtype), "dweight": (dy * n).sum(0)}
    if op == "head":
        acc = torch.matmul(s["codes"].float(), s["w_codes"].float().t())
        return (acc * s["scales"][:, None] * s["w_scales"]).to(TYPES[c["out"]])
    if op == "embed":
        return (s["table"][s["ids"].long()].float() * s["scale"]).to(s["table"].dtype)
    if op == "embed_grad":
        d = torch.zeros(c["V"], c["D"], device=DEV)
        d.index_add_(0, s["ids"].long(), s["dout"].float())
        return (d * s["scale"]).to(s["dout"].dtype)
    hidden, weight, targets = s["hidden"].float(), s["weight"].float(), s["targets"].long()
    live = targets >= 0
    z = torch.matmul(hidden, weight.t())
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp().sum(1).log() + top[:, 0]
    at = targets.clamp(min=0)[:, None]
    loss = torch.where(live, lse - z.gather(1, at)[:, 0], 0.0)
    if not c["grad"]:
        return {"loss": loss, "lse": lse}
    g = (z - lse[:, None]).exp()
    g.scatter_add_(1, at, torch.full_like(lse[:, None], -1.0))
    g = g * torch.where(live, s["dloss"], 0.0)[:, None]
    return {"loss": loss, "lse": lse, "dhidden": torch.matmul(g, weight).to(BF16), "dweight": torch.matmul(g.t(), hidden).to(BF16)}


def _own(s):
    from paper_2512_00719_amd import vocab
    c = s["case"]
    op = c["op"]
    if op == "norm8":
        codes, scales, h = vocab.rms_norm_int8(s["x"], s["weight"], eps=EPS, residual=s["residual"])
        return {"h": h, "values": codes * scales[:, None]}
    if op == "norm":
        y, h, _ = vocab.rms_norm(s["x"], s["weight"], eps=EPS, residual=s["residual"])
        return {"h": h, "y": y}
    if op == "norm_grad":
        dx, dweight = vocab.rms_norm_grad(s["dy"], s["h"], s["weight"], s["rstd"], dh=s["dh"])
        return {"dx": dx, "dweight": dweight}
    if op == "head":
        return vocab.linear_int8(s["codes"], s["scales"], s["w_codes"], s["w_scales"], out_dtype=TYPES[c["out"]])
    if op == "embed":
        return vocab.embed(s["ids"], s["table"], scale=s["scale"])
    if op == "embed_grad":
        return vocab.embed_grad(s["ids"], s["dout"], c["V"], scale=s["scale"])
    loss, lse = vocab.linear_xent(s["hidden"], s["weight"], s["targets"])
    if not c["grad"]:
        return {"loss": loss, "lse": lse}
    dhidden, dweight = vocab.linear_xent_grad(s["dloss"], s["hidden"], s["weight"], s["targets"], lse)
    return {"loss": loss, "lse": lse, "dhidden": dhidden, "dweight": dweight}


def run(state):
    return _own(state) if own else _plain(state)


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    s = prepare(case, seed)
    op, T = case["op"], case["T"]
    f64 = torch.float64
    if op in ("norm8", "norm"):
        total = s["x"].to(f64) if s["residual"] is None else s["x"].to(f64) + s["residual"].to(f64)
        h = total.to(s["x"].dtype).to(f64)  # the stream is kept in its own type, and the norm is of what is kept
        norm = torch.sqrt((h * h).sum(1, keepdim=True) / case["D"] + EPS)
        y = h / norm * s["weight"].to(f64)
        if op == "norm":
            return {"h": total, "y": y}
        step = y.abs().max(1, keepdim=True).values / 127
        return {"h": total, "values": torch.round(y / step) * step}
    if op == "norm_grad":
        h, dy, w = s["h"].to(f64), s["dy"].to(f64), s["weight"].to(f64)
        norm = 1 / s["rstd"].to(f64)[:, None]  # (the saved statistic is an input)
        dn = dy * w
        dx = dn / norm - h * (dn * h).sum(1, keepdim=True) / (case["D"] * norm ** 3)
        if s["dh"] is not None:
            dx += s["dh"].to(f64)
        return {"dx": dx, "dweight": (dy * h / norm).sum(0)}
    if op == "head":
        # (sums of at most 8192 products of 7-bit magnitudes: whole numbers far below 2^53)
        acc = s["codes"].to(f64) @ s["w_codes"].to(f64).t()
        return acc * torch.outer(s["scales"].to(f64), s["w_scales"].to(f64))
    if op == "embed":
        return torch.index_select(s["table"], 0, s["ids"].long()).to(f64) * s["scale"]
    if op == "embed_grad":
        order = torch.argsort(s["ids"].long(), stable=True)
        ids, ends = torch.unique_consecutive(s["ids"].long()[order], return_counts=True)
        run_sums = torch.cat([torch.zeros(1, case["D"], dtype=f64, device=DEV), s["dout"].to(f64)[order].cumsum(0)])[torch.cat([ends.new_zeros(1), ends.cumsum(0)])].diff(dim=0)
        d = torch.zeros(case["V"], case["D"], dtype=f64, device=DEV)
        d[ids] = run_sums * s["scale"]
        return d
    live = torch.nonzero(s["targets"] >= 0)[:, 0]
    y = s["targets"][live].long()
    w = s["weight"].to(f64)
    z = s["hidden"].to(f64) @ w.t()
    lse = torch.logsumexp(z, 1)
    loss = torch.zeros(T, dtype=f64, device=DEV)
    loss[live] = lse[live] - z[live, y]
    if not case["grad"]:
        return {"loss": loss, "lse": lse}
    p = torch.exp(z - lse[:, None])
    del z
    p[live, y] -= 1.0
    p *= (s["dloss"].to(f64) * (s["targets"] >= 0))[:, None]
    return {"loss": loss, "lse": lse, "dhidden": p @ w, "dweight": p.t().contiguous() @ s["hidden"].to(f64)}
