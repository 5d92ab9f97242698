"""The clear side of a private decode, as cases that can be timed and compared.

Next to the encrypted tables a program runs a model's other layers in the
clear: the norm that adds the residual and gives 8 bits, the 8-bit product
that reads them, and the loss over the vocabulary that says what the tables
cost (perplexity), with the gradients that fit a model to them.  Each case is
one call of one of these.

The plain forms are elementary torch operations in 32 bits, rounded once.
Widths are those of paper_2609_16915_amd/workloads.py (model widths 768, 2048
and 4096, FFN widths 5632 and 14336); row counts and vocabularies are generic.

Values held in 8 bits are returned as the values they stand for, in bfloat16.
"""
import math

import torch

own = False

EPS = 1e-5
IGNORE = -100
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one decoded token, width 4096: latency
        dict(name="norm_one_4096", op="norm", rows=1, dim=4096, dtype="bf16", pad=0),
        # a ragged set of prompts, odd width, rows that are not next to each other
        dict(name="norm_333_2047", op="norm", rows=333, dim=2047, dtype="f16", pad=9),
        # a long prefill
        dict(name="norm_16384_4096", op="norm", rows=16384, dim=4096, dtype="bf16", pad=0),
        # the norm's gradient in a small training step, 32 bits
        dict(name="norm_back_1023_768", op="norm_back", rows=1023, dim=768, dtype="f32", pad=0),
        # the same over a large batch
        dict(name="norm_back_8192_4096", op="norm_back", rows=8192, dim=4096, dtype="bf16", pad=0),
        # one decoded token through the FFN's first product
        dict(name="q8_one_14336x4096", op="q8", m=1, n=14336, k=4096, out="bf16"),
        # 33 requests decoded together through the FFN's second product
        dict(name="q8_33_4096x14336", op="q8", m=33, n=4096, k=14336, out="bf16"),
        # a ragged prefill through a small model's first product, 32-bit output
        dict(name="q8_1001_5632x2048", op="q8", m=1001, n=5632, k=2048, out="f32"),
        # a long prefill through the FFN's first product
        dict(name="q8_8192_14336x4096", op="q8", m=8192, n=14336, k=4096, out="bf16"),
        # scoring eight candidate tokens over a large vocabulary
        dict(name="loss_8_128000", op="loss", rows=8, dim=4096, vocab=128000, dtype="bf16",
             masked=0),
        # a small model's training step: odd rows and vocabulary
        dict(name="loss_grad_777_50257", op="loss_grad", rows=777, dim=768, vocab=50257,
             dtype="f16", masked=100),
        # a large model's training step
        dict(name="loss_grad_4096_128000", op="loss_grad", rows=4096, dim=4096, vocab=128000,
             dtype="bf16", masked=512),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: one in four odd, the others multiples of 64 where they can be."""
    d = _spread(rng, lo, hi)
    return d | 1 if rng.random() < 0.25 else max(lo, d // 64 * 64)


def draw(rng):
    op = rng.choice(["norm", "norm_back", "q8", "q8", "loss", "loss_grad"])
    if op in ("norm", "norm_back"):
        while True:
            rows, dim = _spread(rng, 1, 32768), _width(rng, 64, 16384)
            if rows * dim <= 32 << 20:
                break
        return dict(op=op, rows=rows, dim=dim, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    pad=rng.choice([0, 0, 8, rng.randrange(1, 40)]))
    if op == "q8":
        while True:
            m, n, k = _spread(rng, 1, 16384), _width(rng, 64, 16384), _width(rng, 64, 16384)
            if m * n * k <= 8192 * 14336 * 4096 // 2:
                break
        return dict(op=op, m=m, n=n, k=k, out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    while True:
        rows, dim, vocab = _spread(rng, 1, 8192), _width(rng, 64, 4096), _spread(rng, 500, 131072)
        if rows * dim * vocab <= 4096 * 4096 * 128000 // 4 and rows * vocab <= 1 << 29:
            break
    return dict(op=op, rows=rows, dim=dim, vocab=vocab, dtype=rng.choice(["bf16", "bf16", "f16"]),
                masked=rng.choice([0, rows // 10, rows // 2]))


def _normal(gen, rows, cols, dtype, scale=1.0, pad=0):
    """[rows][cols] of a buffer whose rows are cols + pad long."""
    t = torch.randn((rows, cols + pad), generator=gen, device="cuda", dtype=torch.float32)
    return (t * scale).to(dtype)[:, :cols]


def _int8(gen, rows, cols):
    """What rounding a normal row to 8 bits gives: a third of the range deviation."""
    t = torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.float32)
    return (t * 36.0).round_().clamp_(-127, 127).to(torch.int8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op = case["op"]
    s = {"op": op}
    if op in ("norm", "norm_back"):
        rows, dim, dt, pad = case["rows"], case["dim"], DTYPES[case["dtype"]], case["pad"]
        s["weight"] = (1 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).to(dt)
        s["x"] = _normal(gen, rows, dim, dt, 1.0, pad)
        s["residual"] = _normal(gen, rows, dim, dt, 2.0, pad)
        if op == "norm_back":
            # what the forward pass left: the sum and 1 / rms
            h = s.pop("x").float() + s.pop("residual").float()
            s["inv_rms"] = (h.square().mean(1) + EPS).rsqrt()
            s["h"] = h.to(dt)
            s["gy"] = _normal(gen, rows, dim, dt, 1e-2, pad)
            s["gh"] = _normal(gen, rows, dim, dt, 1e-2, pad)
        return s
    if op == "q8":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], s["b"] = _int8(gen, m, k), _int8(gen, n, k)
        s["a_scale"] = 0.01 + 0.02 * torch.rand(m, generator=gen, device="cuda")
        s["b_scale"] = 1e-4 + 4e-4 * torch.rand(n, generator=gen, device="cuda")
        s["bias"] = torch.randn(n, generator=gen, device="cuda")
        s["dtype"] = DTYPES[case["out"]]
        return s
    rows, dim, vocab, dt = case["rows"], case["dim"], case["vocab"], DTYPES[case["dtype"]]
    s["h"] = _normal(gen, rows, dim, dt)
    s["w"] = _normal(gen, vocab, dim, dt, 1.5 / math.sqrt(dim))
    s["targets"] = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    if case["masked"]:
        at = torch.randperm(rows, generator=gen, device="cuda")[:case["masked"]]
        s["targets"][at] = IGNORE
    # the gradient of the mean over the rows that count
    counts = max(1, rows - case["masked"])
    s["gloss"] = torch.full((rows,), 1.0 / counts, device="cuda")
    return s


def _run_own(s):
    from paper_2609_16915_amd import rosetta as R
    op = s["op"]
    if op == "norm":
        o = R.rms_norm_q8(s["x"], s["weight"], EPS, residual=s["residual"])
        return {"h": o.h, "scale": o.scale, "inv_rms": o.inv_rms,
                "values": R.dequantize_rows(o.q, o.scale, torch.bfloat16)}
    if op == "norm_back":
        gx, gw = R.rms_norm_backward(s["gy"], s["h"], s["weight"], s["inv_rms"], gh=s["gh"])
        return {"gx": gx, "gw": gw}
    if op == "q8":
        return R.q8_matmul(s["a"], s["a_scale"], s["b"], s["b_scale"], bias=s["bias"],
                           out_dtype=s["dtype"])
    loss, lse = R.cross_entropy(s["h"], s["w"], s["targets"], IGNORE)
    if op == "loss":
        return {"loss": loss, "lse": lse}
    gh, gw = R.cross_entropy_backward(s["h"], s["w"], s["targets"], lse, s["gloss"], IGNORE)
    return {"loss": loss, "lse": lse, "gh": gh, "gw": gw}


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "norm":
        dt = s["x"].dtype
        h = s["x"].float() + s["residual"].float()
        inv = 1.0 / torch.sqrt((h * h).mean(1) + EPS)
        y = h * inv[:, None] * s["weight"].float()
        scale = y.abs().amax(1) / 127.0
        q = torch.round(y / scale[:, None])
        return {"h": h.to(dt), "scale": scale, "inv_rms": inv,
                "values": (q * scale[:, None]).to(torch.bfloat16)}
    if op == "norm_back":
        h, gy, w, inv = s["h"].float(), s["gy"].float(), s["weight"].float(), s["inv_rms"][:, None]
        g = gy * w
        c = (g * h).sum(1, keepdim=True) * inv * inv * inv / h.shape[1]
        gx = s["gh"].float() + g * inv - h * c
        return {"gx": gx.to(s["h"].dtype), "gw": (gy * h * inv).sum(0)}
    if op == "q8":
        acc = s["a"].float() @ s["b"].float().t()
        return (acc * s["a_scale"][:, None] * s["b_scale"][None, :] + s["bias"]).to(s["dtype"])
    h, w, t = s["h"].float(), s["w"].float(), s["targets"]
    logits = h @ w.t()
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    z = e.sum(1, keepdim=True)
    lse = top[:, 0] + torch.log(z[:, 0])
    counts = t != IGNORE
    at = torch.where(counts, t, torch.zeros_like(t))[:, None]
    loss = torch.where(counts, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    if op == "loss":
        return {"loss": loss, "lse": lse}
    g = torch.where(counts, s["gloss"], torch.zeros_like(lse))[:, None]
    p = e.div_(z)
    p.scatter_add_(1, at, torch.full_like(z, -1.0))
    p *= g
    return {"loss": loss, "lse": lse, "gh": (p @ w).to(s["h"].dtype),
            "gw": (p.t() @ h).to(s["w"].dtype)}


def work(case):
    op = case["op"]
    if op in ("norm", "norm_back"):
        e, b = case["rows"] * case["dim"], BYTES[case["dtype"]]
        if op == "norm":  # x, residual, h; the values as returned
            return {"bytes": e * (3 * b + 2) + case["dim"] * b + 8 * case["rows"], "flops": 9 * e}
        return {"bytes": e * 4 * b + case["dim"] * (b + 4) + 4 * case["rows"], "flops": 12 * e}
    if op == "q8":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + m * n * BYTES[case["out"]] + 4 * m + 8 * n,
                "flops": 2 * m * n * k}
    t, d, v = case["rows"], case["dim"], case["vocab"]
    ends = (t + v) * d * BYTES[case["dtype"]]
    if op == "loss":
        return {"bytes": ends + 16 * t, "flops": 2 * t * d * v + 4 * t * v}
    return {"bytes": 2 * ends + 20 * t, "flops": 6 * t * d * v + 8 * t * v}


def exact(case, seed):
    """The definitions in 64 bits, written apart from run()."""
    s = prepare(case, seed)
    op, D = s["op"], torch.float64
    if op == "norm":
        h = s["x"].to(D).add_(s["residual"].to(D))
        inv = h.pow(2).sum(1).div_(h.shape[1]).add_(EPS).pow_(-0.5)
        y = torch.mul(h, inv.unsqueeze(1)).mul_(s["weight"].to(D))
        scale = torch.maximum(y.max(1).values, -y.min(1).values) / 127
        steps = torch.floor(y / scale.unsqueeze(1) + 0.5)
        return {"h": h, "scale": scale, "inv_rms": inv, "values": steps * scale.unsqueeze(1)}
    if op == "norm_back":
        h, gy, inv = s["h"].to(D), s["gy"].to(D), s["inv_rms"].to(D).unsqueeze(1)
        n = h * inv  # the normalised rows
        gn = gy * s["weight"].to(D)
        gx = s["gh"].to(D) + inv * (gn - n * (gn * n).mean(1, keepdim=True))
        return {"gx": gx, "gw": (gy * n).sum(0)}
    if op == "q8":
        acc = torch.matmul(s["a"].to(D), s["b"].to(D).t().contiguous())
        return torch.outer(s["a_scale"].to(D), s["b_scale"].to(D)).mul_(acc).add_(s["bias"].to(D))
    h, w, t = s["h"].to(D), s["w"].to(D), s["targets"]
    logp = torch.matmul(h, w.t().contiguous())
    rows = (t >= 0).nonzero()[:, 0]
    lse = torch.logsumexp(logp, 1)
    loss = torch.zeros_like(lse)
    loss[rows] = lse[rows] - logp[rows, t[rows]]
    if op == "loss":
        return {"loss": loss, "lse": lse}
    p = logp.sub_(lse.unsqueeze(1)).exp_()
    p[rows, t[rows]] -= 1
    g = torch.zeros_like(lse)
    g[rows] = s["gloss"].to(D)[rows]
    p.mul_(g.unsqueeze(1))
    gh = torch.matmul(p, w)
    return {"loss": loss, "lse": lse, "gh": gh, "gw": torch.matmul(p.t().contiguous(), h)}
