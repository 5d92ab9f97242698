"""What a table costs a model, in the clear: relative perplexity.

    python -m paper_2609_16915_amd.relative_perplexity [--tokens 1024] [--steps 8]

Sec. 5 judges an encrypted activation by the perplexity of the model that uses
it over that of the exact one.  This runs both in the clear on one GPU: a stack
of SwiGLU layers whose activation is either exact or the workload's table (what
rosetta_pbs_batch returns for the same quantised input), everything around it in
8 bits

    norm of the residual sum to 8 bits -> gate and up products -> activation
    -> 8 bits -> down product -> ... -> norm -> loss over the vocabulary,

then fits the last norm and the head to the table with the gradients of both.
Weights and inputs are synthetic and seeded; targets are drawn from the exact
model's own distribution, so that its perplexity means something.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import rosetta as R
from . import workloads as W

EPS = 1e-5


def make_model(layers: int, dim: int, ffn: int, vocab: int, seed: int = 1) -> dict:
    """Random weights of the named sizes: layers in 8 bits, norms and head in
    bfloat16."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rows(n, k, scale):
        w = torch.randn((n, k), generator=gen, device="cuda") * scale
        return R.quantize_rows(w)

    return {"layers": [{"norm": torch.ones(dim, device="cuda", dtype=torch.bfloat16),
                        "gate": rows(ffn, dim, dim ** -0.5), "up": rows(ffn, dim, dim ** -0.5),
                        "down": rows(dim, ffn, ffn ** -0.5)} for _ in range(layers)],
            "norm": torch.ones(dim, device="cuda", dtype=torch.bfloat16),
            "head": (torch.randn((vocab, dim), generator=gen, device="cuda")
                     * 3.0 * dim ** -0.5).to(torch.bfloat16)}


def exact_silu(x):
    return x * torch.sigmoid(x)


def table_silu(w: W.Workload):
    """The workload's table as the encrypted path applies it: the input's interval
    (Workload.quantize), and the value that entry stands for."""
    table = torch.tensor(w.table().astype("int64"), device="cuda")

    def apply(x):
        m = torch.clamp(torch.floor((x - w.lo) / w.dx), 0, w.M - 1).long()
        return w.lo + (table[m] + 0.5) * w.dx
    return apply


def hidden(model: dict, x, activation):
    """What the last norm reads: (the last layer's output, the residual sum)."""
    residual, y = None, x
    for layer in model["layers"]:
        o = R.rms_norm_q8(y, layer["norm"], EPS, residual=residual)
        residual = y if o.h is None else o.h
        gate = R.q8_matmul(o.q, o.scale, *layer["gate"])
        up = R.q8_matmul(o.q, o.scale, *layer["up"])
        q, scale = R.quantize_rows(activation(gate.float()) * up)
        y = R.q8_matmul(q, scale, *layer["down"])
    return y, residual


def loss_and_gradients(model: dict, y, residual, targets):
    """Mean loss over the rows that count, and the gradients of the head and of the
    last norm's weight."""
    z, h, inv_rms = R.rms_norm(y, model["norm"], EPS, residual=residual)
    loss, lse = R.cross_entropy(z, model["head"], targets)
    counts = (targets != -100).sum()
    gloss = (targets != -100) / counts.float()
    gz, g_head = R.cross_entropy_backward(z, model["head"], targets, lse, gloss)
    _, g_norm = R.rms_norm_backward(gz, h, model["norm"], inv_rms)
    return loss.sum() / counts, g_head, g_norm


def perplexity(model: dict, y, residual, targets) -> float:
    z, _, _ = R.rms_norm(y, model["norm"], EPS, residual=residual)
    loss, _ = R.cross_entropy(z, model["head"], targets)
    return math.exp(float(loss.sum() / (targets != -100).sum()))


def sample_targets(model: dict, y, residual, seed: int = 3):
    """A word for each row from the exact model's distribution; the first row, as a
    prompt's, does not count."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    z, _, _ = R.rms_norm(y, model["norm"], EPS, residual=residual)
    p = torch.softmax(z.float() @ model["head"].float().t(), 1)
    t = torch.multinomial(p, 1, generator=gen)[:, 0].contiguous()
    t[0] = -100
    return t


def run(workload: str = "llama3_8b_silu", layers: int = 2, dim: int = 2048, ffn: int = 5632,
        vocab: int = 32000, tokens: int = 1024, steps: int = 8, rate: float = 0.5) -> dict:
    model = make_model(layers, dim, ffn, vocab)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    x = torch.randn((tokens, dim), generator=gen, device="cuda").to(torch.bfloat16)
    exact = hidden(model, x, exact_silu)
    table = hidden(model, x, table_silu(W.get(workload)))
    targets = sample_targets(model, *exact)
    out = {"perplexity_exact": perplexity(model, *exact, targets),
           "perplexity_table": perplexity(model, *table, targets), "losses": []}
    out["relative_perplexity"] = out["perplexity_table"] / out["perplexity_exact"]
    head, norm = model["head"].float(), model["norm"].float()
    for _ in range(steps):
        loss, g_head, g_norm = loss_and_gradients(model, *table, targets)
        out["losses"].append(float(loss))
        head -= rate * g_head.float()
        norm -= rate * g_norm
        model["head"], model["norm"] = head.to(torch.bfloat16), norm.to(torch.bfloat16)
    out["perplexity_fitted"] = perplexity(model, *table, targets)
    return out


def main():
    p = argparse.ArgumentParser(description=__doc__,
                                formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--workload", default="llama3_8b_silu")
    for name, value in (("layers", 2), ("dim", 2048), ("ffn", 5632), ("vocab", 32000),
                        ("tokens", 1024), ("steps", 8)):
        p.add_argument(f"--{name}", type=int, default=value)
    for k, v in run(**vars(p.parse_args())).items():
        print(f"{k}: {v}")


if __name__ == "__main__":
    main()
