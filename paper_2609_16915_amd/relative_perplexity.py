"""What a table costs a model, in the clear: relative perplexity.

    python -m paper_2609_16915_amd.relative_perplexity [--tokens 1024] [--steps 8]
        [--heads 32 --kv-heads 4] [--drafts 4]

Sec. 5 judges an encrypted activation by the perplexity of the model that uses
it over that of the exact one.  This runs both in the clear on one GPU: a stack
of SwiGLU layers whose activation is either exact or the workload's table (what
rosetta_pbs_batch returns for the same quantised input), everything around it in
8 bits

    norm of the residual sum to 8 bits -> gate and up products -> activation
    -> 8 bits -> down product -> ... -> norm -> loss over the vocabulary,

then fits the last norm and the head to the table with the gradients of both.
With --heads each layer begins with attention over an 8-bit cache of its keys and
values

    norm to 8 bits -> q, k, v product -> cache -> attention -> 8 bits -> product,

and with --drafts the model with the table then drafts tokens, that many one after
the other and a second choice for each, which the exact model verifies in one pass a
step: how many it accepts is another measure of the table (of one draft a token it
would be 1 - total variation; the second choices add to that).  Weights and inputs are
synthetic and seeded; targets are drawn from the exact model's own distribution, so
that its perplexity means something.
"""
from __future__ import annotations

import argparse
import math
from typing import NamedTuple

import torch

from . import rosetta as R
from . import workloads as W

EPS = 1e-5


PAGE = 64


class Rows(NamedTuple):
    """Where the rows of a pass are: a cache for each layer, and the packed batch."""
    caches: list
    table: object
    starts: object
    lens: object
    masks: object
    max_rows: int


def make_caches(model: dict, batch: int, positions: int):
    """(caches, table): for each layer a cache, `positions` of each sequence."""
    per = -(-positions // PAGE)
    _, kv_heads, dim = model["heads"]
    table = torch.arange(batch * per, device="cuda", dtype=torch.int32).view(batch, per)
    return [R.kv_cache(batch * per, kv_heads, PAGE, dim) for _ in model["layers"]], table


def make_model(layers: int, dim: int, ffn: int, vocab: int, seed: int = 1, heads: int = 0,
               kv_heads: int = 0) -> dict:
    """Random weights of the named sizes: layers in 8 bits, norms and head in
    bfloat16; with `heads`, attention of that many heads over `kv_heads`."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rows(n, k, scale):
        w = torch.randn((n, k), generator=gen, device="cuda") * scale
        return R.quantize_rows(w)

    model = {"layers": [{"norm": torch.ones(dim, device="cuda", dtype=torch.bfloat16),
                        "gate": rows(ffn, dim, dim ** -0.5), "up": rows(ffn, dim, dim ** -0.5),
                        "down": rows(dim, ffn, ffn ** -0.5)} for _ in range(layers)],
            "norm": torch.ones(dim, device="cuda", dtype=torch.bfloat16),
            "head": (torch.randn((vocab, dim), generator=gen, device="cuda")
                     * 3.0 * dim ** -0.5).to(torch.bfloat16)}
    if heads:
        kv_heads = kv_heads or heads
        each = dim // heads
        model["heads"] = heads, kv_heads, each
        for layer in model["layers"]:
            layer["attention_norm"] = torch.ones(dim, device="cuda", dtype=torch.bfloat16)
            layer["qkv"] = rows((heads + 2 * kv_heads) * each, dim, 2 * dim ** -0.5)
            layer["out"] = rows(dim, heads * each, dim ** -0.5)
    return model


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


def attention(model: dict, layer: dict, o, rows: Rows, cache):
    """A layer's attention of 8-bit rows over its cache, which takes their keys and
    values."""
    heads, kv_heads, each = model["heads"]
    qkv = R.q8_matmul(o.q, o.scale, *layer["qkv"]).view(-1, heads + 2 * kv_heads, each)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    R.kv_write(k, v, cache, rows.table, rows.starts, rows.lens)
    a, _ = R.kv_attention(q, cache, rows.table, rows.starts, rows.lens, masks=rows.masks,
                          max_rows=rows.max_rows, want_lse=False)
    q, scale = R.quantize_rows(a.view(-1, heads * each))
    return R.q8_matmul(q, scale, *layer["out"])


def hidden(model: dict, x, activation, rows: Rows = None):
    """What the last norm reads: (the last layer's output, the residual sum).  A model
    with attention takes `rows`; without, x is one sequence."""
    residual, y = None, x
    if rows is None and "heads" in model:
        rows = one_sequence(model, x.shape[0])
    for i, layer in enumerate(model["layers"]):
        if rows is not None:
            o = R.rms_norm_q8(y, layer["attention_norm"], EPS, residual=residual)
            residual = y if o.h is None else o.h
            y = attention(model, layer, o, rows, rows.caches[i])
        o = R.rms_norm_q8(y, layer["norm"], EPS, residual=residual)
        residual = y if o.h is None else o.h
        gate = R.q8_matmul(o.q, o.scale, *layer["gate"])
        up = R.q8_matmul(o.q, o.scale, *layer["up"])
        q, scale = R.quantize_rows(activation(gate.float()) * up)
        y = R.q8_matmul(q, scale, *layer["down"])
    return y, residual


def one_sequence(model: dict, tokens: int) -> Rows:
    """A pass over one sequence from its beginning, with caches of its own."""
    caches, table = make_caches(model, 1, tokens)
    starts = torch.tensor([0, tokens], device="cuda", dtype=torch.int32)
    return Rows(caches, table, starts, starts[1:].clone(), None, tokens)


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


def probabilities(model: dict, tokens, activation, rows: Rows):
    """The model's distribution after each token; a token's embedding is its row of the
    head."""
    x = model["head"][tokens]
    y, residual = hidden(model, x, activation, rows)
    z, _, _ = R.rms_norm(y, model["norm"], EPS, residual=residual)
    return torch.softmax(z.float() @ model["head"].float().t(), 1)


def draft_and_verify(model: dict, target, drafter, drafts: int, batch: int = 4, prompt: int = 64,
                     steps: int = 8, seed: int = 4) -> dict:
    """Decodes `batch` sequences: the model with the activation `drafter` drafts, that
    with `target` verifies.  A step's tree: node 0 is the last certain token; of the
    2 l - 1 and 2 l, two draws after node 2 l - 3 (0 at first), the first goes on."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    nodes = 1 + 2 * drafts
    parents = torch.tensor([-1, 0, 0] + [p for l in range(2, drafts + 1)
                                         for p in (2 * l - 3,) * 2],
                           device="cuda", dtype=torch.int32)[:nodes].repeat(batch)
    most = prompt + (steps + 1) * (drafts + 1) + nodes
    caches = [make_caches(model, batch, most) for _ in range(2)]  # target's, drafter's

    def at(counts):
        return torch.tensor([0] + counts, device="cuda").cumsum(0).to(torch.int32)

    def each(n):  # n rows for every sequence
        return at([n] * batch)

    def lens_of(values):
        return torch.tensor(values, device="cuda", dtype=torch.int32)

    words = torch.randint(0, model["head"].shape[0], (batch, prompt + 1), generator=gen,
                          device="cuda")
    # all but the last certain token are in both caches
    lens = [prompt] * batch
    for (c, table), activation in zip(caches, (target, drafter)):
        hidden(model, model["head"][words[:, :-1].reshape(-1)], activation,
               Rows(c, table, each(prompt), lens_of(lens), None, prompt))
    new = [[w] for w in words[:, -1].tolist()]  # tokens that the drafter has not read
    masks = R.tree_masks(parents, each(nodes), nodes)
    accepted, said = 0, []
    for _ in range(steps):
        starts = each(nodes)
        tokens = torch.empty((batch, nodes), device="cuda", dtype=torch.int64)
        q = torch.zeros((batch, nodes, model["head"].shape[0]), device="cuda")
        # the drafter reads what is new, then its own first choices
        counts = [len(n) for n in new]
        fed, starts_fed = torch.tensor(sum(new, []), device="cuda"), at(counts)
        tokens[:, 0] = fed[starts_fed[1:].long() - 1]
        known = list(lens)  # positions that the target has without the new root
        node = 0
        for level in range(1, drafts + 1):
            ends = lens_of([k + level for k in known])
            p = probabilities(model, fed, drafter, Rows(*caches[1], starts_fed, ends, None,
                                                        max(counts)))
            q[:, node] = p[starts_fed[1:].long() - 1]
            two = torch.multinomial(q[:, node], 2, replacement=True, generator=gen)
            tokens[:, 2 * level - 1:2 * level + 1] = two
            node = 2 * level - 1
            fed, starts_fed, counts = two[:, 0].contiguous(), each(1), [1] * batch
        # the target reads the tree in one pass
        ends = lens_of([k + nodes for k in known])
        p = probabilities(model, tokens.view(-1), target, Rows(*caches[0], starts, ends, masks,
                                                               nodes))
        u = torch.rand(batch * nodes, generator=gen, device="cuda")
        out, path, count = R.verify_drafts(p, q.view(batch * nodes, -1), tokens.view(-1), u, starts,
                                           parents=parents)
        for cache in caches[0][0]:
            kept = R.kv_keep(cache, caches[0][1], starts, ends, path, count)
        lens = kept.tolist()
        new = [r[:n] for r, n in zip(out.view(batch, nodes).tolist(), count.tolist())]
        accepted += sum(len(n) - 1 for n in new)
        said.append(new)
    return {"accepted_per_step": accepted / (batch * steps), "tokens": said}


def run(workload: str = "llama3_8b_silu", layers: int = 2, dim: int = 2048, ffn: int = 5632,
        vocab: int = 32000, tokens: int = 1024, steps: int = 8, rate: float = 0.5,
        heads: int = 0, kv_heads: int = 0, drafts: int = 0) -> dict:
    if drafts and not heads:
        raise ValueError("drafts are for a model with attention: heads")
    model = make_model(layers, dim, ffn, vocab, heads=heads, kv_heads=kv_heads)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    x = torch.randn((tokens, dim), generator=gen, device="cuda").to(torch.bfloat16)
    exact = hidden(model, x, exact_silu)
    table = hidden(model, x, table_silu(W.get(workload)))
    targets = sample_targets(model, *exact)
    out = {"perplexity_exact": perplexity(model, *exact, targets),
           "perplexity_table": perplexity(model, *table, targets), "losses": []}
    out["relative_perplexity"] = out["perplexity_table"] / out["perplexity_exact"]
    if drafts:
        out["accepted_per_step"] = draft_and_verify(
            model, exact_silu, table_silu(W.get(workload)), drafts)["accepted_per_step"]
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
                        ("tokens", 1024), ("steps", 8), ("heads", 0), ("kv-heads", 0),
                        ("drafts", 0)):
        p.add_argument(f"--{name}", type=int, default=value)
    for k, v in run(**vars(p.parse_args())).items():
        print(f"{k}: {v}")


if __name__ == "__main__":
    main()
