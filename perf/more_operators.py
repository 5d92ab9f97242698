"""Decoding in the clear over an 8-bit cache, as cases that can be timed and compared.

Next to the encrypted tables a program decodes tokens in the clear: it writes
their keys and values to a paged cache in 8 bits, attends over it (one token, a
prompt, or a tree of drafted tokens), and verifies the drafted tokens against the
target's probabilities from given random numbers, after which the cache keeps the
accepted ones.  Each case is one call of one of these, or, for the cache, writing
with what reads it back.

A batch is packed: sequence b has rows starts[b] .. starts[b + 1], the last of its
lens[b] positions; position t lies at place t % page of page table[b][t / page].

The plain forms are elementary torch operations, in 32 bits (verification in 64,
whose draws lie next to borders), rounded once.  Head layouts are those of the
models that paper_2609_16915_amd/workloads.py names (12 heads of 64; 32 over 4 of
64; 32 over 8 of 128); lengths, batches and vocabularies are generic.

Values held in 8 bits are returned as the values they stand for.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one decoded token of one sequence: latency
        dict(name="cache_one_8x128", op="cache", batch=1, n=1, longest=4096, ragged=0, page=64,
             kv_heads=8, dim=128, dtype="bf16", keep=0),
        # trees of drafted tokens: written, the accepted ones kept
        dict(name="cache_trees_16x33_4x64", op="cache", batch=16, n=33, longest=3001, ragged=1,
             page=16, kv_heads=4, dim=64, dtype="f16", keep=1),
        # four long prompts
        dict(name="cache_prompts_4x8192_8x128", op="cache", batch=4, n=8192, longest=8192,
             ragged=0, page=64, kv_heads=8, dim=128, dtype="bf16", keep=0),
        # one decoded token of one sequence: latency
        dict(name="attend_one_4095", op="attend", batch=1, n=1, longest=4095, ragged=0, page=64,
             heads=32, kv_heads=8, dim=128, dtype="bf16", tree=0),
        # the same at the end of a long context
        dict(name="attend_one_131072", op="attend", batch=1, n=1, longest=131072, ragged=0,
             page=64, heads=32, kv_heads=8, dim=128, dtype="bf16", tree=0),
        # 64 requests decoded together, of 2048 to 8192 positions
        dict(name="attend_64_8192", op="attend", batch=64, n=1, longest=8192, ragged=1, page=64,
             heads=32, kv_heads=8, dim=128, dtype="bf16", tree=0),
        # trees of 25 drafted tokens of eight requests
        dict(name="attend_trees_8x25_4097", op="attend", batch=8, n=25, longest=4097, ragged=1,
             page=16, heads=32, kv_heads=4, dim=64, dtype="f16", tree=1),
        # five ragged prompts of a small model, small pages
        dict(name="attend_prompts_5x777", op="attend", batch=5, n=777, longest=777, ragged=1,
             page=16, heads=12, kv_heads=12, dim=64, dtype="f16", tree=0),
        # a long prompt
        dict(name="attend_prompt_8192", op="attend", batch=1, n=8192, longest=8192, ragged=0,
             page=64, heads=32, kv_heads=8, dim=128, dtype="bf16", tree=0),
        # four drafted tokens after each other, one sequence: latency
        dict(name="verify_chain_5_50257", op="verify", batch=1, n=5, vocab=50257, tree=0),
        # trees of 32 tokens over a large vocabulary
        dict(name="verify_trees_16x32_128000", op="verify", batch=16, n=32, vocab=128000, tree=1),
        # a large batch with a few drafted tokens each
        dict(name="verify_chains_64x4_32000", op="verify", batch=64, n=4, vocab=32000, tree=0),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["cache", "attend", "attend", "attend", "verify"])
    if op == "verify":
        while True:
            batch, n, vocab = _spread(rng, 1, 64), _spread(rng, 1, 64), _spread(rng, 500, 131072)
            if batch * n * vocab <= 16 * 32 * 128000:
                break
        return dict(op=op, batch=batch, n=n, vocab=vocab, tree=rng.randrange(2))
    heads, kv_heads, dim = rng.choice([(12, 12, 64), (32, 4, 64), (32, 8, 128), (16, 2, 256),
                                       (25, 5, 80), (8, 1, 96), (20, 20, 16)])
    case = dict(op=op, ragged=rng.randrange(2), page=rng.choice([16, 32, 64, 256]),
                kv_heads=kv_heads, dim=dim)
    while True:
        batch, longest = _spread(rng, 1, 128), _spread(rng, 1, 131072)
        n = min(longest, _spread(rng, 1, 64) if rng.random() < 0.6 else _spread(rng, 64, 8192))
        case.update(batch=batch, longest=longest, n=n)
        if batch * longest * kv_heads * dim > 64 * 8192 * 8 * 128:
            continue
        if batch * n * kv_heads * dim > 4 * 8192 * 8 * 128:
            continue
        if op == "cache" or _pairs(case) * heads * dim <= 8192 * 8192 * 32 * 128 // 2:
            break
    if op == "cache":
        return dict(case, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), keep=rng.randrange(2))
    return dict(case, heads=heads, dtype=rng.choice(["bf16", "bf16", "f16"]),
                tree=rng.randrange(2) if n <= 256 else 0)


def _sizes(case):
    """Rows and positions of each sequence: ragged ones go down to a quarter."""
    out = []
    for b in range(case["batch"]):
        n, length = case["n"], case.get("longest", 0)
        if case.get("ragged"):
            length -= 3 * length * b // (4 * case["batch"])
            n = n if n <= 64 else n - 3 * n * b // (4 * case["batch"])
        out.append((min(n, length) if length else n, length))
    return out


def _pairs(case):
    """Queries times positions that they see (a tree's tokens counted as in a row)."""
    return sum(n * length - n * (n - 1) // 2 for n, length in _sizes(case))


def _parents(rng, n, tree):
    """Node 0 is the last certain token; a later node's parent is an earlier node."""
    return [-1] + [rng.randrange(max(0, i - 6), i) if tree else i - 1 for i in range(1, n)]


def _masks(parents, words):
    """Bit j of row i: whether node i is node j or comes after it."""
    rows = []
    for i, p in enumerate(parents):
        rows.append((rows[p] if p >= 0 else 0) | 1 << i)
    signed = [[(r >> 64 * w) % (1 << 64) for w in range(words)] for r in rows]
    return [[v - (1 << 64) if v >> 63 else v for v in row] for row in signed]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    rng = random.Random(int(seed))
    op, sizes = case["op"], _sizes(case)
    starts = [0]
    for n, _ in sizes:
        starts.append(starts[-1] + n)
    rows = starts[-1]
    s = {"op": op, "sizes": sizes, "rows": rows, "max_rows": max(n for n, _ in sizes),
         "starts": _int32(starts)}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if op == "verify":
        vocab = case["vocab"]
        trees = [_parents(rng, n, case["tree"]) for n, _ in sizes]
        s["host_parents"] = trees
        s["parents"] = _int32([p for t in trees for p in t]) if case["tree"] else None
        # the drafter's logits are the target's with some noise; it drew each token
        # from its distribution at the token's parent
        logits = normal(rows, vocab) * 2
        s["q"] = torch.softmax(logits + normal(rows, vocab) * 0.7, 1)
        s["p"] = torch.softmax(logits, 1)
        at = [starts[b] + max(p, 0) for b, t in enumerate(trees) for p in t]
        s["drafts"] = torch.multinomial(s["q"][torch.tensor(at, device="cuda")], 1,
                                        generator=gen)[:, 0].contiguous()
        s["u"] = torch.rand(rows, generator=gen, device="cuda")
        return s

    heads_kv, dim, page = case["kv_heads"], case["dim"], case["page"]
    dt = DTYPES[case["dtype"]]
    s["lens"] = _int32([length for _, length in sizes])
    # pages lie anywhere; some are of other sequences
    per = max(-(-length // page) for _, length in sizes)
    used = sum(-(-length // page) for _, length in sizes)
    pages = used + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((len(sizes), per), dtype=torch.int32, device="cuda")
    at = 0
    for b, (_, length) in enumerate(sizes):
        c = -(-length // page)
        table[b, :c] = order[at:at + c]
        at += c
    s["table"], s["page"] = table, page
    shape = (pages, heads_kv, page, dim)
    fill = [torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=torch.int8)
            for _ in range(2)]
    scales = [0.005 + 0.02 * torch.rand(shape[:3], generator=gen, device="cuda") for _ in range(2)]
    s["cache"] = (fill[0], fill[1], scales[0], scales[1])
    if op == "cache":
        # keys and values as parts of one projection's output
        kv = normal(rows, 2 * heads_kv * dim).to(dt)
        s["k"] = kv[:, :heads_kv * dim].view(rows, heads_kv, dim)
        s["v"] = kv[:, heads_kv * dim:].view(rows, heads_kv, dim)
        s["dtype"], s["path"], s["count"] = dt, None, None
        if case["keep"]:
            path, count = [], []
            for n, _ in sizes:
                kept = [0] + [i for i in range(1, n) if rng.random() < 0.2]
                path += kept + [-1] * (n - len(kept))
                count.append(len(kept))
            s["path"], s["count"] = _int32(path), _int32(count)
        return s
    heads = case["heads"]
    qkv = (normal(rows, (heads + 2 * heads_kv) * dim) * 2).to(dt)
    s["q"] = qkv[:, :heads * dim].view(rows, heads, dim)
    s["masks"] = None
    if case["tree"]:
        words = -(-s["max_rows"] // 64)
        s["masks"] = torch.tensor([m for n, _ in sizes
                                   for m in _masks(_parents(rng, n, 1), words)],
                                  dtype=torch.int64, device="cuda")
    return s


def _run_own(s):
    from paper_2609_16915_amd import rosetta as R
    if s["op"] == "verify":
        tokens, path, count = R.verify_drafts(s["p"], s["q"], s["drafts"], s["u"], s["starts"],
                                              parents=s["parents"])
        return {"tokens": tokens, "path": path, "count": count}
    cache = R.KVCache(*s["cache"])
    where = (cache, s["table"], s["starts"], s["lens"])
    if s["op"] == "attend":
        out, lse = R.kv_attention(s["q"], *where, masks=s["masks"], max_rows=s["max_rows"])
        return {"out": out, "lse": lse}
    R.kv_write(s["k"], s["v"], *where)
    lens = s["lens"]
    if s["path"] is not None:
        lens = R.kv_keep(*where, s["path"], s["count"])
    k, v = R.kv_read(cache, s["table"], s["starts"], lens, s["rows"], s["dtype"])
    return {"k": k, "v": v, "lens": lens}


# ------------------------------------------------------------- plain forms

def _places(s, lens):
    """(page, place in it, whether there is one) of every row's position."""
    starts = s["starts"].long()
    r = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(starts[1:], r, right=True)
    pos = lens.long()[b] - (starts[b + 1] - r)
    there = pos >= 0
    pos = pos.clamp_min(0)
    return s["table"][b, pos // s["page"]].long(), pos % s["page"], there, b, r - starts[b]


def _cache_plain(s):
    pages, at, _, b, i = _places(s, s["lens"])
    for x, q, scale in ((s["k"], s["cache"][0], s["cache"][2]),
                        (s["v"], s["cache"][1], s["cache"][3])):
        x = x.float()
        sc = x.abs().amax(2) / 127.0
        q[pages, :, at] = torch.round(x / sc[:, :, None]).to(torch.int8)
        scale[pages, :, at] = sc
    lens = s["lens"]
    if s["path"] is not None:
        # row i takes what row path[i] has, the rest their own
        r = torch.arange(s["rows"], device="cuda")
        src = torch.where(i < s["count"].long()[b], r - i + s["path"].long(), r)
        for t in s["cache"]:
            t[pages, :, at] = t[pages[src], :, at[src]]
        n = s["starts"][1:] - s["starts"][:-1]
        lens = s["lens"] - n + s["count"]
    pages, at, there, _, _ = _places(s, lens)
    out = []
    for q, scale in ((s["cache"][0], s["cache"][2]), (s["cache"][1], s["cache"][3])):
        x = q[pages, :, at].float() * scale[pages, :, at][:, :, None]
        out.append(torch.where(there[:, None, None], x, torch.zeros_like(x)).to(s["dtype"]))
    return {"k": out[0], "v": out[1], "lens": lens}


def _gathered(s, b, length, dtype):
    """Keys and values of a sequence, [kv_heads][length][dim]."""
    c = -(-length // s["page"])
    at = s["table"][b, :c].long()
    out = []
    for q, scale in ((s["cache"][0], s["cache"][2]), (s["cache"][1], s["cache"][3])):
        x = q[at].to(dtype) * scale[at].to(dtype)[..., None]
        out.append(x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :length])
    return out


def _seen(s, start, n, length, lo, hi):
    """Which of the positions rows lo .. hi of a sequence see."""
    i = torch.arange(lo, hi, device="cuda")[:, None]
    j = torch.arange(length, device="cuda")[None, :] - (length - n)
    if s["masks"] is None:
        return j <= i
    words = s["masks"][start + lo:start + hi]
    bits = torch.gather(words, 1, (j.clamp_min(0) // 64).expand(hi - lo, length))
    return (j < 0) | (bits >> (j.clamp_min(0) % 64) & 1).bool()


def _attend_plain(s):
    q, rows = s["q"], s["rows"]
    heads, dim = q.shape[1], q.shape[2]
    out = torch.empty((rows, heads, dim), dtype=q.dtype, device="cuda")
    lse = torch.empty((rows, heads), device="cuda")
    start = 0
    for b, (n, length) in enumerate(s["sizes"]):
        k, v = _gathered(s, b, length, torch.float32)
        group, block = heads // k.shape[0], max(1, (1 << 28) // (length * heads))
        for lo in range(0, n, block):
            hi = min(n, lo + block)
            m = hi - lo
            x = q[start + lo:start + hi].float().view(m, -1, group, dim)
            x = x.permute(1, 2, 0, 3).reshape(-1, group * m, dim)
            scores = torch.bmm(x, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(dim))
            scores = scores.view(-1, group, m, length)
            scores.masked_fill_(~_seen(s, start, n, length, lo, hi), -math.inf)
            top = scores.amax(3, keepdim=True)
            e = torch.exp(scores - top)
            z = e.sum(3, keepdim=True)
            o = torch.bmm((e / z).view(-1, group * m, length), v.contiguous())
            o = o.view(-1, group, m, dim).permute(2, 0, 1, 3).reshape(m, heads, dim)
            out[start + lo:start + hi] = o.to(q.dtype)
            lse[start + lo:start + hi] = (top + torch.log(z))[..., 0].permute(2, 0, 1).reshape(
                m, heads)
        start += n
    return {"out": out, "lse": lse}


def _verify_plain(s):
    """At a node, with r = (p - c q)+ and its sum z (c = 0 and z = 1 at first): a child
    with token x is accepted if u z q(x) < p(x) - c q(x); else c grows by z.  The last
    token is drawn from what is left."""
    p, q, drafts = s["p"], s["q"], s["drafts"]
    start, at = 0, []
    for t in s["host_parents"]:
        at += [start + max(i, 0) for i in t]
        start += len(t)
    at = torch.tensor(at, device="cuda")
    px, qx, u, x = (t.tolist() for t in (p[at, drafts].double(), q[at, drafts].double(),
                                         s["u"].double(), drafts))
    tokens, path, count = [], [], []
    start = 0
    for tree in s["host_parents"]:
        node, i, c, z, kept = 0, 1, 0.0, 1.0, [0]
        left = None
        while i < len(tree):
            if tree[i] == node:
                r = start + i
                if u[r] * z * qx[r] < px[r] - c * qx[r]:
                    kept.append(i)
                    node, c, z, left = i, 0.0, 1.0, None
                else:
                    c += z
                    left = (p[start + node].double() - c * q[start + node].double()).clamp_min(0)
                    z = left.sum().item()
            i += 1
        if left is None:
            left = p[start + node].double()
        if not left.sum() > 0:
            left = p[start + node].double()
        total = torch.cumsum(left, 0)
        last = int((total > u[start] * total[-1]).to(torch.int32).argmax())
        n, a = len(tree), len(kept)
        tokens += [x[start + i] for i in kept[1:]] + [last] + [-1] * (n - a)
        path += kept + [-1] * (n - a)
        count.append(a)
        start += n
    return {"tokens": torch.tensor(tokens, device="cuda"), "path": _int32(path),
            "count": _int32(count)}


def run(s):
    if own:
        return _run_own(s)
    return {"cache": _cache_plain, "attend": _attend_plain, "verify": _verify_plain}[s["op"]](s)


def work(case):
    sizes = _sizes(case)
    rows = sum(n for n, _ in sizes)
    if case["op"] == "verify":
        # one node's two distributions for each sequence, the drafted tokens' places
        b, v = case["batch"], case["vocab"]
        return {"bytes": 8 * b * v + 36 * rows, "flops": 3 * b * v}
    entries = 2 * case["kv_heads"] * case["dim"]
    if case["op"] == "cache":
        # in, 8 bits and scales; those, out again
        e, b = rows * entries, BYTES[case["dtype"]]
        places = 2 * rows * case["kv_heads"] * 4
        moved = 2 * sum(case["n"] // 5 for _ in sizes) * entries if case["keep"] else 0
        return {"bytes": e * (2 * b + 2) + 2 * places + moved, "flops": 5 * e}
    e = sum(length for _, length in sizes)
    ends = rows * case["heads"] * (2 * case["dim"] * BYTES[case["dtype"]] + 4)
    return {"bytes": e * (entries + 8 * case["kv_heads"]) + ends,
            "flops": 4 * _pairs(case) * case["heads"] * case["dim"]}


# ------------------------------------------------- the definitions in 64 bits

def _exact_cache(s):
    sizes, page = s["sizes"], s["page"]
    table, starts = s["table"].tolist(), s["starts"].tolist()
    path = s["path"].tolist() if s["path"] is not None else None
    keep = s["count"].tolist() if path else None
    new = [length - n + keep[b] if path else length for b, (n, length) in enumerate(sizes)]
    out = []
    for x, q, scale in ((s["k"], s["cache"][0], s["cache"][2]),
                        (s["v"], s["cache"][1], s["cache"][3])):
        x = x.double()
        top = torch.maximum(x.max(2).values, -x.min(2).values)
        step = (top / 127).unsqueeze(2)
        written = torch.floor(x / step + 0.5) * step
        got = []
        for b, (n, length) in enumerate(sizes):
            rows = written[starts[b]:starts[b + 1]]
            if path:
                rows = rows[torch.tensor(path[starts[b]:starts[b] + keep[b]], device="cuda")]
            more = n - rows.shape[0]  # positions from before the rows
            first = length - n - more
            old = []
            for t in range(first, length - n):
                if t < 0:
                    old.append(torch.zeros_like(rows[0]))
                else:
                    pg = table[b][t // page]
                    old.append(q[pg, :, t % page].double() * scale[pg, :, t % page, None].double())
            got.append(torch.cat([torch.stack(old), rows]) if old else rows)
        out.append(torch.cat(got))
    return {"k": out[0], "v": out[1], "lens": torch.tensor(new, dtype=torch.int32, device="cuda")}


def _exact_attend(s):
    q, D = s["q"], torch.float64
    heads, dim = q.shape[1], q.shape[2]
    outs, lses, start = [], [], 0
    for b, (n, length) in enumerate(s["sizes"]):
        k, v = _gathered(s, b, length, D)
        group = heads // k.shape[0]
        out = torch.empty((n, heads, dim), dtype=D, device="cuda")
        lse = torch.empty((n, heads), dtype=D, device="cuda")
        block = max(1, (1 << 26) // length)
        for lo in range(0, n, block):
            hi = min(n, lo + block)
            hidden = ~_seen(s, start, n, length, lo, hi)
            for h in range(heads):
                a = torch.matmul(k[h // group], q[start + lo:start + hi, h].to(D).t().contiguous())
                a = a.t().div(math.sqrt(dim)).masked_fill(hidden, -math.inf)
                z = torch.logsumexp(a, 1)
                lse[lo:hi, h] = z
                out[lo:hi, h] = torch.matmul(torch.exp(a - z.unsqueeze(1)), v[h // group])
        outs.append(out)
        lses.append(lse)
        start += n
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_verify(s):
    """By the distributions themselves, normalised after every rejection."""
    D, starts = torch.float64, s["starts"].tolist()
    x, u = s["drafts"].tolist(), s["u"].to(D)
    tokens, path, count = [], [], []
    for b, tree in enumerate(s["host_parents"]):
        first, n = starts[b], len(tree)
        node, kept, tokens_here = 0, [0], []
        while True:
            left, q = s["p"][first + node].to(D), s["q"][first + node].to(D)
            whole, target = left, left
            for i in (i for i in range(1, n) if tree[i] == node):
                if (u[first + i] * q[x[first + i]] < target[x[first + i]]).item():
                    break
                left = torch.relu(target - q)
                target = left / left.sum()
            else:
                break
            node = i
            kept.append(i)
            tokens_here.append(x[first + i])
        if not left.sum() > 0:
            left = whole
        edges = left.cumsum(0)
        tokens_here.append(int(torch.searchsorted(edges, u[first] * edges[-1], right=True)))
        tokens += tokens_here + [-1] * (n - len(kept))
        path += kept + [-1] * (n - len(kept))
        count.append(len(kept))
    return {"tokens": torch.tensor(tokens, device="cuda"),
            "path": torch.tensor(path, dtype=torch.int32, device="cuda"),
            "count": torch.tensor(count, dtype=torch.int32, device="cuda")}


def exact(case, seed):
    """The definitions in 64 bits, written apart from run()."""
    s = prepare(case, seed)
    if case["op"] == "cache" and case["keep"] and s["rows"] > 20000:
        return None
    if case["op"] == "attend" and 4 * _pairs(case) * case["heads"] * case["dim"] > 6e12:
        return None
    return {"cache": _exact_cache, "attend": _exact_attend, "verify": _exact_verify}[s["op"]](s)
