"""The example's models with attention: their layers against the same model in 64 bits,
a pass in pieces against one pass, and drafts that the exact model verifies."""
import math

import pytest

from paper_2609_16915_amd import relative_perplexity as RP
from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
D = torch.float64
SIZES = dict(layers=2, dim=256, ffn=704, vocab=1000)


def values(rows):
    q, scale = rows
    return q.to(D) * scale.to(D)[:, None]


def rounded(x):
    """8 bits with a scale per row, in 64 bits."""
    scale = x.abs().amax(-1, keepdim=True) / 127
    return torch.round(x / scale) * scale


def hidden64(model, x, activation):
    heads, kv, each = model["heads"]
    residual, y = torch.zeros_like(x, dtype=D), x.to(D)

    def normed(weight):
        n = residual / torch.sqrt((residual ** 2).mean(1, keepdim=True) + RP.EPS)
        return rounded(n * weight.to(D))

    for layer in model["layers"]:
        residual = residual + y
        qkv = (normed(layer["attention_norm"]) @ values(layer["qkv"]).t()).view(-1, heads + 2 * kv,
                                                                               each)
        q, k, v = qkv.split([heads, kv, kv], 1)
        k, v = (rounded(t).repeat_interleave(heads // kv, 1) for t in (k, v))
        s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(each)
        s = s.masked_fill(~torch.ones_like(s[0]).tril().bool(), -math.inf)
        a = torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), v).reshape(-1, heads * each)
        y = rounded(a) @ values(layer["out"]).t()
        residual = residual + y
        n = normed(layer["norm"])
        f = activation(n @ values(layer["gate"]).t()) * (n @ values(layer["up"]).t())
        y = rounded(f) @ values(layer["down"]).t()
    return y, residual


@pytest.fixture(scope="module")
def model():
    require_gpu()
    return RP.make_model(**SIZES, heads=4, kv_heads=2)


def inputs(tokens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((tokens, SIZES["dim"]), device="cuda", generator=g).to(torch.bfloat16)


def test_layers_with_attention(model):
    x = inputs(96, 5)
    y, residual = RP.hidden(model, x, RP.exact_silu)
    y64, residual64 = hidden64(model, x, RP.exact_silu)
    # A difference of e (of the values' deviation) before a rounding to 8 bits of step s
    # moves a share of about 0.8 e / s of the values (the mean of |e| over s) by a step:
    # e^2 becomes e^2 + 0.8 e s.  s is the largest value over 127: 3.3 deviations for 256
    # normal values, 10 for the 704 products of the activation.  Between the steps lie
    # roundings to bfloat16, 2^-9 of the values.  Ten roundings to 8 bits then give 0.13.
    e = 2.0 ** -9
    for _ in range(2):
        for s in (3.3, 3.3, 3.3, 3.3, 10.0):  # norm, keys and values, attention, norm, FFN
            e = math.sqrt(e * e + 0.8 * e * s / 127 + 2.0 ** -18)
    assert e < 0.14
    for got, want in ((y, y64), (residual, residual64)):
        assert float((got.to(D) - want).norm() / want.norm()) < e


def test_attention_of_one_layer(model):
    """From the same 8-bit rows: queries, keys and values rounded to bfloat16 (2^-9 each),
    which moves keys and values by steps of 8 bits (0.8 2^-9 3.3 / 127, the root of it),
    the output to bfloat16 and to 8 bits: together 0.04 of the norm, by the root of the
    sum of their squares, the scores' part taken three times over."""
    layer, x = model["layers"][0], inputs(96, 7)
    o = R.rms_norm_q8(x, layer["attention_norm"], RP.EPS)
    rows = RP.one_sequence(model, 96)
    got = RP.attention(model, layer, o, rows, rows.caches[0])
    heads, kv, each = model["heads"]
    n = values((o.q, o.scale))
    q, k, v = (n @ values(layer["qkv"]).t()).view(-1, heads + 2 * kv, each).split([heads, kv, kv], 1)
    k, v = (rounded(t).repeat_interleave(heads // kv, 1) for t in (k, v))
    s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(each)
    s = s.masked_fill(~torch.ones_like(s[0]).tril().bool(), -math.inf)
    a = torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), v).reshape(-1, heads * each)
    want = rounded(a) @ values(layer["out"]).t()
    assert float((got.to(D) - want).norm() / want.norm()) < 0.04


def test_a_pass_in_pieces_is_the_pass(model):
    """A sequence that comes in pieces of 40, 1 and 55 rows through the cache."""
    x = inputs(96, 6)
    whole = RP.hidden(model, x, RP.exact_silu)[1]
    caches, table = RP.make_caches(model, 1, 96)
    at = 0
    for n in (40, 1, 55):
        starts = torch.tensor([0, n], device="cuda", dtype=torch.int32)
        lens = torch.tensor([at + n], device="cuda", dtype=torch.int32)
        rows = RP.Rows(caches, table, starts, lens, None, n)
        part = RP.hidden(model, x[at:at + n], RP.exact_silu, rows)[1]
        # the same sums in other orders: single roundings to bfloat16 and to 8 bits differ
        d = part.to(D) - whole[at:at + n].to(D)
        assert float(d.norm() / whole[at:at + n].to(D).norm()) < 0.02
        at += n


def test_drafts(model):
    same = RP.draft_and_verify(model, RP.exact_silu, RP.exact_silu, 3, batch=3, prompt=33, steps=4)
    for step in same["tokens"]:
        assert len(step) == 3
        for new in step:
            assert 1 <= len(new) <= 4 and all(0 <= t < SIZES["vocab"] for t in new)
    # the same model drafts and verifies: its distributions differ by roundings alone, and
    # a first child is rejected with the total variation between them, a few percent
    assert same["accepted_per_step"] > 2.4
    # one that drafts from another distribution altogether is rejected often
    other = RP.draft_and_verify(model, RP.exact_silu, lambda x: -3 * x, 3, batch=3, prompt=33, steps=4)
    assert 0 <= other["accepted_per_step"] < same["accepted_per_step"]


def test_run_with_attention_and_drafts(model):
    out = RP.run(**SIZES, tokens=96, steps=3, heads=4, kv_heads=2, drafts=2)
    assert 1 < out["perplexity_exact"] < SIZES["vocab"]
    assert math.isfinite(out["relative_perplexity"]) and len(out["losses"]) == 3
    assert 0 <= out["accepted_per_step"] <= 2
    with pytest.raises(ValueError, match="heads"):
        RP.run(**SIZES, drafts=2)


def test_without_attention_nothing_changes():
    """The models of before, weight by weight."""
    require_gpu()
    a, b = RP.make_model(**SIZES), RP.make_model(**SIZES, heads=4)
    assert "heads" not in a and "qkv" not in a["layers"][0]
    assert torch.equal(a["head"], b["head"])
    for x, y in zip(a["layers"], b["layers"]):
        for name in ("gate", "up", "down"):
            assert all(torch.equal(s, t) for s, t in zip(x[name], y[name]))
    assert R.KVCache._fields == ("k", "v", "k_scale", "v_scale")
