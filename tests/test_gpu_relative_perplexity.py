"""The example that runs the clear side together: its layers against the same
model in 64 bits, its perplexities, and that its gradients fit."""
import math

import pytest

from paper_2609_16915_amd import relative_perplexity as RP
from paper_2609_16915_amd import rosetta as R
from paper_2609_16915_amd import workloads as W

from gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
D = torch.float64


def values(rows):
    q, scale = rows
    return q.to(D) * scale.to(D)[:, None]


def rounded(x):
    """8 bits with a scale per row, in 64 bits."""
    scale = x.abs().amax(1, keepdim=True) / 127
    return torch.round(x / scale) * scale


def hidden64(model, x, activation):
    residual, y = torch.zeros_like(x, dtype=D), x.to(D)
    for layer in model["layers"]:
        residual = residual + y
        n = residual / torch.sqrt((residual ** 2).mean(1, keepdim=True) + RP.EPS)
        n = rounded(n * layer["norm"].to(D))
        a = activation(n @ values(layer["gate"]).t()) * (n @ values(layer["up"]).t())
        y = rounded(a) @ values(layer["down"]).t()
    return y, residual


def test_layers_perplexities_and_fit():
    require_gpu()
    dim, ffn, vocab, tokens = 256, 704, 1000, 96
    model = RP.make_model(2, dim, ffn, vocab)
    x = torch.randn((tokens, dim), device="cuda",
                    generator=torch.Generator(device="cuda").manual_seed(5)).to(torch.bfloat16)
    y, residual = RP.hidden(model, x, RP.exact_silu)
    y64, residual64 = hidden64(model, x, RP.exact_silu)
    # bfloat16 between the steps: 2^-8 relative at each of a layer's four, which
    # move some values by a step of 8 bits (1/127 of a row's largest, four
    # deviations): together 3 % of the norm is far outside what they can do
    for got, want in ((y, y64), (residual, residual64)):
        assert float((got.to(D) - want).norm() / want.norm()) < 0.03
    out = RP.run(layers=2, dim=dim, ffn=ffn, vocab=vocab, tokens=tokens, steps=12)
    assert 1 < out["perplexity_exact"] < vocab
    assert math.isfinite(out["relative_perplexity"]) and out["relative_perplexity"] > 0.5
    assert out["losses"][-1] < out["losses"][0]
    assert out["perplexity_fitted"] < out["perplexity_table"]
    assert out["losses"][0] == pytest.approx(math.log(out["perplexity_table"]), rel=1e-6)


def test_table_is_what_the_encrypted_path_returns():
    """table_silu against Workload.quantize and Workload.table entry by entry."""
    require_gpu()
    w = W.get("llama3_8b_silu")
    x = torch.linspace(-9, 9, 4001, dtype=torch.float64, device="cuda")
    got = RP.table_silu(w)(x).cpu().numpy()
    m = w.quantize(x.cpu().numpy())
    assert (got == w.lo + (w.table()[m] + 0.5) * w.dx).all()
    assert R.lut_build(w.params(), w.table()).shape == (w.N,)
