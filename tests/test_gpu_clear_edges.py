"""Edges of the clear side on the GPU."""
import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_clear import BF16, EPS, F16, F32, normal

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


# ---------------------------------------------------------------- norm ---

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [1, 33, 1024, 3000, 4096, 16384, 17000])
def test_norm_weight_of_nan_and_infinity(dtype, dim):
    """A weight that is not finite leaves no finite scale: a NaN anywhere, NaN
    everywhere, an infinity on a column of zeros (their product is NaN) and on others."""
    rows, at = 5, dim - 1 - dim // 3
    x, r = normal(1, rows, dim, dtype), normal(2, rows, dim, dtype)
    x[:, at] = r[:, at] = 1
    zero = x.clone()
    zero[:, at] = -r[:, at]
    _, h0, inv0 = R.rms_norm(x.cuda(), None, EPS, residual=r.cuda())
    for wt in {dtype, F32}:
        for fill, where, h in ((float("nan"), [at], x), (float("nan"), slice(None), x),
                               (float("inf"), [at], zero), (float("-inf"), [at], x)):
            w = torch.ones(dim, dtype=wt)
            w[where] = fill
            o = R.rms_norm_q8(h.cuda(), w.cuda(), EPS, residual=r.cuda(), want_y=True)
            assert not torch.isfinite(o.scale).any()
            bad = ~torch.isfinite(o.y)
            assert bad[:, where].all() and int(bad.sum()) == rows * w[where].numel()
            if h is x:  # the weight has no part in these
                assert torch.equal(o.inv_rms, inv0) and torch.equal(o.h, h0)
            assert not torch.isfinite(R.dequantize_rows(o.q, o.scale, F32))[:, at].any()
