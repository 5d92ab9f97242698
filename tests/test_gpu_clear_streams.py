"""The clear side's chain of operators on a stream of its own, with every tensor that it
reads made on that stream, or before the stream waited for the current one."""
import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_clear import BF16, EPS, gen, int8, normal, targets

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def chain(x, r, w, wq, ws, head, t, g, stream=None):
    o = R.rms_norm_q8(x, w, EPS, residual=r, stream=stream)
    y = R.q8_matmul(o.q, o.scale, wq, ws, stream=stream)
    z, h, inv = R.rms_norm(y, w, EPS, residual=o.h, stream=stream)
    loss, lse = R.cross_entropy(z, head, t, stream=stream)
    if g is None:
        with torch.cuda.stream(stream):
            g = torch.ones_like(loss)
    gz, gw = R.cross_entropy_backward(z, head, t, lse, g, stream=stream)
    gx, gn = R.rms_norm_backward(gz, h, w, inv, stream=stream)
    return loss, gw, gx, gn


@pytest.mark.parametrize("made", ["before the wait", "on the stream"])
@pytest.mark.parametrize("rows,dim,vocab", [(90, 256, 1000), (4000, 640, 8100)])
def test_factors_that_are_ready_on_the_stream(rows, dim, vocab, made):
    args = [normal(90, rows, dim, BF16), normal(91, rows, dim, BF16),
            normal(92, 1, dim, BF16)[0], int8(93, dim, dim),
            1e-3 * torch.rand(dim, generator=gen(94)),
            normal(95, vocab, dim, BF16, 0.1), targets(96, rows, vocab, 9)]
    args = [a.cuda() for a in args]
    ones = torch.ones(rows, device="cuda")
    want = [t.clone() for t in chain(*args, ones)]
    for _ in range(10):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = chain(*args, ones if made == "before the wait" else None, stream=side)
        side.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
