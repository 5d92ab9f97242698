"""Caches whose keys and values, or their scales, alternate within a page, and outputs that
alternate within a row: the same bits as with arrays of their own."""
import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_decode import BF16, F32, Batch, ints, packed

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def alternating(kind, pages, heads, page, dim):
    """(k, v) views of one buffer, [pages][heads][page][dim], and the buffer."""
    if kind == "in a place":
        buf = torch.zeros((pages, page, 2, heads, dim), dtype=torch.int8, device="cuda")
        return buf[:, :, 0].transpose(1, 2), buf[:, :, 1].transpose(1, 2)
    if kind == "in a head of a place":
        buf = torch.zeros((pages, page, heads, 2, dim), dtype=torch.int8, device="cuda")
        return buf[:, :, :, 0].transpose(1, 2), buf[:, :, :, 1].transpose(1, 2)
    if kind == "in a head":
        buf = torch.zeros((pages, heads, 2, page, dim), dtype=torch.int8, device="cuda")
        return buf[:, :, 0], buf[:, :, 1]
    buf = torch.zeros((pages, heads, page, 2, dim), dtype=torch.int8, device="cuda")
    return buf[:, :, :, 0], buf[:, :, :, 1]


@pytest.mark.parametrize("kind", ["in a place", "in a head of a place", "in a head", "in a row"])
@pytest.mark.parametrize("heads,dim,page", [(2, 64, 16), (4, 128, 32), (1, 16, 16), (3, 80, 64)])
def test_keys_and_values_that_alternate(kind, heads, dim, page):
    b = Batch([(20, 50), (1, 33), (0, 7), (40, 40)], heads, dim, page, seed=121)
    plain, table, starts, lens = b.cuda()
    k, v = alternating(kind, b.pages, heads, page, dim)
    scales = torch.zeros((b.pages, heads, 2, page), device="cuda")
    both = R.KVCache(k, v, scales[:, :, 0], scales[:, :, 1])
    for t, s in zip(both, plain):
        t.copy_(s)
    where = (table, starts, lens)
    (x, xc), (y, yc), (q, qc) = packed(b.rows, [heads, heads, 2 * heads], dim, BF16, 122)
    for cache in (plain, both):
        R.kv_write(xc, yc, cache, *where)
    path = ints([0] + list(range(3, 20)) + [-1] * 2 + [0] + list(range(0, 40, 2)) + [-1] * 20).cuda()
    count = ints([18, 1, 0, 20]).cuda()
    new = [R.kv_keep(cache, *where, path, count) for cache in (plain, both)]
    assert torch.equal(*new)
    for t, s in zip(both, plain):
        assert torch.equal(t, s)
    outs = [R.kv_attention(qc, cache, *where) for cache in (plain, both)]
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    # keys and values read side by side, [rows][heads][2][dim]
    want = R.kv_read(plain, *where, b.rows, F32)
    buf = torch.full((b.rows, heads, 2, dim), 7.0, device="cuda")
    R.kv_read(both, *where, b.rows, F32, buf[:, :, 0], buf[:, :, 1])
    for got, w in zip((buf[:, :, 0], buf[:, :, 1]), want):
        assert torch.equal(got, w)


def test_an_output_beside_the_queries():
    """[rows][heads][2][dim]: queries and outputs in turn."""
    b = Batch([(5, 60), (64, 64)], 2, 64, 16, seed=123)
    (q, qc), = packed(b.rows, [4], 64, BF16, 124)
    want, _ = R.kv_attention(qc, *b.cuda())
    buf = torch.zeros((b.rows, 4, 2, 64), dtype=BF16, device="cuda")
    buf[:, :, 0] = qc
    R.kv_attention(buf[:, :, 0], *b.cuda(), out=buf[:, :, 1])
    assert torch.equal(buf[:, :, 1], want) and torch.equal(buf[:, :, 0], qc)
