"""Attention of many rows of up to 64: the kernel of tiles, which is taken from 512
workgroups of 128 rows on, over everything that the other kernels are tested with."""
import math
import random

import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_decode import (BF16, F16, Batch, ancestors, attend64, check, gen, packed, tree,
                             within, words_of)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# sequences, heads, heads of the cache
CALLS = [([(130 + 5 * i, 130 + 13 * i) for i in range(16)], 16, 16),
         ([(140, 300), (65, 700), (1, 9), (0, 40), (129, 129), (128, 500), (33, 64)] * 3, 26, 13),
         ([(200, 210)] * 4, 128, 16)]


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def made(which, dim, page, seed, dtype, size=2.0):
    sizes, heads, kv = CALLS[which]
    rows = max(n for n, _ in sizes) * (heads // kv)
    # what the choice goes by (plan_of in kv_attention.hip)
    assert dim <= 64 and rows > 128 and len(sizes) * kv * -(-rows // 128) >= 512
    b = Batch(sizes, kv, dim, page, seed=seed)
    (q, qc), _ = packed(b.rows, [heads, 1], dim, dtype, seed + 1, size)
    return b, q, qc, max(n for n, _ in sizes)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,page", [(16, 16), (48, 64), (64, 32)])
@pytest.mark.parametrize("which", range(len(CALLS)))
def test_prompts(which, dim, page, dtype):
    b, q, qc, most = made(which, dim, page, 141, dtype)
    check(b, q, qc, max_rows=most)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [16, 48, 64])
@pytest.mark.parametrize("which", range(len(CALLS)))
def test_trees(which, dim, dtype):
    b, q, qc, most = made(which, dim, 16, 142, dtype)
    rng = random.Random(143)
    masks = words_of([r for n, _ in b.sizes if n for r in ancestors(tree(rng, n))], -(-most // 64))
    check(b, q, qc, masks, max_rows=most)
    # bits of any kind, rows without any, and nothing before the rows of one sequence
    masks = words_of([rng.getrandbits(64 * masks.shape[1]) if i % 3 else 0 for i in range(b.rows)],
                     masks.shape[1])
    check(b, q, qc, masks, max_rows=most)


@pytest.mark.parametrize("dim", [16, 48, 64])
def test_entries_that_name_no_page(dim):
    b, q, qc, most = made(0, dim, 16, 144, BF16)
    for i in range(0, 16, 2):
        b.table[i, i // 2] = [-1, b.pages, 1 << 30, -(1 << 31)][i // 2 % 4]
    b.table[3] = -7
    out, lse = check(b, q, qc, max_rows=most)
    at = slice(b.starts[3], b.starts[4])
    assert (out[at] == 0).all() and torch.isinf(lse[at]).all()


@pytest.mark.parametrize("dim", [48, 64])
def test_scales_of_either_sign(dim):
    b, q, qc, most = made(0, dim, 32, 145, F16)
    g = gen(146)
    for w in range(2):
        b.scale[w] *= torch.where(torch.rand(b.scale[w].shape, generator=g) < 0.5, -1.0, 1.0)
    pg, at = b.place(2, 60)
    b.scale[1][pg, :, at] = -300.0
    check(b, q, qc, max_rows=most)


@pytest.mark.parametrize("dim", [16, 64])
@pytest.mark.parametrize("which,value", [(0, math.nan), (0, math.inf), (0, -math.inf), (1, math.nan),
                                         (1, math.inf)])
def test_scales_that_are_no_numbers(dim, which, value):
    """Rows that see such a position are NaN; rows before it, other sequences, and what lies
    behind a length or in other pages are not touched."""
    b, q, qc, most = made(0, dim, 16, 147, BF16)
    o, z, bo, bl = attend64(b, q, None, dim ** -0.5)
    n, length = b.sizes[4]
    t = length - n + 70  # row 70 of the sequence is the first to see it
    pg, at = b.place(4, t)
    b.scale[which][pg, :, at] = value
    used = {b.place(i, t) for i, (_, length) in enumerate(b.sizes) for t in range(length)}
    for page in range(b.pages):
        for place in range(16):
            if (page, place) not in used:
                b.scale[which][page, :, place] = value
    out, lse = R.kv_attention(qc, *b.cuda(), max_rows=most)
    bad = slice(b.starts[4] + 70, b.starts[5])
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    keep = torch.ones(b.rows, dtype=torch.bool)
    keep[bad] = False
    within(out[keep.cuda()], o[keep], bo[keep])
    within(lse[keep.cuda()], z[keep], bl[keep])


def test_queries_that_are_no_numbers():
    b, q, qc, most = made(0, 64, 32, 148, F16)
    want, z = R.kv_attention(qc, *b.cuda(), max_rows=most)
    bad = qc.clone()
    bad[7, 3, 5], bad[900, 0, 63], bad[1500, 15, 0] = math.nan, math.inf, -math.inf
    out, lse = R.kv_attention(bad, *b.cuda(), max_rows=most)
    for r, h in ((7, 3), (900, 0), (1500, 15)):
        assert torch.isnan(out[r, h]).all() and torch.isnan(lse[r, h])
        out[r, h], lse[r, h] = want[r, h], z[r, h]
    assert torch.equal(out, want) and torch.equal(lse, z)


def test_rows_behind_and_rows_left_out():
    b, q, qc, most = made(0, 64, 32, 149, BF16)
    want, _ = R.kv_attention(qc, *b.cuda(), max_rows=most)
    more = torch.cat([qc, qc[:5]])
    out = torch.full_like(more, 7.0)
    R.kv_attention(more, *b.cuda(), max_rows=140, out=out)
    for i, (n, _) in enumerate(b.sizes):
        at = b.starts[i]
        assert torch.equal(out[at:at + min(n, 140)], want[at:at + min(n, 140)])
        assert (out[at + min(n, 140):b.starts[i + 1]] == 7).all()
    assert (out[b.rows:] == 7).all()
    # lengths behind the table: all of it is seen
    cache, table, starts, lens = b.cuda()
    short = table[:, :2].contiguous()
    out, lse = R.kv_attention(qc, cache, short, starts, lens, max_rows=most)
    i = 15
    assert b.sizes[i][1] > 64
    c = Batch([(1, 64)], 16, 64, 32, seed=149)
    c.table, c.q8, c.scale, c.pages = b.table[i:i + 1, :2], b.q8, b.scale, b.pages
    last = q[b.starts[i + 1] - 1:b.starts[i + 1]]
    o, z, bo, bl = attend64(c, last, None, 0.125)
    within(out[b.starts[i + 1] - 1:b.starts[i + 1]], o, bo)
    within(lse[b.starts[i + 1] - 1:b.starts[i + 1]], z, bl)
