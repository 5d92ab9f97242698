"""Decoding in the clear at its edges: alignments, strides, signs and sizes of scales,
parts of long sequences, caches past 32 bits, graphs, streams and shared workspaces."""
import math
import random

import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_decode import (BF16, D, F16, F32, Batch, ancestors, attend64, check, drafted,
                             eight_bits, gen, ints, packed, tree, verify, verify64, within,
                             words_of)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def shifted(t, by, pad):
    """The same [rows][heads][dim] on the GPU, `by` elements into a buffer whose rows are
    `pad` further apart than their elements need."""
    rows, heads, dim = t.shape
    width = heads * dim + pad
    buf = torch.full((by + rows * width,), 7.0, dtype=t.dtype, device="cuda")
    m = buf[by:by + rows * width].view(rows, width)[:, :heads * dim].view(rows, heads, dim) \
        if pad == 0 else buf[by:].view(rows, width)[:, :heads * dim].unflatten(1, (heads, dim))
    m.copy_(t)
    return m


@pytest.mark.parametrize("by,pad", [(1, 0), (3, 5), (0, 1), (8, 16)])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (5, 5, 80), (2, 1, 256), (8, 2, 128)])
def test_elements_off_every_alignment(by, pad, heads, kv, dim):
    b = Batch([(3, 40), (1, 1), (20, 33)], kv, dim, 16, seed=61)
    q = torch.randn((b.rows, heads, dim), generator=gen(62)).to(BF16)
    qc = shifted(q, by, pad)
    want, lse = check(b, q, q.cuda())
    out = shifted(torch.zeros_like(q), by, pad)
    got, lse2 = R.kv_attention(qc, *b.cuda(), out=out)
    assert torch.equal(got, want) and torch.equal(lse2, lse)
    for dtype in (BF16, F32):
        k = torch.randn((b.rows, kv, dim), generator=gen(63)).to(dtype)
        cache = b.cuda()
        R.kv_write(shifted(k, by, pad), shifted(k, by + 1, pad), *cache)
        ko, vo = (shifted(torch.zeros_like(k), by, pad) for _ in range(2))
        R.kv_read(*cache, b.rows, dtype, ko, vo)
        e, s = eight_bits(k)
        for t in (ko, vo):
            assert torch.equal(t.cpu(), (e.float() * s[..., None]).to(dtype))


# rows on both sides of every choice between the kernels, lengths with and without parts
SIZES = [[(1, 5000)], [(16, 4000)], [(17, 600)], [(33, 700), (1, 3000)], [(128, 2500)], [(129, 129)],
         [(300, 2300), (5, 5), (64, 1111)], [(700, 700)]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 64), (8, 1, 64), (2, 1, 128), (3, 1, 256)])
def test_every_kernel(sizes, heads, kv, dim):
    b = Batch(sizes, kv, dim, 32, seed=64)
    (q, qc), _ = packed(b.rows, [heads, 1], dim, F16, 65, 2.0)
    check(b, q, qc, max_rows=max(n for n, _ in sizes))


@pytest.mark.parametrize("sizes", [[(130, 900)], [(64, 3000), (200, 260)]])
@pytest.mark.parametrize("heads,kv,dim", [(4, 1, 128), (2, 2, 256), (32, 16, 64)])
def test_trees_in_every_kernel(sizes, heads, kv, dim):
    b = Batch(sizes, kv, dim, 16, seed=66)
    rng = random.Random(67)
    most = max(n for n, _ in sizes)
    masks = words_of([r for n, _ in sizes for r in ancestors(tree(rng, n))], -(-most // 64) + 1)
    (q, qc), _ = packed(b.rows, [heads, 1], dim, BF16, 68, 2.0)
    check(b, q, qc, masks, max_rows=most)


def test_large_batches_of_ragged_prompts_over_all_xcds():
    """Enough work for the kernel of many rows of 64, with sequences of every length."""
    sizes = [(n, n + 7 * n % 50) for n in (513, 700, 64, 1, 300, 511, 129, 640)]
    b = Batch(sizes, 16, 64, 16, seed=69)
    (q, qc), = packed(b.rows, [128], 64, BF16, 70, 2.0)
    check(b, q, qc, max_rows=700)


@pytest.mark.parametrize("n,length,heads,dim", [(1, 4000, 4, 64), (3, 9000, 4, 128), (200, 3000, 2, 128),
                                                (1, 5000, 2, 256)])
def test_no_numbers_in_parts(n, length, heads, dim):
    """What is no number in one row, or one position, shows though the sequence is cut."""
    b = Batch([(n, length)], 1, dim, 64, seed=71)
    (q, qc), _ = packed(n, [heads, 1], dim, BF16, 72)
    bad = qc.clone()
    bad[0, 0, 3] = math.nan
    out, lse = R.kv_attention(bad, *b.cuda())
    want, z = R.kv_attention(qc, *b.cuda())
    assert torch.isnan(out[0, 0]).all() and torch.isnan(lse[0, 0])
    out[0, 0], lse[0, 0] = want[0, 0], z[0, 0]
    assert torch.equal(out, want) and torch.equal(lse, z)
    for which, value in ((0, math.inf), (0, -math.inf), (0, math.nan), (1, math.inf), (1, math.nan)):
        pg, at = b.place(0, length // 2)
        kept = b.scale[which][pg, 0, at].item()
        b.scale[which][pg, 0, at] = value
        out, lse = R.kv_attention(qc, *b.cuda())
        assert torch.isnan(out).all()
        b.scale[which][pg, 0, at] = kept


@pytest.mark.parametrize("n,heads,dim", [(1, 4, 64), (40, 4, 128), (200, 2, 128), (30, 3, 256)])
def test_scales_of_either_sign(n, heads, dim):
    """value = scale q, whatever the scale's sign; a large negative one sets the range."""
    b = Batch([(n, 500)], 1, dim, 16, seed=73)
    g = gen(74)
    for w in range(2):
        b.scale[w] *= torch.where(torch.rand(b.scale[w].shape, generator=g) < 0.5, -1.0, 1.0)
    pg, at = b.place(0, 123)
    b.scale[1][pg, 0, at] = -3e4
    (q, qc), _ = packed(n, [heads, 1], dim, BF16, 75)
    check(b, q, qc)


def test_a_cache_past_32_bits():
    """Pages whose keys and values lie past 2^32 bytes, first and last of the cache."""
    pages, heads, page, dim = 8400, 8, 256, 256
    k, v = (torch.empty((pages, heads, page, dim), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((pages, heads, page), math.nan, device="cuda") for _ in range(2))
    cache = R.KVCache(k, v, ks, vs)
    assert (pages - 1) * heads * page * dim > 1 << 32
    rows = 600
    (x, xc), (y, yc), (q, qc) = packed(rows, [heads, heads, 16], dim, BF16, 76)
    table = ints([pages - 1, 0, pages // 2]).view(1, 3).cuda()
    starts, lens = ints([0, rows]).cuda(), ints([rows]).cuda()
    R.kv_write(xc, yc, cache, table, starts, lens)
    for got, want in zip(R.kv_read(cache, table, starts, lens, rows, F32), (x, y)):
        e, s = eight_bits(want)
        assert torch.equal(got.cpu(), e.float() * s[..., None])
    out, lse = R.kv_attention(qc, cache, table, starts, lens)
    small = Batch([(rows, rows)], heads, dim, page, seed=77)
    for w, t in enumerate((x, y)):
        e, s = eight_bits(t)
        for r in range(rows):
            pg, at = small.place(0, r)
            small.q8[w][pg, :, at], small.scale[w][pg, :, at] = e[r], s[r]
    again, lse2 = R.kv_attention(qc, *small.cuda())
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    path = ints([0] + list(range(2, 301)) + [-1] * 300).cuda()
    new = R.kv_keep(cache, table, starts, lens, path, ints([300]).cuda())
    assert new.tolist() == [300]
    got, _ = R.kv_read(cache, table, ints([0, 300]).cuda(), new, 300, F32)
    e, s = eight_bits(x[[0] + list(range(2, 301))])
    assert torch.equal(got.cpu(), e.float() * s[..., None])


def test_many_sequences():
    """More than the starts that a workgroup keeps at hand."""
    sizes = [(i % 3, 20 + i % 40) for i in range(1500)]
    b = Batch(sizes, 1, 16, 16, seed=78)
    cache, table, starts, lens = b.cuda()
    (k, kc), (q, qc) = packed(b.rows, [1, 2], 16, BF16, 79)
    R.kv_write(kc, kc, cache, table, starts, lens)
    for i, (n, length) in enumerate(sizes):
        for j in range(n):
            pg, at = b.place(i, length - n + j)
            for w in range(2):
                b.q8[w][pg, :, at], b.scale[w][pg, :, at] = eight_bits(k[b.starts[i] + j])
    b.same(cache)
    check(b, q, qc, max_rows=2)
    parents = ints([j - 1 for n, _ in sizes for j in range(n)])
    masks = R.tree_masks(parents.cuda(), starts, 2)
    assert masks[:, 0].tolist() == [(1 << j + 1) - 1 for n, _ in sizes for j in range(n)]


@pytest.mark.parametrize("most", [1, 65, 3000])
def test_masks_of_deep_trees(most):
    """Chains of many words, and of fewer words than rows; a row behind them."""
    parents, follows = [], []
    for n in (3000, 1, 700):
        parents += list(range(-1, n - 1))
        follows += [(1 << i + 1) - 1 for i in range(n)]
    starts = ints([0, 3000, 3001, 3001, 3701]).cuda()
    words = -(-most // 64)
    got = R.tree_masks(ints(parents + [0]).cuda(), starts, most).cpu()
    assert torch.equal(got, words_of([m % (1 << 64 * words) for m in follows + [0]], words))


def test_heads_of_one_group():
    b = Batch([(1, 300), (3, 77)], 1, 128, 32, seed=80)
    (q, qc), = packed(b.rows, [128], 128, BF16, 81)
    check(b, q, qc, max_rows=3)


def test_scale_zero_and_lse_not_wanted():
    b = Batch([(2, 50)], 2, 64, 16, seed=82)
    (q, qc), = packed(2, [4], 64, BF16, 83)
    out, lse = check(b, q, qc, scale=0.0)  # the mean of what is seen
    got, none = R.kv_attention(qc, *b.cuda(), scale=0.0, want_lse=False)
    assert none is None and torch.equal(got, out)


def test_prompts_captured_and_workspaces_shared():
    """Graphs of the kernels of many rows and of parts, which share one workspace, replayed
    in turn with eager calls between."""
    calls = []
    for sizes, heads, kv, dim in (([(300, 2300), (64, 1111)], 4, 1, 128), ([(1, 5000)], 4, 2, 64),
                                  ([(70, 4000)], 2, 1, 256), ([(700, 700)] * 2, 64, 64, 64)):
        b = Batch(sizes, kv, dim, 32, seed=84)
        (q, qc), _ = packed(b.rows, [heads, 1], dim, BF16, 85)
        calls.append((qc, b.cuda(), max(n for n, _ in sizes)))
    want = [R.kv_attention(q, *c, max_rows=m) for q, c, m in calls]
    work = torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for q, _, _ in calls]
    graphs = []
    torch.cuda.synchronize()
    for (q, c, m), out in zip(calls, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            R.kv_attention(q, *c, max_rows=m, out=out, workspace=work)
        graphs.append(g)
    for turn in range(3):
        for i in (0, 1, 2, 3, 1, 0, 3, 2):
            outs[i].fill_(3)
            graphs[i].replay()
            if turn == 1:
                R.kv_attention(calls[0][0], *calls[0][1], max_rows=calls[0][2])
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i][0])


def test_two_streams_at_once():
    calls = []
    for seed in (86, 87):
        b = Batch([(1, 6000), (40, 900)], 2, 128, 16, seed=seed)
        (q, qc), _ = packed(b.rows, [8, 1], 128, BF16, seed)
        calls.append((qc, b.cuda()))
    want = [R.kv_attention(q, *c) for q, c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for _ in range(10):
        got = [R.kv_attention(q, *c, stream=s) for (q, c), s in zip(calls, streams)]
    for s in streams:
        s.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_what_a_captured_step_reads_may_change():
    """Lengths, tables and starts are read when a graph runs: a token more each time."""
    b = Batch([(1, 30), (1, 61)], 2, 64, 16, seed=88, more=3)
    cache, table, starts, lens = b.cuda()
    (q, qc), (k, kc) = packed(2, [4, 2], 64, BF16, 89)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        R.kv_write(kc, kc, cache, table, starts, lens)
        out, lse = R.kv_attention(qc, cache, table, starts, lens, max_rows=1)
    e, s = eight_bits(k)
    for step in range(40):
        graph.replay()
        for i, (n, length) in enumerate(b.sizes):
            at = b.place(i, length - 1)
            for w in range(2):
                b.q8[w][at[0], :, at[1]], b.scale[w][at[0], :, at[1]] = e[i], s[i]
        if step % 8 == 7:
            o, z, bo, bl = attend64(b, q, None, 0.125)
            within(out, o, bo)
            within(lse, z, bl)
        lens += 1
        torch.cuda.synchronize()
        b.sizes = [(n, length + 1) for n, length in b.sizes]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distributions_in_rows_apart(dtype):
    p, q, drafts, u, starts, parents = drafted([9, 14], 30001, 90, False, dtype=dtype)
    far = []
    for t in (p, q):
        buf = torch.full((t.shape[0], t.shape[1] + 7), math.nan, dtype=dtype, device="cuda")
        m = buf[:, 3:3 + t.shape[1]]
        m.copy_(t)
        far.append(m)
    got = R.verify_drafts(far[0], far[1], drafts.cuda(), u.cuda(), ints(starts).cuda(),
                          parents=ints(parents).cuda())
    assert tuple(t.tolist() for t in got) == verify64(p, q, drafts, u, starts, parents)


def test_more_nodes_than_take_part():
    """1500 nodes in a row with the drafter's distribution that of the target: all of the
    first 1024 are kept, and none behind."""
    n, vocab = 1500, 50
    p = torch.softmax(torch.randn((n, vocab), generator=gen(91)), 1)
    drafts = torch.cat([torch.zeros(1).long(), torch.multinomial(p[:-1], 1, generator=gen(92))[:, 0]])
    u = torch.rand(n, generator=gen(93))
    got = verify(p, p, drafts, u, [0, n], None)
    assert got == verify64(p, p, drafts, u, [0, n], None)
    assert got[2] == [1024] and got[1][1023] == 1023 and got[1][1024] == -1


def test_verification_with_a_shared_workspace_and_replayed():
    sets = [drafted([20, 3, 31], 70001, s, False) for s in (94, 95)]
    work = torch.full((1 << 16,), 255, dtype=torch.uint8, device="cuda")
    graphs, outs, want = [], [], []
    for p, q, drafts, u, starts, parents in sets:
        args = (p.cuda(), q.cuda(), drafts.cuda(), u.cuda(), ints(starts).cuda())
        par = ints(parents).cuda()
        want.append(verify64(p, q, drafts, u, starts, parents))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(R.verify_drafts(*args, parents=par, workspace=work))
        graphs.append((g, args, par))
    for _ in range(3):
        for i in (0, 1, 1, 0):
            for t in outs[i]:
                t.fill_(5)
            graphs[i][0].replay()
            torch.cuda.synchronize()
            assert tuple(t.tolist() for t in outs[i]) == want[i]
            work.fill_(255)


def test_results_do_not_depend_on_what_lies_around():
    """A sequence alone, and among others: the same bits where the parts are the same."""
    b = Batch([(1, 700)] * 5, 2, 64, 16, seed=96)
    (q, qc), = packed(5, [4], 64, F16, 97)
    cache, table, starts, lens = b.cuda()
    o, z, bo, bl = attend64(b, q, None, 0.125)
    out, _ = R.kv_attention(qc, cache, table, starts, lens, max_rows=1)
    within(out, o, bo)
    for i in range(5):
        one, _ = R.kv_attention(qc[i:i + 1], cache, table[i:i + 1], ints([0, 1]).cuda(), lens[i:i + 1])
        within(one, o[i:i + 1], bo[i:i + 1])
    assert D is torch.float64
