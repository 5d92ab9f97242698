"""Decoding calls that leave something out, or have nothing to do."""
import random

import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_decode import BF16, Batch, ancestors, attend64, ints, packed, tree, within, words_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def test_trees_with_more_rows_together_than_a_mask_has_bits():
    sizes = [(33, 100)] * 5 + [(64, 64), (1, 9)]
    b = Batch(sizes, 2, 64, 16, seed=131)
    rng = random.Random(132)
    trees = [tree(rng, n) for n, _ in sizes]
    cache, table, starts, lens = b.cuda()
    masks = R.tree_masks(ints([p for t in trees for p in t]).cuda(), starts, 64)
    assert torch.equal(masks.cpu(), words_of([r for t in trees for r in ancestors(t)], 1))
    (q, qc), = packed(b.rows, [4], 64, BF16, 133)
    out, lse = R.kv_attention(qc, cache, table, starts, lens, masks=masks)
    o, z, bo, bl = attend64(b, q, masks.cpu(), 0.125)
    within(out, o, bo)
    within(lse, z, bl)


def test_no_sequence_at_all():
    """A batch that is all padding: starts of one element, and starts without rows."""
    p = torch.rand((9, 50), device="cuda")
    drafts, u = torch.zeros(9, device="cuda").long(), torch.zeros(9, device="cuda")
    parents = ints([-1] + list(range(8))).cuda()
    for starts in ([0], [0, 0, 0]):
        junk = [torch.full((9,), 7, dtype=t, device="cuda") for t in (torch.int64, torch.int32) * 4]
        del junk  # (so that new tensors hold 7)
        s = ints(starts).cuda()
        tokens, path, count = R.verify_drafts(p, p, drafts, u, s, parents=parents)
        assert (tokens == -1).all() and (path == -1).all() and count.tolist() == [0] * (len(starts) - 1)
        assert not R.tree_masks(parents, s, 9).any()
