"""Verification where the drafter has no distribution: rows of q whose node has no
children, or none that takes part, may hold anything."""
import math

import pytest

from gpu_helpers import require_gpu
from test_gpu_decode import BF16, F16, F32, drafted, verify, verify64

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def leaves(drafts, starts, parents, vocab):
    """Rows that no node with a token of the vocabulary has for its parent."""
    inner = set()
    for b in range(len(starts) - 1):
        for i in range(1, starts[b + 1] - starts[b]):
            r = starts[b] + i
            if 0 <= int(drafts[r]) < vocab:
                inner.add(starts[b] + (i - 1 if parents is None else parents[r]))
    return [r for r in range(starts[-1]) if r not in inner]


def poisoned(q, rows, value):
    bad = q.clone()
    if value == "each":
        few = torch.tensor([math.nan, math.inf, -math.inf, 1.0]).to(q.dtype)
        bad[rows] = few.repeat(-(-q.shape[1] // 4))[:q.shape[1]]
    else:
        bad[rows] = value
    return bad


@pytest.mark.parametrize("chain", [False, True])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, "each"])
@pytest.mark.parametrize("vocab", [37, 5000, 8193, 50257])  # without and with launches before the last
def test_leaf_rows_of_q_may_hold_anything(chain, value, vocab):
    # noise 0: q is p, and every walk goes on to a leaf
    for seed, sizes, noise in ((1, [5], 0.0), (2, [1, 12, 0, 33, 2] * 2, 0.0), (3, [20] * 4, 0.7)):
        p, q, drafts, u, starts, parents = drafted(sizes, vocab, 200 * seed + vocab % 89, chain,
                                                   noise=noise)
        want = verify64(p, q, drafts, u, starts, parents)
        if noise == 0.0 and chain:
            assert want[2] == sizes
        rows = leaves(drafts, starts, parents, vocab)
        assert verify(p, poisoned(q, rows, value), drafts, u, starts, parents) == want


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_every_row_a_leaf(dtype):
    """Tokens that no vocabulary has: the last token is drawn from p at the root."""
    vocab = 9001
    p, q, drafts, u, starts, parents = drafted([4, 4, 9], vocab, 48, False, dtype=dtype)
    drafts[:] = torch.tensor([-1, vocab, 1 << 40])[torch.arange(17) % 3]
    want = verify64(p, q, drafts, u, starts, parents)
    assert want[2] == [1, 1, 1]
    for value in (math.nan, math.inf):
        assert verify(p, torch.full_like(q, value), drafts, u, starts, parents) == want


def test_nothing_left_is_drawn_from_p_whatever_q_holds():
    """A rejection that leaves nothing (q at least p everywhere) draws from p itself: where
    q is infinite, too."""
    vocab = 8500
    p, q, drafts, u, starts, _ = drafted([2, 2], vocab, 49, True)
    q = 2 * p + 1
    q[2, 7:] = math.inf
    u[1] = u[3] = 0.9999
    drafts[:] = 5
    assert verify(p, q, drafts, u, starts, None) == verify64(p, q, drafts, u, starts, None)


@pytest.mark.parametrize("shift", [0, 64, 256])
def test_a_draw_on_a_border_next_to_words_without_weight(shift):
    """1, then words of 2^-53 among words of 0: partial sums differ by their order in the last
    bit, and a draw that is exactly 1 lies between two of them, at a word of weight 0.  What
    follows is the next word that has any, not the last of all."""
    p = torch.zeros((1, 600))
    for at, w in ((0, 1.0), (1, 2.0 ** -53), (3, 2.0 ** -53), (13, 1.0), (150, 1.0), (199, 1.0)):
        p[0, shift + at] = w
    u = torch.tensor([0.25])  # of 4
    tokens, path, count = verify(p, p, torch.zeros(1).long(), u, [0, 1], None)
    assert tokens[0] - shift in (1, 3, 13) and path == [0] and count == [1]
