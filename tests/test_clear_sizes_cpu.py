"""Sizes that the entry points take but one launch would not (2^32 threads): refused before
anything is enqueued.  Through the C ABI with addresses that no device has."""
import pytest

from paper_2609_16915_amd import rosetta as R

UNSUPPORTED, BF16 = 3, 1
AT = [i << 50 for i in range(1, 10)]
MOST = (1 << 31) - 1


@pytest.mark.parametrize("m,n,k", [(1, MOST, 64), (100, MOST, 8), (1 << 20, (1 << 19) - 8, 16),
                                   (1, 1 << 29, 4096), (MOST, 200, 16)])
def test_products(m, n, k):
    st = R.lib().rosetta_q8_matmul(AT[0], k, AT[1], AT[2], k, AT[3], None, AT[4], n, BF16, m, n, k, None,
                                   0, None)
    assert st == UNSUPPORTED


# (tiles; the joining of their parts; a vocabulary for few rows)
@pytest.mark.parametrize("rows,dim,vocab", [(1 << 23, 64, 1 << 15), (1 << 27, 8, 100),
                                            (3, 1024, 1 << 30)])
def test_losses(rows, dim, vocab):
    L = R.lib()
    need = L.rosetta_cross_entropy_workspace_bytes(rows, dim, vocab)
    st = L.rosetta_cross_entropy(AT[0], dim, AT[1], dim, BF16, AT[2], -100, rows, dim, vocab, AT[3], AT[4],
                                 AT[5], need, None)
    assert st == UNSUPPORTED


# (the joining of gh's parts; h turned; h packed)
@pytest.mark.parametrize("rows,dim,vocab,gh,gw,stride", [
    (1 << 22, 1 << 12, 1000, True, True, 1 << 12), (1 << 24, 1 << 12, 1000, False, True, 1 << 12),
    (1 << 23, 1 << 12, 1000, False, True, (1 << 12) + 1)])
def test_gradients(rows, dim, vocab, gh, gw, stride):
    L = R.lib()
    need = L.rosetta_cross_entropy_backward_workspace_bytes(rows, dim, vocab)
    st = L.rosetta_cross_entropy_backward(
        AT[0], stride, AT[1], stride, BF16, AT[2], -100, AT[3], AT[4], rows, dim, vocab,
        AT[5] if gh else None, dim, AT[6] if gw else None, dim, AT[7], need, None)
    assert st == UNSUPPORTED
