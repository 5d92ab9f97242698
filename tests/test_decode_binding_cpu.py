"""The decoding binding where a call leaves something out, or has nothing to do: what the
library is given, and what comes back."""
import pytest
import torch

from paper_2609_16915_amd import rosetta as R
from test_decode_cpu import OnDevice, machine  # noqa: F401


@pytest.fixture
def given(machine, monkeypatch):  # noqa: F811
    """The arguments of every call that the library gets, by name."""
    calls = {}

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: calls.setdefault(name, a) and 0
            return lambda *a: calls.setdefault(name, a) and 0

    monkeypatch.setattr(R, "lib", Library)
    return calls


def on(t):
    return OnDevice(t, 0)


def ints(*v):
    return on(torch.tensor(v, dtype=torch.int32))


def cache():
    return R.KVCache(*(on(torch.zeros((2, 1, 16, 64), dtype=torch.int8)) for _ in range(2)),
                     *(on(torch.zeros((2, 1, 16))) for _ in range(2)))


MAX_ROWS, MASKS, WORDS = 7, 8, 9  # of rosetta_kv_attention


@pytest.mark.parametrize("rows,words,given_rows,want", [
    (528, 1, None, 64),   # sixteen trees of 33
    (528, 3, None, 192), (100, 2, None, 100), (528, 1, 33, 33), (40, 1, 99, 40),
    (5, 0, None, 5),      # (masks of no words: refused by the library)
])
def test_rows_of_a_sequence_follow_from_the_masks(given, rows, words, given_rows, want):
    q = on(torch.zeros((rows, 1, 64), dtype=torch.bfloat16))
    masks = on(torch.zeros((rows, words), dtype=torch.int64))
    R.kv_attention(q, cache(), on(torch.zeros((2, 2), dtype=torch.int32)), ints(0, 3, rows),
                   ints(5, 5), masks=masks, max_rows=given_rows)
    a = given["rosetta_kv_attention"]
    assert (a[MAX_ROWS], a[WORDS]) == (want, words) and a[MASKS] == masks.data_ptr()


def test_without_masks_all_rows(given):
    q = on(torch.zeros((528, 1, 64), dtype=torch.bfloat16))
    R.kv_attention(q, cache(), on(torch.zeros((1, 2), dtype=torch.int32)), ints(0, 528), ints(600))
    assert given["rosetta_kv_attention"][MAX_ROWS] == 528


def test_nothing_verified_and_no_masks_where_there_is_no_sequence(given, monkeypatch):
    """Rows of no sequence hold -1, and no bits, where there is no sequence at all."""
    monkeypatch.setattr(OnDevice, "new_empty", lambda self, shape, dtype=None: on(
        torch.full(shape if isinstance(shape, tuple) else (shape,), 7, dtype=dtype or self.dtype)))
    p = on(torch.zeros((3, 9)))
    tokens, path, count = R.verify_drafts(p, p, on(torch.zeros(3).long()), on(torch.zeros(3)), ints(0))
    assert tokens.tolist() == [-1] * 3 and path.tolist() == [-1] * 3 and count.numel() == 0
    assert tokens.dtype is torch.int64 and path.dtype is torch.int32
    assert R.tree_masks(ints(-1, 0, 1), ints(0), 70).tolist() == [[0, 0]] * 3
