"""Attention over caches whose scales are of any size: past 2^100, far apart from each
other, and keys whose scales make up for tiny queries.

Bounds: a score as in attend64 (test_gpu_decode).  The products p_t v_scale[t] become
weights of f16, the largest of a row's between 2^-2 and 2^15, so that a weight is off by
2^-11 of itself or, where it is small, by 2^-25, which is at most 2^-23 of the largest."""
import math

import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_decode import (BF16, D, E, F16, F32, U, Batch, ancestors, gen, packed,
                             seen_fast, tree, within, words_of)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def attend64(b, q, masks, scale):
    """(out, lse, bound of out, bound of lse)."""
    rows, heads, dim = q.shape
    group = heads // b.heads
    zero = torch.zeros((), dtype=D)
    out, lse = torch.zeros((rows, heads, dim), dtype=D), torch.full((rows, heads), -math.inf, dtype=D)
    bo, bl = torch.zeros_like(out), torch.zeros((rows, heads), dtype=D)
    for i, (n, length) in enumerate(b.sizes):
        k, there = b.values(i, 0, length)
        v, _ = b.values(i, 1, length)
        finite = torch.isfinite(k).all(2) & torch.isfinite(v).all(2)
        k, v = (torch.where(finite[..., None], t, zero) for t in (k, v))
        vs = torch.stack([b.scale[1][b.place(i, t)[0], :, b.place(i, t)[1]].abs().to(D)
                          if there[t] else torch.zeros(b.heads, dtype=D) for t in range(length)], 1)
        seen = seen_fast(b, i, masks) & there[None]
        at = slice(b.starts[i], b.starts[i] + n)
        for h in range(heads):
            x, g = q[at, h].to(D), h // group
            sees = seen & finite[g][None] if masks is not None else seen
            s = (x @ k[g].t() * scale).masked_fill(~sees, -math.inf)
            z = torch.logsumexp(s, 1)
            p = torch.where(sees, torch.exp(s - z.nan_to_num(0, 0, 0)[:, None]), zero)
            lse[at, h] = z
            out[at, h] = p @ v[g]
            mags = (x.abs() @ k[g].abs().t() * scale).masked_fill(~sees, 0).amax(1)
            es = ((dim + 9) * E * mags + 8 * E)[:, None]
            largest = (p * torch.where(finite[g], vs[g], zero)[None]).amax(1)
            few = sees.sum(1) * 2.0 ** -23 * largest * 128
            bo[at, h] = p @ v[g].abs() * (U[F16] + 2 * es + (length + 64) * E) + few[:, None]
            # (reference and logarithm of the sum: up to 128 each beside the result)
            bl[at, h] = es[:, 0] + (length + 64) * E + 4 * E * (160 + z.abs().nan_to_num(0, 0, 0))
    bo = bo + U[q.dtype] * (out.abs() + bo) + (2.0 ** -25 if q.dtype == F16 else 0)
    return out, lse, bo, bl


def check(b, q, masks=None, scale=None):
    qc = q.cuda()
    out, lse = R.kv_attention(qc, *b.cuda(), scale=scale, max_rows=max(n for n, _ in b.sizes),
                              masks=None if masks is None else masks.cuda())
    o, z, bo, bl = attend64(b, q, masks, b.dim ** -0.5 if scale is None else scale)
    within(lse, z, bl)
    within(out, o, bo)
    return out, lse


# (sizes, heads, heads of the cache, dim): a kernel each, with and without parts
CALLS = {
    "one row": ([(1, 700)], 4, 1, 64),
    "one row, parts": ([(1, 3000)], 4, 1, 128),
    "rows": ([(20, 500), (3, 260)], 4, 2, 128),
    "rows of 80": ([(9, 300)], 6, 2, 80),
    "rows of 256": ([(7, 400)], 4, 1, 256),
    "tiles of 128": ([(140, 900), (33, 33)], 2, 1, 128),
    "tiles of 96": ([(140, 300)], 2, 1, 96),
    "tiles of 256": ([(40, 500), (70, 71)], 2, 1, 256),
    "tiles of 64": ([(130 + i, 130 + 3 * i) for i in range(16)], 16, 16, 64),
}


def call(name, seed, page=16):
    sizes, heads, kv, dim = CALLS[name]
    if name == "tiles of 64":  # (the kernel of tiles is taken from 512 workgroups on)
        assert len(sizes) * kv * -(-max(n for n, _ in sizes) * heads // kv // 128) >= 512
    b = Batch(sizes, kv, dim, page, seed=seed)
    q = torch.randn((b.rows, heads, dim), generator=gen(seed + 1))
    return b, q


def at_places(b, f):
    """f(i, t, page, place) for every position of every sequence."""
    for i, (_, length) in enumerate(b.sizes):
        for t in range(length):
            pg, at = b.place(i, t)
            f(i, t, pg, at)


def masks_of(b):
    import random
    rng = random.Random(5)
    most = max(n for n, _ in b.sizes)
    return words_of([r for n, _ in b.sizes for r in ancestors(tree(rng, n))], -(-most // 64))


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("low,high", [(100, 121), (60, 121), (-60, 119), (99, 101)])
def test_scales_of_values_past_2_to_the_100(name, masked, low, high):
    b, q = call(name, 101)
    g = gen(102)
    size = torch.randint(low, high, b.scale[1].shape, generator=g).float()
    b.scale[1] = torch.exp2(size) * (1 + torch.rand(size.shape, generator=g)) / 2
    check(b, q.to(BF16), masks_of(b) if masked else None)


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("where", ["first", "last", "spread"])
def test_a_huge_value_among_ordinary_ones(name, where):
    """Rows before it keep their values, rows behind it take its."""
    b, q = call(name, 103)
    for i, (n, length) in enumerate(b.sizes):
        for t in {"first": [0], "last": [length - 1], "spread": [length // 3, length - n // 2 - 1]}[where]:
            pg, at = b.place(i, t)
            b.scale[1][pg, :, at] = -(2.0 ** 118)
    out, _ = check(b, q.to(BF16))
    if where == "last":
        assert (out[0].abs() < 100).all() or b.sizes[0][0] == 1


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("power", [105, 125])
def test_huge_scales_of_keys_and_tiny_queries(name, masked, power):
    """Scores of some tens from queries of 2^-power and keys of 2^power, beside keys of
    ordinary size, whose scores are 0."""
    b, q = call(name, 104)
    b.scale[0] *= torch.where(torch.rand(b.scale[0].shape, generator=gen(105)) < 0.3, 2.0 ** power, 1.0)
    check(b, (q * 2.0 ** -power).to(BF16), masks_of(b) if masked else None, scale=4.0 * b.dim ** -0.5)


@pytest.mark.parametrize("name", list(CALLS))
def test_tiny_queries(name):
    """Scores of some tens from queries of 2^-123, scales of keys of 2^93 and a scale of 2^28."""
    b, q = call(name, 115)
    b.scale[0] *= 2.0 ** 99
    check(b, (q * 2.0 ** -123).to(BF16), scale=2.0 ** 24)


@pytest.mark.parametrize("name", list(CALLS))
def test_unseen_keys_of_every_size_beside_huge_queries(name):
    b, q = call(name, 116)
    b.scale[0] *= 2.0 ** -112
    used = set()
    at_places(b, lambda i, t, pg, at: used.add((pg, at)))
    for pg in range(b.pages):
        for at in range(b.page):
            if (pg, at) not in used:
                b.scale[0][pg, :, at] = [2.0 ** 120, -(2.0 ** 126), 0.0][(pg + at) % 3]
    check(b, (q * 2.0 ** 112).to(BF16))


@pytest.mark.parametrize("name", list(CALLS))
def test_tiny_scales_of_keys_and_huge_queries(name):
    b, q = call(name, 106)
    b.scale[0] *= 2.0 ** -112
    check(b, (q * 2.0 ** 112).to(BF16))


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("power", [97, 125])
def test_no_scale_gives_the_mean_whatever_the_keys_are(name, power):
    b, q = call(name, 107)
    b.scale[0] *= 2.0 ** power
    check(b, q.to(BF16), scale=0.0)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("power", [20, 32, 48, 70])
@pytest.mark.parametrize("where", [0.0, 0.5, 1.0])
def test_a_large_value_that_weighs_nothing(name, dtype, power, where):
    """A position whose value is 2^power times the others' and whose weight is some e^-70
    of theirs: the output is that of the others."""
    b, q = call(name, 108)
    q = q.abs() + 0.5  # (so that keys of one sign score below all others)
    dim = b.dim
    b.scale[0] *= 0.1  # the others' scores near each other
    for i, (n, length) in enumerate(b.sizes):
        if n == length and dtype == F16:
            continue  # (its first row would see nothing else, and its type does not hold that)
        pg, at = b.place(i, int((length - n) * where))
        b.q8[0][pg, :, at] = -127
        b.scale[0][pg, :, at] = 70 / (127 * math.sqrt(dim) * 1.2)
        b.scale[1][pg, :, at] = 2.0 ** (power - 6)
    out, _ = check(b, q.to(dtype))
    assert out[b.sizes[0][0] - 1].abs().max() < 5


@pytest.mark.parametrize("name", list(CALLS))
def test_scales_of_values_over_the_whole_range(name):
    """From 2^-75 to 2^90, in any order, zeros among them."""
    b, q = call(name, 109)
    g = gen(110)
    size = torch.rand(b.scale[1].shape, generator=g) * 165 - 75
    b.scale[1] = torch.exp2(size)
    b.scale[1][torch.rand(size.shape, generator=g) < 0.1] = 0
    b.scale[0] *= 8  # scores of some tens
    check(b, q.to(BF16))


def test_what_is_written_may_be_as_large_as_its_type():
    """Keys and values of a bfloat16's largest, written, read and attended."""
    b = Batch([(5, 200), (200, 200)], 2, 128, 16, seed=111)
    top = torch.finfo(BF16).max
    (v, vc), (k, kc) = packed(b.rows, [2, 2], 128, F32, 112)
    v = (v.clamp(-3, 3) / 3 * top).to(BF16)
    k = k.to(BF16)
    where = b.cuda()
    R.kv_write(k.cuda(), v.cuda(), *where)
    got = R.kv_read(*where, b.rows, F32)[1].cpu()
    # half a step, and three roundings to 32 bits: the scale, the quotient, the product
    most = v.to(D).abs().amax(2, keepdim=True)
    assert ((got.to(D) - v.to(D)).abs() <= most * (1 / 254 + 4 * E)).all()
    b.q8 = [t.cpu() for t in where[0][:2]]
    b.scale = [t.cpu() for t in where[0][2:]]
    q = torch.randn((b.rows, 4, 128), generator=gen(113)).to(BF16)
    out, lse = R.kv_attention(q.cuda(), *where)
    o, z, bo, bl = attend64(b, q, None, 128 ** -0.5)
    within(lse, z, bl)
    within(out, o, bo)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("name", list(CALLS))
def test_unseen_scales_of_every_size_beside_small_ones(name):
    """Rows that see values of 2^-70 alone keep them, whatever lies in their tiles."""
    b, q = call(name, 114)
    b.scale[1] *= 2.0 ** -64
    used = set()
    at_places(b, lambda i, t, pg, at: used.add((pg, at)))
    for pg in range(b.pages):
        for at in range(b.page):
            if (pg, at) not in used:
                b.scale[1][pg, :, at] = [2.0 ** 120, 2.0 ** 60, 0.0, math.inf][(pg + at) % 4]
                b.scale[0][pg, :, at] = [2.0 ** 120, 0.0, 2.0 ** -120][(pg + 2 * at) % 3]
    check(b, q.to(BF16))


@pytest.mark.parametrize("small", range(4))
@pytest.mark.parametrize("heads,dim", [(2, 64), (20, 64), (4, 128), (3, 256)])
def test_thirty_two_positions_of_small_values_among_large_ones(heads, dim, small):
    """What one wave of four goes through has scales 2^148 below the others', whichever it is:
    its exponentials count in every row's sum."""
    b = Batch([(1, 128)], 1, dim, 16, seed=117)
    for t in range(128):
        pg, at = b.place(0, t)
        b.scale[1][pg, :, at] *= 2.0 ** -58 if t // 32 == small else 2.0 ** 90
    q = torch.randn((1, heads, dim), generator=gen(118)).to(BF16)
    check(b, q)


@pytest.mark.parametrize("name", list(CALLS))
def test_huge_scales_of_keys_beside_tiny_ones_of_values(name):
    """That keys' scales are past 2^100 takes nothing from values of 2^-78."""
    b, q = call(name, 119)
    b.scale[0] *= torch.where(torch.rand(b.scale[0].shape, generator=gen(120)) < 0.3, 2.0 ** 120, 1.0)
    b.scale[1] *= 2.0 ** -72
    check(b, (q * 2.0 ** -120).to(BF16))


@pytest.mark.parametrize("heads", [1, 40])
def test_words_of_few_positions_keep_their_bits(heads):
    """Thirty-two positions: one of a large scale and no weight, one that weighs almost all, and
    ones of 2^-12 of its product, which alone make some of the outputs."""
    b = Batch([(1, 32)], 1, 64, 16, seed=121)
    q = torch.ones((1, heads, 64))
    for t in range(32):
        pg, at = b.place(0, t)
        b.q8[0][pg, :, at] = 100 if t == 9 else -100 if t == 3 else 0
        b.scale[0][pg, :, at] = 10 / 800  # scores of 10, 0 and -10
        # (0.878 e^-10 2^-6 is 10.4 of f16's steps of 2^-24)
        b.scale[1][pg, :, at] = 2.0 ** 14 if t == 3 else 2.0 ** -8 if t == 9 else 0.878 * 2.0 ** -6
        b.q8[1][pg, :, at, :32] = 0 if t in (3, 9) else b.q8[1][pg, :, at, :32]
    b.scale[0][b.place(0, 3)[0], :, b.place(0, 3)[1]] *= 3
    check(b, q.to(BF16))
