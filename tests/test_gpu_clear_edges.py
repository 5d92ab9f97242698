"""Edges of the clear side on the GPU."""
import math

import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu
from test_gpu_clear import BF16, D, E, EPS, F16, F32, TINY, U, gen, int8, normal, targets, within

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


# ---------------------------------------------------------------- loss ---

@pytest.fixture
def given_back():
    """What the test took of the card's memory is free again."""
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,rows,dim,vocab", [(BF16, 8_700_001, 512, 250),
                                                  (F16, 17_000_003, 128, 100)])
def test_cross_entropy_gradients_of_millions_of_rows(given_back, dtype, rows, dim, vocab):
    """More rows than a row of h, turned, may hold with 256 (128) of them in 32-bit
    offsets; bounds as for any other sum of 32-bit terms (test_gpu_clear.check_loss).
    A row's word goes by the sign of its last column, so that this column of gw, the
    furthest one, is large against its bound."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    h = torch.empty((rows, dim), dtype=dtype, device="cuda")
    for r in range(0, rows, 1 << 20):
        h[r:r + (1 << 20)] = torch.randn(h[r:r + (1 << 20)].shape, generator=g, device="cuda")
    w = normal(4, vocab, dim, dtype, 1.0 / math.sqrt(dim)).cuda()
    t = torch.randint(0, vocab // 2, (rows,), generator=g, device="cuda") * 2 + (h[:, -1] > 0)
    t[::7] = -100
    c = torch.rand(rows, generator=g, device="cuda") / rows
    loss, lse = R.cross_entropy(h, w, t)
    gh, gw = R.cross_entropy_backward(h, w, t, lse, c)
    u, W = U[dtype], w.to(D)
    want = torch.zeros((vocab, dim), dtype=D, device="cuda")
    bound = torch.zeros_like(want)
    for r in range(0, rows, 1 << 19):
        rs = slice(r, r + (1 << 19))
        H, counts = h[rs].to(D), t[rs] >= 0
        logits = H @ W.t().contiguous()
        lse64 = torch.logsumexp(logits, 1)
        delta = 4 * E * math.sqrt(dim) * H.norm(dim=1) * W.norm(dim=1).max() \
            + 64 * E * (1 + lse64.abs() + logits.abs().amax(1))
        within(lse[rs], lse64, delta)
        p = torch.exp(logits - lse64[:, None])
        f = torch.where(counts, c[rs].to(D), 0.0)[:, None]
        gl = p.clone()
        gl.scatter_add_(1, t[rs].clamp(min=0)[:, None], torch.full_like(f, -1.0))
        gl, p = gl * f, p * f
        off = u * gl.abs() + p * 2 * delta[:, None] + float(c.max()) * 2.0 ** -39
        want_h = gl @ W
        within(gh[rs], want_h, u * want_h.abs() + (off + 64 * E * gl.abs()) @ W.abs() + TINY[dtype])
        want += gl.t().contiguous() @ H
        bound += (off + 64 * E * gl.abs()).t().contiguous() @ H.abs()
    bound += u * want.abs() + TINY[dtype]
    assert (want[:, -1].abs() > 10 * bound[:, -1]).all()
    within(gw, want, bound)


def loss_case(dtype, rows, dim, vocab, mean=0.0):
    """Hidden states, head, targets among the first eighth of the words; `mean`: that of
    the other words' weights."""
    h = normal(10, rows, dim, dtype)
    w = normal(11, vocab, dim, D, 1.0 / math.sqrt(dim))
    t = targets(12, rows, max(1, vocab // 8), rows // 9)
    w[vocab // 8:] += mean
    return h, w.to(dtype), t


def check_gh_by_row(dtype, h, w, t, g, judged):
    """gh of the rows `judged`, each against its own factor: f16 holds gl in half steps of
    2^-38 of the row's factor, or of 2^-63 of the largest where that is more (bf16 in
    relative ones)."""
    td, gd = t.cuda(), g.cuda()
    _, lse = R.cross_entropy(h.cuda(), w.cuda(), td)
    gh, gw = R.cross_entropy_backward(h.cuda(), w.cuda(), td, lse, gd)
    H, W, G = h.cuda().to(D)[judged], w.cuda().to(D), gd.to(D)
    t, valid = td[judged], (td >= 0)[judged]
    logits = H @ W.t().contiguous()
    lse = torch.logsumexp(logits, 1)
    delta = 4 * E * math.sqrt(h.shape[1]) * H.norm(dim=1) * W.norm(dim=1).max() \
        + 64 * E * (1 + lse.abs() + logits.abs().amax(1))
    p = torch.exp(logits - lse[:, None])
    f = torch.where(valid, G[judged], 0.0)[:, None]
    gl = p.clone()
    gl.scatter_add_(1, t.clamp(min=0)[:, None], torch.full_like(f, -1.0))
    gl, p, u = gl * f, p * f.abs(), U[dtype]
    top = G[torch.isfinite(G) & (td >= 0)].abs().max()
    off = u * gl.abs() + p * 2 * delta[:, None]
    if dtype == F16:
        off += torch.maximum(f.abs() * 2.0 ** -38, top * 2.0 ** -63)
    want = gl @ W
    within(gh[judged], want,
           u * want.abs() + (off + 64 * E * gl.abs()) @ W.abs() + TINY[dtype] + 2.0 ** -140)
    return gh, gw, want


def gw64(dtype, h, w, t, g):
    """gw in 64 bits and its bound: gl rounded once on its row's scale and, in f16, once
    more in half steps of 2^-39 of the largest factor."""
    H, W, t, f = h.cuda().to(D), w.cuda().to(D), t.cuda(), g.cuda().to(D)
    want = torch.zeros_like(W)
    bound = torch.zeros_like(W)
    f = torch.where(t >= 0, f, 0.0)
    for r in range(0, len(t), 4096):
        X, c = H[r:r + 4096], f[r:r + 4096, None]
        logits = X @ W.t().contiguous()
        lse = torch.logsumexp(logits, 1)
        delta = 4 * E * math.sqrt(h.shape[1]) * X.norm(dim=1) * W.norm(dim=1).max() \
            + 64 * E * (1 + lse.abs() + logits.abs().amax(1))
        p = torch.exp(logits - lse[:, None])
        gl = p.clone()
        gl.scatter_add_(1, t[r:r + 4096].clamp(min=0)[:, None], torch.full_like(c, -1.0))
        gl, p = gl * c, p * c.abs()
        off = (U[dtype] + 64 * E) * gl.abs() + p * 2 * delta[:, None]
        if dtype == F16:
            off += c.abs() * 2.0 ** -38 + f.abs().max() * 2.0 ** -39
        want += gl.t().contiguous() @ X
        bound += off.t().contiguous() @ X.abs()
    return want, bound + U[dtype] * want.abs() + TINY[dtype]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,dim,vocab", [(20, 64, 300), (9, 1024, 2000), (500, 256, 4000),
                                            (4000, 640, 8100)])
@pytest.mark.parametrize("fill", [float("inf"), float("-inf"), float("nan")])
def test_cross_entropy_factor_of_infinity_stays_in_its_row(dtype, rows, dim, vocab, fill):
    """A factor that is not finite: its row's gh and gw are not, the other rows' are what
    they are without it."""
    h, w, t = loss_case(dtype, rows, dim, vocab)
    g = 0.5 + torch.rand(rows, generator=gen(13))
    t[3] = 1
    g[3] = fill
    judged = torch.arange(rows, device="cuda") != 3
    gh, gw, _ = check_gh_by_row(dtype, h, w, t, g, judged)
    assert not torch.isfinite(gh[3]).any() and not torch.isfinite(gw).any()
    # ignored, it has no part in anything
    t[3] = -100
    gh, gw, _ = check_gh_by_row(dtype, h, w, t, g, judged)
    assert not gh[3].any() and torch.isfinite(gw).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,dim,vocab", [(20, 64, 300), (9, 1024, 2000), (500, 256, 4000),
                                            (4000, 640, 8100), (4000, 641, 8100), (12000, 64, 50000)])
def test_cross_entropy_of_rows_that_weigh_little(dtype, rows, dim, vocab):
    """Row factors from 1 down to 2^-30 of the largest: gh row by row against its own
    factor, and its softmax part there; gw against all of them."""
    h, w, t = loss_case(dtype, rows, dim, vocab, mean=2.0)
    g = 2.0 ** 10 * 2.0 ** -torch.randint(0, 31, (rows,), generator=gen(14)).float()
    g *= 1 - 0.49 * torch.rand(rows, generator=gen(15))
    g[0] = 2.0 ** 10
    # row 1 weighs 2^-24 of row 0, and its softmax is on the words of mean 2
    g[1], t[1], h[1] = -(2.0 ** -14), 0, h[1].abs() * 4 / dim
    gh, gw, want = check_gh_by_row(dtype, h, w, t, g, slice(None))
    assert float(want[1].mean()) * -(2.0 ** 14) > 1
    want_w, bound = gw64(dtype, h, w, t, g)
    within(gw, want_w, bound)
    # gradients alone, bit for bit
    args = h.cuda(), w.cuda(), t.cuda(), R.cross_entropy(h.cuda(), w.cuda(), t.cuda())[1], g.cuda()
    assert torch.equal(R.cross_entropy_backward(*args, want_gw=False)[0], gh)
    assert torch.equal(R.cross_entropy_backward(*args, want_gh=False)[1], gw)


@pytest.mark.parametrize("rows,dim,vocab", [(8, 512, 3000), (24, 1024, 3000), (20, 64, 300),
                                            (130, 100, 20000), (4000, 640, 8100)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_cross_entropy_of_infinite_logits(dtype, rows, dim, vocab):
    """Logits of either infinity give what log, exp and sum of them give in 64 bits: lse is
    infinite where the largest logit is, and rows of finite logits are as they were."""
    h, w = normal(20, rows, dim, dtype), normal(21, vocab, dim, dtype, 0.3)
    t = targets(22, rows, vocab)
    inf = float("inf")
    big = 2.0 ** 100 if dtype == BF16 else inf
    w[:, 0] = 2.0 ** 100 if dtype == BF16 else 1  # (their product leaves 32 bits)
    w[vocab // 2:, 0] *= -1
    h[:, 0] = 0
    h[1:5, 0] = torch.tensor([big, big, -big, -big]).to(dtype)
    t[1:5] = torch.tensor([0, vocab - 1, 0, vocab - 1])
    loss, lse = R.cross_entropy(h.cuda(), w.cuda(), t.cuda())
    assert (lse[1:5] == inf).all()
    assert torch.isnan(loss[[1, 4]]).all() and (loss[[2, 3]] == inf).all()
    rest = torch.tensor([r for r in range(rows) if not 1 <= r < 5])
    same = R.cross_entropy(h[:, 1:].cuda(), w[:, 1:].cuda(), t.cuda())
    assert torch.allclose(lse[rest], same[1][rest], rtol=1e-5) and torch.isfinite(loss[rest]).all()
    # words left out by a logit of -infinity, and rows of nothing else
    w[:, 0] = w[:, 0].abs()
    if dtype == BF16:  # (0 times infinity is NaN)
        w[vocab // 3:, 0] = 0
    loss, lse = R.cross_entropy(h.cuda(), w.cuda(), t.cuda())
    if dtype == BF16:
        kept = R.cross_entropy(h[:, 1:].cuda(), w[vocab // 3:, 1:].cuda(), torch.zeros_like(t).cuda())
        assert torch.allclose(lse[3:5], kept[1][3:5], rtol=1e-5)
        assert loss[3] == inf and torch.isfinite(loss[4])
        assert (lse[1:3] == inf).all() and torch.isnan(loss[1]) and loss[2] == inf
    else:
        assert (lse[3:5] == -inf).all() and torch.isnan(loss[3:5]).all()


# ------------------------------------------------- shared buffers and workspaces ---

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(2, 64), (7, 600), (300, 1031), (5, 17000)])
def test_outputs_beside_inputs_in_one_buffer(dtype, rows, dim):
    """Columns of one buffer: rows that lie between each other's do not overlap."""
    buf = normal(30, rows, 5 * dim + 3, dtype).cuda()
    x, r, h, y, g = (buf[:, i * dim:(i + 1) * dim] for i in range(5))
    w = normal(31, 1, dim, dtype)[0].cuda()
    want = R.rms_norm(x.clone(), w, EPS, residual=r.clone())
    R.rms_norm(x, w, EPS, residual=r, h=h, y=y)
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
    back = R.rms_norm_backward(y.clone(), h.clone(), w, want[2])
    gx, gw = R.rms_norm_backward(y, h, w, want[2], gx=g)
    assert torch.equal(g, back[0]) and torch.equal(gw, back[1])
    a, sa = R.quantize_rows(x)
    product = R.q8_matmul(a, sa, a, sa, out_dtype=dtype)
    both = torch.empty((rows, 2 * max(rows, dim)), dtype=torch.int8, device="cuda")
    both[:, :dim] = a
    q, s = R.quantize_rows(x, q=both[:, dim:2 * dim])
    assert torch.equal(q, a) and torch.equal(both[:, :dim], a) and torch.equal(s, sa)
    assert torch.equal(R.q8_matmul(both[:, :dim], sa, both[:, dim:2 * dim], sa, out_dtype=dtype),
                       product)
    with pytest.raises(R.RosettaError) as e:  # one column of x's
        R.rms_norm(x, w, EPS, y=buf[:, dim - 1:2 * dim - 1])
    assert e.value.status == 4


@pytest.mark.parametrize("rows,dim,vocab", [(40, 64, 300), (300, 256, 1000)])
def test_gradients_beside_their_inputs(rows, dim, vocab):
    hb, wb = normal(32, rows, 2 * dim, BF16).cuda(), normal(33, vocab, 2 * dim, BF16, 0.1).cuda()
    t, g = targets(34, rows, vocab, 3).cuda(), torch.rand(rows, generator=gen(35)).cuda()
    h, w = hb[:, :dim], wb[:, :dim]
    lse = R.cross_entropy(h, w, t)[1]
    want = R.cross_entropy_backward(h.clone(), w.clone(), t, lse, g)
    got = R.cross_entropy_backward(h, w, t, lse, g, gh=hb[:, dim:], gw=wb[:, dim:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim", [(700, 64), (3000, 63), (900, 128), (1000, 129), (50, 250), (33, 768),
                                      (600, 1021), (1100, 2048), (515, 4099), (1100, 4096), (540, 8191),
                                      (20, 16384), (30, 16381), (515, 16390), (3, 40000)])
def test_norm_gradient_in_gh_and_in_gy(dtype, rows, dim):
    """gx at the address of gh or gy, every length class: the bits of a gx of its own."""
    h, gy, gh = (normal(40 + i, rows, dim, dtype, s).cuda() for i, s in ((0, 2.0), (1, 0.5), (2, 0.25)))
    w = normal(43, 1, dim, dtype)[0].cuda()
    inv = 0.5 + torch.rand(rows, generator=gen(44)).cuda()
    want, want_w = R.rms_norm_backward(gy, h, w, inv, gh=gh)
    for which in (0, 1):
        a, b = gy.clone(), gh.clone()
        gx, gw = R.rms_norm_backward(a, h, w, inv, gh=b, gx=(a, b)[which])
        assert gx.data_ptr() == (a, b)[which].data_ptr()
        assert torch.equal(gx, want) and torch.equal(gw, want_w)
        assert torch.equal((b, a)[which], (gh, gy)[which])


@pytest.mark.parametrize("m,n,k", [(33, 4096, 14336), (17, 200, 9000), (100, 300, 20001),
                                   (128, 512, 8192), (700, 1111, 9008)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_q8_matmul_without_a_workspace(m, n, k, dtype):
    """Sums that a workspace would split, whole: the same bits."""
    L = R.lib()
    assert L.rosetta_q8_matmul_workspace_bytes(m, n, k) > 0
    a, b = int8(50, m, k).cuda(), int8(51, n, k).cuda()
    sa, sb = torch.rand(m, generator=gen(52)).cuda(), torch.rand(n, generator=gen(53)).cuda()
    bias = torch.randn(n, generator=gen(54)).cuda()
    want = R.q8_matmul(a, sa, b, sb, bias=bias, out_dtype=dtype)
    got = torch.full_like(want, float("nan"))
    st = L.rosetta_q8_matmul(a.data_ptr(), k, sa.data_ptr(), b.data_ptr(), k, sb.data_ptr(),
                             bias.data_ptr(), got.data_ptr(), n, {F32: 0, BF16: 1}[dtype], m, n, k,
                             None, 0, torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(got, want)


@pytest.mark.parametrize("dtype,size", [(F32, 1e20), (BF16, 1e20), (F32, 3e38), (BF16, 3e38)])
@pytest.mark.parametrize("dim", [1, 33, 1024, 4096, 17000])
def test_norm_whose_squares_overflow(dtype, size, dim):
    """Such a row says so in its scale; the others do not notice."""
    x = normal(60, 3, dim, dtype)
    x[1] = size
    want = R.rms_norm_q8(x[[0, 2]].cuda(), None, EPS)
    got = R.rms_norm_q8(x.cuda(), None, EPS)
    assert not torch.isfinite(got.scale[1])
    assert torch.equal(got.scale[[0, 2]], want.scale) and torch.equal(got.q[[0, 2]], want.q)
