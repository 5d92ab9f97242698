"""The clear side (norm to 8 bits, 8-bit product, vocabulary loss) on the GPU
against its formulas in 64 bits on the host.

Bounds come from the arithmetic: U[T] is half a unit in the last place of an
output's type, E that of the 32-bit sums; a sum of positive terms taken in
chains of c is off by at most c E of itself, a dot product by about sqrt(n) E of
the product of its norms (taken four times over here)."""
import math

import pytest

from paper_2609_16915_amd import rosetta as R

from gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

E = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {t: torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}  # half a step of the smallest values
D = torch.float64
EPS = 1e-5


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(seed, rows, cols, dtype, scale=1.0):
    return (torch.randn((rows, cols), generator=gen(seed)) * scale).to(dtype)


def placed(t, pad=0, offset=0):
    """The same matrix on the GPU, rows `pad` elements further apart and the first
    `offset` elements into its buffer; what surrounds it is NaN or 99."""
    rows, cols = t.shape
    fill = float("nan") if t.is_floating_point() else 99
    buf = torch.full((offset + rows * (cols + pad),), fill, dtype=t.dtype, device="cuda")
    m = buf[offset:].view(rows, cols + pad)[:, :cols]
    m.copy_(t)
    return m


def within(got, want, bound):
    d = (got.detach().to(want.device, D) - want).abs()
    worst = float((d - bound).max()) if d.numel() else 0.0
    assert not torch.isnan(d).any() and worst <= 0, \
        f"off by {worst:.3g} more than the bound (largest difference {float(d.max()):.3g})"


# ---------------------------------------------------------------- norm ---

def norm64(x, r, w, eps):
    h = x.to(D) + (r.to(D) if r is not None else 0)
    inv = 1 / torch.sqrt((h * h).mean(1) + eps)
    y = h * inv[:, None] * (w.to(D) if w is not None else 1)
    return h, inv, y


def chain(dim):
    """Longest chain of 32-bit additions over a row."""
    return dim / 1024 + 64


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim,pad,offset", [
    (1, 1, 0, 0), (3, 7, 0, 0), (5, 64, 8, 0), (4, 511, 1, 1), (9, 512, 0, 0), (2, 513, 3, 2),
    (7, 2047, 9, 0), (3, 2048, 0, 0), (3, 2049, 0, 1), (5, 4096, 0, 0), (2, 4104, 0, 0),
    (2, 8191, 5, 3), (2, 8200, 0, 0), (3, 14336, 0, 0), (2, 16384, 0, 0), (2, 16385, 0, 1),
    (2, 40000, 8, 0), (301, 768, 0, 0)])
def test_norm(dtype, rows, dim, pad, offset):
    x, r = normal(1, rows, dim, dtype), normal(2, rows, dim, dtype, 2.0)
    w = (1 + 0.3 * torch.randn(dim, generator=gen(3))).to(dtype)
    h, inv, y = norm64(x, r, w, EPS)
    o = R.rms_norm_q8(placed(x, pad, offset), w.cuda(), EPS, residual=placed(r, pad, offset),
                      want_y=True, q=placed(torch.zeros(rows, dim, dtype=torch.int8), pad, offset))
    assert torch.equal(o.h.cpu(), (x.float() + r.float()).to(dtype))
    e = chain(dim) * E
    within(o.inv_rms, inv, e * inv)
    scale = y.abs().amax(1) / 127
    within(o.scale, scale, 2 * e * scale)
    within(o.y, y, (U[dtype] + 2 * e) * y.abs() + TINY[dtype])
    steps = y / scale[:, None]
    within(o.q, steps, torch.full_like(steps, 0.5 + 127 * 8 * E))
    assert o.q.abs().max() == 127  # the largest value of a row is a whole 127
    values = R.dequantize_rows(o.q, o.scale, dtype)
    within(values, o.q.cpu().to(D) * o.scale.cpu().to(D)[:, None],
           (U[dtype] + 2 * E) * values.cpu().to(D).abs() + TINY[dtype])
    y2, h2, inv2 = R.rms_norm(placed(x, pad, offset), w.cuda(), EPS,
                              residual=placed(r, pad, offset))
    assert torch.equal(y2, o.y) and torch.equal(h2, o.h) and torch.equal(inv2, o.inv_rms)


@pytest.mark.parametrize("dim", [100, 4096, 20000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_variants(dtype, dim):
    rows = 6
    x, r = normal(4, rows, dim, dtype), normal(5, rows, dim, dtype)
    w = 1 + 0.3 * torch.randn(dim, generator=gen(6))
    # no weight, no residual
    o = R.rms_norm_q8(x.cuda(), None, EPS, want_y=True)
    _, inv, y = norm64(x, None, None, EPS)
    assert o.h is None
    within(o.inv_rms, inv, chain(dim) * E * inv)
    within(o.y, y, (U[dtype] + 2 * chain(dim) * E) * y.abs())
    # a 32-bit weight
    o = R.rms_norm_q8(x.cuda(), w.cuda(), EPS, residual=r.cuda(), want_y=True)
    _, _, y = norm64(x, r, w, EPS)
    within(o.y, y, (U[dtype] + 2 * chain(dim) * E) * y.abs())
    # h in the residual's place, and in x's
    for which in (0, 1):
        xs, rs = x.cuda(), r.cuda()
        p = R.rms_norm_q8(xs, w.cuda(), EPS, residual=rs, h=(xs, rs)[which])
        assert p.h.data_ptr() == (xs, rs)[which].data_ptr()
        assert torch.equal(p.h, o.h) and torch.equal(p.q, o.q) and torch.equal(p.scale, o.scale)


@pytest.mark.parametrize("dim", [33, 3000, 17000])
def test_norm_edge_rows(dim):
    x = normal(7, 8, dim, F32)
    x[0] = 0
    x[1] = 1e-30
    x[2, dim // 2] = float("nan")
    x[3, dim - 1] = float("inf")
    x[4] *= 1e-18
    x[5] = 0
    x[5, 0] = -3
    x[6] *= 1e15
    for norm in (True, False):
        if norm:
            o = R.rms_norm_q8(x.cuda(), None, EPS)
            q, scale = o.q, o.scale
        else:
            q, scale = R.quantize_rows(x.cuda())
        q, scale = q.cpu(), scale.cpu()
        y = norm64(x, None, None, EPS)[2] if norm else x.to(D)
        assert scale[0] == 0 and not q[0].any()
        assert not math.isfinite(scale[2]) and not math.isfinite(scale[3])
        for row in (1, 4, 5, 6, 7):
            want = y[row].abs().max() / 127
            assert abs(float(scale[row]) - want) <= 2 * chain(dim) * E * want, row
            steps = y[row] / want
            assert ((q[row].to(D) - steps).abs() <= 0.5 + 127 * 8 * E).all(), row
    # eps = 0 on a row of zeros: 0 * inf
    o = R.rms_norm_q8(torch.zeros(1, dim, device="cuda"), None, 0.0)
    assert math.isnan(float(o.scale[0])) or float(o.scale[0]) == 0


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim", [(1, 1), (5, 96), (40, 2048), (3, 5000), (600, 130),
                                      (2, 16385)])
def test_quantize_rows(dtype, rows, dim):
    x = normal(8, rows, dim, dtype, 3.0)
    q, scale = R.quantize_rows(placed(x, 3, 1))
    want = x.to(D).abs().amax(1) / 127
    within(scale, want, 2 * E * want)
    steps = x.to(D) / want[:, None]
    within(q, steps, torch.full_like(steps, 0.5 + 127 * 8 * E))


def norm_back64(gy, gh, h, inv, w):
    inv = inv[:, None]
    g = gy * w
    gx = gh + g * inv - h * inv ** 3 * (g * h).mean(1, keepdim=True)
    return gx, (gy * h * inv).sum(0)


def test_norm_gradient_formula_against_differences():
    rows, dim = 3, 11
    x, w = normal(9, rows, dim, D), 1 + normal(10, 1, dim, D)[0]
    a, b = normal(11, rows, dim, D), normal(12, rows, dim, D)
    f = lambda x, w: float((norm64(x, None, w, EPS)[2] * a + x * b).sum())  # noqa: E731
    gx, gw = norm_back64(a, b, x, norm64(x, None, w, EPS)[1], w)
    d = 1e-5
    for t, g in ((x, gx), (w, gw)):
        for at in range(t.numel()):
            old = float(t.view(-1)[at])
            t.view(-1)[at] = old + d
            up = f(x, w)
            t.view(-1)[at] = old - d
            down = f(x, w)
            t.view(-1)[at] = old
            assert abs((up - down) / (2 * d) - float(g.reshape(-1)[at])) < 1e-7


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim,pad,offset", [
    (1, 1, 0, 0), (2, 9, 0, 0), (700, 64, 0, 0), (5, 512, 1, 1), (33, 768, 8, 0), (3, 2048, 0, 0),
    (4, 2049, 0, 0), (1100, 4096, 0, 0), (2, 8000, 3, 5), (2, 16384, 0, 0), (515, 16390, 0, 0)])
def test_norm_backward(dtype, rows, dim, pad, offset):
    h, gy, gh = (normal(20 + i, rows, dim, dtype, s) for i, s in ((0, 2.0), (1, 0.5), (2, 0.25)))
    w = (1 + 0.3 * torch.randn(dim, generator=gen(23))).to(dtype)
    inv = norm64(h, None, None, EPS)[1].float()
    args = placed(gy, pad, offset), placed(h, pad, offset), w.cuda(), inv.cuda()
    gx, gw = R.rms_norm_backward(*args, gh=placed(gh, pad, offset))
    H, GY, GH, W, I = (t.to(D) for t in (h, gy, gh, w, inv))
    want, want_w = norm_back64(GY, GH, H, I, W)
    e = chain(dim) * E
    I = I[:, None]
    size = GH.abs() + (GY * W * I).abs() + H.abs() * I ** 3 * (GY * W * H).abs().mean(1, keepdim=True)
    within(gx, want, U[dtype] * want.abs() + 2 * e * size + TINY[dtype])
    within(gw, want_w, (rows / 512 + 64) * E * (GY * H * I).abs().sum(0))
    # without gh, without the weight's gradient, in place of gy
    gx0, none = R.rms_norm_backward(*args, want_gweight=False)
    assert none is None
    zero, _ = R.rms_norm_backward(*args, gh=torch.zeros(rows, dim, dtype=dtype, device="cuda"))
    assert torch.equal(gx0, zero)
    again, gw2 = R.rms_norm_backward(*args, gx=args[0])
    assert again.data_ptr() == args[0].data_ptr() and torch.equal(again, gx0)
    assert torch.equal(gw, gw2)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim,pad,offset", [
    (1, 3, 0, 0), (5, 8, 0, 0), (67, 15, 2, 1), (3000, 63, 1, 0), (20000, 64, 8, 0), (31, 65, 0, 0),
    (900, 128, 0, 0), (1000, 129, 0, 1), (50, 250, 0, 0), (4100, 256, 8, 0), (600, 257, 0, 0),
    (1030, 1000, 0, 0), (1029, 1021, 3, 1), (300, 1025, 0, 0), (60, 9001, 0, 0)])
def test_norm_of_short_and_ragged_rows(dtype, rows, dim, pad, offset):
    """Rows side by side in a workgroup, and rows that end at any place of a vector:
    both directions."""
    x, r, gy = (normal(24 + i, rows, dim, dtype, s) for i, s in ((0, 1.0), (1, 2.0), (2, 0.5)))
    w = (1 + 0.3 * torch.randn(dim, generator=gen(27))).to(dtype)
    y, h, inv = R.rms_norm(placed(x, pad, offset), w.cuda(), EPS, residual=placed(r, pad, offset))
    want_h, want_inv, want_y = norm64(x, r, w, EPS)
    e = chain(dim) * E
    within(inv, want_inv, e * want_inv)
    within(h, want_h, U[dtype] * want_h.abs() + TINY[dtype])
    within(y, want_y, (U[dtype] + 2 * e) * want_y.abs() + TINY[dtype])
    gx, gw = R.rms_norm_backward(placed(gy, pad, offset), placed(h.cpu(), pad, offset), w.cuda(), inv,
                                 gh=placed(r, pad, offset))
    H, GY, GH, W, I = (t.cpu().to(D) for t in (h, gy, r, w, inv))
    want, want_w = norm_back64(GY, GH, H, I, W)
    I = I[:, None]
    size = GH.abs() + (GY * W * I).abs() + H.abs() * I ** 3 * (GY * W * H).abs().mean(1, keepdim=True)
    within(gx, want, U[dtype] * want.abs() + 2 * e * size + TINY[dtype])
    # at most rows / 512 terms to a thread, 32 rows side by side, 512 groups by 16
    within(gw, want_w, (rows / 512 + 96) * E * (GY * H * I).abs().sum(0))


# ------------------------------------------------------------- product ---

def int8(seed, rows, cols):
    return torch.randint(-128, 128, (rows, cols), generator=gen(seed), dtype=torch.int8)


@pytest.mark.parametrize("m,n,k,pad,offset", [
    (1, 1, 1, 0, 0), (1, 16, 64, 0, 0), (1, 300, 4096, 0, 0), (2, 33, 127, 0, 0),
    (5, 17, 1000, 8, 0), (16, 128, 128, 0, 0), (17, 129, 144, 16, 16), (33, 500, 2048, 0, 0),
    (64, 70, 96, 3, 1), (65, 257, 4097, 0, 0), (100, 64, 16, 0, 0), (127, 1000, 640, 0, 0),
    (128, 256, 512, 0, 0), (129, 130, 1111, 1, 7), (300, 700, 320, 0, 0), (257, 259, 2064, 0, 0),
    (520, 1030, 200, 0, 0), (1000, 513, 768, 0, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_q8_matmul(m, n, k, pad, offset, dtype):
    a, b = int8(30, m, k), int8(31, n, k)
    sa = 0.01 + 0.02 * torch.rand(m, generator=gen(32))
    sb = 1e-3 + 4e-3 * torch.rand(n, generator=gen(33))
    bias = torch.randn(n, generator=gen(34))
    out = placed(torch.zeros(m, n, dtype=dtype), pad, offset)
    got = R.q8_matmul(placed(a, pad, offset), sa.cuda(), placed(b, pad, offset), sb.cuda(),
                      bias=bias.cuda(), out=out)
    prod = (a.to(D) @ b.to(D).t()) * sa.to(D)[:, None] * sb.to(D)
    want = prod + bias.to(D)
    within(got, want, U[dtype] * want.abs() + 4 * E * (prod.abs() + want.abs()) + TINY[dtype])
    plain = R.q8_matmul(a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), out_dtype=dtype)
    within(plain, prod, (U[dtype] + 4 * E) * prod.abs() + TINY[dtype])
    if pad:  # nothing beside the rows is written
        beside = torch.as_strided(out, (m - 1, pad), (n + pad, 1), out.storage_offset() + n)
        assert torch.isnan(beside).all()


@pytest.mark.parametrize("m,n,k,pad", [(4090, 4095, 300, 0), (4090, 4095, 304, 16),
                                       (3968, 4096, 512, 0), (2049, 2047, 4112, 0),
                                       (700, 1111, 9008, 16), (100, 300, 20001, 0)])
def test_q8_matmul_large(m, n, k, pad):
    """Enough outputs for the large tiles, and few enough that small ones have a CU
    each; products taken in 64 bits on the GPU."""
    a, b = int8(35, m, k), int8(36, n, k)
    sa, sb = 0.01 + torch.rand(m, generator=gen(37)), 0.01 + torch.rand(n, generator=gen(38))
    got = R.q8_matmul(placed(a, pad), sa.cuda(), placed(b, pad), sb.cuda(), out_dtype=F32)
    prod = a.cuda().to(D) @ b.cuda().to(D).t().contiguous()
    want = prod * sa.cuda().to(D)[:, None] * sb.cuda().to(D)
    within(got, want, 4 * E * want.abs())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,n,k,pad", [(4090, 4095, 304, 16), (3968, 4096, 512, 0)])
def test_q8_matmul_large_in_16_bits(m, n, k, pad, dtype):
    a, b = int8(39, m, k), int8(40, n, k)
    sa, sb = 0.01 + torch.rand(m, generator=gen(41)), 1e-4 + 1e-4 * torch.rand(n, generator=gen(42))
    got = R.q8_matmul(placed(a, pad), sa.cuda(), placed(b, pad), sb.cuda(), out_dtype=dtype)
    prod = a.cuda().to(D) @ b.cuda().to(D).t().contiguous()
    want = prod * sa.cuda().to(D)[:, None] * sb.cuda().to(D)
    within(got, want, (U[dtype] + 4 * E) * want.abs() + TINY[dtype])


@pytest.mark.parametrize("m", [1, 40, 200])
def test_q8_matmul_largest_sums(m):
    k = 131071
    a = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    b = torch.full((130, k), -128, dtype=torch.int8, device="cuda")
    b[1] = 127
    one = torch.ones(130, device="cuda")
    got = R.q8_matmul(a, one[:1].expand(m).contiguous(), b, one, out_dtype=F32).cpu()
    want = torch.full((m, 130), 128.0 * 128 * k)
    want[:, 1] = -128.0 * 127 * k
    assert torch.equal(got, want.float())


def test_q8_matmul_without_terms_and_with_a_nan_scale():
    none = torch.empty((3, 0), dtype=torch.int8, device="cuda")
    bias = torch.arange(5, dtype=F32, device="cuda")
    got = R.q8_matmul(none, torch.ones(3, device="cuda"), none.new_empty((5, 0)),
                      torch.ones(5, device="cuda"), bias=bias, out_dtype=F32)
    assert torch.equal(got, bias.expand(3, 5))
    a, b = int8(40, 20, 64), int8(41, 50, 64)
    sa = torch.ones(20)
    sa[3] = float("nan")
    got = R.q8_matmul(a.cuda(), sa.cuda(), b.cuda(), torch.ones(50).cuda(), out_dtype=F32).cpu()
    assert torch.isnan(got[3]).all() and torch.isfinite(got[[0, 1, 2, 4, 19]]).all()


# ---------------------------------------------------------------- loss ---

def loss64(h, w, t, ignore):
    logits = h.to(D) @ w.to(D).t()
    lse = torch.logsumexp(logits, 1)
    v = w.shape[0]
    valid = (t != ignore) & (t >= 0) & (t < v)
    at = torch.where(valid, t, torch.zeros_like(t))
    loss = lse - logits.gather(1, at[:, None])[:, 0]
    loss = torch.where(valid, loss, torch.where(t == ignore, 0.0, float("nan")).to(D))
    return logits, lse, loss, valid, at


def check_loss(h, w, t, g, ignore, dtype, pad=0, offset=0, dev="cpu"):
    """`dev`: where the 64-bit products are taken."""
    rows, dim = h.shape
    hd, wd, td, gd = placed(h, pad, offset), placed(w, pad, offset), t.cuda(), g.cuda()
    h, w, t, g = (x.to(dev) for x in (h, w, t, g))
    logits, lse, loss, valid, at = loss64(h, w, t, ignore)
    got, got_lse = R.cross_entropy(hd, wd, td, ignore)
    # a logit's error, and with it a log-sum's; exp and log add units of E
    delta = 4 * E * math.sqrt(dim) * h.to(D).norm(dim=1) * w.to(D).norm(dim=1).max() \
        + 64 * E * (1 + lse.abs() + logits.abs().amax(1))
    within(got_lse, lse, delta)
    got = got.to(dev)
    assert torch.equal(torch.isnan(got), torch.isnan(loss))
    fine = ~torch.isnan(loss)
    within(got[fine], loss[fine], 2 * delta[fine])
    assert not got[t == ignore].any()

    gh, gw = R.cross_entropy_backward(hd, wd, td, got_lse, gd, ignore)
    p = torch.exp(logits - lse[:, None])
    gl = p.clone()
    gl[torch.arange(rows, device=dev), at] -= 1
    c = torch.where(valid, g.to(D), torch.zeros(rows, dtype=D, device=dev))[:, None]
    gl, p = gl * c, p * c.abs()
    u = U[dtype]
    # gl is rounded once; p is off by its logit's error; f16 holds it in steps of
    # 2^-39 of the largest factor
    off = u * gl.abs() + p * 2 * delta[:, None] + c.abs().max() * 2.0 ** -39
    W, H = w.to(D).abs(), h.to(D).abs()
    want_h, want_w = gl @ w.to(D), gl.t() @ h.to(D)
    within(gh, want_h, u * want_h.abs() + off @ W + 64 * E * (gl.abs() @ W) + TINY[dtype])
    within(gw, want_w, u * want_w.abs() + off.t() @ H + 64 * E * (gl.abs().t() @ H) + TINY[dtype])
    # one of the two alone
    only_h, none = R.cross_entropy_backward(hd, wd, td, got_lse, gd, ignore, want_gw=False)
    assert none is None and torch.equal(only_h, gh)
    none, only_w = R.cross_entropy_backward(hd, wd, td, got_lse, gd, ignore, want_gh=False)
    assert none is None and torch.equal(only_w, gw)


def targets(seed, rows, vocab, masked=0, ignore=-100):
    t = torch.randint(0, vocab, (rows,), generator=gen(seed))
    t[torch.randperm(rows, generator=gen(seed + 1))[:masked]] = ignore
    return t


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,dim,vocab,pad,offset,masked", [
    (1, 1, 1, 0, 0, 0), (1, 8, 5, 0, 0, 0), (1, 512, 5000, 0, 0, 0), (3, 33, 127, 0, 0, 1),
    (8, 256, 3001, 8, 0, 0), (17, 64, 128, 8, 8, 3), (40, 72, 129, 0, 0, 40), (65, 100, 1000, 1, 3, 9),
    (128, 128, 256, 0, 0, 0), (129, 320, 777, 0, 0, 64), (300, 96, 5003, 0, 0, 30),
    (260, 513, 513, 0, 0, 0), (600, 640, 1500, 0, 0, 100)])
def test_cross_entropy(dtype, rows, dim, vocab, pad, offset, masked):
    h = normal(50, rows, dim, dtype)
    w = normal(51, vocab, dim, dtype, 2.0 / math.sqrt(dim))
    g = 1e-3 + torch.rand(rows, generator=gen(52)) / rows
    check_loss(h, w, targets(53, rows, vocab, masked), g, -100, dtype, pad, offset)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_cross_entropy_large_logits_and_uneven_factors(dtype):
    rows, dim, vocab = 70, 128, 900
    h, w = normal(60, rows, dim, dtype, 4.0), normal(61, vocab, dim, dtype, 2.0)
    g = torch.exp(4 * torch.randn(rows, generator=gen(62)))
    g[5] = 0
    g[6] = -2
    check_loss(h, w, targets(63, rows, vocab, 7, 3), g, 3, dtype)


@pytest.mark.parametrize("dtype,dim", [(BF16, 64), (F16, 192)])
def test_cross_entropy_gradients_in_pieces(dtype, dim):
    """Enough rows that gl is held for a part of the vocabulary at a time, the last
    part shorter than the others by more than a tile."""
    rows, vocab = 16384, 40000
    one = R.lib().rosetta_cross_entropy_backward_workspace_bytes(rows, dim, vocab)
    assert one < 2 * rows * vocab  # (not all of gl)
    g = torch.full((rows,), 1.0 / rows)
    check_loss(normal(64, rows, dim, dtype), normal(65, vocab, dim, dtype, 1.0 / math.sqrt(dim)),
               targets(66, rows, vocab, 1000), g, -100, dtype, dev="cuda")


@pytest.mark.parametrize("dtype,rows,dim,vocab,pad", [
    (BF16, 4000, 640, 8100, 0), (F16, 4001, 648, 8111, 8), (BF16, 4001, 649, 8111, 0)])
def test_cross_entropy_large(dtype, rows, dim, vocab, pad):
    """Enough rows and words for the large tiles."""
    g = torch.rand(rows, generator=gen(67)) / rows
    check_loss(normal(68, rows, dim, dtype), normal(69, vocab, dim, dtype, 2.0 / math.sqrt(dim)),
               targets(70, rows, vocab, 500), g, -100, dtype, pad, dev="cuda")


@pytest.mark.parametrize("dtype,rows,dim,vocab,pad", [
    (BF16, 64, 1024, 3000, 0), (F16, 100, 1032, 2500, 8), (F16, 2500, 64, 500, 0),
    (BF16, 4500, 192, 700, 0), (F16, 42, 256, 50000, 0), (BF16, 20, 520, 34000, 0),
    (BF16, 24, 1024, 3000, 0), (F16, 3, 704, 40000, 0)])
def test_cross_entropy_of_few_tiles_and_few_rows(dtype, rows, dim, vocab, pad):
    """Few enough tiles that each has a CU, sums over many rows, many parts of few
    outputs, and rows that weigh unlike each other."""
    g = torch.exp(2 * torch.randn(rows, generator=gen(76))) / rows
    check_loss(normal(77, rows, dim, dtype), normal(78, vocab, dim, dtype, 2.0 / math.sqrt(dim)),
               targets(79, rows, vocab, rows // 9), g, -100, dtype, pad, dev="cuda")


def test_cross_entropy_targets_out_of_range():
    rows, dim, vocab = 40, 64, 100
    t = targets(70, rows, vocab)
    t[0], t[1], t[2], t[3] = -1, vocab, 1 << 40, -(1 << 40)
    check_loss(normal(71, rows, dim, BF16), normal(72, vocab, dim, BF16, 0.2), t,
               torch.full((rows,), 1.0 / rows), -100, BF16)


def test_cross_entropy_nan_stays_in_its_row():
    rows, dim, vocab = 20, 64, 300
    h, w = normal(73, rows, dim, BF16), normal(74, vocab, dim, BF16, 0.2)
    h[4, 7] = float("nan")
    t = targets(75, rows, vocab)
    t[9] = -100
    loss, lse = R.cross_entropy(h.cuda(), w.cuda(), t.cuda())
    bad = torch.isnan(loss).cpu()
    assert bad[4] and bad.sum() == 1
    # an ignored row's NaN reaches nothing
    t[4] = -100
    loss, lse = R.cross_entropy(h.cuda(), w.cuda(), t.cuda())
    g = torch.full((rows,), 0.1, device="cuda")
    gh, gw = R.cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), lse, g)
    assert not loss.cpu()[4] and not gh[4].any() and torch.isfinite(gh).all()


@pytest.mark.parametrize("rows,dim,vocab", [(20, 64, 300), (500, 256, 4000)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_cross_entropy_rows_without_part_leave_no_trace(dtype, rows, dim, vocab):
    """NaN and infinities in rows whose target does not count change no bit of any
    other row's results, or of the weights' gradient."""
    h, w = normal(110, rows, dim, dtype), normal(111, vocab, dim, dtype, 0.2)
    t = targets(112, rows, vocab, rows // 3)
    t[3], t[rows - 1] = -7, vocab + 1
    out = (t < 0) | (t >= vocab)
    g = torch.rand(rows, generator=gen(113)).cuda()
    got = []
    for fill in (0.0, float("nan"), float("inf")):
        x = h.clone()
        x[out] = fill
        loss, lse = R.cross_entropy(x.cuda(), w.cuda(), t.cuda())
        gh, gw = R.cross_entropy_backward(x.cuda(), w.cuda(), t.cuda(), lse, g)
        assert not gh[out.cuda()].any()
        got.append((loss[~out.cuda()], gh, gw))
    for other in got[1:]:
        for a, b in zip(other, got[0]):
            assert torch.isfinite(a).all() and torch.equal(a, b)


def test_cross_entropy_gradient_against_differences():
    rows, dim, vocab = 6, 16, 40
    h, w = normal(76, rows, dim, F16), normal(77, vocab, dim, F16, 0.5)
    t = targets(78, rows, vocab, 1)
    g = torch.rand(rows, generator=gen(79))
    lse = R.cross_entropy(h.cuda(), w.cuda(), t.cuda())[1]
    gh, gw = R.cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), lse, g.cuda())
    H, Wt = h.to(D), w.to(D)
    f = lambda: float((loss64(H, Wt, t, -100)[2] * g.to(D)).sum())  # noqa: E731
    d = 1e-5
    for m, got in ((H, gh), (Wt, gw)):
        for at in range(0, m.numel(), 7):
            old = float(m.view(-1)[at])
            m.view(-1)[at] = old + d
            hi = f()
            m.view(-1)[at] = old - d
            lo = f()
            m.view(-1)[at] = old
            # every product has norms below 16: f16 rounding of gl and of the result
            assert abs((hi - lo) / (2 * d) - float(got.view(-1)[at])) < 16 * 2.0 ** -11


# -------------------------------------------------- streams and memory ---

def far(t, stride):
    """The same rows `stride` elements apart: a stride that takes the last row past
    what 32 bits count."""
    rows, cols = t.shape
    buf = torch.empty((rows - 1) * stride + cols, dtype=t.dtype, device="cuda")
    m = torch.as_strided(buf, (rows, cols), (stride, 1))
    m.copy_(t)
    return m


@pytest.mark.parametrize("dim", [72, 20000])
def test_norm_of_rows_far_apart(dim):
    x, r, w = normal(120, 3, dim, BF16).cuda(), normal(121, 3, dim, BF16).cuda(), None
    want = R.rms_norm_q8(x, w, EPS, residual=r)
    got = R.rms_norm_q8(far(x, (1 << 31) + 8), w, EPS, residual=r,
                        q=far(torch.zeros_like(want.q), (1 << 31) + 24))
    assert torch.equal(got.h, want.h) and torch.equal(got.q, want.q)
    assert torch.equal(R.dequantize_rows(got.q, got.scale, F32),
                       R.dequantize_rows(want.q, want.scale, F32))
    back = R.rms_norm_backward(r, want.h, w, want.inv_rms)
    over = R.rms_norm_backward(r, far(want.h, (1 << 31) + 8), w, want.inv_rms,
                               gx=far(torch.zeros_like(r), 1 << 31))
    assert torch.equal(back[0], over[0]) and torch.equal(back[1], over[1])


@pytest.mark.parametrize("m", [2, 70])
def test_products_of_rows_far_apart(m):
    a, b = int8(122, m, 1040).cuda(), int8(123, 5, 1040).cuda()
    sa, sb = torch.rand(m, device="cuda"), torch.rand(5, device="cuda")
    want = R.q8_matmul(a, sa, b, sb, out_dtype=F32)
    assert torch.equal(R.q8_matmul(a, sa, far(b, (1 << 30) + 16), sb, out_dtype=F32), want)
    h, w = normal(124, m, 520, BF16).cuda(), normal(125, 5, 520, BF16).cuda()
    t, g = targets(126, m, 5).cuda(), torch.rand(m, generator=gen(127)).cuda()
    wf = far(w, (1 << 30) + 8)
    loss, lse = R.cross_entropy(h, w, t)
    loss2, lse2 = R.cross_entropy(h, wf, t)
    assert torch.allclose(lse, lse2, rtol=0, atol=1e-5) and torch.allclose(loss, loss2, atol=1e-5)
    gh, gw = R.cross_entropy_backward(h, w, t, lse, g)
    gh2, gw2 = R.cross_entropy_backward(h, wf, t, lse, g, gw=far(torch.zeros_like(w), 1 << 30))
    assert torch.equal(gh, gh2) and torch.equal(gw, gw2)



def test_rows_of_none():
    e = torch.empty((0, 64), dtype=BF16, device="cuda")
    one = torch.ones(64, dtype=BF16, device="cuda")
    assert R.rms_norm_q8(e, one, EPS).q.shape == (0, 64)
    gx, gw = R.rms_norm_backward(e, e, one, torch.empty(0, device="cuda"))
    assert gx.shape == (0, 64) and not gw.any()
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    w = normal(80, 30, 64, BF16).cuda()
    loss, lse = R.cross_entropy(e, w, t)
    gh, gw = R.cross_entropy_backward(e, w, t, lse, loss)
    assert gh.shape == (0, 64) and not gw.any() and gw.shape == (30, 64)
    q = torch.empty((0, 32), dtype=torch.int8, device="cuda")
    assert R.q8_matmul(q, loss, torch.zeros((7, 32), dtype=torch.int8, device="cuda"),
                       torch.ones(7, device="cuda")).shape == (0, 7)


def _chain(x, r, w, wq, ws, head, t, stream=None):
    """Norm, product, norm again, loss and gradients, as a program joins them."""
    o = R.rms_norm_q8(x, w, EPS, residual=r, stream=stream)
    y = R.q8_matmul(o.q, o.scale, wq, ws, stream=stream)
    z, h, inv = R.rms_norm(y, w, EPS, residual=o.h, stream=stream)
    loss, lse = R.cross_entropy(z, head, t, stream=stream)
    gz, gw = R.cross_entropy_backward(z, head, t, lse, torch.ones_like(loss), stream=stream)
    gx, gn = R.rms_norm_backward(gz, h, w, inv, stream=stream)
    return loss, gw, gx, gn


@pytest.mark.parametrize("rows,dim,vocab", [(90, 256, 1000), (4000, 640, 8100)])
def test_another_stream_and_a_captured_graph(rows, dim, vocab):
    args = [normal(90, rows, dim, BF16), normal(91, rows, dim, BF16),
            normal(92, 1, dim, BF16)[0], int8(93, dim, dim),
            1e-3 * torch.rand(dim, generator=gen(94)),
            normal(95, vocab, dim, BF16, 0.1), targets(96, rows, vocab, 9)]
    args = [a.cuda() for a in args]
    want = [t.clone() for t in _chain(*args)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _chain(*args, stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = _chain(*args)
    for k in range(3):
        args[0].copy_(normal(100 + k, rows, dim, BF16))
        want = [t.clone() for t in _chain(*args)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
