"""The clear side's refusals: every wrong argument is an error before anything
is enqueued.  Through the C ABI with addresses that no device has, and through
the binding with CPU tensors, which stop at its device check at the latest."""
import pytest
import torch

from paper_2609_16915_amd import rosetta as R

OK, NULL, PARAMS, UNSUPPORTED, ALIAS, SIZE = 0, 1, 2, 3, 4, 7
F32, BF16, F16 = 0, 1, 2
AT = [1 << 40, 2 << 40, 3 << 40, 4 << 40, 5 << 40, 6 << 40, 7 << 40, 8 << 40]  # far apart


@pytest.fixture(scope="module")
def L():
    return R.lib()


def norm(L, x=AT[0], xs=64, r=None, rs=64, w=None, wt=BF16, t=BF16, rows=4, dim=64, eps=1e-5,
         h=AT[1], hs=64, y=None, ys=64, q=AT[2], qs=64, scale=AT[3], inv=AT[4]):
    return L.rosetta_rms_norm(x, xs, r, rs, w, wt, t, rows, dim, eps, h, hs, y, ys, q, qs, scale,
                              inv, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), OK), (dict(rows=0, x=None, h=None, q=None, scale=None, inv=None), OK),
    (dict(x=None), NULL), (dict(scale=None), NULL), (dict(q=None), NULL),
    (dict(t=3), PARAMS), (dict(t=-1), PARAMS), (dict(w=AT[5], wt=F16), PARAMS),
    (dict(dim=0), PARAMS), (dict(eps=-1.0), PARAMS), (dict(eps=float("nan")), PARAMS),
    (dict(xs=63), PARAMS), (dict(hs=63), PARAMS), (dict(qs=1), PARAMS), (dict(y=AT[5], ys=8), PARAMS),
    (dict(r=AT[5], rs=2), PARAMS), (dict(xs=(1 << 32) + 1), PARAMS),
    (dict(x=AT[0] + 1), PARAMS), (dict(scale=AT[3] + 2), PARAMS),
    (dict(dim=(1 << 24) + 1, xs=1 << 25, hs=1 << 25, qs=1 << 25), UNSUPPORTED),
    (dict(rows=1 << 31), UNSUPPORTED),
    (dict(h=AT[0] + 64), ALIAS), (dict(h=AT[0], hs=128), ALIAS), (dict(q=AT[0] + 128), ALIAS),
    (dict(y=AT[0]), ALIAS), (dict(y=AT[1]), ALIAS), (dict(inv=AT[3] + 12), ALIAS),
    (dict(r=AT[5], h=AT[5] + 2), ALIAS), (dict(w=AT[5], q=AT[5]), ALIAS),
])
def test_norm(L, kw, status):
    assert norm(L, **kw) == status
    assert bool(L.rosetta_last_error()) == (status != OK)


def back(L, gy=AT[0], gys=64, gh=None, ghs=64, h=AT[1], hs=64, w=None, wt=BF16, inv=AT[2], t=BF16,
         rows=4, dim=64, gx=AT[3], gxs=64, gw=AT[4], ws=AT[5], wsb=1 << 30):
    return L.rosetta_rms_norm_backward(gy, gys, gh, ghs, h, hs, w, wt, inv, t, rows, dim, gx, gxs,
                                       gw, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0, gw=None), OK), (dict(gy=None), NULL), (dict(h=None), NULL),
    (dict(inv=None), NULL), (dict(gx=None), NULL), (dict(ws=None), NULL),
    (dict(wsb=4 * 64 * 4 - 1), SIZE), (dict(t=7), PARAMS), (dict(gxs=63), PARAMS),
    (dict(gx=AT[1]), ALIAS), (dict(gx=AT[0] + 2), ALIAS), (dict(gx=AT[0], gxs=80), ALIAS),
    (dict(gw=AT[2]), ALIAS), (dict(ws=AT[3]), ALIAS), (dict(gh=AT[6], gx=AT[6] + 16), ALIAS),
])
def test_norm_backward(L, kw, status):
    assert back(L, **kw) == status


def test_rows_to_8_bits_and_back(L):
    q = lambda x=AT[0], xs=64, t=BF16, rows=3, dim=64, q=AT[1], qs=64, s=AT[2]: \
        L.rosetta_quantize_rows(x, xs, t, rows, dim, q, qs, s, None)  # noqa: E731
    d = lambda q=AT[0], qs=64, s=AT[1], t=BF16, rows=3, dim=64, o=AT[2], os=64: \
        L.rosetta_dequantize_rows(q, qs, s, t, rows, dim, o, os, None)  # noqa: E731
    for f in (q, d):
        assert f(rows=0) == OK and f(t=5) == PARAMS and f(dim=0) == PARAMS
        assert f(s=None) == NULL and f(q=None) == NULL and f(qs=63) == PARAMS
    assert q(q=AT[0] + 10) == ALIAS and q(s=AT[0]) == ALIAS and q(x=None) == NULL
    assert d(o=AT[0]) == ALIAS and d(o=AT[1]) == ALIAS and d(o=None) == NULL


def q8(L, a=AT[0], as_=64, sa=AT[1], b=AT[2], bs=64, sb=AT[3], bias=None, o=AT[4], os=96, t=BF16,
       m=5, n=96, k=64, ws=None, wsb=0):
    return L.rosetta_q8_matmul(a, as_, sa, b, bs, sb, bias, o, os, t, m, n, k, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(m=0), OK), (dict(n=0), PARAMS), (dict(t=3), PARAMS), (dict(a=None), NULL),
    (dict(b=None), NULL), (dict(sa=None), NULL), (dict(sb=None), NULL), (dict(o=None), NULL),
    (dict(as_=63), PARAMS), (dict(bs=63), PARAMS), (dict(os=95), PARAMS),
    (dict(k=131072, as_=1 << 18, bs=1 << 18), UNSUPPORTED), (dict(m=1 << 31), UNSUPPORTED),
    (dict(m=1 << 20, n=1 << 20, os=1 << 20), UNSUPPORTED), (dict(o=AT[4] + 1), PARAMS),
    (dict(o=AT[0]), ALIAS), (dict(o=AT[2] + 64), ALIAS), (dict(bias=AT[4] + 4), ALIAS),
    (dict(sb=AT[4]), ALIAS),
])
def test_q8_matmul(L, kw, status):
    assert q8(L, **kw) == status


def loss(L, h=AT[0], hs=64, w=AT[1], ws=64, t=BF16, tg=AT[2], rows=5, dim=64, vocab=100, o=AT[3],
         lse=AT[4], sp=AT[5], sb=1 << 30):
    return L.rosetta_cross_entropy(h, hs, w, ws, t, tg, -100, rows, dim, vocab, o, lse, sp, sb,
                                   None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), OK), (dict(t=F32), UNSUPPORTED), (dict(t=9), PARAMS), (dict(vocab=0), PARAMS),
    (dict(dim=0), PARAMS), (dict(h=None), NULL), (dict(w=None), NULL), (dict(tg=None), NULL),
    (dict(o=None), NULL), (dict(lse=None), NULL), (dict(sp=None), NULL), (dict(sb=8), SIZE),
    (dict(hs=63), PARAMS), (dict(ws=63), PARAMS), (dict(vocab=1 << 31), UNSUPPORTED),
    (dict(dim=1 << 21, hs=1 << 21, ws=1 << 21), UNSUPPORTED),
    (dict(o=AT[4]), ALIAS), (dict(sp=AT[1] + 256), ALIAS), (dict(tg=AT[2] + 4), PARAMS),
])
def test_cross_entropy(L, kw, status):
    assert loss(L, **kw) == status


def grad(L, h=AT[0], hs=64, w=AT[1], ws=64, t=F16, tg=AT[2], lse=AT[3], g=AT[4], rows=5, dim=64,
         vocab=100, gh=AT[5], ghs=64, gw=AT[6], gws=64, sp=AT[7], sb=1 << 40):
    return L.rosetta_cross_entropy_backward(h, hs, w, ws, t, tg, -100, lse, g, rows, dim, vocab,
                                            gh, ghs, gw, gws, sp, sb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0, gw=None), OK), (dict(t=F32), UNSUPPORTED), (dict(lse=None), NULL),
    (dict(g=None), NULL), (dict(sb=0), SIZE), (dict(sp=None), NULL), (dict(ghs=1), PARAMS),
    (dict(gws=1), PARAMS), (dict(gh=AT[0]), ALIAS), (dict(gw=AT[1]), ALIAS),
    (dict(gh=AT[6] + 128), ALIAS), (dict(sp=AT[6]), ALIAS),
])
def test_cross_entropy_backward(L, kw, status):
    assert grad(L, **kw) == status


def test_workspaces_grow_with_the_work_and_stay_bounded(L):
    f, b = (L.rosetta_cross_entropy_workspace_bytes, L.rosetta_cross_entropy_backward_workspace_bytes)
    assert f(0, 64, 100) == b(0, 64, 100) == 0
    assert 0 < f(8, 4096, 1000) < f(8, 4096, 128000) < f(800, 4096, 128000)
    # gradients hold a piece of the vocabulary, never all of it
    assert b(8192, 4096, 128000) < 8192 * 128000 * 2
    n = L.rosetta_rms_norm_backward_workspace_bytes
    assert n(0, 64) == 0 and n(3, 64) == 3 * 64 * 4
    assert n(10 ** 6, 64) == n(10 ** 5, 64)  # one part per workgroup, not per row


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_checks_types_and_sizes_first():
    x, w, f = z(4, 64), z(64), z(4, dtype=torch.float32)
    i8, t = z(4, 64, dtype=torch.int8), z(4, dtype=torch.int64)
    with pytest.raises(TypeError, match="ROCm device"):
        R.rms_norm_q8(x, w, 1e-5)
    with pytest.raises(TypeError, match="ROCm device"):
        R.q8_matmul(i8, f, i8, f)
    with pytest.raises(TypeError, match="torch.int8"):
        R.q8_matmul(x, f, i8, f)
    with pytest.raises(ValueError, match="matrix"):
        R.quantize_rows(z(2, 2, 64))
    for call in (lambda: R.rms_norm(x, w, 1e-5), lambda: R.quantize_rows(x),
                 lambda: R.dequantize_rows(i8, f, torch.float32),
                 lambda: R.rms_norm_backward(x, x, w, f),
                 lambda: R.cross_entropy(x, x, t),
                 lambda: R.cross_entropy_backward(x, x, t, f, f)):
        with pytest.raises(TypeError, match="ROCm device"):
            call()
    with pytest.raises(TypeError):
        R.rms_norm_q8([1.0], w, 1e-5)
