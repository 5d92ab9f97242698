"""Decoding in the clear: refusals through the C ABI with addresses that no device has
and through the binding with CPU tensors; and, in C++ built from the library's own
header, where rows and positions are put whatever starts, lens and the table hold."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_16915_amd import build as B
from paper_2609_16915_amd import rosetta as R

OK, NULL, PARAMS, UNSUPPORTED, ALIAS, SIZE = 0, 1, 2, 3, 4, 7
F32, BF16, F16 = 0, 1, 2
AT = [i << 40 for i in range(1, 17)]  # far apart


@pytest.fixture(scope="module")
def L():
    return R.lib()


CACHE = dict(k=AT[0], v=AT[1], k_scale=AT[2], v_scale=AT[3], pages=9, kv_heads=2, page=16, dim=64,
             page_stride=2048, head_stride=1024, place_stride=64, scale_page_stride=32,
             scale_head_stride=16)
ROWS = dict(table=AT[4], table_stride=3, table_len=3, starts=AT[5], lens=AT[6], batch=4, rows=10)


def given(kw):
    c = R.CacheStruct(**{**CACHE, **{n: kw.pop(n) for n in list(kw) if n in CACHE}})
    r = R.RowsStruct(**{**ROWS, **{n: kw.pop(n) for n in list(kw) if n in ROWS}})
    return c, r


def write(L, t=BF16, kp=AT[7], krs=128, khs=64, vp=AT[8], vrs=128, vhs=64, **kw):
    c, r = given(kw)
    return L.rosetta_kv_write(kp, krs, khs, vp, vrs, vhs, t, c, r, None)


def read(L, t=BF16, kp=AT[7], krs=128, khs=64, vp=AT[8], vrs=128, vhs=64, **kw):
    c, r = given(kw)
    return L.rosetta_kv_read(c, r, t, kp, krs, khs, vp, vrs, vhs, None)


def keep(L, path=AT[7], count=AT[8], out=AT[9], **kw):
    c, r = given(kw)
    return L.rosetta_kv_keep(c, r, path, count, out, None)


def attend(L, t=BF16, q=AT[7], qrs=512, qhs=64, heads=8, most=10, masks=None, words=0, scale=0.125,
           out=AT[8], ors=512, ohs=64, lse=AT[9], ws=AT[10], wsb=1 << 40, **kw):
    c, r = given(kw)
    return L.rosetta_kv_attention(q, qrs, qhs, t, heads, c, r, most, masks, words, scale, out, ors,
                                  ohs, lse, ws, wsb, None)


LONG = dict(table_len=5000, table_stride=5000)  # (parts to join)
COMMON = [
    (dict(pages=0), PARAMS), (dict(kv_heads=0), PARAMS), (dict(dim=0), UNSUPPORTED),
    (dict(dim=8, place_stride=16), UNSUPPORTED), (dict(dim=72, place_stride=80), UNSUPPORTED),
    (dict(dim=272), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED),
    (dict(page=0), UNSUPPORTED), (dict(pages=1 << 31), UNSUPPORTED),
    (dict(batch=65536), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED),
    (dict(table_len=0), PARAMS),
    (dict(table_len=(1 << 26) + 1, table_stride=1 << 27), UNSUPPORTED), (dict(table_stride=2), PARAMS),
    (dict(place_stride=56), PARAMS), (dict(place_stride=48), PARAMS),
    (dict(head_stride=1008), PARAMS), (dict(page_stride=2032), PARAMS),
    (dict(head_stride=1032), PARAMS), (dict(page_stride=2056), PARAMS),
    (dict(place_stride=1 << 27, head_stride=1 << 32, page_stride=1 << 33), PARAMS),
    (dict(scale_head_stride=15), PARAMS), (dict(scale_page_stride=31), PARAMS),
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scale=None), NULL),
    (dict(v_scale=None), NULL), (dict(table=None), NULL), (dict(starts=None), NULL),
    (dict(lens=None), NULL), (dict(k=AT[0] + 8), PARAMS), (dict(v=AT[1] + 4), PARAMS),
    (dict(k_scale=AT[2] + 2), PARAMS), (dict(starts=AT[5] + 1), PARAMS),
]
WRITTEN = [(dict(v=AT[0]), ALIAS), (dict(v=AT[0] + 1024), ALIAS), (dict(k_scale=AT[1]), ALIAS),
           (dict(v_scale=AT[2] + 64), ALIAS), (dict(table=AT[0]), ALIAS), (dict(lens=AT[3]), ALIAS)]


@pytest.mark.parametrize("kw,status", COMMON + WRITTEN + [
    (dict(rows=0, kp=None, vp=None), OK), (dict(batch=0, table=None, starts=None, lens=None), OK),
    (dict(t=3), PARAMS), (dict(t=-1), PARAMS), (dict(kp=None), NULL), (dict(vp=None), NULL),
    (dict(krs=127), PARAMS), (dict(khs=63), PARAMS), (dict(vrs=64), PARAMS), (dict(vhs=0), PARAMS),
    (dict(kp=AT[7] + 1), PARAMS), (dict(t=F32, vp=AT[8] + 2), PARAMS), (dict(kp=AT[0] + 512), ALIAS),
    (dict(vp=AT[3]), ALIAS),
    # keys and values in one buffer, page by page: apart; with pages too near: not
    (dict(rows=0, page_stride=4096, v=AT[0] + 2048), OK),
    (dict(page_stride=4096, v=AT[0] + 2032), ALIAS),
    # places of heads; heads of rows
    (dict(rows=0, place_stride=128, head_stride=64), OK),
    (dict(rows=0, krs=64, khs=640), OK), (dict(krs=64, khs=639), PARAMS),
])
def test_write(L, kw, status):
    assert write(L, **kw) == status
    assert bool(L.rosetta_last_error()) == (status != OK)


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(rows=0, kp=None, vp=None), OK), (dict(batch=0), OK), (dict(t=7), PARAMS),
    (dict(kp=None), NULL), (dict(vp=None), NULL), (dict(krs=100), PARAMS), (dict(vhs=16), PARAMS),
    (dict(vp=AT[7]), ALIAS), (dict(vp=AT[7] + 128), ALIAS), (dict(kp=AT[1] + 64), ALIAS),
    (dict(kp=AT[5]), ALIAS), (dict(kp=AT[4]), ALIAS),
])
def test_read(L, kw, status):
    assert read(L, **kw) == status


@pytest.mark.parametrize("kw,status", COMMON + WRITTEN + [
    (dict(batch=0), OK), (dict(path=None), NULL), (dict(count=None), NULL), (dict(out=None), NULL),
    (dict(out=AT[6]), ALIAS), (dict(out=AT[8] + 4), ALIAS), (dict(path=AT[0] + 64), ALIAS),
    (dict(out=AT[7]), ALIAS), (dict(count=AT[8] + 2), PARAMS),
])
def test_keep(L, kw, status):
    assert keep(L, **kw) == status


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(rows=0, q=None, out=None), OK), (dict(batch=0), OK), (dict(most=0), OK),
    (dict(t=F32), UNSUPPORTED), (dict(t=5), PARAMS), (dict(heads=0), PARAMS), (dict(heads=7), PARAMS),
    (dict(heads=1 << 16, qrs=1 << 23, ors=1 << 23), UNSUPPORTED), (dict(most=1 << 30), UNSUPPORTED),
    (dict(rows=1 << 29), UNSUPPORTED), (dict(scale=-1.0), PARAMS),
    (dict(scale=float("nan")), PARAMS), (dict(scale=float("inf")), PARAMS),
    (dict(masks=AT[11], words=0), PARAMS), (dict(masks=AT[11], words=1, most=65, rows=70), PARAMS),
    (dict(masks=AT[11] + 4, words=1), PARAMS), (dict(q=None), NULL), (dict(out=None), NULL),
    (dict(qrs=511), PARAMS), (dict(ohs=32), PARAMS), (dict(q=AT[7] + 1), PARAMS),
    (dict(ws=None, **LONG), NULL), (dict(wsb=64, **LONG), SIZE),
    (dict(ws=AT[10] + 8, **LONG), PARAMS),
    (dict(out=AT[7]), ALIAS), (dict(out=AT[7] + 128), ALIAS), (dict(lse=AT[8]), ALIAS),
    (dict(ws=AT[9], **LONG), ALIAS), (dict(out=AT[1]), ALIAS), (dict(ws=AT[5], **LONG), ALIAS),
    (dict(masks=AT[8], words=1), ALIAS), (dict(lse=AT[9] + 2), PARAMS),
])
def test_attention(L, kw, status):
    assert attend(L, **kw) == status


def test_nothing_given(L):
    c, r = given({})
    assert L.rosetta_kv_keep(None, r, AT[7], AT[8], AT[9], None) == NULL
    assert L.rosetta_kv_keep(c, None, AT[7], AT[8], AT[9], None) == NULL


def masks(L, parents=AT[0], starts=AT[1], batch=4, rows=10, words=2, out=AT[2]):
    return L.rosetta_tree_masks(parents, starts, batch, rows, words, out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), OK), (dict(batch=0), OK), (dict(words=0), PARAMS), (dict(parents=None), NULL),
    (dict(starts=None), NULL), (dict(out=None), NULL), (dict(out=AT[0]), ALIAS),
    (dict(out=AT[1] + 8), ALIAS), (dict(out=AT[2] + 4), PARAMS), (dict(batch=65536), UNSUPPORTED),
    (dict(rows=1 << 30), UNSUPPORTED), (dict(words=(1 << 20) + 1), UNSUPPORTED),
    (dict(rows=(1 << 30) - 1, words=1 << 10), UNSUPPORTED),
])
def test_tree_masks(L, kw, status):
    assert masks(L, **kw) == status


def verify(L, p=AT[0], ps=100, q=AT[1], qs=100, t=F32, drafts=AT[2], parents=AT[3], u=AT[4],
           starts=AT[5], batch=4, rows=10, vocab=100, tokens=AT[6], path=AT[7], count=AT[8],
           ws=AT[9], wsb=1 << 20):
    return L.rosetta_verify_drafts(p, ps, q, qs, t, drafts, parents, u, starts, batch, rows, vocab,
                                   tokens, path, count, ws, wsb, None)


BIG = dict(vocab=50000, ps=50000, qs=50000)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), OK), (dict(t=3), PARAMS), (dict(vocab=0), PARAMS), (dict(ps=99), PARAMS),
    (dict(qs=1), PARAMS), (dict(vocab=(1 << 30) + 1, ps=1 << 31, qs=1 << 31), UNSUPPORTED),
    (dict(batch=65536), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED), (dict(p=None), NULL),
    (dict(q=None), NULL), (dict(drafts=None), NULL), (dict(u=None), NULL), (dict(starts=None), NULL),
    (dict(tokens=None), NULL), (dict(path=None), NULL), (dict(count=None), NULL),
    (dict(ws=None, **BIG), NULL), (dict(wsb=8, **BIG), SIZE), (dict(ws=AT[9] + 4, **BIG), PARAMS),
    (dict(drafts=AT[2] + 4), PARAMS), (dict(tokens=AT[0]), ALIAS), (dict(path=AT[6] + 40), ALIAS),
    (dict(count=AT[4]), ALIAS), (dict(path=AT[3]), ALIAS), (dict(ws=AT[8], **BIG), ALIAS),
])
def test_verify_drafts(L, kw, status):
    assert verify(L, **kw) == status


def test_workspaces(L):
    w = L.rosetta_kv_attention_workspace_bytes
    assert w(32, 8, 128, 1, 0, 0, 4096) == 0 and w(32, 7, 128, 1, 1, 1, 4096) == 0
    assert w(32, 8, 128, 1, 1, 1, 16) == 0  # nothing to split
    assert w(32, 8, 128, 1, 1, 1, 1 << 17) > 0
    assert L.rosetta_verify_drafts_workspace_bytes(3, 0) == 0


# ------------------------------------------------------------ the binding

def cpu_cache():
    return R.KVCache(torch.zeros((2, 1, 16, 64), dtype=torch.int8),
                     torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.zeros((2, 1, 16)),
                     torch.zeros((2, 1, 16)))


def test_host_tensors_are_refused():
    i = torch.zeros((1, 2), dtype=torch.int32)
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    c = cpu_cache()
    for call in (lambda: R.kv_write(x, x, c, i, i[0], i[0, :1]),
                 lambda: R.kv_read(c, i, i[0], i[0, :1], 1, torch.float32),
                 lambda: R.kv_keep(c, i, i[0], i[0, :1], i[0, :1], i[0, :1]),
                 lambda: R.kv_attention(x, c, i, i[0], i[0, :1]),
                 lambda: R.tree_masks(i[0], i[0], 4),
                 lambda: R.verify_drafts(x[0].float(), x[0].float(), i[0, :1].long(),
                                         torch.zeros(1), i[0])):
        with pytest.raises(TypeError, match="ROCm device"):
            call()


def test_wrong_kinds_of_argument():
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: R.kv_write(None, None, None, i, i, i),
                 lambda: R.kv_read((1, 2, 3, 4), i, i, i, 1, torch.float32),
                 lambda: R.kv_attention(None, cpu_cache(), i, i, i),
                 lambda: R.tree_masks(None, i, 4), lambda: R.verify_drafts(None, i, i, i, i)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError, match="max_rows"):
        R.tree_masks(i, i, 0)


# ---------------------------------------------- where rows and positions are put

PROGRAM = r"""
#include <cstdio>
#include "decode.hpp"
using namespace rosetta;
int main() {
  const int64_t odd[] = {-2147483648LL, -100, -1, 0, 1, 2, 5, 9, 10, 11, 1000, 2147483647LL};
  long bad = 0, spans = 0, places = 0;
  for (int64_t s : odd)
    for (int64_t e : odd)
      for (int64_t l : odd)
        for (size_t rows : {(size_t)0, (size_t)1, (size_t)10}) {
          const int starts[2] = {(int)s, (int)e}, lens[1] = {(int)l};
          const Span sp = span_of(starts, lens, 0, rows);
          ++spans;
          // inside the call's rows, in order, and as given where that makes sense
          if (sp.first < 0 || sp.n < 0 || (size_t)(sp.first + (int64_t)sp.n) > rows) ++bad;
          if (s >= 0 && e >= s && e <= (int64_t)rows && (sp.first != s || sp.n != e - s)) ++bad;
          if (sp.base != l - sp.n) ++bad;
          const int table[3] = {(int)s, 1, (int)e};
          for (int log : {4, 5, 10})
            for (size_t pages : {(size_t)1, (size_t)2, (size_t)10})
              for (int64_t t : {sp.base - 1, sp.base, sp.base + sp.n - 1, (int64_t)-1, (int64_t)0,
                                ((int64_t)1 << log) - 1, (int64_t)1 << log, ((int64_t)3 << log) - 1,
                                (int64_t)3 << log, (int64_t)1 << 40}) {
                const int64_t pg = page_of(table, 3, log, pages, t);
                ++places;
                const bool in = t >= 0 && t < (int64_t)3 << log;
                const int64_t entry = in ? table[t >> log] : -1;
                const int64_t want = entry >= 0 && entry < (int64_t)pages ? entry : -1;
                if (pg != want) ++bad;
              }
        }
  std::printf("%ld spans %ld places %ld bad\n", spans, places, bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")),
                    reason="needs hipcc")
def test_rows_and_positions_stay_inside(tmp_path):
    src, exe = tmp_path / "places.hip", tmp_path / "places"
    src.write_text(PROGRAM)
    subprocess.run([B.hipcc(), "-O1", "-std=c++17", f"--offload-arch={B.ARCH}", f"-I{B.INCLUDE}",
                    f"-I{B.CSRC}", str(src), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    assert out.stdout.startswith("5184 spans")


# ------------------------------------------------- streams and devices, stood in for

CALLS = ["kv_write", "kv_read", "kv_keep", "tree_masks", "kv_attention", "verify_drafts"]


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_is_entered_however_it_is_passed(monkeypatch, name):
    """What a call allocates comes from the memory of the stream that it runs on."""
    import inspect

    class Entered(Exception):
        pass

    stream = object()

    def enter(s):
        assert s is stream
        raise Entered

    monkeypatch.setattr(torch.cuda, "stream", enter)
    call = getattr(R, name)
    at = list(inspect.signature(call).parameters).index("stream")
    args = [torch.zeros(4, 64)] * at
    with pytest.raises(Entered):
        call(*args[:2], stream=stream)
    with pytest.raises(Entered):
        call(*args, stream)
    with pytest.raises(TypeError, match="stream"):
        call(*args, stream, stream=stream)


class OnDevice(torch.Tensor):
    """A tensor that says it lies on a ROCm device."""
    @staticmethod
    def __new__(cls, t, index):
        f = torch.Tensor._make_subclass(cls, t)
        f.at = index
        return f

    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.at))

    def get_device(self):
        return getattr(self, "at", 0)

    def new_empty(self, *args, **kw):
        return OnDevice(torch.empty(*args, **kw), self.at)


@pytest.fixture
def machine(monkeypatch):
    """Two devices, 0 the current one, and a library that notes where it is called."""
    class Machine:
        current = 0

        def __init__(self):
            self.calls = []

        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: 64
            return lambda *a: self.calls.append((name, self.current, a[-1])) or 0

    m = Machine()

    class On:
        def __init__(self, index):
            self.index = index if isinstance(index, int) else index.index

        def __enter__(self):
            self.before, m.current = m.current, self.index

        def __exit__(self, *a):
            m.current = self.before

    monkeypatch.setattr(R, "lib", lambda: m)
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: m.current, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 100 + i, raising=False)
    return m


def made(on, cache_on=None):
    """The arguments of every call, on device `on` (the cache on another, if given)."""
    t = lambda x: OnDevice(x, on)  # noqa: E731
    c = lambda x: OnDevice(x, on if cache_on is None else cache_on)  # noqa: E731
    cache = R.KVCache(c(torch.zeros((2, 1, 16, 64), dtype=torch.int8)),
                      c(torch.zeros((2, 1, 16, 64), dtype=torch.int8)),
                      c(torch.zeros((2, 1, 16))), c(torch.zeros((2, 1, 16))))
    i = lambda *v: t(torch.tensor(v, dtype=torch.int32))  # noqa: E731
    table, starts, lens = t(torch.zeros((1, 2), dtype=torch.int32)), i(0, 3), i(5)
    x = t(torch.zeros((3, 1, 64), dtype=torch.bfloat16))
    p = t(torch.zeros((3, 9)))
    return {"kv_write": (x, x, cache, table, starts, lens),
            "kv_read": (cache, table, starts, lens, 3, torch.bfloat16),
            "kv_keep": (cache, table, starts, lens, i(0, 1, -1), i(2)),
            "tree_masks": (i(-1, 0, 1), starts, 3),
            "kv_attention": (x, cache, table, starts, lens),
            "verify_drafts": (p, p, t(torch.zeros(3).long()), t(torch.zeros(3)), starts)}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("on", [0, 1])
def test_a_call_runs_on_its_tensors_device(machine, name, on):
    getattr(R, name)(*made(on)[name])
    assert machine.calls == [("rosetta_" + name, on, 100 + on)] and machine.current == 0


@pytest.mark.parametrize("name", ["kv_write", "kv_read", "kv_keep", "kv_attention"])
def test_a_cache_of_another_device_is_refused(machine, name):
    with pytest.raises(ValueError, match="device"):
        getattr(R, name)(*made(0, cache_on=1)[name])
    assert not machine.calls


@pytest.mark.parametrize("name", ["kv_write", "kv_attention", "verify_drafts"])
def test_a_stream_of_another_device_is_refused(machine, monkeypatch, name):
    class Stream:
        device_index, cuda_stream = 1, 7

    class Entered:
        def __init__(self, s):
            pass

        def __enter__(self):
            pass

        def __exit__(self, *a):
            pass

    monkeypatch.setattr(torch.cuda, "stream", Entered)
    with pytest.raises(ValueError, match="stream"):
        getattr(R, name)(*made(0)[name], stream=Stream())
    assert not machine.calls


def test_wrong_sizes_and_types(machine):
    m = made(0)
    x, _, cache, table, starts, lens = m["kv_write"]
    wide = OnDevice(torch.zeros((3, 2, 64), dtype=torch.bfloat16), 0)
    f32 = OnDevice(torch.zeros((3, 1, 64)), 0)
    ints64 = OnDevice(torch.zeros(2).long(), 0)
    for error, call in (
            (ValueError, lambda: R.kv_write(wide, wide, cache, table, starts, lens)),
            (TypeError, lambda: R.kv_write(x, f32, cache, table, starts, lens)),
            (TypeError, lambda: R.kv_write(x, x, cache, table, ints64, lens)),
            (TypeError, lambda: R.kv_write(x, x, cache, table.long(), starts, lens)),
            (ValueError, lambda: R.kv_write(x, x, cache, table, lens, lens)),
            (ValueError, lambda: R.kv_write(x, x, cache, table[0], starts, lens)),
            (ValueError, lambda: R.kv_write(x.transpose(0, 2), x, cache, table, starts, lens)),
            (ValueError, lambda: R.kv_attention(x, cache, table, starts, lens, out=wide)),
            (TypeError, lambda: R.kv_attention(x, cache, table, starts, lens, out=f32)),
            (TypeError, lambda: R.kv_attention(x, cache, table, starts, lens, masks=starts)),
            (ValueError, lambda: R.kv_attention(x, cache, table, starts, lens, max_rows=-1)),
            (TypeError, lambda: R.kv_attention(x.int(), cache, table, starts, lens)),
            (TypeError, lambda: R.kv_read(cache, table, starts, lens, 3, torch.int8)),
            (ValueError, lambda: R.kv_write(x, x, cache._replace(v=cache.v[:1]), table, starts, lens)),
            (TypeError, lambda: R.kv_write(x, x, cache._replace(v=f32), table, starts, lens)),
            (ValueError, lambda: R.kv_write(x, x, cache._replace(
                k_scale=cache.k_scale[:, :, :8], v_scale=cache.v_scale[:, :, :8]), table, starts, lens)),
            (TypeError, lambda: R.verify_drafts(*m["verify_drafts"][:2], starts,
                                                *m["verify_drafts"][3:])),
            (ValueError, lambda: R.verify_drafts(*m["verify_drafts"],
                                                 workspace=OnDevice(torch.zeros(3), 0)))):
        with pytest.raises(error):
            call()
    assert not machine.calls
