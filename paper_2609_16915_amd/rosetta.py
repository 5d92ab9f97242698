"""Python binding of librosetta (batched TFHE PBS on MI355X).

Argument marshalling only: every step of the PBS runs in the library's HIP
kernels.  Device buffers are torch tensors on a ROCm device (dtype uint64, or
int64 read as raw 64-bit words), passed by data_ptr() together with the
current HIP stream; host helpers take and return numpy arrays.  There is no
fallback: if the library is not built, or a call fails, an exception is
raised.

A call given a `stream` is put on that stream and waits for nothing on any
other: what it reads must be ready there (made on it, or before its
wait_stream(); torch.ones() beside the call is on the current stream, and is
not), and must stay until it has run.
"""
from __future__ import annotations

import ctypes as C
import functools
import inspect
import os
from typing import NamedTuple

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librosetta.so")
P = 0xFFFFFFFF00000001

STATUS = {0: "ROSETTA_OK", 1: "ROSETTA_ERR_NULL", 2: "ROSETTA_ERR_PARAMS",
          3: "ROSETTA_ERR_UNSUPPORTED", 4: "ROSETTA_ERR_ALIAS", 5: "ROSETTA_ERR_NOMEM",
          6: "ROSETTA_ERR_DEVICE", 7: "ROSETTA_ERR_SIZE"}


class RosettaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class Params(C.Structure):
    """rosetta_params (include/rosetta.h)."""

    _fields_ = [(name, C.c_uint32) for name in
                ("n", "k", "N", "pbs_level", "pbs_base_log", "ks_level", "ks_base_log",
                 "msg_bits")]

    @classmethod
    def from_dict(cls, d: dict) -> "Params":
        d = dict(d)
        d.setdefault("k", 1)
        return cls(**d)

    @property
    def M(self) -> int:
        return 1 << self.msg_bits


# Every symbol the header declares, with its ctypes signature.
_u64p = C.c_void_p
_pp = C.POINTER(Params)
_ST = C.c_int
SIGNATURES = {
    "rosetta_version": (C.c_char_p, []),
    "rosetta_status_string": (C.c_char_p, [C.c_int]),
    "rosetta_last_error": (C.c_char_p, []),
    "rosetta_check_params": (_ST, [_pp]),
    "rosetta_bsk_words": (C.c_size_t, [_pp]),
    "rosetta_bsk_device_words": (C.c_size_t, [_pp]),
    "rosetta_ksk_words": (C.c_size_t, [_pp]),
    "rosetta_ksk_device_words": (C.c_size_t, [_pp]),
    "rosetta_bsk_prepare": (_ST, [_u64p, _u64p, _pp, C.c_void_p]),
    "rosetta_ksk_prepare": (_ST, [_u64p, _u64p, _pp, C.c_void_p]),
    "rosetta_pbs_batch": (_ST, [_u64p, _u64p, _u64p, _u64p, _u64p, C.c_size_t, _pp,
                                C.c_void_p]),
    "rosetta_pbs_workspace_bytes": (C.c_size_t, [_pp, C.c_size_t]),
    "rosetta_pbs_batch_ws": (_ST, [_u64p, _u64p, _u64p, _u64p, _u64p, C.c_size_t, _pp,
                                   C.c_void_p, C.c_size_t, C.c_void_p]),
    "rosetta_pbs_batch_noalloc": (_ST, [_u64p, _u64p, _u64p, _u64p, _u64p, C.c_size_t, _pp,
                                        C.c_void_p]),
    "rosetta_blind_rotate": (_ST, [_u64p, _u64p, _u64p, _u64p, C.c_size_t, _pp, C.c_void_p]),
    "rosetta_blind_rotate_extract": (_ST, [_u64p, _u64p, _u64p, _u64p, C.c_size_t, _pp,
                                           C.c_void_p]),
    "rosetta_keyswitch": (_ST, [_u64p, _u64p, _u64p, C.c_size_t, _pp, C.c_void_p]),
    "rosetta_ntt_forward": (_ST, [_u64p, _u64p, C.c_size_t, C.c_uint32, C.c_void_p]),
    "rosetta_ntt_inverse": (_ST, [_u64p, _u64p, C.c_size_t, C.c_uint32, C.c_void_p]),
    "rosetta_poly_mul": (_ST, [_u64p, _u64p, _u64p, C.c_size_t, C.c_uint32, C.c_void_p]),
    "rosetta_field_op": (_ST, [C.c_int, _u64p, _u64p, _u64p, _u64p, C.c_size_t, C.c_void_p]),
    "rosetta_modmul_chain": (_ST, [C.c_uint64, C.c_uint32, C.c_uint32, _u64p, C.c_void_p]),
    "rosetta_keygen": (_ST, [C.c_uint64, _pp, C.c_double, C.c_double, _u64p, _u64p, _u64p,
                             _u64p]),
    "rosetta_lwe_encrypt": (_ST, [C.c_uint64, _pp, C.c_double, _u64p, C.c_uint32, _u64p,
                                  C.c_size_t, _u64p]),
    "rosetta_lwe_decrypt": (_ST, [_pp, _u64p, C.c_uint32, _u64p, C.c_size_t, _u64p]),
    "rosetta_lwe_encrypt_plain": (_ST, [C.c_uint64, C.c_double, _u64p, C.c_uint32, _u64p,
                                        C.c_size_t, _u64p]),
    "rosetta_lut_build": (_ST, [_pp, _u64p, _u64p]),
    "rosetta_shutdown": (_ST, []),
    "rosetta_blind_rotate_glwe": (_ST, [_u64p, _u64p, _u64p, _u64p, C.c_size_t, C.c_uint32,
                                        _pp, C.c_int, C.c_void_p]),
    "rosetta_lwe_add_consts": (_ST, [_u64p, _u64p, _u64p, C.c_size_t, C.c_uint32, C.c_uint32,
                                     C.c_void_p]),
    "rosetta_lwe_sum_groups": (_ST, [_u64p, C.c_uint64, _u64p, C.c_size_t, C.c_uint32,
                                     C.c_uint32, C.c_void_p]),
    "rosetta_lwe_combine": (_ST, [_u64p, C.c_uint64, _u64p, C.c_uint64, _u64p, C.c_uint64, _u64p,
                                  C.c_size_t, C.c_void_p]),
    "rosetta_autk_words": (C.c_size_t, [_pp, C.c_uint32]),
    "rosetta_autk_prepare": (_ST, [_u64p, _u64p, _pp, C.c_uint32, C.c_void_p]),
    "rosetta_trace": (_ST, [_u64p, _u64p, _u64p, C.c_size_t, _pp, C.c_uint32, C.c_uint32,
                            C.c_void_p]),
    "rosetta_plain_prepare": (_ST, [_u64p, _u64p, C.c_size_t, C.c_uint32, C.c_void_p]),
    "rosetta_glwe_mul_plain": (_ST, [_u64p, _u64p, _u64p, _u64p, C.c_size_t, C.c_uint32,
                                     C.c_uint32, C.c_void_p]),
    "rosetta_glwe_recombine": (_ST, [_u64p, _u64p, _u64p, C.c_size_t, C.c_uint32, C.c_uint32,
                                     C.c_void_p]),
    "rosetta_glwe_monomial_mul": (_ST, [_u64p, _u64p, _u64p, C.c_size_t, C.c_uint32,
                                        C.c_uint32, C.c_void_p]),
    "rosetta_sample_extract": (_ST, [_u64p, _u64p, C.c_size_t, C.c_uint32, C.c_void_p]),
    "rosetta_glwe_encrypt": (_ST, [C.c_uint64, _pp, C.c_double, _u64p, _u64p, C.c_size_t,
                                   _u64p]),
    "rosetta_glwe_phase": (_ST, [_pp, _u64p, _u64p, C.c_size_t, _u64p]),
    "rosetta_autk_keygen": (_ST, [C.c_uint64, _pp, C.c_uint32, C.c_uint32, C.c_double, _u64p,
                                  _u64p]),
    "rosetta_seglut_boundaries": (_ST, [C.c_double, C.c_double, C.c_uint32, C.c_int, _u64p]),
    "rosetta_seglut_build": (_ST, [C.c_int, _u64p, C.c_uint32, C.c_uint32, C.c_int, _u64p,
                                   _u64p]),
    "rosetta_seglut_protocol_polys": (_ST, [_u64p, C.c_uint32, C.c_uint32, _u64p, _u64p]),
    "rosetta_seglut_eval": (_ST, [_u64p, C.c_uint32, C.c_uint32, _u64p, _u64p, _u64p, _u64p,
                                  C.c_size_t, _u64p]),
    "rosetta_seglut_precision": (_ST, [C.c_int, _u64p, C.c_uint32, C.c_uint32, _u64p, _u64p,
                                       _u64p, _u64p, C.c_size_t, _u64p]),
    "rosetta_encode_fixed": (_ST, [_u64p, C.c_size_t, C.c_int, _u64p]),
}



class LookupParams(C.Structure):
    """rosetta_lookup_params (include/rosetta.h)."""

    _fields_ = [(name, C.c_uint32) for name in
                ("nseg", "nbr", "margin", "x_scale_log", "coef_scale_log", "val_scale_log",
                 "cmp_scale_log", "trace_level", "trace_base_log", "cmp_refine_log")]


_lpp = C.POINTER(LookupParams)
SIGNATURES.update({
    "rosetta_lookup_plain_words": (C.c_size_t, [_pp, _lpp]),
    "rosetta_lookup_encode": (_ST, [_pp, _lpp, _u64p, _u64p, _u64p, _u64p, _u64p]),
    "rosetta_lookup_prepare": (_ST, [_u64p, _u64p, _pp, _lpp, C.c_void_p]),
    "rosetta_lookup_workspace_bytes": (C.c_size_t, [_pp, _lpp, C.c_size_t]),
    "rosetta_lookup_workspace_offset": (C.c_size_t, [_pp, _lpp, C.c_size_t, C.c_uint32]),
    "rosetta_lookup_eval": (_ST, [_u64p, _u64p, _u64p, _u64p, _u64p, _u64p, _u64p, _u64p,
                                  C.c_size_t, _pp, _lpp, _u64p, C.c_size_t, C.c_void_p]),
})

_sz, _i32, _i64, _f32 = C.c_size_t, C.c_int, C.c_int64, C.c_float
SIGNATURES.update({
    "rosetta_rms_norm": (_ST, [_u64p, _sz, _u64p, _sz, _u64p, _i32, _i32, _sz, _sz, _f32, _u64p,
                               _sz, _u64p, _sz, _u64p, _sz, _u64p, _u64p, C.c_void_p]),
    "rosetta_rms_norm_backward": (_ST, [_u64p, _sz, _u64p, _sz, _u64p, _sz, _u64p, _i32, _u64p,
                                        _i32, _sz, _sz, _u64p, _sz, _u64p, _u64p, _sz,
                                        C.c_void_p]),
    "rosetta_rms_norm_backward_workspace_bytes": (_sz, [_sz, _sz]),
    "rosetta_quantize_rows": (_ST, [_u64p, _sz, _i32, _sz, _sz, _u64p, _sz, _u64p, C.c_void_p]),
    "rosetta_dequantize_rows": (_ST, [_u64p, _sz, _u64p, _i32, _sz, _sz, _u64p, _sz,
                                      C.c_void_p]),
    "rosetta_q8_matmul": (_ST, [_u64p, _sz, _u64p, _u64p, _sz, _u64p, _u64p, _u64p, _sz, _i32,
                                _sz, _sz, _sz, _u64p, _sz, C.c_void_p]),
    "rosetta_q8_matmul_workspace_bytes": (_sz, [_sz, _sz, _sz]),
    "rosetta_cross_entropy": (_ST, [_u64p, _sz, _u64p, _sz, _i32, _u64p, _i64, _sz, _sz, _sz,
                                    _u64p, _u64p, _u64p, _sz, C.c_void_p]),
    "rosetta_cross_entropy_workspace_bytes": (_sz, [_sz, _sz, _sz]),
    "rosetta_cross_entropy_backward": (_ST, [_u64p, _sz, _u64p, _sz, _i32, _u64p, _i64, _u64p,
                                             _u64p, _sz, _sz, _sz, _u64p, _sz, _u64p, _sz, _u64p,
                                             _sz, C.c_void_p]),
    "rosetta_cross_entropy_backward_workspace_bytes": (_sz, [_sz, _sz, _sz]),
})



class CacheStruct(C.Structure):
    """rosetta_kv_cache (include/rosetta.h)."""

    _fields_ = ([(name, C.c_void_p) for name in ("k", "v", "k_scale", "v_scale")] +
                [(name, C.c_size_t) for name in
                 ("pages", "kv_heads", "page", "dim", "page_stride", "head_stride",
                  "place_stride", "scale_page_stride", "scale_head_stride")])


class RowsStruct(C.Structure):
    """rosetta_kv_rows (include/rosetta.h)."""

    _fields_ = [("table", C.c_void_p), ("table_stride", C.c_size_t), ("table_len", C.c_size_t),
                ("starts", C.c_void_p), ("lens", C.c_void_p), ("batch", C.c_size_t),
                ("rows", C.c_size_t)]


_cp, _rp = C.POINTER(CacheStruct), C.POINTER(RowsStruct)
SIGNATURES.update({
    "rosetta_kv_write": (_ST, [_u64p, _sz, _sz, _u64p, _sz, _sz, _i32, _cp, _rp, C.c_void_p]),
    "rosetta_kv_read": (_ST, [_cp, _rp, _i32, _u64p, _sz, _sz, _u64p, _sz, _sz, C.c_void_p]),
    "rosetta_kv_keep": (_ST, [_cp, _rp, _u64p, _u64p, _u64p, C.c_void_p]),
    "rosetta_tree_masks": (_ST, [_u64p, _u64p, _sz, _sz, _sz, _u64p, C.c_void_p]),
    "rosetta_kv_attention": (_ST, [_u64p, _sz, _sz, _i32, _sz, _cp, _rp, _sz, _u64p, _sz, _f32,
                                   _u64p, _sz, _sz, _u64p, _u64p, _sz, C.c_void_p]),
    "rosetta_kv_attention_workspace_bytes": (_sz, [_sz] * 7),
    "rosetta_verify_drafts": (_ST, [_u64p, _sz, _u64p, _sz, _i32, _u64p, _u64p, _u64p, _u64p, _sz,
                                    _sz, _sz, _u64p, _u64p, _u64p, _u64p, _sz, C.c_void_p]),
    "rosetta_verify_drafts_workspace_bytes": (_sz, [_sz, _sz]),
})

FUNCTIONS = {"inv": 0, "inv_sqrt": 1, "silu": 2, "gelu": 3, "exp": 4}
SPACINGS = {"uniform": 0, "log": 1}
FITS = {"linear": 0, "constant": 1}

_lib = None


def lib():
    """Load librosetta.so (built in-tree by paper_2609_16915_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run "
                               "`python -m paper_2609_16915_amd.build` first")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise RosettaError(status, lib().rosetta_last_error().decode())


def _params(p) -> Params:
    return p if isinstance(p, Params) else Params.from_dict(p)


# --------------------------------------------------------------------------
# device buffers (torch)
# --------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _torch():
    import torch
    return torch


def _dev(t, name: str) -> int:
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a torch tensor on a ROCm device")
    if t.element_size() != 8 or not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous with 64-bit elements")
    return t.data_ptr()


def _stream(stream) -> int:
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _words(t) -> int:
    """Element count of a tensor (or numpy array)."""
    return int(t.numel()) if hasattr(t, "numel") else int(t.size)


def _expect(t, name: str, words: int):
    """Raise ValueError unless `t` holds exactly `words` elements.  Runs before
    any library call, so that a buffer of the wrong size never reaches a
    kernel (which would read or write out of its bounds)."""
    got = _words(t)
    if got != words:
        raise ValueError(f"{name} holds {got} words, the call needs {words}")


def _batch_of(t, name: str, row: int, allow_empty: bool = True) -> int:
    """Rows of `row` words in `t`; ValueError if the size is not a multiple."""
    got = _words(t)
    if got % row or (got == 0 and not allow_empty):
        raise ValueError(f"{name} holds {got} words, not a whole number of {row}-word rows")
    return got // row


def empty(words, device="cuda"):
    torch = _torch()
    return torch.empty(words, dtype=torch.uint64, device=device)


def to_device(a: np.ndarray, device="cuda"):
    torch = _torch()
    a = np.ascontiguousarray(a, dtype=np.uint64)
    return torch.from_numpy(a).to(device)


def to_host(t) -> np.ndarray:
    return t.cpu().numpy().view(np.uint64)


def bsk_words(params) -> int:
    return lib().rosetta_bsk_words(C.byref(_params(params)))


def version() -> str:
    """rosetta_version(): the version and the digest of the sources built."""
    return lib().rosetta_version().decode()


def ksk_words(params) -> int:
    return lib().rosetta_ksk_words(C.byref(_params(params)))


def ksk_device_words(params) -> int:
    return lib().rosetta_ksk_device_words(C.byref(_params(params)))


def check_params(params):
    _check(lib().rosetta_check_params(C.byref(_params(params))))


def bsk_prepare(bsk_std, params, out=None, stream=None):
    p = _params(params)
    _expect(bsk_std, "bsk_std", bsk_words(p))
    if out is None:
        out = empty(bsk_words(p), bsk_std.device)
    _expect(out, "bsk_dev", bsk_words(p))
    _check(lib().rosetta_bsk_prepare(_dev(bsk_std, "bsk_std"), _dev(out, "bsk_dev"), C.byref(p),
                                     _stream(stream)))
    return out


def ksk_prepare(ksk_std, params, out=None, stream=None):
    p = _params(params)
    _expect(ksk_std, "ksk_std", ksk_words(p))
    if out is None:
        out = empty(ksk_device_words(p), ksk_std.device)
    _expect(out, "ksk_dev", ksk_device_words(p))
    _check(lib().rosetta_ksk_prepare(_dev(ksk_std, "ksk_std"), _dev(out, "ksk_dev"), C.byref(p),
                                     _stream(stream)))
    return out


def _check_pbs_args(p, lwe_in, bsk_dev, ksk_dev, lut) -> int:
    """Sizes of the PBS inputs against the parameters; returns the batch."""
    batch = _batch_of(lwe_in, "lwe_in", p.n + 1)
    _expect(bsk_dev, "bsk_dev", bsk_words(p))
    _expect(ksk_dev, "ksk_dev", ksk_device_words(p))
    _expect(lut, "lut", p.N)
    return batch


def pbs_batch(lwe_in, bsk_dev, ksk_dev, lut, params, out=None, stream=None):
    p = _params(params)
    batch = _check_pbs_args(p, lwe_in, bsk_dev, ksk_dev, lut)
    if out is None:
        out = empty((batch, p.n + 1), lwe_in.device)
    _expect(out, "lwe_out", batch * (p.n + 1))
    _check(lib().rosetta_pbs_batch(_dev(lwe_in, "lwe_in"), _dev(bsk_dev, "bsk_dev"),
                                   _dev(ksk_dev, "ksk_dev"), _dev(lut, "lut"),
                                   _dev(out, "lwe_out"), batch, C.byref(p), _stream(stream)))
    return out


def pbs_workspace_bytes(params, batch: int) -> int:
    return lib().rosetta_pbs_workspace_bytes(C.byref(_params(params)), batch)


def pbs_batch_ws(lwe_in, bsk_dev, ksk_dev, lut, params, workspace, out=None, stream=None):
    p = _params(params)
    batch = _check_pbs_args(p, lwe_in, bsk_dev, ksk_dev, lut)
    if out is None:
        out = empty((batch, p.n + 1), lwe_in.device)
    _expect(out, "lwe_out", batch * (p.n + 1))
    if _words(workspace) * 8 < pbs_workspace_bytes(p, batch):
        raise ValueError(f"workspace holds {_words(workspace) * 8} bytes, the call needs "
                         f"{pbs_workspace_bytes(p, batch)}")
    _check(lib().rosetta_pbs_batch_ws(_dev(lwe_in, "lwe_in"), _dev(bsk_dev, "bsk_dev"),
                                      _dev(ksk_dev, "ksk_dev"), _dev(lut, "lut"),
                                      _dev(out, "lwe_out"), batch, C.byref(p),
                                      _dev(workspace, "workspace"),
                                      workspace.numel() * workspace.element_size(),
                                      _stream(stream)))
    return out


NOALLOC_SCRATCH_BYTES = 64 << 20


def pbs_batch_noalloc(lwe_in, bsk_dev, ksk_dev, lut, params, out, stream=None):
    """rosetta_pbs_batch_noalloc: the PBS with the library's static scratch
    (the caller passes the output buffer; nothing is allocated)."""
    p = _params(params)
    batch = _check_pbs_args(p, lwe_in, bsk_dev, ksk_dev, lut)
    _expect(out, "lwe_out", batch * (p.n + 1))
    _check(lib().rosetta_pbs_batch_noalloc(_dev(lwe_in, "lwe_in"), _dev(bsk_dev, "bsk_dev"),
                                           _dev(ksk_dev, "ksk_dev"), _dev(lut, "lut"),
                                           _dev(out, "lwe_out"), batch, C.byref(p),
                                           _stream(stream)))
    return out


def blind_rotate(lwe_in, bsk_dev, lut, params, out=None, stream=None):
    p = _params(params)
    batch = _batch_of(lwe_in, "lwe_in", p.n + 1)
    _expect(bsk_dev, "bsk_dev", bsk_words(p))
    _expect(lut, "lut", p.N)
    if out is None:
        out = empty((batch, 2 * p.N), lwe_in.device)
    _expect(out, "glwe_out", batch * 2 * p.N)
    _check(lib().rosetta_blind_rotate(_dev(lwe_in, "lwe_in"), _dev(bsk_dev, "bsk_dev"),
                                      _dev(lut, "lut"), _dev(out, "glwe_out"), batch, C.byref(p),
                                      _stream(stream)))
    return out


def blind_rotate_extract(lwe_in, bsk_dev, lut, params, out=None, stream=None):
    p = _params(params)
    batch = _batch_of(lwe_in, "lwe_in", p.n + 1)
    _expect(bsk_dev, "bsk_dev", bsk_words(p))
    _expect(lut, "lut", p.N)
    if out is None:
        out = empty((batch, p.N + 1), lwe_in.device)
    _expect(out, "big_out", batch * (p.N + 1))
    _check(lib().rosetta_blind_rotate_extract(_dev(lwe_in, "lwe_in"), _dev(bsk_dev, "bsk_dev"),
                                              _dev(lut, "lut"), _dev(out, "big_out"), batch,
                                              C.byref(p), _stream(stream)))
    return out


def keyswitch(big_in, ksk_dev, params, out=None, stream=None):
    p = _params(params)
    batch = _batch_of(big_in, "big_in", p.N + 1)
    _expect(ksk_dev, "ksk_dev", ksk_device_words(p))
    if out is None:
        out = empty((batch, p.n + 1), big_in.device)
    _expect(out, "lwe_out", batch * (p.n + 1))
    _check(lib().rosetta_keyswitch(_dev(big_in, "big_in"), _dev(ksk_dev, "ksk_dev"),
                                   _dev(out, "lwe_out"), batch, C.byref(p), _stream(stream)))
    return out


def ntt_forward(x, N: int, out=None, stream=None):
    count = _batch_of(x, "in", N)
    out = empty(x.shape, x.device) if out is None else out
    _expect(out, "out", count * N)
    _check(lib().rosetta_ntt_forward(_dev(x, "in"), _dev(out, "out"), count, N, _stream(stream)))
    return out


def ntt_inverse(x, N: int, out=None, stream=None):
    count = _batch_of(x, "in", N)
    out = empty(x.shape, x.device) if out is None else out
    _expect(out, "out", count * N)
    _check(lib().rosetta_ntt_inverse(_dev(x, "in"), _dev(out, "out"), count, N, _stream(stream)))
    return out


def poly_mul(a, b, N: int, out=None, stream=None):
    count = _batch_of(a, "a", N)
    _expect(b, "b", count * N)
    out = empty(a.shape, a.device) if out is None else out
    _expect(out, "c", count * N)
    _check(lib().rosetta_poly_mul(_dev(a, "a"), _dev(b, "b"), _dev(out, "c"), count, N,
                                  _stream(stream)))
    return out


FIELD_ADD, FIELD_SUB, FIELD_MUL, FIELD_MUL_ADD, FIELD_ADD_WEAK = 0, 1, 2, 3, 4
FIELD_MUL_ADD_WEAK, FIELD_MUL_POW2, FIELD_ROUND_TOP = 5, 256, 512


def field_op(op: int, a, b=None, c=None, out=None, stream=None):
    """Elementwise Goldilocks arithmetic with the kernels' device routines
    (op: FIELD_ADD, FIELD_SUB, FIELD_MUL, FIELD_MUL_ADD, FIELD_ADD_WEAK,
    FIELD_MUL_ADD_WEAK, FIELD_MUL_POW2 + e, FIELD_ROUND_TOP + s; the last
    returns int64 values as uint64)."""
    count = _words(a)
    for t, name in ((b, "b"), (c, "c")):
        if t is not None:
            _expect(t, name, count)
    out = empty(a.shape, a.device) if out is None else out
    _expect(out, "out", count)
    _check(lib().rosetta_field_op(op, _dev(a, "a"), None if b is None else _dev(b, "b"),
                                  None if c is None else _dev(c, "c"), _dev(out, "out"), count,
                                  _stream(stream)))
    return out


def modmul_chain(seed: int, threads: int, iters: int, out=None, stream=None):
    """Throughput probe: 8 register-resident product chains per thread
    (see rosetta_modmul_chain); returns out[threads]."""
    out = empty(threads) if out is None else out
    if _words(out) < threads:
        raise ValueError(f"out holds {_words(out)} words, the call needs {threads}")
    _check(lib().rosetta_modmul_chain(seed, threads, iters, _dev(out, "out"), _stream(stream)))
    return out


def shutdown():
    _check(lib().rosetta_shutdown())


# lookup-protocol primitives ------------------------------------------------

def blind_rotate_glwe(lwe_in, bsk_dev, glwe_tp, params, extract=False, group=1, out=None,
                      stream=None):
    """Blind rotation of GLWE test polynomials glwe_tp [batch*group][2N], each
    LWE selector of lwe_in [batch][n+1] serving `group` consecutive ones."""
    p = _params(params)
    batch = _batch_of(lwe_in, "lwe_in", p.n + 1)
    _expect(bsk_dev, "bsk_dev", bsk_words(p))
    _expect(glwe_tp, "glwe_tp", batch * group * 2 * p.N)
    shape = (batch * group, p.N + 1) if extract else (batch * group, 2 * p.N)
    if out is None:
        out = empty(shape, lwe_in.device)
    _expect(out, "out", shape[0] * shape[1])
    _check(lib().rosetta_blind_rotate_glwe(_dev(lwe_in, "lwe_in"), _dev(bsk_dev, "bsk_dev"),
                                           _dev(glwe_tp, "glwe_tp"), _dev(out, "out"), batch,
                                           group, C.byref(p), 1 if extract else 0,
                                           _stream(stream)))
    return out


def lwe_add_consts(lwe_in, consts, dim: int, out=None, stream=None):
    """out[q][j] = lwe_in[q] + (0, .., 0, consts[j])."""
    batch = _batch_of(lwe_in, "lwe_in", dim + 1)
    c = np.ascontiguousarray(consts, dtype=np.uint64)
    if out is None:
        out = empty((batch, c.size, dim + 1), lwe_in.device)
    _expect(out, "lwe_out", batch * c.size * (dim + 1))
    _check(lib().rosetta_lwe_add_consts(_dev(lwe_in, "lwe_in"), _np_ptr(c), _dev(out, "lwe_out"),
                                        batch, c.size, dim, _stream(stream)))
    return out


def lwe_sum_groups(lwe_in, count: int, dim: int, c0: int = 0, out=None, stream=None):
    """out[q] = sum_j lwe_in[q][j] + (0, .., 0, c0)."""
    batch = _batch_of(lwe_in, "lwe_in", (dim + 1) * count)
    if out is None:
        out = empty((batch, dim + 1), lwe_in.device)
    _expect(out, "lwe_out", batch * (dim + 1))
    _check(lib().rosetta_lwe_sum_groups(_dev(lwe_in, "lwe_in"), c0, _dev(out, "lwe_out"), batch,
                                        count, dim, _stream(stream)))
    return out


def lwe_combine(a, alpha: int, b=None, beta: int = 0, c=None, gamma: int = 0, out=None,
                stream=None):
    """out = alpha a + beta b + gamma c mod p, word by word (b, c optional)."""
    words = _words(a)
    for t, name in ((b, "b"), (c, "c")):
        if t is not None:
            _expect(t, name, words)
    out = empty(a.shape, a.device) if out is None else out
    _expect(out, "out", words)
    _check(lib().rosetta_lwe_combine(_dev(a, "a"), alpha, None if b is None else _dev(b, "b"),
                                     beta, None if c is None else _dev(c, "c"), gamma,
                                     _dev(out, "out"), words, _stream(stream)))
    return out


def autk_words(params, level: int) -> int:
    return lib().rosetta_autk_words(C.byref(_params(params)), level)


def autk_prepare(autk_std, params, level: int, out=None, stream=None):
    p = _params(params)
    _expect(autk_std, "autk_std", autk_words(p, level))
    if out is None:
        out = empty(autk_words(p, level), autk_std.device)
    _expect(out, "autk_dev", autk_words(p, level))
    _check(lib().rosetta_autk_prepare(_dev(autk_std, "autk_std"), _dev(out, "autk_dev"),
                                      C.byref(p), level, _stream(stream)))
    return out


def trace(glwe_in, autk_dev, params, level: int, base_log: int, out=None, stream=None):
    p = _params(params)
    batch = _batch_of(glwe_in, "glwe_in", 2 * p.N)
    _expect(autk_dev, "autk_dev", autk_words(p, level))
    if out is None:
        out = empty((batch, 2 * p.N), glwe_in.device)
    _expect(out, "glwe_out", batch * 2 * p.N)
    _check(lib().rosetta_trace(_dev(glwe_in, "glwe_in"), _dev(autk_dev, "autk_dev"),
                               _dev(out, "glwe_out"), batch, C.byref(p), level, base_log,
                               _stream(stream)))
    return out


def plain_prepare(plain, N: int, out=None, stream=None):
    count = _batch_of(plain, "plain", N)
    out = empty(plain.shape, plain.device) if out is None else out
    _expect(out, "plain_prep", count * N)
    _check(lib().rosetta_plain_prepare(_dev(plain, "plain"), _dev(out, "plain_prep"), count, N,
                                       _stream(stream)))
    return out


def glwe_mul_plain(glwe_in, pa_prep, pb, N: int, out=None, stream=None):
    """out[q][s] = pa_s * glwe_in[q] + (0, pb_s); pb may be None."""
    batch = _batch_of(glwe_in, "glwe_in", 2 * N)
    npoly = _batch_of(pa_prep, "pa_prep", N)
    if pb is not None:
        _expect(pb, "pb", npoly * N)
    if out is None:
        out = empty((batch, npoly, 2 * N), glwe_in.device)
    _expect(out, "glwe_out", batch * npoly * 2 * N)
    _check(lib().rosetta_glwe_mul_plain(_dev(glwe_in, "glwe_in"), _dev(pa_prep, "pa_prep"),
                                        None if pb is None else _dev(pb, "pb"),
                                        _dev(out, "glwe_out"), batch, npoly, N, _stream(stream)))
    return out


def _exps(exps, count):
    if exps is None:
        return None, None
    e = np.ascontiguousarray(exps, dtype=np.uint32)
    if e.size != count:
        raise ValueError("need one exponent per ciphertext")
    return e, _np_ptr(e)


def glwe_recombine(glwe_in, count: int, N: int, exps=None, out=None, stream=None):
    """out[q] = sum_s X^(exps[s]) glwe_in[q][s] (exps None: X^s)."""
    batch = _batch_of(glwe_in, "glwe_in", 2 * N * count)
    if out is None:
        out = empty((batch, 2 * N), glwe_in.device)
    _expect(out, "glwe_out", batch * 2 * N)
    e, ep = _exps(exps, count)
    _check(lib().rosetta_glwe_recombine(_dev(glwe_in, "glwe_in"), ep, _dev(out, "glwe_out"),
                                        batch, count, N, _stream(stream)))
    return out


def glwe_monomial_mul(glwe_in, exps, N: int, out=None, stream=None):
    """out[q][s] = X^(exps[s]) glwe_in[q]."""
    batch = _batch_of(glwe_in, "glwe_in", 2 * N)
    e, ep = _exps(exps, len(exps))
    if out is None:
        out = empty((batch, e.size, 2 * N), glwe_in.device)
    _expect(out, "glwe_out", batch * e.size * 2 * N)
    _check(lib().rosetta_glwe_monomial_mul(_dev(glwe_in, "glwe_in"), ep, _dev(out, "glwe_out"),
                                           batch, e.size, N, _stream(stream)))
    return out


def sample_extract(glwe_in, N: int, out=None, stream=None):
    batch = _batch_of(glwe_in, "glwe_in", 2 * N)
    if out is None:
        out = empty((batch, N + 1), glwe_in.device)
    _expect(out, "big_out", batch * (N + 1))
    _check(lib().rosetta_sample_extract(_dev(glwe_in, "glwe_in"), _dev(out, "big_out"), batch, N,
                                        _stream(stream)))
    return out


# --------------------------------------------------------------------------
# the clear side: 8-bit layers and the vocabulary loss (device)
# --------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _types():
    torch = _torch()
    return {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _type(dtype, name: str) -> int:
    code = _types().get(dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, not {dtype}")
    return code


@functools.lru_cache(maxsize=None)
def _tensor_class():
    return _torch().Tensor


def _misplaced(t, name: str, device):
    """Raises for a tensor that lies on no ROCm device (TypeError) or on another one than
    the call's (its index; ValueError)."""
    if t.get_device() < 0:
        raise TypeError(f"{name} must be a torch tensor on a ROCm device")
    raise ValueError(f"{name} lies on device {t.get_device()}, the call runs on device {device}")


def _mat(t, name: str, dtype=None, shape=None, device=None):
    """(address, row stride, rows, columns) of a device matrix with contiguous
    rows; a vector is one row.  TypeError for the wrong kind of tensor,
    ValueError for the wrong size or device, before any library call."""
    if not isinstance(t, _tensor_class()):
        raise TypeError(f"{name} must be a torch tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    size, strides = t.shape, t.stride()
    if len(size) == 2:
        rows, cols = size
        stride = strides[0] if rows > 1 else cols
    elif len(size) == 1:
        rows, cols, stride = 1, size[0], size[0]
    else:
        raise ValueError(f"{name} must be a matrix or one row, not {tuple(size)}")
    if shape is not None and (rows != shape[0] or cols != shape[1]):
        raise ValueError(f"{name} is {rows} x {cols}, the call needs {shape[0]} x {shape[1]}")
    at = t.get_device()
    if at < 0 or (device is not None and at != device):
        _misplaced(t, name, device)
    if cols > 1 and strides[-1] != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    return t.data_ptr(), stride, rows, cols


def _vec(t, name: str, dtype, count: int, device) -> int:
    """Address of a contiguous device vector of `count` elements."""
    if not isinstance(t, _tensor_class()) or t.dtype != dtype:
        raise TypeError(f"{name} must be a torch tensor of {dtype}")
    if t.numel() != count:
        _expect(t, name, count)
    if t.get_device() != device:
        _misplaced(t, name, device)
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t.data_ptr()


def _made(out, name: str, shape, dtype, like):
    """`out` checked, or a new tensor of that shape and type: (tensor, address,
    row stride)."""
    if out is None:
        out = like.new_empty(shape, dtype=dtype)
        return out, out.data_ptr(), shape[1]
    return out, *_mat(out, name, dtype, shape, like.get_device())[:2]


def _weight(weight, dtype, code: int, dim: int, device):
    """(address, type) of a norm's weight, of x's type or float32; None is ones."""
    if weight is None:
        return None, code
    if not isinstance(weight, _tensor_class()):
        raise TypeError("weight must be a torch tensor")
    if weight.dtype != dtype and weight.dtype != _torch().float32:
        raise TypeError(f"weight must be {dtype} or float32, not {weight.dtype}")
    return _vec(weight, "weight", weight.dtype, dim, device), _type(weight.dtype, "weight")


def _stream_of(t, stream) -> int:
    """The stream given, or the current one of the tensor's device (read as a plain
    number: a Stream object takes 2.6 us to make, as long as the launch)."""
    if stream is not None:
        if stream.device_index != t.get_device():
            raise ValueError(f"the stream is of device {stream.device_index}, the tensors lie on "
                             f"device {t.get_device()}")
        return stream.cuda_stream
    return _torch()._C._cuda_getCurrentRawStream(t.device.index)


def _scratch(workspace, need: int, like):
    """`workspace` checked, or a new one: (address, bytes, tensor)."""
    if workspace is None:
        workspace = like.new_empty(need, dtype=_torch().uint8)
    if not isinstance(workspace, _tensor_class()):
        raise TypeError("workspace must be a torch tensor")
    have = workspace.numel() * workspace.element_size()
    if have < need:
        raise ValueError(f"workspace holds {have} bytes, the call needs {need}")
    if workspace.get_device() != like.get_device():
        _misplaced(workspace, "workspace", like.get_device())
    if not workspace.is_contiguous():
        raise TypeError("workspace must be contiguous")
    return workspace.data_ptr(), have, workspace


def _on_its_stream(call):
    """With a stream given, what `call` allocates (outputs, workspaces) belongs to
    that stream, so that no memory is reused while its work still runs.  Without one,
    the device of its first tensor is the current one while it runs."""
    names = list(inspect.signature(call).parameters)
    at = names.index("stream")  # (the last one)

    @functools.wraps(call)
    def on_stream(*args, stream=None, **kw):
        if len(args) > at:
            if stream is not None or len(args) > at + 1:
                raise TypeError(f"{call.__name__} takes {at + 1} arguments, stream the last of them")
            stream, args = args[at], args[:at]
        torch = _torch()
        if stream is None:
            first = args[0] if args else kw.get(names[0])
            if isinstance(first, KVCache):
                first = first.k
            device = first.get_device() if isinstance(first, _tensor_class()) else -1
            if device < 0 or device == torch._C._cuda_getDevice():
                return call(*args, **kw)
            with torch.cuda.device(device):
                return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, stream=stream, **kw)
    return on_stream


class NormQ8(NamedTuple):
    """What rms_norm_q8 returns: the 8-bit rows and their scales, h = x +
    residual (None without a residual), 1 / rms, and y where it was asked for."""
    q: object
    scale: object
    h: object
    inv_rms: object
    y: object


def _norm(x, weight, eps, residual, h, y, want_y, q, want_q, stream):
    torch = _torch()
    xp, xs, rows, dim = _mat(x, "x")
    dtype = x.dtype
    code, on = _type(dtype, "x"), x.get_device()
    rp, rs = None, dim
    if residual is not None:
        rp, rs = _mat(residual, "residual", dtype, (rows, dim), on)[:2]
    wp, wt = _weight(weight, dtype, code, dim, on)
    hp, hs, yp, ys, qp, qs, scale, sp = None, dim, None, dim, None, dim, None, None
    if h is not None or residual is not None:
        h, hp, hs = _made(h, "h", (rows, dim), dtype, x)
    if want_y:
        y, yp, ys = _made(y, "y", (rows, dim), dtype, x)
    if want_q:
        q, qp, qs = _made(q, "q", (rows, dim), torch.int8, x)
        scale = x.new_empty(rows, dtype=torch.float32)
        sp = scale.data_ptr()
    inv_rms = x.new_empty(rows, dtype=torch.float32)
    _check(lib().rosetta_rms_norm(xp, xs, rp, rs, wp, wt, code, rows, dim, eps, hp, hs, yp, ys, qp,
                                  qs, sp, inv_rms.data_ptr(), _stream_of(x, stream)))
    return q, scale, h, inv_rms, y


@_on_its_stream
def rms_norm_q8(x, weight, eps: float, residual=None, h=None, want_y: bool = False, q=None,
                stream=None) -> NormQ8:
    """RMS norm of x + residual ([rows][dim], float32, bfloat16 or float16) to
    8 bits with a scale per row.  weight [dim] (None: ones) has x's type or
    float32.  h may be x or residual, which it then replaces."""
    return NormQ8(*_norm(x, weight, eps, residual, h, None, want_y, q, True, stream))


@_on_its_stream
def rms_norm(x, weight, eps: float, residual=None, h=None, y=None, stream=None):
    """The same without the 8 bits: (y, h, inv_rms)."""
    _, _, h, inv_rms, y = _norm(x, weight, eps, residual, h, y, True, None, False, stream)
    return y, h, inv_rms


@_on_its_stream
def rms_norm_backward(gy, h, weight, inv_rms, gh=None, gx=None, want_gweight: bool = True,
                      workspace=None, stream=None):
    """(gx, gweight) from gy, the gradient of y (or, passed straight through the
    rounding, of the 8-bit values), and gh, that of h.  h is rms_norm's h, or its
    x where there was no residual.  gx may be gy or gh; gweight is float32."""
    torch = _torch()
    yp, ys, rows, dim = _mat(gy, "gy")
    dtype = gy.dtype
    code, on = _type(dtype, "gy"), gy.get_device()
    hp, hs = _mat(h, "h", dtype, (rows, dim), on)[:2]
    gp, gs = (None, dim) if gh is None else _mat(gh, "gh", dtype, (rows, dim), on)[:2]
    wp, wt = _weight(weight, dtype, code, dim, on)
    ip = _vec(inv_rms, "inv_rms", torch.float32, rows, on)
    gx, xp, xs = _made(gx, "gx", (rows, dim), dtype, gy)
    gweight, gwp, wsp, wsb = None, None, None, 0
    if want_gweight:
        gweight = gy.new_empty(dim, dtype=torch.float32)
        gwp = gweight.data_ptr()
        wsp, wsb, workspace = _scratch(
            workspace, lib().rosetta_rms_norm_backward_workspace_bytes(rows, dim), gy)
    _check(lib().rosetta_rms_norm_backward(yp, ys, gp, gs, hp, hs, wp, wt, ip, code, rows, dim, xp,
                                           xs, gwp, wsp, wsb, _stream_of(gy, stream)))
    return gx, gweight


@_on_its_stream
def quantize_rows(x, q=None, scale=None, stream=None):
    """Rows to 8 bits: (q, scale)."""
    torch = _torch()
    xp, xs, rows, dim = _mat(x, "x")
    code = _type(x.dtype, "x")
    q, qp, qs = _made(q, "q", (rows, dim), torch.int8, x)
    if scale is None:
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(lib().rosetta_quantize_rows(xp, xs, code, rows, dim, qp, qs,
                                       _vec(scale, "scale", torch.float32, rows, x.get_device()),
                                       _stream_of(x, stream)))
    return q, scale


@_on_its_stream
def dequantize_rows(q, scale, dtype, out=None, stream=None):
    """The values that 8-bit rows stand for."""
    torch = _torch()
    qp, qs, rows, dim = _mat(q, "q", torch.int8)
    sp = _vec(scale, "scale", torch.float32, rows, q.get_device())
    out, op, os_ = _made(out, "out", (rows, dim), dtype, q)
    _check(lib().rosetta_dequantize_rows(qp, qs, sp, _type(dtype, "dtype"), rows, dim, op, os_,
                                         _stream_of(q, stream)))
    return out


@_on_its_stream
def q8_matmul(a, a_scale, b, b_scale, bias=None, out_dtype=None, out=None, workspace=None,
              stream=None):
    """a [m][k] times b [n][k] (a row per channel), both int8, with a scale per
    row of each: [m][n] of out_dtype (default bfloat16)."""
    torch = _torch()
    if out_dtype is None:
        out_dtype = getattr(out, "dtype", torch.bfloat16)
    ap, as_, m, k = _mat(a, "a", torch.int8)
    on = a.get_device()
    bp, bs, n, kb = _mat(b, "b", torch.int8, device=on)
    if kb != k:
        raise ValueError(f"b is {n} x {kb}, the call needs rows of {k}")
    sa = _vec(a_scale, "a_scale", torch.float32, m, on)
    sb = _vec(b_scale, "b_scale", torch.float32, n, on)
    bi = None if bias is None else _vec(bias, "bias", torch.float32, n, on)
    out, op, os_ = _made(out, "out", (m, n), out_dtype, a)
    need = lib().rosetta_q8_matmul_workspace_bytes(m, n, k)
    wp, wb = None, 0
    if need:
        wp, wb, workspace = _scratch(workspace, need, a)
    _check(lib().rosetta_q8_matmul(ap, as_, sa, bp, bs, sb, bi, op, os_,
                                   _type(out_dtype, "out_dtype"), m, n, k, wp, wb,
                                   _stream_of(a, stream)))
    return out


@_on_its_stream
def cross_entropy(h, w, targets, ignore_index: int = -100, workspace=None, stream=None):
    """(loss, lse) per row, float32, of hidden states h [rows][dim] under head
    weights w [vocab][dim] (bfloat16 or float16); targets int64."""
    torch = _torch()
    hp, hs, rows, dim = _mat(h, "h")
    dt, on = _type(h.dtype, "h"), h.get_device()
    wp, ws, vocab, dw = _mat(w, "w", h.dtype, device=on)
    if dw != dim:
        raise ValueError(f"w is {vocab} x {dw}, the call needs rows of {dim}")
    tp = _vec(targets, "targets", torch.int64, rows, on)
    loss, lse = (h.new_empty(rows, dtype=torch.float32) for _ in range(2))
    sp, sb, workspace = _scratch(
        workspace, lib().rosetta_cross_entropy_workspace_bytes(rows, dim, vocab), h)
    _check(lib().rosetta_cross_entropy(hp, hs, wp, ws, dt, tp, ignore_index, rows, dim, vocab,
                                       loss.data_ptr(), lse.data_ptr(), sp, sb,
                                       _stream_of(h, stream)))
    return loss, lse


@_on_its_stream
def cross_entropy_backward(h, w, targets, lse, gloss, ignore_index: int = -100,
                           want_gh: bool = True, want_gw: bool = True, gh=None, gw=None,
                           workspace=None, stream=None):
    """(gh, gw) from gloss [rows], the gradient of each row's loss, and lse as
    cross_entropy returned it."""
    torch = _torch()
    hp, hs, rows, dim = _mat(h, "h")
    dt, on = _type(h.dtype, "h"), h.get_device()
    wp, ws, vocab, dw = _mat(w, "w", h.dtype, device=on)
    if dw != dim:
        raise ValueError(f"w is {vocab} x {dw}, the call needs rows of {dim}")
    tp = _vec(targets, "targets", torch.int64, rows, on)
    ep = _vec(lse, "lse", torch.float32, rows, on)
    gp = _vec(gloss, "gloss", torch.float32, rows, on)
    gh, ghp, ghs = _made(gh, "gh", (rows, dim), h.dtype, h) if want_gh else (None, None, dim)
    gw, gwp, gws = _made(gw, "gw", (vocab, dim), w.dtype, w) if want_gw else (None, None, dim)
    sp, sb, workspace = _scratch(
        workspace, lib().rosetta_cross_entropy_backward_workspace_bytes(rows, dim, vocab), h)
    _check(lib().rosetta_cross_entropy_backward(hp, hs, wp, ws, dt, tp, ignore_index, ep, gp, rows,
                                                dim, vocab, ghp, ghs, gwp, gws, sp, sb,
                                                _stream_of(h, stream)))
    return gh, gw


# --------------------------------------------------------------------------
# the clear side, decoding: an 8-bit cache and drafted tokens (device)
# --------------------------------------------------------------------------

class KVCache(NamedTuple):
    """Keys and values in 8 bits: k and v int8 [pages][kv_heads][page][dim] (views
    with any strides that are multiples of 16, the last dimension contiguous), and
    their scales float32 [pages][kv_heads][page], contiguous over a page."""
    k: object
    v: object
    k_scale: object
    v_scale: object


def kv_cache(pages: int, kv_heads: int, page: int, dim: int, device="cuda") -> KVCache:
    """A cache of zeros.  page: a power of two from 16 on; dim: a multiple of 16 up
    to 256."""
    torch = _torch()
    shape = (pages, kv_heads, page, dim)
    k, v = (torch.zeros(shape, dtype=torch.int8, device=device) for _ in range(2))
    ks, vs = (torch.zeros(shape[:3], dtype=torch.float32, device=device) for _ in range(2))
    return KVCache(k, v, ks, vs)


def _tensor(t, name: str, dtype, dims: int, device):
    """A device tensor's (shape, strides), of `dims` dimensions, the last contiguous."""
    if not isinstance(t, _tensor_class()) or (dtype is not None and t.dtype is not dtype):
        raise TypeError(f"{name} must be a torch tensor" + (f" of {dtype}" if dtype else ""))
    size, strides = t.shape, t.stride()
    if len(size) != dims:
        raise ValueError(f"{name} must have {dims} dimensions, not {tuple(size)}")
    at = t.get_device()
    if at < 0 or (device is not None and at != device):
        _misplaced(t, name, device)
    if strides[-1] != 1 and size[-1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return size, strides


def _cache(cache):
    """(struct, device) of a cache; strides over one element alone are any."""
    if not isinstance(cache, KVCache):
        raise TypeError("cache must be a KVCache")
    torch = _torch()
    k, v, ks, vs = cache
    size, st = _tensor(k, "cache.k", torch.int8, 4, None)
    on = k.get_device()
    ssize, ss = _tensor(ks, "cache.k_scale", torch.float32, 3, on)
    if not (isinstance(v, _tensor_class()) and v.dtype is torch.int8 and v.get_device() == on and
            v.shape == size and v.stride() == st):
        _tensor(v, "cache.v", torch.int8, 4, on)
        raise ValueError("cache.v must have the shape and strides of cache.k")
    if not (isinstance(vs, _tensor_class()) and vs.dtype is torch.float32 and
            vs.get_device() == on and vs.shape == ssize and vs.stride() == ss):
        _tensor(vs, "cache.v_scale", torch.float32, 3, on)
        raise ValueError("cache.v_scale must have the shape and strides of cache.k_scale")
    if ssize != size[:3]:
        raise ValueError(f"cache.k_scale is {tuple(ssize)}, the call needs {tuple(size[:3])}")
    pages, heads, page, dim = size
    if pages > 1 and heads > 1 and page > 1:
        return CacheStruct(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, heads,
                           page, dim, st[0], st[1], st[2], ss[0], ss[1]), on
    return CacheStruct(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, heads, page,
                       dim, st[0] if pages > 1 else 0, st[1] if heads > 1 else 0,
                       st[2] if page > 1 else 0, ss[0] if pages > 1 else 0,
                       ss[1] if heads > 1 else 0), on


def _rows(table, starts, lens, rows: int, device):
    torch = _torch()
    size, st = _tensor(table, "table", torch.int32, 2, device)
    batch = size[0]
    return RowsStruct(table.data_ptr(), st[0] if batch > 1 else size[1], size[1],
                      _vec(starts, "starts", torch.int32, batch + 1, device),
                      _vec(lens, "lens", torch.int32, batch, device), batch, rows)


def _heads(t, name: str, dtype, shape, device):
    """(address, row stride, head stride) of [rows][heads][dim]."""
    size, st = _tensor(t, name, dtype, 3, device)
    if tuple(size) != tuple(shape):
        raise ValueError(f"{name} is {tuple(size)}, the call needs {tuple(shape)}")
    return (t.data_ptr(), st[0] if size[0] > 1 else size[1] * size[2],
            st[1] if size[1] > 1 else size[2])


def _made_heads(out, name: str, dtype, shape, like):
    """`out` checked, or a new tensor: (tensor, address, row stride, head stride)."""
    if out is None:
        out = like.new_empty(shape, dtype=dtype)
        return out, out.data_ptr(), shape[1] * shape[2], shape[2]
    return out, *_heads(out, name, dtype, shape, like.get_device())


@_on_its_stream
def kv_write(k, v, cache, table, starts, lens, stream=None):
    """Keys and values [rows][kv_heads][dim] (float32, bfloat16 or float16) to the
    cache in 8 bits, a scale per row and head.  The batch is packed: sequence b has
    rows starts[b] .. starts[b + 1], the last of its lens[b] positions; position t
    lies at place t % page of page table[b][t // page] (all int32)."""
    c, on = _cache(cache)
    dtype = getattr(k, "dtype", None)
    rows = k.shape[0] if isinstance(k, _tensor_class()) and k.dim() == 3 else 0
    shape = (rows, c.kv_heads, c.dim)
    ka = _heads(k, "k", dtype, shape, on)
    va = _heads(v, "v", dtype, shape, on)
    r = _rows(table, starts, lens, rows, on)
    _check(lib().rosetta_kv_write(*ka, *va, _type(dtype, "k"), c, r, _stream_of(cache.k, stream)))


@_on_its_stream
def kv_read(cache, table, starts, lens, rows: int, dtype, k=None, v=None, stream=None):
    """(k, v) [rows][kv_heads][dim]: the values that the rows' positions hold.  Rows of
    no sequence are not written."""
    c, on = _cache(cache)
    shape = (rows, c.kv_heads, c.dim)
    code = _type(dtype, "dtype")
    r = _rows(table, starts, lens, rows, on)
    k, kp, ks, kh = _made_heads(k, "k", dtype, shape, cache.k)
    v, vp, vs, vh = _made_heads(v, "v", dtype, shape, cache.k)
    _check(lib().rosetta_kv_read(c, r, code, kp, ks, kh, vp, vs, vh, _stream_of(cache.k, stream)))
    return k, v


@_on_its_stream
def kv_keep(cache, table, starts, lens, path, count, stream=None):
    """Of each sequence's rows (drafted tokens, say) the accepted ones moved together:
    row i's position takes what row path[starts[b] + i]'s holds, i < count[b].  Returns
    the new lens, lens[b] - n + count[b].  path and count as verify_drafts gives them."""
    torch = _torch()
    c, on = _cache(cache)
    rows = path.numel() if isinstance(path, _tensor_class()) else 0
    pp = _vec(path, "path", torch.int32, rows, on)
    r = _rows(table, starts, lens, rows, on)
    cp = _vec(count, "count", torch.int32, r.batch, on)
    out = lens.new_empty(r.batch, dtype=torch.int32)
    _check(lib().rosetta_kv_keep(c, r, pp, cp, out.data_ptr(), _stream_of(cache.k, stream)))
    return out


@_on_its_stream
def tree_masks(parents, starts, max_rows: int, stream=None):
    """int64 [rows][ceil(max_rows / 64)]: bit j of a row says whether it is its
    sequence's row j or has it among its ancestors.  parents int32 [rows]: the place of
    each row's parent among its sequence's rows, -1 for none.  (Zeros for rows of no
    sequence.)"""
    torch = _torch()
    rows = parents.numel() if isinstance(parents, _tensor_class()) else 0
    on = parents.get_device() if isinstance(parents, _tensor_class()) else -1
    if max_rows < 1:
        raise ValueError("max_rows must be at least 1")
    if on < 0 and isinstance(parents, _tensor_class()):
        _misplaced(parents, "parents", None)
    pp = _vec(parents, "parents", torch.int32, rows, on)
    batch = starts.numel() - 1 if isinstance(starts, _tensor_class()) else 0
    if batch < 0:
        raise ValueError("starts holds nothing")
    sp = _vec(starts, "starts", torch.int32, batch + 1, on)
    words = -(-max_rows // 64)
    masks = parents.new_empty((rows, words), dtype=torch.int64)
    if batch == 0:  # (the library then does nothing)
        masks.zero_()
    _check(lib().rosetta_tree_masks(pp, sp, batch, rows, words, masks.data_ptr(),
                                    _stream_of(parents, stream)))
    return masks


@_on_its_stream
def kv_attention(q, cache, table, starts, lens, masks=None, scale: float = None,
                 max_rows: int = None, out=None, want_lse: bool = True, workspace=None,
                 stream=None):
    """(out, lse) of queries q [rows][heads][dim] (bfloat16 or float16) over the cache,
    the rows' own entries among it: row i of a sequence sees the positions before its
    rows, and its rows up to i, or with `masks` (int64 [rows][words], as tree_masks
    makes them) those whose bit is set.  A row that sees nothing gives zeros and -inf.
    scale: 1 / sqrt(dim) where not given.  max_rows: the most rows of any sequence (where
    not given all rows, or with masks as many as they have bits for; a batch of single
    tokens that names 1 leaves less to launch).  A table that is longer than the longest
    sequence (a narrower view of it will do) is cut in more parts than there is to do.  lse
    is float32 [rows][heads], or None.  Rows of no sequence, or behind max_rows, are not
    written."""
    torch = _torch()
    c, on = _cache(cache)
    if not isinstance(q, _tensor_class()):
        raise TypeError("q must be a torch tensor")
    dtype = q.dtype
    code = _type(dtype, "q")
    rows, heads = q.shape[:2] if q.dim() == 3 else (0, 0)
    shape = (rows, heads, c.dim)
    qa = _heads(q, "q", dtype, shape, on)
    r = _rows(table, starts, lens, rows, on)
    mp, words = None, 0
    if masks is not None:
        size, _ = _tensor(masks, "masks", torch.int64, 2, on)
        words = size[1]
        mp = _vec(masks, "masks", torch.int64, rows * words, on)
    if max_rows is None:
        max_rows = min(rows, 64 * max(words, 1)) if masks is not None else rows
    max_rows = min(max_rows, rows)
    if max_rows < 0:
        raise ValueError("max_rows must not be negative")
    if scale is None:
        scale = c.dim ** -0.5
    L = lib()
    need = L.rosetta_kv_attention_workspace_bytes(heads, c.kv_heads, c.dim, r.batch, rows, max_rows,
                                                  r.table_len * c.page)
    wp, wb = None, 0
    if need:
        wp, wb, workspace = _scratch(workspace, need, q)
    out, op, os_, oh = _made_heads(out, "out", dtype, shape, q)
    lse = q.new_empty((rows, heads), dtype=torch.float32) if want_lse else None
    _check(L.rosetta_kv_attention(*qa, code, heads, c, r, max_rows, mp, words, scale, op, os_, oh,
                                  lse.data_ptr() if want_lse else None, wp, wb,
                                  _stream_of(q, stream)))
    return out, lse


@_on_its_stream
def verify_drafts(p, q, drafts, u, starts, parents=None, workspace=None, stream=None):
    """(tokens, path, count): drafted tokens verified against the target's probabilities.
    p, q [rows][vocab] (of one type): the target's after each row, and those that the
    row's children were drawn from (anything, where it has none); drafts int64 [rows] the
    tokens, u float32 [rows] numbers of [0, 1).  A sequence's rows are the nodes of a tree
    whose node 0 is the last certain token; parents int32 [rows] as for tree_masks (None:
    each follows the one before).  count int32 [batch]: how many nodes are kept, node 0
    among them, and how many new tokens there are; path int32 and tokens int64 [rows]:
    those, from each sequence's first row on, -1 behind, and in rows of no sequence."""
    torch = _torch()
    pp, ps, rows, vocab = _mat(p, "p")
    dtype, on = p.dtype, p.get_device()
    qp, qs = _mat(q, "q", dtype, (rows, vocab), on)[:2]
    dp = _vec(drafts, "drafts", torch.int64, rows, on)
    up = _vec(u, "u", torch.float32, rows, on)
    ap = None if parents is None else _vec(parents, "parents", torch.int32, rows, on)
    batch = starts.numel() - 1 if isinstance(starts, _tensor_class()) else 0
    if batch < 0:
        raise ValueError("starts holds nothing")
    sp = _vec(starts, "starts", torch.int32, batch + 1, on)
    L = lib()
    need = L.rosetta_verify_drafts_workspace_bytes(batch, vocab)
    wp, wb = None, 0
    if need:
        wp, wb, workspace = _scratch(workspace, need, p)
    tokens = drafts.new_empty(rows)
    path = starts.new_empty(rows)
    count = starts.new_empty(batch)
    if batch == 0:  # (the library then does nothing)
        tokens.fill_(-1)
        path.fill_(-1)
    _check(L.rosetta_verify_drafts(pp, ps, qp, qs, _type(dtype, "p"), dp, ap, up, sp, batch, rows,
                                   vocab, tokens.data_ptr(), path.data_ptr(), count.data_ptr(), wp,
                                   wb, _stream_of(p, stream)))
    return tokens, path, count


# --------------------------------------------------------------------------
# host helpers (numpy)
# --------------------------------------------------------------------------

def _np_ptr(a: np.ndarray) -> int:
    return a.ctypes.data


def keygen(seed: int, params, sigma_lwe: float, sigma_glwe: float) -> dict:
    p = _params(params)
    keys = dict(lwe_key=np.zeros(p.n, np.uint64), glwe_key=np.zeros(p.N, np.uint64),
                bsk=np.zeros(bsk_words(p), np.uint64), ksk=np.zeros(ksk_words(p), np.uint64))
    _check(lib().rosetta_keygen(seed, C.byref(p), sigma_lwe, sigma_glwe,
                                _np_ptr(keys["lwe_key"]), _np_ptr(keys["glwe_key"]),
                                _np_ptr(keys["bsk"]), _np_ptr(keys["ksk"])))
    return keys


def lwe_encrypt(seed: int, params, sigma: float, key: np.ndarray, msgs) -> np.ndarray:
    p = _params(params)
    key = np.ascontiguousarray(key, np.uint64)
    msgs = np.ascontiguousarray(msgs, np.uint32)
    dim = key.shape[0]
    out = np.zeros((msgs.shape[0], dim + 1), np.uint64)
    _check(lib().rosetta_lwe_encrypt(seed, C.byref(p), sigma, _np_ptr(key), dim, _np_ptr(msgs),
                                     msgs.shape[0], _np_ptr(out)))
    return out


def lwe_encrypt_plain(seed: int, params, sigma: float, key: np.ndarray, plain) -> np.ndarray:
    """LWE encryptions of plaintexts already in Z_p (params unused beyond
    symmetry with lwe_encrypt)."""
    key = np.ascontiguousarray(key, np.uint64)
    plain = np.ascontiguousarray(plain, np.uint64)
    dim = key.shape[0]
    out = np.zeros((plain.shape[0], dim + 1), np.uint64)
    _check(lib().rosetta_lwe_encrypt_plain(seed, sigma, _np_ptr(key), dim, _np_ptr(plain),
                                           plain.shape[0], _np_ptr(out)))
    return out


def lwe_decrypt(params, key: np.ndarray, cts: np.ndarray) -> np.ndarray:
    p = _params(params)
    key = np.ascontiguousarray(key, np.uint64)
    dim = key.shape[0]
    cts = np.ascontiguousarray(cts, np.uint64).reshape(-1, dim + 1)
    out = np.zeros(cts.shape[0], np.uint32)
    _check(lib().rosetta_lwe_decrypt(C.byref(p), _np_ptr(key), dim, _np_ptr(cts), cts.shape[0],
                                     _np_ptr(out)))
    return out


def lut_build(params, table) -> np.ndarray:
    p = _params(params)
    table = np.ascontiguousarray(table, np.uint32)
    if table.shape[0] != p.M:
        raise ValueError(f"table must have {p.M} entries")
    v = np.zeros(p.N, np.uint64)
    _check(lib().rosetta_lut_build(C.byref(p), _np_ptr(table), _np_ptr(v)))
    return v


def glwe_encrypt(seed: int, params, sigma: float, glwe_key: np.ndarray, msgs) -> np.ndarray:
    p = _params(params)
    key = np.ascontiguousarray(glwe_key, np.uint64)
    msgs = np.ascontiguousarray(msgs, np.uint64).reshape(-1, p.N)
    out = np.zeros((msgs.shape[0], 2 * p.N), np.uint64)
    _check(lib().rosetta_glwe_encrypt(seed, C.byref(p), sigma, _np_ptr(key), _np_ptr(msgs),
                                      msgs.shape[0], _np_ptr(out)))
    return out


def glwe_phase(params, glwe_key: np.ndarray, cts) -> np.ndarray:
    p = _params(params)
    key = np.ascontiguousarray(glwe_key, np.uint64)
    cts = np.ascontiguousarray(cts, np.uint64).reshape(-1, 2 * p.N)
    out = np.zeros((cts.shape[0], p.N), np.uint64)
    _check(lib().rosetta_glwe_phase(C.byref(p), _np_ptr(key), _np_ptr(cts), cts.shape[0],
                                    _np_ptr(out)))
    return out


def autk_keygen(seed: int, params, level: int, base_log: int, sigma: float,
                glwe_key: np.ndarray) -> np.ndarray:
    p = _params(params)
    key = np.ascontiguousarray(glwe_key, np.uint64)
    out = np.zeros(autk_words(p, level), np.uint64)
    _check(lib().rosetta_autk_keygen(seed, C.byref(p), level, base_log, sigma, _np_ptr(key),
                                     _np_ptr(out)))
    return out


# segmented LUT (host) --------------------------------------------------------

def _f64(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.float64)


def seglut_boundaries(lo: float, hi: float, nseg: int, spacing: str) -> np.ndarray:
    tau = np.zeros(nseg + 1, np.float64)
    _check(lib().rosetta_seglut_boundaries(lo, hi, nseg, SPACINGS[spacing], _np_ptr(tau)))
    return tau


def seglut_build(function: str, tau, nbr: int, fit: str = "linear"):
    tau = _f64(tau)
    nseg = tau.shape[0] - 1
    a = np.zeros((nseg, nbr), np.float64)
    b = np.zeros((nseg, nbr), np.float64)
    _check(lib().rosetta_seglut_build(FUNCTIONS[function], _np_ptr(tau), nseg, nbr, FITS[fit],
                                      _np_ptr(a), _np_ptr(b)))
    return a, b


def seglut_protocol_polys(tau, nbr: int):
    tau = _f64(tau)
    nseg = tau.shape[0] - 1
    p = np.zeros(nseg, np.float64)
    q = np.zeros(nseg, np.float64)
    _check(lib().rosetta_seglut_protocol_polys(_np_ptr(tau), nseg, nbr, _np_ptr(p), _np_ptr(q)))
    return p, q


def _offsets(index_offset, count):
    if index_offset is None:
        return None, None
    off = np.ascontiguousarray(index_offset, dtype=np.int32)
    if off.size != count:
        raise ValueError("index_offset must have one entry per input")
    return off, _np_ptr(off)


def seglut_eval(tau, a, b, x, index_offset=None) -> np.ndarray:
    tau, a, b, x = _f64(tau), _f64(a), _f64(b), _f64(x)
    y = np.zeros_like(x)
    off, off_p = _offsets(index_offset, x.size)
    _check(lib().rosetta_seglut_eval(_np_ptr(tau), tau.shape[0] - 1, a.shape[1], _np_ptr(a),
                                     _np_ptr(b), _np_ptr(x), off_p, x.size, _np_ptr(y)))
    return y


def seglut_precision(function: str, tau, a, b, x, index_offset=None) -> float:
    tau, a, b, x = _f64(tau), _f64(a), _f64(b), _f64(x)
    bits = np.zeros(1, np.float64)
    off, off_p = _offsets(index_offset, x.size)
    _check(lib().rosetta_seglut_precision(FUNCTIONS[function], _np_ptr(tau), tau.shape[0] - 1,
                                          a.shape[1], _np_ptr(a), _np_ptr(b), _np_ptr(x), off_p,
                                          x.size, _np_ptr(bits)))
    return float(bits[0])


def encode_fixed(v, scale_log: int) -> np.ndarray:
    v = _f64(v)
    out = np.zeros(v.shape, np.uint64)
    _check(lib().rosetta_encode_fixed(_np_ptr(v), v.size, scale_log, _np_ptr(out)))
    return out


# lookup protocol (Algorithm 1, Steps 1-3) ----------------------------------

def lookup_encode(params, lp: LookupParams, tau, a, b):
    """Host plaintext block [(4 + 2 nseg) N] and constants [nseg]."""
    p = _params(params)
    tau, a, b = _f64(tau), _f64(a), _f64(b)
    plain = np.zeros(lib().rosetta_lookup_plain_words(C.byref(p), C.byref(lp)), np.uint64)
    consts = np.zeros(lp.nseg, np.uint64)
    _check(lib().rosetta_lookup_encode(C.byref(p), C.byref(lp), _np_ptr(tau), _np_ptr(a),
                                       _np_ptr(b), _np_ptr(plain), _np_ptr(consts)))
    return plain, consts


def lookup_prepare(plain_dev, params, lp: LookupParams, out=None, stream=None):
    p = _params(params)
    _expect(plain_dev, "plain", lib().rosetta_lookup_plain_words(C.byref(p), C.byref(lp)))
    out = empty(plain_dev.shape, plain_dev.device) if out is None else out
    _expect(out, "plain_prep", _words(plain_dev))
    _check(lib().rosetta_lookup_prepare(_dev(plain_dev, "plain"), _dev(out, "plain_prep"),
                                        C.byref(p), C.byref(lp), _stream(stream)))
    return out


def lookup_workspace_bytes(params, lp: LookupParams, batch: int) -> int:
    return lib().rosetta_lookup_workspace_bytes(C.byref(_params(params)), C.byref(lp), batch)


LOOKUP_PART_CMP, LOOKUP_PART_S, LOOKUP_PART_I = 2, 3, 6


def lookup_workspace_offset(params, lp: LookupParams, batch: int, part: int) -> int:
    """Word offset of an intermediate of rosetta_lookup_eval in its workspace
    (LOOKUP_PART_CMP, LOOKUP_PART_S or LOOKUP_PART_I)."""
    off = lib().rosetta_lookup_workspace_offset(C.byref(_params(params)), C.byref(lp), batch,
                                                part)
    if off == (1 << 64) - 1:
        raise ValueError(f"unknown lookup workspace part {part}")
    return off


def lookup_eval(x_rlwe, x_cmp, bsk_dev, ksk_dev, autk_dev, plain_prep, consts, params,
                lp: LookupParams, workspace=None, out=None, stream=None):
    p = _params(params)
    batch = _batch_of(x_cmp, "x_cmp", p.n + 1)
    _expect(x_rlwe, "x_rlwe", batch * 2 * p.N)
    _expect(bsk_dev, "bsk_dev", bsk_words(p))
    _expect(ksk_dev, "ksk_dev", ksk_device_words(p))
    _expect(autk_dev, "autk_dev", autk_words(p, lp.trace_level))
    _expect(plain_prep, "plain_prep", lib().rosetta_lookup_plain_words(C.byref(p), C.byref(lp)))
    if out is None:
        out = empty((batch, 2 * p.N), x_cmp.device)
    _expect(out, "out", batch * 2 * p.N)
    if workspace is None:
        workspace = empty(lookup_workspace_bytes(p, lp, batch) // 8, x_cmp.device)
    if _words(workspace) * 8 < lookup_workspace_bytes(p, lp, batch):
        raise ValueError(f"workspace holds {_words(workspace) * 8} bytes, the call needs "
                         f"{lookup_workspace_bytes(p, lp, batch)}")
    c = np.ascontiguousarray(consts, np.uint64)
    _expect(c, "consts", lp.nseg)
    _check(lib().rosetta_lookup_eval(_dev(x_rlwe, "x_rlwe"), _dev(x_cmp, "x_cmp"),
                                     _dev(bsk_dev, "bsk"), _dev(ksk_dev, "ksk"),
                                     _dev(autk_dev, "autk"), _dev(plain_prep, "plain_prep"),
                                     _np_ptr(c), _dev(out, "out"), batch, C.byref(p),
                                     C.byref(lp), _dev(workspace, "workspace"),
                                     workspace.numel() * 8, _stream(stream)))
    return out
