"""Thin ctypes binding over the C ABI declared in ``include/dodo.h``.

Argument marshalling only: device tensors become raw pointers, host offset/length tables become
``int32`` arrays, and the current torch CUDA stream is passed along.  Every step of the path runs
in the library's kernels; there is no CPU or PyTorch fallback, and importing this module fails
loudly when ``libdodo.so`` has not been built (``python -m paper_2310_02409_b200.build``).
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import numpy as np
import torch

LIB_PATH = Path(__file__).resolve().parent / "libdodo.so"

F32, BF16 = 0, 1
FORCE_LAST = 1
ACT_IDENTITY, ACT_RELU, ACT_GELU_TANH = 0, 1, 2
TUNE_ATTEND_TARGET_BLOCKS, TUNE_DENSE_MIN_QUERIES, TUNE_DENSE_BALANCE = 1, 3, 4
DEV_WAIT_TIMEOUT, DEV_BAD_INDEX = 1, 2
Q4_GROUP = 32
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CAPACITY, ERR_CUDA = 0, -1, -2, -3, -4

# every symbol include/dodo.h declares: name -> (restype, argtypes)
_vp, _i, _u, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint32, ctypes.c_float, ctypes.c_size_t
SIGNATURES = {
    "dodo_create": (_i, [ctypes.POINTER(_vp), _i]),
    "dodo_destroy": (_i, [_vp]),
    "dodo_last_error": (ctypes.c_char_p, [_vp]),
    "dodo_reset": (_i, [_vp, _vp]),
    "dodo_device_status": (_i, [_vp, ctypes.POINTER(_i)]),
    "dodo_set_tuning": (_i, [_vp, _i, _i]),
    "dodo_cache_written": (_i, [_vp]),
    "dodo_num_nuggets": (_i, [_i, _i]),
    "dodo_score": (_i, [_vp, _vp, _i, _i, _vp, _f, _vp, _i, _vp, _vp]),
    "dodo_select": (_i, [_vp, _vp, _vp, _vp, _i, _u, _vp, _vp]),
    "dodo_score_mlp_workspace_bytes": (_sz, [_i, _i]),
    "dodo_score_mlp": (_i, [_vp, _vp, _i, _i, _vp, _vp, _vp, _f, _i, _i, _vp, _i, _vp, _vp, _sz, _vp]),
    "dodo_score_mlp_select": (_i, [_vp, _vp, _i, _i, _vp, _vp, _vp, _f, _i, _i, _vp, _vp, _i, _u, _vp, _vp, _vp, _sz, _vp]),
    "dodo_count_threshold": (_i, [_vp, _vp, _vp, _i, _f, _vp, _vp]),
    "dodo_select_threshold": (_i, [_vp, _vp, _vp, _vp, _i, _f, _vp, _vp]),
    "dodo_estimate_threshold": (_i, [_vp, _vp, _i, _i, _vp, _vp]),
    "dodo_score_select": (_i, [_vp, _vp, _i, _i, _vp, _f, _vp, _vp, _i, _u, _vp, _vp, _vp]),
    "dodo_gather_kv": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dodo_compress": (_i, [_vp, _vp, _i, _i, _vp, _f, _vp, _vp, _i, _i, _vp, _vp, _vp, _i, _u, _vp, _vp, _vp, _vp, _vp, _vp,
                           _vp, _vp]),
    "dodo_gather_kv_layers": (_i, [_vp, _i, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dodo_pool_kv": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dodo_attend_workspace_bytes": (_sz, [_vp, _i]),
    "dodo_attend": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                         _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "dodo_attend_indexed": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                 _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "dodo_attend_backward_workspace_bytes": (_sz, [_vp, _i, _i, _i, _i]),
    "dodo_attend_backward": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i,
                                  _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dodo_gather_kv_q4": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dodo_expand_kv_q4": (_i, [_vp, _vp, _vp, _i, _i, _vp, _vp, _i, _i, _vp, _vp, _vp]),
    "dodo_attend_q4_workspace_bytes": (_sz, [_vp, _i, _i, _i]),
    "dodo_attend_q4": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                            _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "dodo_host_arena_bytes": (_sz, [_vp, _i, _i, _i, _i, _i, _i, _i, _i, _i]),
    "dodo_compress_decode_host": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _vp, _i, _vp, _vp, _i, _vp, _i, _f,
                                       _vp, _vp, _sz, _vp]),
    "dodo_attend_noalloc": (_i, [_vp, _vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                 _i, _i, _vp, _vp, _vp, ctypes.c_char_p, _sz]),
}

_lib = None


def load() -> ctypes.CDLL:
    """Load ``libdodo.so`` and attach the signatures.  Raises if the library is missing."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2310_02409_b200.build` "
                              "(there is no fallback path)")
        lib = ctypes.CDLL(str(LIB_PATH))
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


class DodoError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"dodo status {status}: {message}")
        self.status = status


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev(t: torch.Tensor | None):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device arguments must be contiguous CUDA tensors")
    return t.data_ptr()


_I32 = np.dtype(np.int32)


def _table(a) -> bytes | None:
    """A host table as the bytes of an int32 array: a read-only pointer argument without the cost of ``ndarray.ctypes``."""
    if a is None:
        return None
    if type(a) is not np.ndarray or a.dtype is not _I32:
        a = np.asarray(a, dtype=np.int32)
    return a.tobytes()


def _in_place(a) -> int:
    """Address of an int32 table that the call updates."""
    if not (isinstance(a, np.ndarray) and a.dtype == np.int32 and a.flags.c_contiguous and a.flags.writeable):
        raise TypeError("cache_len must be a contiguous, writeable int32 numpy array (updated in place)")
    return ctypes.addressof(ctypes.c_char.from_buffer(a)) if a.size else 0


def _bound(table: bytes | None, sequences: int, rows: int, what: str):
    """Raises unless an offset table describes ``sequences`` regions inside ``rows`` rows."""
    if table is None or len(table) != 4 * (sequences + 1):
        raise ValueError(f"{what} must have {sequences + 1} entries")
    if int.from_bytes(table[-4:], "little", signed=True) > rows:
        raise ValueError(f"{what} ends behind row {rows}, the last of its array")


def _entries(table: bytes | None, sequences: int, what: str):
    if table is None or len(table) < 4 * sequences:
        raise ValueError(f"{what} must have {sequences} entries")


def _cache_tables(off: bytes | None, length: bytes | None, sequences: int, rows: int | None):
    """Checks an attention call's cache tables; rows None: there is no cache tensor, but the library reads tables that it is given."""
    if rows is not None:
        _bound(off, sequences, rows, "cache_off")
    elif length is None:
        return
    elif off is None or len(off) != 4 * (sequences + 1):
        raise ValueError(f"cache_off must have {sequences + 1} entries")
    _entries(length, sequences, "cache_len")


def _local_tables(off: bytes | None, length: bytes | None, pos0: bytes | None, sequences: int, given: bool):
    """Checks an attention call's tables of local tokens; given: there are tensors beside them."""
    if length is None and not given:
        return
    _entries(length, sequences, "loc_len")
    for table, what in ((off, "loc_off"), (pos0, "loc_pos0")):
        if given or table is not None:
            _entries(table, sequences, what)


def _host_i32(a) -> np.ndarray | None:
    if a is None:
        return None
    return np.ascontiguousarray(a, dtype=np.int32)


def _hp(a: np.ndarray | None):
    return None if a is None else a.ctypes.data


try:        # the current stream's handle without building a Stream object around it (0.1 instead of 3.3 us per call)
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _current_device
except ImportError:
    _raw_stream = _current_device = None


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


class Dodo:
    """One library context on one CUDA device.  Methods mirror the C entry points one to one."""

    def __init__(self, device: int = 0):
        self._lib = load()
        self._ctx = _vp()
        rc = self._lib.dodo_create(ctypes.byref(self._ctx), int(device))
        if rc != OK:
            msg = self._lib.dodo_last_error(self._ctx).decode() if self._ctx else "no context"
            self._lib.dodo_destroy(self._ctx)
            self._ctx = None
            raise DodoError(rc, msg)
        self.device = torch.device("cuda", device)
        self._index = int(device)

    def close(self):
        if getattr(self, "_ctx", None):
            self._lib.dodo_destroy(self._ctx)
            self._ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != OK:
            raise DodoError(rc, self._lib.dodo_last_error(self._ctx).decode())

    # -- helpers -------------------------------------------------------------------------------
    def num_nuggets(self, n: int, r: int) -> int:
        return int(self._lib.dodo_num_nuggets(int(n), int(r)))

    def device_status(self) -> int:
        out = _i(0)
        self._check(self._lib.dodo_device_status(self._ctx, ctypes.byref(out)))
        return int(out.value)

    def reset(self):
        self._check(self._lib.dodo_reset(self._ctx, _stream()))

    def cache_written(self):
        self._check(self._lib.dodo_cache_written(self._ctx))

    def set_tuning(self, knob: int, value: int):
        self._check(self._lib.dodo_set_tuning(self._ctx, int(knob), int(value)))

    def attend_workspace_bytes(self, dh: int) -> int:
        return int(self._lib.dodo_attend_workspace_bytes(self._ctx, int(dh)))

    def host_arena_bytes(self, dtype_code, d, H, dh, total_tokens, total_nuggets, B, local, steps) -> int:
        return int(self._lib.dodo_host_arena_bytes(self._ctx, dtype_code, d, H, dh, total_tokens, total_nuggets, B,
                                                   local, steps))

    def compress_decode_host(self, hX, hw, hK, hV, seq_off, nug_off, hLocK, hLocV, local, hQ, sm_scale, hO, arena):
        """``dodo_compress_decode_host``: the whole path of one layer on HOST tensors (pinned for
        asynchronous copies); ``arena`` is a device uint8 tensor of ``host_arena_bytes`` bytes."""
        so, no = _host_i32(seq_off), _host_i32(nug_off)
        for t in (hX, hw, hK, hV, hLocK, hLocV, hQ, hO):
            if t.is_cuda or not t.is_contiguous():
                raise ValueError("host arguments must be contiguous CPU tensors")
        steps, B, H, dh = hQ.shape
        self._check(self._lib.dodo_compress_decode_host(
            self._ctx, hX.data_ptr(), hw.data_ptr(), hK.data_ptr(), hV.data_ptr(), _dtype_code(hX), hX.shape[-1], H, dh,
            _hp(so), _hp(no), B, hLocK.data_ptr(), hLocV.data_ptr(), int(local), hQ.data_ptr(), steps, float(sm_scale),
            hO.data_ptr(), _dev(arena), arena.numel() * arena.element_size(), _stream()))

    # -- the path ------------------------------------------------------------------------------
    def score(self, X, w, bias, seq_off, scores):
        so = _host_i32(seq_off)
        self._check(self._lib.dodo_score(self._ctx, _dev(X), _dtype_code(X), X.shape[-1], _dev(w), float(bias),
                                         _hp(so), len(so) - 1, _dev(scores), _stream()))

    def select(self, scores, seq_off, nug_off, flags, idx):
        so, no = _host_i32(seq_off), _host_i32(nug_off)
        self._check(self._lib.dodo_select(self._ctx, _dev(scores), _hp(so), _hp(no), len(so) - 1, int(flags),
                                          _dev(idx), _stream()))

    def score_mlp_workspace_bytes(self, rows: int, dh: int) -> int:
        return int(self._lib.dodo_score_mlp_workspace_bytes(int(rows), int(dh)))

    def score_mlp(self, X, W1, b1, w2, b2, act, seq_off, scores, workspace):
        so = _host_i32(seq_off)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self._check(self._lib.dodo_score_mlp(self._ctx, _dev(X), _dtype_code(X), int(X.shape[1]), _dev(W1), _dev(b1), _dev(w2),
                                             float(b2), int(W1.shape[0]), int(act), _hp(so), len(so) - 1, _dev(scores),
                                             _dev(workspace), ws_bytes, _stream()))

    def score_mlp_select(self, X, W1, b1, w2, b2, act, seq_off, nug_off, flags, scores, idx, workspace):
        so, no = _host_i32(seq_off), _host_i32(nug_off)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self._check(self._lib.dodo_score_mlp_select(self._ctx, _dev(X), _dtype_code(X), int(X.shape[1]), _dev(W1), _dev(b1), _dev(w2),
                                                    float(b2), int(W1.shape[0]), int(act), _hp(so), _hp(no), len(so) - 1, int(flags),
                                                    _dev(scores), _dev(idx), _dev(workspace), ws_bytes, _stream()))

    def count_threshold(self, scores, seq_off, lam, counts):
        so = _host_i32(seq_off)
        self._check(self._lib.dodo_count_threshold(self._ctx, _dev(scores), _hp(so), len(so) - 1, float(lam),
                                                   _dev(counts), _stream()))

    def select_threshold(self, scores, seq_off, nug_off, lam, idx):
        so, no = _host_i32(seq_off), _host_i32(nug_off)
        self._check(self._lib.dodo_select_threshold(self._ctx, _dev(scores), _hp(so), _hp(no), len(so) - 1, float(lam),
                                                    _dev(idx), _stream()))

    def estimate_threshold(self, sample, r, lam_out):
        self._check(self._lib.dodo_estimate_threshold(self._ctx, _dev(sample), int(sample.numel()), int(r),
                                                      _dev(lam_out), _stream()))

    def score_select(self, X, w, bias, seq_off, nug_off, flags, scores, idx):
        so, no = _host_i32(seq_off), _host_i32(nug_off)
        self._check(self._lib.dodo_score_select(self._ctx, _dev(X), _dtype_code(X), X.shape[-1], _dev(w),
                                                float(bias), _hp(so), _hp(no), len(so) - 1, int(flags),
                                                _dev(scores), _dev(idx), _stream()))

    def gather_kv(self, K, V, seq_off, idx, nug_off, pos_base, cacheK, cacheV, cache_pos, cache_off, cache_len):
        """``cache_len`` must be an int32 numpy array; it is updated in place."""
        so, no, pb, co = _host_i32(seq_off), _host_i32(nug_off), _host_i32(pos_base), _host_i32(cache_off)
        if not (isinstance(cache_len, np.ndarray) and cache_len.dtype == np.int32 and cache_len.flags.c_contiguous):
            raise TypeError("cache_len must be a contiguous int32 numpy array (updated in place)")
        H, dh = K.shape[-2], K.shape[-1]
        self._check(self._lib.dodo_gather_kv(self._ctx, _dev(K), _dev(V), _dtype_code(K), H, dh, _hp(so), _dev(idx),
                                             _hp(no), _hp(pb), len(so) - 1, _dev(cacheK), _dev(cacheV),
                                             _dev(cache_pos), _hp(co), _hp(cache_len), _stream()))

    def compress(self, X, w, bias, K, V, seq_off, nug_off, pos_base, flags, scores, idx, cacheK, cacheV, cache_pos,
                 cache_off, cache_len):
        """``dodo_compress``: score, TopK and gather in one call; ``cache_len`` (int32 numpy array) is updated in place."""
        so, no, pb, co = _host_i32(seq_off), _host_i32(nug_off), _host_i32(pos_base), _host_i32(cache_off)
        if not (isinstance(cache_len, np.ndarray) and cache_len.dtype == np.int32 and cache_len.flags.c_contiguous):
            raise TypeError("cache_len must be a contiguous int32 numpy array (updated in place)")
        H, dh = K.shape[-2], K.shape[-1]
        self._check(self._lib.dodo_compress(self._ctx, _dev(X), _dtype_code(X), X.shape[-1], _dev(w), float(bias), _dev(K),
                                            _dev(V), H, dh, _hp(so), _hp(no), _hp(pb), len(so) - 1, int(flags), _dev(scores),
                                            _dev(idx), _dev(cacheK), _dev(cacheV), _dev(cache_pos), _hp(co), _hp(cache_len),
                                            _stream()))

    def pool_kv(self, K, V, seq_off, r, pos_base, cacheK, cacheV, cache_pos, cache_off, cache_len):
        """``dodo_pool_kv``: mean of every even chunk of r tokens appended to the caches; ``cache_len`` (int32 numpy
        array) is updated in place."""
        so, pb, co = _host_i32(seq_off), _host_i32(pos_base), _host_i32(cache_off)
        if not (isinstance(cache_len, np.ndarray) and cache_len.dtype == np.int32 and cache_len.flags.c_contiguous):
            raise TypeError("cache_len must be a contiguous int32 numpy array (updated in place)")
        H, dh = K.shape[-2], K.shape[-1]
        self._check(self._lib.dodo_pool_kv(self._ctx, _dev(K), _dev(V), _dtype_code(K), H, dh, _hp(so), int(r), _hp(pb),
                                           len(so) - 1, _dev(cacheK), _dev(cacheV), _dev(cache_pos), _hp(co), _hp(cache_len),
                                           _stream()))

    def gather_kv_layers(self, Ks, Vs, seq_off, idx, nug_off, pos_base, cacheKs, cacheVs, cache_pos, cache_off,
                         cache_len):
        """One shared selection, L layers: ``Ks``, ``Vs``, ``cacheKs``, ``cacheVs`` are sequences of L tensors of
        one shape and dtype each.  ``cache_len`` (int32 numpy array) is updated in place, once."""
        so, no, pb, co = _host_i32(seq_off), _host_i32(nug_off), _host_i32(pos_base), _host_i32(cache_off)
        if not (isinstance(cache_len, np.ndarray) and cache_len.dtype == np.int32 and cache_len.flags.c_contiguous):
            raise TypeError("cache_len must be a contiguous int32 numpy array (updated in place)")
        L = len(Ks)
        if not (len(Vs) == len(cacheKs) == len(cacheVs) == L):
            raise ValueError("Ks, Vs, cacheKs and cacheVs must name the same number of layers")
        if L == 0:
            return
        H, dh = Ks[0].shape[-2], Ks[0].shape[-1]
        for t in (*Ks, *Vs, *cacheKs, *cacheVs):
            if t.dtype != Ks[0].dtype or tuple(t.shape[-2:]) != (H, dh):
                raise ValueError("every layer's K, V and caches must share dtype, H and dh")
        ptrs = lambda ts: (ctypes.c_void_p * L)(*[_dev(t) for t in ts])
        self._check(self._lib.dodo_gather_kv_layers(self._ctx, L, ptrs(Ks), ptrs(Vs), _dtype_code(Ks[0]), H, dh, _hp(so),
                                                    _dev(idx), _hp(no), _hp(pb), len(so) - 1, ptrs(cacheKs),
                                                    ptrs(cacheVs), _dev(cache_pos), _hp(co), _hp(cache_len), _stream()))

    def attend(self, Q, q_off, q_pos0, sm_scale, cacheK, cacheV, cache_pos, cache_off, cache_len,
               locK, locV, loc_off, loc_len, loc_pos0, O, lse, workspace):
        qo, qp = _host_i32(q_off), _host_i32(q_pos0)
        co, cl = _host_i32(cache_off), _host_i32(cache_len)
        lo, ll, lp = _host_i32(loc_off), _host_i32(loc_len), _host_i32(loc_pos0)
        H, dh = Q.shape[-2], Q.shape[-1]
        loc_rows = 0 if locK is None else locK.shape[0]
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self._check(self._lib.dodo_attend(self._ctx, _dev(Q), _hp(qo), _hp(qp), _dtype_code(Q), H, dh, float(sm_scale),
                                          _dev(cacheK), _dev(cacheV), _dev(cache_pos), _hp(co), _hp(cl),
                                          _dev(locK), _dev(locV), _hp(lo), _hp(ll), _hp(lp), loc_rows,
                                          len(qo) - 1, _dev(O), _dev(lse), _dev(workspace), ws_bytes, _stream()))

    # -- checks of the methods below ------------------------------------------------------------------
    def _ptr(self, t, dtype, numel, name):
        """Address of a dense tensor on this context's device with its dtype and (None: any) number of elements."""
        if t.dtype is not dtype:
            raise TypeError(f"{name} must be {dtype}, is {t.dtype}")
        if t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous tensor on {self.device}")
        if numel is not None and t.numel() != numel:
            raise ValueError(f"{name} must have {numel} elements, has {t.numel()} (shape {tuple(t.shape)})")
        return t.data_ptr()

    def _workspace(self, t):
        if t is None:
            return None, 0
        return self._ptr(t, t.dtype, None, "workspace"), t.numel() * t.element_size()

    def _heads(self, t, name):
        if t.dim() != 3:
            raise ValueError(f"{name} must have shape [rows, H, dh], has {tuple(t.shape)}")
        return t.shape

    # -- the gradient of attend --------------------------------------------------------------------
    def attend_backward_workspace_bytes(self, q_rows: int, H: int, dh: int, cache_rows: int) -> int:
        return int(self._lib.dodo_attend_backward_workspace_bytes(self._ctx, int(q_rows), int(H), int(dh), int(cache_rows)))

    def attend_backward(self, Q, q_off, q_pos0, sm_scale, cacheK, cacheV, cache_pos, cache_off, cache_len,
                        locK, locV, loc_off, loc_len, loc_pos0, O, lse, dO, dQ, dcacheK, dcacheV, dlocK, dlocV, dscore, workspace):
        """``dodo_attend_backward``: gradients of ``attend`` from its inputs, ``O``, ``lse`` and ``dO``; ``dscore`` (float, one
        entry a cache row) may be None, and the cache's or the local tokens' tensors where the call has none."""
        qo, qp = _table(q_off), _table(q_pos0)
        co, cl = _table(cache_off), _table(cache_len)
        lo, ll, lp = _table(loc_off), _table(loc_len), _table(loc_pos0)
        rows_q, H, dh = self._heads(Q, "Q")
        code, B, dt, row = _dtype_code(Q), len(qo) // 4 - 1, Q.dtype, H * dh
        _bound(qo, B, rows_q, "q_off")
        _entries(qp, B, "q_pos0")
        n, ptr = rows_q * row, self._ptr
        q, o, g, dq = ptr(Q, dt, n, "Q"), ptr(O, dt, n, "O"), ptr(dO, dt, n, "dO"), ptr(dQ, dt, n, "dQ")
        ls = ptr(lse, torch.float32, rows_q * H, "lse")
        ck = cv = dk = dv = pos = ds = rows = None
        if cacheK is not None:
            rows = self._heads(cacheK, "cacheK")[0]
            n = rows * row
            ck, cv = ptr(cacheK, dt, n, "cacheK"), ptr(cacheV, dt, n, "cacheV")
            dk, dv = ptr(dcacheK, dt, n, "dcacheK"), ptr(dcacheV, dt, n, "dcacheV")
            pos = ptr(cache_pos, torch.int32, None, "cache_pos")
            rows = min(rows, cache_pos.numel())
            if dscore is not None:
                ds = ptr(dscore, torch.float32, None, "dscore")
                rows = min(rows, dscore.numel())
        _cache_tables(co, cl, B, rows)
        lk = lv = dlk = dlv = None
        loc_rows = 0
        if locK is not None:
            loc_rows = self._heads(locK, "locK")[0]
            n = loc_rows * row
            lk, lv = ptr(locK, dt, n, "locK"), ptr(locV, dt, n, "locV")
            dlk, dlv = ptr(dlocK, dt, n, "dlocK"), ptr(dlocV, dt, n, "dlocV")
        _local_tables(lo, ll, lp, B, locK is not None)
        w, ws_bytes = self._workspace(workspace)
        self._check(self._lib.dodo_attend_backward(
            self._ctx, q, qo, qp, code, H, dh, sm_scale, ck, cv, pos, co, cl, lk, lv, lo, ll, lp, loc_rows, B, o, ls, g, dq, dk, dv,
            dlk, dlv, ds, w, ws_bytes, _stream()))

    # -- the 4-bit nugget cache ----------------------------------------------------------------------
    def _q4_cache(self, cache_q4, cache_scale, H, dh):
        rows = cache_q4.shape[0]
        return rows, self._ptr(cache_q4, torch.uint8, rows * H * dh, "cache_q4"), self._ptr(cache_scale, torch.int32, rows * H * (dh // 16), "cache_scale")

    def gather_kv_q4(self, K, V, seq_off, idx, nug_off, pos_base, cache_q4, cache_scale, cache_pos, cache_off, cache_len):
        """``dodo_gather_kv_q4``: append the selected rows to a 4-bit cache (``cache_q4`` uint8 [rows, H, 2, dh/2],
        ``cache_scale`` int32 [rows, H, 2, dh/32]); ``cache_len`` (int32 numpy array) is updated in place."""
        so, no, pb, co, cl = _table(seq_off), _table(nug_off), _table(pos_base), _table(cache_off), _in_place(cache_len)
        tokens, H, dh = self._heads(K, "K")
        code, dt, B, ptr = _dtype_code(K), K.dtype, len(so) // 4 - 1, self._ptr
        rows, q4, sc = self._q4_cache(cache_q4, cache_scale, H, dh)
        k, v = ptr(K, dt, None, "K"), ptr(V, dt, K.numel(), "V")
        ix, pos = ptr(idx, torch.int32, None, "idx"), ptr(cache_pos, torch.int32, None, "cache_pos")
        _bound(so, B, tokens, "seq_off")
        _bound(no, B, idx.numel(), "nug_off")
        _bound(co, B, min(rows, cache_pos.numel()), "cache_off")
        _entries(pb, B, "pos_base")
        if cache_len.size < B:
            raise ValueError(f"cache_len must have {B} entries")
        self._check(self._lib.dodo_gather_kv_q4(self._ctx, k, v, code, H, dh, so, ix, no, pb, B, q4, sc, pos, co, cl, _stream()))

    def expand_kv_q4(self, cache_q4, cache_scale, cache_off, cache_len, K, V):
        """``dodo_expand_kv_q4``: the rows in use of a 4-bit cache as rows of K and V (their dtype, the cache's row layout)."""
        co, cl = _table(cache_off), _table(cache_len)
        rows_k, H, dh = self._heads(K, "K")
        code, dt, B = _dtype_code(K), K.dtype, len(co) // 4 - 1
        rows, q4, sc = self._q4_cache(cache_q4, cache_scale, H, dh)
        k, v = self._ptr(K, dt, None, "K"), self._ptr(V, dt, K.numel(), "V")
        _bound(co, B, min(rows, rows_k), "cache_off")
        _entries(cl, B, "cache_len")
        self._check(self._lib.dodo_expand_kv_q4(self._ctx, q4, sc, H, dh, co, cl, B, code, k, v, _stream()))

    def attend_q4_workspace_bytes(self, H: int, dh: int, cache_rows: int) -> int:
        return int(self._lib.dodo_attend_q4_workspace_bytes(self._ctx, int(H), int(dh), int(cache_rows)))

    def attend_q4(self, Q, q_off, q_pos0, sm_scale, cache_q4, cache_scale, cache_pos, cache_off, cache_len,
                  locK, locV, loc_off, loc_len, loc_pos0, O, lse, workspace):
        """``dodo_attend_q4``: ``attend`` over a 4-bit nugget cache and uncompressed local tokens."""
        qo, qp = _table(q_off), _table(q_pos0)
        co, cl = _table(cache_off), _table(cache_len)
        lo, ll, lp = _table(loc_off), _table(loc_len), _table(loc_pos0)
        rows_q, H, dh = self._heads(Q, "Q")
        code, B, dt, ptr = _dtype_code(Q), len(qo) // 4 - 1, Q.dtype, self._ptr
        _bound(qo, B, rows_q, "q_off")
        _entries(qp, B, "q_pos0")
        q, o = ptr(Q, dt, None, "Q"), ptr(O, dt, Q.numel(), "O")
        ls = None if lse is None else ptr(lse, torch.float32, rows_q * H, "lse")
        q4 = sc = pos = lk = lv = rows = None
        if cache_q4 is not None:
            rows, q4, sc = self._q4_cache(cache_q4, cache_scale, H, dh)
            pos = ptr(cache_pos, torch.int32, None, "cache_pos")
            rows = min(rows, cache_pos.numel())
        _cache_tables(co, cl, B, rows)
        loc_rows = 0
        if locK is not None:
            loc_rows = self._heads(locK, "locK")[0]
            lk, lv = ptr(locK, dt, loc_rows * H * dh, "locK"), ptr(locV, dt, loc_rows * H * dh, "locV")
        _local_tables(lo, ll, lp, B, locK is not None)
        w, ws_bytes = self._workspace(workspace)
        self._check(self._lib.dodo_attend_q4(self._ctx, q, qo, qp, code, H, dh, sm_scale, q4, sc, pos, co, cl, lk, lv, lo, ll, lp, loc_rows,
                                             B, o, ls, w, ws_bytes, _stream()))

    def attend_indexed(self, Q, q_off, q_pos0, sm_scale, K, V, seq_off, idx, nug_off, pos_base,
                       locK, locV, loc_off, loc_len, loc_pos0, O, lse, workspace):
        """``dodo_attend_indexed``: queries attend the rows ``idx`` names in the uncompressed K / V, then the local tokens."""
        qo, qp = _host_i32(q_off), _host_i32(q_pos0)
        so, no, pb = _host_i32(seq_off), _host_i32(nug_off), _host_i32(pos_base)
        lo, ll, lp = _host_i32(loc_off), _host_i32(loc_len), _host_i32(loc_pos0)
        H, dh = Q.shape[-2], Q.shape[-1]
        loc_rows = 0 if locK is None else locK.shape[0]
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self._check(self._lib.dodo_attend_indexed(self._ctx, _dev(Q), _hp(qo), _hp(qp), _dtype_code(Q), H, dh, float(sm_scale),
                                                  _dev(K), _dev(V), _hp(so), _dev(idx), _hp(no), _hp(pb), _dev(locK), _dev(locV),
                                                  _hp(lo), _hp(ll), _hp(lp), loc_rows, len(qo) - 1, _dev(O), _dev(lse),
                                                  _dev(workspace), ws_bytes, _stream()))


def attend_noalloc(Q, q_off, q_pos0, sm_scale, cacheK, cacheV, cache_pos, cache_off, cache_len,
                   locK, locV, loc_off, loc_len, loc_pos0, O, lse):
    """``dodo_attend_noalloc``: attention without a context or a workspace, for callers that are not
    allowed to allocate device memory (the scratch is a fixed array inside the library).  Runs on the
    current device and stream; at most 64 sequences per call; calls must not overlap on the GPU."""
    lib = load()
    qo, qp = _host_i32(q_off), _host_i32(q_pos0)
    co, cl = _host_i32(cache_off), _host_i32(cache_len)
    lo, ll, lp = _host_i32(loc_off), _host_i32(loc_len), _host_i32(loc_pos0)
    H, dh = Q.shape[-2], Q.shape[-1]
    loc_rows = 0 if locK is None else locK.shape[0]
    err = ctypes.create_string_buffer(512)
    rc = lib.dodo_attend_noalloc(_dev(Q), _hp(qo), _hp(qp), _dtype_code(Q), H, dh, float(sm_scale),
                                 _dev(cacheK), _dev(cacheV), _dev(cache_pos), _hp(co), _hp(cl),
                                 _dev(locK), _dev(locV), _hp(lo), _hp(ll), _hp(lp), loc_rows, len(qo) - 1,
                                 _dev(O), _dev(lse), _stream(), err, len(err))
    if rc != OK:
        raise DodoError(rc, err.value.decode())
