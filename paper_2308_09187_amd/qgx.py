"""Thin ctypes binding over libqgx.so (include/qgx.h): argument marshalling only.

Every step of the path runs in the library's gfx950 kernels; torch is used for device memory and
streams.  Loading fails loudly when the library has not been built
(``python -m paper_2308_09187_amd.build``); there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqgx.so")

OK = 0
ERR_ARG, ERR_LEVELS, ERR_CAPACITY, ERR_STREAM, ERR_NONFINITE, ERR_HIP, ERR_STATE = -1, -2, -3, -4, -5, -6, -7
EBIT_CAPACITY, EBIT_STREAM, EBIT_NONFINITE, EBIT_STATE = 1, 2, 4, 8
CALL_FIRST_HALF, CALL_SECOND_HALF = 0xFFFFFFFE, 0xFFFFFFFF   # call numbers taken from the iteration counter on the device
NORM_LINF, NORM_L2 = 0, 2
CODE_ELIAS_OMEGA, CODE_TABLE = 0, 1
CHUNK, SUB, SUBS, MAX_SYM, MAX_BINS = 4096, 32, 128, 127, 4096
STATIC_MAX_CHUNKS = 65536
MAX_INTERVALS = 128
FEW_TENSORS = 16
DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

EXPORTS = [
    "qgx_create", "qgx_destroy", "qgx_stream_sizes", "qgx_slot_words", "qgx_compact", "qgx_select_table", "qgx_set_levels", "qgx_get_levels", "qgx_set_code_table",
    "qgx_quantize", "qgx_encode", "qgx_quantize_encode", "qgx_decode", "qgx_decode_average", "qgx_fit_levels", "qgx_fit_code",
    "qgx_state_init", "qgx_eg_step", "qgx_eg_step_static", "qgx_average_reset", "qgx_average_export", "qgx_get_scalars", "qgx_stream_bits", "qgx_debug_set_waves_per_position", "qgx_state_export", "qgx_state_import",
    "qgx_poll_error", "qgx_last_error",
    "qgx_tensor_list_size", "qgx_tensor_list_set", "qgx_clip_gradients", "qgx_layer_norm", "qgx_layer_norm_scratch", "qgx_layer_norm_backward",
    "qgx_position_bias", "qgx_position_bias_scratch", "qgx_position_bias_backward",
    "qgx_game_operator", "qgx_game_dual_vectors", "qgx_quantize_encode_game", "qgx_norm2", "qgx_game_gap", "qgx_quantization_metrics",
]


class QgxError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__("qgx status %d: %s" % (status, text))
        self.status = status


class _Config(C.Structure):
    _fields_ = [("d", C.c_uint64), ("K", C.c_uint32), ("bucket", C.c_uint32), ("n_segments", C.c_uint32),
                ("segment_len", C.POINTER(C.c_uint64)), ("norm", C.c_int32), ("code", C.c_int32),
                ("seed", C.c_uint64)]


class _Game(C.Structure):
    _fields_ = [("z", C.c_void_p), ("a", C.c_void_p), ("b", C.c_void_p), ("mu", C.c_float), ("sigma", C.c_float),
                ("noise_seed", C.c_uint64)]


class _Stream(C.Structure):
    _fields_ = [("norms", C.c_void_p), ("chunk_off", C.c_void_p), ("sub_end", C.c_void_p),
                ("payload", C.c_void_p), ("payload_words_per_worker", C.c_uint64), ("slot_words", C.c_uint64)]


class _Tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("n", C.c_uint64), ("stride", C.c_uint64), ("offset", C.c_uint64), ("dtype", C.c_int32)]


class _TensorList(C.Structure):
    _fields_ = [("table", C.c_void_p), ("table_bytes", C.c_uint64), ("n_pieces", C.c_uint64), ("d", C.c_uint64), ("K", C.c_uint32),
                ("n_tensors", C.c_uint32), ("shared_rows", C.c_uint32), ("dtype", C.c_int32), ("n_few", C.c_uint32),
                ("few", C.c_uint64 * 3 * FEW_TENSORS)]


class _Buckets(C.Structure):
    _fields_ = [("n", C.c_uint32), ("bounds", C.POINTER(C.c_int32)), ("rows", C.POINTER(C.c_uint32))]


class _Scores(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("heads", C.c_uint32), ("workers", C.c_uint64), ("batch", C.c_uint64),
                ("q", C.c_uint64), ("k", C.c_uint64), ("s_worker", C.c_uint64), ("s_batch", C.c_uint64), ("s_head", C.c_uint64),
                ("s_row", C.c_uint64)]


_lib = None


def load():
    """Loads libqgx.so; raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libqgx.so is not built: run `python -m paper_2308_09187_amd.build` "
                              "(hipcc, gfx950); there is no fallback path")
        lib = C.CDLL(LIB_PATH)
        for name in EXPORTS:
            getattr(lib, name)
        lib.qgx_destroy.restype = None
        lib.qgx_poll_error.restype = C.c_uint32
        lib.qgx_last_error.restype = C.c_char_p
        u64, ptr, f32 = C.c_uint64, C.c_void_p, C.c_float    # (argument types given once: plain numbers then pass as they are)
        lib.qgx_clip_gradients.argtypes = [ptr, ptr, C.c_int, f32, ptr, ptr, ptr]
        lib.qgx_layer_norm.argtypes = [ptr, C.c_int, u64, u64, u64, ptr, u64, u64, ptr, ptr, f32, ptr, u64, u64, ptr, ptr, ptr]
        lib.qgx_layer_norm_scratch.argtypes = [ptr, C.c_int, u64, u64, u64, ptr]
        lib.qgx_layer_norm_backward.argtypes = [ptr, C.c_int, u64, u64, u64, ptr, u64, u64, ptr, u64, u64, ptr, ptr, ptr, ptr, u64, u64,
                                                ptr, ptr, u64, ptr, u64, ptr]
        lib.qgx_position_bias.argtypes = [ptr, ptr, ptr, C.c_uint32, ptr, ptr, C.c_int64, ptr, ptr]
        lib.qgx_position_bias_scratch.argtypes = [ptr, ptr, ptr, C.c_int64, ptr]
        lib.qgx_position_bias_backward.argtypes = [ptr, ptr, ptr, C.c_int64, ptr, C.c_uint32, u64, ptr, u64, ptr]
        _lib = lib
    return _lib


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream_handle(stream):
    if stream is None:                       # the handle alone: a Stream object around it takes 3 us, a call with its launch 4.6
        return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return C.c_void_p(stream.cuda_stream)


def _need(ok, text, *what):
    if not ok:
        raise QgxError(ERR_ARG, text % what if what else text)


def _handle(stream, t):
    """The stream's handle as a number, for the functions whose argument types are given; None: the current one of t's device."""
    return torch._C._cuda_getCurrentRawStream(t.get_device()) if stream is None else stream.cuda_stream


def _empty(like, shape, dtype, stream):
    """Memory on like's device (new_empty: 1.5 us, torch.empty 2.3).  Made for a call on `stream` it comes from that
    stream's pool, so that its next use is in order after the call."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _parameter(t, shape, name):
    """Address of a contiguous binary32 parameter, or of a run of one; None stays None."""
    if t is None:
        return None
    _need(t.is_cuda and t.dtype == torch.float32 and t.shape == shape and t.is_contiguous(), "%s: contiguous float32 of shape %s on the GPU", name, tuple(shape))
    return t.data_ptr()


def _dense_last(t):
    return t.dim() == 0 or t.shape[-1] <= 1 or t.stride(-1) == 1


def _empty_like(t, stream):
    """The same of t's shape and type, contiguous (1.3 us)."""
    if stream is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    with torch.cuda.stream(stream):
        return torch.empty_like(t, memory_format=torch.contiguous_format)


class Buckets:
    """Buckets of the relative position delta = key - query: interval b holds bounds[b] <= delta < bounds[b + 1] and takes
    row rows[b] of the table; a delta outside [bounds[0], bounds[-1]) is masked."""

    def __init__(self, bounds, rows):
        _need(len(bounds) == len(rows) + 1, "Buckets: one bound more than rows")
        bounds, rows = [int(x) for x in bounds], [int(x) for x in rows]
        _need(all(-(1 << 31) <= x < 1 << 31 for x in bounds) and all(0 <= x < 1 << 32 for x in rows), "Buckets: bounds and rows of 32 bits")
        self._bounds = (C.c_int32 * len(bounds))(*bounds)
        self._rows = (C.c_uint32 * max(1, len(rows)))(*rows)
        self._c = _Buckets(len(rows), self._bounds, self._rows)
        self._ref = C.addressof(self._c)

    @classmethod
    def logarithmic(cls, rows, far, both=False, window=None):
        """Buckets of a table of `rows` rows: of m rows for keys at and before the query, the first m // 2 have a distance
        each (0, 1, ..), the others start at m // 2 times equal powers of far / (m // 2), the last of them holding all that is
        further.  both=False: m = rows, keys after the query are masked; both=True: m = rows // 2, and as many rows again,
        m .., for the keys after it, by the same distances.  window: keys that far before (and after) or further are masked.
        The starts are worked out in whole numbers: exact, whatever the machine's logarithm.  Where several rows start within one
        distance, the last of them has it and the others have none."""
        m = rows // 2 if both else rows
        exact = m // 2
        _need(m >= 2 and far > exact, "Buckets.logarithmic: two rows a side at least, and far beyond those of one distance each")
        start = list(range(exact))
        for t in range(m - exact):                       # the smallest n with (n / exact)^(m - exact) >= (far / exact)^t
            n = start[-1]
            while n ** (m - exact) < exact ** (m - exact - t) * far ** t:
                n += 1
            start.append(n)
        end = (1 << 30) if window is None else min(int(window), (1 << 31) - 1)       # (no delta is further)
        _need(end >= 1, "Buckets.logarithmic: a window of one key at least")
        start = [n for n in start if n < end]
        stop = start[1:] + [end]                         # (where powers are less than one apart, rows have no distance)
        bounds, ids = [1 - end], []
        for b in range(len(start) - 1, -1, -1):          # keys before the query, the furthest first
            if start[b] < stop[b]:
                ids.append(b)
                bounds.append(1 - start[b])
        if both:
            for b in range(len(start)):
                if max(1, start[b]) < stop[b]:           # (distance 0 is with the keys before)
                    ids.append(m + b)
                    bounds.append(stop[b])
        return cls(bounds, ids)


class TensorList:
    """Gradient tensors of the K workers and where they belong in V; made by Context.tensor_list.  Holds the tensors."""

    def __init__(self, tensors, table, struct):
        self.tensors, self.table, self._c = tensors, table, struct
        self._ref = C.addressof(struct)


class Stream:
    """Device buffers of one CODE o Q result for K workers."""

    def __init__(self, K, NB, NC, cap_words, device="cuda", slot_words=0):
        cap_words = (int(cap_words) + 3) // 4 * 4
        self.slot_words = int(slot_words)
        self.norms = torch.zeros((K, NB), dtype=torch.float32, device=device)
        self.chunk_off = torch.zeros((K, NC + 1), dtype=torch.int32, device=device)
        self.sub_end = torch.zeros((K, NC, SUBS), dtype=torch.int16, device=device)
        self.payload = torch.zeros((K, cap_words), dtype=torch.int32, device=device)
        self.cap_words = cap_words

    def c_struct(self):
        return _Stream(self.norms.data_ptr(), self.chunk_off.data_ptr(), self.sub_end.data_ptr(),
                       self.payload.data_ptr(), self.cap_words, self.slot_words)

    def to_host(self):
        """numpy views in the container's unsigned types."""
        return dict(norms=self.norms.cpu().numpy(),
                    chunk_off=self.chunk_off.cpu().numpy().view(np.uint32),
                    sub_end=self.sub_end.cpu().numpy().view(np.uint16),
                    payload=self.payload.cpu().numpy().view(np.uint32))


class Context:
    def __init__(self, d, K, bucket, norm=NORM_L2, code=CODE_ELIAS_OMEGA, seed=0, segment_len=None, device="cuda"):
        self.lib = load()
        self.d, self.K, self.bucket, self.device = int(d), int(K), int(bucket), device
        seg = None
        nseg = 0
        if segment_len is not None:
            seg = (C.c_uint64 * len(segment_len))(*[int(x) for x in segment_len])
            nseg = len(segment_len)
        cfg = _Config(self.d, self.K, self.bucket, nseg, seg, norm, code, seed)
        self._h = C.c_void_p()
        self._need_bytes = C.c_uint64()           # where the scratch functions answer
        self._need_ref = C.addressof(self._need_bytes)
        self._table, self._n_sym = 0, {}          # the table selected; symbols of each table that was set
        with torch.cuda.device(device):
            st = self.lib.qgx_create(C.byref(self._h), C.byref(cfg))
        if st != OK:
            raise QgxError(st, "qgx_create rejected the configuration")
        nb, nc, ww = C.c_uint64(), C.c_uint64(), C.c_uint64()
        self._check(self.lib.qgx_stream_sizes(self._h, C.byref(nb), C.byref(nc), C.byref(ww)))
        self.NB, self.NC, self.worst_words = nb.value, nc.value, ww.value

    def _check(self, st):
        if st != OK:
            raise QgxError(st, self.lib.qgx_last_error(self._h).decode())

    def close(self):
        if self._h:
            self.lib.qgx_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def slot_words(self):
        sw = C.c_uint64()
        self._check(self.lib.qgx_slot_words(self._h, C.byref(sw)))
        return sw.value

    def new_stream(self, cap_words=None, slotted=False):
        """Compact stream (worst-case capacity unless cap_words is given), or a slotted one."""
        if slotted:
            sw = self.slot_words()
            return Stream(self.K, self.NB, self.NC, sw * self.NC, self.device, slot_words=sw)
        return Stream(self.K, self.NB, self.NC, self.worst_words if cap_words is None else cap_words, self.device)

    def compact(self, src: Stream, dst: Stream, stream=None):
        a, b = src.c_struct(), dst.c_struct()
        self._check(self.lib.qgx_compact(self._h, C.byref(a), C.byref(b), _stream_handle(stream)))
        return dst

    # -- tables ---------------------------------------------------------------------------------
    def set_levels(self, levels, stream=None):
        lv = np.ascontiguousarray(levels, dtype=np.float32)
        self._check(self.lib.qgx_set_levels(self._h, lv.ctypes.data_as(C.c_void_p), C.c_uint32(len(lv)),
                                            _stream_handle(stream)))
        self._n_sym[self._table] = len(lv)

    def get_levels(self, stream=None):
        lv = np.zeros(MAX_SYM, np.float32)
        n = C.c_uint32()
        self._check(self.lib.qgx_get_levels(self._h, lv.ctypes.data_as(C.c_void_p), C.byref(n), _stream_handle(stream)))
        return lv[: n.value].copy()

    def set_code_table(self, code_len, code_bits, stream=None):
        cl = np.ascontiguousarray(code_len, dtype=np.uint8)
        cb = np.ascontiguousarray(code_bits, dtype=np.uint32)
        self._check(self.lib.qgx_set_code_table(self._h, cl.ctypes.data_as(C.c_void_p), cb.ctypes.data_as(C.c_void_p),
                                                C.c_uint32(len(cl)), _stream_handle(stream)))

    # -- CODE o Q -------------------------------------------------------------------------------
    def quantize(self, V, call_id, norms_in=None, stream=None):
        norms = torch.empty((self.K, self.NB), dtype=torch.float32, device=V.device)
        sym = torch.empty((self.K, self.d), dtype=torch.uint8, device=V.device)
        self._check(self.lib.qgx_quantize(self._h, _ptr(V), C.c_uint32(call_id), _ptr(norms_in), _ptr(norms),
                                          _ptr(sym), _stream_handle(stream)))
        return norms, sym

    def encode(self, norms, sym, out: Stream, stream=None):
        s = out.c_struct()
        self._check(self.lib.qgx_encode(self._h, _ptr(norms), _ptr(sym), C.byref(s), _stream_handle(stream)))
        return out

    def quantize_encode(self, V, call_id, out: Stream, norms_in=None, stream=None):
        s = out.c_struct()
        self._check(self.lib.qgx_quantize_encode(self._h, _ptr(V), C.c_uint32(call_id), _ptr(norms_in), C.byref(s),
                                                 _stream_handle(stream)))
        return out

    # -- the large quadratic game's operator, dual vectors and residual norm on the device -------------
    @staticmethod
    def _game(z, a, b, mu, sigma, noise_seed):
        return _Game(z.data_ptr(), a.data_ptr(), b.data_ptr(), mu, sigma, noise_seed)

    def game_operator(self, z, a, b, mu, out=None, stream=None):
        if out is None:
            out = torch.empty(self.d, dtype=torch.float32, device=z.device)
        g = self._game(z, a, b, mu, 0.0, 0)
        self._check(self.lib.qgx_game_operator(self._h, C.byref(g), _ptr(out), _stream_handle(stream)))
        return out

    def game_gap(self, z, a, b, mu, centre, radius, stream=None):
        r = C.c_double()
        g = self._game(z, a, b, mu, 0.0, 0)
        self._check(self.lib.qgx_game_gap(self._h, C.byref(g), _ptr(centre), C.c_double(radius), C.byref(r), _stream_handle(stream)))
        return r.value

    def game_dual_vectors(self, z, a, b, mu, sigma, noise_seed, call_id, out=None, stream=None):
        if out is None:
            out = torch.empty((self.K, self.d), dtype=torch.float32, device=z.device)
        g = self._game(z, a, b, mu, sigma, noise_seed)
        self._check(self.lib.qgx_game_dual_vectors(self._h, C.byref(g), C.c_uint32(call_id), _ptr(out), _stream_handle(stream)))
        return out

    def quantize_encode_game(self, z, a, b, mu, sigma, noise_seed, call_id, out: Stream, V_out=None, stream=None):
        g, s = self._game(z, a, b, mu, sigma, noise_seed), out.c_struct()
        self._check(self.lib.qgx_quantize_encode_game(self._h, C.byref(g), C.c_uint32(call_id), C.byref(s), _ptr(V_out),
                                                      _stream_handle(stream)))
        return out

    def norm2(self, x, stream=None):
        r = C.c_double()
        self._check(self.lib.qgx_norm2(self._h, _ptr(x), C.c_uint64(x.numel()), C.byref(r), _stream_handle(stream)))
        return r.value

    def quantization_metrics(self, V, Vhat, stream=None):
        """Per worker: (number of nonzeros of Q(v), ||Q(v) - v||^2, ||v||^2) as three numpy arrays of K."""
        import numpy as np
        nnz = np.zeros(self.K, np.uint64)
        err = np.zeros(self.K, np.float64)
        nrm = np.zeros(self.K, np.float64)
        self._check(self.lib.qgx_quantization_metrics(self._h, _ptr(V), _ptr(Vhat), C.c_void_p(nnz.ctypes.data),
                                                      C.c_void_p(err.ctypes.data), C.c_void_p(nrm.ctypes.data),
                                                      _stream_handle(stream)))
        return nnz, err, nrm

    # -- between a model's backward pass and the dual vectors -----------------------------------------
    def tensor_list(self, tensors, offsets=None, stream=None):
        """The K workers' gradient tensors, each [K, n] or [n] for K = 1 (rows contiguous, any step between them), for
        clip_gradients.  offsets[i]: where tensor i's elements belong in a worker's row of V; None: one after the other."""
        tensors = list(tensors)
        if offsets is None:
            offsets, at = [], 0
            for t in tensors:
                offsets.append(at)
                at += t.shape[-1] if t.dim() else 1
        _need(len(offsets) == len(tensors), "tensor_list: an offset for every tensor")
        arr = (_Tensor * max(1, len(tensors)))()
        for i, (t, off) in enumerate(zip(tensors, offsets)):
            _need(t.is_cuda and t.dtype in DTYPES, "tensor %d: float32, float16 or bfloat16 on the GPU", i)
            _need((t.dim() == 2 and t.shape[0] == self.K) or (t.dim() == 1 and self.K == 1), "tensor %d: shape [K, n]", i)
            _need(_dense_last(t), "tensor %d: a worker's elements must be contiguous", i)
            _need(0 <= int(off) < 1 << 64, "tensor %d: offset outside the coordinates", i)
            arr[i] = _Tensor(t.data_ptr(), t.shape[-1], t.stride(0) if t.dim() == 2 and self.K > 1 else 0, int(off), DTYPES[t.dtype])
        need, out = C.c_uint64(), _TensorList()
        self._check(self.lib.qgx_tensor_list_size(self._h, arr, C.c_uint32(len(tensors)), C.byref(need)))
        table = _empty(torch.empty(0, device=self.device), (need.value,), torch.uint8, stream)
        self._check(self.lib.qgx_tensor_list_set(self._h, arr, C.c_uint32(len(tensors)), _ptr(table), need, C.byref(out), _stream_handle(stream)))
        return TensorList(tensors, table, out)

    def clip_gradients(self, tensors: TensorList, max_norm, norm=NORM_L2, out=None, stream=None):
        """Clips every worker's gradients to the global norm max_norm, into out = V [K, d] or, without it, in place.
        Returns the workers' norms before, [K]."""
        if out is not None:
            _need(out.is_cuda and out.dtype == torch.float32 and out.shape == (self.K, self.d) and out.is_contiguous(),
                  "clip_gradients: out is V [K, d], contiguous float32 on the GPU")
        norms = _empty(tensors.table, (self.K,), torch.float32, stream)
        st = self.lib.qgx_clip_gradients(self._h, tensors._ref, norm, max_norm, None if out is None else out.data_ptr(),
                                         norms.data_ptr(), _handle(stream, norms))
        if st:
            self._check(st)
        return norms

    @staticmethod
    def _rows(t, name):
        """(type, workers, rows, cols, step between workers, between rows) of [workers, rows, cols], [rows, cols] or [cols]."""
        code, shape, step = DTYPES.get(t.dtype), t.shape, t.stride()
        _need(code is not None and t.is_cuda, "%s: float32, float16 or bfloat16 on the GPU", name)
        _need(1 <= len(shape) <= 3 and (step[-1] == 1 or shape[-1] <= 1), "%s: [workers, rows, cols], [rows, cols] or [cols], rows contiguous", name)
        if len(shape) == 3:
            return code, shape[0], shape[1], shape[2], step[0], step[1]
        return (code, 1, shape[0], shape[1], 0, step[0]) if len(shape) == 2 else (code, 1, 1, shape[0], 0, 0)

    @staticmethod
    def _rows_like(t, x, name):
        """The steps of a tensor of x's shape and type."""
        _need(t.shape == x.shape and t.dtype == x.dtype and t.is_cuda, "%s: of x's shape and type, on the GPU", name)
        step = t.stride()
        _need(step[-1] == 1 or t.shape[-1] <= 1, "%s: rows must be contiguous", name)
        return (step[0], step[1]) if len(step) == 3 else (0, step[0] if len(step) == 2 else 0)

    def layer_norm(self, x, weight=None, bias=None, eps=1e-5, out=None, save=True, stream=None):
        """Layer norm over the last dimension of x.  Returns (y, mean, rstd), the last two what the backward pass takes
        (save=False: None); weight and bias float32 [cols], runs of X say, or None."""
        code, wk, rows, cols, xw, xr = self._rows(x, "x")
        w, b = _parameter(weight, (cols,), "weight"), _parameter(bias, (cols,), "bias")
        if out is None:
            out, yw, yr = _empty_like(x, stream), rows * cols, cols
        else:
            yw, yr = self._rows_like(out, x, "out")
        mean = rstd = None
        if save:
            mean, rstd = _empty(x, (2,) + x.shape[:-1], torch.float32, stream).unbind(0)
        st = self.lib.qgx_layer_norm(self._h, code, wk, rows, cols, x.data_ptr(), xw, xr, w, b, eps, out.data_ptr(), yw, yr,
                                     mean.data_ptr() if save else None, rstd.data_ptr() if save else None, _handle(stream, x))
        if st:
            self._check(st)
        return out, mean, rstd

    def layer_norm_backward(self, dy, x, weight, mean, rstd, dw=None, db=None, dx=None, need_dx=True, stream=None):
        """Returns dx (None with need_dx=False) and writes the workers' weight and bias gradients, the sums over their
        rows, to dw and db: float32 [workers, cols], runs of V's rows say (or [cols] where x has no worker dimension)."""
        code, wk, rows, cols, xw, xr = self._rows(x, "x")
        gw, gr = self._rows_like(dy, x, "dy")
        w = _parameter(weight, (cols,), "weight")
        lead = x.shape[:-1]
        m, r = _parameter(mean, lead, "mean"), _parameter(rstd, lead, "rstd")
        step = None
        for t, name in ((dw, "dw"), (db, "db")):
            if t is None:
                continue
            _need(t.is_cuda and t.dtype == torch.float32 and (t.shape == (wk, cols) or (wk == 1 and t.shape == (cols,))) and _dense_last(t),
                  "%s: float32 [workers, cols] on the GPU", name)
            s = t.stride(0) if wk > 1 else cols
            _need(step is None or step == s, "dw and db: one step between workers")
            step = s
        ow = orow = 0
        if dx is not None:
            ow, orow = self._rows_like(dx, x, "dx")
        elif need_dx:
            dx, ow, orow = _empty_like(x, stream), rows * cols, cols
        need, scratch = self._need_bytes, None
        st = self.lib.qgx_layer_norm_scratch(self._h, code, wk, rows, cols, self._need_ref)
        if not st:
            if need.value:
                scratch = _empty(x, (need.value,), torch.uint8, stream)
            st = self.lib.qgx_layer_norm_backward(
                self._h, code, wk, rows, cols, dy.data_ptr(), gw, gr, x.data_ptr(), xw, xr, w, m, r,
                None if dx is None else dx.data_ptr(), ow, orow, None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                cols if step is None else step, None if scratch is None else scratch.data_ptr(), need.value, _handle(stream, x))
        if st:
            self._check(st)
        return dx

    @staticmethod
    def _scores(t, name):
        """[workers, batch, heads, q, k], [batch, heads, q, k] or [heads, q, k], keys contiguous."""
        code, sh, st = DTYPES.get(t.dtype), t.shape, t.stride()
        _need(code is not None and t.is_cuda, "%s: float32, float16 or bfloat16 on the GPU", name)
        n = len(sh)
        _need(3 <= n <= 5 and (st[-1] == 1 or sh[-1] <= 1), "%s: [workers, batch, heads, q, k], the last dimension contiguous", name)
        return _Scores(t.data_ptr(), code, sh[-3], sh[0] if n == 5 else 1, sh[-4] if n > 3 else 1, sh[-2], sh[-1],
                       st[0] if n == 5 else 0, st[-4] if n > 3 else 0, st[-3], st[-2])

    def _bias(self, table, buckets, src, out, q_offset, positions, stream):
        o = self._scores(out, "out")
        _need(abs(q_offset) <= 1 << 30, "q_offset: beyond +-2^30")
        _need(table.dim() == 2 and table.shape[1] == o.heads, "table: [rows, heads]")
        tab = _parameter(table, table.shape, "table")
        pos = None
        if positions is not None:
            _need(positions.is_cuda and positions.dtype == torch.int32 and positions.is_contiguous() and
                  positions.numel() == o.workers * o.batch, "positions: contiguous int32, one for every sequence, on the GPU")
            pos = positions.data_ptr()
        i = None if src is None else self._scores(src, "scores")
        st = self.lib.qgx_position_bias(self._h, buckets._ref, tab, table.shape[0], None if i is None else C.addressof(i),
                                        C.addressof(o), q_offset, pos, _handle(stream, out))
        if st:
            self._check(st)
        return out

    def position_bias(self, table, buckets: Buckets, q, k, dtype=torch.float32, q_offset=0, out=None, stream=None):
        """The bias alone, [heads, q, k]: table[row of (j - i - q_offset)][head], -inf where that is masked."""
        if out is None:
            out = _empty(table, (table.shape[1], q, k), dtype, stream)
        return self._bias(table, buckets, None, out, q_offset, None, stream)

    def add_position_bias(self, scores, table, buckets: Buckets, q_offset=0, positions=None, out=None, stream=None):
        """scores [.., batch, heads, q, k] plus the bias, -inf where a place is masked.  positions int32 [.., batch]: added to
        q_offset sequence by sequence (the position of its first query).  out may be scores."""
        if out is None:
            out = _empty_like(scores, stream)
        return self._bias(table, buckets, scores, out, q_offset, positions, stream)

    def position_bias_backward(self, grad, buckets: Buckets, dtable, q_offset=0, stream=None):
        """Writes the table's gradient, float32 [workers, rows, heads] (a run of V's rows say; [rows, heads] where grad has
        no worker dimension), from the gradient of the biased scores."""
        g = self._scores(grad, "grad")
        _need(abs(q_offset) <= 1 << 30, "q_offset: beyond +-2^30")
        sh, step = dtable.shape, dtable.stride()
        _need(dtable.is_cuda and dtable.dtype == torch.float32 and len(sh) == (3 if grad.dim() == 5 else 2) and sh[-1] == g.heads and
              (len(sh) == 2 or sh[0] == g.workers), "dtable: float32 [workers, rows, heads] on the GPU")
        rows = sh[-2]
        _need((rows <= 1 or step[-2] == g.heads) and (step[-1] == 1 or g.heads == 1), "dtable: a worker's table must be contiguous")
        need, scratch = self._need_bytes, None
        st = self.lib.qgx_position_bias_scratch(self._h, buckets._ref, C.addressof(g), q_offset, self._need_ref)
        if not st:
            if need.value:
                scratch = _empty(grad, (need.value,), torch.uint8, stream)
            st = self.lib.qgx_position_bias_backward(self._h, buckets._ref, C.addressof(g), q_offset, dtable.data_ptr(), rows,
                                                     step[0] if len(sh) == 3 and g.workers > 1 else rows * g.heads,
                                                     None if scratch is None else scratch.data_ptr(), need.value, _handle(stream, grad))
        if st:
            self._check(st)
        return dtable

    # -- DEQ o CODE and the fused updates ---------------------------------------------------------
    def decode(self, st: Stream, out=None, stream=None):
        if out is None:
            out = torch.empty((self.K, self.d), dtype=torch.float32, device=st.payload.device)
        s = st.c_struct()
        self._check(self.lib.qgx_decode(self._h, C.byref(s), _ptr(out), _stream_handle(stream)))
        return out

    def decode_average(self, st: Stream, out=None, stream=None):
        if out is None:
            out = torch.empty(self.d, dtype=torch.float32, device=st.payload.device)
        s = st.c_struct()
        self._check(self.lib.qgx_decode_average(self._h, C.byref(s), _ptr(out), _stream_handle(stream)))
        return out

    def fit_levels(self, V, n_sym, n_bins=4096, sweeps=10, hist_out=None, stream=None):
        self._check(self.lib.qgx_fit_levels(self._h, _ptr(V), C.c_uint32(n_sym), C.c_uint32(n_bins),
                                            C.c_uint32(sweeps), _ptr(hist_out), _stream_handle(stream)))

    def fit_code(self, stream=None):
        """Returns (p, code_len, code_bits) of the code the context now uses."""
        n = self._n_sym.get(self._table) or len(self.get_levels(stream))
        p = np.zeros(MAX_SYM, np.float64); cl = np.zeros(MAX_SYM, np.uint8); cb = np.zeros(MAX_SYM, np.uint32)
        self._check(self.lib.qgx_fit_code(self._h, p.ctypes.data_as(C.c_void_p), cl.ctypes.data_as(C.c_void_p),
                                          cb.ctypes.data_as(C.c_void_p), _stream_handle(stream)))
        return p[:n].copy(), cl[:n].copy(), cb[:n].copy()

    def state_init(self, X1=None, stream=None):
        self._check(self.lib.qgx_state_init(self._h, _ptr(X1), _stream_handle(stream)))

    def eg_step(self, half, cur: Stream, prev: Stream = None, X_out=None, stream=None, static=False):
        """static: through qgx_eg_step_static (scratch in the library's device image, nothing allocated)."""
        c = cur.c_struct()
        p = prev.c_struct() if prev is not None else None
        fn = self.lib.qgx_eg_step_static if static else self.lib.qgx_eg_step
        self._check(fn(self._h, C.c_int(half), C.byref(c), C.byref(p) if p is not None else None,
                       _ptr(X_out), _stream_handle(stream)))
        return X_out

    def select_table(self, table, prev_table=None):
        self._check(self.lib.qgx_select_table(self._h, C.c_uint32(table),
                                              C.c_uint32(table if prev_table is None else prev_table)))
        self._table = table

    def average_reset(self, on=True, stream=None):
        self._check(self.lib.qgx_average_reset(self._h, C.c_int(1 if on else 0), _stream_handle(stream)))

    def average_export(self, out=None, stream=None):
        """(X_bar [d], number of half-steps averaged)."""
        if out is None:
            out = torch.empty(self.d, dtype=torch.float32, device=self.device)
        n = C.c_uint64()
        self._check(self.lib.qgx_average_export(self._h, _ptr(out), C.byref(n), _stream_handle(stream)))
        return out, n.value

    def scalars(self, stream=None):
        S, g, t = C.c_double(), C.c_double(), C.c_uint64()
        self._check(self.lib.qgx_get_scalars(self._h, C.byref(S), C.byref(g), C.byref(t), _stream_handle(stream)))
        return dict(S=S.value, gamma=g.value, t=t.value)

    def stream_bits(self, coded: Stream, stream=None):
        """Code-word and sign bits of a coded stream over all workers (no padding, no norms)."""
        c, b = coded.c_struct(), C.c_uint64()
        self._check(self.lib.qgx_stream_bits(self._h, C.byref(c), C.byref(b), _stream_handle(stream)))
        return b.value

    def debug_set_waves_per_position(self, waves):
        self._check(self.lib.qgx_debug_set_waves_per_position(self._h, C.c_int(waves)))

    def state_export(self, stream=None):
        Y = torch.empty(self.d, dtype=torch.float32, device=self.device)
        A = torch.empty(self.d, dtype=torch.float32, device=self.device)
        self._check(self.lib.qgx_state_export(self._h, _ptr(Y), _ptr(A), _stream_handle(stream)))
        return Y, A

    def state_import(self, Y, anchor, S, t, stream=None):
        self._check(self.lib.qgx_state_import(self._h, _ptr(Y), _ptr(anchor), C.c_double(S), C.c_uint64(t),
                                              _stream_handle(stream)))

    def poll_error(self, stream=None):
        return int(self.lib.qgx_poll_error(self._h, _stream_handle(stream)))
