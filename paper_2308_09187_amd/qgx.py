"""Thin ctypes binding over libqgx.so (include/qgx.h): argument marshalling only.

Every step of the path runs in the library's gfx950 kernels; torch is used for device memory and
streams.  Loading fails loudly when the library has not been built
(``python -m paper_2308_09187_amd.build``); there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
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
KEPT_BLOCK = 32
ACTIVATIONS = {"none": 0, "silu": 1, "leaky": 2}
MAX_AXES, MAX_PAIRS = 4, 256
DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

EXPORTS = [
    "qgx_create", "qgx_destroy", "qgx_stream_sizes", "qgx_slot_words", "qgx_compact", "qgx_select_table", "qgx_set_levels", "qgx_get_levels", "qgx_set_code_table",
    "qgx_quantize", "qgx_encode", "qgx_quantize_encode", "qgx_decode", "qgx_decode_average", "qgx_fit_levels", "qgx_fit_code",
    "qgx_state_init", "qgx_eg_step", "qgx_eg_step_static", "qgx_average_reset", "qgx_average_export", "qgx_get_scalars", "qgx_stream_bits", "qgx_debug_set_waves_per_position", "qgx_state_export", "qgx_state_import",
    "qgx_poll_error", "qgx_last_error",
    "qgx_tensor_list_size", "qgx_tensor_list_set", "qgx_clip_gradients", "qgx_layer_norm", "qgx_layer_norm_scratch", "qgx_layer_norm_backward",
    "qgx_position_bias", "qgx_position_bias_scratch", "qgx_position_bias_backward",
    "qgx_checkpoint", "qgx_restore", "qgx_weight_gradient_scratch", "qgx_weight_gradient", "qgx_group_norm_scratch", "qgx_group_norm",
    "qgx_group_norm_backward", "qgx_rotate",
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


class _Kept(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("powers", C.c_void_p), ("rows", C.c_uint64), ("cols", C.c_uint64), ("tensor", C.c_uint32)]


class _GroupShape(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("activation", C.c_int32), ("slope", C.c_float), ("groups", C.c_uint32), ("workers", C.c_uint64),
                ("batch", C.c_uint64), ("places", C.c_uint64), ("channels", C.c_uint64)]


class _Places(C.Structure):
    _fields_ = [("data", C.c_void_p), ("s_worker", C.c_uint64), ("s_batch", C.c_uint64), ("s_place", C.c_uint64)]


class _Rotary(C.Structure):
    _fields_ = [("axes", C.c_uint32), ("pairs", C.c_uint32 * MAX_AXES), ("neighbours", C.c_int32), ("frequencies", C.POINTER(C.c_double))]


class _Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("heads", C.c_uint32), ("dim", C.c_uint32), ("workers", C.c_uint64),
                ("batch", C.c_uint64), ("tokens", C.c_uint64), ("s_worker", C.c_uint64), ("s_batch", C.c_uint64), ("s_token", C.c_uint64),
                ("s_head", C.c_uint64)]


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
        lib.qgx_checkpoint.argtypes = [ptr, C.c_int, u64, u64, u64, ptr, u64, u64, C.c_int, C.c_uint32, ptr, ptr]
        lib.qgx_restore.argtypes = [ptr, ptr, C.c_int, ptr, u64, ptr]
        lib.qgx_weight_gradient_scratch.argtypes = [ptr, C.c_int, u64, u64, u64, u64, u64, ptr]
        lib.qgx_weight_gradient.argtypes = [ptr, ptr, C.c_int, u64, u64, u64, ptr, u64, u64, ptr, u64, ptr, u64, ptr, u64, ptr]
        lib.qgx_group_norm_scratch.argtypes = [ptr, ptr, C.c_int, ptr]
        lib.qgx_group_norm.argtypes = [ptr, ptr, ptr, ptr, ptr, f32, ptr, ptr, ptr, ptr, C.c_int, C.c_uint32, ptr, u64, ptr]
        lib.qgx_group_norm_backward.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, u64, ptr, u64, ptr]
        lib.qgx_rotate.argtypes = [ptr, ptr, ptr, u64, u64, u64, ptr, ptr, C.c_int, ptr]
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


def _more(like, shape, stream):
    """Memory of like's type on its device (1.2 us)."""
    if stream is None:
        return like.new_empty(shape)
    with torch.cuda.stream(stream):
        return like.new_empty(shape)


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


class Checkpoint:
    """An activation kept in 8 bits, rows of `cols` elements in blocks of 32: codes uint8 [.., 32 * blocks] and powers uint8
    [.., blocks], contiguous; an element is (code - 128) * 2^(power - 127).  tensor: which of those kept under one call number, a
    number of its own for each.  Made by Context.new_checkpoint or Context.checkpoint, or from such tensors."""

    def __init__(self, codes, powers, cols, tensor=0):
        cols = int(cols)
        blocks = (cols + KEPT_BLOCK - 1) // KEPT_BLOCK
        for t, n, name in ((codes, KEPT_BLOCK * blocks, "codes"), (powers, blocks, "powers")):
            _need(t.is_cuda and t.dtype == torch.uint8 and t.is_contiguous() and t.dim() >= 1 and t.shape[-1] == n, "%s: contiguous uint8 [.., %d] on the GPU", name, n)
        _need(codes.shape[:-1] == powers.shape[:-1] and codes.get_device() == powers.get_device(), "codes and powers: of the same rows")
        self.shape, self._device = codes.shape[:-1] + (cols,), codes.get_device()
        self._memory, self._codes, self._powers = codes, codes, powers
        self._c = _Kept(codes.data_ptr(), powers.data_ptr(), math.prod(self.shape[:-1]), cols, _tensor_number(tensor))
        self._ref = C.addressof(self._c)

    @classmethod
    def _made(cls, like, shape, stream, tensor):
        """Memory for rows of this shape on the device of like, of bytes: one piece, of which codes and powers become tensors when they are asked for."""
        rows, split, size = _kept_layout(shape)
        k = cls.__new__(cls)
        k.shape, k._device, k._codes = shape, like.get_device(), None
        k._memory = _more(like, size, stream)
        at = k._memory.data_ptr()
        k._c = _Kept(at, at + split, rows, shape[-1], tensor)
        k._ref = C.addressof(k._c)
        return k

    def view(self, shape):
        """The same rows with other leading dimensions, for a call that counts them in another way; no memory of its own."""
        shape = torch.Size(shape)
        _need(len(shape) >= 1 and shape[-1] == self.shape[-1] and math.prod(shape[:-1]) == math.prod(self.shape[:-1]),
              "view: as many rows, of %d columns", self.shape[-1])
        k = Checkpoint.__new__(Checkpoint)
        k.shape, k._device, k._codes = shape, self._device, None
        if self._codes is None:
            k._memory = self._memory
        else:                                              # (codes and powers may be memory of their own)
            lead = shape[:-1]
            k._memory = k._codes = self._codes.view(lead + self._codes.shape[-1:])
            k._powers = self._powers.view(lead + self._powers.shape[-1:])
        k._c = _Kept(self._c.codes, self._c.powers, self._c.rows, self._c.cols, self._c.tensor)
        k._ref = C.addressof(k._c)
        return k

    def _parts(self):
        split = _kept_layout(self.shape)[1]
        lead = self.shape[:-1]
        blocks = (self.shape[-1] + KEPT_BLOCK - 1) // KEPT_BLOCK
        self._codes, self._powers = self._memory[:split].view(lead + (KEPT_BLOCK * blocks,)), self._memory[split:].view(lead + (blocks,))

    @property
    def tensor(self):
        return self._c.tensor

    @property
    def codes(self):
        if self._codes is None:
            self._parts()
        return self._codes

    @property
    def powers(self):
        if self._codes is None:
            self._parts()
        return self._powers


def _tensor_number(n):
    _need(0 <= n < 1 << 24, "tensor: a number below 2^24")
    return n


@functools.lru_cache(maxsize=256)
def _kept_layout(shape):
    """Rows, and bytes of their codes and of both."""
    rows, blocks = math.prod(shape[:-1]), (shape[-1] + KEPT_BLOCK - 1) // KEPT_BLOCK
    return rows, rows * blocks * KEPT_BLOCK, rows * blocks * (KEPT_BLOCK + 1)


class Rotary:
    """Rotary positions with several axes: the first pairs[0] pairs of a head turn with the token's position along axis 0, the next
    pairs[1] along axis 1, and so on, pair p by position * frequencies[p] radians.  neighbours: pair p is elements 2 p and
    2 p + 1 of a head, else p and p + the number of pairs."""

    def __init__(self, pairs, frequencies, neighbours=False):
        pairs, frequencies = [int(n) for n in pairs], [float(f) for f in frequencies]
        _need(1 <= len(pairs) <= MAX_AXES and all(n >= 0 for n in pairs) and 1 <= sum(pairs) <= MAX_PAIRS, "Rotary: 1 .. %d axes, 1 .. %d pairs", MAX_AXES, MAX_PAIRS)
        _need(len(frequencies) == sum(pairs) and all(math.isfinite(f * 2.0 ** 31) for f in frequencies),
              "Rotary: a frequency for every pair, finite at every position")
        self.pairs, self.neighbours = pairs, bool(neighbours)
        self.frequencies = (C.c_double * len(frequencies))(*frequencies)
        self._c = _Rotary(len(pairs), (C.c_uint32 * MAX_AXES)(*pairs), int(self.neighbours), self.frequencies)
        self._ref = C.addressof(self._c)

    @classmethod
    def by_base(cls, pairs, base=10000.0, neighbours=False):
        """Frequencies base^(-i / n), i = 0 .. n - 1, for an axis of n pairs."""
        return cls(pairs, [base ** (-i / n) for n in pairs for i in range(n)], neighbours)


class _GroupCall:
    """What is the same in every group norm of tensors of one shape, one type and the same steps."""

    def __init__(self, ctx, t, groups, activation, slope, backward, name):
        code, sh, act = DTYPES.get(t.dtype), t.shape, ACTIVATIONS.get(activation)
        n = len(sh)
        _need(code is not None and t.is_cuda and 2 <= n <= 4, "%s: [workers, batch, places, channels] of float32, float16 or bfloat16 on the GPU", name)
        _need(act is not None and 0 < groups < 1 << 32 and sh[-1] % groups == 0, "activation: none, silu or leaky; groups: a divisor of the channels")
        self.workers, batch = sh[0] if n == 4 else 1, sh[-3] if n > 2 else 1
        self.shape = _GroupShape(code, act, slope, groups, self.workers, batch, sh[-2], sh[-1])
        self.device, self.channels, self.statistics = t.get_device(), sh[-1:], sh[:-2] + (groups,)
        self.like = t.new_empty(0, dtype=torch.float32)
        self.both, self.gradients = (2,) + self.statistics, sh[:1] + sh[-1:] if n == 4 else sh[-1:]
        self.first = Context._places(t, name)            # t itself, x or dy
        run = sh[-2] * sh[-1]
        self.new = _Places(None, batch * run, run, sh[-1])                     # a new tensor of its shape
        self.shape_ref, self.first_ref, self.new_ref = C.addressof(self.shape), C.addressof(self.first), C.addressof(self.new)
        st = ctx.lib.qgx_group_norm_scratch(ctx._h, self.shape_ref, backward, ctx._need_ref)
        if st:
            ctx._check(st)
        self.scratch = ctx._need_bytes.value


def _looks(t):
    """All that a call's checks see of a tensor: shape, steps, type and device."""
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


class _GradientCall:
    """What is the same in every weight gradient of tensors that look alike."""

    def __init__(self, ctx, kept, dy, dw, db):
        _need(dy.dim() >= 2 and kept.shape[:-1] == dy.shape[:-1] and kept._device == dy.get_device(), "dy: [.., out] of the kept rows, on their device")
        cols, lead = kept.shape[-1], dy.shape[:1] if dy.dim() > 2 else ()
        if dy.dim() > 3:                                   # a worker's rows one step apart
            try:
                dy = dy.view(dy.shape[0], math.prod(dy.shape[1:-1]), dy.shape[-1])
            except RuntimeError:
                raise QgxError(ERR_ARG, "dy: dimensions between the first and the last that come down to rows of one step") from None
        self.rows = code, wk, rows, out, _, step = ctx._rows(dy, "dy")
        _need(dw is not None, "dw: where the gradient goes")
        for t, shape, name in ((dw, lead + (cols, out), "dw"), (db, lead + (out,), "db")):
            _need(t is None or (t.get_device() == dy.get_device() and t.dtype == torch.float32 and t.shape == shape and
                                (wk == 0 or (t[0] if lead else t).is_contiguous())),
                  "%s: float32 of shape %s, each worker's contiguous, on dy's device", name, tuple(shape))
        self.dw_step, self.db_step = dw.stride(0) if lead else 0, db.stride(0) if lead and db is not None else 0
        ctx._check(ctx.lib.qgx_weight_gradient_scratch(ctx._h, code, wk, rows, cols, out, step, ctx._need_ref))
        self.scratch = ctx._need_bytes.value


class _RotaryCall:
    """What is the same in every rotation of tensors that look alike.  out None: a new tensor."""

    def __init__(self, x, out, positions, axes):
        self.src = src = Context._heads(x, "x")
        if out is None:
            step = src.heads * src.dim
            self.dst = _Heads(None, src.dtype, src.heads, src.dim, src.workers, src.batch, src.tokens, src.batch * src.tokens * step, src.tokens * step, step, src.dim)
        else:
            _need(out.shape == x.shape and out.dtype == x.dtype and out.get_device() == x.get_device(), "out: of x's shape and type, on its device")
            self.dst = Context._heads(out, "out")
        ps, step, sh = positions.shape, positions.stride(), x.shape
        n = len(ps)
        _need(positions.dtype == torch.int32 and positions.get_device() == x.get_device() and n >= 2 and ps[0] == axes and ps[-1] == sh[-3] and
              (n == 2 or ps[1:] == sh[:-2]) and (ps[-1] <= 1 or step[-1] == 1),
              "positions: int32 [axes, tokens] or [axes, .., tokens], tokens contiguous, on x's device")
        self.steps = step[0], step[1] if n == 4 else 0, step[-2] if n > 2 else 0
        self.src_ref, self.dst_ref = C.addressof(self.src), C.addressof(self.dst)


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
        self._calls = {}                          # what calls of the same shapes share, by how their tensors look
        self._like = torch.empty(0, dtype=torch.uint8, device=device)
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

    # -- an image or video model's block --------------------------------------------------------------
    def _laid_out(self, key, call):
        if len(self._calls) >= 512:
            self._calls.clear()
        self._calls[key] = call
        return call

    def new_checkpoint(self, shape, stream=None, tensor=0):
        """Memory for an activation of this shape, the last dimension its columns (its contents are what checkpoint or group_norm put
        there).  tensor: its number in the draws, another for each of the activations that are kept under one call number."""
        shape = torch.Size(shape)
        _need(len(shape) >= 1 and shape[-1] >= 1, "new_checkpoint: columns")
        return Checkpoint._made(self._like, shape, stream, _tensor_number(tensor))

    @staticmethod
    def _kept_rows(x, name):
        """(type, workers, rows, cols, step between workers, between rows) of [.., cols] whose leading dimensions come down to two."""
        if x.dim() > 3:
            lead = [(n, s) for n, s in zip(x.shape[:-1], x.stride()[:-1]) if n != 1]          # (the step of a single index is nothing's)
            for cut in range(len(lead) + 1):               # [a .., b ..]: each run of dimensions one
                if x.numel() == 0 or all(lead[i - 1][1] == lead[i][1] * lead[i][0] for i in range(1, len(lead)) if i != cut):
                    x = x.view(math.prod(n for n, _ in lead[:cut]), math.prod(n for n, _ in lead[cut:]), x.shape[-1])
                    break
            _need(x.dim() == 3, "%s: leading dimensions that come down to two of one step each", name)
        return Context._rows(x, name)

    def checkpoint(self, x, call_id=None, out=None, stream=None, tensor=None):
        """Keeps x [.., cols] in 8 bits.  call_id None: rounded to nearest; a number (or CALL_FIRST_HALF, CALL_SECOND_HALF): without bias, by
        draws of that call and of the tensor's number (None: out's, or 0).  Tensors kept under one call number need numbers of their own: by the same
        draws, a gradient that has passed through the one would not be independent of the other."""
        code, wk, rows, cols, xw, xr = self._kept_rows(x, "x")
        if out is None:
            _need(cols >= 1, "x: columns")
            like = self._like
            if x.get_device() != like.get_device():
                like = x.new_empty(0, dtype=torch.uint8)
            out = Checkpoint._made(like, x.shape, stream, 0 if tensor is None else _tensor_number(tensor))
        else:
            _need(out.shape == x.shape and out._device == x.get_device(), "out: a checkpoint of x's shape, on its device")
            _need(tensor is None or tensor == out.tensor, "tensor: out has a number of its own")
        _need(call_id is None or 0 <= call_id < 1 << 32, "call_id: 32 bits")
        st = self.lib.qgx_checkpoint(self._h, code, wk, rows, cols, x.data_ptr(), xw, xr, call_id is not None, call_id or 0, out._ref, _handle(stream, x))
        if st:
            self._check(st)
        return out

    def restore(self, kept: Checkpoint, dtype=torch.float32, out=None, stream=None):
        """The kept elements, rounded once to dtype."""
        cols = kept.shape[-1]
        step = cols
        if out is None:
            _need(dtype in DTYPES, "dtype: float32, float16 or bfloat16")
            out = _empty(kept._memory, kept.shape, dtype, stream)
        else:
            _need(out.shape == kept.shape and out.dtype in DTYPES and out.get_device() == kept._device, "out: of the kept shape, on its device")
            if not out.is_contiguous():
                _need(out.dim() == 2 and out.stride(1) == 1, "out: contiguous, or [rows, cols] with contiguous rows")
                step = out.stride(0)
        st = self.lib.qgx_restore(self._h, kept._ref, DTYPES[out.dtype], out.data_ptr(), step, _handle(stream, out))
        if st:
            self._check(st)
        return out

    def weight_gradient(self, kept: Checkpoint, dy, dw, db=None, stream=None):
        """Gradients of x W + b from the kept x [workers, rows, cols] and dy [workers, rows, out], or [workers, batch, places, ..] of both, or [rows, ..]
        without workers (Checkpoint.view gives x the dimensions it needs): dw float32 [workers, cols, out] and db [workers, out], runs
        of V's rows say, are written.  Returns dw."""
        key = (kept.shape, kept._device, _looks(dy), _looks(dw), _looks(db))
        call = self._calls.get(key) or self._laid_out(key, _GradientCall(self, kept, dy, dw, db))
        code, wk, rows, out, gw, gr = call.rows
        size = call.scratch
        scratch = _empty(dy, (size,), torch.uint8, stream) if size else None
        st = self.lib.qgx_weight_gradient(self._h, kept._ref, code, wk, rows, out, dy.data_ptr(), gw, gr, dw.data_ptr(), call.dw_step,
                                          None if db is None else db.data_ptr(), call.db_step, scratch.data_ptr() if size else None, size, _handle(stream, dy))
        if st:
            self._check(st)
        return dw

    # (Checks of the calls below are written out, several to a condition: a call of a function for each costs as much as the launch.)
    @staticmethod
    def _places(t, name):
        """Address and steps of [workers, batch, places, channels], [batch, places, channels] or [places, channels]."""
        step = t.stride()
        n = len(step)
        if not (2 <= n <= 4 and (step[-1] == 1 or t.shape[-1] <= 1)):
            raise QgxError(ERR_ARG, "%s: [workers, batch, places, channels], channels contiguous" % name)
        if n == 4:
            return _Places(t.data_ptr(), step[0], step[1], step[2])
        return _Places(t.data_ptr(), 0, step[0] if n == 3 else 0, step[-2])

    @classmethod
    def _places_like(cls, t, like, name):
        """The same of a tensor of like's shape and type."""
        if not (t.shape == like.shape and t.dtype == like.dtype and t.get_device() == like.get_device()):
            raise QgxError(ERR_ARG, "%s: of x's shape and type, on its device" % name)
        return cls._places(t, name)

    def _group_call(self, t, groups, activation, slope, backward, name):
        """The call for tensors of t's shape, steps, type and device."""
        key = (t.shape, t.stride(), t.dtype, t.get_device(), groups, activation, slope, backward)
        return self._calls.get(key) or self._laid_out(key, _GroupCall(self, t, groups, activation, slope, backward, name))

    @staticmethod
    def _channel_parameter(t, call, name):
        """Address of a contiguous binary32 parameter of the channels, or of a run of one; None stays None."""
        if t is None:
            return None
        if not (t.shape == call.channels and t.dtype == torch.float32 and t.get_device() == call.device and (t.stride(0) == 1 or call.channels[0] == 1)):
            raise QgxError(ERR_ARG, "%s: contiguous float32 of %d channels on the device of the others" % (name, call.channels[0]))
        return t.data_ptr()

    @staticmethod
    def _group_statistic(t, call, name):
        """Address of a contiguous binary32 [workers, batch, groups], without the dimensions that dy has not."""
        if not (t is not None and t.shape == call.statistics and t.dtype == torch.float32 and t.get_device() == call.device and t.is_contiguous()):
            raise QgxError(ERR_ARG, "%s: contiguous float32 [.., groups] on dy's device" % name)
        return t.data_ptr()

    def group_norm(self, x, groups, weight=None, bias=None, eps=1e-5, activation="none", slope=0.01, keep=None, call_id=None, out=None, save=True,
                   stream=None):
        """Group norm of x [workers, batch, places, channels] (or without workers, or without both) and an activation: "none", "silu",
        "leaky" (slope).  Returns (y, mean, rstd), the last two [.., groups] for the backward pass (save=False: None; NaNs of no places).  keep: a
        Checkpoint in which x is kept as well, as checkpoint(x, call_id, out=keep) would."""
        call = self._group_call(x, groups, activation, slope, 0, "x")
        call.first.data = x.data_ptr()
        w, b = self._channel_parameter(weight, call, "weight"), self._channel_parameter(bias, call, "bias")
        if out is None:
            out, to = _empty_like(x, stream), call.new_ref
            call.new.data = out.data_ptr()
        else:
            dst = self._places_like(out, x, "out")
            to = C.addressof(dst)
        kept, unbiased = None, 0
        if keep is not None:
            unbiased = call_id is not None
            if keep.shape != x.shape or keep._device != call.device or (unbiased and not 0 <= call_id < 1 << 32):
                raise QgxError(ERR_ARG, "keep: a checkpoint of x's shape, on its device; call_id: 32 bits")
            kept = keep._ref
        mean = rstd = m = r = None
        if save:
            mean, rstd = _more(call.like, call.both, stream).unbind(0)
            m, r = mean.data_ptr(), rstd.data_ptr()
        size = call.scratch
        scratch = _empty(x, (size,), torch.uint8, stream) if size else None
        st = self.lib.qgx_group_norm(self._h, call.shape_ref, call.first_ref, w, b, eps, to, m, r, kept, unbiased, call_id or 0,
                                     scratch.data_ptr() if size else None, size, _handle(stream, x))
        if st:
            self._check(st)
        return out, mean, rstd

    def group_norm_backward(self, dy, x, groups, weight, bias, mean, rstd, activation="none", slope=0.01, dw=None, db=None, dx=None, need_dx=True,
                            stream=None):
        """Returns dx (None with need_dx=False) and writes the workers' weight and bias gradients to dw and db, float32 [workers, channels], runs
        of V's rows say ([channels] where dy has no worker dimension).  x: the forward pass's input, or a Checkpoint of it."""
        call = self._group_call(dy, groups, activation, slope, 1, "dy")
        dev, src, kept = call.device, None, None
        call.first.data = dy.data_ptr()
        if isinstance(x, Checkpoint):
            if x.shape != dy.shape or x._device != dev:
                raise QgxError(ERR_ARG, "x: a checkpoint of dy's shape, on its device")
            kept = x._ref
        else:
            places = self._places_like(x, dy, "x")
            src = C.addressof(places)
        w, b = self._channel_parameter(weight, call, "weight"), self._channel_parameter(bias, call, "bias")
        m, r = self._group_statistic(mean, call, "mean"), self._group_statistic(rstd, call, "rstd")
        step, to = None, [None, None]
        for i, t in enumerate((dw, db)):
            if t is None:
                continue
            if not (t.shape == call.gradients and t.dtype == torch.float32 and t.get_device() == dev and (t.stride(-1) == 1 or call.channels[0] == 1)):
                raise QgxError(ERR_ARG, "dw and db: float32 [workers, channels] on dy's device")
            one = t.stride(0) if call.workers > 1 else call.channels[0]
            if step is not None and step != one:
                raise QgxError(ERR_ARG, "dw and db: one step between workers")
            step = one
            to[i] = t.data_ptr()
        dst = None
        if dx is not None:
            out = self._places_like(dx, dy, "dx")
            dst = C.addressof(out)
        elif need_dx:
            dx, dst = _empty_like(dy, stream), call.new_ref
            call.new.data = dx.data_ptr()
        size = call.scratch
        scratch = _empty(dy, (size,), torch.uint8, stream) if size else None
        st = self.lib.qgx_group_norm_backward(self._h, call.shape_ref, call.first_ref, src, kept, w, b, m, r, dst, to[0], to[1],
                                              call.channels[0] if step is None else step, scratch.data_ptr() if size else None, size, _handle(stream, dy))
        if st:
            self._check(st)
        return dx

    @staticmethod
    def _heads(t, name):
        """[workers, batch, tokens, heads, dim], [batch, tokens, heads, dim] or [tokens, heads, dim], a head's elements contiguous."""
        code, sh, st = DTYPES.get(t.dtype), t.shape, t.stride()
        n = len(sh)
        if not (code is not None and t.is_cuda and 3 <= n <= 5 and (st[-1] == 1 or sh[-1] <= 1) and sh[-2] < 1 << 32 and sh[-1] < 1 << 32):
            raise QgxError(ERR_ARG, "%s: [workers, batch, tokens, heads, dim] of float32, float16 or bfloat16 on the GPU, the last dimension contiguous" % name)
        return _Heads(t.data_ptr(), code, sh[-2], sh[-1], sh[0] if n == 5 else 1, sh[-4] if n > 3 else 1, sh[-3], st[0] if n == 5 else 0,
                      st[-4] if n > 3 else 0, st[-3], st[-2])

    def rotary(self, x, rotary: Rotary, positions, back=False, out=None, stream=None):
        """x [.., batch, tokens, heads, dim] turned by its tokens' positions, int32 [axes, tokens] (the same for all sequences) or [axes, ..,
        tokens] of x's leading dimensions.  back: by the angles' negatives, the backward pass.  out may be x."""
        new = out is None
        if new:
            out = _empty_like(x, stream)
        key = (_looks(x), _looks(positions), len(rotary.pairs), None if new else _looks(out))
        call = self._calls.get(key) or self._laid_out(key, _RotaryCall(x, None if new else out, positions, len(rotary.pairs)))
        call.src.data, call.dst.data = x.data_ptr(), out.data_ptr()
        axis, worker, batch = call.steps
        st = self.lib.qgx_rotate(self._h, rotary._ref, positions.data_ptr(), axis, worker, batch, call.src_ref, call.dst_ref, back, _handle(stream, x))
        if st:
            self._check(st)
        return out

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
