"""ctypes binding of ``libsirllm.so``: same names as the C ABI, argument marshalling only.

Every function takes CUDA torch tensors (device memory owned by the caller), checks
dtypes and contiguity, passes raw pointers and the current CUDA stream to the library
and raises :class:`SirllmError` on a negative return code.  There is no CPU fallback:
if the library is missing or a tensor is not on a CUDA device the call raises.
"""
from __future__ import annotations

import ctypes
import os
import threading
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsirllm.so")

F32, BF16, F16 = 0, 1, 2
OK, ERR_NULL, ERR_BAD_CONFIG, ERR_ALIGN, ERR_CUDA, ERR_TOO_LARGE = 0, -1, -2, -3, -4, -5
STATUS_TOKEN_RANGE, STATUS_OVERFLOW, STATUS_TIMEOUT, STATUS_BAD_KEEP, STATUS_BAD_SOURCE = 1, 2, 4, 8, 16
MAX_CAPACITY = 49152
MAX_ATTEND_HEAD_DIM = 256
MAX_BEAMS, MAX_GROUP, MAX_BEAM_VOCAB = 64, 256, 1 << 26
POLICY_STREAM, POLICY_RANDOM, POLICY_INTERVAL = 1, 2, 3
ROPE_HALF, ROPE_INTERLEAVED = 0, 1

EXPORTS = ["sirllm_workspace_bytes", "sirllm_workspace_init", "sirllm_score", "sirllm_score_static",
           "sirllm_score_partial",
           "sirllm_score_pairs", "sirllm_step_pairs", "sirllm_decay_select", "sirllm_keep_policy", "sirllm_rerotate_keys",
           "sirllm_append_kv", "sirllm_attend_workspace_bytes", "sirllm_attend_workspace_init", "sirllm_attend",
           "sirllm_attend_shared_workspace_bytes", "sirllm_attend_shared_workspace_init", "sirllm_attend_shared",
           "sirllm_beam_workspace_bytes", "sirllm_beam_workspace_init", "sirllm_beam_select", "sirllm_reorder_streams",
           "sirllm_head_tiles", "sirllm_head_pairs",
           "sirllm_compact_kv", "sirllm_step", "sirllm_step_phases", "sirllm_step_host",
           "sirllm_selftest_bounded_wait", "sirllm_status", "sirllm_strerror",
           "sirllm_last_cuda_error"]

_DTYPE_CODE = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_KV = (torch.bfloat16, torch.float16)


class SirllmError(RuntimeError):
    def __init__(self, code: int, detail: str = ""):
        self.code = code
        super().__init__(f"sirllm error {code}: {detail}")


class Config(ctypes.Structure):
    """Mirror of ``sirllm_config``."""
    _fields_ = [("n_streams", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32),
                ("threshold", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("logits_dtype", ctypes.c_int32),
                ("vocab", ctypes.c_int64), ("logits_row_stride", ctypes.c_int64)]

    @property
    def planes_per_stream(self) -> int:
        return self.n_layers * self.n_kv_heads


def make_config(n_streams, n_layers, n_kv_heads, head_dim, capacity, budget, n_sink, n_recent,
                max_new, vocab, logits_dtype, kv_dtype, threshold=None, logits_row_stride=None) -> Config:
    code = lambda d: _DTYPE_CODE[d] if isinstance(d, torch.dtype) else {"f32": F32, "bf16": BF16, "f16": F16}[d]
    return Config(n_streams, n_layers, n_kv_heads, head_dim, capacity, budget, n_sink, n_recent,
                  budget if threshold is None else threshold, max_new, code(kv_dtype),
                  code(logits_dtype), vocab, vocab if logits_row_stride is None else logits_row_stride)


def config_from_workload(w, **overrides) -> Config:
    """Config for a :class:`workloads.Workload`."""
    kw = dict(n_streams=w.n_streams, n_layers=w.n_layers, n_kv_heads=w.n_kv_heads,
              head_dim=w.head_dim, capacity=w.capacity, budget=w.budget, n_sink=w.n_sink,
              n_recent=w.n_recent, max_new=w.new_tokens, vocab=w.vocab,
              logits_dtype=w.logits_dtype, kv_dtype=w.kv_dtype, threshold=w.threshold)
    kw.update(overrides)
    return make_config(**kw)


_lib = None


def lib():
    """The loaded library; raises if it was not built (``python -m paper_2405_12528_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            # a source checkout: compile once with nvcc; without a compiler this fails loudly
            try:
                from . import build as _build
                _build.build()
            except Exception as exc:
                raise SirllmError(ERR_CUDA, f"{_LIB_PATH} is not built and could not be compiled "
                                            f"({exc}); run paper_2405_12528_b200/build.py") from exc
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, cfgp = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(Config)
        L.sirllm_workspace_bytes.restype = ctypes.c_size_t
        L.sirllm_workspace_bytes.argtypes = [cfgp]
        L.sirllm_workspace_init.restype = ctypes.c_int
        L.sirllm_workspace_init.argtypes = [cfgp, vp, vp]
        L.sirllm_score.restype = ctypes.c_int
        L.sirllm_score.argtypes = [cfgp, vp, vp, vp, vp, vp, vp]
        L.sirllm_score_static.restype = ctypes.c_int
        L.sirllm_score_static.argtypes = [cfgp, vp, vp, vp, vp, vp, vp]
        L.sirllm_score_partial.restype = ctypes.c_int
        L.sirllm_score_partial.argtypes = [cfgp, vp, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, vp, vp,
                                           vp, ctypes.c_int64, vp, vp, vp]
        L.sirllm_score_pairs.restype = ctypes.c_int
        L.sirllm_score_pairs.argtypes = [cfgp, vp, i32, ctypes.c_int64, vp, vp, vp, vp, vp, vp]
        L.sirllm_step_pairs.restype = ctypes.c_int
        L.sirllm_step_pairs.argtypes = [cfgp, vp, i32, ctypes.c_int64] + [vp] * 14
        L.sirllm_decay_select.restype = ctypes.c_int
        L.sirllm_decay_select.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
        L.sirllm_keep_policy.restype = ctypes.c_int
        L.sirllm_keep_policy.argtypes = [cfgp, i32, vp, ctypes.c_uint64, i32, i32, vp, vp, vp, vp]
        L.sirllm_rerotate_keys.restype = ctypes.c_int
        L.sirllm_rerotate_keys.argtypes = [cfgp, vp, vp, vp, ctypes.c_double, i32, vp]
        i64, f32 = ctypes.c_int64, ctypes.c_float
        L.sirllm_append_kv.restype = ctypes.c_int
        L.sirllm_append_kv.argtypes = [cfgp, i32, vp, i32, i64, vp, i64, vp, i64, vp, vp, f32, ctypes.c_double,
                                       i32, vp, vp, vp, i64, vp, vp, vp, vp]
        L.sirllm_attend_workspace_bytes.restype = ctypes.c_size_t
        L.sirllm_attend_workspace_bytes.argtypes = [cfgp]
        L.sirllm_attend_workspace_init.restype = ctypes.c_int
        L.sirllm_attend_workspace_init.argtypes = [cfgp, vp, vp]
        L.sirllm_attend.restype = ctypes.c_int
        L.sirllm_attend.argtypes = [cfgp, i32, vp, i32, i64, vp, vp, vp, f32, vp, i64, vp, vp, vp]
        L.sirllm_attend_shared_workspace_bytes.restype = ctypes.c_size_t
        L.sirllm_attend_shared_workspace_bytes.argtypes = [cfgp, i32, i32]
        L.sirllm_attend_shared_workspace_init.restype = ctypes.c_int
        L.sirllm_attend_shared_workspace_init.argtypes = [cfgp, i32, i32, vp, vp]
        L.sirllm_attend_shared.restype = ctypes.c_int
        L.sirllm_attend_shared.argtypes = [cfgp, i32, i32, vp, vp, i32, i64, vp, vp, vp, f32, vp, i64, vp, vp, vp]
        L.sirllm_beam_workspace_bytes.restype = ctypes.c_size_t
        L.sirllm_beam_workspace_bytes.argtypes = [cfgp]
        L.sirllm_beam_workspace_init.restype = ctypes.c_int
        L.sirllm_beam_workspace_init.argtypes = [cfgp, vp, vp]
        L.sirllm_beam_select.restype = ctypes.c_int
        L.sirllm_beam_select.argtypes = [cfgp, vp, i32, i32, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        L.sirllm_reorder_streams.restype = ctypes.c_int
        L.sirllm_reorder_streams.argtypes = [cfgp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.sirllm_head_tiles.restype = i32
        L.sirllm_head_tiles.argtypes = [cfgp, i64]
        L.sirllm_head_pairs.restype = ctypes.c_int
        L.sirllm_head_pairs.argtypes = [cfgp, vp, i64, vp, i64, i32, i32, i64, i64, vp, vp, vp, i64, vp, vp, vp]
        L.sirllm_compact_kv.restype = ctypes.c_int
        L.sirllm_compact_kv.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.sirllm_step.restype = ctypes.c_int
        L.sirllm_step.argtypes = [cfgp] + [vp] * 14
        L.sirllm_step_phases.restype = ctypes.c_int
        L.sirllm_step_phases.argtypes = [cfgp] + [vp] * 14 + [ctypes.POINTER(vp)]
        L.sirllm_step_host.restype = ctypes.c_int
        L.sirllm_step_host.argtypes = [cfgp] + [vp] * 23
        L.sirllm_selftest_bounded_wait.restype = ctypes.c_int
        L.sirllm_selftest_bounded_wait.argtypes = [cfgp, vp, ctypes.c_uint32, vp]
        L.sirllm_status.restype = ctypes.c_int
        L.sirllm_status.argtypes = [vp, vp, ctypes.POINTER(i32), i32]
        L.sirllm_strerror.restype = ctypes.c_char_p
        L.sirllm_strerror.argtypes = [ctypes.c_int]
        L.sirllm_last_cuda_error.restype = ctypes.c_char_p
        L.sirllm_last_cuda_error.argtypes = []
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != OK:
        L = lib()
        detail = L.sirllm_strerror(rc).decode()
        if rc == ERR_CUDA:
            detail += ": " + L.sirllm_last_cuda_error().decode()
        raise SirllmError(rc, detail)


class _Arg:
    """One tensor argument and what the configuration demands of it.  The C side sees plain
    pointers and no sizes, so every call checks ALL its arguments here first - dtype and
    element count, then residence (right kind of memory, contiguous, on the current device) -
    and only then hands out pointers."""

    def __init__(self, t, dtype, name, numel=0, host=False):
        self.t, self.dtype, self.name, self.numel, self.host = t, dtype, name, numel, host

    def check_shape(self):
        t = self.t
        if t is None:
            return
        if self.dtype is not None and t.dtype not in (self.dtype if isinstance(self.dtype, tuple) else (self.dtype,)):
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} has dtype {t.dtype}")
        if t.numel() < self.numel:
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} holds {t.numel()} elements, the "
                                              f"configuration needs {self.numel}")

    def check_residence(self):
        t = self.t
        if t is None:
            return
        if self.host:
            if t.is_cuda or not t.is_contiguous():
                raise SirllmError(ERR_ALIGN, f"{self.name} must be a contiguous host tensor")
            return
        if not t.is_cuda:
            raise SirllmError(ERR_NULL, f"{self.name} must be a CUDA tensor (there is no CPU path)")
        if not t.is_contiguous() and self.dtype is not None:
            raise SirllmError(ERR_ALIGN, f"{self.name} must be contiguous")
        if t.device.index != torch.cuda.current_device():
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} lives on {t.device}, the current device "
                                              f"is cuda:{torch.cuda.current_device()}")

    def ptr(self):
        return None if self.t is None else self.t.data_ptr()


def _dev(t, dtype=None, name="tensor", numel: int = 0) -> _Arg:
    return _Arg(t, dtype, name, numel)


class Prepared:
    """A call whose arguments were checked and marshalled once (see :func:`prepared`): calling
    it again costs one ctypes call.  It keeps its tensors alive and reads the current CUDA
    stream at every call; it refuses to be called with another device current than the one it
    was prepared on, where its pointers mean nothing."""

    def __init__(self, fn, cfg, args):
        self._fn, self._cfg = fn, Config.from_buffer_copy(cfg)
        self._keep = [a.t for a in args if isinstance(a, _Arg)]
        # arguments as instances of the C types, converted once
        self._stream = ctypes.c_void_p()
        raw = [self._stream if isinstance(a, _CurrentStream) else a.ptr() if isinstance(a, _Arg) else a for a in args]
        self._args = [ctypes.byref(self._cfg)] + [
            t(a) if t in _PLAIN and not isinstance(a, t) else a for t, a in zip(fn.argtypes[1:], raw)]
        self._device = _current_device()

    def __call__(self) -> None:
        current = _current_device()
        if current != self._device:
            raise SirllmError(ERR_BAD_CONFIG, f"the call was prepared on cuda:{self._device}, the current device "
                                              f"is cuda:{current}")
        self._stream.value = _raw_stream(self._device)
        rc = self._fn(*self._args)
        if rc != OK:
            _check(rc)


_PLAIN = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float,
          ctypes.c_double)


# The current device's index, and the handle of a device's current stream: torch's short ways where
# this torch has them.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


_preparing = threading.local()


def prepared(func, *args, **kwargs) -> Prepared:
    """``prepared(sirllm_step, cfg, logits, ...)`` checks and marshals the arguments of one of
    this module's calls once and returns a :class:`Prepared` that issues exactly that call
    (same tensors, whatever they hold by then) each time it is invoked - for loops that repeat
    a call thousands of times a second, where the per-argument checks would dominate."""
    _preparing.out = None
    _preparing.on = True
    try:
        func(*args, **kwargs)
    finally:
        _preparing.on = False
    if _preparing.out is None:
        raise SirllmError(ERR_BAD_CONFIG, f"{getattr(func, '__name__', func)} cannot be prepared")
    return _preparing.out


_int32_places = {}   # of every call's arguments, those that are 32-bit numbers


def _fits(n: int) -> bool:
    """Whether ctypes hands ``n`` on as it is (it cuts larger numbers down to 32 bits without a word)."""
    return -2**31 <= n < 2**31


def _call(fn, cfg, *args) -> None:
    """Checks every argument (numbers, then the shapes of all tensors, then their residence), then calls
    ``fn`` (or, under :func:`prepared`, hands back the marshalled call instead of making it)."""
    places = _int32_places.get(fn.__name__)
    if places is None:
        places = _int32_places[fn.__name__] = [i for i, t in enumerate(fn.argtypes[1:]) if t is ctypes.c_int32]
    for i in places:
        if not _fits(args[i]):
            raise SirllmError(ERR_BAD_CONFIG, f"{args[i]} does not fit 32 bits")
    for a in args:
        if isinstance(a, _Arg):
            a.check_shape()
    for a in args:
        if isinstance(a, _Arg):
            a.check_residence()
    if getattr(_preparing, "on", False):
        _preparing.out = Prepared(fn, cfg, args)
        return
    raw = [a.ptr() if isinstance(a, _Arg) else _stream_handle() if isinstance(a, _CurrentStream) else a
           for a in args]
    _check(fn(ctypes.byref(cfg), *raw))


class _CurrentStream:
    """Placeholder for the current CUDA stream's handle, looked up after the argument checks."""


def _stream() -> _CurrentStream:
    return _CurrentStream()


def _stream_handle() -> int:
    return torch.cuda.current_stream().cuda_stream


def _rows(cfg: Config) -> int:
    return cfg.n_streams * cfg.max_new


def _kv_numel(cfg: Config) -> int:
    return cfg.n_streams * cfg.n_layers * cfg.n_kv_heads * cfg.capacity * cfg.head_dim


class _KvArg(_Arg):
    def __init__(self, cfg, t, name):
        super().__init__(t, _KV, name, _kv_numel(cfg))
        self.code = cfg.kv_dtype

    def check_shape(self):
        super().check_shape()
        if self.t is not None and _DTYPE_CODE.get(self.t.dtype) != self.code:
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} dtype {self.t.dtype} does not match the config")


def _kv(cfg: Config, t, name) -> _Arg:
    return _KvArg(cfg, t, name)


def _ws(cfg: Config, ws) -> _Arg:
    return _dev(ws, torch.uint8, "ws", sirllm_workspace_bytes(cfg))


class _LogitsArg(_Arg):
    """A logits matrix [>= rows, vocab] whose rows are logits_row_stride elements apart
    (a column slice of a wider buffer is fine: only the last dimension must be dense)."""

    def __init__(self, cfg, t, name="logits", host=False, rows=None):
        super().__init__(t, None, name, 0, host)
        self.cfg, self.rows = cfg, _rows(cfg) if rows is None else rows

    def check_shape(self):
        cfg, t = self.cfg, self.t
        if t is None:
            return
        if _DTYPE_CODE.get(t.dtype) != cfg.logits_dtype:
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} dtype {t.dtype} does not match the config")
        rows = self.rows
        if t.dim() != 2 or t.shape[1] != cfg.vocab or t.shape[0] < rows:
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} has shape {tuple(t.shape)}, the "
                                              f"configuration needs [>= {rows}, {cfg.vocab}]")
        if t.stride(1) != 1 or (t.shape[0] > 1 and t.stride(0) != cfg.logits_row_stride):
            raise SirllmError(ERR_ALIGN, f"{self.name} rows must be logits_row_stride elements apart")

    def check_residence(self):
        if self.host and self.t is not None:
            if self.t.is_cuda:
                raise SirllmError(ERR_ALIGN, f"{self.name} must be a host tensor")
            return
        super().check_residence()


def _logits(cfg: Config, logits) -> _Arg:
    return _LogitsArg(cfg, logits)


class _PairsArg(_Arg):
    """Per-tile (max, sum exp) pairs [>= rows, n_tiles, 2], fp32, pairs contiguous."""

    def __init__(self, cfg, t):
        super().__init__(t, None, "pairs")
        self.cfg = cfg

    def check_shape(self):
        t = self.t
        if t is None:
            raise SirllmError(ERR_NULL, "pairs is required")
        if t.dtype != torch.float32:
            raise SirllmError(ERR_BAD_CONFIG, "pairs must be float32")
        if t.dim() != 3 or t.shape[2] != 2 or t.stride(2) != 1 or t.stride(1) != 2:
            raise SirllmError(ERR_ALIGN, "pairs must be [rows, n_tiles, 2] with contiguous pairs")
        if t.shape[0] < _rows(self.cfg):
            raise SirllmError(ERR_BAD_CONFIG, f"pairs hold {t.shape[0]} rows, the configuration "
                                              f"needs {_rows(self.cfg)}")

    @property
    def n_tiles(self) -> int:
        return int(self.t.shape[1])

    @property
    def row_stride(self) -> int:
        return int(self.t.stride(0) // 2 if self.t.shape[0] > 1 else self.t.shape[1])


def sirllm_workspace_bytes(cfg: Config) -> int:
    return lib().sirllm_workspace_bytes(ctypes.byref(cfg))


def new_workspace(cfg: Config, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and initialises a workspace for ``cfg``."""
    n = sirllm_workspace_bytes(cfg)
    if n == 0:
        raise SirllmError(ERR_BAD_CONFIG, "invalid configuration")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    sirllm_workspace_init(cfg, ws)
    return ws


def sirllm_workspace_init(cfg: Config, ws: torch.Tensor) -> None:
    _call(lib().sirllm_workspace_init, cfg, _ws(cfg, ws), _stream())


def _score_args(cfg: Config, token_ids, n_new, out_entropy):
    return (_dev(token_ids, torch.int32, "token_ids", _rows(cfg)),
            _dev(n_new, torch.int32, "n_new", cfg.n_streams),
            _dev(out_entropy, torch.float32, "out_entropy", _rows(cfg)))


def sirllm_score(cfg: Config, logits, token_ids, n_new, out_entropy, ws) -> None:
    _call(lib().sirllm_score, cfg, _logits(cfg, logits), *_score_args(cfg, token_ids, n_new, out_entropy),
          _ws(cfg, ws), _stream())


def sirllm_score_static(cfg: Config, logits, token_ids, n_new, out_entropy, status=None) -> None:
    """``sirllm_score`` without a workspace: for callers that cannot allocate device memory
    (the scratch is a fixed array inside the library; at most 16384 logits rows per call,
    and calls that overlap on the GPU race).  ``status``: optional int32 device word."""
    _call(lib().sirllm_score_static, cfg, _logits(cfg, logits),
          *_score_args(cfg, token_ids, n_new, out_entropy), _dev(status, torch.int32, "status", 1),
          _stream())


class _SliceArg(_Arg):
    """One rank's column range of the logits: [>= rows, n_cols], last dimension dense."""

    def __init__(self, cfg, t, col0):
        super().__init__(t, None, "logits_slice")
        self.cfg, self.col0 = cfg, int(col0)

    def check_shape(self):
        cfg, t = self.cfg, self.t
        if t is None:
            raise SirllmError(ERR_NULL, "logits_slice is required")
        if _DTYPE_CODE.get(t.dtype) != cfg.logits_dtype:
            raise SirllmError(ERR_BAD_CONFIG, f"logits_slice dtype {t.dtype} does not match the config")
        if t.dim() != 2 or t.shape[0] < _rows(cfg) or self.col0 < 0 or self.col0 + t.shape[1] > cfg.vocab:
            raise SirllmError(ERR_BAD_CONFIG, f"logits_slice has shape {tuple(t.shape)} at column "
                                              f"{self.col0}, the configuration needs [>= {_rows(cfg)}, "
                                              f"<= {cfg.vocab - self.col0}]")
        if t.shape[1] > 0 and t.stride(1) != 1:
            raise SirllmError(ERR_ALIGN, "logits_slice rows must be dense")

    @property
    def row_stride(self) -> int:
        t = self.t
        return int(t.stride(0)) if t.shape[0] > 1 and t.shape[1] > 0 else max(int(t.shape[1]), 1)


def sirllm_score_partial(cfg: Config, logits_slice, col0: int, token_ids, n_new, pairs_out, target_out,
                         ws, pair_column: int = 0) -> None:
    """One rank's share of vocabulary-parallel scoring: ``logits_slice`` holds columns
    ``[col0, col0 + n_cols)``; ``pairs_out`` is ``[rows, n_ranks, 2]`` fp32 and this call fills
    column ``pair_column`` of it; ``target_out`` is fp32 ``[rows]``."""
    sl = _SliceArg(cfg, logits_slice, col0)
    sl.check_shape()
    pa = _PairsArg(cfg, pairs_out)
    pa.check_shape()
    if not 0 <= pair_column < pa.n_tiles:
        raise SirllmError(ERR_BAD_CONFIG, f"pair_column {pair_column} outside [0, {pa.n_tiles})")
    ids, nn, tgt = _score_args(cfg, token_ids, n_new, target_out)
    tgt.name = "target_out"
    pa.check_residence()
    _call(lib().sirllm_score_partial, cfg, sl, int(col0), int(logits_slice.shape[1]), sl.row_stride,
          ids, nn, pairs_out.data_ptr() + 8 * int(pair_column), pa.row_stride, tgt, _ws(cfg, ws), _stream())


def sirllm_score_pairs(cfg: Config, pairs, target_logit, token_ids, n_new, out_entropy, ws) -> None:
    """Scores from per-tile ``(max, sum exp)`` pairs ``[rows, n_tiles, 2]`` and target logits."""
    pa = _PairsArg(cfg, pairs)
    pa.check_shape()
    _call(lib().sirllm_score_pairs, cfg, pa, pa.n_tiles, pa.row_stride,
          _dev(target_logit, torch.float32, "target_logit", _rows(cfg)),
          *_score_args(cfg, token_ids, n_new, out_entropy), _ws(cfg, ws), _stream())


def _state_args(cfg: Config, scores, serial, live_len, decay):
    per_slot = cfg.n_streams * cfg.capacity
    return (_dev(scores, torch.float32, "scores", per_slot),
            _dev(serial, torch.int64, "serial", per_slot),
            _dev(live_len, torch.int32, "live_len", cfg.n_streams),
            _dev(decay, torch.float32, "decay", cfg.n_streams))


def _keep_args(cfg: Config, keep_idx, n_keep):
    return (_dev(keep_idx, torch.int32, "keep_idx", cfg.n_streams * cfg.threshold),
            _dev(n_keep, torch.int32, "n_keep", cfg.n_streams))


def _round_args(cfg: Config, token_ids, n_new, scores, serial, live_len, decay, k, v, keep_idx, n_keep,
                new_entropy, ws):
    """The arguments sirllm_step, _step_pairs, _step_phases and _step_host share, in ABI order."""
    ids, nn, ent = _score_args(cfg, token_ids, n_new, new_entropy)
    return (ids, nn) + _state_args(cfg, scores, serial, live_len, decay) + \
        (_kv(cfg, k, "k"), _kv(cfg, v, "v")) + _keep_args(cfg, keep_idx, n_keep) + (ent, _ws(cfg, ws))


def sirllm_step_pairs(cfg: Config, pairs, target_logit, token_ids, n_new, scores, serial, live_len,
                      decay, k, v, keep_idx, n_keep, new_entropy, ws) -> None:
    pa = _PairsArg(cfg, pairs)
    pa.check_shape()
    _call(lib().sirllm_step_pairs, cfg, pa, pa.n_tiles, pa.row_stride,
          _dev(target_logit, torch.float32, "target_logit", _rows(cfg)),
          *_round_args(cfg, token_ids, n_new, scores, serial, live_len, decay, k, v, keep_idx, n_keep,
                       new_entropy, ws), _stream())


def sirllm_decay_select(cfg: Config, scores, serial, live_len, decay, keep_idx, n_keep,
                        compact_scores, ws) -> None:
    _call(lib().sirllm_decay_select, cfg, *_state_args(cfg, scores, serial, live_len, decay),
          *_keep_args(cfg, keep_idx, n_keep), int(bool(compact_scores)), _ws(cfg, ws), _stream())


def sirllm_keep_policy(cfg: Config, policy: int, live_len, seed: int, rnd: int, stream_base: int,
                       keep_idx, n_keep, ws) -> None:
    """Keep lists of StreamLLM / RandomLLM / IntervalLLM (``POLICY_*``) for ``sirllm_compact_kv``."""
    _call(lib().sirllm_keep_policy, cfg, int(policy), _dev(live_len, torch.int32, "live_len", cfg.n_streams),
          int(seed), int(rnd), int(stream_base), *_keep_args(cfg, keep_idx, n_keep), _ws(cfg, ws),
          _stream())


def sirllm_rerotate_keys(cfg: Config, k, keep_idx, n_keep, rope_base: float, layout: int) -> None:
    """Turns the moved rows of a compacted post-rotary K cache to their new positions."""
    _call(lib().sirllm_rerotate_keys, cfg, _kv(cfg, k, "k"), *_keep_args(cfg, keep_idx, n_keep),
          float(rope_base), int(layout), _stream())


class _HeadsArg(_Arg):
    """Rows of attention heads [>= rows, heads, head_dim] of the K/V dtype: heads and elements dense,
    rows any multiple of 8 elements apart (a slice of a wider projection is fine)."""

    def __init__(self, cfg, t, name, rows, heads=None):
        super().__init__(t, None, name)
        self.cfg, self.rows, self.want_heads = cfg, rows, heads

    def check_shape(self):
        cfg, t = self.cfg, self.t
        if t is None:
            return
        if _DTYPE_CODE.get(t.dtype) != cfg.kv_dtype:
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} dtype {t.dtype} does not match the config")
        if t.dim() != 3 or t.shape[0] < self.rows or t.shape[2] != cfg.head_dim or \
                (self.want_heads is not None and t.shape[1] != self.want_heads):
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} has shape {tuple(t.shape)}, the configuration needs "
                                              f"[>= {self.rows}, {self.want_heads or 'heads'}, {cfg.head_dim}]")
        if (t.shape[2] > 1 and t.stride(2) != 1) or (t.shape[1] > 1 and t.stride(1) != cfg.head_dim):
            raise SirllmError(ERR_ALIGN, f"{self.name} heads must be dense")
        if t.shape[0] > 1 and t.stride(0) < t.shape[1] * cfg.head_dim:
            raise SirllmError(ERR_ALIGN, f"{self.name} rows overlap")

    @property
    def heads(self) -> int:
        return 0 if self.t is None else int(self.t.shape[1])

    @property
    def row_stride(self) -> int:
        t = self.t
        return 0 if t is None else int(t.stride(0)) if t.shape[0] > 1 else self.heads * self.cfg.head_dim


def sirllm_append_kv(cfg: Config, layer: int, q, k_new, v_new, q_weight, k_weight, eps: float, rope_base: float,
                     layout: int, first_slot, n_new, q_out, k, v, ws) -> None:
    """New tokens into one layer of the cache: norms per head (where a weight is given), rotation to
    the position of the slot, K/V rows written at ``first_slot[s] + t``.  ``q``, ``q_out``
    ``[rows, n_heads, head_dim]`` (or both None), ``k_new``, ``v_new`` ``[rows, n_kv_heads, head_dim]``."""
    rows, D = _rows(cfg), cfg.head_dim
    qa, ka = _HeadsArg(cfg, q, "q", rows), _HeadsArg(cfg, k_new, "k_new", rows, cfg.n_kv_heads)
    va = _HeadsArg(cfg, v_new, "v_new", rows, cfg.n_kv_heads)
    for a in (qa, ka, va):
        a.check_shape()
    oa = _HeadsArg(cfg, q_out, "q_out", rows, qa.heads if q is not None else None)
    oa.check_shape()
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None and _DTYPE_CODE.get(w.dtype) != cfg.kv_dtype:
            raise SirllmError(ERR_BAD_CONFIG, f"{name} dtype {w.dtype} does not match the config")
    _call(lib().sirllm_append_kv, cfg, int(layer), qa, qa.heads, qa.row_stride, ka, ka.row_stride, va, va.row_stride,
          _dev(q_weight, _KV, "q_weight", D), _dev(k_weight, _KV, "k_weight", D), float(eps), float(rope_base),
          int(layout), _dev(first_slot, torch.int32, "first_slot", cfg.n_streams),
          _dev(n_new, torch.int32, "n_new", cfg.n_streams), oa, oa.row_stride, _kv(cfg, k, "k"), _kv(cfg, v, "v"),
          _ws(cfg, ws), _stream())


def sirllm_attend_workspace_bytes(cfg: Config) -> int:
    return lib().sirllm_attend_workspace_bytes(ctypes.byref(cfg))


def _attend_ws(cfg: Config, ws) -> _Arg:
    return _dev(ws, torch.uint8, "ws", sirllm_attend_workspace_bytes(cfg))


def new_attend_workspace(cfg: Config, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and initialises a workspace for :func:`sirllm_attend`."""
    n = sirllm_attend_workspace_bytes(cfg)
    if n == 0:
        raise SirllmError(ERR_BAD_CONFIG, "invalid configuration")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    sirllm_attend_workspace_init(cfg, ws)
    return ws


def sirllm_attend_workspace_init(cfg: Config, ws: torch.Tensor) -> None:
    _call(lib().sirllm_attend_workspace_init, cfg, _attend_ws(cfg, ws), _stream())


def sirllm_attend(cfg: Config, layer: int, q, k, v, kv_len, scale: Optional[float], out, lse, ws) -> None:
    """Attention of one new token per stream over ``kv_len[s]`` slots of a layer's planes.  ``q``, ``out``
    ``[n_streams, n_heads, head_dim]``; ``scale`` None = 1/sqrt(head_dim); ``lse`` fp32
    ``[n_streams, n_heads]`` or None; ``ws`` from :func:`new_attend_workspace`."""
    S = cfg.n_streams
    qa = _HeadsArg(cfg, q, "q", S)
    qa.check_shape()
    oa = _HeadsArg(cfg, out, "out", S, qa.heads if q is not None else None)
    oa.check_shape()
    _call(lib().sirllm_attend, cfg, int(layer), qa, qa.heads, qa.row_stride, _kv(cfg, k, "k"), _kv(cfg, v, "v"),
          _dev(kv_len, torch.int32, "kv_len", S), cfg.head_dim ** -0.5 if scale is None else float(scale), oa,
          oa.row_stride, _dev(lse, torch.float32, "lse", S * qa.heads), _attend_ws(cfg, ws), _stream())


def _groups(cfg: Config, group: int) -> int:
    if int(group) < 1 or cfg.n_streams % int(group) != 0:
        raise SirllmError(ERR_BAD_CONFIG, f"{cfg.n_streams} streams do not divide into groups of {group}")
    return cfg.n_streams // int(group)


def sirllm_attend_shared_workspace_bytes(cfg: Config, group: int, n_heads: int) -> int:
    if not (_fits(group) and _fits(n_heads)):
        return 0
    return lib().sirllm_attend_shared_workspace_bytes(ctypes.byref(cfg), int(group), int(n_heads))


def new_attend_shared_workspace(cfg: Config, group: int, n_heads: int, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and initialises a workspace for :func:`sirllm_attend_shared`."""
    n = sirllm_attend_shared_workspace_bytes(cfg, group, n_heads)
    if n == 0:
        raise SirllmError(ERR_BAD_CONFIG, "invalid configuration")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    sirllm_attend_shared_workspace_init(cfg, group, n_heads, ws)
    return ws


def sirllm_attend_shared_workspace_init(cfg: Config, group: int, n_heads: int, ws: torch.Tensor) -> None:
    _call(lib().sirllm_attend_shared_workspace_init, cfg, int(group), int(n_heads),
          _dev(ws, torch.uint8, "ws", sirllm_attend_shared_workspace_bytes(cfg, group, n_heads)), _stream())


def sirllm_attend_shared(cfg: Config, layer: int, group: int, shared_len, q, k, v, kv_len, scale: Optional[float], out,
                         lse, ws) -> None:
    """:func:`sirllm_attend` for groups of ``group`` consecutive streams whose first ``shared_len[g]`` slots
    are held once, in the planes of the group's first stream.  ``ws`` from :func:`new_attend_shared_workspace`."""
    S, groups = cfg.n_streams, _groups(cfg, group)
    qa = _HeadsArg(cfg, q, "q", S)
    qa.check_shape()
    oa = _HeadsArg(cfg, out, "out", S, qa.heads if q is not None else None)
    oa.check_shape()
    _call(lib().sirllm_attend_shared, cfg, int(layer), int(group), _dev(shared_len, torch.int32, "shared_len", groups), qa,
          qa.heads, qa.row_stride, _kv(cfg, k, "k"), _kv(cfg, v, "v"), _dev(kv_len, torch.int32, "kv_len", S),
          cfg.head_dim ** -0.5 if scale is None else float(scale), oa, oa.row_stride,
          _dev(lse, torch.float32, "lse", S * qa.heads),
          _dev(ws, torch.uint8, "ws", sirllm_attend_shared_workspace_bytes(cfg, group, qa.heads)), _stream())


def sirllm_beam_workspace_bytes(cfg: Config) -> int:
    return lib().sirllm_beam_workspace_bytes(ctypes.byref(cfg))


def new_beam_workspace(cfg: Config, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and initialises a workspace for :func:`sirllm_beam_select`."""
    n = sirllm_beam_workspace_bytes(cfg)
    if n == 0:
        raise SirllmError(ERR_BAD_CONFIG, "invalid configuration")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    sirllm_beam_workspace_init(cfg, ws)
    return ws


def sirllm_beam_workspace_init(cfg: Config, ws: torch.Tensor) -> None:
    _call(lib().sirllm_beam_workspace_init, cfg, _dev(ws, torch.uint8, "ws", sirllm_beam_workspace_bytes(cfg)), _stream())


def sirllm_beam_select(cfg: Config, logits, group: int, n_out: int, totals, ended, end_token: int, places: bool,
                       totals_out, source, token_ids, entropy, ended_out, ws) -> None:
    """The ``n_out`` best continuations of every group of ``group`` beams (one beam per stream): ``logits``
    ``[n_streams, vocab]``, ``totals`` fp32 and ``ended`` int32 (or None) ``[n_streams]``; outputs
    ``[n_streams / group * n_out]``, ``entropy`` and ``ended_out`` may be None.  ``ws`` from
    :func:`new_beam_workspace`."""
    S, n = cfg.n_streams, _groups(cfg, group) * max(int(n_out), 0)
    _call(lib().sirllm_beam_select, cfg, _LogitsArg(cfg, logits, rows=S), int(group), int(n_out),
          _dev(totals, torch.float32, "totals", S), _dev(ended, torch.int32, "ended", S), int(end_token),
          int(bool(places)), _dev(totals_out, torch.float32, "totals_out", n), _dev(source, torch.int32, "source", n),
          _dev(token_ids, torch.int32, "token_ids", n), _dev(entropy, torch.float32, "entropy", n),
          _dev(ended_out, torch.int32, "ended_out", n),
          _dev(ws, torch.uint8, "ws", sirllm_beam_workspace_bytes(cfg)), _stream())


def sirllm_reorder_streams(cfg: Config, group: int, source, shared_len, scores, serial, live_len, k, v, ws) -> None:
    """Stream ``s`` goes on from stream ``source[s]`` of its group (-1: it stays): K/V rows, scores, tags and
    length, in place, from slot ``shared_len[g]`` (None: 0) on."""
    S, groups = cfg.n_streams, _groups(cfg, group)
    per_slot = S * cfg.capacity
    _call(lib().sirllm_reorder_streams, cfg, int(group), _dev(source, torch.int32, "source", S),
          _dev(shared_len, torch.int32, "shared_len", groups), _dev(scores, torch.float32, "scores", per_slot),
          _dev(serial, torch.int64, "serial", per_slot), _dev(live_len, torch.int32, "live_len", S),
          _kv(cfg, k, "k"), _kv(cfg, v, "v"), _ws(cfg, ws), _stream())


class _MatrixArg(_Arg):
    """A matrix [>= rows, width] of 16-bit elements with dense rows any multiple of 8 elements apart."""

    def __init__(self, t, name, rows):
        super().__init__(t, None, name)
        self.rows = rows

    def check_shape(self):
        t = self.t
        if t is None:
            raise SirllmError(ERR_NULL, f"{self.name} is required")
        if t.dtype not in _KV:
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} has dtype {t.dtype}")
        if t.dim() != 2 or t.shape[0] < self.rows or t.shape[1] < 1:
            raise SirllmError(ERR_BAD_CONFIG, f"{self.name} has shape {tuple(t.shape)}, the call needs "
                                              f"[>= {self.rows}, d_model]")
        if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
            raise SirllmError(ERR_ALIGN, f"{self.name} rows must be dense")

    @property
    def row_stride(self) -> int:
        t = self.t
        return int(t.stride(0)) if t.shape[0] > 1 else (int(t.shape[1]) + 7) // 8 * 8


def sirllm_head_tiles(cfg: Config, n_cols: int) -> int:
    """Pairs per row that :func:`sirllm_head_pairs` writes for ``n_cols`` vocabulary columns."""
    return lib().sirllm_head_tiles(ctypes.byref(cfg), int(n_cols))


def sirllm_head_pairs(cfg: Config, hidden, weight, col0: int, token_ids, n_new, pairs_out, target_out, ws) -> None:
    """Per-tile ``(max, sum exp)`` pairs and target logits of ``hidden @ weight.T`` for
    :func:`sirllm_score_pairs` / :func:`sirllm_step_pairs`, without the logits.  ``hidden``
    ``[rows, d_model]``, ``weight`` ``[n_cols, d_model]`` (rows ``[col0, col0 + n_cols)`` of the LM
    head), ``pairs_out`` fp32 ``[rows, sirllm_head_tiles(cfg, n_cols), 2]``, ``target_out`` fp32 ``[rows]``."""
    rows = _rows(cfg)
    ha, wa = _MatrixArg(hidden, "hidden", rows), _MatrixArg(weight, "weight", 1)
    ha.check_shape()
    wa.check_shape()
    if hidden.dtype != weight.dtype or hidden.shape[1] != weight.shape[1]:
        raise SirllmError(ERR_BAD_CONFIG, f"hidden {tuple(hidden.shape)} {hidden.dtype} and weight "
                                          f"{tuple(weight.shape)} {weight.dtype} do not match")
    n_cols = int(weight.shape[0])
    pa = _PairsArg(cfg, pairs_out)
    pa.check_shape()
    tiles = sirllm_head_tiles(cfg, n_cols)
    if tiles == 0 or pa.n_tiles != tiles:
        raise SirllmError(ERR_BAD_CONFIG, f"pairs_out holds {pa.n_tiles} tiles per row, {n_cols} columns need {tiles}")
    _call(lib().sirllm_head_pairs, cfg, ha, ha.row_stride, wa, wa.row_stride, int(hidden.shape[1]),
          _DTYPE_CODE[hidden.dtype], int(col0), n_cols, *_head_out(cfg, token_ids, n_new, pa, target_out),
          _ws(cfg, ws), _stream())


def _head_out(cfg: Config, token_ids, n_new, pa: _PairsArg, target_out):
    ids, nn, tgt = _score_args(cfg, token_ids, n_new, target_out)
    tgt.name = "target_out"
    return ids, nn, pa, pa.row_stride, tgt


def sirllm_compact_kv(cfg: Config, k_src, v_src, k_dst, v_dst, keep_idx, n_keep, ws) -> None:
    _call(lib().sirllm_compact_kv, cfg, _kv(cfg, k_src, "k_src"), _kv(cfg, v_src, "v_src"),
          _kv(cfg, k_dst, "k_dst"), _kv(cfg, v_dst, "v_dst"), *_keep_args(cfg, keep_idx, n_keep),
          _ws(cfg, ws), _stream())


def sirllm_step(cfg: Config, logits, token_ids, n_new, scores, serial, live_len, decay, k, v,
                keep_idx, n_keep, new_entropy, ws) -> None:
    _call(lib().sirllm_step, cfg, _logits(cfg, logits),
          *_round_args(cfg, token_ids, n_new, scores, serial, live_len, decay, k, v, keep_idx, n_keep,
                       new_entropy, ws), _stream())


def sirllm_step_phases(cfg: Config, logits, token_ids, n_new, scores, serial, live_len, decay, k, v,
                       keep_idx, n_keep, new_entropy, ws, events) -> None:
    """``sirllm_step`` that records the four ``torch.cuda.Event`` objects in ``events``
    (created with ``enable_timing=True``) around its three phases."""
    handles = (ctypes.c_void_p * 4)()
    for i, ev in enumerate(events):
        if not ev.cuda_event:          # torch creates the handle lazily, on first record
            ev.record()
        handles[i] = ev.cuda_event
    _call(lib().sirllm_step_phases, cfg, _logits(cfg, logits),
          *_round_args(cfg, token_ids, n_new, scores, serial, live_len, decay, k, v, keep_idx, n_keep,
                       new_entropy, ws), _stream(), handles)


def _host(t, dtype=None, name="tensor", numel: int = 0) -> _Arg:
    return _Arg(t, dtype, name, numel, host=True)


def sirllm_step_host(cfg: Config, h_logits, h_token_ids, h_n_new, h_new_k, h_new_v, h_live_len,
                     d_logits, d_token_ids, d_n_new, scores, serial, live_len, decay, k, v,
                     keep_idx, n_keep, new_entropy, h_keep_idx, h_n_keep, h_new_entropy, ws) -> None:
    """One round with HOST inputs and outputs (``h_*`` are CPU tensors, ideally pinned);
    the results are valid after ``torch.cuda.current_stream().synchronize()``."""
    rows, S = _rows(cfg), cfg.n_streams
    new_rows = S * cfg.n_layers * cfg.n_kv_heads * cfg.max_new * cfg.head_dim
    rest = _round_args(cfg, d_token_ids, d_n_new, scores, serial, live_len, decay, k, v, keep_idx,
                       n_keep, new_entropy, ws)
    _call(lib().sirllm_step_host, cfg, _LogitsArg(cfg, h_logits, "h_logits", host=True),
          _host(h_token_ids, torch.int32, "h_token_ids", rows), _host(h_n_new, torch.int32, "h_n_new", S),
          _host(h_new_k, _KV, "h_new_k", new_rows), _host(h_new_v, _KV, "h_new_v", new_rows),
          _host(h_live_len, torch.int32, "h_live_len", S), _LogitsArg(cfg, d_logits, "d_logits"),
          *rest[:-1], _host(h_keep_idx, torch.int32, "h_keep_idx", S * cfg.threshold),
          _host(h_n_keep, torch.int32, "h_n_keep", S),
          _host(h_new_entropy, torch.float32, "h_new_entropy", rows), rest[-1], _stream())


def sirllm_selftest_bounded_wait(cfg: Config, ws: torch.Tensor, polls: int = 2000) -> None:
    """Lets one device-side bounded wait run out on purpose (raises STATUS_TIMEOUT in ``ws``)."""
    _call(lib().sirllm_selftest_bounded_wait, cfg, _ws(cfg, ws), int(polls), _stream())


def sirllm_status(ws: torch.Tensor, clear: bool = False) -> int:
    """Synchronises the current stream and returns the device status word."""
    out = ctypes.c_int32(0)
    arg = _dev(ws, torch.uint8, "ws", 4)
    arg.check_shape()
    arg.check_residence()
    _check(lib().sirllm_status(arg.ptr(), _stream_handle(), ctypes.byref(out), int(clear)))
    return out.value


def sirllm_strerror(code: int) -> str:
    return lib().sirllm_strerror(code).decode()


def sirllm_last_cuda_error() -> str:
    return lib().sirllm_last_cuda_error().decode()
