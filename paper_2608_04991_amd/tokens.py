"""Python binding of include/rac_tokens.h: rotary positions, and the log
probabilities of drafted tokens with their gradient.  Re-exported by the package.

    cfg = RotaryConfig(rows=n, q_heads=32, k_heads=8, head_dim=128, rotary_dim=128, layout=RAC_ROTARY_HALF)
    freq = torch.tensor(rac_rotary_frequencies(128, 10000.0), dtype=torch.float64, device="cuda")
    rac_rotary(cfg, pos, freq, q, k)                                  # in place

    cfg = LogprobConfig(rows=n, vocab=32000, tokens=m, top=8)
    ws = torch.empty(rac_logprobs_workspace(cfg), dtype=torch.uint8, device="cuda")
    rac_logprobs(cfg, logits, tokens, logprob, lse, ws, token_rows=parents, top_ids=ids, top_logprobs=values)

As in the rest of the package every step runs in HIP kernels; PyTorch supplies
device memory and the stream.
"""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass, fields

import paper_2608_04991_amd as _rac

__all__ = [
    "RAC_TYPE_BF16", "RAC_TYPE_FP16", "RAC_TYPE_FP32", "RAC_ROTARY_INTERLEAVED", "RAC_ROTARY_HALF", "RotaryConfig",
    "LogprobConfig", "rac_rotary_frequencies", "rac_rotary", "rac_logprobs_workspace", "rac_logprobs",
    "rac_logprobs_backward",
]

RAC_TYPE_BF16 = 0
RAC_TYPE_FP16 = 1
RAC_TYPE_FP32 = 2
RAC_ROTARY_INTERLEAVED = 0
RAC_ROTARY_HALF = 1


class _RotaryConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "q_heads", "k_heads", "head_dim", "rotary_dim", "type", "layout",
                                              "transpose")] + [("amplitude", ctypes.c_float)]


class _RotaryTensors(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "q_out", "k_out")] + \
               [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride")]


class _LogprobConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "vocab", "tokens", "top", "type")] + [("scale", ctypes.c_float)]


class _LogprobTensors(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("stride", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("tokens", "token_rows", "logprob", "lse", "entropy", "top_ids",
                                               "top_logprobs")]


class _LogprobGradients(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("stride", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("tokens", "lse", "entropy", "grad_logprob", "grad_entropy",
                                               "grad_logits")] + [("grad_stride", ctypes.c_int64)]


class _Kept:
    """A configuration that keeps the library's struct and a reference to it.  A
    copy or a pickle has the fields alone."""

    def __getstate__(self) -> dict:
        return {f.name: getattr(self, f.name) for f in fields(self)}

    @functools.cached_property
    def _ref(self):
        return ctypes.byref(self._struct)

    @property
    def _bytes(self) -> int:
        return 4 if self.type == RAC_TYPE_FP32 else 2


@dataclass(frozen=True)
class RotaryConfig(_Kept):
    rows: int
    q_heads: int
    k_heads: int
    head_dim: int
    rotary_dim: int
    type: int = RAC_TYPE_BF16
    layout: int = RAC_ROTARY_INTERLEAVED
    transpose: bool = False
    amplitude: float = 1.0

    @functools.cached_property
    def _struct(self) -> _RotaryConfig:
        return _RotaryConfig(self.rows, self.q_heads, self.k_heads, self.head_dim, self.rotary_dim, self.type, self.layout,
                             int(self.transpose), self.amplitude)


@dataclass(frozen=True)
class LogprobConfig(_Kept):
    rows: int
    vocab: int
    tokens: int
    top: int = 0
    type: int = RAC_TYPE_BF16
    scale: float = 0.0

    @functools.cached_property
    def _struct(self) -> _LogprobConfig:
        return _LogprobConfig(self.rows, self.vocab, self.tokens, self.top, self.type, self.scale)

    @functools.cached_property
    def _workspace(self) -> int:
        return int(_rac.library().rac_logprobs_workspace(self._ref))


def declare(L) -> None:
    """The argument types of the library's functions of this part."""
    vp, i32, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double
    rp, lp = ctypes.POINTER(_RotaryConfig), ctypes.POINTER(_LogprobConfig)
    for name, args, res in (
            ("rac_rotary_frequencies", [i32, f64, f64, i32, f64, f64, ctypes.POINTER(f64)], ctypes.c_int),
            ("rac_rotary", [rp, vp, vp, ctypes.POINTER(_RotaryTensors), vp], ctypes.c_int),
            ("rac_logprobs_workspace", [lp], ctypes.c_size_t),
            ("rac_logprobs", [lp, ctypes.POINTER(_LogprobTensors), vp, ctypes.c_size_t, vp], ctypes.c_int),
            ("rac_logprobs_backward", [lp, ctypes.POINTER(_LogprobGradients), vp], ctypes.c_int)):
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res


def _heads(t, what: str, rows: int, heads: int, dim: int, size: int):
    """(address, elements between rows) of a [rows][heads][dim] tensor whose heads
    lie together; its rows may be apart."""
    if t is None or isinstance(t, int):
        return t, heads * dim
    try:
        n, h, d = t.shape
        row, head, one = t.stride()
        if n <= 1:
            row = heads * dim
        if h == heads and d == dim and n >= rows and one == 1 and (head == dim or h == 1) and row >= heads * dim \
                and t.is_cuda and t.element_size() == size:
            return t.data_ptr(), row
    except (AttributeError, ValueError, TypeError):
        pass
    raise ValueError(f"{what}: expected a GPU tensor of {size}-byte elements, [{rows}][{heads}][{dim}], heads and "
                     "channels contiguous")


def _matrix(t, what: str, rows: int, width: int, size: int):
    """(address, elements between rows) of a [rows][width] tensor; its rows may be apart."""
    if t is None or isinstance(t, int):
        return t, width
    try:
        n, w = t.shape
        row, one = t.stride()
        if n <= 1:
            row = width
        if w == width and n >= rows and (one == 1 or w == 1) and row >= width and t.is_cuda and t.element_size() == size:
            return t.data_ptr(), row
    except (AttributeError, ValueError, TypeError):
        pass
    raise ValueError(f"{what}: expected a GPU tensor of {size}-byte elements, [{rows}][{width}], words contiguous")


def rac_rotary_frequencies(rotary_dim: int, base: float, factor: float = 1.0, trained: int = 0, slow: float = 1.0,
                           fast: float = 32.0) -> list:
    """Turns a position of every channel pair (binary64, on the host)."""
    out = (ctypes.c_double * max(1, int(rotary_dim) // 2))()
    _rac._check(_rac.library().rac_rotary_frequencies(int(rotary_dim), float(base), float(factor), int(trained),
                                                      float(slow), float(fast), out), "rac_rotary_frequencies")
    return list(out)


def rac_rotary(cfg: RotaryConfig, pos, freq, q, k=None, *, q_out=None, k_out=None, stream=None) -> None:
    """Turns queries q ([rows][q_heads][head_dim]) and keys k ([rows][k_heads]
    [head_dim]) by their positions pos (int32 [rows]) with the frequencies freq
    (float64 [rotary_dim / 2]), in place or into q_out and k_out.  Rows may be apart
    (views of a larger tensor)."""
    R, D, size = cfg.rows, cfg.head_dim, cfg._bytes
    q_out, k_out = q if q_out is None else q_out, k if k_out is None else k_out
    qp, qs = _heads(q, "q", R, cfg.q_heads, D, size)
    kp, ks = _heads(k, "k", R, cfg.k_heads, D, size)
    qo, qos = _heads(q_out, "q_out", R, cfg.q_heads, D, size)
    ko, kos = _heads(k_out, "k_out", R, cfg.k_heads, D, size)
    t = _RotaryTensors(qp, kp, qo, ko, qs, ks, qos, kos)
    status = _rac.library().rac_rotary(cfg._ref, _rac._dev(pos, "pos", 4, R), _rac._dev(freq, "freq", 8, cfg.rotary_dim // 2),
                                       ctypes.byref(t), _rac._stream(stream))
    if status:
        _rac._check(status, "rac_rotary")


def rac_logprobs_workspace(cfg: LogprobConfig) -> int:
    return cfg._workspace


def rac_logprobs(cfg: LogprobConfig, logits, tokens, logprob, lse, workspace, *, token_rows=None, entropy=None,
                 top_ids=None, top_logprobs=None, stream=None) -> None:
    """Log probabilities logprob (fp32 [tokens]) of tokens (int32 [tokens]) under the
    logits ([rows][vocab], rows may be apart) of rows token_rows (int32 [tokens],
    None: one token a row), with lse and entropy (fp32 [rows]) and the largest
    alternatives top_ids (int32 [rows][top]) and top_logprobs (fp32)."""
    dev, R, n = _rac._dev, cfg.rows, cfg.rows * cfg.top
    lp, ls = _matrix(logits, "logits", R, cfg.vocab, cfg._bytes)
    t = _LogprobTensors(lp, ls, dev(tokens, "tokens", 4, cfg.tokens), dev(token_rows, "token_rows", 4, cfg.tokens),
                        dev(logprob, "logprob", 4, cfg.tokens), dev(lse, "lse", 4, R), dev(entropy, "entropy", 4, R),
                        dev(top_ids, "top_ids", 4, n), dev(top_logprobs, "top_logprobs", 4, n))
    need = cfg._workspace
    status = _rac.library().rac_logprobs(cfg._ref, ctypes.byref(t), dev(workspace, "workspace", 1, need), need,
                                         _rac._stream(stream))
    if status:
        _rac._check(status, "rac_logprobs")


def rac_logprobs_backward(cfg: LogprobConfig, logits, tokens, lse, grad_logits, *, grad_logprob=None, grad_entropy=None,
                          entropy=None, stream=None) -> None:
    """Gradients grad_logits (as the logits, which they may replace) from those of
    logprob and entropy (fp32 [rows], either may be None), for one token a row."""
    dev, R = _rac._dev, cfg.rows
    lp, ls = _matrix(logits, "logits", R, cfg.vocab, cfg._bytes)
    gp, gs = _matrix(grad_logits, "grad_logits", R, cfg.vocab, cfg._bytes)
    g = _LogprobGradients(lp, ls, dev(tokens, "tokens", 4, R), dev(lse, "lse", 4, R), dev(entropy, "entropy", 4, R),
                          dev(grad_logprob, "grad_logprob", 4, R), dev(grad_entropy, "grad_entropy", 4, R), gp, gs)
    status = _rac.library().rac_logprobs_backward(cfg._ref, ctypes.byref(g), _rac._stream(stream))
    if status:
        _rac._check(status, "rac_logprobs_backward")
