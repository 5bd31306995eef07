"""Norm, 8-bit product and log probabilities on torch tensors (bmgd_norm_*, bmgd_product_*, bmgd_logprobs_* of include/bmgd.h).

Checks shapes, types and devices, fills in addresses and strides, and calls the library: no arithmetic happens here.

The objects hold sizes and types only: one may be used on several devices and streams, and from several threads, at once.  Matrices are torch tensors whose rows are any
distance apart, vectors are contiguous, all of a call on one GPU.  Calls are asynchronous and run on `stream` (a torch stream or a handle), by default on torch's current one
of that GPU; the caller orders other streams that operands are made or results read on.  Results overlap neither operands nor each other but where it is said.

Two calls (the norm's weight gradient, log probabilities of few rows of many classes) need a workspace.  It is taken from torch's pool for the stream that the call
runs on; captured with torch's graphs, it belongs to the graph's pool.  A program that captures in other ways gives one (`workspace=`), and keeps it while the graph lives.
"""
from __future__ import annotations

import ctypes as C
import math
import struct

import torch

from . import binding as B
from .network import _CODES, _TYPES, _stream, _tensors

_BYTE, _FLOAT, _INT = torch.int8, torch.float32, torch.int32
_PLACES = struct.Struct("PQ").pack                      # a workspace: its address and its size
_NONE16 = bytes(16)


def _type_of(dtype):
    if dtype not in _TYPES:
        raise ValueError(f"dtype {dtype!r} is not one of BMGD_F32, BMGD_BF16 and BMGD_F16")
    return _TYPES[dtype]


def _refuse(name, t, kind, shape, matrix, index):
    if not isinstance(t, torch.Tensor) or t.dtype is not kind or not t.is_cuda or t.device.index != index:
        what = f"{t.dtype} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name}: a {kind} tensor on one GPU, cuda:{index}, is wanted, not {what}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: shape {shape} is wanted, not {tuple(t.shape)}")
    if matrix:
        raise ValueError(f"{name}: the elements of a row must lie next to each other (strides {t.stride()})")
    raise ValueError(f"{name}: contiguous elements are wanted (strides {t.stride()})")


def _rows_of(name, t):
    """Rows and GPU of a call's first matrix."""
    try:
        index = t.get_device()
        if index >= 0:
            return t.shape[0], index
    except (AttributeError, IndexError):
        pass
    raise ValueError(f"{name}: a matrix on a GPU is wanted")


def _places(names, tensors, kinds, shapes, how, index):
    found = _tensors.operands(tensors, kinds, shapes, how, index, False)
    if type(found) is int:
        _refuse(names[found], tensors[found], kinds[found], shapes[found], how[found] in b"mM", index)
    return found


def _run(fn, args, stream, index, tensors, how):
    """The call on the device of its tensors.  Those that it writes are told so, unless it is refused."""
    stream = _stream(stream, index)
    if torch._C._cuda_getDevice() == index:
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, stream)
    if rc != B.BMGD_OK:
        raise B.BmgdError(rc, B.bmgd_last_error(None))
    _tensors.told(tensors, how)


def _workspace(need, given, stream, index):
    """(tensor to keep until the call is made, its address and size).  From the pool of the stream that the call runs on: torch gives the memory to others
    on that stream only, behind the call."""
    if given is not None:
        if not isinstance(given, torch.Tensor) or not given.is_cuda or given.get_device() != index or not given.is_contiguous():
            raise ValueError(f"workspace: a contiguous tensor on cuda:{index} is wanted")
        return given, _PLACES(given.data_ptr(), given.numel() * given.element_size())
    if not need:
        return None, _NONE16
    if stream is None or B._stream(stream) == torch._C._cuda_getCurrentRawStream(index):
        area = torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", index))
    else:
        with torch.cuda.stream(torch.cuda.ExternalStream(B._stream(stream), device=index)):
            area = torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", index))
    return area, _PLACES(area.data_ptr(), need)


class RMSNorm:
    """y = s w / sqrt(mean s^2 + eps) of the rows s = x + residual, in 16 or 32 bits or as 8-bit codes with a scale for each row; its gradient.

    n: columns.  dtype: of all matrices but codes, and of the weight (BMGD_F32, BMGD_BF16, BMGD_F16).
    """

    _NAMES = ("x", "residual", "sum", "y", "codes", "dy", "dsum", "dx", "weight", "dweight", "scales", "rstd")       # bmgd_norm_tensors

    def __init__(self, n, dtype=B.BMGD_BF16, eps=1e-6):
        self._type = t = _type_of(dtype)
        if not isinstance(n, int) or not 1 <= n <= 1 << 20:
            raise ValueError("n must be in [1, 2^20]")
        if not (eps >= 0.0 and math.isfinite(C.c_float(eps).value)):
            raise ValueError("eps must be finite in 32 bits and >= 0")
        self.n, self.cfg = n, B.bmgd_norm_config(n, eps, dtype, 0)
        self._cfg = C.byref(self.cfg)
        self._kinds = (t, t, t, t, _BYTE, t, t, t, t, t, _FLOAT, _FLOAT)
        self._of_n = (n,)

    def forward(self, x, weight=None, y=None, residual=None, sum=None, codes=None, scales=None, rstd=None, stream=None):
        """Writes y, or codes and scales, or all three; sum <- s and rstd <- 1 / sqrt(mean s^2 + eps) where they are given (`backward` reads both; s is x
        without a residual).  weight None: ones.  sum may be x or residual, y may be x (without sum there) or residual."""
        rows, index = _rows_of("x", x)
        at, of, n = (rows, self.n), (rows,), self._of_n
        tensors, how = (x, residual, sum, y, codes, None, None, None, weight, None, scales, rstd), b"mmMMMmmmvvVV"
        found = _places(self._NAMES, tensors, self._kinds, (at, at, at, at, at, at, at, at, n, n, of, of), how, index)
        _run(B.lib.bmgd_norm_forward, (self._cfg, rows, found + _NONE16), stream, index, tensors, how)

    def backward(self, dy, s, weight, rstd, dx, dweight=None, dsum=None, workspace=None, stream=None):
        """dx <- the gradient of x (and of residual alike) from dy, the s that was normed and the forward call's rstd, plus dsum, the gradient that reaches s besides;
        dweight <- the weight's.  dx may be dy or dsum."""
        rows, index = _rows_of("s", s)
        at, of, n = (rows, self.n), (rows,), self._of_n
        tensors, how = (s, None, None, None, None, dy, dsum, dx, weight, dweight, None, rstd), b"mmmmmmmMvVvv"
        found = _places(self._NAMES, tensors, self._kinds, (at, at, at, at, at, at, at, at, n, n, of, of), how, index)
        keep, place = _workspace(B.lib.bmgd_norm_workspace_bytes(self._cfg, rows) if dweight is not None and rows else 0, workspace, stream, index)
        _run(B.lib.bmgd_norm_backward, (self._cfg, rows, found + place), stream, index, tensors, how)

    def values(self, codes, scales, out, stream=None):
        """out <- scales[i] codes[i, j], in the type of `out` (any of the three)."""
        _values(codes, scales, out, self.n, stream)


def _values(codes, scales, out, n, stream):
    rows, index = _rows_of("codes", codes)
    if not isinstance(out, torch.Tensor) or out.dtype not in _CODES:
        raise ValueError("out: a tensor of 32-bit or 16-bit floats is wanted")
    tensors = codes, out, scales
    found = _places(("codes", "out", "scales"), tensors, (_BYTE, out.dtype, _FLOAT), ((rows, n), (rows, n), (rows,)), b"mMv", index)
    _run(B.lib.bmgd_product_values, (rows, n, found[:16], struct.unpack_from("P", found, 32)[0], found[16:32], _CODES[out.dtype]), stream, index, tensors, b"mMv")


class Int8Product:
    """Y = (x_scales[i] X)(w_scales[j] W)' of 8-bit codes, exact sums, for any number of rows; holds no weights.

    p: columns of both; out_n: outputs; dtype: of y, and of the weights that `quantize` takes.
    """

    def __init__(self, p, out_n, dtype=B.BMGD_BF16):
        self._type = _type_of(dtype)
        if not isinstance(p, int) or not 1 <= p <= 131_071:
            raise ValueError("p must be in [1, 131071]")
        if not isinstance(out_n, int) or not 1 <= out_n <= 1 << 20:
            raise ValueError("out_n must be in [1, 2^20]")
        self.p, self.out_n, self.cfg = p, out_n, B.bmgd_product_config(p, out_n, dtype, 0)
        self._cfg = C.byref(self.cfg)
        self._kinds = (_BYTE, _BYTE, self._type, _FLOAT, _FLOAT)

    def forward(self, x, x_scales, w, w_scales, y, stream=None):
        """y <- the product of the codes x (rows x p, a scale for each row) and w (out_n x p, a scale for each output)."""
        rows, index = _rows_of("x", x)
        tensors = x, w, y, x_scales, w_scales
        found = _places(("x", "w", "y", "x_scales", "w_scales"), tensors, self._kinds,
                        ((rows, self.p), (self.out_n, self.p), (rows, self.out_n), (rows,), (self.out_n,)), b"mmMvv", index)
        _run(B.lib.bmgd_product_forward, (self._cfg, rows, found), stream, index, tensors, b"mmMvv")

    def quantize(self, weights, w, w_scales, stream=None):
        """Lays a layer's weights (p x out_n, as GatedBlock has them) out for the product, once: w <- codes (out_n x p), w_scales <- a scale for each output."""
        _, index = _rows_of("weights", weights)
        tensors = weights, w, w_scales
        found = _places(("weights", "w", "w_scales"), tensors, (self._type, _BYTE, _FLOAT), ((self.p, self.out_n), (self.out_n, self.p), (self.out_n,)), b"mMV", index)
        _run(B.lib.bmgd_product_quantize, (self._cfg, found[:16], found[16:32], struct.unpack_from("P", found, 32)[0]), stream, index, tensors, b"mMV")

    def values(self, codes, scales, out, stream=None):
        """out <- scales[i] codes[i, j] of rows of p codes, in the type of `out` (any of the three)."""
        _values(codes, scales, out, self.p, stream)


class LogProbs:
    """Log probabilities of labels, entropy and the `top` most probable classes of rows of logits; the gradient of the first two.

    classes: columns; dtype: of the logits (BMGD_F32, BMGD_BF16, BMGD_F16); top: up to 64.  Labels are int32: a negative one leaves its row out.
    """

    _NAMES = ("logits", "dlogits", "labels", "logprob", "entropy", "top_classes", "top_logprobs", "kept", "dlogprob", "dentropy")       # bmgd_logprobs_tensors

    def __init__(self, classes, dtype=B.BMGD_BF16, top=0):
        self._type = t = _type_of(dtype)
        if not isinstance(classes, int) or not 1 <= classes <= 1 << 24:
            raise ValueError("classes must be in [1, 2^24]")
        if not isinstance(top, int) or not 0 <= top <= min(64, classes):
            raise ValueError("top must be in [0, 64] and not above classes")
        self.classes, self.top, self.cfg = classes, top, B.bmgd_logprobs_config(classes, dtype, top)
        self._cfg = C.byref(self.cfg)
        self._kinds = (t, t, _INT, _FLOAT, _FLOAT, _INT, _FLOAT, _FLOAT, _FLOAT, _FLOAT)

    def forward(self, logits, labels=None, logprob=None, entropy=None, top_classes=None, top_logprobs=None, kept=None, workspace=None, stream=None):
        """Writes what is given: logprob (of labels, rows of them), entropy (rows), top_classes and top_logprobs (rows x top each; both wanted where top is not 0),
        kept (rows x 3, fp32: what `backward` needs)."""
        rows, index = _rows_of("logits", logits)
        at, of, best = (rows, self.classes), (rows,), (rows, self.top)
        tensors, how = (logits, None, labels, logprob, entropy, top_classes, top_logprobs, kept, None, None), b"mmvVVVVVvv"
        found = _places(self._NAMES, tensors, self._kinds, (at, at, of, of, of, best, best, (rows, 3), of, of), how, index)
        keep, place = _workspace(B.lib.bmgd_logprobs_workspace_bytes(self._cfg, rows), workspace, stream, index)
        _run(B.lib.bmgd_logprobs_forward, (self._cfg, rows, found + place), stream, index, tensors, how)

    def backward(self, logits, kept, dlogits, labels=None, dlogprob=None, dentropy=None, stream=None):
        """dlogits <- dlogprob ([j = label] - p_j) - dentropy p_j (ln p_j + entropy), from the forward call's `kept`.  dlogits may be logits."""
        rows, index = _rows_of("logits", logits)
        at, of = (rows, self.classes), (rows,)
        tensors, how = (logits, dlogits, labels, None, None, None, None, kept, dlogprob, dentropy), b"mMvvvvvvvv"
        found = _places(self._NAMES, tensors, self._kinds, (at, at, of, of, of, of, of, (rows, 3), of, of), how, index)
        _run(B.lib.bmgd_logprobs_backward, (self._cfg, rows, found + _NONE16), stream, index, tensors, how)
