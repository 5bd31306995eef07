"""Gated block and AdamW step on torch tensors (bmgd_gated_*, bmgd_adamw_* of include/bmgd.h).

Checks shapes, types and devices, fills in addresses and strides, and calls the library: no arithmetic happens here.
"""
from __future__ import annotations

import ctypes as C
import itertools
import struct

import numpy as np
import torch

from . import binding as B

try:
    from . import _tensors
except ImportError as e:
    raise ImportError(f"_tensors.so, next to {B.LIB_PATH}, is missing or was built for another torch ({e}): build it first (__graft_entry__.build())") from e

_TYPES = {B.BMGD_BF16: torch.bfloat16, B.BMGD_F16: torch.float16, B.BMGD_F32: torch.float32}
_CODES = {v: k for k, v in _TYPES.items()}
_NAMES = ("x", "gate", "up", "down", "y", "g", "u", "dy", "dx", "dgate", "dup", "ddown")      # bmgd_gated_tensors: an address and a stride each
_FIELDS = [name for name, _ in B.bmgd_adamw_tensor._fields_]                                   # eight bytes each
_STATE = ("m", "s", "m_scale", "s_scale")
_REST = bytes(16 * 5)                 # those behind the first seven, which a forward call does not have


def _stream(stream, index):
    """The handle of `stream`, or of the stream that is torch's current one on device `index`: the one that work on the operands is on."""
    return torch._C._cuda_getCurrentRawStream(index) if stream is None else B._stream(stream)


class GatedBlock:
    """Y = (act(X Wg) * (X Wu)) Wd with its backward pass, for up to `max_rows` rows a call; holds a workspace, no weights.

    Matrices are torch tensors on the block's device, of type `dtype` (BMGD_BF16 or BMGD_F16), rows any distance apart.  Results must not overlap operands or each other.
    Calls run on `stream` (a torch stream or a handle), by default on torch's current one; the caller orders other streams that operands are made or results read on.
    """

    def __init__(self, p, hidden, out_n, max_rows, dtype=B.BMGD_BF16, activation=B.BMGD_ACT_SILU, workspace=None):
        cfg = B.bmgd_gated_config(p, hidden, out_n, max_rows, dtype, activation, None, 0)
        self.h = None
        if workspace is None and torch.cuda.is_available():
            # from torch's pool, where a block of the same size that was closed has left one (an invalid configuration needs 0 bytes and is refused below)
            need = B.bmgd_gated_workspace_bytes(cfg)
            if need:
                workspace = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
                torch.cuda.current_stream().synchronize()      # work of tensors that had this memory before
                at = -workspace.data_ptr() % 256
                workspace = workspace[at:at + need]
        if workspace is not None:
            if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or workspace.device.index != torch.cuda.current_device():
                raise ValueError("workspace: a tensor on the current GPU is wanted")
            cfg.workspace, cfg.workspace_bytes = B._ptr(workspace), workspace.numel() * workspace.element_size()
        self.cfg, self._keep = cfg, workspace
        rc, h = B.bmgd_gated_create(cfg)
        if rc != B.BMGD_OK:
            raise B.BmgdError(rc, B.bmgd_last_error(None))
        self.h = h
        self._type = _TYPES[dtype]
        self._device = torch.device("cuda", torch.cuda.current_device())
        self._index = self._device.index
        self._p, self._hidden, self._out_n, self._in, self._out = p, hidden, out_n, (p, hidden), (hidden, out_n)

    def _refuse(self, name, t, shape):
        if t.dtype is not self._type or t.device != self._device:
            raise ValueError(f"{name}: a {self._type} tensor on {self._device} is wanted, not {t.dtype} on {t.device}")
        if tuple(t.shape) != shape:
            raise ValueError(f"{name}: shape {shape} is wanted, not {tuple(t.shape)}")
        raise ValueError(f"{name}: the elements of a row must lie next to each other (strides {t.stride()})")

    def _addresses(self, tensors, shapes, written):
        found = _tensors.matrices(tensors, shapes, self._type, self._index, written)
        if type(found) is int:
            self._refuse(_NAMES[found], tensors[found], shapes[found])
        return found

    def forward(self, x, gate, up, down, y, g=None, u=None, stream=None):
        """y <- Y (and g <- G, u <- U, which `backward` needs).  Asynchronous."""
        rows = x.shape[0]
        hid = (rows, self._hidden)
        found = self._addresses((x, gate, up, down, y, g, u), ((rows, self._p), self._in, self._in, self._out, (rows, self._out_n), hid, hid), 4)
        rc = B.lib.bmgd_gated_forward(self.h, rows, found + _REST, _stream(stream, self._index))
        if rc != B.BMGD_OK:
            raise B.BmgdError(rc, B.bmgd_gated_last_error(self.h))

    def backward(self, dy, x, gate, up, down, g, u, dx=None, dgate=None, dup=None, ddown=None, stream=None):
        """The gradients that are asked for (dgate and dup together) are written, from dy and the forward call's g and u.  Asynchronous."""
        rows = x.shape[0]
        at, hid, wide = (rows, self._p), (rows, self._hidden), self._in
        out = (rows, self._out_n)
        found = self._addresses((x, gate, up, down, None, g, u, dy, dx, dgate, dup, ddown), (at, wide, wide, self._out, out, hid, hid, out, at, wide, wide, self._out), 8)
        rc = B.lib.bmgd_gated_backward(self.h, rows, found, _stream(stream, self._index))
        if rc != B.BMGD_OK:
            raise B.BmgdError(rc, B.bmgd_gated_last_error(self.h))

    def close(self):
        if getattr(self, "h", None):
            B.bmgd_gated_destroy(self.h)                       # (waits for the device)
            self.h = self._keep = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdamW:
    """AdamW over the fp32 tensors `thetas` with the gradients that stand in the tensors `grads` at the time of a step.

    grads: of one type (fp32, bf16, f16), sized like thetas; `set_grads` names others.
    copies: None, or tensors of one 16-bit type that receive the rounded new values.
    state_bits: 32, or 8 for 8-bit codes with a scale per 256 elements.
    state: None (zeros), or a tuple of tensors per theta that are used in place: (m, s) in fp32, or (m codes int8, s codes uint8,
    m scales, s scales fp32) with ceil(n / 256) scales each.  `self.state` holds them.
    step: the number of updates already made.
    A tensor that is given other memory (`t.data = ...`), or replaced in `thetas`, `grads`, `copies` or `state`, is followed from the next call on.
    All tensors are contiguous and on one device; those that a step writes overlap neither each other nor a gradient.  Calls run on `stream` (a torch stream or a handle), by default on torch's current one; the caller orders other
    streams that the tensors are written or read on.
    """

    def __init__(self, thetas, grads, copies=None, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, state_bits=32,
                 state=None, step=0):
        self.thetas = list(thetas)
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 32 or 8")
        self.device = self.thetas[0].device if self.thetas else None
        self.count, self.steps, self.lr = len(self.thetas), int(step), lr
        self._t = (B.bmgd_adamw_tensor * max(1, self.count))()
        self._rows = np.frombuffer(self._t, dtype=np.int64).reshape(-1, len(_FIELDS))
        cfg = B.bmgd_adamw_default_config()
        cfg.beta1, cfg.beta2, cfg.eps, cfg.weight_decay, cfg.state_bits = beta1, beta2, eps, weight_decay, state_bits
        self.cfg = cfg
        sizes = [t.numel() for t in self.thetas]
        self._n = struct.pack(f"{self.count}q", *sizes)
        blocks = struct.pack(f"{self.count}q", *[-(-n // 256) for n in sizes])
        self._rows[:self.count, _FIELDS.index("n")] = sizes
        self._groups = {}                                      # by field: its tensors and where they were when `_rows` was filled in
        self._fill("theta", self.thetas, torch.float32, self._n)
        self._seen = None                                      # streams that the moments made here are known to be used on
        if state is None:
            state = [self._zeros(t, state_bits) for t in self.thetas]
            if self.thetas and self.thetas[0].is_cuda:
                # the caller does not see these fills, so steps on any stream must find them done
                home = torch.cuda.current_stream(self.device)
                self._seen = {home.cuda_stream}
                if not torch.cuda.is_current_stream_capturing():
                    home.synchronize()
        self.state = [tuple(s) for s in state]
        kinds = (torch.float32, torch.float32) if state_bits == 32 else (torch.int8, torch.uint8, torch.float32, torch.float32)
        if len(self.state) != self.count or any(len(s) != len(kinds) for s in self.state):
            raise ValueError(f"state: {len(kinds)} tensors for each of {self.count} are wanted")
        for i, (field, kind) in enumerate(zip(_STATE, kinds)):
            self._fill(field, self.state, kind, blocks if field.endswith("scale") else self._n, i)
        self.copies = None
        if copies is not None:
            self.copies = list(copies)
            kind = self._same_type("copies", self.copies, (torch.bfloat16, torch.float16))
            self._fill("copy", self.copies, kind, self._n)
            cfg.copy_dtype = _CODES[kind]
        self.set_grads(grads)

    @staticmethod
    def _zeros(t, bits):
        if bits == 32:
            return torch.zeros_like(t), torch.zeros_like(t)
        blocks = -(-t.numel() // 256)
        new = lambda n, kind: torch.zeros(n, dtype=kind, device=t.device)  # noqa: E731
        return new(t.numel(), torch.int8), new(t.numel(), torch.uint8), new(blocks, torch.float32), new(blocks, torch.float32)

    def _check(self, name, t, kind, n):
        if t.dtype is not kind or t.device != self.device or not t.is_cuda:
            raise ValueError(f"{name}: a {kind} tensor on one GPU is wanted, not {t.dtype} on {t.device}")
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{name}: {n} contiguous elements are wanted, not {tuple(t.shape)} with strides {t.stride()}")

    def _addresses(self, read, name, tensors, kind, sizes):
        found = read(tensors, sizes, kind, self.device.index if self.count and self.device.type == "cuda" else -2)
        if type(found) is int:
            n = struct.unpack_from("q", sizes, 8 * found)[0]
            for t in tensors[found] if read is _tensors.pairs else (tensors[found],):
                self._check(name, t, kind, n)
            raise ValueError(f"{name}: tensor {found} is not one that was asked for")
        return found

    def _fill(self, field, tensors, kind, sizes, item=-1):
        found = self._addresses(_tensors.vectors, field, tensors if item < 0 else [s[item] for s in tensors], kind, sizes)
        self._rows[:self.count, _FIELDS.index(field)] = np.frombuffer(found, dtype=np.int64)
        self._groups[field] = tensors, item, sizes, kind, found
        self._watched = tuple(self._groups.values()), tuple(g for name, g in self._groups.items() if name in _STATE)
        self._apart = False
        if field != "grad":
            self._written = None

    def _read_again(self, watched):
        """Addresses, where a tensor of these has been given other memory (`t.data = ...`, `resize_`) or replaced in its list: 10 ns a tensor if none has."""
        if not _tensors.same(watched):
            for field, (tensors, item, sizes, kind, _) in list(self._groups.items()):
                if len(tensors) != self.count:
                    raise ValueError(f"{field}: {self.count} tensors are wanted, not {len(tensors)}")
                self._fill(field, tensors, kind, sizes, item)

    def _spans(self, field):
        """Where the tensors of a field begin and end (at 0 where they have no elements)."""
        _, _, sizes, kind, found = self._groups[field]
        start = np.frombuffer(found, dtype=np.int64)
        return start, start + np.frombuffer(sizes, dtype=np.int64) * kind.itemsize

    def _check_apart(self):
        """What a step writes is written once, and is not a gradient.  Looked at before the first step with these addresses."""
        if self._written is None:
            starts, ends = (np.concatenate(x) for x in zip(*(self._spans(field) for field in self._groups if field != "grad")))
            order = np.argsort(starts)
            starts, ends = starts[order], ends[order]
            if not np.any(starts[1:] < ends[:-1]):
                self._written = starts, np.concatenate([[0], ends])
        if self._written is not None:
            starts, ends = self._spans("grad")
            before = self._written[0].searchsorted(ends)         # how many begin before its end; the last of these ends furthest
            self._apart = not (self._written[1][before] > starts).any()
        if not self._apart:
            raise B.BmgdError(B.BMGD_EINVAL, "AdamW: tensors that a step writes overlap each other or a gradient")

    def _same_type(self, name, tensors, kinds):
        if len(tensors) != self.count:
            raise ValueError(f"{name}: {self.count} tensors are wanted, not {len(tensors)}")
        kind = tensors[0].dtype if tensors else kinds[0]
        if kind not in kinds:
            raise ValueError(f"{name}: type {kind} is not one of {kinds}")
        return kind

    def set_grads(self, grads):
        """The tensors that later steps read gradients from."""
        grads = list(grads)
        kind = self._same_type("grads", grads, (torch.float32, torch.bfloat16, torch.float16))
        self._fill("grad", grads, kind, self._n)
        self.grads, self.cfg.grad_dtype = grads, _CODES[kind]

    def _launch(self, stream, fn, *args):
        if self.device is None:
            rc = fn(*args, None)                               # (no tensors: checks only)
        else:
            stream = _stream(stream, self.device.index)
            if self._seen is not None and stream not in self._seen:
                # torch must not give their memory away, once they are dropped, before the work on this stream has ended
                self._seen.add(stream)
                for t in itertools.chain.from_iterable(self.state):
                    t.record_stream(torch.cuda.ExternalStream(stream, self.device))
            if torch.cuda.current_device() == self.device.index:
                rc = fn(*args, stream)
            else:
                with torch.cuda.device(self.device):
                    rc = fn(*args, stream)
        if rc != B.BMGD_OK:
            raise B.BmgdError(rc, B.bmgd_last_error(None))

    def step(self, lr=None, grad_scale=1.0, stream=None):
        """One update with the gradients as they stand in stream order, times grad_scale.  Asynchronous.  A step that is captured into a graph keeps its number
        (`steps` + 1) and rates: each replay makes that update again, with that bias correction, and `steps` does not count replays."""
        self._read_again(self._watched[0])
        if not self._apart:
            self._check_apart()
        self.cfg.lr, self.cfg.grad_scale = self.lr if lr is None else lr, grad_scale
        self._launch(stream, B.lib.bmgd_adamw_step, C.byref(self.cfg), self._t, self.count, self.steps + 1)
        self.steps += 1
        _tensors.touch(self.thetas)
        if self.copies:
            _tensors.touch(self.copies)

    def moments(self, out=None, stream=None):
        """Pairs (m, s) of fp32 tensors with the values that the state stands for; `out`: pairs to write them to (otherwise new ones, which belong to
        torch's current stream).  With moments in 32 bits the state itself, and `out` is refused."""
        if self.cfg.state_bits == 32:
            if out is not None:
                raise ValueError("moments in 32 bits are the tensors in `state`")
            return self.state
        self._read_again(self._watched[1])
        if out is None:
            out = [(torch.empty(t.numel(), device=t.device), torch.empty(t.numel(), device=t.device)) for t in self.thetas]
            if out and stream is not None:
                # memory that work on the current stream may still use, and that torch must not give away before the work on this one has ended
                here, there = torch.cuda.current_stream(self.device), torch.cuda.ExternalStream(B._stream(stream), self.device)
                if here != there:
                    there.wait_stream(here)
                    for t in itertools.chain.from_iterable(out):
                        t.record_stream(there)
        out = list(out)
        if len(out) != self.count:
            raise ValueError(f"out: {self.count} pairs are wanted, not {len(out)}")
        found = self._addresses(_tensors.pairs, "out", out, torch.float32, self._n)
        self._launch(stream, B.lib.bmgd_adamw_moments, self._t, self.count, found[0], found[1])
        return out
