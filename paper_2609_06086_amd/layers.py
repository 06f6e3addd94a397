"""ctypes binding of ``include/poseidon_layers.h``: layer operators of a pipeline stage.

Every operator runs in the HIP library ``libposeidon.so``; this module checks
and marshals arguments and allocates outputs and workspaces with torch.  All
tensors live on one GPU.  Matrices are 2-D with neighbouring values in a row;
any row pitch is taken as it is, any other layout of an input is copied first,
and so are the experts' rows (``ys``) on a pitch.  Results are new tensors without
a history: autograd does not see these calls, and the backward operators are called
by name.
Work is enqueued on ``stream`` (a ``torch.cuda.Stream`` or a raw ``hipStream_t``
integer, of the tensors' GPU; default: torch's current stream there), on which
the outputs are allocated too.  Nothing synchronises.  What is refused raises
``PoseidonError`` before anything is enqueued.
"""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from . import poseidon as P
from .poseidon import PoseidonError

GROUP = 64
WIDTH_MAX, PITCH_MAX, ROWS_MAX = 1 << 20, 1 << 24, 2 ** 31 - 1
EXPERTS_MAX, RANGES_MAX, VOCAB_MAX, TILES_MAX = 511, 65535, 2 ** 26 - 1, 1 << 22
TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

_p, _u64, _u32 = C.c_void_p, C.c_uint64, C.c_uint32
_ARGS = {
    "poseidon_stash": [_p, _u64, _u32, _u64, _u64, _p, _p, _p],
    "poseidon_restore": [_p, _p, _u64, _u64, _p, _u64, _u32, _p],
    "poseidon_gated_forward": [_p, _u64, _p, _u64, _u32, _u64, _u64, _p, _u64, _p, _p, _p, _p, _p],
    "poseidon_gated_backward": [_p, _u64, _u32, _u64, _u64, _p, _p, _p, _p, _p, _u64, _p, _u64, _p],
    "poseidon_weight_gradient": [_p, _u64, _u32, _u64, _u64, _p, _p, _u64, _p, _u32, _p, _u32, _u32, _p, _u64, _p],
    "poseidon_weight_gradient_workspace": [_u64, _u64, _u64, _u32],
    "poseidon_expert_sort": [_p, _u64, _u32, _u32, _p, _p, _p, _p, _u64, _p],
    "poseidon_expert_sort_workspace": [_u64, _u32, _u32],
    "poseidon_expert_gather": [_p, _u64, _u32, _u64, _u64, _p, _u32, _p, _p, _p, _p, _p],
    "poseidon_expert_combine": [_p, _u32, _u64, _u64, _p, _u32, _p, _p, _u64, _p],
    "poseidon_expert_combine_backward": [_p, _u64, _p, _u32, _u64, _u64, _p, _u32, _p, _p, _p, _p, _p],
    "poseidon_embed": [_p, _u64, _p, _u64, _u32, _u64, _u64, C.c_float, _p, _u64, _p],
    "poseidon_embed_backward": [_p, _u64, _p, _u64, _u32, _u64, _u64, C.c_float, _p, _u64, _u32, _u32, _p, _u64, _p],
    "poseidon_embed_backward_workspace": [_u64, _u64, _u64],
}
EXPORTS = tuple(_ARGS)

_functions = {}


def lib():
    """The loaded HIP library, with the layer operators' signatures."""
    L = P.lib()
    if not _functions:
        made = {}
        for name, args in _ARGS.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = _u64 if name.endswith("_workspace") else C.c_int
            made[name] = f
        _functions.update(made)    # all at once: other threads may be at it too
    return L


def _function(name: str):
    if not _functions:
        lib()
    return _functions[name]


class Stash:
    """Rows kept in 8 bits: int8 codes [rows, groups * 64] on a 16-byte boundary, uint8 scale bytes [rows, groups], the
    rows' width and the type they came from.  The operators make theirs in one piece of memory, of which codes and scales are views."""
    __slots__ = ("rows", "width", "dtype", "_codes", "_scales", "_memory")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, width: int, dtype: torch.dtype):
        self.rows, self.width, self.dtype = scales.shape[0], width, dtype
        self._codes, self._scales, self._memory = codes, scales, None

    @classmethod
    def empty(cls, rows: int, width: int, dtype: torch.dtype, device) -> "Stash":
        s = cls.__new__(cls)
        s.rows, s.width, s.dtype, s._codes, s._scales = rows, width, dtype, None, None
        s._memory = torch.empty(rows * -(-width // GROUP) * (GROUP + 1), dtype=torch.uint8, device=device)
        return s

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            n = self.rows * _groups(self.width) * GROUP
            self._codes = self._memory[:n].view(torch.int8).view(self.rows, _groups(self.width) * GROUP)
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            n = self.rows * _groups(self.width) * GROUP
            self._scales = self._memory[n:].view(self.rows, _groups(self.width))
        return self._scales

    @property
    def nbytes(self) -> int:
        return self.rows * _groups(self.width) * (GROUP + 1)

    @property
    def device(self) -> torch.device:
        return (self._codes if self._memory is None else self._memory).device

    def tensors(self):
        """The memory it holds."""
        return (self._codes, self._scales) if self._memory is None else (self._memory,)

    def addresses(self):
        """(codes, scales) of a stash that _stash has looked over."""
        if self._memory is None:
            return self._codes.data_ptr(), self._scales.data_ptr()
        at = self._memory.data_ptr()
        return at, at + self.rows * _groups(self.width) * GROUP


@dataclass
class ExpertPlan:
    """Order of a batch's choices by expert: order [tokens * k], position [tokens, k] (-1: dropped), offsets
    [experts + 1], all int32."""
    order: torch.Tensor
    position: torch.Tensor
    offsets: torch.Tensor

    def tensors(self):
        """The memory it holds."""
        return self.order, self.position, self.offsets


def _refuse(where: str):
    raise PoseidonError(P.POSEIDON_E_INVAL, where)


def _streamed(f):
    """Runs f with torch's current stream set to `stream`, and keeps its inputs' memory until that stream is past."""

    @functools.wraps(f)
    def g(*args, stream=None, **kw):
        if stream is None:
            return f(*args, **kw)
        held = [t for a in (*args, *kw.values())
                for t in ((a,) if isinstance(a, torch.Tensor) else a.tensors() if isinstance(a, (Stash, ExpertPlan)) else ())
                if t.is_cuda]
        if not isinstance(stream, torch.cuda.Stream):
            device = held[0].device if held else None    # a raw stream is one of the tensors' GPU
            stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
        elif any(t.device != stream.device for t in held):
            _refuse(f"{f.__name__}: stream: not of the tensors' GPU")
        with torch.cuda.stream(stream):
            out = f(*args, **kw)
        for t in held:
            t.record_stream(stream)
        return out

    return g


def _call(name: str, device: torch.device, *args):
    """Calls the library on torch's current stream of `device`; raises what it refuses."""
    index = device.index
    if torch._C._cuda_getDevice() == index:
        rc = _function(name)(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(device):
            rc = _function(name)(*args, torch._C._cuda_getCurrentRawStream(index))
    if rc != P.POSEIDON_OK:
        raise PoseidonError(rc, name)


def _workspace(name: str, device: torch.device, *sizes):
    """(tensor or None, address, bytes) of the workspace that the sizes need."""
    n = _function(name + "_workspace")(*sizes)
    if n == 2 ** 64 - 1:
        raise PoseidonError(P.POSEIDON_E_RANGE, name)
    if not n:
        return None, None, 0
    w = torch.empty(n, dtype=torch.uint8, device=device)
    return w, w.data_ptr(), n


def _rows(x, where: str, device=None, dtype=None, shape=None):
    """A matrix operand with neighbouring values in a row (copied if it has none): (x, rows, width, pitch)."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dim() != 2 or x.dtype not in TYPES:
        _refuse(f"{where}: not a 2-D float32, float16 or bfloat16 tensor on the GPU")
    n, d = size = x.shape
    if (device is not None and x.device != device) or (dtype is not None and x.dtype != dtype) or \
            (shape is not None and size != shape):
        _refuse(f"{where}: device, type or shape differs from what the others ask for")
    pitch, step = x.stride()
    if n <= 1:
        pitch = d
    if (step != 1 and d > 1) or pitch < d:
        return x.contiguous(), n, d, d
    return x, n, d, pitch


def _out(out, where: str, device, dtype, n: int, d: int):
    """A matrix that the caller brought for a result, or a new one: (out, pitch)."""
    if out is None:
        return torch.empty((n, d), dtype=dtype, device=device), d
    if isinstance(out, torch.Tensor) and out.device == device and out.dtype == dtype and out.shape == (n, d):
        pitch, step = out.stride()
        if n <= 1:
            pitch = d
        if (step == 1 or d <= 1) and pitch >= d:
            return out, pitch
    _refuse(f"{where}: device, type, shape or layout differs from the result's")


def _whole(x, where: str, device, dtype, shape) -> torch.Tensor:
    """An operand without gaps (copied if it has some)."""
    if not isinstance(x, torch.Tensor) or x.device != device or x.dtype != dtype or \
            (shape is not None and x.shape != shape):
        _refuse(f"{where}: not a {dtype} tensor of shape {shape} on {device}")
    return x if x.is_contiguous() else x.contiguous()


def _groups(width: int) -> int:
    return -(-width // GROUP)


def _stash(s, where: str, device, rows=None, width=None) -> Stash:
    if not isinstance(s, Stash) or (rows is not None and s.rows != rows) or (width is not None and s.width != width) or \
            s.device != device:
        _refuse(f"{where}: not a Stash of these sizes on {device}")
    if s._memory is not None:
        return s
    n, g = s.rows, _groups(s.width)
    codes = _whole(s.codes, where, device, torch.int8, (n, g * GROUP))
    scales = _whole(s.scales, where, device, torch.uint8, (n, g))
    return s if codes is s.codes and scales is s.scales else Stash(codes, scales, s.width, s.dtype)


# ---- activations kept in 8 bits ----

@_streamed
def poseidon_stash(x) -> Stash:
    """Rows of x [rows, width] kept in 8 bits."""
    x, n, d, pitch = _rows(x, "poseidon_stash: x")
    dev, dt = x.device, x.dtype
    s = Stash.empty(n, d, dt, dev)
    _call("poseidon_stash", dev, x.data_ptr(), pitch, TYPES[dt], n, d, *s.addresses())
    return s


@_streamed
def poseidon_restore(stash: Stash, *, dtype=None, out=None) -> torch.Tensor:
    """What was kept, [rows, width], in its own type or in `dtype`."""
    if not isinstance(stash, Stash) or stash.device.type != "cuda":
        _refuse("poseidon_restore: stash: not a Stash on the GPU")
    dtype = stash.dtype if dtype is None else dtype
    if dtype not in TYPES:
        _refuse("poseidon_restore: a float32, float16 or bfloat16 result")
    device = stash.device
    s = _stash(stash, "poseidon_restore: stash", device)
    out, pitch = _out(out, "poseidon_restore: out", device, dtype, s.rows, s.width)
    _call("poseidon_restore", device, *s.addresses(), s.rows, s.width, out.data_ptr(), pitch, TYPES[dtype])
    return out


@_streamed
def poseidon_gated_forward(gate, up, *, keep: bool = True, out=None) -> Tuple[torch.Tensor, Optional[Stash], Optional[Stash]]:
    """(silu(gate) * up, gate kept in 8 bits, up kept in 8 bits); without `keep` the latter are None."""
    gate, n, d, gate_pitch = _rows(gate, "poseidon_gated_forward: gate")
    dev, dt = gate.device, gate.dtype
    up, _, _, up_pitch = _rows(up, "poseidon_gated_forward: up", dev, dt, (n, d))
    out, pitch = _out(out, "poseidon_gated_forward: out", dev, dt, n, d)
    sg = Stash.empty(n, d, dt, dev) if keep else None
    su = Stash.empty(n, d, dt, dev) if keep else None
    kept = sg.addresses() + su.addresses() if keep else (None,) * 4
    _call("poseidon_gated_forward", dev, gate.data_ptr(), gate_pitch, up.data_ptr(), up_pitch, TYPES[dt], n, d,
          out.data_ptr(), pitch, *kept)
    return out, sg, su


@_streamed
def poseidon_gated_backward(dout, gate: Stash, up: Stash, *, dgate=None, dup=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dgate, dup) at the kept gate and up."""
    dout, n, d, pitch = _rows(dout, "poseidon_gated_backward: dout")
    dev, dt = dout.device, dout.dtype
    gate = _stash(gate, "poseidon_gated_backward: gate", dev, n, d)
    up = _stash(up, "poseidon_gated_backward: up", dev, n, d)
    dgate, dgate_pitch = _out(dgate, "poseidon_gated_backward: dgate", dev, dt, n, d)
    dup, dup_pitch = _out(dup, "poseidon_gated_backward: dup", dev, dt, n, d)
    _call("poseidon_gated_backward", dev, dout.data_ptr(), pitch, TYPES[dt], n, d, *gate.addresses(),
          *up.addresses(), dgate.data_ptr(), dgate_pitch, dup.data_ptr(), dup_pitch)
    return dgate, dup


@_streamed
def poseidon_weight_gradient(dy, x: Stash, *, offsets=None, dtype=torch.float32, out=None,
                             accumulate: bool = False) -> torch.Tensor:
    """dy^T x from the kept x: [out_width, in_width], or with int32 offsets [ranges + 1] one for each range of rows,
    [ranges, out_width, in_width].  With accumulate it is added to `out`."""
    dy, n, o, pitch = _rows(dy, "poseidon_weight_gradient: dy")
    dev = dy.device
    x = _stash(x, "poseidon_weight_gradient: x", dev, n)
    if accumulate and out is None:
        _refuse("poseidon_weight_gradient: accumulate without out")
    ranges = 1
    if offsets is not None:
        offsets = _whole(offsets, "poseidon_weight_gradient: offsets", dev, torch.int32, None)
        if offsets.dim() != 1 or offsets.numel() < 2:
            _refuse("poseidon_weight_gradient: offsets: not int32 [ranges + 1]")
        ranges = offsets.numel() - 1
    dtype = dtype if out is None else getattr(out, "dtype", None)
    if dtype not in TYPES:
        _refuse("poseidon_weight_gradient: a float32, float16 or bfloat16 result")
    shape = (o, x.width) if offsets is None else (ranges, o, x.width)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
    elif out.device != dev or out.shape != shape or not out.is_contiguous():
        _refuse("poseidon_weight_gradient: out: device, shape or layout differs from the result's")
    w, at, size = _workspace("poseidon_weight_gradient", dev, n, o, x.width, ranges)
    _call("poseidon_weight_gradient", dev, dy.data_ptr(), pitch, TYPES[dy.dtype], n, o, *x.addresses(), x.width,
          None if offsets is None else offsets.data_ptr(), ranges, out.data_ptr(), TYPES[dtype], int(accumulate), at, size)
    return out


# ---- tokens by expert ----

@_streamed
def poseidon_expert_sort(choice, n_experts: int) -> ExpertPlan:
    """Stable order of the choices [tokens, k] (int32) by expert; what is outside [0, n_experts) is dropped."""
    if not isinstance(choice, torch.Tensor) or not choice.is_cuda or choice.dim() != 2 or choice.dtype != torch.int32:
        _refuse("poseidon_expert_sort: choice: not an int32 [tokens, k] tensor on the GPU")
    choice = choice.contiguous()
    n, k = choice.shape
    dev = choice.device
    if not 0 < n_experts <= EXPERTS_MAX or not k:
        raise PoseidonError(P.POSEIDON_E_INVAL if n_experts < 1 or not k else P.POSEIDON_E_RANGE, "poseidon_expert_sort")
    plan = ExpertPlan(torch.empty(n * k, dtype=torch.int32, device=dev), torch.empty_like(choice),
                      torch.empty(n_experts + 1, dtype=torch.int32, device=dev))
    w, at, size = _workspace("poseidon_expert_sort", dev, n, k, n_experts)
    _call("poseidon_expert_sort", dev, choice.data_ptr(), n, k, n_experts, plan.order.data_ptr(),
          plan.position.data_ptr(), plan.offsets.data_ptr(), at, size)
    return plan


def _plan(plan, where: str, device, tokens: int):
    """(position, offsets, the address of their last entry, which is the number of kept choices, k)"""
    if not isinstance(plan, ExpertPlan) or plan.position.dim() != 2 or plan.position.shape[0] != tokens or \
            plan.offsets.dim() != 1 or plan.offsets.shape[0] < 2:
        _refuse(f"{where}: not the ExpertPlan of these tokens")
    position = _whole(plan.position, where, device, torch.int32, None)
    offsets = _whole(plan.offsets, where, device, torch.int32, None)
    return position, offsets, offsets.data_ptr() + 4 * (offsets.shape[0] - 1), position.shape[1]


@_streamed
def poseidon_expert_gather(x, plan: ExpertPlan, *, keep: bool = False, rows: bool = True):
    """(x by expert [tokens * k, width], or None without `rows`; the same rows kept in 8 bits, or None without `keep`)."""
    x, n, d, pitch = _rows(x, "poseidon_expert_gather: x")
    dev, dt = x.device, x.dtype
    position, offsets, kept, k = _plan(plan, "poseidon_expert_gather: plan", dev, n)
    xs = torch.empty(n * k, d, dtype=dt, device=dev) if rows else None
    s = Stash.empty(n * k, d, dt, dev) if keep else None
    if xs is None and s is None:
        _refuse("poseidon_expert_gather: neither rows nor keep")
    _call("poseidon_expert_gather", dev, x.data_ptr(), pitch, TYPES[dt], n, d, position.data_ptr(), k,
          kept, xs.data_ptr() if rows else None, *(s.addresses() if keep else (None, None)))
    return xs, s


@_streamed
def poseidon_expert_combine(ys, plan: ExpertPlan, weights=None, *, out=None) -> torch.Tensor:
    """sum over a token's choices of weight * ys row, [tokens, width]; without weights (float32 [tokens, k]) each
    counts once, which is the gradient of the gather."""
    ys, places, d, pitch = _rows(ys, "poseidon_expert_combine: ys")
    ys = ys if pitch == d else ys.contiguous()
    n = plan.position.shape[0] if isinstance(plan, ExpertPlan) else 0
    dev, dt = ys.device, ys.dtype
    position, _, _, k = _plan(plan, "poseidon_expert_combine: plan", dev, n)
    if places != n * k:
        _refuse("poseidon_expert_combine: ys: not a row for each choice")
    if weights is not None:
        weights = _whole(weights, "poseidon_expert_combine: weights", dev, torch.float32, (n, k))
    out, pitch = _out(out, "poseidon_expert_combine: out", dev, dt, n, d)
    _call("poseidon_expert_combine", dev, ys.data_ptr(), TYPES[dt], n, d, position.data_ptr(), k,
          None if weights is None else weights.data_ptr(), out.data_ptr(), pitch)
    return out


@_streamed
def poseidon_expert_combine_backward(dout, ys, plan: ExpertPlan, weights) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dys [tokens * k, width], dweights float32 [tokens, k]) of poseidon_expert_combine."""
    dout, n, d, pitch = _rows(dout, "poseidon_expert_combine_backward: dout")
    dev, dt = dout.device, dout.dtype
    _, offsets, kept, k = _plan(plan, "poseidon_expert_combine_backward: plan", dev, n)
    order = _whole(plan.order, "poseidon_expert_combine_backward: plan", dev, torch.int32, (n * k,))
    ys, _, _, ys_pitch = _rows(ys, "poseidon_expert_combine_backward: ys", dev, dt, (n * k, d))
    ys = ys if ys_pitch == d else ys.contiguous()
    weights = _whole(weights, "poseidon_expert_combine_backward: weights", dev, torch.float32, (n, k))
    dys, dweights = torch.empty((n * k, d), dtype=dt, device=dev), torch.empty_like(weights)
    _call("poseidon_expert_combine_backward", dev, dout.data_ptr(), pitch, ys.data_ptr(), TYPES[dt], n, d,
          order.data_ptr(), k, kept, weights.data_ptr(), dys.data_ptr(), dweights.data_ptr())
    return dys, dweights


# ---- embedding ----

def _ids(ids, where: str, device) -> torch.Tensor:
    if not isinstance(ids, torch.Tensor) or ids.dim() != 1:
        _refuse(f"{where}: not an int32 [tokens] tensor")
    return _whole(ids, where, device, torch.int32, None)


@_streamed
def poseidon_embed(ids, table, scale: float = 1.0, *, out=None) -> torch.Tensor:
    """scale * table[ids], [tokens, width]; ids (int32) outside the table give zeros."""
    table, v, d, table_pitch = _rows(table, "poseidon_embed: table")
    dev, dt = table.device, table.dtype
    ids = _ids(ids, "poseidon_embed: ids", dev)
    n = ids.numel()
    out, pitch = _out(out, "poseidon_embed: out", dev, dt, n, d)
    _call("poseidon_embed", dev, ids.data_ptr(), n, table.data_ptr(), table_pitch, TYPES[dt], v, d, scale,
          out.data_ptr(), pitch)
    return out


@_streamed
def poseidon_embed_backward(ids, dout, vocab: int, scale: float = 1.0, *, dtype=torch.float32, out=None,
                            accumulate: bool = False) -> torch.Tensor:
    """Gradient [vocab, width] of the table.  With accumulate the sums are added to `out` and the rows of no token
    are left alone."""
    dout, n, d, pitch = _rows(dout, "poseidon_embed_backward: dout")
    dev = dout.device
    ids = _ids(ids, "poseidon_embed_backward: ids", dev)
    if ids.numel() != n or (accumulate and out is None):
        _refuse("poseidon_embed_backward: ids: not one for each row of dout, or accumulate without out")
    dtype = dtype if out is None else getattr(out, "dtype", None)
    if dtype not in TYPES or vocab < 0:
        _refuse("poseidon_embed_backward: a float32, float16 or bfloat16 result")
    out, out_pitch = _out(out, "poseidon_embed_backward: out", dev, dtype, vocab, d)
    w, at, size = _workspace("poseidon_embed_backward", dev, n, vocab, d)
    _call("poseidon_embed_backward", dev, ids.data_ptr(), n, dout.data_ptr(), pitch, TYPES[dout.dtype], vocab, d,
          scale, out.data_ptr(), out_pitch, TYPES[dtype], int(accumulate), at, size)
    return out
