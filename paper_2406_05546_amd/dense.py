"""ctypes binding of the dense-layer and optimizer operators of libps_hotpath.so (include/ps_dense.h): same names,
argument checks and marshalling only.  Tensors are torch cuda tensors; work runs on torch's current stream of their device, and results
and workspaces come from torch's allocator on that stream.  There is no fallback: a missing library or a refused call
raises an exception.  Nothing is recorded for autograd, also where tensors require gradients: the backward passes are calls of their own."""
from __future__ import annotations

import ctypes
import struct
import threading
from dataclasses import dataclass, field
from typing import List, Optional, Sequence, Tuple

import torch

from .binding import PS_EINVAL, PS_OK, PsError, load_library

PS_F32, PS_BF16, PS_F16 = range(3)
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
ADAMW_BLOCK = 256
CHECKPOINT_BLOCK = 32

EXPORTS = ["ps_linear_workspace_bytes", "ps_linear_forward", "ps_linear_backward", "ps_checkpoint_encode", "ps_checkpoint_decode",
           "ps_linear_checkpoint_workspace_bytes", "ps_linear_forward_checkpoint", "ps_linear_backward_checkpoint", "ps_adamw_workspace_bytes", "ps_adamw_create",
           "ps_adamw_destroy", "ps_adamw_step", "ps_dense_last_error"]


class ps_matrix(ctypes.Structure):
    _fields_ = [("data_dev", ctypes.c_void_p), ("row", ctypes.c_int64), ("matrix", ctypes.c_int64)]


class ps_linear(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("activation", ctypes.c_int32), ("rows", ctypes.c_int64), ("in_features", ctypes.c_int64),
                ("out_features", ctypes.c_int64), ("n_groups", ctypes.c_int32), ("n_weights", ctypes.c_int32),
                ("offsets_dev", ctypes.c_void_p), ("weight_of_group_dev", ctypes.c_void_p)]


class ps_checkpoint(ctypes.Structure):
    _fields_ = [("codes_dev", ctypes.c_void_p), ("scales_dev", ctypes.c_void_p), ("row", ctypes.c_int64), ("scale_row", ctypes.c_int64)]


class ps_adamw_tensor(ctypes.Structure):
    _fields_ = [("param_dev", ctypes.c_void_p), ("grad_dev", ctypes.c_void_p), ("copy_dev", ctypes.c_void_p), ("m_dev", ctypes.c_void_p),
                ("v_dev", ctypes.c_void_p), ("m_scale_dev", ctypes.c_void_p), ("v_scale_dev", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("grad_row", ctypes.c_int64), ("grad_rows", ctypes.c_int32), ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("copy_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("weight_decay", ctypes.c_float)]


class ps_adamw_options(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("grad_scale", ctypes.c_double), ("step", ctypes.c_int64), ("n_rows", ctypes.c_int32)]


_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib = load_library()
        vp, i32, u64, p = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.POINTER
        for name, args in {
                "ps_linear_workspace_bytes": [vp, i32, vp],
                "ps_linear_forward": 8 * [vp] + [u64, vp],
                "ps_linear_backward": 9 * [vp] + [u64, vp],
                "ps_checkpoint_encode": [i32, ctypes.c_int64, ctypes.c_int64, vp, vp, vp],
                "ps_checkpoint_decode": [i32, ctypes.c_int64, ctypes.c_int64, vp, i32, vp, vp],
                "ps_linear_checkpoint_workspace_bytes": [vp, i32, i32, vp],
                "ps_linear_forward_checkpoint": 8 * [vp] + [u64, vp],
                "ps_linear_backward_checkpoint": 4 * [vp] + [i32] + 7 * [vp] + [u64, vp],
                "ps_adamw_workspace_bytes": [p(ps_adamw_tensor), i32, p(u64)],
                "ps_adamw_create": [p(vp), p(ps_adamw_tensor), i32, vp, u64, vp],
                "ps_adamw_destroy": [vp],
                "ps_adamw_step": [vp, p(ps_adamw_options), vp]}.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ctypes.c_int
        lib.ps_dense_last_error.argtypes, lib.ps_dense_last_error.restype = [], ctypes.c_char_p
        _lib = lib
    return _lib


def _check(call: str, status: int) -> None:
    if status != PS_OK:
        raise PsError(call, status, (_library().ps_dense_last_error() or b"").decode())


def _refuse(call: str, why: str) -> None:
    raise PsError(call, PS_EINVAL, f"{call}: {why}")


_DTYPES = {torch.float32: PS_F32, torch.bfloat16: PS_BF16, torch.float16: PS_F16}


def _dtype(call: str, name: str, t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        _refuse(call, f"{name} is {t.dtype}, not float32, bfloat16 or float16")
    return code


def _matrix(call: str, name: str, t, device, dtype, shape: Tuple[int, ...], matrices: bool = False) -> Tuple[int, int, int]:
    """Checks that `t` has this shape, type and device; the fields of its ps_matrix."""
    if t.dtype is not dtype or t.get_device() != device.index:
        _refuse(call, f"{name} is {t.dtype} on {t.device}, not {dtype} on {device}")
    if t.shape != shape:
        _refuse(call, f"{name} has the shape {tuple(t.shape)}, not {shape}")
    stride = t.stride()
    cols = shape[-1]
    if cols > 1 and stride[-1] != 1 and t.numel():
        _refuse(call, f"{name}'s rows are not contiguous")
    if matrices:
        rows = shape[1] if len(shape) == 3 else 1
        row = stride[1] if rows > 1 else cols
        return t.data_ptr(), row, stride[0] if shape[0] > 1 else rows * row
    return t.data_ptr(), stride[0] if len(shape) == 2 and shape[0] > 1 else cols, 0


def _ints(call: str, name: str, t, device, n: Optional[int] = None) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.int32 or t.device != device or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.numel() != n):
        _refuse(call, f"{name} is a contiguous int32 tensor" + (f" of {n} elements" if n is not None else "") + " next to the others")
    return t.data_ptr()


# The arguments of a call, written in one go: a ps_linear and one ps_matrix for each operand (ctypes structures, made one by one, take
# most of the time of a small layer).
_LAYER, _MATRIX = "<iiqqqiiQQ", "Qqq"
_LAYER_BYTES, _MATRIX_BYTES = struct.calcsize(_LAYER), struct.calcsize("<" + _MATRIX)
_CHECKPOINT = "QQqq"
_CHECKPOINT_BYTES = struct.calcsize("<" + _CHECKPOINT)
assert _LAYER_BYTES == ctypes.sizeof(ps_linear) and _MATRIX_BYTES == ctypes.sizeof(ps_matrix) and _CHECKPOINT_BYTES == ctypes.sizeof(ps_checkpoint)
_PACK = {n: struct.Struct(_LAYER + n * _MATRIX).pack_into for n in (6, 7)}
_PACK_MATRIX, _PACK_CHECKPOINT = struct.Struct("<" + _MATRIX).pack_into, struct.Struct("<" + _CHECKPOINT).pack_into
_ABSENT = (0, 0, 0)


class _Arguments(threading.local):
    def __init__(self):
        self.memory = ctypes.create_string_buffer(_LAYER_BYTES + 7 * _MATRIX_BYTES + 2 * _CHECKPOINT_BYTES)
        self.need = ctypes.c_uint64(0)
        self.options = ps_adamw_options()
        self.at = ctypes.addressof(self.memory)
        self.at_need = ctypes.addressof(self.need)
        self.at_matrices = [self.at + _LAYER_BYTES + i * _MATRIX_BYTES for i in range(7)]
        self.of_checkpoints = [_LAYER_BYTES + 7 * _MATRIX_BYTES + i * _CHECKPOINT_BYTES for i in range(2)]


_arguments = _Arguments()


@dataclass
class Checkpoint:
    """Activations [rows, cols] in 8 bits, as ps_checkpoint_encode gives them: e4m3 codes, and for every 32 columns of a row a power of two
    that scales them.  Rows are contiguous."""
    codes: torch.Tensor   # [rows, cols] float8_e4m3fn (or uint8)
    scales: torch.Tensor  # [rows, ceil(cols / 32)] float8_e8m0fnu (or uint8)

    @property
    def shape(self) -> torch.Size:
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device


_CODES, _SCALES = (torch.float8_e4m3fn, torch.uint8), (torch.float8_e8m0fnu, torch.uint8)


def _kept(call: str, name: str, c: Checkpoint, device, shape) -> Tuple[int, int, int, int]:
    """Checks that `c` has this shape and device; the fields of its ps_checkpoint."""
    codes, scales = c.codes, c.scales
    blocks = -(-shape[1] // CHECKPOINT_BLOCK)
    if codes.dtype not in _CODES or scales.dtype not in _SCALES or codes.device != device or scales.device != device:
        _refuse(call, f"{name} has {codes.dtype} codes on {codes.device} and {scales.dtype} scales on {scales.device}, not e4m3 and e8m0 ones on {device}")
    if codes.shape != shape or scales.shape != (shape[0], blocks):
        _refuse(call, f"{name} has codes {tuple(codes.shape)} and scales {tuple(scales.shape)}, not {tuple(shape)} and {(shape[0], blocks)}")
    row, scale_row = codes.stride(), scales.stride()
    if codes.numel() and (shape[1] > 1 and row[1] != 1 or blocks > 1 and scale_row[1] != 1):
        _refuse(call, f"{name}'s rows are not contiguous")
    several = shape[0] > 1
    return codes.data_ptr(), scales.data_ptr(), row[0] if several else shape[1], scale_row[0] if several else blocks


def _run_checkpoint(call: str, layer: Tuple[int, ...], backward: int, device, matrices, x8, x_act: int, pre8) -> None:
    """`_run` for calls with a checkpoint: x8 or pre8 are the fields of one in the place of x (then None in `matrices`) or pre, or None."""
    index = device.index
    if index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _run_checkpoint(call, layer, backward, device, matrices, x8, x_act, pre8)
    lib, a = _library(), _arguments
    fields = list(layer)
    for m in matrices:
        fields += m or _ABSENT
    _PACK[len(matrices)](a.memory, 0, *fields)
    kept = []
    for of, c in zip(a.of_checkpoints, (x8, pre8)):
        if c:
            _PACK_CHECKPOINT(a.memory, of, *c)
        kept.append(a.at + of if c else None)
    st = lib.ps_linear_checkpoint_workspace_bytes(a.at, backward, 1 if x8 and matrices[5] else 0, a.at_need)
    if st != PS_OK:
        _check(call, st)
    need = a.need.value
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    at, stream = None if ws is None else ws.data_ptr(), torch._C._cuda_getCurrentRawStream(index)
    refs = [at if m else None for m, at in zip(matrices, a.at_matrices)]
    if backward:
        dy, x, w, pre, dx, dw, db = refs
        st = lib.ps_linear_backward_checkpoint(a.at, dy, x, kept[0], x_act, w, pre, kept[1], dx, dw, db, at, need, stream)
    else:
        st = lib.ps_linear_forward_checkpoint(a.at, *refs[:5], kept[1], at, need, stream)
    if st != PS_OK:
        _check(call, st)


def ps_checkpoint_empty(rows: int, cols: int, device) -> Checkpoint:
    """Room for activations [rows, cols], its contents whatever they are."""
    return Checkpoint(torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=device),
                      torch.empty(rows, -(-cols // CHECKPOINT_BLOCK), dtype=torch.float8_e8m0fnu, device=device))


def _code_call(call: str, dtype: int, x, device, shape, kept, encode: bool, act: int) -> None:
    """kept: the fields of the checkpoint."""
    index = device.index
    if index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _code_call(call, dtype, x, device, shape, kept, encode, act)
    a = _arguments
    _PACK_MATRIX(a.memory, _LAYER_BYTES, *_matrix(call, "x", x, device, x.dtype, shape))
    _PACK_CHECKPOINT(a.memory, a.of_checkpoints[0], *kept)
    lib, at, kept, stream = _library(), a.at_matrices[0], a.at + a.of_checkpoints[0], torch._C._cuda_getCurrentRawStream(index)
    st = lib.ps_checkpoint_encode(dtype, *shape, at, kept, stream) if encode else lib.ps_checkpoint_decode(dtype, *shape, kept, act, at, stream)
    if st != PS_OK:
        _check(call, st)


def ps_checkpoint_encode(x, out: Optional[Checkpoint] = None) -> Checkpoint:
    """x [rows, cols] (float32, bfloat16 or float16, contiguous rows) in 8 bits: a value is off by at most 2^-4 of itself from 2^-13 of its block's
    largest (and from 2^-132) on, below by less than 2^-16 of that largest (or 2^-135).  What is not 0 is not held as 0; what is not finite is
    held as NaN."""
    call = "ps_checkpoint_encode"
    dtype = _dtype(call, "x", x)
    device, shape = x.device, x.shape
    if len(shape) != 2 or device.type != "cuda":
        _refuse(call, "x is [rows, cols] on a GPU")
    if out is None:
        out = ps_checkpoint_empty(*shape, device)
        kept = out.codes.data_ptr(), out.scales.data_ptr(), shape[1], -(-shape[1] // CHECKPOINT_BLOCK)
    else:
        kept = _kept(call, "out", out, device, shape)
    _code_call(call, dtype, x, device, shape, kept, True, 0)
    return out


def ps_checkpoint_decode(c: Checkpoint, dtype=torch.bfloat16, activation: str = "none", out=None):
    """The activation of the values that a checkpoint holds, in `dtype` (or out's)."""
    call = "ps_checkpoint_decode"
    if c.codes.dim() != 2 or c.codes.device.type != "cuda":
        _refuse(call, "the checkpoint is [rows, cols] on a GPU")
    act = ACTIVATIONS.get(activation)
    if act is None:
        _refuse(call, f"unknown activation {activation!r}")
    x = torch.empty(c.shape, dtype=dtype, device=c.device) if out is None else out
    if x.shape != c.shape or x.device != c.device:
        _refuse(call, f"out has the shape {tuple(x.shape)} on {x.device}, not {tuple(c.shape)} on {c.device}")
    _code_call(call, _dtype(call, "out", x), x, c.device, c.shape, _kept(call, "the checkpoint", c, c.device, c.shape), False, act)
    return x


def _layer(call: str, x, w, activation: str, offsets, weight_of_group, dtype_of=None) -> Tuple[int, ...]:
    """The fields of the call's ps_linear.  x may be a checkpoint of the type of `dtype_of`."""
    grouped = offsets is not None
    act = ACTIVATIONS.get(activation)
    if act is None:
        _refuse(call, f"unknown activation {activation!r}")
    if len(x.shape) != 2 or w.dim() != (3 if grouped else 2):
        _refuse(call, "x is [rows, in] and w " + ("[matrices, out, in]" if grouped else "[out, in]"))
    dtype, device = _dtype(call, "x", x) if dtype_of is None else _dtype(call, "dy", dtype_of), x.device
    if device.type != "cuda":
        _refuse(call, f"x is on {device}, not on a GPU")
    rows, fin = x.shape
    if not grouped:
        return dtype, act, rows, fin, w.shape[0], 1, 1, 0, 0
    at = _ints(call, "offsets", offsets, device)
    n_groups = offsets.numel() - 1
    if n_groups < 1:
        _refuse(call, "offsets has one element more than there are groups, of which there is at least one")
    return dtype, act, rows, fin, w.shape[1], n_groups, w.shape[0], at, _ints(call, "weight_of_group", weight_of_group, device, n_groups)


def _run(call: str, layer: Tuple[int, ...], backward: int, device, matrices) -> None:
    """Calls the library with what `_layer` and `_matrix` (or None) gave."""
    index = device.index
    if index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _run(call, layer, backward, device, matrices)
    lib, a, n = _library(), _arguments, len(matrices)
    fields = list(layer)
    for m in matrices:
        fields += m or _ABSENT
    _PACK[n](a.memory, 0, *fields)
    st = lib.ps_linear_workspace_bytes(a.at, backward, a.at_need)
    if st != PS_OK:
        _check(call, st)
    need = a.need.value
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    refs = [at if m else None for m, at in zip(matrices, a.at_matrices)]
    st = (lib.ps_linear_backward if backward else lib.ps_linear_forward)(a.at, *refs, None if ws is None else ws.data_ptr(), need,
                                                                         torch._C._cuda_getCurrentRawStream(index))
    if st != PS_OK:
        _check(call, st)


def _forward(x, offsets, w, bias, residual, activation, weight_of_group, pre, out):
    call = "ps_linear_forward"
    if type(x) is Checkpoint:
        _refuse(call, "x is a checkpoint, which the backward pass reads")
    layer = _layer(call, x, w, activation, offsets, weight_of_group)
    grouped, device, dtype, rows, fin, fout = offsets is not None, x.device, x.dtype, layer[2], layer[3], layer[4]
    mats = (w.shape[0],) if grouped else ()
    of_out = (rows, fout)
    y = x.new_empty(of_out) if out is None else out
    kept = type(pre) is Checkpoint
    matrices = [
        _matrix(call, "x", x, device, dtype, (rows, fin)), _matrix(call, "w", w, device, dtype, mats + (fout, fin), grouped),
        None if bias is None else _matrix(call, "bias", bias, device, dtype, mats + (fout,), grouped),
        None if residual is None else _matrix(call, "residual", residual, device, dtype, of_out), _matrix(call, "out", y, device, dtype, of_out),
        None if pre is None or kept else _matrix(call, "pre", pre, device, dtype, of_out)]
    if kept:
        _run_checkpoint("ps_linear_forward_checkpoint", layer, 0, device, matrices, None, 0, _kept(call, "pre", pre, device, of_out))
    else:
        _run(call, layer, 0, device, matrices)
    return y


def ps_linear_forward(x, w, bias=None, residual=None, activation: str = "none", pre=None, out=None):
    """act(x w^T + bias) + residual.  x [rows, in], w [out, in], bias [out], residual [rows, out], all of one type
    (float32, bfloat16, float16) with contiguous rows; activation "none", "relu", "gelu" or "silu".  pre [rows, out]
    receives the value before the activation, which the backward pass reads; given a Checkpoint, in 8 bits.  out may be the residual.  Returns out."""
    return _forward(x, None, w, bias, residual, activation, None, pre, out)


def ps_grouped_linear_forward(x, offsets, w, bias=None, residual=None, activation: str = "none", weight_of_group=None, pre=None, out=None):
    """The same for rows in groups: group g has rows offsets[g] .. offsets[g + 1] - 1 (int32 on the GPU) and uses matrix
    weight_of_group[g] (or g) of w [matrices, out, in] and of bias [matrices, out].  Rows in no group are left as they are."""
    return _forward(x, offsets, w, bias, residual, activation, weight_of_group, pre, out)


def _backward(dy, x, offsets, w, activation, pre, weight_of_group, need_dx, need_dw, need_db, dx, dw, db, x_activation):
    call = "ps_linear_backward"
    x_kept, pre_kept = type(x) is Checkpoint, type(pre) is Checkpoint
    layer = _layer(call, x, w, activation, offsets, weight_of_group, dy if x_kept else None)
    grouped, device, dtype, rows, fin, fout, groups = offsets is not None, x.device, (dy if x_kept else x).dtype, layer[2], layer[3], layer[4], layer[5]
    x_act = ACTIVATIONS.get(x_activation)
    if x_act is None or (x_act and not x_kept):
        _refuse(call, f"unknown activation {x_activation!r} of x" if x_act is None else "the activation of x goes with an x in 8 bits")
    mats, of = ((w.shape[0],), (groups,)) if grouped else ((), ())
    of_in, of_out, of_w, of_b = (rows, fin), (rows, fout), of + (fout, fin), of + (fout,)
    if dx is None and need_dx:
        dx = dy.new_empty(of_in)
    if dw is None and need_dw:
        dw = dy.new_empty(of_w)
    if db is None and need_db:
        db = dy.new_empty(of_b)
    matrices = [
        _matrix(call, "dy", dy, device, dtype, of_out), None if x_kept else _matrix(call, "x", x, device, dtype, of_in), _matrix(call, "w", w, device, dtype, mats + (fout, fin), grouped),
        None if pre is None or pre_kept else _matrix(call, "pre", pre, device, dtype, of_out), None if dx is None else _matrix(call, "dx", dx, device, dtype, of_in),
        None if dw is None else _matrix(call, "dw", dw, device, dtype, of_w, grouped), None if db is None else _matrix(call, "db", db, device, dtype, of_b, grouped)]
    if x_kept or pre_kept:
        _run_checkpoint("ps_linear_backward_checkpoint", layer, 1, device, matrices, _kept(call, "x", x, device, of_in) if x_kept else None, x_act,
                        _kept(call, "pre", pre, device, of_out) if pre_kept else None)
    else:
        _run(call, layer, 1, device, matrices)
    return dx, dw, db


def ps_linear_backward(dy, x, w, activation: str = "none", pre=None, need_dx: bool = True, need_dw: bool = True, need_db: bool = True,
                       dx=None, dw=None, db=None, x_activation: str = "none"):
    """Gradients (dx, dw, db) of ps_linear_forward for dy [rows, out]; pre as the forward pass wrote it, not needed without
    an activation.  What is not needed is None; dx, dw and db may be given tensors.  The residual's gradient is dy.
    pre and x may be Checkpoints; an x so held is x_activation of its values (that of the layer before, where its pre-activations were kept)."""
    return _backward(dy, x, None, w, activation, pre, None, need_dx, need_dw, need_db, dx, dw, db, x_activation)


def ps_grouped_linear_backward(dy, x, offsets, w, activation: str = "none", pre=None, weight_of_group=None, need_dx: bool = True,
                               need_dw: bool = True, need_db: bool = True, dx=None, dw=None, db=None, x_activation: str = "none"):
    """The same for rows in groups: dw [groups, out, in] and db [groups, out] are every group's own (of a worker, say, whatever
    matrix it used), zeros for a group without rows.  dw and db may be views into wider rows, for instance of a gradient buffer."""
    return _backward(dy, x, offsets, w, activation, pre, weight_of_group, need_dx, need_dw, need_db, dx, dw, db, x_activation)


@dataclass
class AdamW:
    """Handle of one table of tensors, and what it refers to: the weights, gradients and states stay alive with it.  Steps may run on any
    stream (the caller orders them); a handle that is dropped may leave steps behind that still run."""
    handle: ctypes.c_void_p
    device: object
    state_bits: int
    params: List[object]
    grads: List[object]
    m: List[object]
    v: List[object]
    m_scale: List[object]
    v_scale: List[object]
    copies: List[object]
    workspace: object = None
    rows: int = 1                    # gradient rows that every tensor has
    streams: set = field(default_factory=set)  # those on which the allocator knows all of these to be used
    closed: bool = field(default=False)

    def __del__(self):
        if not self.closed and self.handle and _lib is not None:
            self.closed = True
            _lib.ps_adamw_destroy(self.handle)


def ps_adamw_create(params: Sequence, grads: Sequence, state_bits: int = 32, weight_decay=0.0, copies: Optional[Sequence] = None,
                    m: Optional[Sequence] = None, v: Optional[Sequence] = None, m_scale: Optional[Sequence] = None,
                    v_scale: Optional[Sequence] = None) -> AdamW:
    """The table of an AdamW step over `params` (contiguous cuda tensors of float32, bfloat16 or float16).  grads[i]: a
    gradient of params[i]'s shape, or buffered rows of it [rows, numel] whose rows may be any distance apart.  weight_decay: a
    number, or one for each tensor.  copies[i] (or None) receives the new weights in its own type.  The states are made as zeros
    unless given: float32 of the parameter's size, or with 8 bits uint8 or float8_e4m3fn codes and float32 scales, one for
    256 elements.  Waits for the table's copy to the GPU."""
    call = "ps_adamw_create"
    params, grads = list(params), list(grads)
    n = len(params)
    decay = [float(weight_decay)] * n if not isinstance(weight_decay, (list, tuple)) else [float(d) for d in weight_decay]
    copies = [None] * n if copies is None else list(copies)
    if state_bits not in (8, 32):
        _refuse(call, "states have 8 or 32 bits")
    if n == 0:
        _refuse(call, "no tensors")
    device = params[0].device
    if device.type != "cuda":
        _refuse(call, "tensors are on the GPU")
    given = {"m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale}
    states = {}
    for name, lst in given.items():
        if lst is None:
            if name.endswith("scale"):
                lst = [torch.zeros(-(-p.numel() // ADAMW_BLOCK) if state_bits == 8 else 0, device=device) for p in params]
            else:
                lst = [torch.zeros(p.numel(), device=device, dtype=torch.uint8 if state_bits == 8 else torch.float32) for p in params]
        states[name] = list(lst)
    if any(len(lst) != n for lst in (grads, decay, copies, *states.values())):
        _refuse(call, "one gradient, decay, copy and state for each tensor")
    table = (ps_adamw_tensor * n)()
    for i, p in enumerate(params):
        g, c = grads[i], copies[i]
        if p.device != device or not p.is_contiguous():
            _refuse(call, f"tensor {i} is not contiguous, or on another device")
        rows = g.dim() == 2 and tuple(g.shape) != tuple(p.shape) and g.shape[1] == p.numel()
        if g.device != device or not (rows or tuple(g.shape) == tuple(p.shape)) or not (g.is_contiguous() if not rows else g.shape[1] <= 1 or g.stride(1) == 1):
            _refuse(call, f"gradient {i} has neither tensor {i}'s shape nor rows of its {p.numel()} elements, or is not contiguous, or on another device")
        if c is not None and (c.device != device or c.numel() != p.numel() or not c.is_contiguous()):
            _refuse(call, f"copy {i} does not fit tensor {i}")
        for name, lst in states.items():
            s = lst[i]
            scale = name.endswith("scale")
            size = (-(-p.numel() // ADAMW_BLOCK) if state_bits == 8 else 0) if scale else p.numel()
            types = (torch.float32,) if scale or state_bits == 32 else (torch.uint8, torch.float8_e4m3fn)
            if s.device != device or not s.is_contiguous() or s.numel() != size or s.dtype not in types:
                _refuse(call, f"{name}[{i}] does not fit tensor {i}")
        table[i] = ps_adamw_tensor(p.data_ptr(), g.data_ptr(), None if c is None else c.data_ptr(), states["m"][i].data_ptr(), states["v"][i].data_ptr(),
                                   states["m_scale"][i].data_ptr() or None, states["v_scale"][i].data_ptr() or None, p.numel(),
                                   g.stride(0) if rows and g.shape[0] > 1 else p.numel(), g.shape[0] if rows else 1, _dtype(call, f"tensor {i}", p),
                                   _dtype(call, f"gradient {i}", g), 0 if c is None else _dtype(call, f"copy {i}", c), state_bits, decay[i])
    lib = _library()
    size = ctypes.c_uint64(0)
    handle = ctypes.c_void_p()
    with torch.cuda.device(device):
        stream = torch.cuda.current_stream(device).cuda_stream
        _check(call, lib.ps_adamw_workspace_bytes(table, n, ctypes.byref(size)))
        ws = torch.empty(size.value, dtype=torch.uint8, device=device)
        _check(call, lib.ps_adamw_create(ctypes.byref(handle), table, n, ctypes.c_void_p(ws.data_ptr()), size.value,
                                         ctypes.c_void_p(stream)))
    return AdamW(handle, device, state_bits, params, grads, states["m"], states["v"], states["m_scale"], states["v_scale"], copies, ws,
                 min(t.grad_rows for t in table), {stream})


def ps_adamw_step(opt: AdamW, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, grad_scale: float = 1.0,
                  n_rows: Optional[int] = None) -> None:
    """Step number `step` (from 1) with the sum of the first n_rows gradient rows (all that every tensor has, if not given).  Captured into a graph,
    every replay repeats this step's number and rates, and the handle has to be kept for as long."""
    call = "ps_adamw_step"
    if opt.closed:
        _refuse(call, "the table was destroyed")
    index = opt.device.index
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return ps_adamw_step(opt, step, lr, beta1, beta2, eps, grad_scale, n_rows)
    stream = torch._C._cuda_getCurrentRawStream(index)
    if stream not in opt.streams:
        # what the handle keeps may be freed with it while this step runs: not for use on its own stream before that
        current = torch.cuda.current_stream(index)
        for t in (opt.workspace, *opt.params, *opt.grads, *opt.m, *opt.v, *opt.m_scale, *opt.v_scale, *opt.copies):
            if t is not None:
                t.record_stream(current)
        opt.streams.add(stream)
    o = _arguments.options
    o.lr, o.beta1, o.beta2, o.eps, o.grad_scale, o.step, o.n_rows = lr, beta1, beta2, eps, grad_scale, step, opt.rows if n_rows is None else n_rows
    st = _library().ps_adamw_step(opt.handle, ctypes.byref(o), stream)
    if st != PS_OK:
        _check(call, st)


def ps_adamw_state(opt: AdamW, i: int):
    """Both moments of tensor i, as float32 values."""
    if opt.state_bits == 32:
        return opt.m[i], opt.v[i]
    def values(codes, scale):
        return codes.view(torch.float8_e4m3fn).float() * scale.repeat_interleave(ADAMW_BLOCK)[:codes.numel()]
    return values(opt.m[i], opt.m_scale[i]), values(opt.v[i], opt.v_scale[i]).square()


def ps_adamw_destroy(opt: AdamW) -> None:
    if not opt.closed:
        opt.closed = True
        _check("ps_adamw_destroy", _library().ps_adamw_destroy(opt.handle))
