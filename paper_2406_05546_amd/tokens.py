"""ctypes binding of the operators on tokens of libps_hotpath.so (include/ps_tokens.h): same names, argument checks and
marshalling only.  Tensors are torch cuda tensors; work runs on torch's current stream of their device, and results and
workspaces come from torch's allocator on that stream.  There is no fallback: a missing library or a refused call raises an
exception.  Nothing is recorded for autograd: the backward passes are calls of their own."""
from __future__ import annotations

import ctypes
import struct
import threading
from dataclasses import dataclass
from typing import Optional

import torch

from .binding import PS_OK, PsError, load_library
from .dense import _dtype, _ints, _matrix, _refuse

LOGPROB_MAX_TOP = 32
MAX_VOCAB = 1 << 22

EXPORTS = ["ps_embedding_forward", "ps_embedding_workspace_bytes", "ps_embedding_backward", "ps_logprob_workspace_bytes", "ps_logprob_forward", "ps_logprob_backward"]


class ps_tokens(ctypes.Structure):
    _fields_ = [("data_dev", ctypes.c_void_p), ("stride", ctypes.c_int64), ("bytes", ctypes.c_int32)]


class ps_vector(ctypes.Structure):
    _fields_ = [("data_dev", ctypes.c_void_p), ("stride", ctypes.c_int64)]


class ps_embedding(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("n_tables", ctypes.c_int32), ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("dim", ctypes.c_int64), ("offsets_dev", ctypes.c_void_p), ("table_of_group_dev", ctypes.c_void_p), ("scale", ctypes.c_double)]


class ps_logprob(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("top", ctypes.c_int32), ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("scale", ctypes.c_double)]


_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib = load_library()
        vp, u64 = ctypes.c_void_p, ctypes.c_uint64
        for name, args in {
                "ps_embedding_forward": 5 * [vp],
                "ps_embedding_workspace_bytes": 2 * [vp],
                "ps_embedding_backward": 5 * [vp] + [u64, vp],
                "ps_logprob_workspace_bytes": 2 * [vp],
                "ps_logprob_forward": 8 * [vp] + [u64, vp],
                "ps_logprob_backward": 8 * [vp]}.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ctypes.c_int
        lib.ps_dense_last_error.argtypes, lib.ps_dense_last_error.restype = [], ctypes.c_char_p
        _lib = lib
    return _lib


# The arguments of a call, written in one go: what is called, its tokens, and two matrices and vectors.
_EMBEDDING, _LOGPROB = struct.Struct("=3i4xqqqQQd" "Qqi4x" "Qqq" "Qqq"), struct.Struct("=iiqqd" "Qqi4x" "Qqq" "Qqq" "Qq" "Qq")


class _Arguments(threading.local):
    def __init__(self):
        self.memory = ctypes.create_string_buffer(256)
        self.need = ctypes.c_uint64(0)
        at = self.at = ctypes.addressof(self.memory)
        self.at_need = ctypes.addressof(self.need)
        e = ctypes.sizeof(ps_embedding)
        self.embedding = (at, at + e, at + e + 24, at + e + 48)
        p = ctypes.sizeof(ps_logprob)
        self.logprob = (at, at + p, at + p + 24, at + p + 48, at + p + 72, at + p + 88)


assert _EMBEDDING.size == ctypes.sizeof(ps_embedding) + 72 and _LOGPROB.size == ctypes.sizeof(ps_logprob) + 104
_arguments = _Arguments()
_TOKEN_BYTES = {torch.int32: 4, torch.int64: 8}


def _tokens(call: str, t, device, rows: Optional[int] = None):
    """The fields of a ps_tokens."""
    size = _TOKEN_BYTES.get(t.dtype)
    if size is None or t.get_device() != device.index:
        _refuse(call, f"tokens are {t.dtype} on {t.device}, not int32 or int64 on {device}")
    if t.dim() != 1 or (rows is not None and t.shape[0] != rows):
        _refuse(call, f"tokens have the shape {tuple(t.shape)}, not one for each" + ("" if rows is None else f" of {rows} rows"))
    return t.data_ptr(), t.stride(0), size


def _call(call: str, device, *args) -> None:
    """Calls the library on the current stream of the device."""
    index = device.index
    if index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _call(call, device, *args)
    st = getattr(_library(), call)(*args, torch._C._cuda_getCurrentRawStream(index))
    if st != PS_OK:
        raise PsError(call, st, (_library().ps_dense_last_error() or b"").decode())


def _workspace(call: str, name: str, device):
    """A workspace for what the arguments describe (None if none is needed), and its size."""
    a = _arguments
    st = getattr(_library(), name)(a.at, a.at_need)
    if st != PS_OK:
        raise PsError(call, st, (_library().ps_dense_last_error() or b"").decode())
    need = a.need.value
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None, need


def _on_gpu(call: str, name: str, t) -> None:
    if t.device.type != "cuda":
        _refuse(call, f"{name} is on {t.device}, not on a GPU")


def _groups(call: str, offsets, device, index=None):
    if offsets is None:
        return 1, 0, 0
    at = _ints(call, "offsets", offsets, device)
    n = offsets.numel() - 1
    if n < 1:
        _refuse(call, "offsets has one element more than there are groups, of which there is at least one")
    return n, at, _ints(call, "table_of_group", index, device, n)


def _embedding_forward(tokens, offsets, table, scale, table_of_group, out):
    call = "ps_embedding_forward"
    _on_gpu(call, "table", table)
    grouped = offsets is not None
    if table.dim() != (3 if grouped else 2):
        _refuse(call, "table is " + ("[tables, vocab, dim]" if grouped else "[vocab, dim]"))
    device, dtype = table.device, _dtype(call, "table", table)
    shape = tuple(table.shape)
    given = _tokens(call, tokens, device)
    groups, at_offsets, at_index = _groups(call, offsets, device, table_of_group)
    of_out = (tokens.shape[0], shape[-1])
    y = table.new_empty(of_out) if out is None else out
    a = _arguments
    _EMBEDDING.pack_into(a.memory, 0, dtype, groups, shape[0] if grouped else 1, of_out[0], shape[-2], shape[-1], at_offsets, at_index, scale, *given,
                         *_matrix(call, "table", table, device, table.dtype, shape, grouped), *_matrix(call, "out", y, device, table.dtype, of_out))
    _call(call, device, *a.embedding)
    return y


def ps_embedding_forward(tokens, table, scale: float = 1.0, out=None):
    """Rows of `table` [vocab, dim] (float32, bfloat16 or float16, contiguous rows) for `tokens` [rows] (int32 or int64), times
    `scale`; a token outside 0 .. vocab - 1 (padding) gives a row of zeros.  Returns out [rows, dim]."""
    return _embedding_forward(tokens, None, table, scale, None, out)


def ps_grouped_embedding_forward(tokens, offsets, table, scale: float = 1.0, table_of_group=None, out=None):
    """The same for rows in groups: group g has rows offsets[g] .. offsets[g + 1] - 1 (int32 on the GPU) and uses table
    table_of_group[g] (or g) of `table` [tables, vocab, dim].  Rows in no group are left as they are."""
    return _embedding_forward(tokens, offsets, table, scale, table_of_group, out)


def _embedding_backward(dy, tokens, offsets, vocab, scale, dtable):
    call = "ps_embedding_backward"
    _on_gpu(call, "dy", dy)
    if dy.dim() != 2:
        _refuse(call, "dy is [rows, dim]")
    device, dtype, (rows, dim) = dy.device, _dtype(call, "dy", dy), dy.shape
    given = _tokens(call, tokens, device, rows)
    groups, at_offsets, _ = _groups(call, offsets, device)
    if not 1 <= vocab <= MAX_VOCAB:
        _refuse(call, f"vocab is {vocab}, not 1 .. {MAX_VOCAB}")
    shape = (vocab, dim) if offsets is None else (groups, vocab, dim)
    if dtable is None:
        dtable = dy.new_empty(shape)
    a = _arguments
    _EMBEDDING.pack_into(a.memory, 0, dtype, groups, 1, rows, vocab, dim, at_offsets, 0, scale, *given,
                         *_matrix(call, "dy", dy, device, dy.dtype, (rows, dim)), *_matrix(call, "dtable", dtable, device, dy.dtype, shape, offsets is not None))
    ws, need = _workspace(call, "ps_embedding_workspace_bytes", device)
    _call(call, device, *a.embedding, None if ws is None else ws.data_ptr(), need)
    return dtable


def ps_embedding_backward(dy, tokens, vocab: int, scale: float = 1.0, dtable=None):
    """Gradient of ps_embedding_forward's table for dy [rows, dim]: for every token `scale` times the sum of its rows, zeros for
    tokens that are not there.  Returns dtable [vocab, dim]."""
    return _embedding_backward(dy, tokens, None, vocab, scale, dtable)


def ps_grouped_embedding_backward(dy, tokens, offsets, vocab: int, scale: float = 1.0, dtable=None):
    """The same for rows in groups: dtable [groups, vocab, dim] is every group's own, whatever table it used.  dtable may be a view
    into wider rows, for instance of a gradient buffer."""
    return _embedding_backward(dy, tokens, offsets, vocab, scale, dtable)


@dataclass
class LogProb:
    """What ps_logprob_forward gives: float32, the tokens int32."""
    logp: Optional[torch.Tensor]        # [rows]
    norm: torch.Tensor                  # [rows, 3]: largest logit, logarithm of the sum, entropy
    top_logp: Optional[torch.Tensor]    # [rows, top]
    top_tokens: Optional[torch.Tensor]  # [rows, top]

    @property
    def entropy(self) -> torch.Tensor:
        return self.norm[:, 2]


def _logprob(call: str, logits, tokens):
    _on_gpu(call, "logits", logits)
    if logits.dim() != 2:
        _refuse(call, "logits are [rows, vocab]")
    device, (rows, vocab) = logits.device, logits.shape
    return device, _dtype(call, "logits", logits), rows, vocab, (0, 0, 4) if tokens is None else _tokens(call, tokens, device, rows)


def ps_logprob_forward(logits, tokens=None, scale: float = 1.0, top: int = 0) -> LogProb:
    """Log probabilities of `tokens` [rows] (int32 or int64; none: logp is None) under softmax(scale * logits), logits [rows, vocab] of float32,
    bfloat16 or float16 with contiguous rows; the entropy of every row; and its `top` (0 .. 32) most probable tokens, most probable
    first, the lower one among equals.  A token outside 0 .. vocab - 1 has 0.  A logit of -inf has probability 0 and is no alternative: behind the
    last one top_tokens is -1 and top_logp -inf.  A row of nothing but -inf has log probability -inf and entropy 0."""
    call = "ps_logprob_forward"
    device, dtype, rows, vocab, given = _logprob(call, logits, tokens)
    if not 0 <= top <= LOGPROB_MAX_TOP:
        _refuse(call, f"top is {top}, not 0 .. {LOGPROB_MAX_TOP}")
    new = torch.empty
    logp = None if tokens is None else new(rows, device=device, dtype=torch.float32)
    norm = new(rows, 3, device=device, dtype=torch.float32)
    top_logp, top_tokens = (new(rows, top, device=device, dtype=torch.float32), new(rows, top, device=device, dtype=torch.int32)) if top else (None, None)
    a = _arguments
    _LOGPROB.pack_into(a.memory, 0, dtype, top, rows, vocab, scale, *given, *_matrix(call, "logits", logits, device, logits.dtype, (rows, vocab)), *7 * (0,))
    at, at_tokens, at_logits = a.logprob[:3]
    ws, need = _workspace(call, "ps_logprob_workspace_bytes", device)
    _call(call, device, at, at_tokens, at_logits, None if logp is None else logp.data_ptr(), norm.data_ptr(), top_logp.data_ptr() if top else None,
          top_tokens.data_ptr() if top else None, None if ws is None else ws.data_ptr(), need)
    return LogProb(logp, norm, top_logp, top_tokens)


def _numbers(call: str, name: str, t, device, rows: int):
    """The fields of a ps_vector."""
    if t is None:
        return 0, 0
    if t.dtype is not torch.float32 or t.get_device() != device.index or t.shape != (rows,):
        _refuse(call, f"{name} is {t.dtype} {tuple(t.shape)} on {t.device}, not float32 ({rows},) on {device}")
    return t.data_ptr(), t.stride(0) if rows > 1 else 0


def ps_logprob_backward(logits, tokens, norm, dlogp=None, dentropy=None, scale: float = 1.0, out=None):
    """Gradient of the logits from those of ps_logprob_forward's logp (dlogp [rows], float32) and entropy (dentropy [rows]), either of which
    may be None or a broadcast number; norm and scale as in the forward call.  out may be the logits themselves.  Returns out [rows, vocab]."""
    call = "ps_logprob_backward"
    device, dtype, rows, vocab, given = _logprob(call, logits, tokens)
    if dlogp is not None and tokens is None:
        _refuse(call, "a gradient of log probabilities, and no tokens")
    if norm.dtype is not torch.float32 or norm.get_device() != device.index or norm.shape != (rows, 3) or not norm.is_contiguous():
        _refuse(call, f"norm is not what the forward pass gives for {rows} rows")
    shape = (rows, vocab)
    d = torch.empty(shape, device=device, dtype=logits.dtype) if out is None else out
    a = _arguments
    _LOGPROB.pack_into(a.memory, 0, dtype, 0, rows, vocab, scale, *given, *_matrix(call, "logits", logits, device, logits.dtype, shape),
                       *_matrix(call, "out", d, device, logits.dtype, shape), *_numbers(call, "dlogp", dlogp, device, rows), *_numbers(call, "dentropy", dentropy, device, rows))
    at, at_tokens, at_logits, at_out, at_dlogp, at_dentropy = a.logprob
    _call(call, device, at, at_tokens, at_logits, norm.data_ptr(), at_dlogp, at_dentropy, at_out)
    return d
