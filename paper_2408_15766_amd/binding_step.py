"""ctypes binding of the operators of a training step (spec_step.h): same names as the C ABI, argument marshalling only.

As in binding.py: torch is used for device memory and for the current HIP stream, every tensor has to be on the current device, what
a call does not support is refused with SpecError before anything is launched.  The functions compute gradients when they are asked to and register nothing
with autograd.
"""
from __future__ import annotations

import ctypes as C
import itertools
import struct
from typing import Optional, Sequence

from .binding import SPEC_EINVAL, SPEC_ROPE_MAX_DIM, SpecError, _INT_MAX, _dtype_code, _fit, _here, _new, _refuse, lib, spec_rotary_plan_t

SPEC_GRAD_SUMS = 1024
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}

lib.spec_k_embed.argtypes = [C.c_int32, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_float, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]
lib.spec_k_embed_grad_scratch_bytes.restype = C.c_uint64
lib.spec_k_embed_grad_scratch_bytes.argtypes = [C.c_int32] * 3
lib.spec_k_embed_grad.argtypes = [C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_int32, C.c_int32, C.c_void_p,
                                  C.c_int64, C.c_void_p, C.c_uint64, C.c_void_p]
lib.spec_k_headnorm_rotary.argtypes = [C.POINTER(spec_rotary_plan_t), C.c_int32, C.c_char_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_float, C.c_void_p]
lib.spec_k_headnorm_rotary_grad_scratch_bytes.restype = C.c_uint64
lib.spec_k_headnorm_rotary_grad_scratch_bytes.argtypes = [C.c_int32] * 2
lib.spec_k_headnorm_rotary_grad.argtypes = [C.POINTER(spec_rotary_plan_t), C.c_int32, C.c_char_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_float,
                                            C.c_void_p, C.c_uint64, C.c_void_p]
lib.spec_k_ffn_gated.argtypes = [C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]
lib.spec_k_ffn_gated_grad_scratch_bytes.restype = C.c_uint64
lib.spec_k_ffn_gated_grad_scratch_bytes.argtypes = [C.c_int32] * 3
lib.spec_k_ffn_gated_grad.argtypes = [C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p,
                                      C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_uint64, C.c_void_p]
lib.spec_k_ffn_gated_plan.argtypes = [C.c_int32] * 3 + [C.POINTER(C.c_int32)] * 7
lib.spec_k_grad_sums.argtypes = [C.c_int32, C.c_char_p, C.c_void_p, C.c_void_p]
lib.spec_k_grad_clip.argtypes = [C.c_int32, C.c_char_p, C.c_void_p, C.c_double, C.c_void_p, C.c_void_p]


def _room(what: str, scratch, n: int, beside):
    """(the scratch tensor, its bytes): the caller's, or a new one of n bytes."""
    import torch
    if scratch is None:
        return (_new((n,), (1,), torch.uint8, beside) if n else None), n
    if not scratch.is_contiguous():
        _refuse(what, "scratch has to be contiguous")
    return scratch, scratch.numel() * scratch.element_size()


def _matrix(what: str, name: str, t, rows: Optional[int] = None, cols: Optional[int] = None) -> int:
    """The row stride of a matrix with dense rows."""
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols) or (t.shape[1] > 1 and t.stride(1) != 1):
        _refuse(what, f"{name} has to be [{'rows' if rows is None else rows}, {'columns' if cols is None else cols}] with dense rows")
    if t.shape[0] > _INT_MAX or t.shape[1] > _INT_MAX:
        _refuse(what, f"{name} is {tuple(t.shape)}")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _tokens(what: str, tok):
    import torch
    if tok.dtype is not torch.int32 or tok.dim() != 1 or not tok.is_contiguous() or tok.shape[0] > _INT_MAX:
        _refuse(what, "tok has to be int32 [rows]")
    return tok.shape[0]


# ---- embedding ----------------------------------------------------------------------------------

def spec_k_embed(table, tok, scale: float = 1.0, out_dtype=None, out=None):
    """table: [vocab, d] (bf16 or fp32, rows may be strided), tok: int32 [rows] -> scale * table[tok] in out_dtype (default: the table's), zeros for
    tokens outside the table (padding).  out: optional [rows, d] tensor (rows may be strided)."""
    what = "spec_k_embed"
    stream = _here(what, table, tok, out)
    ldt, rows = _matrix(what, "table", table), _tokens(what, tok)
    vocab, d = table.shape
    if out is None:
        out = _new((rows, d), (d, 1), table.dtype if out_dtype is None else out_dtype, table)
    elif out_dtype is not None and out_dtype is not out.dtype:
        _refuse(what, "out has to be of out_dtype")
    ldo = _matrix(what, "out", out, rows, d)
    rc = lib.spec_k_embed(_dtype_code(what, table.dtype), table.data_ptr(), ldt, vocab, d, tok.data_ptr(), rows, scale, _dtype_code(what, out.dtype), out.data_ptr(),
                          ldo, stream)
    if rc:
        raise SpecError(rc, f"{what}: {rows} rows of a {vocab} x {d} table")
    return out


def spec_k_embed_grad_scratch_bytes(rows: int, vocab: int, d: int) -> int:
    return int(lib.spec_k_embed_grad_scratch_bytes(rows, vocab, d)) if _fit(rows, vocab, d) else 0


def spec_k_embed_grad(dy, tok, vocab: int, scale: float = 1.0, out_dtype=None, out=None, accumulate: bool = False, scratch=None):
    """The gradient of spec_k_embed's table: dy [rows, d] (bf16 or fp32, rows may be strided), tok int32 [rows] -> [vocab, d] in out_dtype (default:
    dy's).  out: optional tensor for it (rows may be strided); accumulate: the gradient is added to out's values, and rows without a token stay untouched.
    scratch: optional uint8 tensor of spec_k_embed_grad_scratch_bytes(rows, vocab, d)."""
    import torch
    what = "spec_k_embed_grad"
    stream = _here(what, dy, tok, out, scratch)
    rows = _tokens(what, tok)
    ldy = _matrix(what, "dy", dy, rows)
    d = dy.shape[1]
    if out is None:
        if accumulate:
            _refuse(what, "accumulate needs an out")
        if not 1 <= vocab <= _INT_MAX:
            _refuse(what, f"a vocabulary of {vocab}")
        out = _new((vocab, d), (d, 1), dy.dtype if out_dtype is None else out_dtype, dy)
    elif out_dtype is not None and out_dtype is not out.dtype:
        _refuse(what, "out has to be of out_dtype")
    ldt = _matrix(what, "out", out, vocab, d)
    scratch, room = _room(what, scratch, lib.spec_k_embed_grad_scratch_bytes(rows, vocab, d), dy)
    rc = lib.spec_k_embed_grad(_dtype_code(what, dy.dtype), dy.data_ptr(), ldy, tok.data_ptr(), rows, d, vocab, scale, bool(accumulate), _dtype_code(what, out.dtype),
                               out.data_ptr(), ldt, None if scratch is None else scratch.data_ptr(), room, stream)
    if rc:
        raise SpecError(rc, f"{what}: {rows} rows, a {vocab} x {d} table, {room} bytes of scratch")
    return out


# ---- norms of heads, with the rotary embedding -----------------------------------------------------

_part = "QQqqqqiiii"
_norm_parts = [struct.Struct("@" + (_part + "Qif") * n).pack for n in range(4)]          # spec_headnorm_part, as often as there are tensors
_norm_grad_parts = [struct.Struct("@" + (_part + "QifQqqQii") * n).pack for n in range(4)]


def _positions(what: str, pos, rows: int):
    """(pointer, first position) of the rows' positions."""
    import torch
    if isinstance(pos, torch.Tensor):
        if pos.dtype is not torch.int32 or pos.dim() != 1 or pos.shape[0] != rows or not pos.is_contiguous():
            _refuse(what, f"pos has to be int32 [{rows}]")
        return pos.data_ptr(), 0
    if not -_INT_MAX - 1 <= int(pos) <= _INT_MAX:
        _refuse(what, f"position {pos}")
    return None, int(pos)


# (Most of a small call is the host's share, 10 us beside a kernel of 5: each thing is asked once, in the loop.)

def _outs(like, dtypes):
    """New dense tensors [rows, heads, hd] beside those of `like`."""
    made = []
    for t, d in zip(like, dtypes):
        rows, heads, hd = t.shape
        made.append(_new((rows, heads, hd), (heads * hd, hd, 1), d, t))
    return made


def _rotary_fields(what: str, x, o, turn, rows: int, hd: int, name: str):
    """spec_rotary_part of a tensor and its output."""
    import torch
    shape, dtype, out_dtype, bf16, fp32 = x.shape, x.dtype, o.dtype, torch.bfloat16, torch.float32
    if len(shape) != 3 or shape[0] != rows or shape[2] != hd or shape != o.shape or shape[1] > 1024:
        _refuse(what, f"{name} and outputs have to be [{rows}, up to 1024 heads, {hd}]")
    (ldx, hsx, one), (ldo, hso, two) = x.stride(), o.stride()
    if hd > 1 and not one == two == 1:
        _refuse(what, "the dims of a head have to be dense")
    if (dtype is not bf16 and dtype is not fp32) or (out_dtype is not bf16 and out_dtype is not fp32):
        _refuse(what, f"{dtype} to {out_dtype} (float32 and bfloat16 are supported)")
    return (x.data_ptr(), o.data_ptr(), ldx, hsx, ldo, hso, shape[1], dtype is bf16, out_dtype is bf16, bool(turn))


def _weight(what: str, w, hd: int):
    if w is None:
        return 0, 0
    if w.dim() != 1 or w.shape[0] != hd or not w.is_contiguous():
        _refuse(what, f"weights have to be [{hd}]")
    return w.data_ptr(), _dtype_code(what, w.dtype)


def spec_k_headnorm_rotary(plan: spec_rotary_plan_t, xs: Sequence, pos, weights: Sequence, eps: float = 1e-6, offset: float = 0.0, turned: Optional[Sequence[bool]] = None,
                           out_dtypes: Optional[Sequence] = None, outs=None):
    """spec_k_rotary (xs, pos, turned, out_dtypes, outs as there) with a norm of every head before it: x / sqrt(mean x^2 + eps) * (offset + weights[i]), weights[i]
    a [hd] tensor, or None: that tensor is not normed."""
    import torch
    what = "spec_k_headnorm_rotary"
    n = len(xs)
    if not 1 <= n <= 3 or any(x.dim() != 3 for x in xs):
        _refuse(what, "one to three tensors [rows, heads, hd] are needed")
    made = outs is None
    if made:
        outs = _outs(xs, [x.dtype for x in xs] if out_dtypes is None else out_dtypes)
    if len(outs) != n or len(weights) != n or (turned is not None and len(turned) != n):
        _refuse(what, "as many outputs, weights and flags as tensors are needed")
    stream = _here(what, *xs, *(() if made else outs), *weights, pos if isinstance(pos, torch.Tensor) else None)
    rows, _, hd = xs[0].shape
    if rows > _INT_MAX or hd > SPEC_ROPE_MAX_DIM:
        _refuse(what, f"{rows} rows, heads of {hd}")
    at, first = _positions(what, pos, rows)
    fields = []
    for x, o, w, turn in zip(xs, outs, weights, (True,) * n if turned is None else turned):
        fields += _rotary_fields(what, x, o, turn, rows, hd, "tensors")
        fields += _weight(what, w, hd)
        fields.append(offset)
    rc = lib.spec_k_headnorm_rotary(C.byref(plan), n, _norm_parts[n](*fields), hd, rows, at, first, eps, stream)
    if rc:
        raise SpecError(rc, f"{what}: {rows} rows, heads of {hd}, plan over {plan.rot}, eps {eps}")
    return list(outs)


def spec_k_headnorm_rotary_grad_scratch_bytes(n_parts: int, hd: int) -> int:
    return int(lib.spec_k_headnorm_rotary_grad_scratch_bytes(n_parts, hd)) if _fit(n_parts, hd) else 0


def spec_k_headnorm_rotary_grad(plan: spec_rotary_plan_t, dys: Sequence, xs: Sequence, pos, weights: Sequence, eps: float = 1e-6, offset: float = 0.0,
                                turned: Optional[Sequence[bool]] = None, out_dtypes: Optional[Sequence] = None, outs=None, scratch=None):
    """The gradients of spec_k_headnorm_rotary: dys, those of its outputs, and its inputs xs (None where weights[i] is None) -> (gradients of xs, in
    out_dtypes (default: each dy's) or `outs` (an entry may be the dy itself), gradients of weights: fp32 [hd] each, None where weights[i] is None).
    scratch: optional uint8 tensor of spec_k_headnorm_rotary_grad_scratch_bytes(len(dys), hd)."""
    import torch
    what = "spec_k_headnorm_rotary_grad"
    n = len(dys)
    if not 1 <= n <= 3 or any(t.dim() != 3 for t in dys):
        _refuse(what, "one to three tensors [rows, heads, hd] are needed")
    made = outs is None
    if made:
        outs = _outs(dys, [t.dtype for t in dys] if out_dtypes is None else out_dtypes)
    if len(outs) != n or len(xs) != n or len(weights) != n or (turned is not None and len(turned) != n):
        _refuse(what, "as many inputs, outputs, weights and flags as gradients are needed")
    stream = _here(what, *dys, *(() if made else outs), *xs, *weights, scratch, pos if isinstance(pos, torch.Tensor) else None)
    rows, _, hd = dys[0].shape
    if rows > _INT_MAX or hd > SPEC_ROPE_MAX_DIM:
        _refuse(what, f"{rows} rows, heads of {hd}")
    at, first = _positions(what, pos, rows)
    dws, fields = [], []
    for dy, x, o, w, turn in zip(dys, xs, outs, weights, (True,) * n if turned is None else turned):
        fields += _rotary_fields(what, dy, o, turn, rows, hd, "gradients")
        fields += _weight(what, w, hd)
        fields.append(offset)
        if w is None:
            dws.append(None)
            fields += (0, 0, 0, 0, 0, 0)
            continue
        if x is None or x.shape != dy.shape or (hd > 1 and x.stride(2) != 1):
            _refuse(what, f"the input of a normed tensor has to be {tuple(dy.shape)} with dense heads")
        dw = _new((hd,), (1,), torch.float32, dy)
        dws.append(dw)
        fields += (x.data_ptr(), x.stride(0), x.stride(1), dw.data_ptr(), _dtype_code(what, x.dtype), 0)
    need = lib.spec_k_headnorm_rotary_grad_scratch_bytes(n, hd) if any(w is not None for w in weights) else 0
    scratch, room = _room(what, scratch, need, dys[0])
    rc = lib.spec_k_headnorm_rotary_grad(C.byref(plan), n, _norm_grad_parts[n](*fields), hd, rows, at, first, eps, None if scratch is None else scratch.data_ptr(), room,
                                         stream)
    if rc:
        raise SpecError(rc, f"{what}: {rows} rows, heads of {hd}, plan over {plan.rot}, eps {eps}, {room} bytes of scratch")
    return list(outs), dws


# ---- gated feed-forward block -----------------------------------------------------------------------

def _ffn_args(what: str, x, w_gate, w_up, act: str):
    """(rows, d, f, ldx, ldw) of a call."""
    import torch
    if act not in ACTIVATIONS:
        _refuse(what, f"activation {act!r} ({', '.join(ACTIVATIONS)} are supported)")
    for t in (x, w_gate, w_up):
        if t.dtype is not torch.bfloat16:
            _refuse(what, f"{t.dtype} (bfloat16 is supported)")
    ldx, ldw = _matrix(what, "x", x), _matrix(what, "w_gate", w_gate, None, x.shape[1])
    if _matrix(what, "w_up", w_up, *w_gate.shape) != ldw:
        _refuse(what, "w_gate and w_up have to have the same strides")
    return x.shape[0], x.shape[1], w_gate.shape[0], ldx, ldw


def _bf16_out(what: str, name: str, t, rows: int, cols: int, beside):
    """(an output, its row stride): the caller's, or a new one."""
    import torch
    if t is None:
        return _new((rows, cols), (cols, 1), torch.bfloat16, beside), cols
    if t.dtype is not torch.bfloat16:
        _refuse(what, f"{name} has to be bfloat16")
    return t, _matrix(what, name, t, rows, cols)


def spec_k_ffn_gated(x, w_gate, w_up, act: str = "silu", out=None):
    """act(x w_gate^T) * (x w_up^T): x [rows, d], w_gate and w_up [f, d] as they are trained, bf16 (rows may be strided, by multiples of 8; d and f are multiples
    of 8) -> bf16 [rows, f].  act: silu, gelu or gelu_tanh.  out: optional tensor for it (rows may be strided)."""
    what = "spec_k_ffn_gated"
    stream = _here(what, x, w_gate, w_up, out)
    rows, d, f, ldx, ldw = _ffn_args(what, x, w_gate, w_up, act)
    out, ldh = _bf16_out(what, "out", out, rows, f, x)
    rc = lib.spec_k_ffn_gated(x.data_ptr(), ldx, rows, d, w_gate.data_ptr(), w_up.data_ptr(), ldw, f, ACTIVATIONS[act], out.data_ptr(), ldh, stream)
    if rc:
        raise SpecError(rc, f"{what}: {rows} rows, {d} by {f} (multiples of 8, 16-byte aligned), strides {ldx}, {ldw}, {ldh}")
    return out


def spec_k_ffn_gated_grad_scratch_bytes(rows: int, d: int, f: int) -> int:
    return int(lib.spec_k_ffn_gated_grad_scratch_bytes(rows, d, f)) if _fit(rows, d, f) else 0


def spec_k_ffn_gated_grad(x, w_gate, w_up, dh, act: str = "silu", outs: Optional[Sequence] = None, want: Sequence[bool] = (True, True), scratch=None):
    """The gradients of spec_k_ffn_gated for dh [rows, f] (bf16): (dx [rows, d], dw_gate [f, d], dw_up [f, d]), bf16.  want: whether those of x and of the weights are
    formed (None in the place of what is not).  outs: optional three tensors for them (or None each; rows may be strided, both weights' alike).  scratch: optional uint8 tensor of
    spec_k_ffn_gated_grad_scratch_bytes(rows, d, f)."""
    import torch
    what = "spec_k_ffn_gated_grad"
    dx, dwg, dwu = (None, None, None) if outs is None else outs
    stream = _here(what, x, w_gate, w_up, dh, dx, dwg, dwu, scratch)
    rows, d, f, ldx, ldw = _ffn_args(what, x, w_gate, w_up, act)
    if dh.dtype is not torch.bfloat16:
        _refuse(what, f"{dh.dtype} (bfloat16 is supported)")
    lddh = _matrix(what, "dh", dh, rows, f)
    if (dx is not None and not want[0]) or ((dwg is not None or dwu is not None) and not want[1]) or not any(want):
        _refuse(what, "an output that is not wanted")
    lddx = lddw = 0
    if want[0]:
        dx, lddx = _bf16_out(what, "dx", dx, rows, d, x)
    if want[1]:
        (dwg, lddw), (dwu, other) = _bf16_out(what, "dw_gate", dwg, f, d, x), _bf16_out(what, "dw_up", dwu, f, d, x)
        if lddw != other:
            _refuse(what, "dw_gate and dw_up have to have the same strides")
    scratch, room = _room(what, scratch, lib.spec_k_ffn_gated_grad_scratch_bytes(rows, d, f), x)
    rc = lib.spec_k_ffn_gated_grad(x.data_ptr(), ldx, rows, d, w_gate.data_ptr(), w_up.data_ptr(), ldw, f, ACTIVATIONS[act], dh.data_ptr(), lddh,
                                   None if dx is None else dx.data_ptr(), lddx, None if dwg is None else dwg.data_ptr(), None if dwu is None else dwu.data_ptr(), lddw,
                                   None if scratch is None else scratch.data_ptr(), room, stream)
    if rc:
        raise SpecError(rc, f"{what}: {rows} rows, {d} by {f} (multiples of 8, 16-byte aligned), strides {ldx}, {ldw}, {lddh}, {lddx}, {lddw}, {room} bytes of scratch")
    return dx, dwg, dwu


def spec_k_ffn_gated_plan(rows: int, d: int, f: int):
    """How calls of these sizes run: (kernel of the forward call, tiles of g and u formed again, tiles of dx, ranges of its k, tiles of the weights' gradients, ranges of their k, whether a call for all
    gradients forms dx and those in one launch)."""
    out = [C.c_int32() for _ in range(7)]
    rc = lib.spec_k_ffn_gated_plan(rows, d, f, *(C.byref(o) for o in out)) if _fit(rows, d, f) else SPEC_EINVAL
    if rc:
        raise SpecError(rc, f"spec_k_ffn_gated_plan: {rows} rows, {d} by {f}")
    return tuple(o.value for o in out)


# ---- gradient clipping ------------------------------------------------------------------------------

_grad_dtypes = {}                                               # torch's two types -> the C ABI's (torch is imported by the first call)


def _grad_fields(what: str, grads, outs):
    """spec_grad_part, as often as there are tensors.  By maps over the tensors' methods: a loop took 2 us a tensor."""
    import torch
    tensor, device = torch.Tensor, torch.cuda.current_device()
    if not _grad_dtypes:
        _grad_dtypes.update({torch.float32: 0, torch.bfloat16: 1})
    every = grads if outs is grads else [*grads, *outs]
    if not all(map(tensor.is_contiguous, every)):
        _refuse(what, "gradients and outputs have to be contiguous")
    if any(at != device for at in map(tensor.get_device, every)):
        _refuse(what, f"tensors on {sorted({str(t.device) for t in every})}, and the current device is cuda:{device}")
    types = [_grad_dtypes.get(t.dtype) for t in every]
    if None in types:
        _refuse(what, f"{[t.dtype for t in every][types.index(None)]} (float32 and bfloat16 are supported)")
    where, sizes, n = list(map(tensor.data_ptr, every)), list(map(tensor.numel, every)), len(grads)
    if sizes[:n] != sizes[-n:] and n:
        _refuse(what, "outputs have to have as many elements as their gradients")
    return struct.pack("@" + "QQqii" * n, *itertools.chain.from_iterable(zip(where[:n], where[-n:], sizes, types[:n], types[-n:]))) if n else b""


def spec_k_grad_sums(grads: Sequence, sums=None):
    """The squares of all elements of the tensors (bf16 or fp32, contiguous), summed up: a float64 tensor [SPEC_GRAD_SUMS] whose sum is the square of their norm (processes
    that each hold a part of the gradients all-reduce it).  sums: optional tensor for it."""
    import torch
    what = "spec_k_grad_sums"
    if not grads and sums is None:
        _refuse(what, "tensors or sums are needed")
    beside = grads[0] if grads else sums
    if sums is None:
        sums = _new((SPEC_GRAD_SUMS,), (1,), torch.float64, beside)
    elif sums.dtype is not torch.float64 or tuple(sums.shape) != (SPEC_GRAD_SUMS,) or not sums.is_contiguous():
        _refuse(what, f"sums has to be float64 [{SPEC_GRAD_SUMS}]")
    stream = _here(what, sums)
    rc = lib.spec_k_grad_sums(len(grads), _grad_fields(what, grads, grads), sums.data_ptr(), stream)
    if rc:
        raise SpecError(rc, f"{what}: {len(grads)} tensors")
    return sums


def spec_k_grad_clip(grads: Sequence, sums, max_norm: float, outs: Optional[Sequence] = None):
    """The tensors times min(1, max_norm / (norm + 1e-6)), norm^2 the sum of `sums` (spec_k_grad_sums): in place, or into `outs` (of as many elements, bf16 or fp32).  Returns the
    norm before that, a float32 tensor [] on the device; nothing waits for it."""
    import torch
    what = "spec_k_grad_clip"
    if sums.dtype is not torch.float64 or tuple(sums.shape) != (SPEC_GRAD_SUMS,) or not sums.is_contiguous():
        _refuse(what, f"sums has to be float64 [{SPEC_GRAD_SUMS}]")
    if outs is not None and len(outs) != len(grads):
        _refuse(what, "as many outputs as gradients are needed")
    stream = _here(what, sums)
    norm = _new((), (), torch.float32, sums)
    rc = lib.spec_k_grad_clip(len(grads), _grad_fields(what, grads, grads if outs is None else outs), sums.data_ptr(), max_norm, norm.data_ptr(), stream)
    if rc:
        raise SpecError(rc, f"{what}: {len(grads)} tensors, max_norm {max_norm} (outputs may overlap nothing but their own gradient, in place)")
    return norm
