"""Operators of a worker's local step on CUDA tensors: the calls of include/halos_step.h.

    rope, rotary                      rotary positions (rotary: with autograd)
    attention_forward, _backward      masked attention and its gradients; attention: with autograd
    distill_forward, _backward, distill_loss_and_grad      the loss against labels and a teacher's top logits; distill_loss: with autograd
    embedding_forward, _backward      rows of a table by tokens, scaled, and the table's gradient; embedding: with autograd
    rms_norm_forward, _quantized, _backward      root-mean-square norm with the residual's addition; rms_norm: with autograd (not in 8 bits)
    grad_norm, clip_grads, sgd_step   the norm of many gradients at once, clipping by it, and a step of plain descent

As in ``binding``, the arithmetic is the CUDA library's; what happens here is checking, marshalling and output
allocation, on the current stream of the tensors' device.  The caller's current device stays what it was.  There is no CPU path.
Errors are ``HalosError``.  Everything can be captured into CUDA graphs; a backward pass by autograd while no graph of the same leaves that was
built outside the capture is alive, since torch accumulates on that graph's stream.
"""
from __future__ import annotations

import array
import ctypes as C
import functools
import math
import operator
import struct
from typing import Optional

import torch

from .binding import BF16, ERR_INVALID_ARG, ERR_UNSUPPORTED, F32, HalosError, load_library

F16 = 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
_LAYOUTS = {"half": ROPE_HALF, "interleaved": ROPE_INTERLEAVED}
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

EXPORTED = ("halos_step_error", "halos_step_fault", "halos_rope", "halos_attention_fwd", "halos_attention_bwd",
            "halos_attention_workspace", "halos_distill_fwd", "halos_distill_bwd", "halos_distill_fwd_bwd",
            "halos_embedding_fwd", "halos_embedding_bwd", "halos_embedding_workspace", "halos_rms_norm_fwd", "halos_rms_norm_bwd",
            "halos_rms_norm_workspace", "halos_grad_norm", "halos_clip_grads", "halos_sgd_step", "halos_grads_workspace")

_u32, _i32, _i64, _u64, _vp, _f32 = C.c_uint32, C.c_int32, C.c_int64, C.c_uint64, C.c_void_p, C.c_float
_stride3 = _i64 * 3


class RopeArgs(C.Structure):
    _fields_ = [("struct_size", _u32), ("device", _i32), ("stream", _vp), ("dtype", _u32), ("layout", _u32), ("inverse", _u32),
                ("positions_64", _u32), ("batch", _i64), ("seq", _i64), ("n_q", _u32), ("n_k", _u32), ("head_dim", _u32),
                ("rot_dim", _u32), ("magnitude", _f32), ("reserved", _u32), ("freqs", _vp), ("positions", _vp),
                ("position_stride", _i64 * 2), ("position_offset", _i64), ("q_in", _vp), ("k_in", _vp), ("q_out", _vp),
                ("k_out", _vp), ("q_in_stride", _stride3), ("k_in_stride", _stride3), ("q_out_stride", _stride3), ("k_out_stride", _stride3)]


class AttentionArgs(C.Structure):
    _fields_ = [("struct_size", _u32), ("device", _i32), ("stream", _vp), ("dtype", _u32), ("causal", _u32), ("batch", _i64),
                ("sq", _i64), ("sk", _i64), ("n_q", _u32), ("n_kv", _u32), ("head_dim", _u32), ("scale", _f32),
                ("doc_start", _vp), ("lens", _vp), ("q", _vp), ("k", _vp), ("v", _vp), ("o", _vp), ("lse", _vp), ("dout", _vp),
                ("dq", _vp), ("dk", _vp), ("dv", _vp), ("workspace", _vp), ("workspace_bytes", _u64)] + \
               [(n + "_stride", _stride3) for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")]


class DistillArgs(C.Structure):
    _fields_ = [("struct_size", _u32), ("device", _i32), ("stream", _vp), ("dtype", _u32), ("teacher_dtype", _u32), ("labels_64", _u32),
                ("index_64", _u32), ("rows", _i64), ("vocab", _i64), ("k", _u32), ("temperature", _f32), ("mix", _f32), ("reserved", _u32),
                ("ignore_index", _i64), ("logits", _vp), ("logits_stride", _i64), ("labels", _vp), ("teacher_index", _vp),
                ("teacher_logits", _vp), ("teacher_index_stride", _i64), ("teacher_logits_stride", _i64), ("loss", _vp), ("stats", _vp),
                ("dloss", _vp), ("dlogits", _vp), ("dlogits_stride", _i64)]


class EmbeddingArgs(C.Structure):
    _fields_ = [("struct_size", _u32), ("device", _i32), ("stream", _vp), ("dtype", _u32), ("weight_dtype", _u32), ("tokens_64", _u32),
                ("accumulate", _u32), ("tokens", _i64), ("vocab", _i64), ("dim", _u32), ("scale", _f32), ("token", _vp), ("weight", _vp),
                ("weight_stride", _i64), ("out", _vp), ("out_stride", _i64), ("dout", _vp), ("dout_stride", _i64), ("dweight", _vp),
                ("dweight_stride", _i64), ("workspace", _vp), ("workspace_bytes", _u64)]


class RmsNormArgs(C.Structure):
    _fields_ = [("struct_size", _u32), ("device", _i32), ("stream", _vp), ("dtype", _u32), ("weight_dtype", _u32), ("quantized", _u32),
                ("group", _u32), ("size", _stride3), ("dim", _u32), ("eps", _f32), ("x", _vp), ("residual", _vp), ("summed", _vp), ("y", _vp),
                ("scales", _vp), ("rstd", _vp), ("weight", _vp), ("dy", _vp), ("dsummed", _vp), ("dx", _vp), ("dweight", _vp),
                ("workspace", _vp), ("workspace_bytes", _u64)] + \
               [(n + "_stride", _stride3) for n in ("x", "residual", "summed", "y", "dy", "dsummed", "dx")]


class GradsArgs(C.Structure):
    _fields_ = [("struct_size", _u32), ("device", _i32), ("stream", _vp), ("count", _u64), ("grads", _vp), ("outs", _vp), ("numel", _vp),
                ("grad_dtypes", _vp), ("out_dtypes", _vp), ("max_norm", _f32), ("rate", _f32), ("norm", _vp), ("workspace", _vp),
                ("workspace_bytes", _u64)]


def _packer(kind):
    """A struct's fields as one ``struct.Struct``: small calls are bound by what happens here, and packing all values at once costs a third of
    setting them one by one.  The kinds have no gaps, so their sizes agree."""
    codes = {_u32: "I", _i32: "i", _i64: "q", _u64: "Q", _vp: "Q", _f32: "f", _stride3: "3q", _i64 * 2: "2q"}
    packed = struct.Struct("=" + "".join(codes[f[1]] for f in kind._fields_))
    assert packed.size == C.sizeof(kind)
    return packed


def _pack(kind, *values) -> bytes:
    try:
        return kind.pack(*values)
    except (struct.error, OverflowError) as e:
        raise HalosError(ERR_INVALID_ARG, f"an argument out of range: {e}") from None


_ROPE, _ATTENTION, _DISTILL = _packer(RopeArgs), _packer(AttentionArgs), _packer(DistillArgs)
_EMBEDDING, _RMS_NORM, _GRADS = _packer(EmbeddingArgs), _packer(RmsNormArgs), _packer(GradsArgs)
# The stream's handle is asked for without building a stream object around it.
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device, _set_device = torch._C._cuda_getDevice, torch._C._cuda_setDevice
_lib = None


class _Once(torch.autograd.Function):
    """Gradients as a function of what they were formed from, for a graph of them (create_graph=True): the kernels have no derivative of
    their own, and autograd, which does not see them, would take it for zero."""
    @staticmethod
    def forward(ctx, form, *inputs):
        return form(*inputs)

    @staticmethod
    def backward(ctx, *grads):
        raise HalosError(ERR_UNSUPPORTED, "attention, the distillation loss and norms have no second derivative")


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        lib.halos_step_error.restype = C.c_char_p
        lib.halos_step_fault.argtypes = [_i32, C.POINTER(_i32)]
        for name in ("rope", "attention_fwd", "attention_bwd", "distill_fwd", "distill_bwd", "distill_fwd_bwd", "embedding_fwd", "embedding_bwd",
                     "rms_norm_fwd", "rms_norm_bwd", "grad_norm", "clip_grads", "sgd_step"):
            getattr(lib, "halos_" + name).argtypes = [_vp]
        for name in ("attention", "embedding", "rms_norm", "grads"):
            getattr(lib, f"halos_{name}_workspace").argtypes = [_vp, C.POINTER(_u64)]
        _lib = lib
    return _lib


def _refuse(text: str):
    raise HalosError(ERR_INVALID_ARG, text)


def _call(name: str, args: bytes, device: int):
    """The C calls leave their device current; here the caller's stays."""
    lib = _lib or _library()
    before = _current_device()
    rc = getattr(lib, name)(args)
    if before != device:
        _set_device(before)
    if rc:
        raise HalosError(rc, lib.halos_step_error().decode())


def _dtype(x, what: str) -> int:
    d = _DTYPES.get(x.dtype)
    if d is None:
        _refuse(f"{what}: {x.dtype} is not float32, bfloat16 or float16")
    return d


def _on(x, device, what: str):
    if not x.is_cuda:
        _refuse(f"{what} is not a CUDA tensor (there is no CPU path)")
    if x.device != device:
        _refuse(f"{what} is on {x.device}, not on {device}")


def _workspace(name: str, args: bytes, device: int) -> int:
    """Bytes of workspace; the C calls leave their device current, here the caller's stays."""
    lib = _lib or _library()
    size, before = _u64(0), _current_device()
    rc = getattr(lib, name)(args, C.byref(size))
    if before != device:
        _set_device(before)
    if rc:
        raise HalosError(rc, lib.halos_step_error().decode())
    return size.value


def _overwritten(x, what: str):
    """For a tensor that a kernel is about to write over: refused inside a graph, whose history it would no longer agree with, and noted,
    so that autograd notices where it had been saved."""
    if x.requires_grad and torch.is_grad_enabled():
        _refuse(f"{what} requires a gradient and cannot be overwritten (pass it detached if its history does not matter)")
    torch.autograd.graph.increment_version(x)


def fault(device: Optional[int] = None) -> bool:
    """Whether a bounded wait of a kernel has run out on this device since this was last asked; waits for the device.  Until it is asked, the
    calls that follow such a wait raise HalosError: what some call before them returned is undefined."""
    out = _i32(0)
    lib = _library()
    before = torch.cuda.current_device()
    device = before if device is None else int(device)
    rc = lib.halos_step_fault(device, C.byref(out))
    if before != device:
        _set_device(before)
    if rc:
        raise HalosError(rc, lib.halos_step_error().decode())
    return bool(out.value)


# ------------------------------------------------------------------------------------------ rotary positions

def rotary_frequencies(rot_dim: int, *, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained_len: int = 2048,
                       slow_turns: float = 1.0, fast_turns: float = 32.0, device="cuda"):
    """(freqs, magnitude) for ``rope``: radians per position of each of rot_dim/2 pairs, w_p = base^(-2p/rot_dim), and
    the factor on the result.  For contexts ``factor`` times longer than the ``trained_len`` a model was trained on, scaling is

    "linear"  every angle divided by factor
    "base"    the base raised to base factor^(r/(r-2)), so that the slowest pair is slowed by factor and the fastest not at all
    "ramp"    pairs that turn more than fast_turns times within trained_len stay, those that turn less than slow_turns times
              are slowed by factor, with a ramp between, and magnitude = 1 + 0.1 ln(factor)
    """
    if rot_dim <= 0 or rot_dim % 2:
        _refuse("rot_dim must be positive and even")
    if not (base > 0 and factor > 0):
        _refuse("base and factor must be positive")
    if scaling not in ("none", "linear", "base", "ramp"):
        _refuse(f"scaling {scaling!r} is not none, linear, base or ramp")
    if scaling == "base" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    out, magnitude = [], 1.0
    for p in range(rot_dim // 2):
        w = base ** (-2.0 * p / rot_dim)
        if scaling == "linear":
            w /= factor
        elif scaling == "ramp":
            keep = min(1.0, max(0.0, (w * trained_len / (2 * math.pi) - slow_turns) / (fast_turns - slow_turns)))
            w = w * keep + w / factor * (1 - keep)
        out.append(w)
    if scaling == "ramp":
        magnitude = 0.1 * math.log(factor) + 1.0
    return torch.tensor(out, dtype=torch.float64, device=device), magnitude


def _heads_last(x, what: str):
    if x.dim() != 4:
        _refuse(f"{what} must be [batch, seq, heads, head_dim]")
    if x.stride(3) != 1 and x.size(3) > 1:
        _refuse(f"{what}: the elements of a head must lie side by side")


def rope(q, k, freqs, *, positions=None, offset: int = 0, layout: str = "half", magnitude: float = 1.0, inverse: bool = False, inplace: bool = False):
    """Rotates the first 2 len(freqs) elements of every head of q and k ([batch, seq, heads, head_dim], any strides that keep a
    head's elements side by side; k may be None) to their positions: int32 or int64 [seq] or [batch, seq], or offset + 0, 1, ...
    inverse: the gradient's way back.  inplace: q and k are overwritten and returned (neither themselves nor one another may they overlap, nor require a gradient)."""
    device, dtype = q.device, q.dtype
    _heads_last(q, "q")
    _on(q, device, "q")
    kind = _dtype(q, "q")
    batch, seq, n_q, head_dim = q.shape
    n_k = 0
    if k is not None:
        _heads_last(k, "k")
        _on(k, device, "k")
        k_batch, k_seq, n_k, k_dim = k.shape
        if k.dtype != dtype or (k_batch, k_seq, k_dim) != (batch, seq, head_dim):
            _refuse("q and k must agree in type, batch, seq and head_dim")
    _on(freqs, device, "freqs")
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
        _refuse("freqs must be a contiguous float64 vector")
    at, wide, st = 0, False, (0, 0)
    if positions is not None:
        _on(positions, device, "positions")
        wide = positions.dtype == torch.int64
        if not wide and positions.dtype != torch.int32:
            _refuse("positions must be int32 or int64")
        st = positions.stride()
        if positions.shape == (batch, seq):
            pass
        elif positions.shape == (seq,):
            st = (0, st[0])
        else:
            _refuse("positions must be [seq] or [batch, seq]")
        at = positions.data_ptr()
    if inplace:
        for x in (q, k):
            if x is not None and any(s == 0 and n > 1 for s, n in zip(x.stride(), x.shape)):
                _refuse("a broadcast tensor cannot be rotated in place")
        for x, what in ((q, "q"), (k, "k")):
            if x is not None:
                _overwritten(x, what)
        q_out, k_out = q, k
    else:
        q_out, k_out = torch.empty_like(q), None if k is None else torch.empty_like(k)
    none = (0, 0, 0)
    _call("halos_rope", _pack(
        _ROPE, _ROPE.size, device.index, _raw_stream(device.index), kind, _LAYOUTS.get(layout, 99), bool(inverse), wide, batch, seq, n_q, n_k, head_dim, 2 * freqs.numel(), magnitude, 0,
        freqs.data_ptr(), at, *st, offset, q.data_ptr(), 0 if k is None else k.data_ptr(), q_out.data_ptr(), 0 if k is None else k_out.data_ptr(),
        *q.stride()[:3], *(none if k is None else k.stride()[:3]), *q_out.stride()[:3], *(none if k is None else k_out.stride()[:3])), device.index)
    return q_out, k_out


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, freqs, positions, offset, layout, magnitude, inverse):
        ctx.save_for_backward(freqs, positions)
        ctx.how = (offset, layout, magnitude, not inverse)
        return rope(q, k, freqs, positions=positions, offset=offset, layout=layout, magnitude=magnitude, inverse=inverse)

    @staticmethod
    def backward(ctx, dq, dk):
        dq, dk = (x if x is None or x.stride(3) == 1 else x.contiguous() for x in (dq, dk))  # dk is None where k is
        return (*_Rotary.apply(dq, dk, *ctx.saved_tensors, *ctx.how), None, None, None, None, None, None)  # linear: differentiable as often as one likes


def rotary(q, k, freqs, *, positions=None, offset: int = 0, layout: str = "half", magnitude: float = 1.0):
    """``rope`` with autograd; k may be None."""
    return _Rotary.apply(q, k, freqs, positions, offset, layout, magnitude, False)


# ------------------------------------------------------------------------------------------ attention

def _aligned(x):
    """x, or a copy of it that bulk copies can address: 16-byte steps, rows apart, elements side by side."""
    b, s, h, d = x.shape
    sb, ss, sh, sd = x.stride()
    if x.data_ptr() % 16 == 0 and (sd == 1 or d == 1) and (b <= 1 or (sb >= d and sb % 8 == 0)) and (s <= 1 or (ss >= d and ss % 8 == 0)) \
            and (h <= 1 or (sh >= d and sh % 8 == 0)):
        return x
    return x.clone(memory_format=torch.contiguous_format)


def _attention_checked(q, k, v, scale, causal, doc_start, lens):
    """The args' values from dtype to lens, after checks."""
    device, dtype = q.device, q.dtype
    for x, what in ((q, "q"), (k, "k"), (v, "v")):
        if x.dim() != 4:
            _refuse(f"{what} must be [batch, seq, heads, head_dim]")
        _on(x, device, what)
        if x.dtype != dtype:
            _refuse("q, k and v must be of one type")
    batch, sq, n_q, head_dim = q.shape
    k_batch, sk, n_kv, k_dim = k.shape
    if v.shape != k.shape or k_batch != batch or k_dim != head_dim:
        _refuse("k and v must have one shape, and q's batch and head_dim")
    if doc_start is not None:
        _on(doc_start, device, "doc_start")
        if doc_start.dtype != torch.int32 or doc_start.shape != (batch, sq) or not doc_start.is_contiguous():
            _refuse("doc_start must be contiguous int32 [batch, seq of q]")
    if lens is not None:
        _on(lens, device, "lens")
        if lens.dtype != torch.int32 or lens.shape != (batch,) or not lens.is_contiguous():
            _refuse("lens must be contiguous int32 [batch]")
    if scale is None:
        scale = head_dim ** -0.5 if head_dim else 0.0
    return (_dtype(q, "q"), bool(causal), batch, sq, sk, n_q, n_kv, head_dim, scale, 0 if doc_start is None else doc_start.data_ptr(), 0 if lens is None else lens.data_ptr())


def attention_forward(q, k, v, *, scale: Optional[float] = None, causal: bool = True, doc_start=None, lens=None):
    """(o, lse) of q [batch, sq, heads, head_dim] against k, v [batch, sk, key heads, head_dim], bfloat16 or float16; o has q's
    shape, lse is float32 [batch, heads, sq].  Query i stands at i + sk - sq; it sees keys from doc_start[b, i] on (int32), before
    lens[b] (int32), and up to its own position if causal.  A query that sees none, or stands at or past lens[b], has o = 0 and
    lse = -infinity.  What lies at or past lens[b] may hold anything; keys and values that
    some query sees have to be finite, and those between them.  scale: head_dim^-1/2 unless given."""
    values = _attention_checked(q, k, v, scale, causal, doc_start, lens)
    q, k, v = _aligned(q), _aligned(k), _aligned(v)
    o = torch.empty_like(q)
    lse = q.new_empty((values[2], values[5], values[3]), dtype=torch.float32)
    device = q.device.index
    _call("halos_attention_fwd", _pack(
        _ATTENTION, _ATTENTION.size, device, _raw_stream(device), *values, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), 0, 0, 0, 0, 0, 0,
        *q.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3], 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), device)
    return o, lse


def attention_backward(dout, q, k, v, o, lse, *, scale: Optional[float] = None, causal: bool = True, doc_start=None, lens=None):
    """(dq, dk, dv) from the gradient of o, the forward pass's inputs and what it returned.  Deterministic."""
    values = _attention_checked(q, k, v, scale, causal, doc_start, lens)
    for x, what in ((dout, "dout"), (o, "o")):
        _on(x, q.device, what)
        if x.shape != q.shape or x.dtype != q.dtype:
            _refuse(f"{what} must be like q")
    _on(lse, q.device, "lse")
    if lse.dtype != torch.float32 or lse.shape != (values[2], values[5], values[3]) or not lse.is_contiguous():
        _refuse("lse must be contiguous float32 [batch, heads, seq]")
    q, k, v, o, dout = (_aligned(x) for x in (q, k, v, o, dout))
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    device, size = q.device.index, _u64(0)
    tensors = (q, k, v, o, dout, dq, dk, dv)
    strides = [s for x in tensors for s in x.stride()[:3]]
    pointers = [x.data_ptr() for x in (q, k, v, o, lse, dout, dq, dk, dv)]
    head = (_ATTENTION.size, device, _raw_stream(device), *values, *pointers)
    (_lib or _library()).halos_attention_workspace(_pack(_ATTENTION, *head, 0, 0, *strides), C.byref(size))
    space = q.new_empty(size.value, dtype=torch.uint8)
    _call("halos_attention_bwd", _pack(_ATTENTION, *head, space.data_ptr(), size.value, *strides), device)
    return dq, dk, dv


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, causal, doc_start, lens):
        ctx.how = dict(scale=scale, causal=causal)
        o, lse = attention_forward(q, k, v, doc_start=doc_start, lens=lens, **ctx.how)
        ctx.save_for_backward(q, k, v, o, lse, doc_start, lens)  # the masks too, so that autograd notices if they are overwritten
        return o

    @staticmethod
    def backward(ctx, dout):
        *inputs, doc_start, lens = (dout, *ctx.saved_tensors)
        form = functools.partial(attention_backward, doc_start=doc_start, lens=lens, **ctx.how)
        return (*(_Once.apply(form, *inputs) if torch.is_grad_enabled() else form(*inputs)), None, None, None, None)


def attention(q, k, v, *, scale: Optional[float] = None, causal: bool = True, doc_start=None, lens=None):
    """``attention_forward``'s o, with autograd (of first order: a derivative of the gradients is refused)."""
    return _Attention.apply(q, k, v, scale, causal, doc_start, lens)


# ------------------------------------------------------------------------------------------ distillation loss

def _distill_checked(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index):
    """The args' values from the size to teacher_logits_stride, after checks."""
    if logits.dim() != 2:
        _refuse("logits must be [rows, vocab]")
    device = logits.device
    _on(logits, device, "logits")
    rows, vocab = logits.shape
    stride, step_ = logits.stride()
    if vocab > 1 and step_ != 1:
        _refuse("logits: a row's elements must lie side by side")
    kind = _dtype(logits, "logits")
    label_at, labels_64 = 0, False
    if labels is not None:
        _on(labels, device, "labels")
        labels_64 = labels.dtype == torch.int64
        if not labels_64 and labels.dtype != torch.int32 or labels.shape != (rows,) or not labels.is_contiguous():
            _refuse("labels must be contiguous int32 or int64 [rows]")
        label_at = labels.data_ptr()
    if (teacher_idx is None) != (teacher_logits is None):
        _refuse("teacher_idx and teacher_logits come together")
    k, teacher_kind, index_64, index_at, t_at, index_stride, t_stride = 0, 0, False, 0, 0, 0, 0
    if teacher_idx is not None:
        for x, what in ((teacher_idx, "teacher_idx"), (teacher_logits, "teacher_logits")):
            _on(x, device, what)
            if x.dim() != 2 or x.shape != teacher_idx.shape or x.size(0) != rows or (x.size(1) > 1 and x.stride(1) != 1):
                _refuse(f"{what} must be [rows, k], a row's elements side by side")
        index_64 = teacher_idx.dtype == torch.int64
        if not index_64 and teacher_idx.dtype != torch.int32:
            _refuse("teacher_idx must be int32 or int64")
        teacher_kind, k = _dtype(teacher_logits, "teacher_logits"), teacher_idx.size(1)
        index_at, index_stride, t_at, t_stride = teacher_idx.data_ptr(), teacher_idx.stride(0), teacher_logits.data_ptr(), teacher_logits.stride(0)
    return (_DISTILL.size, device.index, _raw_stream(device.index), kind, teacher_kind, labels_64, index_64, rows, vocab, k, temperature, mix, 0, ignore_index, logits.data_ptr(), stride,
            label_at, index_at, t_at, index_stride, t_stride)


def _row_weights(dloss, logits):
    _on(dloss, logits.device, "dloss")
    if dloss.dtype != torch.float32 or dloss.shape != logits.shape[:1] or not dloss.is_contiguous():
        _refuse("dloss must be contiguous float32 [rows]")
    return dloss.data_ptr()


def _gradient_like(logits, out):
    """The gradient's tensor: `out`, or one whose rows start at the same offset from a 16-byte boundary as those of the logits
    do, so that both are read and written in whole vectors."""
    if out is None:
        rows, vocab = logits.shape
        per = 16 // logits.element_size()
        first = logits.data_ptr() % 16 // logits.element_size()
        stride = max(vocab, logits.stride(0)) if rows > 1 else vocab
        if stride > vocab + per:  # keep the remainder only
            stride = vocab + (stride - vocab) % per
        out = logits.new_empty(first + rows * stride).as_strided((rows, vocab), (stride, 1), first)
    else:
        _on(out, logits.device, "out")
        if out.shape != logits.shape or out.dtype != logits.dtype or (out.size(1) > 1 and out.stride(1) != 1):
            _refuse("out must be like logits, a row's elements side by side")
        _overwritten(out, "out")
    return out


def distill_forward(logits, labels, teacher_idx, teacher_logits, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100):
    """(loss [rows], stats [rows, 2]) in float32 of logits [rows, vocab] (float32, bfloat16 or float16, rows any distance apart).

    With p = softmax(teacher_logits / T) over the entries with teacher_idx != -1 ([rows, k], both may be None):
    loss = (1 - mix) (-log softmax(z)[label]) + mix T^2 sum p (log p - log softmax(z / T)[idx]); a row whose label is ignore_index
    has loss 0.  labels None: no first term.  stats = log sum exp of z and of z / T, for ``distill_backward``."""
    values = _distill_checked(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)
    loss = logits.new_empty(values[7], dtype=torch.float32)
    stats = logits.new_empty((values[7], 2), dtype=torch.float32)
    _call("halos_distill_fwd", _pack(_DISTILL, *values, loss.data_ptr(), stats.data_ptr(), 0, 0, 0), values[1])
    return loss, stats


def distill_backward(dloss, logits, stats, labels, teacher_idx, teacher_logits, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100, out=None):
    """dlogits from dloss [rows] and the forward pass's statistics; out may be the logits themselves (detached, if they are in a graph)."""
    values = _distill_checked(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)
    weights = _row_weights(dloss, logits)
    _on(stats, logits.device, "stats")
    if stats.dtype != torch.float32 or stats.shape != (values[7], 2) or not stats.is_contiguous():
        _refuse("stats must be contiguous float32 [rows, 2]")
    out = _gradient_like(logits, out)
    _call("halos_distill_bwd", _pack(_DISTILL, *values, 0, stats.data_ptr(), weights, out.data_ptr(), out.stride(0)), values[1])
    return out


def distill_loss_and_grad(logits, labels, teacher_idx, teacher_logits, dloss, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100, out=None):
    """(loss, dlogits) in one pass over the logits, for weights dloss [rows] that are known beforehand; out may be the logits (detached,
    if they are in a graph)."""
    values = _distill_checked(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)
    weights = _row_weights(dloss, logits)
    loss = logits.new_empty(values[7], dtype=torch.float32)
    out = _gradient_like(logits, out)
    _call("halos_distill_fwd_bwd", _pack(_DISTILL, *values, loss.data_ptr(), 0, weights, out.data_ptr(), out.stride(0)), values[1])
    return loss, out


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index):
        ctx.how = dict(temperature=temperature, mix=mix, ignore_index=ignore_index)
        loss, stats = distill_forward(logits, labels, teacher_idx, teacher_logits, **ctx.how)
        ctx.save_for_backward(logits, stats, labels, teacher_idx, teacher_logits)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        form = functools.partial(distill_backward, **ctx.how)
        inputs = (dloss.contiguous(), *ctx.saved_tensors)
        return (_Once.apply(form, *inputs) if torch.is_grad_enabled() else form(*inputs), None, None, None, None, None, None)


def distill_loss(logits, labels, teacher_idx=None, teacher_logits=None, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100):
    """``distill_forward``'s loss, with autograd for the logits (of first order: a derivative of the gradient is refused)."""
    return _Distill.apply(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)


# ------------------------------------------------------------------------------------------ embedding

_STREAM = struct.Struct("=IiQ")              # what every args struct begins with: its size, device and stream


@functools.lru_cache(maxsize=1024)
def _plain_strides(shape):
    strides, step_ = [], 1
    for n in reversed(shape):
        strides.append(step_)
        step_ *= max(n, 1)
    return tuple(reversed(strides))


def _new(shape, dtype, device):
    """A contiguous tensor: with strides given, half of what torch.empty takes."""
    return torch.empty_strided(shape, _plain_strides(shape), dtype=dtype, device=device)


def _as_rows(x, dim: int):
    """x, or a copy of it, as a matrix of rows whose elements lie side by side."""
    if x.dim() != 2:
        x = x.reshape(-1, dim)
    return x if x.stride(1) == 1 or dim == 1 else x.contiguous()


def _share(a, b) -> bool:
    """Whether two matrices, each (address, rows, distance of rows, bytes of a row), have a byte in common.  Rows of one may lie between those of the other."""
    (a_at, a_rows, a_step, a_row), (b_at, b_rows, b_step, b_row) = a, b
    if not (a_rows and b_rows and a_row and b_row) or a_at + (a_rows - 1) * a_step + a_row <= b_at or b_at + (b_rows - 1) * b_step + b_row <= a_at:
        return False
    starts = a_at + torch.arange(a_rows, device="cpu") * a_step
    before = torch.div(starts - b_at, b_step or 1, rounding_mode="floor")         # b's last row that begins there or in front, and the one behind it
    near = [b_at + (before + k).clamp(0, b_rows - 1) * b_step for k in (0, 1)]
    return any(bool(((x < starts + a_row) & (starts < x + b_row)).any()) for x in near)


def _tokens_checked(tokens, device):
    _on(tokens, device, "tokens")
    wide = tokens.dtype == torch.int64
    if not wide and tokens.dtype != torch.int32:
        _refuse("tokens must be int32 or int64")
    return tokens if tokens.is_contiguous() else tokens.contiguous(), wide


@functools.lru_cache(maxsize=256)
def _embedding_workspace(device: int, dtype: int, weight_dtype: int, tokens: int, vocab: int, dim: int) -> int:
    """Goes by sizes alone, so that they are asked for once."""
    return _workspace("halos_embedding_workspace", _pack(_EMBEDDING, _EMBEDDING.size, device, 0, dtype, weight_dtype, 0, 0, tokens, vocab, dim, 1.0, *(0,) * 11), device)


def embedding_forward(weight, tokens, *, scale: float = 1.0, dtype=None):
    """scale times the rows of weight [vocab, dim] (any distance apart) that tokens (int32 or int64, any shape) name, as [*tokens.shape, dim] of
    dtype (float32, bfloat16 or float16; weight's unless given).  A token outside the vocabulary gives a row of NaN."""
    if weight.dim() != 2:
        _refuse("weight must be [vocab, dim]")
    device = weight.device
    _on(weight, device, "weight")
    vocab, dim = weight.shape
    stride, step_ = weight.stride()
    if step_ != 1 and dim > 1:
        _refuse("weight: a row's elements must lie side by side")
    tokens, wide = _tokens_checked(tokens, device)
    kind = _dtype(weight, "weight")
    out_kind = kind if dtype is None else _DTYPES.get(dtype)
    if out_kind is None:
        _refuse(f"dtype: {dtype} is not float32, bfloat16 or float16")
    out = _new((*tokens.shape, dim), dtype or weight.dtype, device)
    index = device.index
    _call("halos_embedding_fwd", _pack(
        _EMBEDDING, _EMBEDDING.size, index, _raw_stream(index), out_kind, kind, wide, 0, tokens.numel(), vocab, dim, scale,
        tokens.data_ptr(), weight.data_ptr(), stride, out.data_ptr(), dim, 0, 0, 0, 0, 0, 0), index)
    return out


def embedding_backward(dout, tokens, vocab: int, *, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False):
    """The gradient [vocab, dim] of the table from that of the rows, dout [*tokens.shape, dim]: for every token scale times the sum of dout where it
    stands, in a fixed order, 0 where it does not.  Of dtype (dout's unless given), or written to out (rows any distance apart, detached if it is in a graph, sharing no memory with dout or tokens);
    accumulate: added to what out holds, whose other rows are not touched.  Tokens outside the vocabulary take no part."""
    device, vocab = dout.device, int(vocab)
    _on(dout, device, "dout")
    shape = dout.shape
    if not shape or shape[:-1] != tokens.shape:
        _refuse("dout must be [*tokens.shape, dim]")
    tokens, wide = _tokens_checked(tokens, device)
    dim = shape[-1]
    rows, stride = dout, dim
    if dim and not dout.is_contiguous():
        rows = _as_rows(dout, dim)
        stride = rows.stride(0)
    given = out is not None
    if not given:
        if accumulate:
            _refuse("accumulate needs out")
        if vocab < 0 or (dtype is not None and dtype not in _DTYPES):
            _refuse("vocab must be positive and dtype float32, bfloat16 or float16")
        out = _new((vocab, dim), dtype or dout.dtype, device)
    else:
        _on(out, device, "out")
        if out.shape != (vocab, dim) or (dtype is not None and out.dtype != dtype) or (out.stride(1) != 1 and dim > 1) or (vocab > 1 and out.stride(0) < dim):
            _refuse("out must be [vocab, dim] of dtype, a row's elements side by side and rows apart")
    index, count, kind, out_kind = device.index, tokens.numel(), _dtype(dout, "dout"), _dtype(out, "out")
    out_at, out_stride, at, token_at = out.data_ptr(), out.stride(0), rows.data_ptr(), tokens.data_ptr()
    if given:
        # whole runs of memory first: what lies apart, as nearly everything does, is seen at once
        out_size, size, token_bytes = 4 if out_kind == F32 else 2, 4 if kind == F32 else 2, count * (8 if wide else 4)
        end = out_at + ((vocab - 1) * out_stride + dim) * out_size
        if (at < end and out_at < at + ((count - 1) * stride + dim) * size) or (token_at < end and out_at < token_at + token_bytes):
            written = (out_at, vocab, out_stride * out_size, dim * out_size)
            if _share(written, (at, count, stride * size, dim * size)) or _share(written, (token_at, 1, 0, token_bytes)):
                _refuse("out shares memory with dout or tokens")
        _overwritten(out, "out")
    space_bytes = _embedding_workspace(index, kind, out_kind, count, vocab, dim)
    space = torch.empty(space_bytes, dtype=torch.uint8, device=device)
    _call("halos_embedding_bwd", _pack(
        _EMBEDDING, _EMBEDDING.size, index, _raw_stream(index), kind, out_kind, wide, bool(accumulate), count, vocab, dim, scale,
        token_at, 0, 0, 0, 0, at, stride, out_at, out_stride, space.data_ptr(), space_bytes), index)
    return out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, weight, tokens, scale, dtype):
        ctx.save_for_backward(tokens)
        ctx.how = (weight.size(0), scale, weight.dtype)
        return embedding_forward(weight, tokens, scale=scale, dtype=dtype)

    @staticmethod
    def backward(ctx, dout):
        return _EmbeddingBack.apply(dout, *ctx.saved_tensors, *ctx.how), None, None, None


class _EmbeddingBack(torch.autograd.Function):
    """Linear, as the embedding is: differentiable as often as one likes."""
    @staticmethod
    def forward(ctx, dout, tokens, vocab, scale, dtype):
        ctx.save_for_backward(tokens)
        ctx.how = (scale, dout.dtype)
        return embedding_backward(dout, tokens, vocab, scale=scale, dtype=dtype)

    @staticmethod
    def backward(ctx, dweight):
        tokens, = ctx.saved_tensors
        rows = _Embedding.apply(dweight if dweight.stride(1) == 1 else dweight.contiguous(), tokens, *ctx.how)
        none = (tokens < 0) | (tokens >= dweight.size(0))     # take no part in the gradient: its derivative there is 0, not the NaN of their rows
        return rows.masked_fill(none.unsqueeze(-1), 0.0), None, None, None, None


def embedding(weight, tokens, *, scale: float = 1.0, dtype=None):
    """``embedding_forward`` with autograd; the gradient is of weight's type."""
    return _Embedding.apply(weight, tokens, scale, dtype)


# ------------------------------------------------------------------------------------------ root-mean-square norm

_NORM_POINTERS, _NORM_STRIDES = struct.Struct("=13Q"), struct.Struct("=21q")
_NORM_LAYOUT = struct.Struct("=IIII3qIf")


def _side_by_side(x):
    """x, or a copy of it whose rows' elements lie side by side (more than three outer sizes as one), and the strides of its outer sizes, True where it is contiguous."""
    if x.is_contiguous():
        return x, True
    if x.stride(-1) != 1 and x.size(-1) > 1:
        return x.contiguous(), True
    if x.dim() > 4:
        x = x.reshape(-1, x.size(-1))
    return x, x.stride()[:-1]


@functools.lru_cache(maxsize=256)
def _norm_layout(shape, strides, kind: int, weight_kind: int, quantized: bool, group: int, eps: float):
    """The args' part that goes by sizes and strides alone (those of x, residual, summed, y, dy, dsummed, dx without the innermost; None: not there, or
    contiguous where True), the bytes before the pointers and those behind them."""
    dim, outer = shape[-1], shape[:-1]
    size = (1,) * (3 - len(outer)) + tuple(outer) if len(outer) <= 3 else (1, 1, math.prod(outer))
    plain = (size[1] * size[2] * dim, size[2] * dim, dim)
    every = []
    for s in strides:
        every += plain if s is True else (0, 0, 0) if s is None else (0,) * (3 - len(s)) + s
    try:
        return _NORM_LAYOUT.pack(kind, weight_kind, quantized, group, *size, dim, eps), _NORM_STRIDES.pack(*every)
    except (struct.error, OverflowError) as e:
        raise HalosError(ERR_INVALID_ARG, f"an argument out of range: {e}") from None


@functools.lru_cache(maxsize=256)
def _norm_workspace(device: int, shape, kind: int, weight_kind: int) -> int:
    """Goes by sizes alone, so that they are asked for once."""
    layout, strides = _norm_layout(shape, (None,) * 7, kind, weight_kind, False, 0, 0.0)
    return _workspace("halos_rms_norm_workspace", _STREAM.pack(_RMS_NORM.size, device, 0) + layout + _NORM_POINTERS.pack(*(0,) * 13) + strides, device)


def _norm_weight(weight, x, device):
    if weight.device != device:
        _on(weight, device, "weight")
    if weight.dim() != 1 or weight.size(0) != x.size(-1) or not weight.is_contiguous():
        _refuse("weight must be a contiguous vector as long as a row")
    return _dtype(weight, "weight")


def _like(a, b, what: str):
    _on(a, b.device, what)
    if a.shape != b.shape or a.dtype != b.dtype:
        _refuse(f"{what} must be of the same shape and type")


def _rms_norm(x, weight, residual, eps, quantized, group):
    device, shape, eps, group = x.device, x.shape, float(eps), int(group)
    _on(x, device, "x")
    if not shape:
        _refuse("rows must have a last dimension")
    kind, weight_kind = _dtype(x, "x"), _norm_weight(weight, x, device)
    (x3, x_stride), summed, at_r, at_s, r_stride, s_stride = _side_by_side(x), x, 0, 0, None, None
    if residual is not None:
        _like(residual, x, "residual")
        r3, r_stride = _side_by_side(residual)
        summed = torch.empty_like(x) if x.is_contiguous() else _new(shape, x.dtype, device)
        at_r, at_s, s_stride = r3.data_ptr(), summed.data_ptr(), True
    layout, strides = _norm_layout(shape, (x_stride, r_stride, s_stride, True, None, None, None), kind, weight_kind, quantized, group, eps)
    y, scales, at_scales = torch.empty_like(x) if x.is_contiguous() and not quantized else _new(shape, torch.float8_e4m3fn if quantized else x.dtype, device), None, 0
    rstd = _new(shape[:-1], torch.float32, device)
    if quantized:
        scales = _new((*shape[:-1], -(-shape[-1] // (group or shape[-1] or 1))), torch.float32, device)
        at_scales = scales.data_ptr()
    index = device.index
    _call("halos_rms_norm_fwd", b"".join((_STREAM.pack(_RMS_NORM.size, index, _raw_stream(index)), layout, _NORM_POINTERS.pack(
        x3.data_ptr(), at_r, at_s, y.data_ptr(), at_scales, rstd.data_ptr(), weight.data_ptr(), 0, 0, 0, 0, 0, 0), strides)), index)
    return y, scales, summed, rstd


def rms_norm_forward(x, weight, *, residual=None, eps: float = 1e-5):
    """(y, summed, rstd) of the rows of x [..., dim] (float32, bfloat16 or float16; any strides that keep a row's elements side by side): with s = x +
    residual in 32 bits, rstd = 1 / sqrt(mean of s^2 + eps) in float32 [...], y = s rstd weight, and summed = s rounded to x's type (x itself without
    a residual), which the next residual is.  weight [dim] may be of another type."""
    y, _, summed, rstd = _rms_norm(x, weight, residual, eps, False, 0)
    return y, summed, rstd


def rms_norm_quantized(x, weight, *, residual=None, eps: float = 1e-5, group: int = 0):
    """(q, scales, summed, rstd): ``rms_norm_forward`` with y in 8 bits (float8_e4m3fn), q scales being nearest to y.  scales [..., n] in float32 has one value for
    every group (32, 64 or 128) of a row's elements, or one for the row (0): the largest of them over 448.  Without autograd: all four, summed among
    them, are cut from the graph that x, the residual and weight may be in."""
    return _rms_norm(x, weight, residual, eps, True, group)


def rms_norm_backward(dy, summed, weight, rstd, *, dsummed=None):
    """(dx, dweight) from the gradient of y, what the forward pass returned, and the gradient of summed.  dx is the gradient of x and of the
    residual; dweight is of weight's type.  Deterministic."""
    device, shape = dy.device, dy.shape
    _on(dy, device, "dy")
    if not shape:
        _refuse("rows must have a last dimension")
    kind, weight_kind = _dtype(dy, "dy"), _norm_weight(weight, dy, device)
    _like(summed, dy, "summed")
    _on(rstd, device, "rstd")
    if rstd.dtype != torch.float32 or rstd.shape != shape[:-1] or not rstd.is_contiguous():
        _refuse("rstd must be contiguous float32 [...]")
    (dy3, dy_stride), (s3, s_stride), at_d, d_stride = _side_by_side(dy), _side_by_side(summed), 0, None
    if dsummed is not None:
        _like(dsummed, dy, "dsummed")
        d3, d_stride = _side_by_side(dsummed)
        at_d = d3.data_ptr()
    index = device.index
    layout, strides = _norm_layout(shape, (None, None, s_stride, None, dy_stride, d_stride, True), kind, weight_kind, False, 0, 0.0)
    size = _norm_workspace(index, shape, kind, weight_kind)
    dx, dweight, space = torch.empty_like(dy) if dy.is_contiguous() else _new(shape, dy.dtype, device), torch.empty_like(weight), torch.empty(size, dtype=torch.uint8, device=device)
    _call("halos_rms_norm_bwd", b"".join((_STREAM.pack(_RMS_NORM.size, index, _raw_stream(index)), layout, _NORM_POINTERS.pack(
        0, 0, s3.data_ptr(), 0, 0, rstd.data_ptr(), weight.data_ptr(), dy3.data_ptr(), at_d, dx.data_ptr(), dweight.data_ptr(), space.data_ptr(), size), strides)), index)
    return dx, dweight


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, summed, rstd = rms_norm_forward(x, weight, residual=residual, eps=eps)
        ctx.save_for_backward(summed, weight, rstd)
        ctx.added = residual is not None
        ctx.set_materialize_grads(False)
        return (y, summed) if ctx.added else y

    @staticmethod
    def backward(ctx, dy, dsummed=None):
        if dy is None:                   # nobody used the norm: the sum's gradient goes through
            return dsummed, None, dsummed if ctx.added else None, None
        form = lambda dy, summed, weight, rstd, dsummed: rms_norm_backward(dy, summed, weight, rstd, dsummed=dsummed)  # noqa: E731
        inputs = (dy, *ctx.saved_tensors, dsummed)
        dx, dweight = _Once.apply(form, *inputs) if torch.is_grad_enabled() else form(*inputs)
        return dx, dweight, dx if ctx.added else None, None


def rms_norm(x, weight, *, residual=None, eps: float = 1e-5):
    """``rms_norm_forward``'s y, or (y, summed) with a residual, with autograd (of first order: a derivative of the gradients is refused)."""
    return _RmsNorm.apply(x, weight, residual, eps)


# ------------------------------------------------------------------------------------------ gradients

# Many small tensors are bound by what is asked of each: attributes by map, whose loop is not Python's.
_DTYPE_OF, _SHAPE_OF, _REQUIRES = operator.attrgetter("dtype"), operator.attrgetter("shape"), operator.attrgetter("requires_grad")


def _dense(x) -> bool:
    """Whether x's elements fill a run of memory, in whatever order."""
    return x.is_contiguous() or x.permute(sorted(range(x.dim()), key=lambda i: (x.stride(i), x.size(i)), reverse=True)).is_contiguous()


def _listed(tensors, what: str):
    tensors = list(tensors)
    if not tensors or not all([issubclass(kind, torch.Tensor) for kind in set(map(type, tensors))]):
        _refuse(f"{what} must be one tensor or more")
    return tensors


@functools.lru_cache(maxsize=256)
def _grads_workspace(device: int, count: int) -> int:
    """Goes by the number of tensors alone, so that it is asked for once."""
    return _workspace("halos_grads_workspace", _pack(_GRADS, _GRADS.size, device, 0, count, *(0,) * 5, 0.0, 0.0, 0, 0, 0), device)


def _words(values):
    """An array of 64-bit values, and where it lies."""
    words = array.array("Q", values)
    return words, words.buffer_info()[0]


def _grads_call(name: str, grads, outs, max_norm: float, rate: float, with_norm: bool):
    device = grads[0].device
    index = device.index if grads[0].is_cuda else -1
    both = grads if outs is None or outs is grads else grads + outs
    if index < 0 or set(map(torch.Tensor.get_device, both)) != {index}:
        for x in both:
            _on(x, device, "a tensor")
    kinds = [_DTYPES.get(kind, 255) for kind in map(_DTYPE_OF, both)]
    if 255 in kinds:
        _dtype(both[kinds.index(255)], "a tensor")
    in_place = outs is grads
    if not all(map(torch.Tensor.is_contiguous, both)):
        if outs is None:
            grads = [x if _dense(x) else x.contiguous() for x in grads]
        else:
            if not all([_dense(x) for x in outs]):
                _refuse("a tensor that is written must fill a run of memory")
            if not in_place:  # elements side by side in the one are to be so in the other
                grads = [g if (g.is_contiguous() and o.is_contiguous()) or (g.stride() == o.stride()) else torch.empty_like(o, dtype=g.dtype).copy_(g) for g, o in zip(grads, outs)]
    if outs is not None:
        if torch.is_grad_enabled() and any(map(_REQUIRES, outs)):
            _overwritten(next(x for x in outs if x.requires_grad), "a tensor that is written")
        torch.autograd.graph.increment_version(outs)
    n = len(grads)
    g_words, g_at = _words(map(torch.Tensor.data_ptr, grads))
    sizes, sizes_at = _words(map(torch.Tensor.numel, grads))
    g_kinds = bytes(kinds[:n])
    kinds_at = o_kinds_at = C.cast(C.c_char_p(g_kinds), _vp).value
    o_at, norm, space, size = 0, None, 0, 0
    if in_place:
        o_at = g_at
    elif outs is not None:
        o_kinds = bytes(kinds[n:])
        (o_words, o_at), o_kinds_at = _words(map(torch.Tensor.data_ptr, outs)), C.cast(C.c_char_p(o_kinds), _vp).value
    if with_norm:
        norm, size = torch.empty_strided((), (), dtype=torch.float32, device=device), _grads_workspace(index, n)
        space = torch.empty(size, dtype=torch.uint8, device=device)
    _call(name, _pack(_GRADS, _GRADS.size, index, _raw_stream(index), n, g_at, o_at, sizes_at, kinds_at, o_kinds_at, max_norm, rate,
                      norm.data_ptr() if with_norm else 0, space.data_ptr() if with_norm else 0, size), index)
    return norm


def grad_norm(grads):
    """The root of the sum of the squares of every element of `grads` (tensors of float32, bfloat16 and float16, any strides), a float32 scalar on their
    device.  Formed so that neither large nor small gradients leave what 32 bits hold on the way, in a fixed order."""
    grads = _listed(grads, "grads")
    return _grads_call("halos_grad_norm", grads, None, 0.0, 0.0, True)


def clip_grads(grads, max_norm: float, *, out=None):
    """``grad_norm``, and where it is above max_norm the gradients times max_norm / norm: in place, or to the tensors of out (one for each, of the same
    sizes and any of the types).  A norm that is NaN leaves them as they are."""
    grads = _listed(grads, "grads")
    outs = grads if out is None else _paired(_listed(out, "out"), grads)
    return _grads_call("halos_clip_grads", grads, outs, max_norm, 0.0, True)


def sgd_step(params, grads, rate: float, *, max_norm: Optional[float] = None):
    """params -= rate grads, the gradients clipped to max_norm as by ``clip_grads`` if it is given (they themselves stay as they are).  Returns their norm, or
    None without max_norm.  The parameters may be of other types than the gradients, and detached if they are in a graph."""
    grads = _listed(grads, "grads")
    params = _paired(_listed(params, "params"), grads)
    return _grads_call("halos_sgd_step", grads, params, 0.0 if max_norm is None else max_norm, rate, max_norm is not None)


def _paired(tensors, grads):
    if len(tensors) != len(grads) or list(map(_SHAPE_OF, tensors)) != list(map(_SHAPE_OF, grads)):
        _refuse("there must be one tensor for each gradient, of its shape")
    return tensors
