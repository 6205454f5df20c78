"""Operators of a worker's local step on CUDA tensors: the calls of include/halos_step.h.

    rope, rotary                      rotary positions (rotary: with autograd)
    attention_forward, _backward      masked attention and its gradients; attention: with autograd
    distill_forward, _backward, distill_loss_and_grad      the loss against labels and a teacher's top logits; distill_loss: with autograd

As in ``binding``, the arithmetic is the CUDA library's; what happens here is checking, marshalling and output
allocation, on the current stream of the tensors' device.  The caller's current device stays what it was.  There is no CPU path.
Errors are ``HalosError``.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import struct
from typing import Optional

import torch

from .binding import BF16, ERR_INVALID_ARG, ERR_UNSUPPORTED, F32, HalosError, load_library

F16 = 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
_LAYOUTS = {"half": ROPE_HALF, "interleaved": ROPE_INTERLEAVED}
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

EXPORTED = ("halos_step_error", "halos_step_fault", "halos_rope", "halos_attention_fwd", "halos_attention_bwd",
            "halos_attention_workspace", "halos_distill_fwd", "halos_distill_bwd", "halos_distill_fwd_bwd")

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
        raise HalosError(ERR_UNSUPPORTED, "attention and the distillation loss have no second derivative")


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        lib.halos_step_error.restype = C.c_char_p
        lib.halos_step_fault.argtypes = [_i32, C.POINTER(_i32)]
        for name in ("rope", "attention_fwd", "attention_bwd", "distill_fwd", "distill_bwd", "distill_fwd_bwd"):
            getattr(lib, "halos_" + name).argtypes = [_vp]
        lib.halos_attention_workspace.argtypes = [_vp, C.POINTER(_u64)]
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
