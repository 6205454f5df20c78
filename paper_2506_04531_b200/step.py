"""Operators of a worker's local step on CUDA tensors: the calls of include/halos_step.h.

    rope, rotary                      rotary positions (rotary: with autograd)
    attention_forward, _backward      masked attention and its gradients; attention: with autograd
    distill_forward, _backward, distill_loss_and_grad      the loss against labels and a teacher's top logits; distill_loss: with autograd

As in ``binding``, the arithmetic is the CUDA library's; what happens here is checking, marshalling and output
allocation, on the current stream of the tensors' device.  There is no CPU path.  Errors are ``HalosError``.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from .binding import BF16, ERR_INVALID_ARG, F32, HalosError, load_library

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


_ROPE_SIZE, _ATTENTION_SIZE, _DISTILL_SIZE = C.sizeof(RopeArgs), C.sizeof(AttentionArgs), C.sizeof(DistillArgs)
# Small calls are bound by what happens here, so the stream's handle is asked for without building a stream object around it.
_byref, _raw_stream = C.byref, torch._C._cuda_getCurrentRawStream
_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        lib.halos_step_error.restype = C.c_char_p
        lib.halos_step_fault.argtypes = [_i32, C.POINTER(_i32)]
        for name, args in (("rope", RopeArgs), ("attention_fwd", AttentionArgs), ("attention_bwd", AttentionArgs), ("distill_fwd", DistillArgs),
                           ("distill_bwd", DistillArgs), ("distill_fwd_bwd", DistillArgs)):
            getattr(lib, "halos_" + name).argtypes = [C.POINTER(args)]
        lib.halos_attention_workspace.argtypes = [C.POINTER(AttentionArgs), C.POINTER(_u64)]
        _lib = lib
    return _lib


def _refuse(text: str):
    raise HalosError(ERR_INVALID_ARG, text)


def _call(name: str, args):
    lib = _lib or _library()
    rc = getattr(lib, name)(_byref(args))
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


def _begin(args, size: int, device):
    args.struct_size = size
    args.device = device.index
    args.stream = _raw_stream(device.index)


def fault(device: Optional[int] = None) -> bool:
    """Whether a bounded wait of an attention kernel has run out on this device; waits for the device."""
    out = _i32(0)
    lib = _library()
    rc = lib.halos_step_fault(torch.cuda.current_device() if device is None else int(device), C.byref(out))
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
    inverse: the gradient's way back.  inplace: q and k are overwritten and returned (a view must not overlap itself)."""
    device, dtype = q.device, q.dtype
    _heads_last(q, "q")
    _on(q, device, "q")
    a = RopeArgs()
    a.dtype = _dtype(q, "q")
    a.layout = _LAYOUTS.get(layout, 99)
    a.batch, a.seq, a.n_q, a.head_dim = shape = q.shape
    if k is not None:
        _heads_last(k, "k")
        _on(k, device, "k")
        k_shape = k.shape
        if k.dtype != dtype or k_shape[:2] != shape[:2] or k_shape[3] != shape[3]:
            _refuse("q and k must agree in type, batch, seq and head_dim")
        a.n_k = k_shape[2]
    _on(freqs, device, "freqs")
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
        _refuse("freqs must be a contiguous float64 vector")
    a.rot_dim, a.freqs = 2 * freqs.numel(), freqs.data_ptr()
    if positions is not None:
        _on(positions, device, "positions")
        wide = positions.dtype == torch.int64
        if not wide and positions.dtype != torch.int32:
            _refuse("positions must be int32 or int64")
        if positions.shape != shape[:2] and positions.shape != shape[1:2]:
            _refuse("positions must be [seq] or [batch, seq]")
        a.positions, a.positions_64 = positions.data_ptr(), wide
        st = positions.stride()
        a.position_stride[:] = st if len(st) == 2 else (0, st[0])
    a.position_offset, a.magnitude, a.inverse = offset, magnitude, bool(inverse)
    if inplace:
        for x in (q, k):
            if x is not None and any(s == 0 and n > 1 for s, n in zip(x.stride(), x.shape)):
                _refuse("a broadcast tensor cannot be rotated in place")
        q_out, k_out = q, k
    else:
        q_out, k_out = torch.empty_like(q), None if k is None else torch.empty_like(k)
    a.q_in, a.q_out = q.data_ptr(), q_out.data_ptr()
    a.q_in_stride[:], a.q_out_stride[:] = q.stride()[:3], q_out.stride()[:3]
    if k is not None:
        a.k_in, a.k_out = k.data_ptr(), k_out.data_ptr()
        a.k_in_stride[:], a.k_out_stride[:] = k.stride()[:3], k_out.stride()[:3]
    _begin(a, _ROPE_SIZE, device)
    _call("halos_rope", a)
    return q_out, k_out


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, freqs, positions, offset, layout, magnitude):
        ctx.save_for_backward(freqs, positions)
        ctx.how = dict(offset=offset, layout=layout, magnitude=magnitude)
        return rope(q, k, freqs, positions=positions, **ctx.how)

    @staticmethod
    def backward(ctx, dq, dk):
        freqs, positions = ctx.saved_tensors
        dq, dk = (x if x.stride(3) == 1 else x.contiguous() for x in (dq, dk))
        dq, dk = rope(dq, dk, freqs, positions=positions, inverse=True, **ctx.how)
        return dq, dk, None, None, None, None, None


def rotary(q, k, freqs, *, positions=None, offset: int = 0, layout: str = "half", magnitude: float = 1.0):
    """``rope`` with autograd."""
    return _Rotary.apply(q, k, freqs, positions, offset, layout, magnitude)


# ------------------------------------------------------------------------------------------ attention

def _aligned(x):
    """x, or a copy of it that bulk copies can address: 16-byte steps, rows apart, elements side by side."""
    b, s, h, d = x.shape
    sb, ss, sh, sd = x.stride()
    if x.data_ptr() % 16 == 0 and (sd == 1 or d == 1) and (b <= 1 or (sb >= d and sb % 8 == 0)) and (s <= 1 or (ss >= d and ss % 8 == 0)) \
            and (h <= 1 or (sh >= d and sh % 8 == 0)):
        return x
    return x.clone(memory_format=torch.contiguous_format)


def _attention_args(q, k, v, scale, causal, doc_start, lens):
    device, dtype = q.device, q.dtype
    for x, what in ((q, "q"), (k, "k"), (v, "v")):
        if x.dim() != 4:
            _refuse(f"{what} must be [batch, seq, heads, head_dim]")
        _on(x, device, what)
        if x.dtype != dtype:
            _refuse("q, k and v must be of one type")
    q_shape, k_shape = q.shape, k.shape
    if k_shape != v.shape or k_shape[0] != q_shape[0] or k_shape[3] != q_shape[3]:
        _refuse("k and v must have one shape, and q's batch and head_dim")
    a = AttentionArgs()
    a.dtype, a.causal = _dtype(q, "q"), bool(causal)
    a.batch, a.sq, a.n_q, a.head_dim = q_shape
    a.sk, a.n_kv = k_shape[1:3]
    a.scale = q_shape[3] ** -0.5 if scale is None and q_shape[3] else scale or 0.0
    if doc_start is not None:
        _on(doc_start, q.device, "doc_start")
        if doc_start.dtype != torch.int32 or doc_start.shape != q.shape[:2] or not doc_start.is_contiguous():
            _refuse("doc_start must be contiguous int32 [batch, seq of q]")
        a.doc_start = doc_start.data_ptr()
    if lens is not None:
        _on(lens, q.device, "lens")
        if lens.dtype != torch.int32 or lens.shape != q.shape[:1] or not lens.is_contiguous():
            _refuse("lens must be contiguous int32 [batch]")
        a.lens = lens.data_ptr()
    return a


def _set(a, name: str, x):
    setattr(a, name, x.data_ptr())
    getattr(a, name + "_stride")[:] = x.stride()[:3]


def attention_forward(q, k, v, *, scale: Optional[float] = None, causal: bool = True, doc_start=None, lens=None):
    """(o, lse) of q [batch, sq, heads, head_dim] against k, v [batch, sk, key heads, head_dim], bfloat16 or float16; o has q's
    shape, lse is float32 [batch, heads, sq].  Query i stands at i + sk - sq; it sees keys from doc_start[b, i] on (int32), before
    lens[b] (int32), and up to its own position if causal.  A query that sees none, or stands at or past lens[b], has o = 0 and
    lse = -infinity.  What lies at or past lens[b] may hold anything.  scale: head_dim^-1/2 unless given."""
    a = _attention_args(q, k, v, scale, causal, doc_start, lens)
    q, k, v = _aligned(q), _aligned(k), _aligned(v)
    o = torch.empty_like(q)
    lse = q.new_empty((a.batch, a.n_q, a.sq), dtype=torch.float32)
    for n, x in (("q", q), ("k", k), ("v", v), ("o", o)):
        _set(a, n, x)
    a.lse = lse.data_ptr()
    _begin(a, _ATTENTION_SIZE, q.device)
    _call("halos_attention_fwd", a)
    return o, lse


def attention_backward(dout, q, k, v, o, lse, *, scale: Optional[float] = None, causal: bool = True, doc_start=None, lens=None):
    """(dq, dk, dv) from the gradient of o, the forward pass's inputs and what it returned.  Deterministic."""
    a = _attention_args(q, k, v, scale, causal, doc_start, lens)
    for x, what in ((dout, "dout"), (o, "o")):
        _on(x, q.device, what)
        if x.shape != q.shape or x.dtype != q.dtype:
            _refuse(f"{what} must be like q")
    _on(lse, q.device, "lse")
    if lse.dtype != torch.float32 or lse.shape != (q.shape[0], q.shape[2], q.shape[1]) or not lse.is_contiguous():
        _refuse("lse must be contiguous float32 [batch, heads, seq]")
    q, k, v, o, dout = (_aligned(x) for x in (q, k, v, o, dout))
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for n, x in (("q", q), ("k", k), ("v", v), ("o", o), ("dout", dout), ("dq", dq), ("dk", dk), ("dv", dv)):
        _set(a, n, x)
    a.lse = lse.data_ptr()
    size = _u64(0)
    a.struct_size = _ATTENTION_SIZE
    _library().halos_attention_workspace(C.byref(a), C.byref(size))
    space = q.new_empty(size.value, dtype=torch.uint8)
    a.workspace, a.workspace_bytes = space.data_ptr(), size.value
    _begin(a, _ATTENTION_SIZE, q.device)
    _call("halos_attention_bwd", a)
    return dq, dk, dv


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, causal, doc_start, lens):
        ctx.how = dict(scale=scale, causal=causal, doc_start=doc_start, lens=lens)
        o, lse = attention_forward(q, k, v, **ctx.how)
        ctx.save_for_backward(q, k, v, o, lse)
        return o

    @staticmethod
    def backward(ctx, dout):
        return (*attention_backward(dout, *ctx.saved_tensors, **ctx.how), None, None, None, None)


def attention(q, k, v, *, scale: Optional[float] = None, causal: bool = True, doc_start=None, lens=None):
    """``attention_forward``'s o, with autograd."""
    return _Attention.apply(q, k, v, scale, causal, doc_start, lens)


# ------------------------------------------------------------------------------------------ distillation loss

def _distill_args(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index):
    if logits.dim() != 2:
        _refuse("logits must be [rows, vocab]")
    _on(logits, logits.device, "logits")
    if logits.size(1) > 1 and logits.stride(1) != 1:
        _refuse("logits: a row's elements must lie side by side")
    a = DistillArgs()
    a.dtype = _dtype(logits, "logits")
    a.rows, a.vocab = logits.shape
    a.temperature, a.mix, a.ignore_index = temperature, mix, ignore_index
    a.logits, a.logits_stride = logits.data_ptr(), logits.stride(0)
    if labels is not None:
        _on(labels, logits.device, "labels")
        if labels.dtype not in (torch.int32, torch.int64) or labels.shape != logits.shape[:1] or not labels.is_contiguous():
            _refuse("labels must be contiguous int32 or int64 [rows]")
        a.labels, a.labels_64 = labels.data_ptr(), labels.dtype == torch.int64
    if (teacher_idx is None) != (teacher_logits is None):
        _refuse("teacher_idx and teacher_logits come together")
    if teacher_idx is not None:
        for x, what in ((teacher_idx, "teacher_idx"), (teacher_logits, "teacher_logits")):
            _on(x, logits.device, what)
            if x.dim() != 2 or x.shape != teacher_idx.shape or x.shape[0] != logits.shape[0] or (x.size(1) > 1 and x.stride(1) != 1):
                _refuse(f"{what} must be [rows, k], a row's elements side by side")
        if teacher_idx.dtype not in (torch.int32, torch.int64):
            _refuse("teacher_idx must be int32 or int64")
        a.teacher_dtype, a.index_64, a.k = _dtype(teacher_logits, "teacher_logits"), teacher_idx.dtype == torch.int64, teacher_idx.shape[1]
        a.teacher_index, a.teacher_index_stride = teacher_idx.data_ptr(), teacher_idx.stride(0)
        a.teacher_logits, a.teacher_logits_stride = teacher_logits.data_ptr(), teacher_logits.stride(0)
    return a


def _row_weights(dloss, logits):
    _on(dloss, logits.device, "dloss")
    if dloss.dtype != torch.float32 or dloss.shape != logits.shape[:1] or not dloss.is_contiguous():
        _refuse("dloss must be contiguous float32 [rows]")
    return dloss.data_ptr()


def _gradient_like(logits, out, a):
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
    a.dlogits, a.dlogits_stride = out.data_ptr(), out.stride(0)
    return out


def distill_forward(logits, labels, teacher_idx, teacher_logits, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100):
    """(loss [rows], stats [rows, 2]) in float32 of logits [rows, vocab] (float32, bfloat16 or float16, rows any distance apart).

    With p = softmax(teacher_logits / T) over the entries with teacher_idx != -1 ([rows, k], both may be None):
    loss = (1 - mix) (-log softmax(z)[label]) + mix T^2 sum p (log p - log softmax(z / T)[idx]); a row whose label is ignore_index
    has loss 0.  labels None: no first term.  stats = log sum exp of z and of z / T, for ``distill_backward``."""
    a = _distill_args(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)
    loss = logits.new_empty(a.rows, dtype=torch.float32)
    stats = logits.new_empty((a.rows, 2), dtype=torch.float32)
    a.loss, a.stats = loss.data_ptr(), stats.data_ptr()
    _begin(a, _DISTILL_SIZE, logits.device)
    _call("halos_distill_fwd", a)
    return loss, stats


def distill_backward(dloss, logits, stats, labels, teacher_idx, teacher_logits, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100, out=None):
    """dlogits from dloss [rows] and the forward pass's statistics; out may be the logits themselves."""
    a = _distill_args(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)
    a.dloss = _row_weights(dloss, logits)
    _on(stats, logits.device, "stats")
    if stats.dtype != torch.float32 or stats.shape != (logits.shape[0], 2) or not stats.is_contiguous():
        _refuse("stats must be contiguous float32 [rows, 2]")
    a.stats = stats.data_ptr()
    out = _gradient_like(logits, out, a)
    _begin(a, _DISTILL_SIZE, logits.device)
    _call("halos_distill_bwd", a)
    return out


def distill_loss_and_grad(logits, labels, teacher_idx, teacher_logits, dloss, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100, out=None):
    """(loss, dlogits) in one pass over the logits, for weights dloss [rows] that are known beforehand; out may be the logits."""
    a = _distill_args(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)
    a.dloss = _row_weights(dloss, logits)
    loss = logits.new_empty(a.rows, dtype=torch.float32)
    a.loss = loss.data_ptr()
    out = _gradient_like(logits, out, a)
    _begin(a, _DISTILL_SIZE, logits.device)
    _call("halos_distill_fwd_bwd", a)
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
        logits, *rest = ctx.saved_tensors
        return (distill_backward(dloss.contiguous(), logits, *rest, **ctx.how), None, None, None, None, None, None)


def distill_loss(logits, labels, teacher_idx=None, teacher_logits=None, *, temperature: float = 1.0, mix: float = 0.5, ignore_index: int = -100):
    """``distill_forward``'s loss, with autograd for the logits."""
    return _Distill.apply(logits, labels, teacher_idx, teacher_logits, temperature, mix, ignore_index)
