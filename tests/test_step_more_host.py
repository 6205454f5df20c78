"""CPU-side checks of the embedding, the norms and the gradients' calls: struct layouts, refusals that are decided on the host, and what autograd sees of
them, with stand-ins for the kernels."""
from __future__ import annotations

import ctypes as C
import subprocess
from pathlib import Path

import pytest
import torch
import torch.nn.functional as F

from paper_2506_04531_b200 import binding, step

ROOT = Path(__file__).resolve().parent.parent
KINDS = {"halos_embedding_args": step.EmbeddingArgs, "halos_rms_norm_args": step.RmsNormArgs, "halos_grads_args": step.GradsArgs}
CALLS = {"halos_embedding_fwd": step.EmbeddingArgs, "halos_embedding_bwd": step.EmbeddingArgs, "halos_rms_norm_fwd": step.RmsNormArgs, "halos_rms_norm_bwd": step.RmsNormArgs,
         "halos_grad_norm": step.GradsArgs, "halos_clip_grads": step.GradsArgs, "halos_sgd_step": step.GradsArgs}


@pytest.fixture(scope="module")
def lib():
    from paper_2506_04531_b200 import build
    build.build()
    return step._library()


def test_struct_layouts_match_c(tmp_path):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "halos_step.h"', "int main(void){"]
    for name, kind in KINDS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in kind._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-I", str(ROOT / "include"), "-o", str(tmp_path / "layout"), str(src)], check=True)
    out = iter(int(x) for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split())
    for name, kind in KINDS.items():
        assert next(out) == C.sizeof(kind), name
        for f in kind._fields_:
            assert next(out) == getattr(kind, f[0]).offset, (name, f[0])


def test_struct_size_is_checked(lib):
    for call, kind in CALLS.items():
        args = kind()
        args.struct_size = C.sizeof(kind) - 8
        assert getattr(lib, call)(C.byref(args)) == binding.ERR_INVALID_ARG
        assert b"size" in lib.halos_step_error()
        assert getattr(lib, call)(None) == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["embedding", "rms_norm", "grads"])
def test_workspaces_ask_for_whole_args(lib, name):
    n, call = C.c_uint64(0), getattr(lib, f"halos_{name}_workspace")
    args = KINDS[f"halos_{name}_args"]()
    assert call(None, C.byref(n)) == call(C.byref(args), C.byref(n)) == binding.ERR_INVALID_ARG


def _embedding(**kw):
    a = step.EmbeddingArgs()
    a.struct_size, a.dtype, a.weight_dtype, a.tokens_64, a.tokens, a.vocab, a.dim, a.scale = C.sizeof(a), 1, 0, 1, 4, 100, 64, 1.0
    a.token = a.weight = a.out = a.dout = a.dweight = a.workspace = 4096
    a.weight_stride = a.out_stride = a.dout_stride = a.dweight_stride = 64
    for n, v in kw.items():
        setattr(a, n, v)
    return a


@pytest.mark.parametrize("kw,unsupported", [(dict(dtype=3), False), (dict(weight_dtype=9), False), (dict(tokens=-1), False), (dict(vocab=0), False), (dict(vocab=-5), False), (dict(dim=0), False),
                                            (dict(tokens=1 << 31), True), (dict(vocab=(1 << 31) - 1), True), (dict(dim=1 << 30), True), (dict(token=None), False), (dict(token=4100), False)])
def test_embedding_refuses_on_the_host(lib, kw, unsupported):
    want = binding.ERR_UNSUPPORTED if unsupported else binding.ERR_INVALID_ARG
    assert lib.halos_embedding_fwd(C.byref(_embedding(**kw))) == want
    assert lib.halos_embedding_bwd(C.byref(_embedding(**kw))) == want


@pytest.mark.parametrize("back,kw", [(False, dict(weight=None)), (False, dict(out=None)), (False, dict(weight=4098)), (False, dict(out=4097)), (True, dict(dout=None)), (True, dict(dweight=None)),
                                     (True, dict(dout=4097)), (True, dict(dweight=4098))])
def test_embedding_refuses_pointers(lib, back, kw):
    assert (lib.halos_embedding_bwd if back else lib.halos_embedding_fwd)(C.byref(_embedding(**kw))) == binding.ERR_INVALID_ARG


def _norm(**kw):
    a = step.RmsNormArgs()
    a.struct_size, a.dtype, a.weight_dtype, a.dim, a.eps = C.sizeof(a), 1, 0, 64, 1e-5
    a.size[:] = (1, 2, 8)
    for n in ("x", "residual", "summed", "y", "scales", "rstd", "weight", "dy", "dsummed", "dx", "dweight", "workspace"):
        setattr(a, n, 4096)
    for n in ("x", "residual", "summed", "y", "dy", "dsummed", "dx"):
        getattr(a, n + "_stride")[:] = (1024, 512, 64)
    for n, v in kw.items():
        if n == "size":
            a.size[:] = v
        else:
            setattr(a, n, v)
    return a


@pytest.mark.parametrize("kw,unsupported", [(dict(dtype=3), False), (dict(weight_dtype=4), False), (dict(size=(1, -1, 8)), False), (dict(size=(1 << 11, 1 << 10, 1 << 10)), True), (dict(size=(1, 1, 1 << 32)), True),
                                            (dict(size=(1 << 30, 1 << 30, 1 << 30)), True), (dict(dim=0), False), (dict(dim=1 << 30), True), (dict(weight=None), False), (dict(weight=4098), False),
                                            (dict(rstd=None), False), (dict(rstd=4098), False), (dict(summed=None), False), (dict(summed=4097), False)])
def test_norm_refuses_on_the_host(lib, kw, unsupported):
    want = binding.ERR_UNSUPPORTED if unsupported else binding.ERR_INVALID_ARG
    assert lib.halos_rms_norm_fwd(C.byref(_norm(**kw))) == want
    assert lib.halos_rms_norm_bwd(C.byref(_norm(**kw))) == want


@pytest.mark.parametrize("back,kw,unsupported", [(False, dict(eps=-1.0), False), (False, dict(eps=float("inf")), False), (False, dict(quantized=1, group=16), True), (False, dict(quantized=1, scales=None), False),
                                                 (False, dict(quantized=1, scales=4098), False), (False, dict(x=None), False), (False, dict(y=4097), False), (False, dict(residual=4097), False),
                                                 (True, dict(dy=None), False), (True, dict(dx=None), False), (True, dict(dweight=None), False), (True, dict(dsummed=4097), False)])
def test_norm_refuses_one_way(lib, back, kw, unsupported):
    assert (lib.halos_rms_norm_bwd if back else lib.halos_rms_norm_fwd)(C.byref(_norm(**kw))) == (binding.ERR_UNSUPPORTED if unsupported else binding.ERR_INVALID_ARG)


def _grads(run=((4096, 10, 0),), to=((8192, 0),), **kw):
    a, n = step.GradsArgs(), len(run)
    keep = [(C.c_uint64 * n)(*[g[0] for g in run]), (C.c_int64 * n)(*[g[1] for g in run]), (C.c_uint8 * n)(*[g[2] for g in run]),
            (C.c_uint64 * n)(*[o[0] for o in to]), (C.c_uint8 * n)(*[o[1] for o in to])]
    a.struct_size, a.count, a.norm, a.workspace, a.max_norm = C.sizeof(a), n, 4096, 4096, 1.0
    a.grads, a.numel, a.grad_dtypes, a.outs, a.out_dtypes = (C.addressof(x) for x in keep)
    for n, v in kw.items():
        setattr(a, n, v)
    a.keep = keep
    return a


@pytest.mark.parametrize("grads,outs,kw,unsupported", [
    (((4096, 10, 3),), ((8192, 0),), {}, False), (((4096, 10, 0),), ((8192, 5),), {}, False), (((4096, -1, 0),), ((8192, 0),), {}, False), (((4096, 1 << 40, 0),), ((8192, 0),), {}, True),
    (((0, 10, 0),), ((8192, 0),), {}, False), (((4096, 10, 0),), ((0, 0),), {}, False), (((4098, 10, 0),), ((8192, 0),), {}, False), (((4096, 10, 0),), ((8193, 1),), {}, False),
    (((4096, 10, 0),), ((8192, 0),), dict(max_norm=-1.0), False), (((4096, 10, 0),), ((8192, 0),), dict(max_norm=float("nan")), False), (((4096, 10, 0),), ((8192, 0),), dict(grads=None), False),
    (((4096, 10, 0),), ((8192, 0),), dict(outs=None), False), (((4096, 10, 0),), ((8192, 0),), dict(count=1 << 24), True),
    # what is written overlaps: another output, another gradient, the gradient itself at another place or in another type
    (((4096, 10, 0), (5000, 10, 0)), ((8192, 0), (8228, 0)), {}, False), (((4096, 10, 0), (8192, 10, 0)), ((8192, 0), (4096, 0)), {}, False), (((4096, 10, 0),), ((4100, 0),), {}, False),
    (((4096, 10, 0),), ((4096, 1),), {}, False), (((4096, 100, 0), (4096, 100, 0)), ((4096, 0), (8192, 0)), {}, False), (((4096, 100, 0), (9000, 10, 0)), ((9000, 1), (4096 + 396, 0)), {}, False)])
def test_gradients_refuse_on_the_host(lib, grads, outs, kw, unsupported):
    want = binding.ERR_UNSUPPORTED if unsupported else binding.ERR_INVALID_ARG
    for call in (lib.halos_clip_grads, lib.halos_sgd_step):
        assert call(C.byref(_grads(grads, outs, **kw))) == want, lib.halos_step_error()


def test_gradients_refuse_one_way(lib):
    assert lib.halos_sgd_step(C.byref(_grads(rate=float("nan")))) == binding.ERR_INVALID_ARG
    assert lib.halos_clip_grads(C.byref(_grads(norm=None))) == binding.ERR_INVALID_ARG
    assert lib.halos_grad_norm(C.byref(_grads(norm=None))) == binding.ERR_INVALID_ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a host without a device")
def test_without_a_device_valid_calls_fail_with_a_cuda_error(lib):
    a = _norm()
    a.quantized, a.group = 1, 32
    # neighbours that touch, gradients that are their own outputs, and ranges of no elements are no overlap
    fine = _grads(((4096, 10, 0), (4136, 10, 0), (4096, 0, 0)), ((4096, 0), (4136, 0), (4100, 0)))
    for call, args in ((lib.halos_embedding_fwd, _embedding()), (lib.halos_embedding_bwd, _embedding()), (lib.halos_rms_norm_fwd, a), (lib.halos_rms_norm_bwd, _norm()), (lib.halos_clip_grads, fine),
                       (lib.halos_sgd_step, _grads()), (lib.halos_grad_norm, _grads())):
        assert call(C.byref(args)) == binding.ERR_CUDA, lib.halos_step_error()
        assert b"no CPU path" in lib.halos_step_error()


def test_cpu_tensors_are_refused(lib):
    x, t, w = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64), torch.ones(8)
    for call in (lambda: step.embedding_forward(x, t), lambda: step.embedding_backward(x, t, 4), lambda: step.rms_norm_forward(x, w), lambda: step.rms_norm_quantized(x, w),
                 lambda: step.rms_norm_backward(x, x, w, torch.ones(3)), lambda: step.grad_norm([x]), lambda: step.clip_grads([x], 1.0), lambda: step.sgd_step([x], [x.clone()], 1.0)):
        with pytest.raises(binding.HalosError) as e:
            call()
        assert e.value.status == binding.ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------ autograd

@pytest.fixture
def plain(monkeypatch):
    def embedding_forward(weight, tokens, *, scale=1.0, dtype=None):
        return (weight.detach()[tokens] * scale).to(dtype or weight.dtype)

    def embedding_backward(dout, tokens, vocab, *, scale=1.0, dtype=None, **kw):
        return (dout.new_zeros(vocab, dout.size(-1)).index_add(0, tokens.reshape(-1), dout.detach().reshape(-1, dout.size(-1))) * scale).to(dtype or dout.dtype)

    def rms_norm_forward(x, weight, *, residual=None, eps=1e-5):
        s = x.detach() if residual is None else x.detach() + residual.detach()
        rstd = (s.pow(2).mean(-1) + eps).rsqrt()
        return s * rstd[..., None] * weight.detach(), (x if residual is None else s), rstd

    def rms_norm_backward(dy, summed, weight, rstd, *, dsummed=None):
        g, u = dy * weight, summed * rstd[..., None]
        dx = rstd[..., None] * (g - u * (g * u).mean(-1, keepdim=True))
        return dx if dsummed is None else dx + dsummed, (dy * u).flatten(0, -2).sum(0)

    for f in (embedding_forward, embedding_backward, rms_norm_forward, rms_norm_backward):
        monkeypatch.setattr(step, f.__name__, f)


def test_embedding_differentiated_twice(plain):
    w, t, c = torch.randn(6, 4, dtype=torch.float64, requires_grad=True), torch.tensor([[1, 5], [1, 0]]), torch.randn(2, 2, 4, dtype=torch.float64)
    got = [(step.embedding(w, t, scale=2.0), w), (F.embedding(t, w) * 2.0, w)]
    firsts = [torch.autograd.grad((y.pow(3) * c).sum(), x, create_graph=True)[0] for y, x in got]
    seconds = [torch.autograd.grad(g.pow(2).sum(), w)[0] for g in firsts]
    assert torch.allclose(*firsts) and torch.allclose(*seconds)
    assert torch.autograd.gradcheck(lambda w: step.embedding(w, t, scale=2.0), (w,))


def test_embedding_tokens_that_are_overwritten_are_noticed(plain):
    w, t = torch.randn(6, 4, requires_grad=True), torch.tensor([1, 5])
    y = step.embedding(w, t)
    t += 0
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("residual", [True, False])
def test_norm_gradients(plain, residual):
    x, w = torch.randn(3, 5, 4, dtype=torch.float64, requires_grad=True), torch.randn(4, dtype=torch.float64, requires_grad=True)
    if residual:
        r = torch.randn(3, 5, 4, dtype=torch.float64, requires_grad=True)
        for which in (slice(0, 2), slice(0, 1), slice(1, 2)):       # both results, either one
            assert torch.autograd.gradcheck(lambda x, w, r: step.rms_norm(x, w, residual=r)[which], (x, w, r))
    else:
        assert torch.autograd.gradcheck(lambda x, w: step.rms_norm(x, w), (x, w))


def test_a_second_derivative_of_the_norm_is_refused_and_not_left_out(plain):
    x, w, r = (torch.randn(s, requires_grad=True) for s in ((3, 4), (4,), (3, 4)))
    y, s = step.rms_norm(x, w, residual=r)
    g, = torch.autograd.grad(y.sum() + s.pow(2).sum(), x, create_graph=True)
    with pytest.raises(step.HalosError, match="second derivative"):
        (g.pow(2).sum() + x.sum()).backward()


def test_what_the_norm_saved_is_noticed_when_overwritten(plain):
    x, w = torch.randn(3, 4), torch.randn(4, requires_grad=True)
    y = step.rms_norm(x, w)
    x += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("status", [0, 4])
def test_the_callers_device_stays_current(monkeypatch, status):
    """Asking for a workspace makes its device current, as every C call does."""
    class Library:
        current = 0

        def halos_embedding_workspace(self, args, out):
            self.current = 1
            return status

        def halos_step_error(self):
            return b"as asked"

    lib = Library()
    monkeypatch.setattr(step, "_lib", lib)
    monkeypatch.setattr(step, "_current_device", lambda: lib.current)
    monkeypatch.setattr(step, "_set_device", lambda d: setattr(lib, "current", d))
    if status:
        with pytest.raises(step.HalosError):
            step._workspace("halos_embedding_workspace", b"", 1)
    else:
        step._workspace("halos_embedding_workspace", b"", 1)
    assert lib.current == 0
