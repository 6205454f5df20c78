"""CPU-side checks of the local step's operators: exported symbols, struct layouts, and refusals that are decided on the host."""
from __future__ import annotations

import ctypes as C
import re
import subprocess
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parent.parent
HEADER = ROOT / "include" / "halos_step.h"


@pytest.fixture(scope="module")
def lib():
    from paper_2506_04531_b200 import build
    build.build()
    from paper_2506_04531_b200 import step
    return step._library()


def test_every_declared_symbol_is_exported(lib):
    from paper_2506_04531_b200 import step
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    declared = set(re.findall(r"\b(halos_[a-z_0-9]+)\s*\(", text))
    assert declared == set(step.EXPORTED)
    for name in declared:
        assert hasattr(lib, name)


def test_struct_layouts_match_c(tmp_path):
    from paper_2506_04531_b200 import step
    kinds = {"halos_rope_args": step.RopeArgs, "halos_attention_args": step.AttentionArgs, "halos_distill_args": step.DistillArgs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "halos_step.h"', "int main(void){"]
    for name, kind in kinds.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in kind._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-I", str(ROOT / "include"), "-o", str(tmp_path / "layout"), str(src)], check=True)
    out = iter(int(x) for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split())
    for name, kind in kinds.items():
        assert next(out) == C.sizeof(kind), name
        for f in kind._fields_:
            assert next(out) == getattr(kind, f[0]).offset, (name, f[0])


def test_struct_size_is_checked(lib):
    from paper_2506_04531_b200 import binding, step
    for call, kind in (("halos_rope", step.RopeArgs), ("halos_attention_fwd", step.AttentionArgs), ("halos_attention_bwd", step.AttentionArgs),
                       ("halos_distill_fwd", step.DistillArgs), ("halos_distill_bwd", step.DistillArgs), ("halos_distill_fwd_bwd", step.DistillArgs)):
        args = kind()
        args.struct_size = C.sizeof(kind) - 8
        assert getattr(lib, call)(C.byref(args)) == binding.ERR_INVALID_ARG
        assert b"size" in lib.halos_step_error()
        assert getattr(lib, call)(None) == binding.ERR_INVALID_ARG


def _attention(step, **kw):
    a = step.AttentionArgs()
    a.struct_size, a.dtype, a.batch, a.sq, a.sk, a.n_q, a.n_kv, a.head_dim, a.scale = C.sizeof(a), 1, 2, 16, 16, 4, 2, 64, 0.125
    for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv"):
        setattr(a, n, 4096)
        getattr(a, n + "_stride")[:] = (16 * 4 * 64, 4 * 64, 64)
    a.lse = 4096
    for n, v in kw.items():
        setattr(a, n, v)
    return a


@pytest.mark.parametrize("kw,unsupported", [(dict(dtype=7), False), (dict(dtype=0), True), (dict(head_dim=60), True), (dict(head_dim=136), True), (dict(head_dim=0), True), (dict(n_kv=3), False),
                                            (dict(n_kv=0), False), (dict(scale=0.0), False), (dict(scale=float("nan")), False), (dict(scale=float("inf")), False), (dict(batch=-1), False),
                                            (dict(q=None), False), (dict(q=4098), True), (dict(q_stride=(C.c_int64 * 3)(4096, 250, 64)), True), (dict(k_stride=(C.c_int64 * 3)(4096, 0, 64)), True),
                                            (dict(lse=None), False), (dict(sq=1 << 31), True)])
def test_attention_refuses_on_the_host(lib, kw, unsupported):
    from paper_2506_04531_b200 import binding, step
    want = binding.ERR_UNSUPPORTED if unsupported else binding.ERR_INVALID_ARG
    assert lib.halos_attention_fwd(C.byref(_attention(step, **kw))) == want
    assert lib.halos_attention_bwd(C.byref(_attention(step, **kw))) == want


def test_workspace_is_checked(lib):
    from paper_2506_04531_b200 import binding, step
    a, n = _attention(step), C.c_uint64(0)
    assert lib.halos_attention_workspace(C.byref(a), C.byref(n)) == binding.OK and n.value >= 2 * 4 * 16 * 16
    for ptr, size in ((None, n.value), (4096, n.value - 1), (4104, n.value)):
        a.workspace, a.workspace_bytes = ptr, size
        assert lib.halos_attention_bwd(C.byref(a)) == binding.ERR_INVALID_ARG
        assert b"workspace" in lib.halos_step_error()


@pytest.mark.parametrize("kw,unsupported", [(dict(temperature=0.0), False), (dict(temperature=float("nan")), False), (dict(temperature=float("inf")), False), (dict(mix=-0.1), False),
                                            (dict(mix=float("nan")), False), (dict(k=1025), True), (dict(rows=-1), False), (dict(rows=1 << 31), True), (dict(vocab=0), False), (dict(logits=None), False),
                                            (dict(logits=4097), False), (dict(teacher_index=None), False), (dict(dlogits_stride=10), False), (dict(dtype=9), False)])
def test_distill_refuses_on_the_host(lib, kw, unsupported):
    from paper_2506_04531_b200 import binding, step
    a = step.DistillArgs()
    a.struct_size, a.rows, a.vocab, a.k, a.temperature, a.mix = C.sizeof(a), 4, 100, 8, 1.0, 0.5
    a.logits = a.labels = a.teacher_index = a.teacher_logits = a.loss = a.stats = a.dloss = a.dlogits = 4096
    a.logits_stride = a.dlogits_stride = 100
    for n, v in kw.items():
        setattr(a, n, v)
    assert lib.halos_distill_fwd_bwd(C.byref(a)) == (binding.ERR_UNSUPPORTED if unsupported else binding.ERR_INVALID_ARG)


@pytest.mark.parametrize("kw,unsupported", [(dict(rot_dim=3), False), (dict(rot_dim=66), False), (dict(head_dim=300), True), (dict(layout=2), False), (dict(freqs=None), False),
                                            (dict(q_in=None), False), (dict(q_in=4097), False), (dict(dtype=3), False), (dict(batch=-1), False)])
def test_rope_refuses_on_the_host(lib, kw, unsupported):
    from paper_2506_04531_b200 import binding, step
    a = step.RopeArgs()
    a.struct_size, a.dtype, a.batch, a.seq, a.n_q, a.n_k, a.head_dim, a.rot_dim = C.sizeof(a), 1, 1, 2, 2, 2, 64, 16
    a.freqs = a.q_in = a.k_in = a.q_out = a.k_out = 4096
    for n, v in kw.items():
        setattr(a, n, v)
    assert lib.halos_rope(C.byref(a)) == (binding.ERR_UNSUPPORTED if unsupported else binding.ERR_INVALID_ARG)


def test_cpu_tensors_are_refused(lib):
    from paper_2506_04531_b200 import binding, step
    x = torch.zeros(1, 4, 2, 64)
    with pytest.raises(binding.HalosError):
        step.rope(x, None, step.rotary_frequencies(16, device="cpu")[0])
    with pytest.raises(binding.HalosError):
        step.attention_forward(x, x, x)
    with pytest.raises(binding.HalosError):
        step.distill_forward(torch.zeros(2, 8), None, None, None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a host without a device")
def test_without_a_device_valid_calls_fail_with_a_cuda_error(lib):
    from paper_2506_04531_b200 import binding, step
    assert lib.halos_attention_fwd(C.byref(_attention(step))) == binding.ERR_CUDA
    assert b"no CPU path" in lib.halos_step_error()


def test_writing_over_the_input_with_other_strides_is_refused(lib):
    """The rows that are written would be others than those that are still to be read."""
    from paper_2506_04531_b200 import binding, step
    d = step.DistillArgs()
    d.struct_size, d.rows, d.vocab, d.temperature, d.mix = C.sizeof(d), 4, 100, 1.0, 0.5
    d.logits = d.labels = d.loss = d.stats = d.dloss = d.dlogits = 4096
    d.logits_stride, d.dlogits_stride = 108, 100
    for call in (lib.halos_distill_fwd_bwd, lib.halos_distill_bwd):
        assert call(C.byref(d)) == binding.ERR_INVALID_ARG and b"stride" in lib.halos_step_error()
    for which in "qk":
        r = step.RopeArgs()
        r.struct_size, r.dtype, r.batch, r.seq, r.n_q, r.n_k, r.head_dim, r.rot_dim = C.sizeof(r), 1, 1, 2, 2, 2, 64, 16
        r.freqs, r.q_in, r.k_in, r.q_out, r.k_out = 4096, 8192, 16384, 8192, 16384
        for n in ("q_in", "k_in", "q_out", "k_out"):
            getattr(r, n + "_stride")[:] = (256, 128, 64)
        getattr(r, which + "_out_stride")[:] = (256, 192, 64)
        assert lib.halos_rope(C.byref(r)) == binding.ERR_INVALID_ARG and b"strides" in lib.halos_step_error()
