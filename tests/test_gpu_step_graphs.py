"""The local step's operators captured into CUDA graphs, from several threads, and with gradients that are not laid out as usual."""
from __future__ import annotations

import subprocess
import sys
import threading
from pathlib import Path

import pytest
import torch

from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent

# All calls at once on static inputs; and whether a replay after new inputs gives what plain calls give.
CAPTURE = """
import torch
from paper_2506_04531_b200 import step
g = torch.Generator(device="cuda").manual_seed(0)
x = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
def inputs():
    return [x(2, 200, 4, 64) for _ in range(4)] + [x(400, 3000)]
labels, ones = torch.arange(400, device="cuda"), torch.ones(400, device="cuda")
idx, t = torch.arange(8, device="cuda").expand(400, -1).contiguous(), torch.ones(400, 8, device="cuda")
freqs = step.rotary_frequencies(16)[0]
def everything(q, k, v, do, z):
    q2, k2 = step.rope(q, k, freqs, offset=3)
    o, lse = step.attention_forward(q2, k2, v)
    grads = step.attention_backward(do, q2, k2, v, o, lse)
    loss, stats = step.distill_forward(z, labels, idx, t, temperature=2.0)
    dz = step.distill_backward(ones, z, stats, labels, idx, t, temperature=2.0)
    return [q2, k2, o, lse, *grads, loss, stats, dz, *step.distill_loss_and_grad(z, labels, idx, t, ones)]
static = inputs()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):           # the process's first calls
    out = everything(*static)
for _ in range(2):
    fresh = inputs()
    for a, b in zip(static, fresh):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, everything(*fresh)))
assert not step.fault()
print("same")
"""


def test_capture_from_the_first_call_on():
    r = subprocess.run([sys.executable, "-c", CAPTURE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]


def test_threads_with_streams_of_their_own():
    """Vocabularies that need different amounts of shared memory, so that the threads also meet where a kernel's limit is set."""
    vocabs, got, errors = [2500, 9000, 14000, 23000, 30000, 52000], {}, []

    def inputs(V):
        g = torch.Generator(device="cuda").manual_seed(V)
        q = torch.randn((1, 130, 2, 64), generator=g, device="cuda").bfloat16()
        return q, torch.randn((40, V), generator=g, device="cuda"), torch.arange(40, device="cuda"), torch.ones(40, device="cuda")

    def run(V):
        q, z, labels, ones = inputs(V)
        return [*step.attention_forward(q, q, q), *step.distill_loss_and_grad(z, labels, None, None, ones, temperature=1.7)]

    def work(V):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    got[V] = run(V)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(V,)) for V in vocabs]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not errors
    for V in vocabs:
        assert all(torch.equal(a, b) for a, b in zip(got[V], run(V)))


def test_gradients_that_arrive_broadcast_or_transposed():
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((2, 70, 3, 64), generator=g, device="cuda").bfloat16() for _ in range(3))
    for dout in (q.new_ones(()).expand_as(q), torch.randn((3, 2, 64, 70), generator=g, device="cuda").bfloat16().permute(1, 3, 0, 2)):
        strange, plain = ([x.clone().requires_grad_() for x in (q, k, v)] for _ in range(2))
        step.attention(*strange).backward(dout)
        step.attention(*plain).backward(dout.contiguous())
        assert all(torch.equal(a.grad, b.grad) for a, b in zip(strange, plain))
        freqs = step.rotary_frequencies(16)[0]
        strange, plain = ([x.clone().requires_grad_() for x in (q, k)] for _ in range(2))
        torch.autograd.backward(step.rotary(*strange, freqs), (dout, dout))
        torch.autograd.backward(step.rotary(*plain, freqs), (dout.contiguous(), dout.contiguous()))
        assert all(torch.equal(a.grad, b.grad) for a, b in zip(strange, plain))
    z, labels = torch.randn((6, 500), generator=g, device="cuda"), torch.arange(6, device="cuda")
    for dloss in (z.new_ones(()).expand(6), torch.rand((12,), generator=g, device="cuda")[::2]):
        strange, plain = z.clone().requires_grad_(), z.clone().requires_grad_()
        step.distill_loss(strange, labels).backward(dloss)
        step.distill_loss(plain, labels).backward(dloss.contiguous())
        assert torch.equal(strange.grad, plain.grad)
