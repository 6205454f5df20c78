"""The embedding, norms and gradients' operators together: in a local step, captured into CUDA graphs, and from several threads."""
from __future__ import annotations

import subprocess
import sys
import threading
from pathlib import Path

import pytest
import torch
import torch.nn.functional as F

from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


def _x(shape, seed, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def _rms(x, w):
    return x * (x.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w


def test_a_local_step_against_64_bits():
    """Tokens to clipped update, all in 32 bits.  Ten operations lie on the way, each off by some 100 of 2^-24 of its terms' sizes (sums of 48 to 160): 6e-5 in
    all, for which 1e-3 of a tensor's largest gradient leaves room."""
    d, vocab, b, s = 48, 160, 3, 37
    shapes = dict(embed=(vocab, d), n1=(d,), w1=(d, d), n2=(d,), w2=(d, d), n3=(d,), out=(vocab, d))
    tokens = torch.randint(0, vocab, (b, s), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    labels = torch.randint(0, vocab, (b * s,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    start = {n: _x(sh, 3 + i, 0.3) + (1 if len(sh) == 1 else 0) for i, (n, sh) in enumerate(shapes.items())}

    p = {n: t.clone().requires_grad_() for n, t in start.items()}
    x = step.embedding(p["embed"], tokens, scale=2.0)
    y = step.rms_norm(x, p["n1"])
    y, x = step.rms_norm(F.linear(y, p["w1"]), p["n2"], residual=x)
    y, x = step.rms_norm(F.linear(y, p["w2"]), p["n3"], residual=x)
    loss = step.distill_loss(F.linear(y, p["out"]).view(-1, vocab), labels, mix=0.0).mean()
    grads = torch.autograd.grad(loss, list(p.values()))

    q = {n: t.double().requires_grad_() for n, t in start.items()}
    x = F.embedding(tokens, q["embed"]) * 2.0
    x1 = F.linear(_rms(x, q["n1"]), q["w1"]) + x
    x2 = F.linear(_rms(x1, q["n2"]), q["w2"]) + x1
    want = F.cross_entropy(F.linear(_rms(x2, q["n3"]), q["out"]).view(-1, vocab), labels)
    exact = torch.autograd.grad(want, list(q.values()))
    assert abs(loss.item() - want.item()) <= 1e-5 * want.item()
    for n, g, e in zip(shapes, grads, exact):
        assert float((g.double() - e).abs().max()) <= 1e-3 * float(e.abs().max()), n

    norm = float(sum(e.square().sum() for e in exact)) ** 0.5
    params = [t.clone() for t in start.values()]
    got = step.sgd_step(params, grads, 0.5, max_norm=norm / 2)
    assert abs(float(got) - norm) <= 1e-3 * norm
    for t, before, e in zip(params, start.values(), exact):
        assert float((t.double() - (before.double() - 0.25 * e)).abs().max()) <= 2e-3 * float(e.abs().max()) + 1e-6
    assert not step.fault()


def test_the_example_runs_with_them():
    from paper_2506_04531_b200.examples import local_steps
    losses, counters = local_steps.run(rounds=10, h_steps=4, norm="rms", max_norm=0.5, log=None)
    assert all(x == x and x < 20 for x in losses) and counters["t"] >= 0
    assert not step.fault()


def test_the_examples_gradient():
    """Of the decoder with root-mean-square norms, against the same in 32 bits without these operators.  Activations are rounded to 8 bits of mantissa about a
    dozen times on the way there and back, 2^-8 each at worst: 5% together, for which 10% of the gradient's length leaves room."""
    from paper_2506_04531_b200.examples import local_steps as ex
    from paper_2506_04531_b200.inputs import gen, layouts
    layout = layouts.decoder_layout("example", ex.LAYERS, ex.WIDTH, ex.VOCAB)
    flat = torch.from_numpy(gen.theta_init(layout, 0)).cuda()
    flat += _x(flat.shape, 9, 0.02)
    tokens, labels, positions, starts = ex.documents(torch.Generator().manual_seed(0))
    model = ex.Decoder(layout, "rms")
    a = flat.clone().requires_grad_()
    got, = torch.autograd.grad(F.cross_entropy(model.logits(a, tokens, positions, starts).float(), labels.reshape(-1)), a)

    b = flat.clone().requires_grad_()
    w, heads = model.tensors(b), ex.WIDTH // ex.HEAD_DIM
    n, s = tokens.shape
    i = torch.arange(s, device="cuda")
    seen = (i[None, None, :] <= i[None, :, None]) & (i[None, None, :] >= starts[:, :, None])
    angle = (positions.double()[:, :, None] * model.freqs).float()[:, :, None, :]

    def turned(x):
        r, rest = x[..., : ex.ROT_DIM], x[..., ex.ROT_DIM:]
        u, v = r.chunk(2, -1)
        return torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin(), rest], -1)

    x = F.embedding(tokens, w["embed_in"])
    for layer in range(ex.LAYERS):
        p = f"layers.{layer}."
        qkv = F.linear(_rms(x, w[p + "ln1.w"]), w[p + "qkv.w"], w[p + "qkv.b"]).view(n, s, heads, 3, ex.HEAD_DIM)
        q, k, v = turned(qkv[:, :, :, 0]), turned(qkv[:, :, :, 1]), qkv[:, :, :, 2]
        score = torch.einsum("bihd,bjhd->bhij", q, k) * ex.HEAD_DIM ** -0.5
        o = torch.einsum("bhij,bjhd->bihd", score.masked_fill(~seen[:, None], float("-inf")).softmax(-1), v).reshape(n, s, ex.WIDTH)
        x = x + F.linear(o, w[p + "attn_out.w"], w[p + "attn_out.b"])
        y = _rms(x, w[p + "ln2.w"])
        x = x + F.linear(F.gelu(F.linear(y, w[p + "up.w"], w[p + "up.b"])), w[p + "down.w"], w[p + "down.b"])
    want, = torch.autograd.grad(F.cross_entropy(F.linear(_rms(x, w["final_ln.w"]), w["embed_out"]).view(-1, ex.VOCAB), labels.reshape(-1)), b)
    assert float((got - want).norm()) <= 0.1 * float(want.norm())


# All calls at once on static inputs, the process's first ones; two graphs that run side by side; whether replays after new inputs give what plain calls give.
CAPTURE = """
import torch
from paper_2506_04531_b200 import step
g = torch.Generator(device="cuda").manual_seed(0)
x = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
def inputs():
    return [torch.randint(0, 3000, (4, 700), generator=g, device="cuda"), torch.randn(3000, 96, generator=g, device="cuda"), x(4, 700, 96), x(4, 700, 96), x(4, 700, 96), torch.randn(96, generator=g, device="cuda"),
            torch.randint(0, 3000, (70000,), generator=g, device="cuda"), x(70000, 8)]
def everything(tokens, table, a, b, c, w, many, rows):
    e = step.embedding_forward(table, tokens, dtype=torch.bfloat16)
    y, s, rstd = step.rms_norm_forward(e, w, residual=a)
    q, scales, _, _ = step.rms_norm_quantized(b, w, group=32)
    dx, dw = step.rms_norm_backward(c, s, w, rstd, dsummed=b)
    dt = step.embedding_backward(dx, tokens, 3000, dtype=torch.float32)
    dm = step.embedding_backward(rows, many, 3000)
    out = [torch.empty_like(dt), torch.empty_like(dw)]
    norm = step.clip_grads([dt, dw], 1.0, out=out)
    params = [table.clone(), w.clone()]
    return [e, y, s, rstd, q.view(torch.uint8), scales, dx, dw, dt, dm, norm, *out, step.sgd_step(params, [dt, dw], 0.1, max_norm=0.5), *params, step.grad_norm([dm])]
static, graphs, outs = [inputs(), inputs()], [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
for i in range(2):
    with torch.cuda.graph(graphs[i]):
        outs.append(everything(*static[i]))
streams = [torch.cuda.Stream(), torch.cuda.Stream()]
for _ in range(3):
    fresh = [inputs(), inputs()]
    for st, fr in zip(static, fresh):
        for a, b in zip(st, fr):
            a.copy_(b)
    torch.cuda.synchronize()
    for graph, stream in zip(graphs, streams):
        with torch.cuda.stream(stream):
            graph.replay()
    torch.cuda.synchronize()
    for out, fr in zip(outs, fresh):
        for k, (a, b) in enumerate(zip(out, everything(*fr))):
            assert torch.equal(a, b), k
assert not step.fault()
print("same")
"""


def test_capture_from_the_first_call_on():
    r = subprocess.run([sys.executable, "-c", CAPTURE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]


# Forward and backward by autograd on static leaves, then the parameters' clipped step, in one graph: replays walk the way that eager steps walk.
AUTOGRAD = """
import torch
from paper_2506_04531_b200 import step
def state():
    g = torch.Generator(device="cuda").manual_seed(1)
    x = lambda *s: torch.randn(s, generator=g, device="cuda")
    return [x(500, 72), x(72), x(72)], torch.randint(0, 500, (3, 41), generator=g, device="cuda"), x(3, 41, 72)
def one(params, tokens, target):
    leaves = [p.detach().requires_grad_() for p in params]
    e = step.embedding(leaves[0], tokens, scale=2.0)
    y = step.rms_norm(e, leaves[1])
    z, s = step.rms_norm(y, leaves[2], residual=e)
    grads = torch.autograd.grad((z * target).sum() + (s * s).mean(), leaves)
    return step.sgd_step(params, grads, 0.1, max_norm=1.0)
params, tokens, target = state()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    norm = one(params, tokens, target)
eager, _, _ = state()
for k in range(4):
    graph.replay()
    want = one(eager, tokens, target)
    assert torch.equal(norm, want), k
    assert all(torch.equal(a, b) for a, b in zip(params, eager)), k
assert not torch.equal(params[0], state()[0][0])
print("same")
"""


def test_autograd_captured():
    r = subprocess.run([sys.executable, "-c", AUTOGRAD], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]


def test_threads_with_streams_of_their_own():
    widths, got, errors = [96, 1021, 2048, 4096, 9000, 12288], {}, []

    def run(d):
        t = torch.randint(0, 500, (300,), generator=torch.Generator(device="cuda").manual_seed(d), device="cuda")
        x, w = _x((300, d), d, dtype=torch.bfloat16), _x((d,), d + 1)
        y, s, rstd = step.rms_norm_forward(x, w, residual=x)
        dx, dw = step.rms_norm_backward(y, s, w, rstd)
        return [y, dx, dw, step.embedding_backward(dx, t, 500, dtype=torch.float32), step.rms_norm_quantized(x, w, group=64)[1], step.grad_norm([dx, dw])]

    def work(d):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    got[d] = run(d)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(d,)) for d in widths]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not errors
    for d in widths:
        assert all(torch.equal(a, b) for a, b in zip(got[d], run(d)))


def test_tensors_that_come_from_another_stream():
    """Inputs made on one stream, used on another after an event, outputs handed back: what the calls allocate belongs to the stream they run on."""
    side = torch.cuda.Stream()
    for seed in range(5):
        x, w, t = _x((2000, 256), seed), _x((256,), 100 + seed), torch.randint(0, 900, (2000,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y, _, rstd = step.rms_norm_forward(x, w)
            got = [y, step.embedding_backward(y, t, 900), *step.rms_norm_backward(y, x, w, rstd)]
        torch.cuda.current_stream().wait_stream(side)
        y, _, rstd = step.rms_norm_forward(x, w)
        assert all(torch.equal(a, b) for a, b in zip(got, [y, step.embedding_backward(y, t, 900), *step.rms_norm_backward(y, x, w, rstd)]))
