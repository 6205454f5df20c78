"""Workers that train a small decoder and hand their results to the hierarchy.

    python -m paper_2506_04531_b200.examples.local_steps [--rounds 40] [--norm rms] [--max-norm 1.0]

Algorithm 1 end to end on one GPU: a worker restarts from the model it was scheduled with (theta_{t,0}), runs H local steps of
SGD on packed documents, and its result theta_{t,H} goes to its local parameter server.  The local step's operators are those of
``step``: rotary positions that begin anew with each document, attention that stays within documents, and cross-entropy mixed
with distillation from the top logits of the global model, which is what a worker can be sent of it over a slow link.
Matrix products and activations are torch's, and norms and the embedding, unless the decoder is to have root-mean-square norms (--norm rms): then these
are the operators of ``step``, too, and with --max-norm the gradients are clipped on their way into the step.  The data are synthetic: each document counts up by a stride of its own.
"""
from __future__ import annotations

import argparse

import torch
import torch.nn.functional as F

from .. import binding as hb, step
from ..inputs import gen, layouts

LAYERS, WIDTH, HEAD_DIM, ROT_DIM, VOCAB = 2, 128, 64, 16, 512
BATCH, SEQ, DOCUMENT, TOP_K = 8, 256, 64, 16


class Decoder:
    """The decoder of a layout, over flat fp32 parameters; activations in bfloat16.  norm: "layer", or "rms", which leaves the norms' biases unused."""

    def __init__(self, layout, norm="layer"):
        self.layout, self.norm = layout, norm
        self.freqs, self.magnitude = step.rotary_frequencies(ROT_DIM)

    def tensors(self, flat):
        return {t.name: p.view(t.shape) for t, p in zip(self.layout.tensors, torch.split(flat, [t.numel for t in self.layout.tensors]))}

    def attend(self, w, p, x, positions, doc_start):
        b, s = x.shape[:2]
        qkv = F.linear(x, w[p + "qkv.w"], w[p + "qkv.b"]).view(b, s, WIDTH // HEAD_DIM, 3, HEAD_DIM)
        q, k = step.rotary(qkv[:, :, :, 0], qkv[:, :, :, 1], self.freqs, positions=positions, magnitude=self.magnitude)
        o = step.attention(q, k, qkv[:, :, :, 2], doc_start=doc_start)
        return F.linear(o.reshape(b, s, WIDTH), w[p + "attn_out.w"], w[p + "attn_out.b"])

    def logits_rms(self, flat, tokens, positions, doc_start):
        """Each half of a layer is added to the residual by the norm in front of the next one."""
        full = self.tensors(flat)
        w = {n: p.to(torch.bfloat16) for n, p in full.items() if "ln" not in n and n != "embed_in"}
        x = step.embedding(full["embed_in"], tokens, dtype=torch.bfloat16)
        y = step.rms_norm(x, full["layers.0.ln1.w"])
        for i in range(LAYERS):
            p, after = f"layers.{i}.", "final_ln.w" if i + 1 == LAYERS else f"layers.{i + 1}.ln1.w"
            y, x = step.rms_norm(self.attend(w, p, y, positions, doc_start), full[p + "ln2.w"], residual=x)
            half = F.linear(F.gelu(F.linear(y, w[p + "up.w"], w[p + "up.b"])), w[p + "down.w"], w[p + "down.b"])
            y, x = step.rms_norm(half, full[after], residual=x)
        return F.linear(y, w["embed_out"]).view(-1, VOCAB)

    def logits(self, flat, tokens, positions, doc_start):
        if self.norm == "rms":
            return self.logits_rms(flat, tokens, positions, doc_start)
        w = {n: p.to(torch.bfloat16) for n, p in self.tensors(flat).items()}
        b, s = tokens.shape
        x = F.embedding(tokens, w["embed_in"])
        for i in range(LAYERS):
            p = f"layers.{i}."
            norm = lambda n: F.layer_norm(x, (WIDTH,), w[p + n + ".w"], w[p + n + ".b"])  # noqa: E731
            x = x + self.attend(w, p, norm("ln1"), positions, doc_start)
            x = x + F.linear(F.gelu(F.linear(norm("ln2"), w[p + "up.w"], w[p + "up.b"])), w[p + "down.w"], w[p + "down.b"])
        x = F.layer_norm(x, (WIDTH,), w["final_ln.w"], w["final_ln.b"])
        return F.linear(x, w["embed_out"]).view(b * s, VOCAB)


def documents(gen_):
    """Tokens, the next ones as labels, positions within documents, and where each token's document starts."""
    n = SEQ // DOCUMENT
    first, stride = torch.randint(0, VOCAB, (BATCH, n, 1), generator=gen_), torch.randint(1, 4, (BATCH, n, 1), generator=gen_)
    at = torch.arange(DOCUMENT + 1)
    text = (first + stride * at) % VOCAB
    labels = text[:, :, 1:].clone()
    labels[:, :, 0] = -100                                  # the first step of a document cannot be foreseen
    start = (torch.arange(n) * DOCUMENT)[None, :, None].expand(BATCH, n, DOCUMENT)
    place = at[:-1].expand(BATCH, n, DOCUMENT)
    return [x.reshape(BATCH, SEQ).cuda() for x in (text[:, :, :-1], labels, place.to(torch.int32), start.to(torch.int32).contiguous())]


def local_steps(model, flat, teacher, batches, rate, mix, max_norm=None):
    """H steps of SGD from `flat`, the gradients clipped to max_norm if there is one; the result and the last step's cross-entropy."""
    theta = flat.clone().requires_grad_()
    for tokens, labels, positions, starts in batches:
        idx = t = None
        if teacher is not None:
            with torch.no_grad():
                t, idx = model.logits(teacher, tokens, positions, starts).topk(TOP_K, 1)
        z, counted = model.logits(theta, tokens, positions, starts), (labels != -100).sum()
        loss = step.distill_loss(z, labels.reshape(-1), idx, t, temperature=2.0, mix=mix if teacher is not None else 0.0)
        grad, = torch.autograd.grad(loss.sum() / counted, theta)
        if max_norm is None:
            theta = (theta.detach() - rate * grad).requires_grad_()
        else:
            with torch.no_grad():
                step.sgd_step(model.tensors(theta).values(), model.tensors(grad).values(), rate, max_norm=max_norm)
    plain, _ = step.distill_forward(z.detach(), labels.reshape(-1), None, None, mix=0.0)
    return theta.detach(), float(plain.sum() / counted)


def run(rounds: int = 40, h_steps: int = 16, rate: float = 0.3, mix: float = 0.1, seed: int = 0, norm: str = "layer", max_norm=None, log=print):
    layout = layouts.decoder_layout("example", LAYERS, WIDTH, VOCAB)
    model = Decoder(layout, norm)
    worker_lps = [0, 0, 1, 1]
    start = torch.from_numpy(gen.theta_init(layout, seed)).cuda()
    rng = torch.Generator().manual_seed(seed)
    losses = []
    with hb.Halos(start, worker_lps, layout.numel, K=4) as h:
        for r in range(rounds):
            w = r % len(worker_lps)
            lps = worker_lps[w]
            teacher = h.peek(hb.BUF_THETA_G, 0) if r >= 2 * len(worker_lps) else None   # until then it has learned nothing
            result, loss = local_steps(model, h.peek(hb.BUF_THETA0, w), teacher, [documents(rng) for _ in range(h_steps)], rate, mix, max_norm)
            h.worker_delta(w, result)                       # Alg. 1 line 25
            if h.lps_apply(lps, w):                         # lines 10-13
                h.lps_push(lps)                             # line 14
                h.gps_merge(lps)                            # lines 2-4
                h.lps_pull(lps)                             # lines 18-19
            losses.append(loss)
            if log and r % 10 == 9:
                log(f"round {r + 1}: cross-entropy of the last 10 results {sum(losses[-10:]) / 10:.3f}")
        iterations = h.counters(0)
    return losses, iterations


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rounds", type=int, default=40)
    ap.add_argument("--norm", choices=("layer", "rms"), default="layer")
    ap.add_argument("--max-norm", type=float)
    args = ap.parse_args()
    run(args.rounds, norm=args.norm, max_norm=args.max_norm)


if __name__ == "__main__":
    main()
