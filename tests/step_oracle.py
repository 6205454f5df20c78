"""Plain 64-bit forms of the local step's operators, and the error bounds that follow from where the kernels round.

Nothing here comes from the CUDA library.  u is half the spacing of a 16-bit type at 1: every value that is rounded once to
that type is off by at most u of itself."""
from __future__ import annotations

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -24, torch.float32: 1e-38}


def rope(x, freqs, positions, layout, magnitude, inverse):
    """(y, bound) of x [b, s, h, d]; positions [b, s]."""
    r = 2 * freqs.numel()
    x = x.double()
    # the angle modulo a turn in exact integer arithmetic: a turn is 2^64
    turn = [int(math.floor((w / (2 * math.pi)) * 2.0 ** 64)) for w in freqs.tolist()]
    angle = torch.tensor([[((t * w) % 2 ** 64) / 2.0 ** 64 for w in turn] for t in positions.reshape(-1).tolist()], dtype=torch.float64, device=x.device)
    angle = angle.reshape(*positions.shape, 1, r // 2) * (2 * math.pi) * (-1 if inverse else 1)
    first = torch.arange(r // 2, device=x.device) * (1 if layout == "half" else 2)
    second = first + (r // 2 if layout == "half" else 1)
    y, size = x.clone(), torch.zeros_like(x)
    a, b = x[..., first], x[..., second]
    y[..., first] = magnitude * (a * angle.cos() - b * angle.sin())
    y[..., second] = magnitude * (b * angle.cos() + a * angle.sin())
    size[..., first] = size[..., second] = magnitude * (a.abs() + b.abs())
    # angle: 2^-25 half turns of rounding and 2^-32 of a turn cut off; sine and cosine 2 ulp; magnitude, product, sum: 2^-24 each
    return y, size * (2.0 ** -25 * math.pi + 2.0 ** -32 * 2 * math.pi + 5 * 2.0 ** -24)


def visible(b, sq, sk, causal, doc_start, lens, device):
    t = torch.arange(sq, device=device)[:, None] + sk - sq
    j = torch.arange(sk, device=device)[None, :]
    n = sk if lens is None else max(0, min(sk, int(lens[b])))
    see = (j < n) & (t < n)
    if causal:
        see = see & (j <= t)
    if doc_start is not None:
        see = see & (j >= doc_start[b].long()[:, None])
    return see


def attention(q, k, v, dout=None, *, scale, causal, doc_start=None, lens=None):
    """A dict of o, lse (and dq, dk, dv) and, under the name + "_bound", how far the kernels may be off: they round p and ds once to the
    inputs' type before they enter a product, o before D = dout.o is formed from it, and each result once."""
    u, tiny = U[q.dtype], TINY[q.dtype]
    B, sq, H, D = q.shape
    sk, Hk = k.shape[1:3]
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=q.device)  # noqa: E731
    r = {n: z(B, sq, H, D) for n in ("o", "o_bound", "dq", "dq_bound")} | {n: z(B, sk, Hk, D) for n in ("dk", "dk_bound", "dv", "dv_bound")}
    r["lse"] = torch.full((B, H, sq), -math.inf, dtype=torch.float64, device=q.device)
    e32 = 2e-6  # relative, of a probability formed in 32 bits: exponent |s - lse| < 30 times 2^-24, approximations of 2^-22
    for b in range(B):
        see = visible(b, sq, sk, causal, doc_start, lens, q.device)
        rows, cols = see.any(1), see.any(0)
        for h in range(H):
            g = h // (H // Hk)
            qq = torch.where(rows[:, None], q[b, :, h].double(), 0.0)
            kk, vv = (torch.where(cols[:, None], x[b, :, g].double(), 0.0) for x in (k, v))
            s = (qq @ kk.T * scale).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(s, 1) if sk else torch.full((sq,), -math.inf, dtype=torch.float64, device=q.device)
            p = torch.where(see, torch.exp(s - torch.where(rows, lse, 0.0)[:, None]), 0.0)
            o = p @ vv
            spread = p @ vv.abs()
            r["o"][b, :, h], r["lse"][b, h] = o, lse
            r["o_bound"][b, :, h] = (u + 2 * e32) * spread + u * o.abs() + tiny
            if dout is None:
                continue
            do = torch.where(rows[:, None], dout[b, :, h].double(), 0.0)
            dp = do @ vv.T
            delta = (p * dp).sum(1, keepdim=True)
            ds = p * (dp - delta)
            delta_off = 2 * u * (do.abs() * spread).sum(1, keepdim=True)
            ds_off = u * ds.abs() + p * (delta_off + 2 * e32 * (do.abs() @ vv.abs().T + (do.abs() * spread).sum(1, keepdim=True))) + tiny
            r["dq"][b, :, h] = scale * (ds @ kk)
            r["dq_bound"][b, :, h] = scale * (ds_off @ kk.abs()) + u * r["dq"][b, :, h].abs() + tiny
            r["dk"][b, :, g] += scale * (ds.T @ qq)
            r["dk_bound"][b, :, g] += scale * (ds_off.T @ qq.abs())
            r["dv"][b, :, g] += p.T @ do
            r["dv_bound"][b, :, g] += (u + 2 * e32) * (p.T @ do.abs()) + tiny
    for n in ("dk", "dv"):
        r[n + "_bound"] += u * r[n].abs() + tiny
    return r


def distill(z, labels, idx, t, dloss, *, temperature, mix, ignore_index):
    """A dict of loss, stats, dz and their bounds."""
    u, tiny, T = U[z.dtype], TINY[z.dtype], temperature
    n, V = z.shape
    x = z.double()
    counted = torch.ones(n, dtype=torch.bool, device=z.device) if labels is None else labels.long() != ignore_index
    lse1, lseT = torch.logsumexp(x, 1), torch.logsumexp(x / T, 1)
    q1, qT = torch.exp(x - lse1[:, None]), torch.exp(x / T - lseT[:, None])
    loss, size = torch.zeros(n, dtype=torch.float64, device=z.device), torch.zeros(n, dtype=torch.float64, device=z.device)
    dz, dz_size = torch.zeros_like(x), torch.zeros_like(x)
    # a thread adds up to V/128 terms in a row, 2^-24 each at worst (the smallest CTA that takes such rows); differences z - max: 2^-24
    top = torch.where(torch.isfinite(x), x, 0.0).abs().amax(1)
    eps = 2.0 ** -24 * (V / 128 + 64) + 2.0 ** -22 * top * (1 + 1 / T)
    if labels is not None:
        y = labels.long().clamp(0, V - 1)[:, None]
        loss += (1 - mix) * (lse1 - x.gather(1, y)[:, 0])
        size += (1 - mix) * (1 + lse1.abs() + x.gather(1, y)[:, 0].abs())
        dz += (1 - mix) * q1
        dz_size += (1 - mix) * q1
        dz.scatter_add_(1, y, torch.full_like(dz[:, :1], mix - 1))
        dz_size.scatter_add_(1, y, torch.full_like(dz[:, :1], 1 - mix))
    if idx is not None and idx.shape[1]:
        sent = idx >= 0
        w = (t.double() / T).masked_fill(~sent, -math.inf)
        p = torch.softmax(w, 1).nan_to_num(0.0)
        any_ = (p.sum(1) > 0).double()
        at = idx.long().clamp_min(0)
        zk = torch.where(p > 0, x.gather(1, at), 0.0)
        loss += mix * T * T * (torch.special.xlogy(p, p) - p * zk / T + p * lseT[:, None]).sum(1)
        size += mix * T * T * (torch.special.xlogy(p, p).abs() + p * zk.abs() / T + p * lseT[:, None].abs()).sum(1)
        dz += mix * T * any_[:, None] * qT
        dz_size += mix * T * any_[:, None] * qT
        dz.scatter_add_(1, at, -mix * T * p)
        dz_size.scatter_add_(1, at, mix * T * p)
    g = dloss.double() if dloss is not None else torch.ones(n, dtype=torch.float64, device=z.device)
    loss, dz = torch.where(counted, loss, 0.0), torch.where(counted[:, None], dz * g[:, None], 0.0)
    dz_bound = torch.where(counted[:, None], dz_size * g.abs()[:, None] * (8 * eps + 2e-6)[:, None], 0.0) + u * dz.abs() + tiny
    return dict(loss=loss, loss_bound=(eps + 2.0 ** -21) * size + eps * (1 + T * T), stats=torch.stack([lse1, lseT], 1), stats_bound=eps[:, None] * (1 + 0 * torch.stack([lse1, lseT], 1)),
                dz=dz, dz_bound=dz_bound)
