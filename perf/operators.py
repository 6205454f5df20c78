"""The operators of a worker's local step, as they are measured: rotary positions, attention with its backward pass,
and the distillation loss with its gradient.

Sizes: the head counts, widths and the vocabulary follow the decoder layouts of this repository (d = 512 to 2048 in
heads of 64 or 128, V = 50304, sequences of 2048 tokens) and go on from there to odd and ragged ones."""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
IGNORED = -100


def listed():
    return [
        # queries and keys of one layer of the 160m layout for 32 sequences, as views of the fused projection's output;
        # a quarter of each head is rotated
        dict(name="rope_160m", op="rope", back=False, dtype="bf16", batch=32, seq=2048, hq=12, hk=12, d=64, rot=16, layout="half", scaling="none", factor=1.0, packed=True, positions="offset"),
        # one long sequence with shared key heads, whole heads rotated, frequencies scaled for eight times the length trained on
        dict(name="rope_long_f16", op="rope", back=False, dtype="f16", batch=1, seq=16411, hq=16, hk=4, d=128, rot=128, layout="interleaved", scaling="ramp", factor=8.0, packed=False, positions="offset"),
        # the gradient's way back in 32 bits, a head and a rotated part that no vector width divides, packed documents
        dict(name="rope_back_f32_odd", op="rope", back=True, dtype="f32", batch=3, seq=1021, hq=10, hk=5, d=80, rot=22, layout="half", scaling="linear", factor=4.0, packed=False, positions="documents"),
        # one token for each of eight sequences: latency
        dict(name="rope_token", op="rope", back=False, dtype="bf16", batch=8, seq=1, hq=16, hk=16, d=64, rot=16, layout="half", scaling="none", factor=1.0, packed=True, positions="documents"),
        # attention of one layer of the 160m layout over 16 sequences, both directions
        dict(name="attention_160m", op="attention", back=False, dtype="bf16", batch=16, seq=2048, hq=12, hk=12, d=64, causal=True, documents=0, ragged=False, packed=True),
        dict(name="attention_160m_back", op="attention", back=True, dtype="bf16", batch=16, seq=2048, hq=12, hk=12, d=64, causal=True, documents=0, ragged=False, packed=True),
        # the 1p4b layout: heads of 128
        dict(name="attention_1p4b", op="attention", back=False, dtype="bf16", batch=4, seq=2048, hq=16, hk=16, d=128, causal=True, documents=0, ragged=False, packed=True),
        # one long odd sequence of packed documents, four query heads to a key head, backward
        dict(name="attention_docs_back", op="attention", back=True, dtype="f16", batch=1, seq=8197, hq=16, hk=4, d=128, causal=True, documents=5, ragged=False, packed=False),
        # a few short sequences of different lengths, padded with whatever was in memory: latency
        dict(name="attention_short", op="attention", back=False, dtype="f16", batch=5, seq=67, hq=8, hk=2, d=80, causal=True, documents=0, ragged=True, packed=False),
        # the loss of four sequences of 2048 tokens against a teacher's 64 top logits, and its gradient, in one call
        dict(name="distill_step", op="distill", part="both", dtype="bf16", rows=8192, vocab=50304, k=64, temperature=2.0, mix=0.5, spare=0),
        # loss alone (evaluation) in 32 bits over an odd vocabulary
        dict(name="distill_loss_f32", op="distill", part="forward", dtype="f32", rows=1003, vocab=10007, k=20, temperature=1.5, mix=0.7, spare=0),
        # gradient alone, from the statistics that the forward kept, rows with room between them
        dict(name="distill_back_f16", op="distill", part="backward", dtype="f16", rows=2048, vocab=32003, k=100, temperature=1.0, mix=0.3, spare=13),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rope", "attention", "attention", "distill"])
    if op == "rope":
        dtype, d = rng.choice(list(TYPES)), rng.choice([40, 64, 80, 96, 128, 256])
        hk = rng.choice([1, 2, 3, 4, 8, 12])
        hq = hk * rng.choice([1, 1, 2, 4])
        seq = _spread(rng, 1, 16384)
        tokens = 96_000_000 // (BYTES[dtype] * d * (hq + hk))  # at most 192 MB moved
        batch = max(1, min(_spread(rng, 1, 64), tokens // seq))
        return dict(op=op, back=rng.random() < 0.5, dtype=dtype, batch=batch, seq=seq, hq=hq, hk=hk, d=d, rot=rng.choice([d, d // 2, d // 4, 2]) // 2 * 2,
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "base", "ramp"]), factor=rng.choice([2.0, 4.0, 8.0]),
                    packed=rng.random() < 0.5, positions=rng.choice(["offset", "documents"]))
    if op == "attention":
        d = rng.choice([32, 64, 64, 72, 80, 96, 128, 128])
        seq, causal = _spread(rng, 1, 8192), rng.random() < 0.8
        room = 16 * 12 * 2048 * 2048 * 64  # products of the largest listed case
        most = max(1, room // (seq * seq * max(64, d)) // (1 if causal else 2))
        hk = min(rng.choice([1, 2, 3, 4, 8, 12]), most)
        hq = hk * min(rng.choice([1, 1, 2, 3, 4]), most // hk)
        batch = max(1, min(_spread(rng, 1, 32), most // hq))
        return dict(op=op, back=rng.random() < 0.5, dtype=rng.choice(["bf16", "f16"]), batch=batch, seq=seq, hq=hq, hk=hk, d=d, causal=causal,
                    documents=rng.choice([0, 0, 3, 9]), ragged=rng.random() < 0.3, packed=rng.random() < 0.5)
    dtype, vocab = rng.choice(list(TYPES)), _spread(rng, 1000, 128000)
    rows = max(1, min(_spread(rng, 1, 8192), 400_000_000 // (vocab * BYTES[dtype] // 2)))
    return dict(op=op, part=rng.choice(["both", "both", "forward", "backward"]), dtype=dtype, rows=rows, vocab=vocab, k=rng.choice([1, 8, 20, 64, 100]),
                temperature=rng.choice([1.0, 1.5, 2.0, 4.0]), mix=rng.choice([0.0, 0.3, 0.5, 1.0]), spare=rng.choice([0, 0, 8, 13]))


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(shape, gen, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _heads(c, gen, dtype, count, n):
    """`n` tensors [batch, seq, heads, d]: views of one projection's output where the case is packed, else tensors of their own."""
    if c["packed"] and len(set(count)) == 1:
        every = _normal((c["batch"], c["seq"], count[0], n, c["d"]), gen, dtype)
        return [every[:, :, :, i] for i in range(n)]
    return [_normal((c["batch"], c["seq"], h, c["d"]), gen, dtype) for h in count]


def _document_starts(c, gen, documents):
    """[batch, seq]: where the document of each token begins."""
    at = torch.rand((c["batch"], c["seq"]), generator=gen, device="cuda") < documents / max(1, c["seq"])
    place = torch.arange(c["seq"], device="cuda").expand(c["batch"], -1)
    return torch.where(at, place, torch.zeros_like(place)).cummax(1).values


def frequencies(c):
    """Radians per position of each rotated pair, and the factor on the result."""
    r, base, f = c["rot"], 10000.0, c["factor"]
    if c["scaling"] == "base" and r > 2:
        base *= f ** (r / (r - 2))
    w = torch.tensor([base ** (-2.0 * p / r) for p in range(r // 2)], dtype=torch.float64)
    if c["scaling"] == "linear":
        return w / f, 1.0
    if c["scaling"] == "ramp":  # what turns often within 2048 positions stays, what hardly turns is stretched
        keep = ((w * 2048 / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        return w * keep + w / f * (1 - keep), 0.1 * math.log(f) + 1.0
    return w, 1.0


def prepare(case, seed):
    c, gen = case, _generator(seed)
    dtype = TYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "rope":
        s["q"], s["k"] = _heads(c, gen, dtype, [c["hq"], c["hk"]], 2 if c["hq"] != c["hk"] or not c["packed"] else 3)[:2]
        w, s["magnitude"] = frequencies(c)
        s["freqs"] = w.cuda()
        place = torch.arange(c["seq"], device="cuda").expand(c["batch"], -1)
        if c["positions"] == "documents":  # positions begin anew with each document
            s["positions"] = (place - _document_starts(c, gen, 4) + seed % 5).to(torch.int32)
        else:
            s["positions"] = (place + (seed % 1000)).to(torch.int64)
    elif c["op"] == "attention":
        s["q"], s["k"], s["v"] = _heads(c, gen, dtype, [c["hq"], c["hk"], c["hk"]], 3)
        s["doc_start"] = _document_starts(c, gen, c["documents"]).to(torch.int32) if c["documents"] else None
        s["lens"] = None
        if c["ragged"]:  # one sequence may be empty; what lies past the end of each is whatever was there
            lens = torch.randint(0, c["seq"] + 1, (c["batch"],), generator=gen, device="cuda")
            lens[0] = c["seq"]
            s["lens"] = lens.to(torch.int32)
            past = (torch.arange(c["seq"], device="cuda")[None, :] >= lens[:, None])[:, :, None, None]
            for n in "qkv":
                s[n] = s[n].masked_fill(past, float("nan"))
        if c["back"]:
            s["dout"] = _normal((c["batch"], c["seq"], c["hq"], c["d"]), gen, dtype)
            s["out"], s["lse"] = _attention(s)  # what the forward pass left behind
    else:
        n, v, k = c["rows"], c["vocab"], c["k"]
        z = _normal((n, v + c["spare"]), gen, dtype, 2.5)[:, :v]
        s["z"] = z
        s["labels"] = torch.randint(0, v, (n,), generator=gen, device="cuda")
        s["labels"][torch.rand((n,), generator=gen, device="cuda") < 0.05] = IGNORED
        places = torch.randint(0, max(1, v // k), (n, k), generator=gen, device="cuda") + torch.arange(k, device="cuda") * (v // k)
        t = _normal((n, k), gen, torch.float32, 1.5) + 8.0
        t, order = t.sort(1, descending=True)
        s["idx"], s["t"] = places.gather(1, order).to(torch.int32), t.to(dtype)
        s["idx"][torch.rand((n, k), generator=gen, device="cuda") < 0.02] = -1  # the teacher sent fewer
        s["dloss"] = torch.rand((n,), generator=gen, device="cuda") / n * (65536.0 if dtype is torch.float16 else 1.0)  # 16-bit training scales its loss
        if c["part"] == "backward":
            s["stats"] = _distill_stats(s)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _rotate(x, s):
    c = s["case"]
    turns = s["positions"].double()[:, :, None] * (s["freqs"] / (2 * math.pi))  # whole turns leave before the angle is rounded to 32 bits
    angle = ((turns - turns.round()) * (2 * math.pi)).float()[:, :, None, :]
    cos, sin = angle.cos() * s["magnitude"], angle.sin() * (-s["magnitude"] if c["back"] else s["magnitude"])
    f = x.float()
    turned, rest = f[..., : c["rot"]], f[..., c["rot"]:]
    if c["layout"] == "half":
        a, b = turned.chunk(2, -1)
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, rest], -1).to(x.dtype)


def _seen(s):
    """[batch, 1, 1, seq, seq]: whether query i sees key j; and [batch, seq, 1, 1]: whether a token is past its sequence's end."""
    c = s["case"]
    i = torch.arange(c["seq"], device="cuda")
    seen = (i[None, :] <= i[:, None]) if c["causal"] else torch.ones((c["seq"], c["seq"]), dtype=torch.bool, device="cuda")
    seen = seen[None].expand(c["batch"], -1, -1)
    past = torch.zeros((c["batch"], c["seq"]), dtype=torch.bool, device="cuda")
    if s["doc_start"] is not None:
        seen = seen & (i[None, None, :] >= s["doc_start"][:, :, None])
    if s["lens"] is not None:
        past = i[None, :] >= s["lens"][:, None]
        seen = seen & ~past[:, None, :] & ~past[:, :, None]
    return seen[:, None, None], past[:, :, None, None]


def _grouped(x, past, heads):
    """[batch, seq, h, d] in 32 bits as [batch, heads, h / heads, seq, d]; what is past the end does not count."""
    b, n, h, d = x.shape
    return x.float().masked_fill(past, 0.0).reshape(b, n, heads, h // heads, d).permute(0, 2, 3, 1, 4)


def _probabilities(s):
    c = s["case"]
    seen, past = _seen(s)
    q, k, v = (_grouped(s[n], past, c["hk"]) for n in "qkv")
    score = (q * c["d"] ** -0.5 @ k.transpose(-1, -2)).masked_fill(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top.isfinite(), top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1).flatten(1, 2)
    return p / total.clamp_min(1e-38), lse, q, k, v, past


def _ungrouped(x, like):
    return x.permute(0, 3, 1, 2, 4).flatten(2, 3).to(like.dtype)


def _attention(s):
    p, lse, q, k, v, past = _probabilities(s)
    return _ungrouped(p @ v, s["q"]), lse


def _attention_back(s):
    p, lse, q, k, v, past = _probabilities(s)
    do = _grouped(s["dout"], past, s["case"]["hk"])
    dp = do @ v.transpose(-1, -2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["case"]["d"] ** -0.5
    dq = ds @ k
    dk, dv = (x.sum(2, keepdim=True) for x in (ds.transpose(-1, -2) @ q, p.transpose(-1, -2) @ do))
    return [_ungrouped(x, s["q"]) for x in (dq, dk, dv)]


def _log_sum_exp(z):
    top = z.amax(-1, keepdim=True)
    return (top + (z - top).exp().sum(-1, keepdim=True).log()).squeeze(-1)


def _distill_stats(s):
    z = s["z"].float()
    return torch.stack([_log_sum_exp(z), _log_sum_exp(z / s["case"]["temperature"])], 1)


def _teacher(s):
    """The teacher's probabilities over what it sent: [rows, k], zero where it sent nothing; and where to look."""
    sent = s["idx"] >= 0
    t = (s["t"].float() / s["case"]["temperature"]).masked_fill(~sent, float("-inf"))
    top = t.amax(-1, keepdim=True)
    e = torch.exp(t - torch.where(top.isfinite(), top, torch.zeros_like(top)))
    return e / e.sum(-1, keepdim=True).clamp_min(1e-38), s["idx"].clamp_min(0).long()


def _distill_loss(s, stats):
    c = s["case"]
    z, mix, temp = s["z"], c["mix"], c["temperature"]
    p, at = _teacher(s)
    counted = s["labels"] != IGNORED
    ce = stats[:, 0] - z.gather(1, s["labels"].clamp_min(0)[:, None]).float()[:, 0]
    kl = (p * (p.clamp_min(1e-38).log() - z.gather(1, at).float() / temp + stats[:, 1:])).sum(-1)
    return torch.where(counted, (1 - mix) * ce + mix * temp * temp * kl, torch.zeros_like(ce))


def _distill_gradient(s, stats):
    c = s["case"]
    mix, temp = c["mix"], c["temperature"]
    p, at = _teacher(s)
    z = s["z"].float()
    sent = (s["idx"] >= 0).any(1, keepdim=True)
    counted = (s["labels"] != IGNORED)[:, None]
    g = (1 - mix) * torch.exp(z - stats[:, :1]) + mix * temp * sent * torch.exp(z / temp - stats[:, 1:])
    g.scatter_add_(1, at, -mix * temp * p)
    g.scatter_add_(1, s["labels"].clamp_min(0)[:, None], torch.full_like(g[:, :1], mix - 1))
    return torch.where(counted, g * s["dloss"][:, None], torch.zeros_like(g)).to(s["z"].dtype)


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2506_04531_b200 import step
    if c["op"] == "rope":
        if own:
            return step.rope(s["q"], s["k"], s["freqs"], positions=s["positions"], layout=c["layout"], magnitude=s["magnitude"], inverse=c["back"])
        return _rotate(s["q"], s), _rotate(s["k"], s)
    if c["op"] == "attention":
        if own:
            mask = dict(causal=c["causal"], doc_start=s["doc_start"], lens=s["lens"])
            if c["back"]:
                return step.attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], **mask)
            return step.attention_forward(s["q"], s["k"], s["v"], **mask)
        return _attention_back(s) if c["back"] else _attention(s)
    if own:
        what = dict(temperature=c["temperature"], mix=c["mix"], ignore_index=IGNORED)
        if c["part"] == "forward":
            return step.distill_forward(s["z"], s["labels"], s["idx"], s["t"], **what)
        if c["part"] == "backward":
            return step.distill_backward(s["dloss"], s["z"], s["stats"], s["labels"], s["idx"], s["t"], **what)
        return step.distill_loss_and_grad(s["z"], s["labels"], s["idx"], s["t"], s["dloss"], **what)
    if c["part"] == "backward":
        return _distill_gradient(s, s["stats"])
    stats = _distill_stats(s)
    loss = _distill_loss(s, stats)
    return (loss, stats) if c["part"] == "forward" else (loss, _distill_gradient(s, stats))


def work(case):
    c, size = case, BYTES[case["dtype"]]
    if c["op"] == "rope":
        moved = c["batch"] * c["seq"] * (c["hq"] + c["hk"]) * c["d"]
        return {"bytes": 2 * size * moved, "flops": 3 * moved * c["rot"] / c["d"]}
    if c["op"] == "attention":
        pairs = c["batch"] * c["hq"] * (c["seq"] * (c["seq"] + 1) / 2 if c["causal"] else c["seq"] ** 2)
        if c["documents"]:  # as many pairs as documents of equal lengths have, about
            pairs /= min(c["seq"], c["documents"] + 1)
        tokens = c["batch"] * c["seq"] * c["d"] * size
        if c["back"]:
            return {"bytes": tokens * (4 * c["hq"] + 4 * c["hk"]), "flops": 10 * c["d"] * pairs}
        return {"bytes": tokens * (2 * c["hq"] + 2 * c["hk"]), "flops": 4 * c["d"] * pairs}
    values, sent = c["rows"] * c["vocab"] * size, c["rows"] * c["k"] * (4 + size)
    return {"bytes": values * (1 if c["part"] == "forward" else 2) + sent, "flops": 10 * c["rows"] * c["vocab"]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        return [_exact_rope(s[n], s) for n in "qk"]
    if c["op"] == "attention":
        return _exact_attention(s)
    return _exact_distill(s)


def _exact_rope(x, s):
    """Each pair as a complex number, times magnitude e^(i angle)."""
    c, half = s["case"], s["case"]["rot"] // 2
    y = x.double().clone()
    first = torch.arange(half, device="cuda") * (1 if c["layout"] == "half" else 2)
    second = first + (half if c["layout"] == "half" else 1)
    angle = s["positions"].double()[:, :, None, None] * s["freqs"] * (-1 if c["back"] else 1)
    turned = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.full_like(angle, s["magnitude"]), angle)
    y[..., first], y[..., second] = turned.real.clone(), turned.imag.clone()
    return y


def _exact_attention(s):
    """A sequence and a head at a time, gradients by differentiating the definition."""
    c = s["case"]
    n, group = c["seq"], c["hq"] // c["hk"]
    o = torch.zeros((c["batch"], n, c["hq"], c["d"]), dtype=torch.float64, device="cuda")
    lse = torch.full((c["batch"], c["hq"], n), float("-inf"), dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(o), *(torch.zeros((c["batch"], n, c["hk"], c["d"]), dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(c["batch"]):
        end = n if s["lens"] is None else int(s["lens"][b])
        if not end:
            continue
        low = torch.zeros(end, dtype=torch.long, device="cuda") if s["doc_start"] is None else s["doc_start"][b, :end].long()
        j = torch.arange(end, device="cuda")
        hidden = j[None, :] < low[:, None]
        if c["causal"]:
            hidden = hidden | (j[None, :] > j[:, None])
        for h in range(c["hq"]):
            one = [s["q"][b, :end, h], s["k"][b, :end, h // group], s["v"][b, :end, h // group]]
            q, k, v = (t.double().clone().requires_grad_(c["back"]) for t in one)
            score = (q @ k.T / math.sqrt(c["d"])).masked_fill(hidden, float("-inf"))
            out = torch.softmax(score, 1) @ v
            if c["back"]:
                out.backward(s["dout"][b, :end, h].double())
                dq[b, :end, h] = q.grad
                dk[b, :end, h // group] += k.grad
                dv[b, :end, h // group] += v.grad
            else:
                o[b, :end, h] = out
                lse[b, h, :end] = torch.logsumexp(score, 1)
    return [dq, dk, dv] if c["back"] else [o, lse]


def _exact_distill(s):
    """Some rows at a time, the gradient by differentiating the loss."""
    c, temp, mix = s["case"], s["case"]["temperature"], s["case"]["mix"]
    losses, stats, grads = [], [], []
    for at in range(0, c["rows"], 512):
        part = slice(at, at + 512)
        z = s["z"][part].double().clone().requires_grad_(c["part"] != "forward")
        label, idx = s["labels"][part], s["idx"][part]
        dense = torch.full_like(z, float("-inf")).detach()
        row, col = (idx >= 0).nonzero(as_tuple=True)
        dense[row, idx[row, col].long()] = s["t"][part].double()[row, col] / temp
        p = torch.softmax(dense, 1).nan_to_num(0.0)
        soft, hard = torch.log_softmax(z / temp, 1), torch.log_softmax(z, 1)
        kl = torch.special.xlogy(p, p).sum(1) - (p * soft).sum(1)
        ce = -hard.gather(1, label.clamp_min(0)[:, None])[:, 0]
        loss = ((1 - mix) * ce + mix * temp ** 2 * kl) * (label != IGNORED)
        if c["part"] != "forward":
            (loss * s["dloss"][part].double()).sum().backward()
            grads.append(z.grad.to(torch.float32 if c["dtype"] != "f32" else torch.float64))
        losses.append(loss.detach())
        stats.append(torch.stack([torch.logsumexp(z.detach(), 1), torch.logsumexp(z.detach() / temp, 1)], 1))
    if c["part"] == "forward":
        return torch.cat(losses), torch.cat(stats)
    return torch.cat(grads) if c["part"] == "backward" else (torch.cat(losses), torch.cat(grads))
