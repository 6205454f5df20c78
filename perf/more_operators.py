"""What a local step does around its matrix products, as it is measured: the embedding and its gradient, root-mean-square norms
with the residual's addition (their gradient, and their result in 8 bits), and the gradients' global norm with clipping.

Sizes: widths, the vocabulary and the tensors of a model follow the decoder layouts of this repository (d = 512 to 2048, V = 50304,
76 to 292 tensors, sequences of 2048 tokens) and go on from there to odd and ragged ones."""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
RATE = 0.01
LARGEST = 448.0  # of the 8-bit type with 4 bits of exponent


def listed():
    return [
        # the first thing a local step does: 32 sequences of tokens, from 32-bit master parameters to 16-bit activations
        dict(name="embed_160m", op="embed", back=False, dtype="bf16", wtype="f32", vocab=50304, d=768, batch=32, seq=2048, wide=True, padded=False, scaled=False, onto=False),
        # one token for each of eight sequences: latency
        dict(name="embed_token", op="embed", back=False, dtype="bf16", wtype="bf16", vocab=50304, d=2048, batch=8, seq=1, wide=True, padded=False, scaled=True, onto=False),
        # the last thing its backward pass does: the gradient of the 32-bit master parameters
        dict(name="embed_160m_back", op="embed", back=True, dtype="bf16", wtype="f32", vocab=50304, d=768, batch=32, seq=2048, wide=True, padded=False, scaled=False, onto=False),
        # ragged sequences filled up with one token, an odd vocabulary and width, 16 bits throughout
        dict(name="embed_padded_back_f16", op="embed", back=True, dtype="f16", wtype="f16", vocab=32003, d=1021, batch=7, seq=1021, wide=False, padded=True, scaled=True, onto=False),
        # the norm before each half of a layer of the 160m layout: the half before it is added to the residual on the way
        dict(name="norm_160m", op="norm", part="forward", dtype="bf16", wtype="f32", batch=32, seq=2048, heads=0, d=768, residual=True, packed=False, group=0),
        # its backward pass at the 1p4b layout's width, with the gradient that comes down the residual
        dict(name="norm_1p4b_back", op="norm", part="backward", dtype="bf16", wtype="bf16", batch=8, seq=2048, heads=0, d=2048, residual=True, packed=False, group=0),
        # the same norm in front of a product in 8 bits, a scale for every 128 elements
        dict(name="norm_1p4b_quantized", op="norm", part="quantized", dtype="bf16", wtype="bf16", batch=8, seq=2048, heads=0, d=2048, residual=True, packed=False, group=128),
        # one token for each of eight sequences: latency
        dict(name="norm_token", op="norm", part="forward", dtype="bf16", wtype="bf16", batch=8, seq=1, heads=0, d=2048, residual=True, packed=False, group=0),
        # norms of the heads of queries, as views of a fused projection, in 32 bits and of an odd number of tokens: their way back
        dict(name="norm_heads_back_f32", op="norm", part="backward", dtype="f32", wtype="f32", batch=3, seq=1021, heads=10, d=80, residual=False, packed=True, group=0),
        # a step of local SGD on the 160m layout's 148 tensors, the gradients clipped to a norm of 1
        dict(name="grads_160m_step", op="grads", part="step", dtype="f32", layers=12, width=768, vocab=50304, before=3.0),
        # 16-bit gradients of the 70m layout, clipped on their way to the 32-bit vector that further micro-batches are added to
        dict(name="grads_70m_clip", op="grads", part="clip", dtype="bf16", layers=6, width=512, vocab=50304, before=3.0),
        # the norm alone of a small model of odd width, for the log: latency
        dict(name="grads_small_norm", op="grads", part="norm", dtype="f16", layers=2, width=81, vocab=1009, before=0.5),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["embed", "embed", "norm", "norm", "norm", "grads"])
    if op == "embed":
        dtype = rng.choice(list(TYPES))
        wtype, back = rng.choice(["f32", dtype]), rng.random() < 0.6
        d, vocab = rng.choice([_spread(rng, 16, 4096), _spread(rng, 2, 512) * 8]), _spread(rng, 500, 200000)
        vocab = max(1, min(vocab, 200_000_000 // (d * BYTES[wtype])))
        seq = _spread(rng, 1, 8192)
        batch = max(1, min(_spread(rng, 1, 64), 120_000_000 // (d * BYTES[dtype] * seq), 65536 // seq))
        return dict(op=op, back=back, dtype=dtype, wtype=wtype, vocab=vocab, d=d, batch=batch, seq=seq, wide=rng.random() < 0.5, padded=rng.random() < 0.4, scaled=rng.random() < 0.4,
                    onto=back and wtype == "f32" and rng.random() < 0.4)
    if op == "norm":
        dtype, part = rng.choice(list(TYPES)), rng.choice(["forward", "backward", "quantized"])
        heads = rng.choice([0, 0, 1, 5, 12, 16])
        d = rng.choice([64, 80, 128, 256, _spread(rng, 8, 256)]) if heads else rng.choice([_spread(rng, 32, 16384), _spread(rng, 8, 1024) * 16])
        seq = _spread(rng, 1, 8192)
        batch = max(1, min(_spread(rng, 1, 64), 400_000_000 // (4 * BYTES[dtype] * d * max(1, heads) * seq)))
        return dict(op=op, part=part, dtype=dtype, wtype=rng.choice(["f32", dtype]), batch=batch, seq=seq, heads=heads, d=d, residual=rng.random() < 0.6,
                    packed=heads > 0 and rng.random() < 0.6, group=rng.choice([0, 32, 128]) if part == "quantized" else 0)
    width = rng.choice([_spread(rng, 64, 1024), _spread(rng, 4, 64) * 16])
    layers, vocab = _spread(rng, 1, 24), _spread(rng, 500, 60000)
    layers = max(1, min(layers, (150_000_000 - 2 * vocab * width) // (12 * width * width + 13 * width)))
    return dict(op=op, part=rng.choice(["step", "clip", "clip", "norm"]), dtype=rng.choice(list(TYPES)), layers=layers, width=width, vocab=vocab, before=rng.choice([0.5, 3.0, 40.0]))


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(shape, gen, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _share(c):
    """How often each token comes: as the words of a language do, the frequent ones first."""
    return 1.0 / (torch.arange(c["vocab"], dtype=torch.float64) + 3.0)


def _tokens(c, gen):
    upto = _share(c).cumsum(0).cuda()
    at = torch.rand((c["batch"], c["seq"]), generator=gen, device="cuda", dtype=torch.float64) * upto[-1]
    tokens = torch.searchsorted(upto, at).clamp_max(c["vocab"] - 1)
    if c["padded"]:
        lens = torch.randint(1, c["seq"] + 1, (c["batch"], 1), generator=gen, device="cuda")
        tokens = torch.where(torch.arange(c["seq"], device="cuda") < lens, tokens, torch.full_like(tokens, c["vocab"] // 2))
    return tokens if c["wide"] else tokens.to(torch.int32)


def _rows(c, gen, n):
    """`n` tensors [batch, seq, d] or [batch, seq, heads, d]; where the case is packed, views of one projection's output."""
    dtype = TYPES[c["dtype"]]
    if c["packed"]:
        every = _normal((c["batch"], c["seq"], c["heads"], max(3, n), c["d"]), gen, dtype, 1.5)
        return [every[:, :, :, i] for i in range(n)]
    shape = (c["batch"], c["seq"], c["heads"], c["d"]) if c["heads"] else (c["batch"], c["seq"], c["d"])
    return [_normal(shape, gen, dtype, 1.5) for _ in range(n)]


def _shapes(c):
    d, every = c["width"], [(c["vocab"], c["width"])]
    for _ in range(c["layers"]):
        every += [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (4 * d, d), (4 * d,), (d, 4 * d), (d,)]
    return every + [(d,), (d,), (c["vocab"], d)]


def _views(flat, shapes):
    return [x.view(s) for x, s in zip(torch.split(flat, [math.prod(s) for s in shapes]), shapes)]


def prepare(case, seed):
    c, gen = case, _generator(seed)
    dtype, s = TYPES[c["dtype"]], {"case": c}
    if c["op"] == "embed":
        s["tokens"] = _tokens(c, gen)
        s["scale"] = math.sqrt(c["d"]) if c["scaled"] else 1.0
        if c["back"]:
            s["dout"] = _normal((c["batch"], c["seq"], c["d"]), gen, dtype, 0.1)
            if c["onto"]:  # the gradient of the micro-batches before
                s["grad"] = _normal((c["vocab"], c["d"]), gen, TYPES[c["wtype"]], 0.1)
        else:
            s["weight"] = _normal((c["vocab"], c["d"]), gen, TYPES[c["wtype"]], 0.02)
    elif c["op"] == "norm":
        s["weight"] = 1 + _normal((c["d"],), gen, TYPES[c["wtype"]], 0.1)
        if c["part"] == "backward":  # what the forward pass left behind, and the gradients of what it returned
            s["summed"], = _rows(c, gen, 1)
            s["rstd"] = (s["summed"].double().square().mean(-1) + EPS).rsqrt().float()
            s["dy"] = _normal(s["summed"].shape, gen, dtype)
            s["dsummed"] = _normal(s["summed"].shape, gen, dtype) if c["residual"] else None
        else:
            s["x"], s["residual"] = (_rows(c, gen, 2) if c["residual"] else (*_rows(c, gen, 1), None))
    else:
        shapes = _shapes(c)
        total = sum(math.prod(d) for d in shapes)
        # tensors of their own, as a backward pass leaves them; their norm is about `before`, and what is clipped is clipped to 1
        s["grads"] = [_normal(d, gen, dtype, c["before"] / math.sqrt(total)) for d in shapes]
        if c["part"] == "clip":
            s["flat"] = torch.zeros(total, device="cuda")
        elif c["part"] == "step":
            s["flat"] = _normal((total,), gen, torch.float32, 0.02)
        if c["part"] != "norm":
            s["views"] = _views(s["flat"], shapes)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _embedding(s):
    return (s["weight"][s["tokens"].long()].float() * s["scale"]).to(TYPES[s["case"]["dtype"]])


def _embedding_back(s):
    c = s["case"]
    tokens, dout = s["tokens"].reshape(-1).long(), s["dout"].reshape(-1, c["d"]).float() * s["scale"]
    grad = s["grad"] if c["onto"] else torch.zeros((c["vocab"], c["d"]), device="cuda")
    return grad.index_add_(0, tokens, dout).to(TYPES[c["wtype"]])


def _norm(s):
    """The result in 32 bits, the sum that the next residual is, and one over the root of the mean square."""
    x = s["x"].float()
    if s["residual"] is not None:
        x = x + s["residual"].float()
    rstd = (x.square().mean(-1) + EPS).rsqrt()
    return x * rstd[..., None] * s["weight"].float(), x.to(s["x"].dtype), rstd


def _quantized(y, group):
    """y in 8 bits and the scales: what a group's largest is divided by to become the largest 8-bit value."""
    n, d = (group or y.shape[-1]), y.shape[-1]
    pieces = torch.cat([y, y.new_zeros((*y.shape[:-1], -d % n))], -1).unflatten(-1, (-1, n))
    scale = (pieces.abs().amax(-1) / LARGEST).clamp_min(2.0 ** -126)
    return (pieces / scale[..., None]).flatten(-2)[..., :d].to(torch.float8_e4m3fn), scale


def _norm_back(s):
    x, dy, rstd = s["summed"].float(), s["dy"].float(), s["rstd"][..., None]
    unit, g = x * rstd, dy * s["weight"].float()
    dx = rstd * (g - unit * (g * unit).mean(-1, keepdim=True))
    if s["dsummed"] is not None:
        dx = dx + s["dsummed"].float()
    return dx.to(s["dy"].dtype), (dy * unit).flatten(0, -2).sum(0).to(s["weight"].dtype)


def _global_norm(grads):
    return torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()


def _clipped(s):
    norm = _global_norm(s["grads"])
    factor = (1.0 / norm).clamp_max(1.0)
    if s["case"]["part"] == "clip":
        [v.copy_(g.float() * factor) for v, g in zip(s["views"], s["grads"])]
    elif s["case"]["part"] == "step":
        [v.copy_(v - RATE * factor * g.float()) for v, g in zip(s["views"], s["grads"])]
    else:
        return norm
    return norm, s["flat"]


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2506_04531_b200 import step
    if c["op"] == "embed":
        if c["back"]:
            if own:
                return step.embedding_backward(s["dout"], s["tokens"], c["vocab"], scale=s["scale"], dtype=TYPES[c["wtype"]], out=s["grad"] if c["onto"] else None, accumulate=c["onto"])
            return _embedding_back(s)
        return step.embedding_forward(s["weight"], s["tokens"], scale=s["scale"], dtype=TYPES[c["dtype"]]) if own else _embedding(s)
    if c["op"] == "norm":
        if c["part"] == "backward":
            return step.rms_norm_backward(s["dy"], s["summed"], s["weight"], s["rstd"], dsummed=s["dsummed"]) if own else _norm_back(s)
        if own:
            if c["part"] == "quantized":
                y = step.rms_norm_quantized(s["x"], s["weight"], residual=s["residual"], eps=EPS, group=c["group"])
            else:
                y = step.rms_norm_forward(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        else:
            y = _norm(s)
            y = (*_quantized(y[0], c["group"]), *y[1:]) if c["part"] == "quantized" else (y[0].to(s["x"].dtype), *y[1:])
        return y if c["residual"] else (*y[:-2], y[-1])  # without a residual the sum is the input itself
    if own:
        if c["part"] == "norm":
            return step.grad_norm(s["grads"])
        if c["part"] == "clip":
            return step.clip_grads(s["grads"], 1.0, out=s["views"]), s["flat"]
        return step.sgd_step(s["views"], s["grads"], RATE, max_norm=1.0), s["flat"]
    return _clipped(s)


def work(case):
    c, size = case, BYTES[case["dtype"]]
    if c["op"] == "embed":
        n, p = c["batch"] * c["seq"], _share(c)
        # rows of the table that some token asks for, as many as are expected
        met = float((1 - (-n * p / p.sum()).exp()).sum())
        moved, index = n * c["d"], n * (8 if c["wide"] else 4)
        table = BYTES[c["wtype"]] * c["d"] * (met if not c["back"] else 2 * met if c["onto"] else c["vocab"])
        return {"bytes": size * moved + table + index, "flops": (2 if c["back"] else 1) * moved}
    if c["op"] == "norm":
        rows, d = c["batch"] * c["seq"] * max(1, c["heads"]), c["d"]
        if c["part"] == "backward":
            return {"bytes": rows * (d * size * (4 if c["residual"] else 3) + 4) + 2 * d * BYTES[c["wtype"]], "flops": 10 * rows * d}
        moved = size * (3 if c["residual"] else 1) + (1 if c["part"] == "quantized" else size)
        scales = 4 * -(-d // (c["group"] or d)) if c["part"] == "quantized" else 0
        return {"bytes": rows * (d * moved + 4 + scales) + d * BYTES[c["wtype"]], "flops": 5 * rows * d}
    total = sum(math.prod(d) for d in _shapes(c))
    return {"bytes": total * (size + {"norm": 0, "clip": 4, "step": 8}[c["part"]]), "flops": total * (2 if c["part"] == "norm" else 4)}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "embed":
        return _exact_embedding(s)
    if c["op"] == "norm":
        return _exact_norm(s)
    return _exact_grads(s)


def _exact_embedding(s):
    """The table's rows by the tokens, and the gradient by differentiating a weighted sum of them."""
    c, flat = s["case"], s["tokens"].long().flatten()
    if not c["back"]:
        return torch.index_select(s["weight"].double(), 0, flat).mul(s["scale"]).view(c["batch"], c["seq"], c["d"])
    table = torch.zeros((c["vocab"], c["d"]), dtype=torch.float64, device="cuda", requires_grad=True)
    part = 1 << 13
    for at in range(0, flat.numel(), part):
        torch.nn.functional.embedding(flat[at:at + part], table).backward(s["dout"].view(-1, c["d"])[at:at + part].double() * s["scale"])
    return table.grad + s["grad"].double() if c["onto"] else table.grad


def _exact_norm(s):
    """Some rows at a time: each over its length times the root of d, times the weight; gradients by differentiating that."""
    c, d, back = s["case"], s["case"]["d"], s["case"]["part"] == "backward"
    if back:
        rows = [s[n].reshape(-1, d) for n in ("summed", "dy")]
        dsummed = None if s["dsummed"] is None else s["dsummed"].reshape(-1, d)
    else:
        rows = [s[n].reshape(-1, d) for n in ("x", "residual") if s[n] is not None]
    shape = (s["summed"] if back else s["x"]).shape
    w = s["weight"].double().requires_grad_(back)
    got, part = [], max(1, (1 << 24) // d)
    for at in range(0, rows[0].shape[0], part):
        one = [r[at:at + part].double() for r in rows]
        x = (one[0] if back or len(one) == 1 else one[0] + one[1]).requires_grad_(back)
        length = torch.sqrt(torch.linalg.vector_norm(x, dim=1).square() + d * EPS)
        y = x / length[:, None] * math.sqrt(d) * w
        if back:
            y.backward(one[1])
            got.append((x.grad if dsummed is None else x.grad + dsummed[at:at + part].double(),))
        elif c["part"] == "quantized":
            n = c["group"] or d
            top = torch.stack([y[:, i:i + n].abs().amax(1) for i in range(0, d, n)], 1) / LARGEST
            got.append((y / torch.repeat_interleave(top, n, 1)[:, :d], top, x, math.sqrt(d) / length))
        else:
            got.append((y, x, math.sqrt(d) / length))
    got = [torch.cat(v) for v in zip(*got)]
    if back:
        return got[0].view(shape), w.grad
    if not c["residual"]:
        del got[-2]
    return [v.view(*shape[:-1], *v.shape[1:]) for v in got]


def _exact_grads(s):
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"]))
    if s["case"]["part"] == "norm":
        return torch.tensor(norm, dtype=torch.float64)
    clipped = torch.cat([g.double().flatten() for g in s["grads"]]) / max(1.0, norm)
    return torch.tensor(norm, dtype=torch.float64), clipped if s["case"]["part"] == "clip" else s["flat"].double() - RATE * clipped
