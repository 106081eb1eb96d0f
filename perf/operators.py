"""Language-model operators whose time and results are measured.

The operators are the work of a GPT training step around its matrices: the embedding lookup with
scaling and its gradient, the norm and rotation of queries and keys with its gradient, and the loss
of distillation from a teacher's top logits with its gradient.  A case is one call of one of them.
`prepare` makes what a training loop has in hand before the call, `run` makes the call (where `own`
is false: the same in elementary torch operations, in 32 bits), `exact` computes it in 64 bits.

Inputs follow what the operators meet in training: tokens drawn with the 1/rank law of text, with
some padding among them; activations of unit scale with a few large features; logits with a peak
near the teacher's entries; rows that a mask leaves out, entries and labels that are absent.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}
EPS = 1e-6  # of the norms
THETA = 10000.0
ROWS_64 = 1 << 25  # elements that `exact` holds in 64 bits at a time


# ------------------------------------------------------------------------------ the cases ---
def listed():
    return [
        # 64 tokens of one short prompt, bf16 copy of the table: launch and latency
        dict(name="lookup_prompt", op="lookup", tokens=64, vocab=32000, dim=768, table="bf16", out="bf16"),
        # a micro-batch of 32 sequences of 1024 tokens, 1.3B-parameter GPT (d = 2048), fp32 parameters
        dict(name="lookup_train", op="lookup", tokens=32768, vocab=50001, dim=2048, table="fp32", out="bf16"),
        # gradient of one odd-length sequence, 160M-parameter GPT (d = 768): most rows of the table get none
        dict(name="embed_grad_sequence", op="embed_grad", tokens=1023, vocab=32000, dim=768, grad="bf16", out="fp32"),
        # gradient of the training micro-batch: tokens that come thousands of times
        dict(name="embed_grad_train", op="embed_grad", tokens=32768, vocab=50001, dim=2048, grad="bf16", out="fp32"),
        # one new token for each of 16 sequences, grouped heads, positions anywhere in a long context
        dict(name="qk_token", op="qk", batch=16, seq=1, heads=16, kv_heads=4, head_dim=128, rotary=128, dtype="bf16",
             far=131072, layout="packed"),
        # 32 sequences of 1024 tokens of a 1.3B-parameter GPT, q and k inside the packed projection
        dict(name="qk_train", op="qk", batch=32, seq=1024, heads=16, kv_heads=16, head_dim=128, rotary=128, dtype="bf16",
             far=0, layout="packed"),
        # gradient, fp32, 160M-parameter GPT, an odd length, half of each head rotated, heads before tokens
        dict(name="qk_grad_odd", op="qk_grad", batch=3, seq=701, heads=12, kv_heads=12, head_dim=64, rotary=32,
             dtype="fp32", far=0, layout="heads_first"),
        # gradient of the training micro-batch
        dict(name="qk_grad_train", op="qk_grad", batch=32, seq=1024, heads=16, kv_heads=16, head_dim=128, rotary=128,
             dtype="bf16", far=0, layout="packed"),
        # loss of a handful of positions, as an evaluation on a short text
        dict(name="distill_short", op="distill", rows=9, vocab=32000, top=16, dtype="bf16", hard=0.0, temperature=2.0),
        # loss of four sequences of 1024 tokens, fp32 logits, odd vocabulary
        dict(name="distill_eval", op="distill", rows=4096, vocab=50001, top=64, dtype="fp32", hard=0.5, temperature=1.0),
        # loss and gradient of a part of a sequence, mixed with the hard labels, rows at odd addresses
        dict(name="distill_grad_odd", op="distill_grad", rows=509, vocab=50001, top=33, dtype="bf16", hard=0.3,
             temperature=1.5),
        # loss and gradient of a micro-batch of 8 sequences of 1024 tokens
        dict(name="distill_grad_train", op="distill_grad", rows=8192, vocab=50001, top=128, dtype="bf16", hard=0.0,
             temperature=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "embed_grad", "qk", "qk_grad", "distill", "distill_grad"])
    if op in ("lookup", "embed_grad"):
        c = dict(op=op, tokens=_log(rng, 1, 65536), vocab=_log(rng, 1000, 131072),
                 dim=rng.choice([64, 320, 768, 771, 1000, 1024, 1536, 2048, 2050]))
        if op == "lookup":
            c.update(table=rng.choice(["bf16", "fp32"]), out=rng.choice(["bf16", "fp32"]))
        else:
            c.update(grad=rng.choice(["bf16", "fp32"]), out=rng.choice(["fp32", "fp32", "bf16"]))
        while c["tokens"] * c["dim"] > 32768 * 2048 or c["vocab"] * c["dim"] > 50001 * 2048:
            c["tokens"], c["vocab"] = c["tokens"] * 2 // 3, c["vocab"] * 2 // 3
        return c
    if op in ("qk", "qk_grad"):
        head_dim = rng.choice([32, 64, 80, 96, 128, 128, 256])
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        c = dict(op=op, batch=_log(rng, 1, 32), seq=1 if rng.random() < 0.25 else _log(rng, 2, 8192),
                 heads=kv_heads * rng.choice([1, 2, 4]), kv_heads=kv_heads, head_dim=head_dim,
                 rotary=rng.choice([head_dim, head_dim, head_dim // 2, 2 * (head_dim // 5)]),
                 dtype=rng.choice(["bf16", "bf16", "fp32"]), far=rng.choice([0, 0, 131072]),
                 layout=rng.choice(["packed", "heads_first"]))
        while c["batch"] * c["seq"] * (c["heads"] + kv_heads) * head_dim * BYTES[c["dtype"]] > 32768 * 32 * 128 * 2:
            c["batch"], c["seq"] = max(1, c["batch"] * 2 // 3), max(1, c["seq"] * 2 // 3)
        return c
    c = dict(op=op, rows=_log(rng, 1, 8192), vocab=_log(rng, 500, 131072), top=_log(rng, 1, 256),
             dtype=rng.choice(["bf16", "bf16", "fp32"]), hard=rng.choice([0.0, 0.0, 0.25, 1.0]),
             temperature=rng.choice([1.0, 2.0, 3.5]))
    c["rows"] = max(1, min(c["rows"], 8192 * 50001 * 2 // (c["vocab"] * BYTES[c["dtype"]])))
    return c


# ----------------------------------------------------------------------------- the inputs ---
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _embed_inputs(case, g):
    n, v, d = case["tokens"], case["vocab"], case["dim"]
    tokens = (torch.exp(_rand(g, n).double() * math.log(v)).floor().long() - 1).clamp_(0, v - 1)
    tokens[_rand(g, n) < 0.03] = -1  # padding
    s = dict(tokens=tokens, scale=math.sqrt(d))
    if case["op"] == "lookup":
        s["table"] = (_randn(g, v, d) * 0.02).to(DTYPES[case["table"]])
    else:
        s["grad"] = (_randn(g, n, d) * 1e-3).to(DTYPES[case["grad"]])
    return s


def _heads(g, case, heads, into=None):
    """[batch, seq, heads, head_dim] of unit scale with a few large features, in the case's layout."""
    b, t, d = case["batch"], case["seq"], case["head_dim"]
    x = _randn(g, b, t, heads, d) * (1 + 4 * (_rand(g, d) < 0.05).float())
    x = x.to(DTYPES[case["dtype"]])
    if into is not None:
        into.copy_(x)
        return into
    return x.transpose(1, 2).contiguous().transpose(1, 2) if case["layout"] == "heads_first" else x


def _qk_inputs(case, g):
    b, t, hq, hk, d = case["batch"], case["seq"], case["heads"], case["kv_heads"], case["head_dim"]
    if case["layout"] == "packed":  # views of the projection's output, the values' part untouched
        qkv = torch.zeros(b, t, hq + 2 * hk, d, dtype=DTYPES[case["dtype"]], device="cuda")
        q, k = _heads(g, case, hq, qkv[:, :, :hq]), _heads(g, case, hk, qkv[:, :, hq:hq + hk])
    else:
        q, k = _heads(g, case, hq), _heads(g, case, hk)
    start = (_rand(g, b) * max(1, case["far"] - t)).long() if case["far"] else torch.zeros(b, dtype=torch.long, device="cuda")
    s = dict(q=q, k=k, wq=1 + 0.1 * _randn(g, d), wk=1 + 0.1 * _randn(g, d),
             positions=start[:, None] + torch.arange(t, device="cuda")[None])
    if case["op"] == "qk_grad":
        s["gq"], s["gk"] = _heads(g, dict(case, layout="heads_first"), hq), _heads(g, dict(case, layout="heads_first"), hk)
    return s


def _angles(case, positions):
    """cos, sin of the rotation, [batch, seq, rotary / 2], in 64 bits."""
    r = case["rotary"]
    a = positions.double()[..., None] * THETA ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    return a.cos(), a.sin()


def _distill_inputs(case, g):
    n, v, k = case["rows"], case["vocab"], min(case["top"], case["vocab"])
    # distinct entries of each row: an arithmetic progression from a random start
    step = 1 + (_rand(g, n, 1) * max(1, v // k - 1)).long()
    ids = ((_rand(g, n, 1) * v).long() + step * torch.arange(k, device="cuda")[None]) % v
    teacher = 9 - torch.cumsum(_rand(g, n, k) * (8.0 / k), 1)  # descending, as a top-k gives them
    logits = torch.empty(n, v, dtype=DTYPES[case["dtype"]], device="cuda")
    rows = max(1, ROWS_64 // v)
    for i in range(0, n, rows):
        z = _randn(g, min(rows, n - i), v) * 2
        z.scatter_add_(1, ids[i:i + rows], teacher[i:i + rows] * 0.8)
        logits[i:i + rows] = z.to(logits.dtype)
    labels = ids[:, 0].clone()
    labels[_rand(g, n) < 0.05] = -100  # no label
    ids[:, k // 2:][_rand(g, n, k - k // 2) < 0.2] = -1  # shorter lists
    keep = (_rand(g, n) >= 0.05).float()  # positions that the mask leaves out
    s = dict(logits=logits, ids=ids, teacher=teacher, weights=keep / keep.sum().clamp(min=1))
    s["labels"] = labels if case["hard"] > 0 else None
    return s


def _inputs(case, seed):
    g = _generator(seed)
    return {"lookup": _embed_inputs, "embed_grad": _embed_inputs, "qk": _qk_inputs, "qk_grad": _qk_inputs,
            "distill": _distill_inputs, "distill_grad": _distill_inputs}[case["op"]](case, g)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:  # the plans that a training loop makes once
        import paper_2512_13728_gb300 as cd

        s["cd"] = cd
        if case["op"] in ("lookup", "embed_grad"):
            s["plan"] = cd.EmbedPlan(case["vocab"], case["dim"], case["tokens"])
        elif case["op"] in ("qk", "qk_grad"):
            s["plan"] = cd.QKNormPlan(case["head_dim"], case["rotary"], theta=THETA, eps=EPS)
    elif case["op"] in ("qk", "qk_grad"):  # the tables that one keeps instead
        s["cos"], s["sin"] = (a.float() for a in _angles(case, s["positions"]))
    return s


# ------------------------------------------------------------------------------ one call ---
def run(s):
    return (_run_own if own else _run_plain)(s, s["case"])


def _run_own(s, case):
    op = case["op"]
    if op == "lookup":
        return s["plan"].lookup(s["tokens"], s["table"], scale=s["scale"], dtype=DTYPES[case["out"]])
    if op == "embed_grad":
        return s["plan"].gradient(s["tokens"], s["grad"], scale=s["scale"], dtype=DTYPES[case["out"]])
    if op == "qk":
        return s["plan"].forward(s["q"], s["k"], s["wq"], s["wk"], s["positions"])
    if op == "qk_grad":
        return s["plan"].backward(s["gq"], s["gk"], s["q"], s["k"], s["wq"], s["wk"], s["positions"])
    f = s["cd"].distill_loss if op == "distill" else s["cd"].distill_loss_grad
    return f(s["logits"], s["ids"], s["teacher"], temperature=case["temperature"], labels=s["labels"],
             hard=case["hard"], weights=s["weights"])


def _run_plain(s, case):
    op = case["op"]
    if op == "lookup":
        t = s["tokens"]
        rows = s["table"][t.clamp(min=0)].float() * s["scale"]
        return torch.where((t >= 0)[:, None], rows, 0.0).to(DTYPES[case["out"]])
    if op == "embed_grad":
        t = s["tokens"]
        rows = torch.where((t >= 0)[:, None], s["grad"].float() * s["scale"], 0.0)
        out = torch.zeros(case["vocab"], case["dim"], device="cuda")
        return out.index_add_(0, t.clamp(min=0), rows).to(DTYPES[case["out"]])
    if op == "qk":
        return tuple(_norm_rotate(x, w, s["cos"], s["sin"]).to(x.dtype) for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])))
    if op == "qk_grad":
        dq, dwq = _norm_rotate_grad(s["gq"], s["q"], s["wq"], s["cos"], s["sin"])
        dk, dwk = _norm_rotate_grad(s["gk"], s["k"], s["wk"], s["cos"], s["sin"])
        return dq.to(s["q"].dtype), dk.to(s["k"].dtype), dwq, dwk
    return _distill_plain(s, case, op == "distill_grad")


def _rotate(x, cos, sin):
    """The first 2 * cos.shape[-1] elements of each head as pairs (j, j + half), rotated."""
    h = cos.shape[-1]
    a, b, rest = x[..., :h], x[..., h:2 * h], x[..., 2 * h:]
    cos, sin = cos[..., None, :], sin[..., None, :]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _norm_rotate(x, w, cos, sin):
    x = x.float()
    return _rotate(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w, cos, sin)


def _norm_rotate_grad(g, x, w, cos, sin):
    x, g = x.float(), _rotate(g.float(), cos, -sin)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n, u = x * r, g * w
    return r * (u - n * (u * n).mean(-1, keepdim=True)), (g * n).sum((0, 1, 2))


def _distill_plain(s, case, with_grad):
    z, t, h = s["logits"].float(), case["temperature"], case["hard"]
    v = z.shape[1]
    w, ids = s["weights"], s["ids"]
    there = (ids >= 0) & (s["teacher"] > -math.inf)
    e = torch.exp((s["teacher"] - s["teacher"].amax(1, keepdim=True)) / t) * there
    p = e / e.sum(1, keepdim=True).clamp(min=1e-30)
    at = ids.clamp(min=0)
    top = z.amax(1, keepdim=True)
    q = torch.exp((z - top) / t)
    total = q.sum(1, keepdim=True)
    logq = (z.gather(1, at) - top) / t - total.log()
    loss = (1 - h) * t * t * torch.where(p > 0, p * (p.log() - logq), 0.0).sum(1)
    grad = None
    if with_grad:
        grad = (q / total * there.any(1, keepdim=True)).scatter_add_(1, at, -p) * ((1 - h) * t)
    if h > 0:
        y, has = s["labels"].clamp(min=0)[:, None], (s["labels"] >= 0)[:, None]
        q = torch.exp(z - top)
        total = q.sum(1, keepdim=True)
        loss = loss + h * torch.where(has, total.log() - (z.gather(1, y) - top), 0.0)[:, 0]
        if with_grad:
            grad = grad + ((q / total).scatter_add_(1, y, -torch.ones_like(total)) * has) * h
    loss = torch.where(w > 0, loss * w, 0.0)
    return (loss, (grad * w[:, None]).to(s["logits"].dtype)) if with_grad else loss


# ------------------------------------------------------------------------------ 64 bits ---
def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "lookup":
        out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device="cuda")
        real = s["tokens"] >= 0
        out[real] = torch.nn.functional.embedding(s["tokens"][real], s["table"]).double() * s["scale"]
        return out
    if op == "embed_grad":  # differences of running sums over the tokens' order
        order = torch.argsort(s["tokens"], stable=True)
        sums = torch.zeros(case["tokens"] + 1, case["dim"], dtype=torch.float64, device="cuda")
        torch.cumsum(s["grad"][order].double(), 0, out=sums[1:])
        ends = torch.searchsorted(s["tokens"][order], torch.arange(case["vocab"] + 1, device="cuda"))
        return (sums[ends[1:]] - sums[ends[:-1]]) * s["scale"]
    if op in ("qk", "qk_grad"):
        # pairs as complex numbers
        cos, sin = _angles(case, s["positions"])
        turn = torch.complex(cos, sin)[:, :, None]
        half = case["rotary"] // 2
        out, weights = [], []
        for name in ("q", "k"):
            x, w = s[name].double(), s["w" + name].double()
            norm = torch.sqrt((x ** 2).sum(-1, keepdim=True) / case["head_dim"] + EPS)
            if op == "qk":
                u = x / norm * w
                pairs = torch.complex(u[..., :half], u[..., half:2 * half]) * turn
                out.append(torch.cat([pairs.real, pairs.imag, u[..., 2 * half:]], -1))
            else:
                g = s["g" + name].double()
                pairs = torch.complex(g[..., :half].contiguous(), g[..., half:2 * half].contiguous()) * turn.conj()
                gu = torch.cat([pairs.real, pairs.imag, g[..., 2 * half:]], -1)
                weights.append((gu * x / norm).flatten(0, 2).sum(0))
                gx = gu * w / norm
                out.append(gx - x * ((gx * x).sum(-1, keepdim=True) / (case["head_dim"] * norm ** 2)))
        return tuple(out + weights)
    t, h, n, v = case["temperature"], case["hard"], case["rows"], case["vocab"]
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    grad = torch.zeros(n, v, dtype=torch.float64, device="cuda") if op == "distill_grad" else None
    rows = max(1, ROWS_64 // v)
    for i in range(0, n, rows):
        r = slice(i, i + rows)
        z, w, ids = s["logits"][r].double(), s["weights"][r].double(), s["ids"][r]
        teacher = s["teacher"][r].double().masked_fill(ids < 0, -math.inf)
        some = torch.isfinite(teacher).any(1)
        logp = torch.log_softmax(torch.where(some[:, None], teacher, 0.0) / t, 1)
        p = logp.exp() * some[:, None]
        logq = torch.log_softmax(z / t, 1)
        kl = torch.where(p > 0, p * (logp - logq.gather(1, ids.clamp(min=0))), 0.0).sum(1)
        loss[r] = w * (1 - h) * t * t * kl
        if grad is not None:
            target = torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), p)
            grad[r] = (w * (1 - h) * t * some)[:, None] * (logq.exp() - target)
        if h > 0:
            y, wh = s["labels"][r], w * h * (s["labels"][r] >= 0)
            logq = torch.log_softmax(z, 1)
            loss[r] -= wh * logq.gather(1, y.clamp(min=0)[:, None])[:, 0]
            if grad is not None:
                grad[r] += wh[:, None] * logq.exp()
                grad[r] -= torch.zeros_like(z).scatter_(1, y.clamp(min=0)[:, None], wh[:, None])
    return loss if grad is None else (loss, grad)


# ---------------------------------------------------------------------------- least work ---
def work(case):
    """Each input read once and each output written once; of the table, the rows that the tokens name
    (for the 1/rank law: the expected number of them)."""
    op = case["op"]
    if op in ("lookup", "embed_grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        if op == "embed_grad":
            return {"bytes": 8 * n + n * d * BYTES[case["grad"]] + v * d * BYTES[case["out"]], "flops": 2 * n * d}
        share = torch.log1p(1 / torch.arange(1, v + 1, dtype=torch.float64)) / math.log(v)
        rows = float((1 - (1 - share) ** n).sum())
        return {"bytes": 8 * n + rows * d * BYTES[case["table"]] + n * d * BYTES[case["out"]], "flops": n * d}
    if op in ("qk", "qk_grad"):
        tokens = case["batch"] * case["seq"]
        each = tokens * (case["heads"] + case["kv_heads"]) * case["head_dim"]
        passes, flops = (2, 8) if op == "qk" else (3, 20)
        return {"bytes": 8 * tokens + each * passes * BYTES[case["dtype"]], "flops": flops * each}
    n, v = case["rows"], case["vocab"]
    passes, flops = (1, 4) if op == "distill" else (2, 8)
    return {"bytes": n * v * passes * BYTES[case["dtype"]] + n * min(case["top"], v) * 12 + 16 * n,
            "flops": flops * n * v}
