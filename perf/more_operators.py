"""Workloads of the operators at the two ends of a training step on tokens: embedding lookup and its gradient, layer norm
and its backward pass, the log probabilities of given tokens with entropy and top alternatives and their backward pass,
and distillation from a teacher's top logits, loss and gradient.

`run` computes one pass: with `own` false from elementary torch operations in 32 bits, with `own` true through the
library's entry points.  `exact` computes the same outputs in 64 bits from the operators' definitions."""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": F8, "i32": torch.int32, "i64": torch.int64}
BYTES = {"bf16": 2, "f32": 4, "e4m3": 1, "i32": 4, "i64": 8, "none": 0}
E4M3_MAX = 448.0
EPS = 1e-5


# ---- cases ----------------------------------------------------------------------------------------
def listed():
    return [
        # the tokens of one decoding step of 64 sequences: latency
        dict(name="embed_64x4096", op="embed", n=64, vocab=32000, d=4096, table="bf16", out="bf16", ids="i32", scale=1.0, pads=0.0),
        # the tokens of a training step at the Llama-13B-shaped layer's width, rows scaled by the root of the width
        dict(name="embed_16384x5120", op="embed", n=16384, vocab=32000, d=5120, table="bf16", out="bf16", ids="i64", scale=71.5541752799933, pads=0.05),
        # the gradient of a GPT-2-small-shaped table, whole: rows of absent tokens are zeros
        dict(name="embed_bwd_50257x768", op="embed_bwd", n=8192, vocab=50257, d=768, dy="bf16", dtable="f32", ids="i64", scale=1.0, accumulate=False, pads=0.0),
        # a tied table: what the output projection left there grows by the rows of the tokens that occur; padded batch
        dict(name="embed_bwd_tied_32000x4096", op="embed_bwd", n=16384, vocab=32000, d=4096, dy="bf16", dtable="f32", ids="i32", scale=1.0, accumulate=True, pads=0.1),
        # a single token before a projection: latency
        dict(name="layernorm_one_token", op="layernorm", rows=1, cols=4096, x="bf16", res="bf16", y="bf16"),
        # a training step of the GPT-2-small-shaped layer: fp32 residual stream, bf16 output of the block before
        dict(name="layernorm_8192x768", op="layernorm", rows=8192, cols=768, x="bf16", res="f32", y="bf16"),
        # backward at the Llama-13B-shaped layer's tokens and width, with the residual stream's gradient
        dict(name="layernorm_bwd_16384x5120", op="layernorm_bwd", rows=16384, cols=5120, h="bf16", dy="bf16", dres=True),
        # serving: what 16 sequences' next tokens got, and the 20 best alternatives
        dict(name="logprobs_top20_16x128000", op="logprobs", rows=16, vocab=128000, pad=0, x="f32", ids="i64", scale=1.0, top=20, entropy=True, pads=0.0),
        # evaluation and the loss of a training step: odd vocabulary, rows padded as a product leaves them
        dict(name="logprobs_8192x50257", op="logprobs", rows=8192, vocab=50257, pad=47, x="bf16", ids="i64", scale=1.0, top=0, entropy=True, pads=0.05),
        # the loss's gradient with a large vocabulary, with an entropy bonus
        dict(name="logprobs_bwd_8192x128000", op="logprobs_bwd", rows=8192, vocab=128000, pad=0, x="bf16", dx="bf16", ids="i64", scale=1.0, entropy=True, pads=0.05),
        # a student of an odd vocabulary in fp32 with rows that touch, few tokens; the teacher's probabilities as they are
        dict(name="distill_301x50257", op="distill", rows=301, vocab=50257, pad=0, x="f32", dx="f32", t="f32", ids="i64", k=37, scale=1.0, normalize=False, pads=0.05),
        # loss and gradient of a training step against a teacher's 64 best logits at temperature 2
        dict(name="distill_8192x32000", op="distill", rows=8192, vocab=32000, pad=0, x="bf16", dx="bf16", t="bf16", ids="i32", k=64, scale=0.5, normalize=True, pads=0.05),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_bwd", "embed_bwd", "layernorm", "layernorm", "layernorm_bwd", "logprobs", "logprobs", "logprobs_bwd", "distill", "distill"])
    even = rng.random() < 0.6                      # whole vectors; the others are odd
    if op.startswith("embed"):
        n, vocab, d = _spread(rng, 1, 32768), _spread(rng, 500, 131072), _spread(rng, 64, 8192)
        d = d // 8 * 8 if even else d
        vocab = min(vocab, (1 << 28) // d)
        c = dict(op=op, n=n, vocab=vocab, d=d, ids=rng.choice(["i32", "i64"]), scale=rng.choice([1.0, math.sqrt(d)]), pads=rng.choice([0.0, 0.1]))
        if op == "embed":
            c.update(table=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
        else:
            c.update(dy=rng.choice(["bf16", "f32"]), dtable=rng.choice(["f32", "f32", "bf16"]), accumulate=rng.random() < 0.5)
        return c
    if op.startswith("layernorm"):
        rows = _spread(rng, 1, 16384)
        cols = _spread(rng, 64, 16384 if rows <= 8192 else 8192)
        cols = max(8, cols // 8 * 8) if even else cols
        if op == "layernorm":
            return dict(op=op, rows=rows, cols=cols, x=rng.choice(["bf16", "f32"]), res=rng.choice(["none", "bf16", "f32"]), y=rng.choice(["bf16", "f32", "e4m3"]))
        return dict(op=op, rows=rows, cols=min(cols, 8192), h=rng.choice(["bf16", "f32"]), dy=rng.choice(["bf16", "f32"]), dres=rng.random() < 0.7)
    vocab = _spread(rng, 1000, 160000)
    vocab = vocab // 8 * 8 if even else vocab
    rows = _spread(rng, 1, max(1, min(8192, 400_000_000 // vocab)))
    c = dict(op=op, rows=rows, vocab=vocab, pad=rng.choice([0, 0, -vocab % 64]), x=rng.choice(["bf16", "bf16", "f32"]), ids=rng.choice(["i32", "i64"]),
             scale=rng.choice([1.0, 1.0, 0.5, 1.25]), pads=rng.choice([0.0, 0.1]))
    if op == "logprobs":
        c.update(top=rng.choice([0, 1, 5, 20, 50]) if rows * vocab < 1 << 27 else 0, entropy=rng.random() < 0.6)
    elif op == "logprobs_bwd":
        c.update(dx=c["x"] if rng.random() < 0.7 else "bf16", entropy=rng.random() < 0.4)
    else:
        c.update(dx=c["x"] if rng.random() < 0.7 else "bf16", t=rng.choice(["bf16", "f32"]), k=_spread(rng, 1, 128), normalize=rng.random() < 0.7)
    return c


def _distinct(n, vocab):
    """Expected number of different tokens among n of the distribution of `_tokens`."""
    v = np.arange(vocab, dtype=np.float64)
    p = np.log1p(1.0 / (v + 1)) / math.log(vocab + 1)
    return float((1 - np.exp(n * np.log1p(-np.minimum(p, 1 - 1e-12)))).sum())


def work(case):
    b, op = BYTES, case["op"]
    if op == "embed":
        n, d = case["n"], case["d"]
        live = n * (1 - case["pads"])
        return {"bytes": _distinct(live, case["vocab"]) * d * b[case["table"]] + n * (d * b[case["out"]] + b[case["ids"]]), "flops": n * d}
    if op == "embed_bwd":
        n, d = case["n"], case["d"]
        live = n * (1 - case["pads"])
        rows = 2 * _distinct(live, case["vocab"]) if case["accumulate"] else case["vocab"]
        return {"bytes": live * d * b[case["dy"]] + n * b[case["ids"]] + rows * d * b[case["dtable"]], "flops": 2 * n * d}
    if op == "layernorm":
        t, d = case["rows"], case["cols"]
        return {"bytes": t * d * (b[case["x"]] + 2 * b[case["res"]] + b[case["y"]]) + 8 * d + 12 * t, "flops": 8 * t * d}
    if op == "layernorm_bwd":
        t, d = case["rows"], case["cols"]
        return {"bytes": t * d * (b[case["dy"]] + b[case["h"]] * (3 if case["dres"] else 2)) + 12 * d + 8 * t, "flops": 12 * t * d}
    t, v = case["rows"], case["vocab"]
    if op == "logprobs":
        return {"bytes": t * (v * b[case["x"]] + b[case["ids"]] + 12 + 8 * case["top"]), "flops": (6 if case["entropy"] else 4) * t * v}
    if op == "logprobs_bwd":
        return {"bytes": t * (v * (b[case["x"]] + b[case["dx"]]) + b[case["ids"]] + 16), "flops": (7 if case["entropy"] else 4) * t * v}
    # the logits are needed for the sum first and for the gradient after it: twice
    return {"bytes": t * (v * (2 * b[case["x"]] + b[case["dx"]]) + case["k"] * (b[case["t"]] + b[case["ids"]]) + 12), "flops": 8 * t * v}


# ---- inputs ---------------------------------------------------------------------------------------
def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    x = torch.randn(*shape, generator=g, device=DEV)
    return (x.mul_(scale) if scale != 1.0 else x).to(dtype)


def _tokens(g, n, vocab, kind, pads, pad):
    """Tokens whose frequency falls with 1 / rank, as a vocabulary's do, and a share of padding at the end."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    t = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    live = n - int(n * pads)
    t[live:] = pad
    return t.to(TYPES[kind])


def _logits(g, case):
    """Scores with a spread of 2.5; one place in 50 of the vocabulary is masked (special and unused entries)."""
    rows, vocab = case["rows"], case["vocab"]
    x = torch.randn(rows, vocab + case["pad"], generator=g, device=DEV, dtype=torch.float32).mul_(2.5)
    x.masked_fill_(torch.rand(vocab + case["pad"], generator=g, device=DEV) < 0.02, -math.inf)
    return x.to(TYPES[case["x"]])[:, :vocab]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op.startswith("embed"):
        n, vocab, d = case["n"], case["vocab"], case["d"]
        s["tokens"] = _tokens(g, n, vocab, case["ids"], case["pads"], -1)
        if op == "embed":
            s["table_in"] = _randn(g, vocab, d, scale=0.02, dtype=TYPES[case["table"]])
            s["y"] = torch.empty(n, d, dtype=TYPES[case["out"]], device=DEV)
        else:
            s["dy_in"] = _randn(g, n, d, dtype=TYPES[case["dy"]])
            s["dt"] = _randn(g, vocab, d, dtype=TYPES[case["dtable"]])
        return s
    if op == "layernorm":
        t, d = case["rows"], case["cols"]
        s["x_in"] = _randn(g, t, d, dtype=TYPES[case["x"]])
        s["r"] = _randn(g, t, d, scale=3.0).add_(0.5).to(TYPES[case["res"]]) if case["res"] != "none" else None
        s["w"], s["b"] = 1.0 + _randn(g, d, scale=0.1), _randn(g, d, scale=0.1)
        s["yout"] = torch.empty(t, d, dtype=TYPES[case["y"]], device=DEV)
        s["h"] = torch.empty_like(s["r"]) if s["r"] is not None else None
        s["mean"], s["rstd"] = torch.empty(t, device=DEV), torch.empty(t, device=DEV)
        s["codes"] = torch.empty(t, device=DEV) if case["y"] == "e4m3" else None
        return s
    if op == "layernorm_bwd":
        t, d = case["rows"], case["cols"]
        s["h_in"] = _randn(g, t, d, scale=3.0).add_(0.5).to(TYPES[case["h"]])
        h = s["h_in"].float()
        s["mean"] = h.mean(1)
        s["rstd"] = torch.rsqrt((h - s["mean"][:, None]).square().mean(1) + EPS)
        s["w"] = 1.0 + _randn(g, d, scale=0.1)
        s["dy_in"] = _randn(g, t, d, dtype=TYPES[case["dy"]])
        s["dres_in"] = _randn(g, t, d, dtype=TYPES[case["h"]]) if case["dres"] else None
        s["dxout"] = torch.empty(t, d, dtype=TYPES[case["h"]], device=DEV)
        s["dw"], s["db"] = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        return s
    t, vocab = case["rows"], case["vocab"]
    s["logits"] = _logits(g, case)
    f32 = lambda *shape: torch.empty(*shape, device=DEV)  # noqa: E731
    if op == "distill":
        # each row's teacher: k different places, best first; a few places in a row may be empty (index -1)
        k = case["k"]
        first = torch.randint(0, vocab, (t, 1), generator=g, device=DEV)
        step = torch.randint(1, max(2, vocab // k), (t, 1), generator=g, device=DEV)
        at = (first + step * torch.arange(k, device=DEV)) % vocab
        values = -torch.rand(t, k, generator=g, device=DEV).mul_(0.6).cumsum(1)
        values = values - torch.logsumexp(values, 1, keepdim=True) - 0.05
        # the student has an idea of what the teacher says
        s["logits"].scatter_(1, at, (values + 11.0 + _randn(g, t, k)).to(TYPES[case["x"]]))
        at[torch.rand(t, k, generator=g, device=DEV) < 0.02] = -1
        at[t - int(t * case["pads"]):] = -1                                    # a padded batch: nothing to learn there
        s["index"], s["values"] = at.to(TYPES[case["ids"]]), values.to(TYPES[case["t"]])
        s["loss"], s["lse"] = f32(t), f32(t)
        s["dloss"] = torch.full((t,), 1.0 / t, device=DEV)
        s["dxout"] = torch.empty(t, vocab + case["pad"], dtype=TYPES[case["dx"]], device=DEV)[:, :vocab]
        return s
    s["tokens"] = _tokens(g, t, vocab, case["ids"], case["pads"], -100)
    # the given tokens are likely ones, and never masked
    at = s["tokens"].long().clamp_min(0)[:, None]
    s["logits"].scatter_(1, at, (9.0 + _randn(g, t, 1, scale=2.0)).to(TYPES[case["x"]]))
    if op == "logprobs":
        s["logp"], s["lse"] = f32(t), f32(t)
        s["H"] = f32(t) if case["entropy"] else None
        s["tv"] = f32(t, case["top"]) if case["top"] else None
        s["ti"] = torch.empty(t, case["top"], dtype=torch.int32, device=DEV) if case["top"] else None
        return s
    s["lse"], s["H"] = _statistics(s["logits"], case["scale"])
    s["dlogp"] = -torch.rand(t, generator=g, device=DEV) / t
    s["dH"] = torch.full((t,), -0.01 / t, device=DEV) if case["entropy"] else None
    s["dxout"] = torch.empty(t, vocab + case["pad"], dtype=TYPES[case["dx"]], device=DEV)[:, :vocab]
    return s


# ---- plain forms ----------------------------------------------------------------------------------
def _live(tokens, vocab):
    t = tokens.long()
    return (t >= 0) & (t < vocab)


def _plain_embed(s):
    ok = _live(s["tokens"], s["vocab"])
    rows = s["table_in"][s["tokens"].long() * ok].float() * s["scale"] * ok[:, None]
    return {"y": rows.to(TYPES[s["out"]])}


def _plain_embed_bwd(s):
    ok = _live(s["tokens"], s["vocab"])
    g = s["dy_in"].float() * s["scale"] * ok[:, None]
    total = torch.zeros(s["vocab"], s["d"], device=DEV).index_add_(0, s["tokens"].long() * ok, g)
    if s["accumulate"]:
        total += s["dt"].float()
    s["dt"].copy_(total)
    return {"dtable": s["dt"]}


def _row_codes(y):
    top = y.abs().amax(1)
    scale = top * (1 / E4M3_MAX)
    q = y * torch.where(scale == 0, 0.0, 1.0 / scale)[:, None]
    return q.clamp(-E4M3_MAX, E4M3_MAX).to(F8), scale


def _plain_layernorm(s):
    h = s["x_in"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    mean = h.mean(1)
    c = h - mean[:, None]
    rstd = torch.rsqrt(c.square().mean(1) + EPS)
    y = c * rstd[:, None] * s["w"] + s["b"]
    out = {"mean": mean, "rstd": rstd}
    if s["r"] is not None:
        out["h"] = h.to(s["r"].dtype)
    if s["codes"] is not None:
        out["y"], out["codes"] = _row_codes(y)
    else:
        out["y"] = y.to(s["yout"].dtype)
    return out


def _plain_layernorm_bwd(s):
    xh = (s["h_in"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy_in"].float()
    q = dy * s["w"]
    dx = s["rstd"][:, None] * (q - q.mean(1, keepdim=True) - xh * (q * xh).mean(1, keepdim=True))
    if s["dres_in"] is not None:
        dx = dx + s["dres_in"].float()
    return {"dx": dx.to(s["dxout"].dtype), "dw": (dy * xh).sum(0), "db": dy.sum(0)}


def _statistics(logits, scale):
    """lse and entropy of each row, in 32 bits; a masked place (-inf) has probability 0 and adds nothing."""
    x = logits.float()
    top = x.amax(1, keepdim=True)
    d = (x - top).mul_(scale)
    e = torch.exp(d)
    total = e.sum(1)
    mean = e.mul_(d.clamp_min_(-1e30)).sum(1) / total
    log_total = torch.log(total)
    return top[:, 0] * scale + log_total, log_total - mean


def _plain_logprobs(s):
    x = s["logits"]
    ok = _live(s["tokens"], s["vocab"])
    lse, entropy = _statistics(x, s["scale"])
    at = (s["tokens"].long() * ok)[:, None]
    own_score = x.gather(1, at)[:, 0].float() * s["scale"]
    out = {"logp": torch.where(ok, own_score - lse, 0.0), "lse": lse}
    if s["entropy"]:
        out["entropy"] = entropy
    if s["top"]:
        # whole numbers that order like the scores and, among equal ones, by place
        bits = (x.float() + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
        key |= torch.arange(s["vocab"] - 1, -1, -1, device=DEV)
        best = key.topk(s["top"], dim=1).values
        index = s["vocab"] - 1 - (best & 0xFFFFFFFF)
        out["top_index"] = index.int()
        out["top_values"] = x.gather(1, index).float() * s["scale"] - lse[:, None]
    return out


def _plain_logprobs_bwd(s):
    ok = _live(s["tokens"], s["vocab"])
    logp = s["logits"].float() * s["scale"] - s["lse"][:, None]
    p = torch.exp(logp)
    up = s["dlogp"] * ok
    g = p * -up[:, None]
    g.scatter_add_(1, (s["tokens"].long() * ok)[:, None], up[:, None])
    if s["entropy"]:
        g -= p.mul_(logp.clamp_min_(-1e30) + s["H"][:, None]).mul_(s["dH"][:, None])
    return {"dx": (g * s["scale"]).to(s["dxout"].dtype)}


def _plain_distill(s):
    ok = _live(s["index"], s["vocab"])
    at = s["index"].long() * ok
    x = s["logits"].float()
    lse, _ = _statistics(s["logits"], s["scale"])
    t = (s["values"].float() * s["scale"]).masked_fill(~ok, -math.inf)
    if s["normalize"]:
        top = t.amax(1, keepdim=True).clamp_min(-1e30)
        t = t - top
        t = t - torch.log(torch.exp(t).sum(1, keepdim=True)).clamp_min(-1e30)
    q = torch.exp(t)
    logp = x.gather(1, at) * s["scale"] - lse[:, None]
    loss = torch.where(q > 0, q * (t - logp), 0.0).sum(1)
    up = s["dloss"][:, None] * s["scale"]
    g = torch.exp(x * s["scale"] - lse[:, None]) * (q.sum(1, keepdim=True) * up)
    g.scatter_add_(1, at, -q * up)
    return {"loss": loss, "lse": lse, "dx": g.to(s["dxout"].dtype)}


# ---- one pass -------------------------------------------------------------------------------------
def _own_run(s):
    import paper_2512_22142_b200 as cl
    op = s["op"]
    if op == "embed":
        cl.embedding(s["tokens"], s["table_in"], s["y"], scale=s["scale"])
        return {"y": s["y"]}
    if op == "embed_bwd":
        cl.embedding_backward(s["dy_in"], s["tokens"], s["dt"], scale=s["scale"], accumulate=s["accumulate"])
        return {"dtable": s["dt"]}
    if op == "layernorm":
        cl.layernorm(s["x_in"], s["w"], s["b"], s["yout"], residual=s["r"], h=s["h"], mean=s["mean"], rstd=s["rstd"], scale=s["codes"], eps=EPS)
        out = {"y": s["yout"], "mean": s["mean"], "rstd": s["rstd"]}
        if s["h"] is not None:
            out["h"] = s["h"]
        if s["codes"] is not None:
            out["codes"] = s["codes"]
        return out
    if op == "layernorm_bwd":
        cl.layernorm_backward(s["dy_in"], s["h_in"], s["w"], s["mean"], s["rstd"], s["dxout"], s["dw"], s["db"], dres=s["dres_in"])
        return {"dx": s["dxout"], "dw": s["dw"], "db": s["db"]}
    if op == "logprobs":
        cl.token_logprobs(s["logits"], s["tokens"], s["logp"], lse=s["lse"], entropy=s["H"], top_values=s["tv"], top_index=s["ti"], scale=s["scale"])
        out = {"logp": s["logp"], "lse": s["lse"]}
        if s["entropy"]:
            out["entropy"] = s["H"]
        if s["top"]:
            out.update(top_values=s["tv"], top_index=s["ti"])
        return out
    if op == "logprobs_bwd":
        cl.token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["dxout"], dlogp=s["dlogp"], dentropy=s["dH"],
                                   entropy=s["H"] if s["entropy"] else None, scale=s["scale"])
        return {"dx": s["dxout"]}
    cl.distill(s["logits"], s["index"], s["values"], s["loss"], lse=s["lse"], scale=s["scale"], normalize=s["normalize"])
    cl.distill_backward(s["logits"], s["index"], s["values"], s["lse"], s["dloss"], s["dxout"], scale=s["scale"], normalize=s["normalize"])
    return {"loss": s["loss"], "lse": s["lse"], "dx": s["dxout"]}


def run(state):
    if own:
        return _own_run(state)
    return {"embed": _plain_embed, "embed_bwd": _plain_embed_bwd, "layernorm": _plain_layernorm, "layernorm_bwd": _plain_layernorm_bwd,
            "logprobs": _plain_logprobs, "logprobs_bwd": _plain_logprobs_bwd, "distill": _plain_distill}[state["op"]](state)


# ---- 64 bits, from the definitions ----------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        padded = torch.cat([s["table_in"].double() * case["scale"], torch.zeros(1, case["d"], dtype=torch.float64, device=DEV)])
        return {"y": padded[torch.where(_live(s["tokens"], case["vocab"]), s["tokens"].long(), case["vocab"])]}
    if op == "embed_bwd":
        total = s["dt"].double() if case["accumulate"] else torch.zeros(case["vocab"], case["d"], dtype=torch.float64, device=DEV)
        keep = torch.nonzero(_live(s["tokens"], case["vocab"]))[:, 0]
        total.index_put_((s["tokens"].long()[keep],), s["dy_in"][keep].double() * case["scale"], accumulate=True)
        return {"dtable": total}
    if op == "layernorm":
        h = s["x_in"].double() if s["r"] is None else s["x_in"].double() + s["r"].double()
        mean, rstd = h.mean(1), (h.var(1, unbiased=False) + EPS) ** -0.5
        y = torch.einsum("ij,i,j->ij", h - mean[:, None], rstd, s["w"].double()) + s["b"].double()
        out = {"mean": mean, "rstd": rstd, "h": None if s["r"] is None else h, "y": y, "codes": None}
        if case["y"] == "e4m3":
            out["codes"] = y.abs().max(1).values / E4M3_MAX
            out["y"] = y / out["codes"][:, None]
        return out
    if op == "layernorm_bwd":
        n = case["cols"]
        rstd, dy, w = s["rstd"].double(), s["dy_in"].double(), s["w"].double()
        c = s["h_in"].double() - s["mean"].double()[:, None]
        along = torch.einsum("ij,j,ij->i", dy, w, c) * rstd ** 3 / n
        dx = torch.einsum("i,ij,j->ij", rstd, dy, w) - (rstd * (dy @ w) / n)[:, None] - c * along[:, None]
        if s["dres_in"] is not None:
            dx = dx + s["dres_in"].double()
        return {"dx": dx, "dw": torch.einsum("ij,ij,i->j", dy, c, rstd), "db": dy.sum(0)}
    z = s["logits"].double() * case["scale"]
    if op == "logprobs":
        logp = torch.log_softmax(z, 1)
        ok = _live(s["tokens"], case["vocab"])
        at = torch.where(ok, s["tokens"].long(), 0)[:, None]
        out = {"logp": torch.where(ok, logp.gather(1, at)[:, 0], 0.0), "lse": torch.logsumexp(z, 1)}
        if case["entropy"]:
            out["entropy"] = torch.special.entr(logp.exp()).sum(1)
        if case["top"]:
            out["top_values"], out["top_index"] = logp.topk(case["top"], dim=1).values, None
            if case["rows"] * case["vocab"] <= 1 << 24:
                out["top_index"] = z.sort(dim=1, descending=True, stable=True).indices[:, :case["top"]].int()
        return out
    p = torch.exp(z - s["lse"].double()[:, None]) if op == "logprobs_bwd" else torch.softmax(z, 1)
    if op == "logprobs_bwd":
        up = torch.where(_live(s["tokens"], case["vocab"]), s["dlogp"].double(), 0.0)
        g = -up[:, None] * p
        rows = torch.arange(case["rows"], device=DEV)
        g[rows, s["tokens"].long().clamp_min(0)] += up
        if case["entropy"]:
            g += s["dH"].double()[:, None] * (torch.special.entr(p) - s["H"].double()[:, None] * p)
        return {"dx": g * case["scale"]}
    ok = _live(s["index"], case["vocab"])
    logq = torch.where(ok, s["values"].double() * case["scale"], -math.inf)
    if case["normalize"]:
        logq = torch.where(ok, logq - torch.logsumexp(logq, 1, keepdim=True), -math.inf)
    q = logq.exp()
    at = torch.where(ok, s["index"].long(), 0)
    cross = torch.where(ok, q * (z - torch.logsumexp(z, 1, keepdim=True)).gather(1, at), 0.0).sum(1)
    g = torch.einsum("ij,i->ij", p, q.sum(1)) .scatter_add_(1, at, -q)
    return {"loss": -torch.special.entr(q).sum(1) - cross, "lse": torch.logsumexp(z, 1), "dx": g * (s["dloss"].double() * case["scale"])[:, None]}
