"""What is measured of the operators between the lifted weights w and the gradient g that a subspace step takes:
layer norm, embedding lookup, log probabilities of given tokens (each with its backward pass), and the norm of all
gradients with clipping into one flat vector.

`own` false: every operator in its plain form, elementary torch operations in 32 bits, rounded once at the end.
`own` true:  the library's entry points, as a training or scoring program calls them.

A case is a dict: "op" names the operator and direction, the rest are its sizes and types.
"""

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5                    # layer norm
CLIP_EPS = 1e-6               # added to the norm before max_norm is divided by it
IGNORE = -100                 # a target that stands for no token
F32, BF16 = "f32", "bf16"
_DT = {F32: torch.float32, BF16: torch.bfloat16}
_SIZE = {F32: 4, BF16: 2, "i32": 4, "i64": 8}


# ------------------------------------------------------------------------------------------- cases
def _decoder_sizes():
    """Parameter tensors of the 1.3 B decoder workload: 1,315,758,080 elements in 388 tensors."""
    d, ffn, vocab, positions = 2048, 8192, 50272, 2050
    per_block = [d * d, d] * 4 + [d, d, ffn * d, ffn, d * ffn, d, d, d]
    return [vocab * d, positions * d] + per_block * 24 + [d, d]


def _vit_sizes():
    """Parameter tensors of the ViT-B/16 workload: 86,567,656 elements in 152 tensors."""
    d, mlp, patch, tokens, classes = 768, 4 * 768, 16, 197, 1000
    per_block = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, mlp * d, mlp, d * mlp, d]
    return [d, tokens * d, d * 3 * patch * patch, d] + per_block * 12 + [d, d, d * classes, classes]


def _ragged_sizes(count, total, spread):
    """`count` sizes of about `total` elements together, the largest about e^(2 spread) times the smallest."""
    w = [math.exp(spread * math.cos(2.399963 * i)) for i in range(count)]
    s = sum(w)
    return [max(1, int(total * v / s)) for v in w]


def _sizes(case):
    if case["model"] == "decoder":
        return _decoder_sizes()
    if case["model"] == "vit":
        return _vit_sizes()
    return _ragged_sizes(case["tensors"], case["total"], case["spread"])


def _norm(name, back, rows, cols, dtype, wtype=F32, pad=0, shift=0):
    # pad: elements between rows (a column block of a wider activation); shift: where the weights start in the flat vector
    c = {"name": name, "op": "layer_norm_backward" if back else "layer_norm", "rows": rows, "cols": cols, "dtype": dtype,
         "wtype": wtype, "pad": pad, "shift": shift}
    return c if name else {k: v for k, v in c.items() if k != "name"}


def _embed(name, back, tokens, vocab, dim, table, act, ids="i64", scale=1.0, padding=-1, accumulate=False):
    # table: type of the table, or of its gradient; act: type of the rows looked up, or of their gradient
    c = {"name": name, "op": "embedding_backward" if back else "embedding", "tokens": tokens, "vocab": vocab, "dim": dim,
         "table": table, "act": act, "ids": ids, "scale": scale}
    if back:
        c.update(padding=padding, accumulate=accumulate)
    return c if name else {k: v for k, v in c.items() if k != "name"}


def _logp(name, back, rows, vocab, dtype, top=0, entropy=True, masked=0.0, ignored=0.0, ids="i64"):
    # masked: share of the vocabulary at -inf, and then one whole row; ignored: share of rows whose target stands for no token
    c = {"name": name, "op": "token_logprobs_backward" if back else "token_logprobs", "rows": rows, "vocab": vocab,
         "dtype": dtype, "entropy": entropy, "masked": masked, "ignored": ignored, "ids": ids}
    if not back:
        c["top"] = top
    return c if name else {k: v for k, v in c.items() if k != "name"}


def _clip(name, model, grad, flat, max_norm, tensors=0, total=0, spread=0.0):
    # grad: type of the tensors ("mixed": bfloat16, every third float32); flat: type of the flat gradient
    c = {"name": name, "op": "clip_gather", "model": model, "grad": grad, "flat": flat, "max_norm": max_norm,
         "tensors": tensors, "total": total, "spread": spread}
    return c if name else {k: v for k, v in c.items() if k != "name"}


def listed():
    return [
        # the tokens of one image through a ViT-B/16 norm, float32: latency counts
        _norm("norm 197x768 f32", False, 197, 768, F32),
        # a micro-batch of 8 sequences of 2048 tokens through a norm of the decoder, with float32 weights as lifted
        _norm("norm 16384x2048 bf16", False, 16384, 2048, BF16),
        _norm("norm bwd 16384x2048 bf16", True, 16384, 2048, BF16),
        # rows of an odd width, on no 16-byte boundary
        _norm("norm bwd 4099x1023 f32", True, 4099, 1023, F32, shift=1),
        # a sequence looked up in the lifted float32 table, activations in bfloat16
        _embed("embed 2048 tokens bf16", False, 2048, 50272, 2048, F32, BF16),
        # the whole table's gradient for the same micro-batch: most rows stay zero, a few tokens are frequent
        _embed("embed bwd 16384 tokens", True, 16384, 50272, 2048, F32, BF16, padding=1),
        # one decoded token scored: its log probability, the entropy and 20 alternatives
        _logp("logprobs 1x50272 bf16", False, 1, 50272, BF16, top=20),
        # a batch of prompts scored
        _logp("logprobs 8192x50272 bf16", False, 8192, 50272, BF16, top=5, ignored=0.1),
        # a constrained vocabulary in float32, odd sizes
        _logp("logprobs 333x32003 f32", False, 333, 32003, F32, top=20, masked=0.3, ids="i32"),
        # the loss's gradient for a batch of training rows
        _logp("logprobs bwd 8192x50272 bf16", True, 8192, 50272, BF16, entropy=False, ignored=0.1),
        # all gradients of the image model, float32, into the flat gradient of the step
        _clip("clip vit f32", "vit", F32, F32, 1.0),
        # all gradients of the decoder, bfloat16: the largest
        _clip("clip decoder bf16", "decoder", BF16, BF16, 1.0),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_bwd", "embed", "embed_bwd", "logp", "logp_bwd", "clip"])
    if op in ("norm", "norm_bwd"):
        cols = _log_int(rng, 8, 16384)
        rows = _log_int(rng, 1, min(65536, (1 << 25) // cols))
        if rng.random() < 0.5:
            cols = max(8, cols // 8 * 8)
        return _norm("", op == "norm_bwd", rows, cols, rng.choice([F32, BF16]), rng.choice([F32, F32, BF16]),
                     rng.choice([0, 0, 8, 3]), rng.choice([0, 0, 1, 2]))
    if op in ("embed", "embed_bwd"):
        dim = _log_int(rng, 4, 4096)
        if rng.random() < 0.6:
            dim = max(8, dim // 8 * 8)
        vocab = _log_int(rng, 16, min(131072, 100_000_000 // dim))
        tokens = _log_int(rng, 1, 16384)
        return _embed("", op == "embed_bwd", tokens, vocab, dim, rng.choice([F32, BF16]), rng.choice([F32, BF16]),
                      rng.choice(["i32", "i64"]), rng.choice([1.0, round(math.sqrt(dim), 3)]), rng.choice([-1, 1]),
                      rng.choice([False, False, True]))
    if op in ("logp", "logp_bwd"):
        vocab = _log_int(rng, 64, 131072)
        rows = _log_int(rng, 1, min(16384, 300_000_000 // vocab))
        if rng.random() < 0.5:
            vocab = vocab // 8 * 8
        return _logp("", op == "logp_bwd", rows, vocab, rng.choice([F32, BF16]), rng.choice([0, 1, 5, 20]),
                     rng.choice([False, True]), rng.choice([0.0, 0.0, 0.3]), rng.choice([0.0, 0.2]), rng.choice(["i32", "i64"]))
    grad, flat = rng.choice([(F32, F32), (BF16, BF16), (BF16, F32), ("mixed", F32), ("mixed", BF16)])
    return _clip("", "ragged", grad, flat, rng.choice([0.1, 1.0, 1e6]), _log_int(rng, 1, 700), _log_int(rng, 1000, 400_000_000),
                 rng.choice([0.0, 2.0, 4.0]))


# ------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 2654435761 % (1 << 62) + 1)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _activations(g, rows, cols, dtype, pad):
    """Rows with a few columns far from zero and far larger than the rest, as the residual stream of a decoder has."""
    x = _randn(g, rows, cols) * (0.5 + torch.rand((rows, 1), generator=g, device=DEV)) + 0.3 * _randn(g, cols)
    x[:, :: max(1, cols // 7)] *= 8.0
    buf = torch.zeros((rows, cols + pad), dtype=_DT[dtype], device=DEV)
    buf[:, :cols] = x
    return buf[:, :cols]


def _tokens(g, count, vocab, ids):
    """Token numbers whose frequency falls as one over their rank, ranks spread over the vocabulary."""
    u = torch.rand((count,), generator=g, device=DEV, dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab + 1)) - 1).to(torch.int64).clamp_(0, vocab - 1)
    stride = 7919 if math.gcd(7919, vocab) == 1 else 1
    return (rank * stride % vocab).to(torch.int32 if ids == "i32" else torch.int64)


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = {"case": case}
    if op.startswith("layer_norm"):
        rows, cols, dt = case["rows"], case["cols"], _DT[case["dtype"]]
        s["x"] = _activations(g, rows, cols, case["dtype"], case["pad"])
        flat = (_randn(g, case["shift"] + 2 * cols) * 0.1).to(_DT[case["wtype"]])
        s["weight"] = flat[case["shift"]: case["shift"] + cols].add_(1.0)
        s["bias"] = flat[case["shift"] + cols:]
        s["mean"] = torch.empty((rows,), device=DEV)
        s["rstd"] = torch.empty((rows,), device=DEV)
        s["out"] = torch.empty((rows, cols), dtype=dt, device=DEV)
        if op == "layer_norm_backward":
            xf = s["x"].float()
            s["mean"].copy_(xf.mean(1))
            s["rstd"].copy_((xf - s["mean"][:, None]).square().mean(1).add_(EPS).rsqrt_())
            s["dy"] = (_randn(g, rows, cols) * 0.01).to(dt)
            s["dw"] = torch.empty((cols,), device=DEV)
            s["db"] = torch.empty((cols,), device=DEV)
    elif op == "embedding":
        s["table"] = (_randn(g, case["vocab"], case["dim"]) * 0.02).to(_DT[case["table"]])
        s["ids"] = _tokens(g, case["tokens"], case["vocab"], case["ids"])
        s["out"] = torch.empty((case["tokens"], case["dim"]), dtype=_DT[case["act"]], device=DEV)
    elif op == "embedding_backward":
        s["dout"] = (_randn(g, case["tokens"], case["dim"]) * 0.01).to(_DT[case["act"]])
        s["ids"] = _tokens(g, case["tokens"], case["vocab"], case["ids"])
        s["dtable"] = torch.empty((case["vocab"], case["dim"]), dtype=_DT[case["table"]], device=DEV)
        if case["accumulate"]:            # added to what another use of the table has left (an output layer that shares it)
            s["before"] = (_randn(g, case["vocab"], case["dim"]) * 0.001).to(_DT[case["table"]])
    elif op.startswith("token_logprobs"):
        rows, vocab, dt = case["rows"], case["vocab"], _DT[case["dtype"]]
        z = _randn(g, rows, vocab).mul_(2.5)
        t = _tokens(g, rows, vocab, "i64")
        sure = torch.rand((rows,), generator=g, device=DEV)
        z[torch.arange(rows, device=DEV), t] += 12.0 * sure             # some rows are sure of their token
        if case["masked"]:
            off = torch.rand((vocab,), generator=g, device=DEV) < case["masked"]
            z.masked_fill_(off[None, :], -math.inf)
            if rows > 2:
                z[rows // 2] = -math.inf                                # a row whose mask leaves nothing
        if case["ignored"]:
            t[torch.rand((rows,), generator=g, device=DEV) < case["ignored"]] = IGNORE
        s["logits"], s["targets"] = z.to(dt), t.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        del z
        s["lse"] = torch.empty((rows,), device=DEV)
        if op == "token_logprobs":
            s["logp"] = torch.empty((rows,), device=DEV)
            s["entropy"] = torch.empty((rows,), device=DEV) if case["entropy"] else None
            k = min(case["top"], vocab)
            s["top_ids"] = torch.empty((rows, k), dtype=torch.int32, device=DEV) if k else None
            s["top_logp"] = torch.empty((rows, k), device=DEV) if k else None
        else:
            s["lse"], h = _stats(s["logits"])
            s["entropy"] = h if case["entropy"] else None
            s["d_logp"] = -torch.rand((rows,), generator=g, device=DEV) / rows
            s["d_entropy"] = -0.01 * torch.rand((rows,), generator=g, device=DEV) / rows if case["entropy"] else None
            s["dlogits"] = torch.empty((rows, vocab), dtype=dt, device=DEV)
    else:
        sizes = _sizes(case)
        kinds = [BF16 if i % 3 else F32 for i in range(len(sizes))] if case["grad"] == "mixed" else [case["grad"]] * len(sizes)
        s["grads"] = [(_randn(g, n) * (1e-4 * math.exp(2.0 * math.sin(i)))).to(_DT[k]) for i, (n, k) in enumerate(zip(sizes, kinds))]
        s["g"] = torch.empty((sum(sizes),), dtype=_DT[case["flat"]], device=DEV)
        s["norm"] = torch.empty((1,), device=DEV)
    return s


def _stats(logits):
    """Log of the sum of exponentials and entropy of every row, in rows few enough for the temporaries; float32."""
    lse, ent = [], []
    for z in logits.split(max(1, (1 << 26) // logits.shape[1])):
        z = z.double()
        m = z.max(1, keepdim=True).values
        m = torch.where(m == -math.inf, 0.0, m)
        e = torch.exp(z - m)
        total = e.sum(1)
        lse.append((m[:, 0] + total.log()).float())
        w = torch.where(e > 0, e * (z - m), 0.0).sum(1)
        ent.append(torch.where(total > 0, total.log() - w / total, 0.0).float())
    return torch.cat(lse), torch.cat(ent)


# ------------------------------------------------------------------------------------------- one pass
_kept = {}


def _library(need=0):
    """The binding, a context on the current stream and a workspace of at least `need` bytes, kept as a program keeps them."""
    if "ctx" not in _kept:
        from paper_2205_13104_b200 import twa
        _kept["twa"], _kept["ctx"], _kept["ws"] = twa, twa.twa_create(0), torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    if _kept["ws"].numel() < need:
        _kept["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return _kept["twa"], _kept["ctx"], _kept["ws"]


def _own(s):
    c, op = s["case"], s["case"]["op"]
    twa, ctx, ws = _library()
    if op == "layer_norm":
        twa.twa_layer_norm(ctx, s["x"], s["weight"], s["bias"], EPS, s["out"], s["mean"], s["rstd"])
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "layer_norm_backward":
        if "ws_bytes" not in s:
            s["ws_bytes"] = twa.twa_layer_norm_workspace_bytes(c["rows"], c["cols"])
        ws = _library(s["ws_bytes"])[2]
        twa.twa_layer_norm_backward(ctx, s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["out"], s["dw"], s["db"], ws)
        return {"dx": s["out"], "dw": s["dw"], "db": s["db"]}
    if op == "embedding":
        twa.twa_embedding(ctx, s["table"], s["ids"], c["scale"], s["out"])
        return s["out"]
    if op == "embedding_backward":
        if "ws_bytes" not in s:
            s["ws_bytes"] = twa.twa_embedding_workspace_bytes(c["tokens"], c["vocab"], c["dim"])
        ws = _library(s["ws_bytes"])[2]
        if c["accumulate"]:
            s["dtable"].copy_(s["before"])
        twa.twa_embedding_backward(ctx, s["dout"], s["ids"], c["scale"], s["dtable"], ws, padding_id=c["padding"],
                                   accumulate=c["accumulate"])
        return s["dtable"]
    if op == "token_logprobs":
        twa.twa_token_logprobs(ctx, s["logits"], s["targets"], s["logp"], s["lse"], entropy=s["entropy"],
                               top_ids=s["top_ids"], top_logp=s["top_logp"], ignore_id=IGNORE)
        return {k: s[k] for k in ("logp", "lse", "entropy", "top_ids", "top_logp") if s[k] is not None}
    if op == "token_logprobs_backward":
        twa.twa_token_logprobs_backward(ctx, s["logits"], s["targets"], s["lse"], s["d_logp"], s["dlogits"],
                                        entropy=s["entropy"], d_entropy=s["d_entropy"], ignore_id=IGNORE)
        return s["dlogits"]
    if "tensors" not in s:                               # the list of gradients, kept while they stay where they are
        s["tensors"] = twa.Tensors(s["grads"])
        s["ws_bytes"] = twa.twa_grad_norm_workspace_bytes(s["tensors"])
    ws = _library(s["ws_bytes"])[2]
    twa.twa_clip_gather(ctx, s["tensors"], c["max_norm"], s["g"], s["norm"], ws, eps=CLIP_EPS)
    return {"g": s["g"], "norm": s["norm"]}


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "layer_norm":
        x = s["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = torch.rsqrt((d * d).mean(1) + EPS)
        y = d * rstd[:, None] * s["weight"].float() + s["bias"].float()
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if op == "layer_norm_backward":
        dy = s["dy"].float()
        xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        v = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (v - v.mean(1, keepdim=True) - xhat * (v * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dw": (dy * xhat).sum(0), "db": dy.sum(0)}
    if op == "embedding":
        return (s["table"][s["ids"].long()].float() * c["scale"]).to(s["out"].dtype)
    if op == "embedding_backward":
        keep = s["ids"] != c["padding"]
        rows = s["dout"].float() * (c["scale"] * keep)[:, None]
        total = torch.zeros((c["vocab"], c["dim"]), device=DEV).index_add_(0, s["ids"].long(), rows)
        if c["accumulate"]:
            total = total + s["before"].float()
        return total.to(s["dtable"].dtype)
    if op == "token_logprobs":
        z, t = s["logits"].float(), s["targets"].long()
        m = z.max(1).values
        m = torch.where(m == -math.inf, 0.0, m)
        d = z - m[:, None]
        e = torch.exp(d)
        total = e.sum(1)
        lse = m + torch.log(total)
        none = total == 0
        at = z.gather(1, t.clamp(min=0)[:, None])[:, 0]
        logp = torch.where(none, -math.inf, at - lse)
        out = {"logp": torch.where(t == IGNORE, 0.0, logp), "lse": lse}
        if c["entropy"]:
            h = torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1) / total
            out["entropy"] = torch.where(none, 0.0, h)
        k = min(c["top"], c["vocab"])
        if k:                                            # one number per value and place: equal values fall to the lowest index
            b = z.view(torch.int32).long()
            key = torch.where(b < 0, -(b & 0x7FFFFFFF), b) * (1 << 20) - torch.arange(c["vocab"], device=DEV)
            ids = key.topk(k, 1).indices
            top = z.gather(1, ids) - lse[:, None]
            out["top_ids"], out["top_logp"] = ids.int(), torch.where(none[:, None], -math.inf, top)
        return out
    if op == "token_logprobs_backward":
        z, t = s["logits"].float(), s["targets"].long()
        lse = torch.where(s["lse"] == -math.inf, 0.0, s["lse"])[:, None]
        live = t != IGNORE
        p = torch.exp(z - lse)
        dlp = torch.where(live & (s["lse"] > -math.inf), s["d_logp"], 0.0)
        dz = -dlp[:, None] * p
        dz.scatter_add_(1, t.clamp(min=0)[:, None], dlp[:, None])
        if c["entropy"]:
            dz = dz - s["d_entropy"][:, None] * torch.where(p > 0, p * (z - lse + s["entropy"][:, None]), 0.0)
        return dz.to(s["logits"].dtype)
    flat = torch.cat([t.float() for t in s["grads"]])
    norm = (flat * flat).sum().sqrt()
    factor = torch.clamp(c["max_norm"] / (norm + CLIP_EPS), max=1.0)
    return {"g": (flat * factor).to(s["g"].dtype), "norm": norm.reshape(1)}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- floors
def work(case):
    op = case["op"]
    if op.startswith("layer_norm"):
        n, e = case["rows"] * case["cols"], _SIZE[case["dtype"]]
        w = case["cols"] * _SIZE[case["wtype"]]
        if op == "layer_norm":
            return {"bytes": 2 * n * e + 2 * w + 8 * case["rows"], "flops": 8 * n}
        return {"bytes": 3 * n * e + w + 8 * case["cols"] + 8 * case["rows"], "flops": 14 * n}
    if op.startswith("embedding"):
        n = case["tokens"] * case["dim"]
        ids, act, row = case["tokens"] * _SIZE[case["ids"]], n * _SIZE[case["act"]], case["dim"] * _SIZE[case["table"]]
        if op == "embedding":                            # a row of the table is read once, however often it is looked up
            return {"bytes": ids + act + _distinct(case) * row, "flops": n}
        table = (2 if case["accumulate"] else 1) * case["vocab"] * row
        return {"bytes": ids + act + table, "flops": 2 * n}
    if op.startswith("token_logprobs"):
        n, rows = case["rows"] * case["vocab"], case["rows"]
        b = n * _SIZE[case["dtype"]] + rows * _SIZE[case["ids"]]
        if op == "token_logprobs":
            k = min(case["top"], case["vocab"])
            return {"bytes": b + rows * (8 + 4 * case["entropy"] + 8 * k), "flops": (6 if case["entropy"] else 4) * n}
        return {"bytes": b + n * _SIZE[case["dtype"]] + rows * (8 + 8 * case["entropy"]), "flops": (8 if case["entropy"] else 4) * n}
    total, sizes = 0, _sizes(case)
    for i, n in enumerate(sizes):
        total += n * (_SIZE[BF16 if i % 3 else F32] if case["grad"] == "mixed" else _SIZE[case["grad"]])
    return {"bytes": total + sum(sizes) * _SIZE[case["flat"]] + 4, "flops": 3 * sum(sizes)}


def _distinct(case):
    """Rows of the table that a lookup meets on average, by the tokens' distribution."""
    v, n = case["vocab"], case["tokens"]
    scale = math.log(v + 1)
    return sum(1.0 - (1.0 - math.log((r + 2) / (r + 1)) / scale) ** n for r in range(v))


# ------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions, row by row or token by token, in 64 bits."""
    s, op = prepare(case, seed), case["op"]
    if op == "layer_norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = torch.addcmul(s["bias"].double(), ((x.T - mean) * rstd).T, s["weight"].double())
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "layer_norm_backward":
        # vjp of w * xhat + b through xhat = (x - mean) rstd: P v rstd, P the projection off the constants and off xhat
        r, n = s["rstd"].double(), case["cols"]
        h = ((s["x"].double().T - s["mean"].double()) * r).T
        dy = s["dy"].double()
        v = dy * s["weight"].double()
        along = torch.einsum("rc,rc->r", v, h) / n
        dx = ((v.T - v.sum(1) / n - h.T * along) * r).T
        return {"dx": dx, "dw": torch.einsum("rc,rc->c", dy, h), "db": torch.einsum("rc->c", dy)}
    if op == "embedding":
        return torch.index_select(s["table"], 0, s["ids"].long()).double() * case["scale"]
    if op == "embedding_backward":
        out = s["before"].double() if case["accumulate"] else torch.zeros((case["vocab"], case["dim"]), dtype=torch.float64, device=DEV)
        token, order = torch.sort(s["ids"].long(), stable=True)
        run_sum = torch.cumsum(s["dout"].double()[order], 0)            # sums of a token's rows as differences of running sums
        last = torch.cat([token[1:] != token[:-1], torch.ones(1, dtype=torch.bool, device=DEV)])
        ends = run_sum[last]
        ends[1:] -= run_sum[last][:-1]
        token = token[last]
        live = token != case["padding"]
        out[token[live]] += case["scale"] * ends[live]
        return out
    if op == "token_logprobs":
        rows, k = case["rows"], min(case["top"], case["vocab"])
        got = {n: [] for n in ("logp", "lse", "entropy", "top_logp")}
        step = max(1, (1 << 26) // case["vocab"])
        for a in range(0, rows, step):
            z, t = s["logits"][a: a + step].double(), s["targets"][a: a + step].long()
            lse = torch.logsumexp(z, 1)
            lp = torch.where(lse[:, None] == -math.inf, -math.inf, z - lse[:, None])
            got["lse"].append(lse)
            got["logp"].append(torch.where(t == IGNORE, 0.0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0]))
            got["entropy"].append(-torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(1))
            if k:
                got["top_logp"].append(lp.topk(k, 1).values)
        out = {n: torch.cat(v) for n, v in got.items() if v}
        if not case["entropy"]:
            del out["entropy"]
        if k:
            out["top_ids"] = None                        # whole numbers: they have to be the plain form's
        return out
    if op == "token_logprobs_backward":
        out = torch.zeros((case["rows"], case["vocab"]), dtype=torch.float64, device=DEV)
        step = max(1, (1 << 26) // case["vocab"])
        for a in range(0, case["rows"], step):
            lse, t = s["lse"][a: a + step].double(), s["targets"][a: a + step].long()
            some = lse > -math.inf
            lp = torch.where(some[:, None], s["logits"][a: a + step].double() - lse[:, None], -math.inf)
            p = lp.exp()
            weight = torch.where((t != IGNORE) & some, s["d_logp"][a: a + step].double(), 0.0)
            one = torch.zeros_like(p).scatter_(1, t.clamp(min=0)[:, None], 1.0)
            out[a: a + step] = weight[:, None] * (one - p)
            if case["entropy"]:
                rest = torch.where(p > 0, lp + s["entropy"][a: a + step].double()[:, None], 0.0)
                out[a: a + step] -= s["d_entropy"][a: a + step].double()[:, None] * p * rest
        return out
    norm = math.sqrt(sum(torch.linalg.vector_norm(t.double()).item() ** 2 for t in s["grads"]))
    factor = min(1.0, case["max_norm"] / (norm + CLIP_EPS))
    g = torch.empty((s["g"].numel(),), dtype=torch.float64, device=DEV)
    at = 0
    for t in s["grads"]:
        torch.mul(t.double(), factor, out=g[at: at + t.numel()])
        at += t.numel()
    return {"g": g, "norm": torch.tensor([norm], dtype=torch.float64)}
