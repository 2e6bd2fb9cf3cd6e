"""What is measured of the operators that a sequence model needs beside those of perf/operators.py: the gated linear
recurrence, dropout, tokens sorted by expert, and the experts' results brought back with weights.

`own` false: every operator in its plain form, elementary torch operations in 32 bits (the recurrence in 64), rounded
             once at the end.
`own` true:  the library's entry points, as a training or serving program calls them.

A case is a dict: "op" names the operator and direction, the rest are its sizes and types.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
F32, BF16 = "f32", "bf16"
_DT = {F32: torch.float32, BF16: torch.bfloat16}
_SIZE = {F32: 4, BF16: 2, "i32": 4, "i64": 8}
SITE = 5                      # the dropout of a model that is drawn here


# ------------------------------------------------------------------------------------------- cases
def _named(name, c):
    return {"name": name, **c} if name else c


def _scan(name, train, sequences, tokens, channels, dtype, ragged=False, state=False, pad=0):
    # tokens: of all sequences together; ragged: lengths between about 1/50 and 3 times the mean, from offsets on the device
    # state: given and returned; pad: elements between rows (x, f, h as column blocks of a wider activation)
    return _named(name, {"op": "scan_train" if train else "scan", "sequences": sequences, "tokens": tokens, "channels": channels,
                         "dtype": dtype, "ragged": ragged, "state": state, "pad": pad})


def _drop(name, back, rows, cols, dtype, p, residual=False, pad=0):
    c = {"op": "dropout_backward" if back else "dropout", "rows": rows, "cols": cols, "dtype": dtype, "p": p, "pad": pad}
    if not back:
        c["residual"] = residual
    return _named(name, c)


def _moe(name, op, tokens, dim, top, experts, dtype, none=0.0, ids="i64", weights=True, pad=0):
    # none: share of the assignments that have no expert (dropped by a capacity limit)
    c = {"op": op, "tokens": tokens, "dim": dim, "top": top, "experts": experts, "dtype": dtype, "none": none, "pad": pad}
    if op == "dispatch":
        c["ids"] = ids
    if op == "combine":
        c["weights"] = weights
    return _named(name, c)


def listed():
    return [
        # one token of each of 64 sequences that are being generated: the state goes one step, latency counts
        _scan("scan step 64x2048 bf16", False, 64, 64, 2048, BF16, state=True),
        # a micro-batch of 8 sequences of 2048 tokens, forward and backward
        _scan("scan train 8x2048x2048 bf16", True, 8, 16384, 2048, BF16),
        # one long sequence in float32, few channels: little work side by side, a long axis
        _scan("scan train 1x65536x512 f32", True, 1, 65536, 512, F32),
        # prompts of uneven lengths read in, the state kept for the tokens to come; an odd width
        _scan("scan ragged 37x20011x771 bf16", False, 37, 20011, 771, BF16, ragged=True, state=True),
        # the tokens of one image behind a ViT-B/16 block, with the residual: latency counts
        _drop("dropout 197x768 bf16", False, 197, 768, BF16, 0.1, residual=True),
        # the residual stream of a large micro-batch
        _drop("dropout 32768x2048 bf16", False, 32768, 2048, BF16, 0.1, residual=True),
        # its gradient in float32, rows on no 16-byte boundary
        _drop("dropout bwd 4099x1023 f32", True, 4099, 1023, F32, 0.25),
        # sixteen tokens being generated, two experts of eight: latency counts
        _moe("dispatch 16x512 2 of 8 bf16", "dispatch", 16, 512, 2, 8, BF16, ids="i32"),
        # the largest: many fine experts
        _moe("dispatch 32768x2048 8 of 128 bf16", "dispatch", 32768, 2048, 8, 128, BF16),
        # an odd width in float32, some assignments dropped
        _moe("combine 1000x515 3 of 17 f32", "combine", 1000, 515, 3, 17, F32, none=0.1),
        # a training micro-batch, two experts a token
        _moe("combine 16384x1024 2 of 16 bf16", "combine", 16384, 1024, 2, 16, BF16, none=0.02),
        # the gradient through the weights, many experts a token
        _moe("combine bwd 16384x2048 8 of 64 bf16", "combine_backward", 16384, 2048, 8, 64, BF16),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["scan", "scan_train", "drop", "drop_bwd", "dispatch", "combine", "combine_backward"])
    dtype = rng.choice([F32, BF16, BF16])
    pad = rng.choice([0, 0, 8, 3])
    if op in ("scan", "scan_train"):
        channels = _log_int(rng, 16, 4096)
        if rng.random() < 0.6:
            channels = channels // 8 * 8
        tokens = _log_int(rng, 1, min(65536, (1 << 25) // channels))
        sequences = _log_int(rng, 1, min(tokens, 256))
        ragged = rng.random() < 0.5
        if not ragged:
            tokens = tokens // sequences * sequences
        return _scan("", op == "scan_train", sequences, tokens, channels, dtype, ragged, rng.random() < 0.5, pad)
    if op in ("drop", "drop_bwd"):
        cols = _log_int(rng, 8, 16384)
        if rng.random() < 0.6:
            cols = cols // 8 * 8
        rows = _log_int(rng, 1, min(65536, (1 << 26) // cols))
        return _drop("", op == "drop_bwd", rows, cols, dtype, rng.choice([0.05, 0.1, 0.2, 0.5]), rng.random() < 0.6, pad)
    dim = _log_int(rng, 16, 4096)
    if rng.random() < 0.6:
        dim = max(8, dim // 8 * 8)
    experts = _log_int(rng, 2, 256)
    top = rng.choice([t for t in (1, 2, 3, 4, 6, 8) if t <= experts])
    tokens = _log_int(rng, 1, min(32768, (1 << 28) // (dim * top)))
    return _moe("", op, tokens, dim, top, experts, dtype, rng.choice([0.0, 0.0, 0.1]), rng.choice(["i32", "i64"]), rng.random() < 0.6, pad)


# ------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 2654435761 % (1 << 62) + 1)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _matrix(values, dtype, pad):
    """The values in that type, rows `pad` elements apart."""
    rows, cols = values.shape
    buf = torch.zeros((rows, cols + pad), dtype=_DT[dtype], device=DEV)
    buf[:, :cols] = values
    return buf[:, :cols]


def _lengths(case):
    n, total = case["sequences"], case["tokens"]
    if not case["ragged"]:
        return [total // n] * n
    w = [math.exp(2.0 * math.cos(2.399963 * i + 1.0)) for i in range(n)]
    ends, at = [], 0.0
    for v in w:
        at += v
        ends.append(int(total * at / sum(w)))
    ends[-1] = total
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def _chosen(g, case):
    """Experts of every token, some in demand and some not; -1 where an assignment was dropped."""
    tokens, top, experts = case["tokens"], case["top"], case["experts"]
    ids = (_randn(g, tokens, experts) + 0.7 * _randn(g, experts)).topk(top, 1).indices
    if case["none"]:
        ids[torch.rand(ids.shape, generator=g, device=DEV) < case["none"]] = -1
    return ids


def _order(ids, experts):
    """Sort key and stable order of the assignments by expert, those without one at the end."""
    key = torch.where(ids < 0, experts, ids.long()).flatten()
    return torch.sort(key, stable=True)


def prepare(case, seed):
    g, op, dt, pad = _gen(seed), case["op"], _DT[case["dtype"]], case["pad"]
    s = {"case": case}
    if op in ("scan", "scan_train"):
        n, c, q = case["tokens"], case["channels"], case["sequences"]
        s["x"] = _matrix(_randn(g, n, c), case["dtype"], pad)
        # gates of channels that forget at once up to ones that remember some hundred tokens
        s["f"] = _matrix(1.5 * _randn(g, n, c) + 5.0 * torch.rand((c,), generator=g, device=DEV), case["dtype"], pad)
        s["h"] = _matrix(torch.zeros((n, c), device=DEV), case["dtype"], pad)
        s["lengths"] = _lengths(case)
        s["starts"] = torch.tensor([0] + s["lengths"], device=DEV).cumsum(0).int() if case["ragged"] else None
        s["first"] = torch.tensor([0] + s["lengths"][:-1], device=DEV).cumsum(0)
        s["h0"] = 0.5 * _randn(g, q, c) if case["state"] else None
        s["h_last"] = torch.empty((q, c), device=DEV) if case["state"] else None
        if op == "scan_train":
            s["dh"] = _matrix(0.01 * _randn(g, n, c), case["dtype"], pad)
            s["dx"], s["df"] = (_matrix(torch.zeros((n, c), device=DEV), case["dtype"], pad) for _ in range(2))
            s["d_last"] = 0.01 * _randn(g, q, c) if case["state"] else None
            s["dh0"] = torch.empty((q, c), device=DEV) if case["state"] else None
    elif op in ("dropout", "dropout_backward"):
        rows, cols = case["rows"], case["cols"]
        s["x"] = _matrix(_randn(g, rows, cols), case["dtype"], pad)
        s["residual"] = _matrix(2.0 * _randn(g, rows, cols), case["dtype"], pad) if case.get("residual") else None
        s["y"] = _matrix(torch.zeros((rows, cols), device=DEV), case["dtype"], pad)
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=g, device=DEV)
        s["rng"][1] %= 100000                                          # seed, step
    else:
        tokens, top, dim, experts = case["tokens"], case["top"], case["dim"], case["experts"]
        rows = tokens * top
        ids = _chosen(g, case)
        if op == "dispatch":
            s["ids"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
            s["x"] = _matrix(_randn(g, tokens, dim), case["dtype"], pad)
            s["place"] = torch.empty((tokens, top), dtype=torch.int32, device=DEV)
            s["starts"] = torch.empty((experts + 1,), dtype=torch.int32, device=DEV)
            s["order"] = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
            s["out"] = _matrix(torch.zeros((rows, dim), device=DEV), case["dtype"], pad)
        else:
            key, order = _order(ids, experts)
            place = torch.empty((rows,), dtype=torch.int32, device=DEV)
            place[order] = torch.where(key < experts, torch.arange(rows, device=DEV), -1).int()
            s["place"] = place.view(tokens, top)
            s["y"] = _matrix(_randn(g, rows, dim), case["dtype"], pad)
            s["weights"] = torch.softmax(_randn(g, tokens, top), 1) if case.get("weights", True) else None
            if op == "combine":
                s["out"] = _matrix(torch.zeros((tokens, dim), device=DEV), case["dtype"], pad)
            else:
                s["dout"] = _matrix(0.01 * _randn(g, tokens, dim), case["dtype"], pad)
                s["dy"] = _matrix(torch.zeros((rows, dim), device=DEV), case["dtype"], pad)
                s["dw"] = torch.empty((tokens, top), device=DEV)
    return s


# ------------------------------------------------------------------------------------------- one pass
_kept = {}


def _library():
    """The binding and a context on the current stream, kept as a program keeps them."""
    if "ctx" not in _kept:
        from paper_2205_13104_b200 import twa
        _kept["twa"], _kept["ctx"] = twa, twa.twa_create(0)
    return _kept["twa"], _kept["ctx"]


def _own(s):
    c, op = s["case"], s["case"]["op"]
    twa, ctx = _library()
    if op == "scan":
        twa.twa_gated_scan(ctx, s["x"], s["f"], s["h"], s["starts"], c["sequences"], s["h0"], s["h_last"])
        return {"h": s["h"], "h_last": s["h_last"]} if c["state"] else s["h"]
    if op == "scan_train":
        if "states" not in s:                            # what the forward call leaves for the backward one
            s["states"] = torch.empty(twa.twa_gated_scan_states_bytes(c["tokens"], c["sequences"], c["channels"]), dtype=torch.uint8,
                                      device=DEV)
        twa.twa_gated_scan(ctx, s["x"], s["f"], s["h"], s["starts"], c["sequences"], s["h0"], s["h_last"], s["states"])
        twa.twa_gated_scan_backward(ctx, s["dh"], s["x"], s["f"], s["states"], s["dx"], s["df"], s["starts"], c["sequences"],
                                    s["d_last"], s["dh0"])
        out = {k: s[k] for k in ("h", "dx", "df")}
        if c["state"]:
            out.update(h_last=s["h_last"], dh0=s["dh0"])
        return out
    if op == "dropout":
        twa.twa_dropout(ctx, s["x"], c["p"], s["rng"], SITE, s["y"], s["residual"])
        return s["y"]
    if op == "dropout_backward":
        twa.twa_dropout_backward(ctx, s["x"], c["p"], s["rng"], SITE, s["y"])
        return s["y"]
    if op == "dispatch":
        twa.twa_expert_dispatch(ctx, s["x"], s["ids"], c["experts"], s["place"], s["starts"], s["out"], s["order"])
        return {k: s[k] for k in ("place", "starts", "order", "out")}
    if op == "combine":
        twa.twa_expert_combine(ctx, s["y"], s["place"], s["weights"], s["out"])
        return s["out"]
    twa.twa_expert_combine_backward(ctx, s["dout"], s["y"], s["place"], s["weights"], s["dy"], s["dw"])
    return {"dy": s["dy"], "dw": s["dw"]}


def _recur(a, b, longest):
    """v_t = a_t v_{t-1} + b_t along the rows by doubling: after the round of distance d, b_t holds what the last 2 d rows give.
    A sequence begins where a_t is 0."""
    d = 1
    while d < longest:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _plain_scan(s):
    # in 64 bits: gates next to one are multiplied over thousands of tokens, and in 32 bits each has lost the digits of 1 - a
    c, n = s["case"], s["x"].shape[0]
    x, a = s["x"].double(), 1.0 / (1.0 + torch.exp(-s["f"].double()))
    some = torch.tensor([v > 0 for v in s["lengths"]], device=DEV)
    first = s["first"]
    at = torch.where(some, first, n)                     # rows where a sequence begins; n: one behind the rows, for empty ones
    begins = torch.zeros((n + 1,), dtype=torch.bool, device=DEV)
    begins[at] = True
    begins = begins[:n, None]
    h0 = torch.zeros((c["sequences"], c["channels"]), dtype=torch.float64, device=DEV) if s["h0"] is None else s["h0"].double()
    entry = torch.zeros((n + 1, c["channels"]), dtype=torch.float64, device=DEV)
    entry[at] = h0
    entry = entry[:n]                                    # the state that enters at those rows
    inner = torch.where(begins, 0.0, a)
    longest = max(s["lengths"])
    h = _recur(inner, (1.0 - a) * x + a * entry, longest)
    last = (first + torch.tensor(s["lengths"], device=DEV) - 1).clamp(min=0)
    dt = s["x"].dtype
    out = {"h": h.to(dt)}
    if c["state"]:
        out["h_last"] = torch.where(some[:, None], h[last], h0).float()
    if c["op"] == "scan":
        return out if c["state"] else out["h"]
    dh = s["dh"].double()
    if c["state"]:
        dh = dh.index_add(0, last, torch.where(some[:, None], s["d_last"].double(), 0.0))
    # G_t = dh_t + a_{t+1} G_{t+1}: the same recurrence over the rows in reverse order
    after = torch.cat([inner[1:], torch.zeros_like(a[:1])])
    grad = _recur(after.flip(0), dh.flip(0), longest).flip(0)
    before = torch.where(begins, entry, torch.cat([torch.zeros_like(h[:1]), h[:-1]]))
    out["dx"] = ((1.0 - a) * grad).to(dt)
    out["df"] = (a * (1.0 - a) * (before - x) * grad).to(dt)
    if c["state"]:
        f = first.clamp(max=n - 1)
        out["dh0"] = torch.where(some[:, None], a[f] * grad[f], s["d_last"].double()).float()
    return out


def _numbers(rng, rows, cols):
    """16 random bits for every element: the words of Philox4x32-10 with the counter (column / 8, row, SITE, step) and the
    seed as its key, low half first.  Products of 32-bit words fit the 64 bits of an integer as bit patterns."""
    low = 0xFFFFFFFF
    groups = (cols + 7) // 8
    c0 = torch.arange(groups, device=DEV).expand(rows, groups)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(rows, groups)
    c2 = torch.full((rows, groups), SITE, device=DEV)
    c3 = (rng[1] & low).expand(rows, groups)
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, groups * 8)[:, :cols]


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op in ("scan", "scan_train"):
        return _plain_scan(s)
    if op in ("dropout", "dropout_backward"):
        t = min(65535, int(round(c["p"] * 65536)))
        kept = _numbers(s["rng"], c["rows"], c["cols"]) >= t
        y = torch.where(kept, s["x"].float() * (65536.0 / (65536 - t)), 0.0)
        if s["residual"] is not None:
            y = s["residual"].float() + y
        return y.to(s["x"].dtype)
    if op == "dispatch":
        experts, rows = c["experts"], c["tokens"] * c["top"]
        key, order = _order(s["ids"], experts)
        live = key < experts
        place = torch.empty((rows,), dtype=torch.int32, device=DEV)
        place[order] = torch.where(live, torch.arange(rows, device=DEV), -1).int()
        starts = (key[None, :] < torch.arange(experts + 1, device=DEV)[:, None]).sum(1).int()
        out = torch.where(live[:, None], s["x"][order // c["top"]], 0.0).to(s["x"].dtype)
        return {"place": place.view(c["tokens"], c["top"]), "starts": starts, "order": torch.where(live, order, -1).int(), "out": out}
    place = s["place"].long()
    live = place >= 0
    rows = torch.where(live[..., None], s["y"][place.clamp(min=0)].float(), 0.0)         # tokens, top, dim
    if op == "combine":
        if s["weights"] is not None:
            rows = rows * s["weights"][..., None]
        return rows.sum(1).to(s["y"].dtype)
    dout = s["dout"].float()
    dy = torch.zeros((c["tokens"] * c["top"] + 1, c["dim"]), dtype=s["y"].dtype, device=DEV)
    dy[torch.where(live, place, c["tokens"] * c["top"])] = (s["weights"][..., None] * dout[:, None]).to(s["y"].dtype)
    return {"dy": dy[:-1], "dw": (rows * dout[:, None]).sum(2)}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- floors
def work(case):
    op, e = case["op"], _SIZE[case["dtype"]]
    if op in ("scan", "scan_train"):
        n = case["tokens"] * case["channels"]
        b = 3 * n * e + (4 * (case["sequences"] + 1) if case["ragged"] else 0)
        if case["state"]:
            b += 8 * case["sequences"] * case["channels"]
        if op == "scan":
            return {"bytes": b, "flops": 8 * n}
        b += 3 * n * e                                   # dh in, dx and df out
        if case["state"]:
            b += 8 * case["sequences"] * case["channels"]
        return {"bytes": b, "flops": 22 * n}
    if op in ("dropout", "dropout_backward"):
        n = case["rows"] * case["cols"]
        return {"bytes": (3 if case.get("residual") else 2) * n * e + 16, "flops": 2 * n}
    rows, n = case["tokens"] * case["top"], case["tokens"] * case["dim"] * e
    kept = int(n * case["top"] * (1.0 - case["none"]))   # the experts' rows
    if op == "dispatch":
        return {"bytes": n + kept + rows * (_SIZE[case["ids"]] + 8) + 4 * (case["experts"] + 1), "flops": 4 * rows}
    if op == "combine":
        return {"bytes": kept + n + rows * (8 if case["weights"] else 4), "flops": 2 * kept // e}
    return {"bytes": n + 2 * kept + 12 * rows, "flops": 3 * kept // e}


# ------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions: the recurrence token by token, the generator in numpy's unsigned words, the experts one by one."""
    s, op = prepare(case, seed), case["op"]
    if op in ("scan", "scan_train"):
        return _exact_scan(case, s)
    if op in ("dropout", "dropout_backward"):
        t = min(65535, int(round(case["p"] * 65536)))
        kept = torch.from_numpy(_exact_numbers(s["rng"].cpu().numpy(), case["rows"], case["cols"]) >= t).to(DEV)
        y = s["x"].double() * 65536.0 / (65536 - t)
        y = y.masked_fill_(~kept, 0.0)
        return y if s["residual"] is None else y + s["residual"]
    if op == "dispatch":
        out = torch.zeros((case["tokens"] * case["top"], case["dim"]), dtype=torch.float64, device=DEV)
        at = 0
        for e in range(case["experts"]):
            token = (s["ids"] == e).nonzero()[:, 0]      # in the order of the tokens
            out[at: at + len(token)] = s["x"][token].double()
            at += len(token)
        return {"place": None, "starts": None, "order": None, "out": out}
    w = s["weights"]
    if op == "combine":
        out = torch.zeros((case["tokens"], case["dim"]), dtype=torch.float64, device=DEV)
        for j in range(case["top"]):
            token = (s["place"][:, j] >= 0).nonzero()[:, 0]
            y = s["y"][s["place"][token, j].long()].double()
            out[token] += y if w is None else y * w[token, j].double()[:, None]
        return out
    dy = torch.zeros((case["tokens"] * case["top"], case["dim"]), dtype=torch.float64, device=DEV)
    dw = torch.zeros((case["tokens"], case["top"]), dtype=torch.float64, device=DEV)
    for j in range(case["top"]):
        token = (s["place"][:, j] >= 0).nonzero()[:, 0]
        row = s["place"][token, j].long()
        d = s["dout"][token].double()
        dy[row] = d * w[token, j].double()[:, None]
        dw[token, j] = torch.einsum("td,td->t", d, s["y"][row].double())
    return {"dy": dy, "dw": dw}


def _exact_scan(case, s):
    lengths, q, c = torch.tensor(s["lengths"], device=DEV), case["sequences"], case["channels"]
    longest = max(s["lengths"])
    step = torch.arange(longest, device=DEV)
    inside = step < lengths[:, None]
    row = (s["first"][:, None] + step)[inside]

    def apart(rows, fill):
        """sequences, tokens of the longest, channels; `fill` behind the end of the shorter ones."""
        out = torch.full((q, longest, c), fill, dtype=torch.float64, device=DEV)
        out[inside] = rows.double()[row]
        return out

    def together(padded):
        out = torch.zeros((case["tokens"], c), dtype=torch.float64, device=DEV)
        out[row] = padded[inside]
        return out

    def state(given):
        return torch.zeros((q, c), dtype=torch.float64, device=DEV) if given is None else given.double()

    a, x = torch.sigmoid(apart(s["f"], math.inf)), apart(s["x"], 0.0)          # behind the end the state stays
    h = torch.empty((longest + 1, q, c), dtype=torch.float64, device=DEV)
    h[0] = state(s["h0"])
    for t in range(longest):
        torch.lerp(x[:, t], h[t], a[:, t], out=h[t + 1])
    out = {"h": together(h[1:].transpose(0, 1))}
    if case["state"]:
        out["h_last"] = h[longest].clone()
    if case["op"] == "scan":
        return out if case["state"] else out["h"]
    dh, k = apart(s["dh"], 0.0), state(s["d_last"])
    for t in reversed(range(longest)):
        dh[:, t] += k                                    # now the gradient of h_t from its own output and all later ones
        k = a[:, t] * dh[:, t]
    slope = (1.0 - a) * dh
    out["dx"], out["df"] = together(slope), together(slope * a * (h[:-1].transpose(0, 1) - x))
    if case["state"]:
        out["dh0"] = k
    return out


def _exact_numbers(rng, rows, cols):
    groups, seed, step = (cols + 7) // 8, int(rng[0]), int(rng[1])
    u32 = np.uint32
    x = np.empty((4, rows, groups), u32)
    x[0], x[1], x[2], x[3] = np.arange(groups, dtype=u32), np.arange(rows, dtype=u32)[:, None], SITE, step & 0xFFFFFFFF
    for i in range(10):
        key0, key1 = u32((seed + i * 0x9E3779B9) & 0xFFFFFFFF), u32(((seed >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)
        a = x[0].astype(np.uint64) * np.uint64(0xD2511F53)
        b = x[2].astype(np.uint64) * np.uint64(0xCD9E8D57)
        x = np.stack([(b >> np.uint64(32)).astype(u32) ^ x[1] ^ key0, b.astype(u32), (a >> np.uint64(32)).astype(u32) ^ x[3] ^ key1, a.astype(u32)])
    return np.moveaxis(x, 0, -1).copy().view("<u2").reshape(rows, groups * 8)[:, :cols]
