"""The operators of a sequence model (gated scan, dropout, expert dispatch and combine) against their definitions in 64 bits, at
the sizes, types, strides and offsets where they can go wrong.

Tolerances are worst-case bounds of the arithmetic, element by element: U = 2^-24 is half a unit in the last place of float32,
and an output is rounded once to its type (relative 2^-8 for bfloat16, U for float32).
"""

import numpy as np
import pytest
import torch

from paper_2205_13104_b200 import twa
from philox import dropout_numbers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: U, BF16: 2.0 ** -8}
FILL = 7.0


@pytest.fixture(scope="module")
def ctx():
    torch.cuda.set_device(0)
    c = twa.twa_create(0)
    yield c
    twa.twa_destroy(c)


@pytest.fixture(autouse=True)
def clean(ctx):
    twa.twa_clear_status(ctx)
    yield
    twa.twa_clear_status(ctx)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def strided(values, dtype, pad=0, shift=0):
    """The matrix as a view whose rows are `pad` elements apart, beginning `shift` elements into a buffer of FILL."""
    rows, cols = values.shape
    buf = torch.full((shift + rows * (cols + pad),), FILL, dtype=dtype, device=DEV)
    view = buf[shift:].view(rows, cols + pad)[:, :cols]
    view.copy_(values)
    return buf, view


def blank(rows, cols, dtype, pad=0, shift=0):
    return strided(torch.full((rows, cols), FILL, device=DEV), dtype, pad, shift)


def untouched(buf, view, rows=None):
    """Nothing outside the view, or outside its rows marked in `rows`, was written."""
    keep = view.clone()
    if rows is None:
        view.fill_(FILL)
    else:
        view[rows] = FILL
    same = bool((buf == FILL).all())
    view.copy_(keep)
    return same


def close(got, want, tol):
    got = got.double()
    same = (got == want) | ((got - want).abs() <= tol)
    assert bool(same.all()), float(((got - want).abs() / tol)[~same].max())


def ok(ctx):
    assert twa.twa_get_status(ctx)[0] == 0


# ------------------------------------------------------------------------------------------- gated scan
def scan_64(x, f, lengths, first, h0, dh=None, d_last=None):
    """Definition and error bounds, sequence by sequence, token by token.  A dict of (value, bound) without the final rounding."""
    x, f = x.double(), f.double()
    a, b = torch.sigmoid(f), torch.sigmoid(-f)
    s = torch.minimum(a, b)
    # relative error of s: of the exponential (expf one unit; the fast one 2 + 1.2 |f| units), then of the sum and the quotient
    # (a gate beyond 128, an infinite one too: s is below 2^-184, zero in float32, so that its error counts for nothing)
    es = 2 * U * ((3.0 if x_dtype(x, f) == F32 else 0) + 3 + 1.2 * f.abs().clamp(max=128.0))
    n, c = x.shape
    q = len(lengths)
    zero = torch.zeros((q, c), dtype=torch.float64, device=DEV)
    h, eh, last, elast = torch.zeros_like(x), torch.zeros_like(x), zero.clone(), zero.clone()
    before, ebefore = torch.zeros_like(x), torch.zeros_like(x)
    size = torch.zeros_like(x)
    for i, (at, length) in enumerate(zip(first, lengths)):
        v, e = (zero[i] if h0 is None else h0[i].double()), zero[i]
        big = torch.maximum(v.abs(), x[at: at + length].abs().amax(0)) if length else v.abs()
        for t in range(at, at + length):
            before[t], ebefore[t], size[t] = v, e, big
            v = a[t] * v + b[t] * x[t]
            # a step's difference, product and sum, for the state and for the factor A; then the joins of segments
            e = a[t] * e + 4 * big * (s[t] * (U + es[t]) + U)
            h[t], eh[t] = v, e
        last[i], elast[i] = v, e + U * big
    out = {"h": (h, eh), "h_last": (last, elast)}
    if dh is None:
        return out
    dh = dh.double()
    g, eg, mag = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    k0, ek0 = zero.clone(), zero.clone()
    for i, (at, length) in enumerate(zip(first, lengths)):
        k = zero[i] if d_last is None else d_last[i].double()
        e, m = zero[i], k.abs()
        for t in reversed(range(at, at + length)):
            g[t], mag[t] = dh[t] + k, dh[t].abs() + m
            eg[t] = e + U * mag[t]
            k, m = a[t] * g[t], a[t] * mag[t]
            e = a[t] * eg[t] + 4 * mag[t] * (s[t] * (U + es[t]) + U)
        k0[i], ek0[i] = k, e + U * m
    slope, big = a * b, before.abs() + x.abs() + size
    out["dx"] = b * g, b * eg + (es + 4 * U) * b * mag + U * mag * b
    out["df"] = slope * (before - x) * g, slope * (big * eg + mag * (ebefore + 4 * U * big) + (es + 8 * U) * big * mag)
    out["dh0"] = k0, ek0
    return out


def x_dtype(x, f):
    return scan_64.dtype


LENGTHS = [[1], [2, 1, 3], [8], [9], [7, 0, 8, 1, 9, 0], [63, 64, 65], [129, 5, 128, 0, 200], [1] * 70, [3, 1, 2, 64, 1, 1, 8, 2, 1, 1, 9, 1],
           [700], [0, 0], [5] * 9, [64, 64, 64], [130, 130]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: "-".join(map(str, v))[:24])
@pytest.mark.parametrize("channels,dtype,pad,shift", [(64, BF16, 0, 0), (130, F32, 0, 0), (1, F32, 0, 0), (63, BF16, 3, 1), (70, BF16, 2, 2),
                                                      (200, F32, 1, 1), (257, BF16, 0, 0)])
@pytest.mark.parametrize("state", [False, True])
def test_gated_scan_and_its_gradient(ctx, lengths, channels, dtype, pad, shift, state):
    q = len(lengths)
    g = gen(sum(lengths) * 7 + channels + state)
    equal = len(set(lengths)) == 1
    lead, tail = (0, 0) if equal else (2, 3)                        # rows before the first and behind the last sequence
    n = lead + sum(lengths) + tail
    first = [lead + sum(lengths[:i]) for i in range(q)]
    rows = torch.zeros(n, dtype=torch.bool, device=DEV)
    rows[lead: n - tail] = True
    starts = None if equal else torch.tensor(first + [lead + sum(lengths)], device=DEV, dtype=torch.int32 if channels % 2 else torch.int64)
    _, x = strided(randn(g, n, channels), dtype, pad, shift)
    # gates from shut to open, some at either end of what a sigmoid has left of 32 bits
    fv = 2.0 * randn(g, n, channels) + 3.0 * randn(g, channels)
    fv[torch.rand(fv.shape, generator=g, device=DEV) < 0.02] = 200.0
    fv[torch.rand(fv.shape, generator=g, device=DEV) < 0.02] = -200.0
    _, f = strided(fv, dtype, pad, shift)
    _, dh = strided(0.1 * randn(g, n, channels), dtype, pad, shift)
    h0 = randn(g, q, channels) if state else None
    d_last = randn(g, q, channels) if state else None
    h_last = torch.full((q, channels), FILL, device=DEV) if state else None
    dh0 = torch.full((q, channels), FILL, device=DEV) if state else None
    hbuf, h = blank(n, channels, dtype, pad, shift)
    dxbuf, dx = blank(n, channels, dtype, pad, shift)
    dfbuf, df = blank(n, channels, dtype, pad, shift)
    size = twa.twa_gated_scan_states_bytes(n, q, channels)
    states = torch.full((size // 4 + 4,), FILL, device=DEV)
    twa.twa_gated_scan(ctx, x, f, h, starts, q, h0, h_last, states[:size // 4])
    twa.twa_gated_scan_backward(ctx, dh, x, f, states[:size // 4], dx, df, starts, q, d_last, dh0)
    scan_64.dtype = dtype
    want = scan_64(x, f, lengths, first, h0, dh, d_last)
    for name, got in (("h", h), ("dx", dx), ("df", df)):
        v, e = want[name]
        # values below the smallest normal numbers may be taken for zero
        close(got[rows], v[rows], (e + ROUND[dtype] * (v.abs() + e) + 1e-37)[rows])
    if state:
        close(h_last, want["h_last"][0], want["h_last"][1] + 1e-37)
        close(dh0, want["dh0"][0], want["dh0"][1] + 1e-37)
    for buf, view in ((hbuf, h), (dxbuf, dx), (dfbuf, df)):
        assert untouched(buf, view, rows)
    assert bool((states[size // 4:] == FILL).all())

    # again, bit for bit, without states, the state in place; then every output in the place of an input
    again = torch.empty_like(h)
    again.fill_(FILL)
    carried = None if h0 is None else h0.clone()
    twa.twa_gated_scan(ctx, x, f, again, starts, q, carried, carried)
    assert torch.equal(again, h) and (carried is None or torch.equal(carried, h_last))
    for dx_at, df_at in ((0, 1), (1, 2), (2, 0)):
        t = [strided(v, dtype, pad, shift)[1] for v in (dh, x, f)]
        twa.twa_gated_scan_backward(ctx, *t, states[:size // 4], t[dx_at], t[df_at], starts, q, d_last, dh0)
        assert torch.equal(t[dx_at][rows], dx[rows]) and torch.equal(t[df_at][rows], df[rows])
    for at in (0, 1):
        t = [strided(v, dtype, pad, shift)[1] for v in (x, f)]
        twa.twa_gated_scan(ctx, *t, t[at], starts, q, h0)
        assert torch.equal(t[at][rows], h[rows])
    ok(ctx)


@pytest.mark.parametrize("sequences,length,channels,dtype", [(1, 9000, 64, F32), (1, 5000, 200, BF16), (3, 3001, 96, BF16), (2, 2500, 1100, F32),
                                                             (700, 3, 130, BF16), (40, 100, 513, F32), (1, 20000, 33, BF16), (5, 1999, 450, F32)])
@pytest.mark.parametrize("ragged", [False, True])
def test_gated_scan_over_long_axes(ctx, sequences, length, channels, dtype, ragged):
    """Against doubling in 64 bits: many tiles, sequences side by side, few channels."""
    g = gen(length + channels)
    n = sequences * length
    cut = sorted(torch.randint(0, n + 1, (sequences - 1,), generator=torch.Generator().manual_seed(n)).tolist()) if ragged else \
        [i * length for i in range(1, sequences)]
    edges = [0] + cut + [n]
    lengths = [b - a for a, b in zip(edges, edges[1:])]
    x, dh = randn(g, n, channels).to(dtype), (0.1 * randn(g, n, channels)).to(dtype)
    f = (1.5 * randn(g, n, channels) + 4.0 * torch.rand((channels,), generator=g, device=DEV)).to(dtype)
    h0, d_last = randn(g, sequences, channels), randn(g, sequences, channels)
    h, dx, df = (torch.empty_like(x) for _ in range(3))
    h_last, dh0 = torch.empty_like(h0), torch.empty_like(h0)
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, sequences, channels), dtype=torch.uint8, device=DEV)
    starts = torch.tensor(edges, device=DEV) if ragged else None
    twa.twa_gated_scan(ctx, x, f, h, starts, sequences, h0, h_last, states)
    twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, sequences, d_last, dh0)
    x64, f64 = x.double(), f.double()
    a, b = torch.sigmoid(f64), torch.sigmoid(-f64)
    s = torch.minimum(a, b)
    es = 2 * U * (6 + 1.2 * f64.abs())
    some = torch.tensor([v > 0 for v in lengths], device=DEV)
    first, last = torch.tensor(edges[:-1], device=DEV)[some], (torch.tensor(edges[1:], device=DEV) - 1)[some]
    inner = a.clone()
    inner[first] = 0.0

    def recur(decay, v):
        d = 1
        while d < max(lengths):
            v = torch.cat([v[:d], v[d:] + decay[d:] * v[:-d]])
            decay = torch.cat([decay[:d], decay[d:] * decay[:-d]])
            d *= 2
        return v

    entry = torch.zeros_like(a)
    entry[first] = h0[some].double()
    h64 = recur(inner, b * x64 + a * entry)
    big = max(float(x64.abs().max()), float(h0.abs().max()))
    eh = recur(inner, 4 * big * (s * (U + es) + U))                  # as scan_64 bounds it
    close(h, h64, eh + ROUND[dtype] * (h64.abs() + eh))
    want_last = h0.double()
    want_last[some] = h64[last]
    elast = torch.zeros_like(want_last)
    elast[some] = eh[last] + U * big
    close(h_last, want_last, elast)
    d = dh.double()
    d[last] += d_last[some].double()
    mag = dh.double().abs()
    mag[last] += d_last[some].double().abs()
    after = torch.cat([inner[1:], torch.zeros_like(a[:1])]).flip(0)
    g64, mag = recur(after, d.flip(0)).flip(0), recur(after, mag.flip(0)).flip(0)
    eg = recur(after, (4 * mag * (s * (U + es) + 2 * U)).flip(0)).flip(0)
    before = torch.cat([torch.zeros_like(a[:1]), h64[:-1]])
    before[first] = h0[some].double()
    ebefore = torch.cat([torch.zeros_like(a[:1]), eh[:-1]])
    close(dx, b * g64, b * eg + (es + 5 * U) * b * mag + ROUND[dtype] * (b * g64.abs() + b * eg))
    want = a * b * (before - x64) * g64
    e = a * b * (3 * big * eg + mag * (ebefore + 12 * U * big) + (es + 8 * U) * 3 * big * mag)
    close(df, want, e + ROUND[dtype] * (want.abs() + e))
    want = d_last.double()
    want[some] = (a * g64)[first]
    e = torch.zeros_like(want)
    e[some] = (a * eg + 4 * mag * (s * (U + es) + 2 * U))[first]
    close(dh0, want, e)
    keep = [t.clone() for t in (h, h_last, dx, df, dh0)]
    twa.twa_gated_scan(ctx, x, f, h, starts, sequences, h0, h_last, states)
    twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, sequences, d_last, dh0)
    assert all(torch.equal(p, t) for p, t in zip(keep, (h, h_last, dx, df, dh0)))
    ok(ctx)


@pytest.mark.parametrize("cluster", [1, 2, 8])
@pytest.mark.parametrize("channels", [16, 32, 64])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gated_scan_however_it_is_shared(ctx, cluster, channels, dtype):
    """Every number of blocks along a sequence and of channels a block, with ragged sequences, tails of channels and empty sequences."""
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, cluster)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CHANNELS, channels)
    try:
        for state in (False, True):
            test_gated_scan_and_its_gradient(ctx, [700, 1, 0, 1025, 130], 72, dtype, 0, 0, state)
            test_gated_scan_and_its_gradient(ctx, [2100], 24, dtype, 8, 8, state)
            test_gated_scan_and_its_gradient(ctx, [129, 400, 64], 71, dtype, 0, 1, state)
    finally:
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, 0)
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CHANNELS, 0)


def test_gated_scan_of_constant_gates_keeps_its_digits(ctx):
    """A gate next to one over many tokens: h_t = 1 - a^t for x = 1.  A gate held as a float32 would be off by 2^-25 each step."""
    n, q = 40000, torch.tensor([8.0, 9.0, 10.0, 11.0], device=DEV)
    f = q.expand(n, 4).contiguous()
    x, h = torch.ones_like(f), torch.empty_like(f)
    twa.twa_gated_scan(ctx, x, f, h)
    t = torch.arange(1, n + 1, device=DEV, dtype=torch.float64)[:, None]
    want = -torch.expm1(-t * torch.log1p(torch.exp(-f.double())))
    # a product's and a sum's rounding a token, of independent sign, over the tokens remembered, and the error of s itself: far less
    # than the 1 - a = 1.7e-5 .. 3.4e-4 apart a step is.  A rounded gate would be off by up to 2^-25 / 1.7e-5 = 1.8e-3.
    assert float((h.double() - want).abs().max()) < 1e-4
    ok(ctx)


def test_gated_scan_gradient_against_differences(ctx):
    g = gen(3)
    lengths = [5, 70, 1]
    n, c, q = sum(lengths), 6, 3
    x, f, dh, h0, d_last = randn(g, n, c), 2 * randn(g, n, c), randn(g, n, c), randn(g, q, c), randn(g, q, c)
    starts = torch.tensor([0, 5, 75, 76], device=DEV)
    h, dx, df, dh0 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, q, c), dtype=torch.uint8, device=DEV)
    twa.twa_gated_scan(ctx, x, f, h, starts, q, h0, None, states)
    twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, q, d_last, dh0)
    edges = starts.tolist()

    def loss(x, f, h0):
        total = 0.0
        a = torch.sigmoid(f)
        for i in range(q):
            v = h0[i]
            for t in range(edges[i], edges[i + 1]):
                v = a[t] * v + (1 - a[t]) * x[t]
                total = total + (v * dh[t]).sum()
            total = total + (v * d_last[i]).sum()
        return float(total)

    # central differences of step 1e-4 in 64 bits: the third derivative's share is below 1e-6 of gradients of order one
    args = [x.double(), f.double(), h0.double()]
    for which, grad in enumerate((dx, df, dh0)):
        for i in range(0, args[which].numel(), 37 if which < 2 else 5):
            up, down = [v.clone() for v in args], [v.clone() for v in args]
            up[which].view(-1)[i] += 1e-4
            down[which].view(-1)[i] -= 1e-4
            assert abs((loss(*up) - loss(*down)) / 2e-4 - float(grad.view(-1)[i])) < 3e-5
    ok(ctx)


def test_gated_scan_token_by_token_is_the_scan(ctx):
    """A sequence that is generated, one call a token with the state in place, against the whole sequence at once."""
    g = gen(9)
    q, n, c = 5, 150, 96
    x, f, h0 = randn(g, q, n, c), 2 * randn(g, q, n, c) + 2, randn(g, q, c)
    whole, last = torch.empty(q * n, c, device=DEV), torch.empty_like(h0)
    twa.twa_gated_scan(ctx, x.view(-1, c), f.view(-1, c), whole, None, q, h0, last)
    state = h0.clone()
    out = torch.empty(q, n, c, device=DEV)
    for t in range(n):
        twa.twa_gated_scan(ctx, x[:, t], f[:, t], out[:, t], None, q, state, state)      # rows n * c elements apart
    lengths, first = [n] * q, [i * n for i in range(q)]
    scan_64.dtype = F32
    want, e = scan_64(x.view(-1, c), f.view(-1, c), lengths, first, h0)["h"]
    close(whole, want, e + U * want.abs())
    close(out.view(-1, c), want, e + U * want.abs())
    close(state, last.double(), 2 * (e.view(q, n, c)[:, -1] + U * 5))
    ok(ctx)


def test_gated_scan_keeps_what_is_not_finite_to_its_channel_and_sequence(ctx):
    g = gen(4)
    n, c = 300, 70
    x, f = randn(g, n, c), randn(g, n, c)
    clean_h, h = torch.empty_like(x), torch.empty_like(x)
    starts = torch.tensor([0, 100, 300], device=DEV)
    twa.twa_gated_scan(ctx, x, f, clean_h, starts, 2)
    x[120, 7], f[30, 9], x[299, 69] = float("nan"), float("nan"), float("inf")
    twa.twa_gated_scan(ctx, x, f, h, starts, 2)
    spoilt = torch.zeros(n, c, dtype=torch.bool, device=DEV)
    spoilt[120:, 7] = spoilt[30:100, 9] = spoilt[299:, 69] = True
    assert torch.equal(h[~spoilt], clean_h[~spoilt])
    assert not bool(torch.isfinite(h[spoilt]).any())
    ok(ctx)


@pytest.mark.parametrize("edges", [[0, 5, 3, 20], [-1, 5, 10, 20], [0, 5, 21, 22], [0, 10, 10, 1 << 40]])
@pytest.mark.parametrize("few", [False, True])
def test_gated_scan_reports_wrong_starts(ctx, edges, few):
    n, c = 20, 8
    x = torch.ones(n, c, device=DEV)
    if not few:
        edges = edges + [edges[-1]] * 40                              # mostly short sequences: the other launch
    q = len(edges) - 1
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, q, c), dtype=torch.uint8, device=DEV)
    starts = torch.tensor(edges, device=DEV)
    good = [i for i in range(q) if 0 <= edges[i] <= edges[i + 1] <= n]
    bad = [i for i in range(q) if i not in good]
    mine = torch.zeros(n, dtype=torch.bool, device=DEV)
    for i in good:
        mine[edges[i]: edges[i + 1]] = True
    for back in (False, True):
        h, dx, last = torch.full_like(x, FILL), torch.full_like(x, FILL), torch.full((q, c), FILL, device=DEV)
        if back:
            states.zero_()
            twa.twa_gated_scan_backward(ctx, x, x, x, states, h, dx, starts, q, None, last)
        else:
            twa.twa_gated_scan(ctx, x, x, h, starts, q, None, last, states)
        code, detail = twa.twa_get_status(ctx)
        assert code == twa.TWA_ERR_INVALID_ARG and detail in bad
        assert bool((h[~mine] == FILL).all()) and not bool((h[mine] == FILL).any())
        assert bool((last[bad] == FILL).all()) and not bool((last[good] == FILL).any())
        twa.twa_clear_status(ctx)


# ------------------------------------------------------------------------------------------- dropout
DROP_SIZES = [(1, 1), (1, 8), (3, 7), (5, 31), (197, 768), (1000, 129), (33, 512), (9, 1023), (2, 40001), (2, 40000), (3001, 24), (1, 257), (700, 2048)]


@pytest.mark.parametrize("rows,cols", DROP_SIZES)
@pytest.mark.parametrize("dtype,pad,shift", [(F32, 0, 0), (BF16, 0, 0), (BF16, 8, 8), (F32, 3, 1), (BF16, 5, 3)])
def test_dropout_and_its_gradient(ctx, rows, cols, dtype, pad, shift):
    g = gen(rows + cols)
    seed, step, site, p = -5 * rows + (cols << 33), (1 << 32) * 3 + rows, cols * 1000003 % (1 << 32), 0.1 + 0.3 * (rows % 3)
    rng = torch.tensor([seed, step], device=DEV)
    t = round(p * 65536)
    kept = torch.from_numpy(dropout_numbers(seed, step, site, rows, cols) >= t).to(DEV)
    scale = 65536 / (65536 - t)
    xv, rv = randn(g, rows, cols), randn(g, rows, cols)
    xv[~kept & (torch.rand(xv.shape, generator=g, device=DEV) < 0.1)] = float("nan")      # what is dropped does not count
    _, x = strided(xv, dtype, pad, shift)
    _, res = strided(rv, dtype, pad, shift)
    for residual in (None, res):
        ybuf, y = blank(rows, cols, dtype, pad, shift)
        twa.twa_dropout(ctx, x, p, rng, site, y, residual)
        want = torch.where(kept, x.double() * scale, 0.0) + (0.0 if residual is None else residual.double())
        # the scale rounded once, the product and sum once, then the type
        terms = torch.where(kept, x.double().abs() * scale, 0.0)
        close(y, want, ROUND[dtype] * want.abs() + 2 * U * (terms + want.abs()) * (1 + ROUND[dtype]))
        assert untouched(ybuf, y)
        first = y.clone()
        for at in (0, 1):
            t2 = [strided(v, dtype, pad, shift)[1] for v in (x, res)]
            twa.twa_dropout(ctx, t2[0], p, rng, site, t2[at if residual is not None else 0], None if residual is None else t2[1])
            assert torch.equal(t2[at if residual is not None else 0], first)
    dxbuf, dx = blank(rows, cols, dtype, pad, shift)
    dyv = randn(g, rows, cols)
    _, dy = strided(dyv, dtype, pad, shift)
    twa.twa_dropout_backward(ctx, dy, p, rng, site, dx)
    want = torch.where(kept, dy.double() * scale, 0.0)
    close(dx, want, ROUND[dtype] * want.abs() + 3 * U * want.abs())
    assert untouched(dxbuf, dx)
    ok(ctx)


@pytest.mark.parametrize("rows,cols", [(7, 1), (5, 2), (300, 255), (31, 256), (9, 257), (64, 515), (3, 4099)])
def test_dropout_of_rows_at_other_places_between_words(ctx, rows, cols):
    """bfloat16 matrices whose rows begin on 4-byte words and between them, alike in all matrices or not."""
    g = gen(rows * cols)
    rng = torch.tensor([9, 8], device=DEV)
    kept = torch.from_numpy(dropout_numbers(9, 8, 7, rows, cols) >= 32768).to(DEV)
    xv, rv = randn(g, rows, cols), randn(g, rows, cols)
    for places in (((0, 0),) * 3, ((0, 1),) * 3, ((1, 1),) * 3, ((2, 1), (4, 3), (0, 1)), ((1, 1), (3, 3), (1, 1)), ((0, 0), (0, 1), (0, 0)), ((1, 0), (0, 0), (1, 0))):
        (_, x), (_, res) = strided(xv, BF16, *places[0]), strided(rv, BF16, *places[1])
        for residual in (None, res):
            ybuf, y = blank(rows, cols, BF16, *places[2])
            twa.twa_dropout(ctx, x, 0.5, rng, 7, y, residual)
            want = torch.where(kept, 2 * x.float(), 0.0) + (0.0 if residual is None else residual.float())
            assert torch.equal(y, want.to(BF16))                      # twice a value and one sum: rounded as float32 does
            assert untouched(ybuf, y)
    ok(ctx)


def test_dropout_at_the_ends_of_its_probability(ctx):
    x = torch.ones(64, 1024, device=DEV)
    rng, y = torch.tensor([1, 2], device=DEV), torch.empty(64, 1024, device=DEV)
    numbers = torch.from_numpy(dropout_numbers(1, 2, 3, 64, 1024).astype(np.int64)).to(DEV)
    twa.twa_dropout(ctx, x, 0.0, rng, 3, y)
    assert torch.equal(y, x)
    twa.twa_dropout(ctx, x, 2.0 ** -18, rng, 3, y)                      # below half a step: nothing is dropped
    assert torch.equal(y, x)
    twa.twa_dropout(ctx, x, 1.0 - 2.0 ** -24, rng, 3, y)                # one number of 65536 is left
    assert torch.equal(y, torch.where(numbers == 65535, 65536.0, 0.0))
    twa.twa_dropout(ctx, x, 0.5, rng, 3, y)
    assert torch.equal(y, torch.where(numbers >= 32768, 2.0, 0.0))
    assert abs(float(y.mean()) - 1) < 6 / 256                          # 65536 draws of deviation one
    ok(ctx)


def test_dropout_draws_anew_from_a_graph_and_by_site(ctx):
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        own = twa.twa_create(0)
        x, rng = torch.ones(300, 200, device=DEV), torch.tensor([77, 0], device=DEV)
        y = [torch.empty_like(x) for _ in range(2)]
        back = torch.empty_like(x)

        def step():
            rng[1] += 1
            for site in (0, 1):
                twa.twa_dropout(own, x, 0.3, rng, site, y[site])
            twa.twa_dropout_backward(own, x, 0.3, rng, 1, back)

        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        seen = []
        for replay in range(3):
            graph.replay()
            stream.synchronize()
            for site in (0, 1):
                kept = torch.from_numpy(dropout_numbers(77, int(rng[1]), site, 300, 200) >= round(0.3 * 65536)).to(DEV)
                assert torch.equal(y[site] != 0, kept)
                seen.append(kept)
            assert torch.equal(back, y[1])
        assert not any(torch.equal(a, b) for i, a in enumerate(seen) for b in seen[:i])
        assert twa.twa_get_status(own)[0] == 0
        del graph
        twa.twa_destroy(own)
    torch.cuda.current_stream().wait_stream(stream)


# ------------------------------------------------------------------------------------------- experts
def chosen(g, tokens, top, experts, none=0.0):
    ids = (randn(g, tokens, experts) + randn(g, experts)).topk(min(top, experts), 1).indices if top <= experts else \
        torch.randint(0, experts, (tokens, top), generator=g, device=DEV)
    ids[torch.rand(ids.shape, generator=g, device=DEV) < none] = -1
    return ids


def sorted_64(ids, experts):
    """place, starts and order by a stable sort."""
    flat = ids.long().flatten()
    key = torch.where((flat < 0) | (flat >= experts), experts, flat)
    order = torch.sort(key, stable=True).indices
    live = int((key < experts).sum())
    place = torch.full_like(flat, -1)
    place[order[:live]] = torch.arange(live, device=DEV)
    starts = torch.tensor([int((key < e).sum()) for e in range(experts + 1)], device=DEV)
    return place.view(ids.shape).int(), starts.int(), order[:live].int()


EXPERT_SIZES = [(1, 1, 1, 8), (1, 2, 8, 512), (16, 2, 8, 512), (5, 3, 3, 7), (100, 4, 64, 129), (1000, 2, 17, 40), (513, 1, 1024, 16), (999, 8, 600, 33),
                (4097, 8, 256, 24), (30000, 6, 100, 8), (7, 32, 5, 12), (2000, 1, 2, 1000), (65, 2, 4, 4100)]


@pytest.mark.parametrize("tokens,top,experts,dim", EXPERT_SIZES)
@pytest.mark.parametrize("dtype,itype,none,pad,shift", [(BF16, torch.int64, 0.0, 0, 0), (F32, torch.int32, 0.2, 0, 0), (BF16, torch.int32, 0.1, 5, 3),
                                                        (F32, torch.int64, 0.0, 1, 1), (BF16, torch.int64, 0.5, 2, 2)])
def test_dispatch_and_combine(ctx, tokens, top, experts, dim, dtype, itype, none, pad, shift):
    g = gen(tokens + experts)
    ids = chosen(g, tokens, top, experts, none).to(itype)
    _, x = strided(randn(g, tokens, dim), dtype, pad, shift)
    n = tokens * top
    obuf, out = blank(n + 3, dim, dtype, pad, shift)
    place = torch.full((tokens, top), -7, dtype=torch.int32, device=DEV)
    starts, order = torch.full((experts + 1,), -7, dtype=torch.int32, device=DEV), torch.full((n,), -7, dtype=torch.int32, device=DEV)
    twa.twa_expert_dispatch(ctx, x, ids, experts, place, starts, out, order)
    place64, starts64, order64 = sorted_64(ids, experts)
    live = len(order64)
    assert torch.equal(place, place64) and torch.equal(starts, starts64)
    assert torch.equal(order[:live], order64) and bool((order[live:] == -7).all())
    assert torch.equal(out[:live], x[order64.long() // top])
    mine = torch.arange(n + 3, device=DEV) < live
    assert untouched(obuf, out, mine)
    only = torch.empty_like(place)
    twa.twa_expert_dispatch(ctx, None, ids, experts, only, starts, None)      # places only, no order
    assert torch.equal(only, place)

    # what the experts made of the rows, brought back; rows that no place names hold NaN
    _, y = strided(randn(g, n + 3, dim), dtype, pad, shift)
    y[live:] = float("nan")
    weights = torch.softmax(randn(g, tokens, top), 1)
    weights[place < 0] = float("nan")                                        # of no consequence
    rows = torch.where((place >= 0)[..., None], y[place.long().clamp(min=0)].double(), 0.0)
    w64 = torch.where(place >= 0, weights.double(), 0.0)
    for w in (weights, None):
        bbuf, back = blank(tokens, dim, dtype, pad, shift)
        twa.twa_expert_combine(ctx, y, place, w, back)
        terms = rows * (w64 if w is not None else 1.0 * (place >= 0))[..., None]
        want = terms.sum(1)
        close(back, want, ROUND[dtype] * want.abs() + 2 * top * U * terms.abs().sum(1) + 1e-37)
        assert untouched(bbuf, back)
    _, dout = strided(randn(g, tokens, dim), dtype, pad, shift)
    dybuf, dy = blank(n + 3, dim, dtype, pad, shift)
    dw = torch.full((tokens, top), FILL, device=DEV)
    twa.twa_expert_combine_backward(ctx, dout, y, place, weights, dy, dw)
    prod = rows * dout.double()[:, None]
    close(dw, prod.sum(2), (dim + 8) * U * prod.abs().sum(2) + 1e-37)
    want = torch.zeros(n + 3, dim, dtype=torch.float64, device=DEV)
    flat = place.flatten().long()
    grads = (w64[..., None] * dout.double()[:, None]).view(n, dim)
    want[flat[flat >= 0]] = grads[flat >= 0]
    close(dy[:live], want[:live], (ROUND[dtype] + U) * want[:live].abs() + 1e-37)
    assert untouched(dybuf, dy, mine)
    first = dy[:live].clone(), dw.clone()
    held = strided(y, dtype, pad, shift)[1]
    twa.twa_expert_combine_backward(ctx, dout, held, place, weights, held)            # in the place of y, without dw
    assert torch.equal(held[:live], first[0])
    twa.twa_expert_combine_backward(ctx, dout, y, place, weights, dy, dw)
    assert torch.equal(dy[:live], first[0]) and torch.equal(dw, first[1])
    ok(ctx)


@pytest.mark.parametrize("tokens", [3000, 20011])
def test_combine_gradient_of_many_tokens(ctx, tokens):
    """More tokens than blocks for each of them: a token a warp."""
    test_dispatch_and_combine(ctx, tokens, 5, 40, 136, BF16, torch.int64, 0.1, 0, 0)
    test_dispatch_and_combine(ctx, tokens, 9, 40, 35, F32, torch.int32, 0.1, 1, 1)


@pytest.mark.parametrize("count,experts", [(1 << 20, 256), (700001, 1000), (300000, 1)])
def test_sort_of_many_assignments(ctx, count, experts):
    g = gen(count)
    ids = torch.randint(-1, experts, (count, 1), generator=g, device=DEV)
    place, starts = torch.empty((count, 1), dtype=torch.int32, device=DEV), torch.empty(experts + 1, dtype=torch.int32, device=DEV)
    order = torch.empty(count, dtype=torch.int32, device=DEV)
    twa.twa_expert_dispatch(ctx, None, ids, experts, place, starts, None, order)
    place64, starts64, order64 = sorted_64(ids, experts)
    assert torch.equal(place, place64) and torch.equal(starts, starts64) and torch.equal(order[: len(order64)], order64)
    ok(ctx)


def test_experts_with_nothing_and_with_wrong_numbers(ctx):
    starts = torch.full((5,), 9, dtype=torch.int32, device=DEV)
    none = torch.empty((0, 2), dtype=torch.int32, device=DEV)
    empty = torch.empty(0, 8, device=DEV)
    twa.twa_expert_dispatch(ctx, empty, none, 4, none, starts, empty)
    assert bool((starts == 0).all())
    twa.twa_expert_combine(ctx, empty, none, None, empty)
    twa.twa_expert_combine_backward(ctx, empty, empty, none, torch.empty(0, 2, device=DEV), empty)
    # no assignment at all: nothing is copied, sums are zero
    place, out, x = torch.empty((6, 2), dtype=torch.int32, device=DEV), torch.full((12, 8), FILL, device=DEV), torch.ones(6, 8, device=DEV)
    twa.twa_expert_dispatch(ctx, x, torch.full((6, 2), -1, device=DEV), 4, place, starts, out)
    assert bool((place == -1).all()) and bool((starts == 0).all()) and bool((out == FILL).all())
    back, dw = torch.full((6, 8), FILL, device=DEV), torch.full((6, 2), FILL, device=DEV)
    twa.twa_expert_combine(ctx, out, place, dw, back)
    assert bool((back == 0).all())
    twa.twa_expert_combine_backward(ctx, x, out, place, dw.clone(), out, dw)
    assert bool((dw == 0).all()) and bool((out == FILL).all())
    ok(ctx)
    # ids outside the experts count as none and are reported by their token
    ids = torch.tensor([[0, 3], [4, 1], [2, 2], [-2, 1 << 40], [3, 3], [-1, 0]], device=DEV)
    twa.twa_expert_dispatch(ctx, x, ids, 4, place, starts, out)
    code, detail = twa.twa_get_status(ctx)
    assert code == twa.TWA_ERR_INVALID_ARG and detail in (1, 3)
    want = sorted_64(ids, 4)
    assert torch.equal(place, want[0]) and torch.equal(starts, want[1])
    twa.twa_clear_status(ctx)
    # so are places that are not among the rows
    place[2, 1], place[4, 0] = 12, 2 ** 31 - 1
    y, w = torch.ones(12, 8, device=DEV), torch.ones(6, 2, device=DEV)
    twa.twa_expert_combine(ctx, y, place, w, back)
    code, detail = twa.twa_get_status(ctx)
    assert code == twa.TWA_ERR_INVALID_ARG and detail in (2, 4)
    good = (place >= 0) & (place < 12)
    assert torch.equal(back[:, 0], good.sum(1).float())
    twa.twa_clear_status(ctx)
    twa.twa_expert_combine_backward(ctx, x, y, place, w, torch.empty_like(y), dw)
    code, detail = twa.twa_get_status(ctx)
    assert code == twa.TWA_ERR_INVALID_ARG and detail in (2, 4)
    assert torch.equal(dw, 8.0 * good)


# ------------------------------------------------------------------------------------------- together
def test_operators_replay_from_a_graph_on_another_stream(ctx):
    g = gen(12)
    n, c, top, experts = 512, 64, 2, 8
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        own = twa.twa_create(0)
        x, f, logits = randn(g, n, c), randn(g, n, c), randn(g, n, experts)
        rng = torch.tensor([5, 0], device=DEV)
        h, dropped, back, dh, dx, df = (torch.empty(n, c, device=DEV) for _ in range(6))
        states = torch.empty(twa.twa_gated_scan_states_bytes(n, 4, c), dtype=torch.uint8, device=DEV)
        place, starts = torch.empty((n, top), dtype=torch.int32, device=DEV), torch.empty(experts + 1, dtype=torch.int32, device=DEV)
        rows, dy, dw = torch.empty(n * top, c, device=DEV), torch.empty(n * top, c, device=DEV), torch.empty(n, top, device=DEV)
        outs = (h, dropped, place, starts, rows, back, dy, dw, dh, dx, df)

        def step():
            w, ids = torch.softmax(logits, 1).topk(top, 1)
            twa.twa_gated_scan(own, x, f, h, None, 4, states=states)
            twa.twa_dropout(own, h, 0.2, rng, 0, dropped, x)
            twa.twa_expert_dispatch(own, dropped, ids, experts, place, starts, rows)
            twa.twa_expert_combine(own, rows, place, w, back)
            twa.twa_expert_combine_backward(own, back, rows, place, w, dy, dw)
            twa.twa_expert_combine(own, dy, place, None, dh)
            twa.twa_dropout_backward(own, dh, 0.2, rng, 0, dh)
            twa.twa_gated_scan_backward(own, dh, x, f, states, dx, df, None, 4)

        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for _ in range(3):
            x.copy_(randn(g, n, c))
            logits.copy_(randn(g, n, experts))
            step()
            want = [t.clone() for t in outs]
            for t in outs:
                t.zero_()
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(want, outs))
        assert twa.twa_get_status(own)[0] == 0
        del graph
        twa.twa_destroy(own)
    torch.cuda.current_stream().wait_stream(stream)


def test_gated_scan_with_shut_gates_begins_anew(ctx):
    """Gates of -inf part sequences that share a row range: whatever the state was, the next one begins from the token."""
    g = gen(21)
    for dtype, c in ((F32, 64), (BF16, 37)):
        n = 1000
        x, f = randn(g, n, c).to(dtype), randn(g, n, c).to(dtype)
        h0 = 1e8 * torch.ones(1, c, device=DEV)                     # as far from the tokens as float32 has digits
        f[0], f[300], f[301], f[900] = -float("inf"), -float("inf"), float("inf"), -float("inf")
        h, parts = torch.empty_like(x), torch.empty_like(x)
        twa.twa_gated_scan(ctx, x, f, h, None, 1, h0)
        assert torch.equal(h[0], x[0]) and torch.equal(h[300], x[300]) and torch.equal(h[301], h[300]) and torch.equal(h[900], x[900])
        starts = torch.tensor([0, 300, 900, n], device=DEV)
        twa.twa_gated_scan(ctx, x, f, parts, starts, 3)
        scan_64.dtype = dtype
        want, e = scan_64(x, f, [300, 600, 100], [0, 300, 900], None)["h"]
        for got in (h, parts):
            close(got, want, e + ROUND[dtype] * (want.abs() + e) + 1e-37)
    ok(ctx)


def test_two_graphs_of_one_context_and_two_contexts_at_once(ctx):
    """Calls that a cluster of blocks shares, captured twice from one context and replayed together with a second context's."""
    g = gen(31)
    side = [torch.cuda.Stream() for _ in range(3)]
    cases = []
    for i, s in enumerate(side):
        n, c, tokens, experts = 6000 + 64 * i, 48, 9000 + i, 40 + i
        x, f, dh = (randn(g, n, c).to(BF16) for _ in range(3))
        cases.append(dict(x=x, f=f, dh=dh, h=torch.empty_like(x), dx=torch.empty_like(x), df=torch.empty_like(x),
                          states=torch.empty(twa.twa_gated_scan_states_bytes(n, 1, c), dtype=torch.uint8, device=DEV),
                          ids=torch.randint(-1, experts, (tokens, 4), generator=g, device=DEV), experts=experts,
                          place=torch.empty((tokens, 4), dtype=torch.int32, device=DEV), starts=torch.empty(experts + 1, dtype=torch.int32, device=DEV),
                          rows=randn(g, tokens, 24), out=torch.zeros(tokens * 4, 24, device=DEV)))
    torch.cuda.synchronize()

    def step(own, v):
        twa.twa_gated_scan(own, v["x"], v["f"], v["h"], states=v["states"])
        twa.twa_expert_dispatch(own, v["rows"], v["ids"], v["experts"], v["place"], v["starts"], v["out"])
        twa.twa_gated_scan_backward(own, v["dh"], v["x"], v["f"], v["states"], v["dx"], v["df"])

    names = ("h", "dx", "df", "place", "starts", "out")
    want, contexts, graphs = [], {}, []
    for s, v in zip(side, cases):
        with torch.cuda.stream(s):
            one = twa.twa_create(0)
            step(one, v)
            s.synchronize()
            assert twa.twa_get_status(one)[0] == 0
            twa.twa_destroy(one)
        want.append([v[k].clone() for k in names])
    with torch.cuda.stream(side[0]):
        contexts[0] = contexts[1] = twa.twa_create(0)               # the first two graphs are this context's
    with torch.cuda.stream(side[2]):
        contexts[2] = twa.twa_create(0)
    for i, v in enumerate(cases):
        s = side[0] if i < 2 else side[2]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(contexts[i], v)
        graphs.append(graph)
    for _ in range(5):
        for v in cases:
            for k in names:
                v[k].zero_()
        torch.cuda.synchronize()
        for s, graph in zip(side, graphs):                          # all three at once
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for v, w in zip(cases, want):
            assert all(torch.equal(v[k], t) for k, t in zip(names, w))
    for c in (contexts[0], contexts[2]):
        assert twa.twa_get_status(c)[0] == 0
    del graphs
    twa.twa_destroy(contexts[0])
    twa.twa_destroy(contexts[2])


def test_scan_knobs_take_what_they_mean(ctx):
    for key, good in ((twa.TWA_TUNE_SCAN_CLUSTER, (1, 2, 4, 8)), (twa.TWA_TUNE_SCAN_CHANNELS, (16, 32, 64))):
        for value in good + (0,):
            twa.twa_set_tuning(ctx, key, value)
        for value in (3, 12, 128):
            with pytest.raises(twa.TwaError):
                twa.twa_set_tuning(ctx, key, value)
        twa.twa_set_tuning(ctx, key, 0)


def test_offsets_beyond_32_bits(ctx):
    """Matrices of more than 2^31 elements, looked at near their ends."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    g = gen(1)
    n, c = (1 << 20) + 129, 2304
    x = torch.zeros(n, c, dtype=BF16, device=DEV)
    x[-400:] = randn(g, 400, c).to(BF16)
    y = torch.empty_like(x)
    rng = torch.tensor([3, 4], device=DEV)
    twa.twa_dropout(ctx, x, 0.5, rng, 9, y)
    kept = torch.from_numpy(dropout_numbers(3, 4, 9, 2, c, n - 2) >= 32768).to(DEV)
    assert torch.equal(y[-2:], torch.where(kept, 2 * x[-2:], 0))
    # the state comes from the row 300 rows before the end: everything before is zero
    f = torch.zeros(n, c, dtype=BF16, device=DEV)
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, 2, c), dtype=torch.uint8, device=DEV)
    starts = torch.tensor([0, n - 300, n], device=DEV)
    twa.twa_gated_scan(ctx, x, f, y, starts, 2, states=states)
    small, fs, want = x[-300:].clone(), f[-300:].clone(), torch.empty(300, c, dtype=BF16, device=DEV)
    s2 = torch.empty(twa.twa_gated_scan_states_bytes(300, 1, c), dtype=torch.uint8, device=DEV)
    twa.twa_gated_scan(ctx, small, fs, want, states=s2)
    assert torch.equal(y[-300:], want)
    dx, df = torch.empty_like(small), torch.empty_like(small)
    twa.twa_gated_scan_backward(ctx, small, small, fs, s2, dx, df)
    twa.twa_gated_scan_backward(ctx, x, x, f, states, y, f, starts, 2)
    assert torch.equal(y[-300:], dx) and torch.equal(f[-300:], df)
    del f, states
    ids = torch.arange(n, device=DEV)[:, None] % 2
    place, edges = torch.empty((n, 1), dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    twa.twa_expert_dispatch(ctx, x, ids, 2, place, edges, y)
    odd = n // 2
    assert torch.equal(y[-150:], x[1::2][-150:]) and int(edges[1]) == n - odd
    back = torch.empty_like(x)
    twa.twa_expert_combine(ctx, y, place, None, back)
    assert torch.equal(back[-400:], x[-400:])
    dw, w = torch.empty(n, 1, device=DEV), torch.ones(n, 1, device=DEV)
    twa.twa_expert_combine_backward(ctx, x, y, place, w, y, dw)
    assert torch.equal(y[-150:], x[1::2][-150:])
    want = (x[-400:].double() ** 2).sum(1)
    close(dw[-400:, 0], want, (c + 8) * U * want)
    ok(ctx)


def test_refusals(ctx):
    lib, bad, mis, uns, space = twa.load(), twa.TWA_ERR_INVALID_ARG, twa.TWA_ERR_MISALIGNED, twa.TWA_ERR_UNSUPPORTED, twa.TWA_ERR_WORKSPACE
    d = torch.zeros(4096, device=DEV).data_ptr()                      # long enough for every call that is meant well
    drop = lambda x=d, ldx=8, dt=0, rows=4, cols=8, p=0.1, rng=d, site=0, res=None, ldr=0, y=d, ldy=8: lib.twa_dropout(
        ctx, x, ldx, dt, rows, cols, p, rng, site, res, ldr, y, ldy)
    for kw, want in ((dict(dt=7), bad), (dict(rows=-1), bad), (dict(cols=0), bad), (dict(p=1.0), bad), (dict(p=-0.1), bad), (dict(p=float("nan")), bad),
                     (dict(site=-1), bad), (dict(site=1 << 32), bad), (dict(x=None), bad), (dict(y=None), bad), (dict(rng=None), bad), (dict(ldx=7), bad),
                     (dict(ldy=7), bad), (dict(res=d, ldr=7), bad), (dict(x=d + 2), mis), (dict(y=d + 1), mis), (dict(rng=d + 4), mis), (dict(res=d + 2, ldr=8), mis),
                     (dict(rows=twa.TWA_DROPOUT_MAX_ROWS + 1), uns), (dict(cols=twa.TWA_DROPOUT_MAX_COLS + 1, ldx=1 << 30, ldy=1 << 30), uns),
                     (dict(rows=0, x=None, y=None, rng=None), 0), (dict(), 0)):
        assert drop(**kw) == want, kw
    scan = lambda x=d, ldx=8, f=d, ldf=8, dt=0, n=4, c=8, starts=None, st=0, q=2, h0=None, h=d, ldh=8, last=None, states=None, size=0: lib.twa_gated_scan(
        ctx, x, ldx, f, ldf, dt, n, c, starts, st, q, h0, h, ldh, last, states, size)
    for kw, want in ((dict(dt=2), bad), (dict(n=-1), bad), (dict(c=0), bad), (dict(q=-1), bad), (dict(q=3), bad), (dict(q=0), bad), (dict(starts=d, st=5), bad),
                     (dict(x=None), bad), (dict(f=None), bad), (dict(h=None), bad), (dict(ldx=7), bad), (dict(ldf=7), bad), (dict(ldh=7), bad),
                     (dict(x=d + 2), mis), (dict(f=d + 2), mis), (dict(h=d + 2), mis), (dict(h0=d + 2), mis), (dict(last=d + 2), mis), (dict(starts=d + 2), mis),
                     (dict(starts=d + 4, st=1), mis), (dict(states=d, size=2 * 8 * 4 - 1), space), (dict(states=d + 4, size=2 * 8 * 4), mis),
                     (dict(c=twa.TWA_SCAN_MAX_CHANNELS + 1), uns), (dict(q=twa.TWA_SCAN_MAX_SEQUENCES + 1), uns), (dict(n=twa.TWA_SCAN_MAX_TOKENS + 1), uns),
                     (dict(n=0, q=1 << 24, c=1 << 20), uns), (dict(n=0, q=0, x=None, f=None, h=None), 0), (dict(n=0, x=None, f=None, h=None), 0), (dict(), 0)):
        assert scan(**kw) == want, kw
    back = lambda dh=d, x=d, f=d, dt=0, n=4, c=8, starts=None, st=0, q=2, states=d, size=64, last=None, dx=d + 4096, df=d + 8192, ld=8, dh0=None: \
        lib.twa_gated_scan_backward(ctx, dh, ld, x, ld, f, ld, dt, n, c, starts, st, q, states, size, last, dx, ld, df, ld, dh0)
    for kw, want in ((dict(dt=-1), bad), (dict(q=3), bad), (dict(dh=None), bad), (dict(x=None), bad), (dict(f=None), bad), (dict(dx=None), bad), (dict(df=None), bad),
                     (dict(ld=7), bad), (dict(states=None), space), (dict(size=63), space), (dict(states=d + 4), mis), (dict(dh=d + 2), mis), (dict(df=d + 2), mis),
                     (dict(last=d + 1), mis), (dict(dh0=d + 1), mis), (dict(), 0)):
        assert back(**kw) == want, kw
    send = lambda x=d, ldx=8, dt=0, n=4, dim=8, ids=d, it=0, top=2, e=4, place=d + 4096, starts=d + 8192, order=None, out=d + 12288, ldo=8: lib.twa_expert_dispatch(
        ctx, x, ldx, dt, n, dim, ids, it, top, e, place, starts, order, out, ldo)
    for kw, want in ((dict(dt=3), bad), (dict(it=2), bad), (dict(n=-1), bad), (dict(top=0), bad), (dict(e=0), bad), (dict(dim=0), bad), (dict(ids=None), bad),
                     (dict(place=None), bad), (dict(starts=None), bad), (dict(x=None), bad), (dict(out=None), bad), (dict(ldx=7), bad), (dict(ldo=7), bad),
                     (dict(ids=d + 4, it=1), mis), (dict(place=d + 2), mis), (dict(starts=d + 2), mis), (dict(order=d + 2), mis), (dict(x=d + 2), mis),
                     (dict(out=d + 2), mis), (dict(e=twa.TWA_EXPERTS_MAX + 1), uns), (dict(top=33), uns), (dict(n=twa.TWA_EXPERTS_MAX_ASSIGNMENTS), uns),
                     (dict(dim=twa.TWA_EXPERTS_MAX_DIM + 1), uns), (dict(n=0, x=None, out=None, ids=None, place=None), 0), (dict(), 0)):
        assert send(**kw) == want, kw
    join = lambda y=d, ldy=8, dt=0, rows=8, place=d, w=d, n=4, top=2, dim=8, out=d + 4096, ldo=8: lib.twa_expert_combine(
        ctx, y, ldy, dt, rows, place, w, n, top, dim, out, ldo)
    for kw, want in ((dict(dt=3), bad), (dict(rows=-1), bad), (dict(n=-1), bad), (dict(top=0), bad), (dict(dim=0), bad), (dict(y=None), bad), (dict(place=None), bad),
                     (dict(out=None), bad), (dict(ldy=7), bad), (dict(ldo=7), bad), (dict(place=d + 2), mis), (dict(w=d + 2), mis), (dict(y=d + 2), mis),
                     (dict(out=d + 2), mis), (dict(top=33), uns), (dict(dim=twa.TWA_EXPERTS_MAX_DIM + 1), uns), (dict(n=0, y=None, place=None, out=None), 0), (dict(), 0)):
        assert join(**kw) == want, kw
    grad = lambda dout=d, ldd=8, y=d, dt=0, rows=8, place=d, w=d, n=4, top=1, dim=8, dy=d + 4096, dw=None: lib.twa_expert_combine_backward(
        ctx, dout, ldd, y, 8, dt, rows, place, w, n, top, dim, dy, 8, dw)
    for kw, want in ((dict(dt=3), bad), (dict(dout=None), bad), (dict(ldd=7), bad), (dict(y=None), bad), (dict(dy=None), bad), (dict(place=None), bad), (dict(w=None), bad),
                     (dict(dout=d + 2), mis), (dict(y=d + 2), mis), (dict(dy=d + 2), mis), (dict(place=d + 2), mis), (dict(w=d + 2), mis), (dict(dw=d + 2), mis),
                     (dict(top=33), uns), (dict(n=0, dout=None), 0)):
        assert grad(**kw) == want, kw
    torch.cuda.synchronize()
    ok(ctx)


@pytest.mark.parametrize("channels,pads,step", [(71, (0, 3, 2), 1), (5, (2, 0, 7), 1), (129, (1, 1, 0), 1), (70, (2, 4, 0), 2), (130, (0, 6, 2), 2)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gated_scan_takes_rows_from_any_place(ctx, channels, pads, step, dtype):
    # every place of a row in the 16 bytes around it, another one for each matrix, between values that must not reach a result:
    # the same numbers at the head of an allocation give the same bits
    lengths = [129, 5, 0, 128, 17, 40]
    n, q = sum(lengths), len(lengths)
    starts = torch.tensor([sum(lengths[:i]) for i in range(q + 1)], device=DEV, dtype=torch.int32)
    g = gen(channels)
    src = [randn(g, n, channels).to(dtype), (2.0 * randn(g, n, channels) + 2.0).to(dtype), randn(g, n, channels).to(dtype)]
    size = twa.twa_gated_scan_states_bytes(n, q, channels)

    def run(x, f, dh):
        states = torch.empty(size, dtype=torch.uint8, device=DEV)
        h, dx, df = (torch.empty((n, channels), dtype=dtype, device=DEV) for _ in range(3))
        twa.twa_gated_scan(ctx, x, f, h, starts, q, states=states)
        twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, q)
        return h, dx, df

    def lain(v, pad, shift):
        ld = channels + pad
        buf = torch.full((shift + (n - 1) * ld + channels + 9,), float("nan"), dtype=dtype, device=DEV)
        view = buf[shift:].as_strided((n, channels), (ld, 1), buf.storage_offset() + shift)
        view.copy_(v)
        return view

    # rows `step` elements longer than the matrix is wide: not in units of 16 bytes there either
    want = run(*(lain(v, step, 0) for v in src))
    for shift in range(0, 9, step):
        got = run(*(lain(v, pad, (shift * k) % 9 // step * step) for k, (v, pad) in enumerate(zip(src, pads), 1)))
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    ok(ctx)
