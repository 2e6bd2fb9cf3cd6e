"""The model's operators between w and g (layer norm, embedding, token log probabilities, gradient norm and clipping)
against their definitions in 64 bits, at the sizes, types, strides and masks where they can go wrong.

Tolerances are worst-case bounds of the arithmetic, element by element: U = 2^-24 is half a unit in the last place of
float32, a sum of float32 terms whose longest chain of additions is k errs by at most k U times the sum of their
magnitudes, and an output is rounded once to its type (relative 2^-8 for bfloat16, U for float32).
"""

import ctypes
import math

import pytest
import torch

from paper_2205_13104_b200 import twa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: U, BF16: 2.0 ** -8}


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


def strided(values, dtype, pad=0, shift=0, fill=7.0):
    """The matrix as a view whose rows are `pad` elements apart, beginning `shift` elements into a buffer of `fill`."""
    rows, cols = values.shape
    buf = torch.full((shift + rows * (cols + pad),), fill, dtype=dtype, device=DEV)
    view = buf[shift:].view(rows, cols + pad)[:, :cols]
    view.copy_(values)
    return buf, view


def untouched(buf, view, fill=7.0):
    """Nothing outside the view was written."""
    keep = view.clone()
    view.fill_(fill)
    ok = bool((buf == fill).all())
    view.copy_(keep)
    return ok


def close(got, want, tol):
    """|got - want| <= tol everywhere; equal infinities count as equal."""
    got = got.double()
    same = (got == want) | ((got - want).abs() <= tol)
    assert bool(same.all()), float(((got - want).abs() / tol)[~same].max())


def ok(ctx):
    assert twa.twa_get_status(ctx)[0] == 0


# ------------------------------------------------------------------------------------------- layer norm
def layer_norm_64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    h = (x - mean) * rstd
    return h * (1.0 if w is None else w.double()) + (0.0 if b is None else b.double()), mean[:, 0], rstd[:, 0], h


def norm_tolerances(x, w, b, y, rstd, chain):
    big = x.double().abs().max(1, keepdim=True).values
    h = rstd[:, None] * big                                    # the mean errs by chain U big, the variance likewise
    wa = 1.0 if w is None else w.double().abs()
    return 3 * chain * U * (h + 1.0) * (1.0 + h) * wa + (ROUND[x.dtype] + 4 * U) * (y.abs() + (0.0 if b is None else b.double().abs()))


NORM_SIZES = [(1, 1), (1, 8), (3, 2), (5, 31), (7, 64), (2, 768), (197, 768), (1000, 127), (33, 512), (9, 1023), (64, 1024),
              (5, 1025), (301, 2048), (3, 4096), (4, 8191), (2, 8192), (3, 16384), (2, 16385), (2, 32768), (2, 40001)]


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dtype,wtype,pad,shift", [(F32, F32, 0, 0), (BF16, F32, 0, 0), (BF16, BF16, 8, 8), (F32, BF16, 3, 1),
                                                   (BF16, F32, 5, 3)])
def test_layer_norm_forward_and_backward(ctx, rows, cols, dtype, wtype, pad, shift):
    g = gen(rows * 131 + cols)
    xv = randn(g, rows, cols) * 2.0 + 0.5 * randn(g, cols) + 1.0
    xbuf, x = strided(xv, dtype, pad, shift)
    dybuf, dy = strided(randn(g, rows, cols) * 0.1, dtype, pad, shift)
    flat = randn(g, shift + 2 * cols).to(wtype)                 # weights as slices of one flat vector
    w, b = flat[shift: shift + cols], flat[shift + cols:]
    ybuf, y = strided(torch.zeros_like(xv), dtype, pad, shift)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    eps = 1e-5
    twa.twa_layer_norm(ctx, x, w, b, eps, y, mean, rstd)
    y64, mean64, rstd64, _ = layer_norm_64(x, w, b, eps)
    chain = 64 + cols / 512                                     # registers of a thread or the loop's strides, then the reductions
    big = x.double().abs().max(1).values
    close(mean, mean64, chain * U * big + 1e-30)
    close(rstd, rstd64, 3 * chain * U * rstd64 * (1 + big * rstd64))
    close(y, y64, norm_tolerances(x, w, b, y64, rstd64, chain))
    assert untouched(ybuf, y)

    # backward, from the statistics that the forward call left
    ws = torch.empty(twa.twa_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    dxbuf, dx = strided(torch.zeros_like(xv), dtype, pad, shift)
    dw, db = torch.full((cols + 2,), 5.0, device=DEV), torch.full((cols + 2,), 5.0, device=DEV)
    twa.twa_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx, dw[1:-1], db[1:-1], ws)
    r, m, d = rstd.double()[:, None], mean.double()[:, None], dy.double()
    h = (x.double() - m) * r
    v = d * w.double()
    dx64 = r * (v - v.mean(1, keepdim=True) - h * (v * h).mean(1, keepdim=True))
    vb, hb = v.abs().max(1, keepdim=True).values, (r * (x.double().abs() + m.abs())).max(1, keepdim=True).values
    close(dx, dx64, ROUND[dtype] * dx64.abs() + 3 * chain * U * r * vb * (1 + hb) ** 2 + 1e-30)
    long = rows + 64
    herr = 4 * U * r * (x.double().abs() + m.abs())
    close(dw[1:-1], (d * h).sum(0), long * U * (d * h).abs().sum(0) + (d.abs() * herr).sum(0) + 1e-30)
    close(db[1:-1], d.sum(0), long * U * d.abs().sum(0) + 1e-30)
    for t in (dw, db):
        assert t[0] == 5.0 and t[-1] == 5.0
    assert untouched(dxbuf, dx)

    # in place, repeated bit for bit, and added to what is there
    first, dw0, db0 = dx.clone(), dw[1:-1].clone(), db[1:-1].clone()
    inplace = dy.clone() if pad == 0 else strided(dy, dtype, pad, shift)[1]
    twa.twa_layer_norm_backward(ctx, inplace, x, w, mean, rstd, inplace, dw[1:-1], db[1:-1], ws)
    assert torch.equal(inplace, first) and torch.equal(dw[1:-1], dw0) and torch.equal(db[1:-1], db0)
    twa.twa_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx, dw[1:-1], db[1:-1], ws, accumulate=True)
    close(dw[1:-1], 2 * dw0.double(), 4 * U * dw0.double().abs() + long * U * (d * h).abs().sum(0))
    first = y.clone()
    twa.twa_layer_norm(ctx, x, w, b, eps, x)
    assert torch.equal(x, first)
    ok(ctx)


@pytest.mark.parametrize("rows,cols,dtype,wtype,pad,shift", [
    (16384, 2048, BF16, F32, 0, 0), (3000, 2048, F32, F32, 0, 0), (9000, 768, BF16, BF16, 0, 0), (20000, 256, F32, F32, 0, 0),
    (3001, 512, BF16, F32, 8, 8), (40000, 12, F32, F32, 0, 0), (30011, 96, BF16, F32, 0, 0), (6007, 1023, BF16, F32, 5, 3),
    (20011, 37, F32, BF16, 3, 1), (60013, 3, F32, F32, 0, 0),
    (1201, 8192, BF16, F32, 0, 0), (1500, 4099, F32, F32, 3, 2), (600, 12000, BF16, F32, 0, 0), (500, 16384, F32, F32, 0, 0),
    (1300, 16400, BF16, F32, 0, 0), (700, 9001, F32, F32, 0, 1)])
def test_layer_norm_of_many_rows(ctx, rows, cols, dtype, wtype, pad, shift):
    """Several rows for every team of threads: the ring's second round, the row that is fetched ahead, sums over rows."""
    test_layer_norm_forward_and_backward(ctx, rows, cols, dtype, wtype, pad, shift)


ALIKE, APART = ((0, 1),) * 4, ((1, 1), (2, 0), (0, 2), (3, 1))


@pytest.mark.parametrize("rows,cols,dtype,places", [(4099, 1023, F32, ALIKE), (50021, 7, BF16, ALIKE), (2000, 300, F32, APART),
                                                    (6000, 64, F32, APART), (1000, 2047, F32, APART), (700, 9000, F32, APART),
                                                    (9001, 5, F32, APART)])
def test_layer_norm_of_rows_between_16_byte_boundaries(ctx, rows, cols, dtype, places):
    """x, dy, y and dx with their rows at the same place between boundaries, or each at another (padding, start)."""
    g = gen(rows + cols)
    xv, dv, w = randn(g, rows, cols) + 0.5, randn(g, rows, cols), randn(g, cols)
    _, x = strided(xv, dtype, *places[0])
    _, dy = strided(dv, dtype, *places[1])
    ybuf, y = strided(torch.zeros_like(xv), dtype, *places[2])
    mean, rstd, dw, db = (torch.empty(n, device=DEV) for n in (rows, rows, cols, cols))
    ws = torch.empty(twa.twa_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    twa.twa_layer_norm(ctx, x, w, None, 1e-5, y, mean, rstd)
    y64, _, rstd64, _ = layer_norm_64(x, w, None, 1e-5)
    chain = 64 + cols / 512
    close(y, y64, norm_tolerances(x, w, None, y64, rstd64, chain))
    assert untouched(ybuf, y)
    dxbuf, dx = strided(torch.zeros_like(xv), dtype, *places[3])
    twa.twa_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx, dw, db, ws)
    r, m, d = rstd.double()[:, None], mean.double()[:, None], dy.double()
    h, v = (x.double() - m) * r, d * w.double()
    dx64 = r * (v - v.mean(1, keepdim=True) - h * (v * h).mean(1, keepdim=True))
    vb, hb = v.abs().max(1, keepdim=True).values, (r * (x.double().abs() + m.abs())).max(1, keepdim=True).values
    close(dx, dx64, ROUND[dtype] * dx64.abs() + 3 * chain * U * r * vb * (1 + hb) ** 2 + 1e-30)
    herr = 4 * U * r * (x.double().abs() + m.abs())
    close(dw, (d * h).sum(0), (rows + 64) * U * (d * h).abs().sum(0) + (d.abs() * herr).sum(0) + 1e-30)
    close(db, d.sum(0), (rows + 64) * U * d.abs().sum(0) + 1e-30)
    assert untouched(dxbuf, dx)
    ok(ctx)


def test_layer_norm_without_weights_and_with_bfloat16_gradients(ctx):
    g = gen(5)
    x = randn(g, 40, 96)
    dy = randn(g, 40, 96)
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(40, device=DEV), torch.empty(40, device=DEV)
    twa.twa_layer_norm(ctx, x, None, None, 1e-6, y, mean, rstd)
    y64, _, rstd64, h = layer_norm_64(x, None, None, 1e-6)
    close(y, y64, norm_tolerances(x, None, None, y64, rstd64, 64))
    dw = torch.empty(96, dtype=BF16, device=DEV)
    ws = torch.empty(twa.twa_layer_norm_workspace_bytes(40, 96), dtype=torch.uint8, device=DEV)
    twa.twa_layer_norm_backward(ctx, dy, x, None, mean, rstd, dx, dw, None, ws)
    want = (dy.double() * h).sum(0)
    close(dw, want, 2.0 ** -8 * want.abs() + 200 * U * (dy.double() * h).abs().sum(0))
    again = torch.empty_like(dx)
    twa.twa_layer_norm_backward(ctx, dy, x, None, mean, rstd, again, None, None, None)     # no weights' gradient: no workspace
    assert torch.equal(again, dx)
    # constant rows: nothing but eps in the root
    one = torch.full((3, 100), 4.0, device=DEV)
    yo = torch.empty_like(one)
    twa.twa_layer_norm(ctx, one, None, None, 1e-5, yo, mean[:3], rstd[:3])
    assert bool((yo == 0).all()) and bool((rstd[:3] - 1e-5 ** -0.5).abs().max() < 1e-3)
    ok(ctx)


def test_layer_norm_sums_are_added_to_what_the_kernel_before_left(ctx):
    """Launches may begin while the kernel before them ends: what that one writes last is not to be read too early."""
    big, cols = torch.empty(1 << 26, device=DEV), 512
    dw, db = big[-cols:], big[-2 * cols: -cols]
    none, ws = torch.empty(0, device=DEV), torch.empty(twa.twa_layer_norm_workspace_bytes(0, cols), dtype=torch.uint8, device=DEV)
    x = torch.empty(0, cols, device=DEV)
    wrong = torch.zeros((), device=DEV)
    for i in range(50):
        big.fill_(float(i))
        twa.twa_layer_norm_backward(ctx, x, x, None, none, none, x, dw, db, ws, accumulate=True)
        wrong += (big[-2 * cols:] != float(i)).sum()
    assert float(wrong) == 0
    ok(ctx)


def test_layer_norm_gradient_against_differences(ctx):
    g = gen(11)
    x, w, b, dy = randn(g, 6, 20), randn(g, 20), randn(g, 20), randn(g, 6, 20)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dw, db = (torch.empty(n, device=DEV) for n in (6, 6, 20, 20))
    ws = torch.empty(twa.twa_layer_norm_workspace_bytes(6, 20), dtype=torch.uint8, device=DEV)
    twa.twa_layer_norm(ctx, x, w, b, 1e-5, y, mean, rstd)
    twa.twa_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx, dw, db, ws)

    def loss(x, w, b):
        return float((layer_norm_64(x, w, b, 1e-5)[0] * dy.double()).sum())

    # central differences of step 1e-4 in 64 bits: the third derivative's share is below 1e-7 of gradients of order one
    step = 1e-4
    args = [x.double(), w.double(), b.double()]
    for which, grad in enumerate((dx, dw, db)):
        for i in range(0, args[which].numel(), 7):
            up, down = [a.clone() for a in args], [a.clone() for a in args]
            up[which].view(-1)[i] += step
            down[which].view(-1)[i] -= step
            assert abs((loss(*up) - loss(*down)) / (2 * step) - float(grad.view(-1)[i])) < 3e-5


# ------------------------------------------------------------------------------------------- embedding
EMB_SIZES = [(1, 1, 1), (1, 5, 8), (3, 2, 7), (32, 3, 16), (33, 9, 24), (100, 700, 129), (257, 50, 512), (2048, 17, 40), (2049, 1000, 33),
             (5000, 513, 64), (4096, 50272, 16), (9000, 300000, 8), (70000, 40, 8), (3000, 1, 72), (20, 60, 4100)]


@pytest.mark.parametrize("tokens,vocab,dim", EMB_SIZES)
@pytest.mark.parametrize("ttype,atype,itype,pad,shift", [(F32, F32, torch.int64, 0, 0), (F32, BF16, torch.int32, 0, 0),
                                                         (BF16, BF16, torch.int64, 8, 8), (BF16, F32, torch.int32, 3, 1)])
def test_embedding_and_its_gradient(ctx, tokens, vocab, dim, ttype, atype, itype, pad, shift):
    g = gen(tokens + vocab)
    tbuf, table = strided(randn(g, vocab, dim), ttype, pad, shift)
    u = torch.rand(tokens, generator=g, device=DEV)
    ids = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1).to(itype)      # some ids often, most rarely
    scale = math.sqrt(dim)
    obuf, out = strided(torch.zeros(tokens, dim, device=DEV), atype, pad, shift)
    twa.twa_embedding(ctx, table, ids, scale, out)
    scale32 = torch.tensor(scale, dtype=F32, device=DEV)
    assert torch.equal(out, (table[ids.long()].float() * scale32).to(atype))
    assert untouched(obuf, out)

    dbuf, dout = strided(randn(g, tokens, dim), atype, pad, shift)
    ws = torch.empty(twa.twa_embedding_workspace_bytes(tokens, vocab, dim), dtype=torch.uint8, device=DEV)
    chain = 32 + tokens / 256 + 16                              # a run, a stretch of runs, the stretches
    for padding in (-1, 0):
        want = torch.zeros(vocab, dim, dtype=torch.float64, device=DEV)
        size = torch.zeros_like(want)
        keep = ids.long() != padding
        want.index_add_(0, ids.long()[keep], dout.double()[keep])
        size.index_add_(0, ids.long()[keep], dout.double()[keep].abs())
        want, size = want * float(scale32), size * float(scale32)
        gbuf, grad = strided(torch.full((vocab, dim), 3.0, device=DEV), ttype, pad, shift)
        twa.twa_embedding_backward(ctx, dout, ids, scale, grad, ws, padding_id=padding)
        close(grad, want, chain * U * size + ROUND[ttype] * want.abs())
        assert untouched(gbuf, grad)
        first = grad.clone()
        ws.fill_(0xAB)                                          # the workspace carries nothing from call to call
        twa.twa_embedding_backward(ctx, dout, ids, scale, grad, ws, padding_id=padding)
        assert torch.equal(grad, first)
        held = randn(g, vocab, dim).to(ttype)
        grad.copy_(held)
        twa.twa_embedding_backward(ctx, dout, ids, scale, grad, ws, padding_id=padding, accumulate=True)
        want = want + held.double()
        close(grad, want, (chain + 2) * U * (size + held.double().abs()) + ROUND[ttype] * want.abs())
        rest = torch.ones(vocab, dtype=torch.bool, device=DEV)
        rest[ids.long()[keep]] = False
        assert torch.equal(grad[rest], held[rest])
    ok(ctx)


@pytest.mark.parametrize("tokens,vocab,dim", [(20000, 300000, 8), (40000, 1000, 24), (130001, 50272, 8), (16385, 513, 7), (6, (1 << 20) + 5, 4)])
@pytest.mark.parametrize("ttype,atype,itype,pad,shift", [(F32, BF16, torch.int64, 0, 0), (BF16, F32, torch.int32, 3, 1)])
def test_embedding_gradient_of_many_tokens(ctx, tokens, vocab, dim, ttype, atype, itype, pad, shift):
    """More ids than a cluster of blocks sorts, in one to three passes, and a vocabulary beyond its bitmap."""
    test_embedding_and_its_gradient(ctx, tokens, vocab, dim, ttype, atype, itype, pad, shift)


def test_embedding_gradient_of_many_tokens_replays_from_a_graph(ctx):
    g = gen(77)
    tokens, vocab, dim = 40000, 70000, 32
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        own = twa.twa_create(0)
        ids = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
        dout = torch.randint(-4, 5, (tokens, dim), generator=g, device=DEV).float()       # sums of whole numbers are exact
        grad, added = torch.empty(vocab, dim, device=DEV), torch.zeros(vocab, dim, device=DEV)
        ws = torch.empty(twa.twa_embedding_workspace_bytes(tokens, vocab, dim), dtype=torch.uint8, device=DEV)

        def step():
            twa.twa_embedding_backward(own, dout, ids, 1.0, grad, ws)
            twa.twa_embedding_backward(own, dout, ids, 1.0, added, ws, accumulate=True)

        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        added.zero_()
        want = torch.zeros(vocab, dim, device=DEV)
        for again in range(3):
            ids.copy_(torch.randint(0, vocab >> again, (tokens,), generator=g, device=DEV))
            graph.replay()
            now = torch.zeros(vocab, dim, dtype=torch.float64, device=DEV).index_add_(0, ids, dout.double())
            want += now.float()
            assert torch.equal(grad.double(), now) and torch.equal(added, want)
        assert twa.twa_get_status(own)[0] == 0
        del graph
        twa.twa_destroy(own)


@pytest.mark.parametrize("tokens,vocab", [(20000, 5), (65536, 1), (6000, 70000)])
def test_embedding_gradient_of_whole_numbers_is_exact(ctx, tokens, vocab):
    """Small whole numbers add without rounding, so each sum is one number: a token that is lost or counted twice shows."""
    g = gen(tokens)
    ids = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    dout = torch.randint(-4, 5, (tokens, 24), generator=g, device=DEV).float()
    grad = torch.empty(vocab, 24, device=DEV)
    ws = torch.empty(twa.twa_embedding_workspace_bytes(tokens, vocab, 24), dtype=torch.uint8, device=DEV)
    twa.twa_embedding_backward(ctx, dout, ids, 1.0, grad, ws)
    assert torch.equal(grad.double(), torch.zeros(vocab, 24, dtype=torch.float64, device=DEV).index_add_(0, ids, dout.double()))


def test_embedding_with_ids_outside_the_table(ctx):
    table = torch.arange(12.0, device=DEV).view(6, 2)
    ids = torch.tensor([0, 6, 5, -1, 2 ** 40, 3], device=DEV)
    out = torch.full((6, 2), 9.0, device=DEV)
    twa.twa_embedding(ctx, table, ids, 1.0, out)
    code, detail = twa.twa_get_status(ctx)
    assert code == twa.TWA_ERR_INVALID_ARG and detail in (1, 3, 4)
    assert torch.equal(out[[0, 2, 5]], table[[0, 5, 3]]) and bool((out[[1, 3, 4]] == 0).all())
    twa.twa_clear_status(ctx)
    grad = torch.empty_like(table)
    ws = torch.empty(twa.twa_embedding_workspace_bytes(6, 6, 2), dtype=torch.uint8, device=DEV)
    twa.twa_embedding_backward(ctx, torch.ones(6, 2, device=DEV), ids, 2.0, grad, ws)
    code, detail = twa.twa_get_status(ctx)
    assert code == twa.TWA_ERR_INVALID_ARG and detail in (1, 3, 4)
    want = torch.zeros_like(table)
    want[[0, 5, 3]] = 2.0
    assert torch.equal(grad, want)


def test_embedding_rows_beyond_2_31_elements(ctx):
    vocab, dim = (1 << 20) + 77, 2056
    table = torch.empty(vocab, dim, dtype=BF16, device=DEV)
    ids = torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1], device=DEV)
    rows = torch.randint(-8, 9, (4, dim), device=DEV).to(BF16)
    table[ids] = rows
    out = torch.empty(4, dim, dtype=BF16, device=DEV)
    twa.twa_embedding(ctx, table, ids, 1.0, out)
    assert torch.equal(out, table[ids])
    table[ids] = 1.0
    ws = torch.empty(twa.twa_embedding_workspace_bytes(4, vocab, dim), dtype=torch.uint8, device=DEV)
    twa.twa_embedding_backward(ctx, rows, ids, 1.0, table, ws, accumulate=True)
    assert torch.equal(table[vocab - 1], (1.0 + rows[0].float() + rows[3].float()).to(BF16))
    assert torch.equal(table[vocab - 2], 1.0 + rows[2])
    ok(ctx)


# ------------------------------------------------------------------------------------------- token log probabilities
def logprobs_64(z, t, top, ignore=-100):
    z = z.double()
    lse = torch.logsumexp(z, 1)
    none = lse == -math.inf
    lp = torch.where(none[:, None], -math.inf, z - lse[:, None])
    logp = torch.where(t == ignore, 0.0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0])
    h = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(1)
    ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
    return logp, lse, h, ids, lp.gather(1, ids), lp


def logprob_tolerances(z, vocab):
    # longest chain of a thread (16-byte units over 512 threads, unrolled into single additions), ex2 (2^-22), the
    # exponent's argument rounded twice at a magnitude below 2 (|max| + 40)
    some = torch.where(z.double().abs() < 1e30, z.double().abs(), 0.0).max(1).values
    return (vocab / 512 + 48 + 4 * (some + 40.0)) * U, some


LOGP_SIZES = [(1, 1, 1), (2, 2, 2), (3, 7, 7), (5, 33, 32), (4, 100, 20), (1, 1000, 5), (3, 4099, 20), (2, 16384, 32), (1, 50272, 20),
              (7, 50257, 5), (150, 32003, 3), (300, 1031, 20), (1, 200001, 32), (2, 131072, 1)]


@pytest.mark.parametrize("rows,vocab,top", LOGP_SIZES)
@pytest.mark.parametrize("dtype,itype,pad,shift", [(F32, torch.int64, 0, 0), (BF16, torch.int32, 0, 0), (BF16, torch.int64, 5, 3),
                                                   (F32, torch.int32, 3, 1)])
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_token_logprobs_and_gradient(ctx, rows, vocab, top, dtype, itype, pad, shift, masked):
    g = gen(rows * 7 + vocab)
    zv = randn(g, rows, vocab) * 3.0 + 5.0 * randn(g, rows, 1)
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    zv[torch.arange(rows, device=DEV), t] += 10.0 * torch.rand(rows, generator=g, device=DEV)
    if masked:
        off = torch.rand(rows, vocab, generator=g, device=DEV) < masked
        low = -math.inf if rows % 2 else torch.finfo(dtype).min       # masks of -inf, or of the type's lowest value
        zv.masked_fill_(off, low)
        if rows > 1:
            zv[rows // 2] = -math.inf                                 # a row whose mask leaves nothing
            zv[0, 1:] = -math.inf                                     # and one that leaves a single token
    if rows > 2:
        t[2] = -100
    zbuf, z = strided(zv, dtype, pad, shift)
    logp, lse, ent = (torch.empty(rows, device=DEV) for _ in range(3))
    ids, tlp = torch.empty(rows, top, dtype=torch.int32, device=DEV), torch.empty(rows, top, device=DEV)
    twa.twa_token_logprobs(ctx, z, t.to(itype), logp, lse, entropy=ent, top_ids=ids, top_logp=tlp)
    want = logprobs_64(z, t, top)
    tol, big = logprob_tolerances(z, vocab)
    lse_tol = tol + 2 * U * want[1].abs().nan_to_num(posinf=0.0, neginf=0.0)
    close(lse, want[1], lse_tol)
    close(logp, want[0], lse_tol + 4 * U * (big + want[0].abs().nan_to_num(posinf=0.0)) )
    close(ent, want[2], 4 * tol * (1.0 + want[2] + math.log(vocab)))
    assert torch.equal(ids.long(), want[3])
    close(tlp, want[4], (lse_tol + 4 * U * big)[:, None] + 4 * U * want[4].abs().nan_to_num(posinf=0.0))
    # each part alone gives the same
    only = [torch.empty_like(logp), torch.empty_like(lse)]
    twa.twa_token_logprobs(ctx, z, t.to(itype), *only)
    assert torch.equal(only[0], logp) and torch.equal(only[1], lse)

    d_logp, d_ent = randn(g, rows), 0.1 * randn(g, rows)
    lp = torch.where(lse.double()[:, None] == -math.inf, -math.inf, z.double() - lse.double()[:, None])
    p = lp.exp()
    live = ((t != -100) & (lse > -math.inf)).double() * d_logp.double()
    one = torch.zeros_like(p).scatter_(1, t.clamp(min=0)[:, None], 1.0)
    first = live[:, None] * (one - p)
    inner = torch.where(p > 0, lp + ent.double()[:, None], 0.0)
    second = -d_ent.double()[:, None] * p * inner
    # p errs by the exponent's argument (rounded against lse log2 e) and ex2; flushed below 2^-126
    rel = 2.0 ** -21 + 4 * U * (big + 40.0)[:, None] + 4 * U * lse.double().abs().nan_to_num(posinf=0.0)[:, None]
    for with_entropy in (False, True):
        dz64 = first + (second if with_entropy else 0.0)
        scale = live.abs()[:, None] * p + (d_ent.double().abs()[:, None] * p * (inner.abs() + 1.0) if with_entropy else 0.0)
        dtol = rel * scale + 2 * U * live.abs()[:, None] * one + ROUND[dtype] * dz64.abs() + 1e-36
        dbuf, dz = strided(torch.zeros_like(zv), dtype, pad, shift)
        extra = dict(entropy=ent, d_entropy=d_ent) if with_entropy else {}
        twa.twa_token_logprobs_backward(ctx, z, t.to(itype), lse, d_logp, dz, **extra)
        close(dz, dz64, dtol)
        assert untouched(dbuf, dz)
        _, other = strided(torch.zeros_like(zv), dtype, pad + 1, shift + 1)            # rows that lie differently
        twa.twa_token_logprobs_backward(ctx, z, t.to(itype), lse, d_logp, other, **extra)
        close(other, dz64, dtol)
        same = z.clone() if pad == 0 else strided(z, dtype, pad, shift)[1]
        twa.twa_token_logprobs_backward(ctx, same, t.to(itype), lse, d_logp, same, **extra)
        assert torch.equal(same, dz)
    ok(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [75, 2840, 20011])
@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("with_entropy", [False, True])
def test_logprobs_of_many_rows(ctx, dtype, vocab, top, with_entropy):
    """Several rows for every block, with and without the search and the entropy: every output of every row."""
    rows = 4001
    g = gen(vocab + top)
    z = (2.5 * randn(g, rows, vocab) + 4.0 * randn(g, rows, 1)).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    t[::7] = -100
    logp, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ent = torch.empty(rows, device=DEV) if with_entropy else None
    ids = torch.empty(rows, top, dtype=torch.int32, device=DEV) if top else None
    tlp = torch.empty(rows, top, device=DEV) if top else None
    twa.twa_token_logprobs(ctx, z, t, logp, lse, entropy=ent, top_ids=ids, top_logp=tlp)
    want = logprobs_64(z, t, max(top, 1))
    tol, big = logprob_tolerances(z, vocab)
    lse_tol = tol + 2 * U * want[1].abs()
    close(lse, want[1], lse_tol)
    close(logp, want[0], lse_tol + 4 * U * (big + want[0].abs()))
    if with_entropy:
        close(ent, want[2], 4 * tol * (1.0 + want[2] + math.log(vocab)))
    if top:
        assert torch.equal(ids.long(), want[3])
        close(tlp, want[4], (lse_tol + 4 * U * big)[:, None] + 4 * U * want[4].abs())
    ok(ctx)


FAR = [8191.5, 8192.0, 8193.0, 20000.0, 1e5, 1e30, 3e38]


@pytest.mark.parametrize("vocab", [333, 20011, 200001])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [2 * len(FAR) + 2, 700])
@pytest.mark.parametrize("mixed", [False, True])
def test_logprobs_of_logits_far_from_zero(ctx, vocab, dtype, rows, mixed):
    """Rows whose largest logit is far above or below zero, whole rows at the type's lowest value, and (mixed) with half of a row's
    logits near zero; few rows, which clusters share, and many."""
    if vocab > 100000 and rows > 100:
        rows = 320
    g = gen(vocab + rows)
    base = torch.tensor([s * v for v in FAR for s in (1.0, -1.0)] + [0.0, 0.0], device=DEV).repeat(rows // (2 * len(FAR) + 2) + 1)[:rows]
    z = randn(g, rows, vocab)
    near = z[:, vocab // 2:].clone()
    z += base[:, None]
    if mixed:
        z[:, vocab // 2:] = near
    z[-1] = torch.finfo(dtype).min
    z = z.to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    logp, lse, ent = (torch.empty(rows, device=DEV) for _ in range(3))
    ids, tlp = torch.empty(rows, 4, dtype=torch.int32, device=DEV), torch.empty(rows, 4, device=DEV)
    twa.twa_token_logprobs(ctx, z, t, logp, lse, entropy=ent, top_ids=ids, top_logp=tlp)
    want = logprobs_64(z, t, 4)
    # Differences to the maximum come first, so its size does not count: a sum's longest chain is a warp's lane over the whole
    # row, ex2 (2^-22), the exponent rounded twice at a magnitude below 2 x 40 where it counts; lse itself is rounded
    tol = (vocab / 32 + 48 + 4 * 40.0) * U
    close(lse, want[1], tol + 2 * U * want[1].abs())
    # the result in 64 bits from the target's difference to the maximum, which 64 bits hold exactly
    m = z.double().max(1, keepdim=True).values
    d = z.double() - m
    logs = torch.log(torch.exp(d).sum(1))
    at = d.gather(1, t[:, None])[:, 0] - logs
    close(logp, at, tol + 4 * U * at.abs())
    p = torch.exp(d - logs[:, None])
    h = -torch.where(p > 0, p * (d - logs[:, None]), 0.0).sum(1)
    close(ent, h, 4 * tol * (1.0 + h + math.log(vocab)))
    assert torch.equal(ids.long(), want[3])
    best = d.gather(1, want[3]) - logs[:, None]
    close(tlp, best, tol + 4 * U * best.abs())
    only = [torch.empty_like(logp), torch.empty_like(lse)]
    twa.twa_token_logprobs(ctx, z, t, *only)
    assert torch.equal(only[0], logp) and torch.equal(only[1], lse)
    # the gradient, from lse as it is in float32
    d_logp, dz = randn(g, rows), torch.empty_like(z)
    twa.twa_token_logprobs_backward(ctx, z, t, lse, d_logp, dz)
    p = torch.exp(z.double() - lse.double()[:, None])
    one = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    dz64 = d_logp.double()[:, None] * (one - p)
    scale = d_logp.double().abs()[:, None]
    # z - lse is one rounding of at most 40 where p counts (88 where lse, rounded, lies so far below the logits that p is that large)
    close(dz, dz64, (2.0 ** -21 + 4 * 128 * U) * scale * p + 2 * U * scale * one + ROUND[dtype] * dz64.abs() + 1e-36)
    ok(ctx)


@pytest.mark.parametrize("vocab", [40, 3000, 60000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_top_tokens_of_equal_logits_are_the_lowest_indices(ctx, vocab, dtype):
    rows, top = 4, 32
    z = torch.zeros(rows, vocab, dtype=dtype, device=DEV)
    z[1, ::2] = -0.0                                              # zeros of both signs are equal
    z[2] = torch.arange(vocab, device=DEV) % 3                    # a third of the vocabulary at the maximum
    z[3, vocab - 1] = 1.0
    z[3, 0] = -1.0
    t = torch.zeros(rows, dtype=torch.int64, device=DEV)
    logp, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ids, tlp = torch.empty(rows, top, dtype=torch.int32, device=DEV), torch.empty(rows, top, device=DEV)
    twa.twa_token_logprobs(ctx, z, t, logp, lse, top_ids=ids, top_logp=tlp)
    assert torch.equal(ids.long(), torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :top])
    ok(ctx)


def test_top_tokens_of_sorted_logits(ctx):
    """Every element better than all before it, and the reverse."""
    vocab, top = 30011, 20
    z = torch.stack([torch.arange(vocab, device=DEV) * 1e-3, torch.arange(vocab, 0, -1, device=DEV) * 1e-3])
    t = torch.tensor([vocab - 1, 0], device=DEV)
    logp, lse = torch.empty(2, device=DEV), torch.empty(2, device=DEV)
    ids, tlp = torch.empty(2, top, dtype=torch.int32, device=DEV), torch.empty(2, top, device=DEV)
    twa.twa_token_logprobs(ctx, z, t, logp, lse, top_ids=ids, top_logp=tlp)
    assert torch.equal(ids[0].long(), torch.arange(vocab - 1, vocab - 1 - top, -1, device=DEV))
    assert torch.equal(ids[1].long(), torch.arange(top, device=DEV))
    assert torch.equal(tlp[:, 0], logp)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_logprobs_report_logits_that_are_no_numbers(ctx, bad):
    z = torch.zeros(3, 5000, device=DEV)
    z[1, 4321] = bad
    t = torch.tensor([1, 2, 3], device=DEV)
    logp, lse, ent = (torch.empty(3, device=DEV) for _ in range(3))
    twa.twa_token_logprobs(ctx, z, t, logp, lse, entropy=ent)
    assert twa.twa_get_status(ctx) == (twa.TWA_ERR_NONFINITE, 1)
    assert abs(float(lse[0]) - math.log(5000)) < 1e-5 and abs(float(lse[2]) - math.log(5000)) < 1e-5


def test_logprobs_report_targets_outside_the_vocabulary(ctx):
    z = torch.zeros(2, 10, device=DEV)
    logp, lse = torch.empty(2, device=DEV), torch.empty(2, device=DEV)
    t = torch.tensor([3, 10], device=DEV)
    twa.twa_token_logprobs(ctx, z, t, logp, lse)
    assert twa.twa_get_status(ctx) == (twa.TWA_ERR_INVALID_ARG, 1)
    assert math.isnan(float(logp[1])) and abs(float(logp[0]) + math.log(10)) < 1e-6
    twa.twa_clear_status(ctx)
    dz = torch.empty_like(z)
    twa.twa_token_logprobs_backward(ctx, z, t, lse, torch.ones(2, device=DEV), dz)
    assert twa.twa_get_status(ctx) == (twa.TWA_ERR_INVALID_ARG, 1)


def test_logprobs_gradient_against_differences(ctx):
    g = gen(3)
    z = randn(g, 4, 12)
    z[1, 5] = -math.inf
    t = torch.tensor([0, 3, -100, 11], device=DEV)
    logp, lse, ent = (torch.empty(4, device=DEV) for _ in range(3))
    twa.twa_token_logprobs(ctx, z, t, logp, lse, entropy=ent)
    a, b = randn(g, 4), randn(g, 4)
    dz = torch.empty_like(z)
    twa.twa_token_logprobs_backward(ctx, z, t, lse, a, dz, entropy=ent, d_entropy=b)

    def loss(zz):
        got = logprobs_64(zz, t, 1)
        return float((a.double() * got[0]).sum() + (b.double() * got[2]).sum())

    step = 1e-4
    for i in range(z.numel()):
        if z.view(-1)[i] == -math.inf:
            continue
        up, down = z.double().clone(), z.double().clone()
        up.view(-1)[i] += step
        down.view(-1)[i] -= step
        assert abs((loss(up) - loss(down)) / (2 * step) - float(dz.view(-1)[i])) < 1e-5


def test_rows_beyond_2_31_elements(ctx):
    """Three rows that lie 1.5 G elements apart: layer norm, log probabilities and their gradient reach the last."""
    ld, cols = 3 << 29, 2048
    buf = torch.empty(2 * ld + cols, dtype=BF16, device=DEV)
    x = torch.as_strided(buf, (3, cols), (ld, 1))
    near = randn(gen(1), 3, cols).to(BF16)
    x.copy_(near)
    y, y2 = torch.empty_like(near), torch.empty_like(near)
    twa.twa_layer_norm(ctx, x, None, None, 1e-5, y)
    twa.twa_layer_norm(ctx, near, None, None, 1e-5, y2)
    assert torch.equal(y, y2)
    t = torch.tensor([5, 6, 7], device=DEV)
    far, close_by = [torch.empty(3, device=DEV) for _ in range(2)], [torch.empty(3, device=DEV) for _ in range(2)]
    twa.twa_token_logprobs(ctx, x, t, *far)
    twa.twa_token_logprobs(ctx, near, t, *close_by)
    assert torch.equal(far[0], close_by[0]) and torch.equal(far[1], close_by[1])
    ones = torch.ones(3, device=DEV)
    dz = torch.empty_like(near)
    twa.twa_token_logprobs_backward(ctx, near, t, far[1], ones, dz)
    twa.twa_token_logprobs_backward(ctx, x, t, far[1], ones, x)
    assert torch.equal(x, dz)
    ok(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 7), (300, 1023), (40, 5000)])
def test_what_lies_between_rows_does_not_count(ctx, dtype, rows, cols):
    """NaN between the rows of every input gives what zeros there give, bit for bit."""
    g = gen(rows)
    xv, dv, t, w = randn(g, rows, cols), randn(g, rows, cols), torch.randint(0, cols, (rows,), generator=g, device=DEV), randn(g, cols)
    ws = torch.empty(max(twa.twa_layer_norm_workspace_bytes(rows, cols), twa.twa_embedding_workspace_bytes(rows, rows, cols)),
                     dtype=torch.uint8, device=DEV)
    got = []
    for fill in (0.0, math.nan):
        x, dy = (strided(v, dtype, 3, 1, fill)[1] for v in (xv, dv))
        y, dx, dz = (strided(torch.zeros_like(xv), dtype, 3, 1, fill)[1] for _ in range(3))
        out = torch.empty(rows, cols, device=DEV)
        mean, rstd, logp, lse, ent = (torch.empty(rows, device=DEV) for _ in range(5))
        dw, db, grad = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV), torch.empty(rows, cols, device=DEV)
        ids, tlp = torch.empty(rows, 5, dtype=torch.int32, device=DEV), torch.empty(rows, 5, device=DEV)
        twa.twa_layer_norm(ctx, x, w, None, 1e-5, y, mean, rstd)
        twa.twa_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx, dw, db, ws)
        twa.twa_token_logprobs(ctx, x, t, logp, lse, entropy=ent, top_ids=ids, top_logp=tlp)
        twa.twa_token_logprobs_backward(ctx, x, t, lse, lse, dz, entropy=ent, d_entropy=lse)
        where = torch.arange(rows, device=DEV) // 2
        twa.twa_embedding(ctx, x, where, 1.5, out)
        twa.twa_embedding_backward(ctx, dy, where, 1.5, grad, ws)
        got.append([a.clone() for a in (y, mean, rstd, dx, dw, db, logp, lse, ent, ids, tlp, dz, out, grad)])
    for a, b in zip(*got):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    ok(ctx)


# ------------------------------------------------------------------------------------------- gradient norm and clipping
def gradients(g, sizes, kinds, shift):
    out = []
    for i, (n, k) in enumerate(zip(sizes, kinds)):
        buf = (randn(g, n + shift + 1) * 0.01 * (1 + i % 5)).to(k)
        out.append(buf[shift: shift + n])                        # on no particular boundary
    return out


CLIP_SETS = [[1], [5], [16384], [16385, 3], [0, 7, 0, 100000, 1], [1000, 999, 998, 1, 2, 3] * 30, [33] * 513, [20] * 1024 + [70001],
             [3_000_001, 8]]


@pytest.mark.parametrize("sizes", CLIP_SETS, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("kinds,flat", [((F32,), F32), ((BF16,), BF16), ((BF16, F32), F32), ((F32, BF16, BF16), BF16)])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_and_clipping(ctx, sizes, kinds, flat, shift):
    g = gen(len(sizes) + shift)
    kinds = [kinds[i % len(kinds)] for i in range(len(sizes))]
    grads = gradients(g, sizes, kinds, shift)
    ts = twa.Tensors(grads)
    ws = torch.empty(twa.twa_grad_norm_workspace_bytes(ts), dtype=torch.uint8, device=DEV)
    norm = torch.empty(1, device=DEV)
    twa.twa_grad_norm(ctx, ts, norm, ws)
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    assert abs(float(norm) - want) <= 16 * U * want
    total = sum(sizes)
    for max_norm in (0.5 * want, 2.0 * want):
        g_out = torch.full((total + 2,), 5.0, dtype=flat, device=DEV)
        twa.twa_clip_gather(ctx, ts, max_norm, g_out[1: 1 + total] if shift else g_out[:total], norm, ws)
        part = g_out[1: 1 + total] if shift else g_out[:total]
        factor = min(1.0, max_norm / (want + 1e-6))
        ref = torch.cat([t.double() for t in grads]) * factor
        close(part, ref, (20 * U + ROUND[flat]) * ref.abs() + 1e-38)
        if factor == 1.0:
            assert torch.equal(part, torch.cat([t.float() for t in grads]).to(flat))
        assert g_out[-1] == 5.0 and (not shift or g_out[0] == 5.0)
        first = g_out.clone()
        twa.twa_clip_gather(ctx, ts, max_norm, part, norm, ws)
        assert torch.equal(g_out, first)
    before = [t.clone() for t in grads]
    twa.twa_clip_grads(ctx, ts, 2.0 * want, norm, ws)
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    twa.twa_clip_grads(ctx, ts, 0.5 * want, norm, ws)
    factor = 0.5 * want / (want + 1e-6)
    for a, b in zip(before, grads):
        close(b, a.double() * factor, (20 * U + ROUND[a.dtype]) * a.double().abs() * factor + 1e-38)
    ok(ctx)


LARGE_SETS = [[20_000_001], [20_000_003, 5, 7_000_001], [1 + (i * 7919) % 85703 for i in range(700)],
              [40_000 + 8 * i for i in range(450)] + [1] * 70]


@pytest.mark.parametrize("sizes", LARGE_SETS, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("kinds,flat", [((F32,), F32), ((BF16,), BF16), ((BF16, F32), F32), ((F32, BF16, BF16), BF16)])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_and_clipping_of_many_chunks(ctx, sizes, kinds, flat, shift):
    """Several chunks, and several tensors, for every block of either kernel."""
    test_norm_and_clipping(ctx, sizes, kinds, flat, shift)


def test_norm_of_nothing_and_of_what_is_no_number(ctx):
    norm = torch.full((1,), 3.0, device=DEV)
    ts = twa.Tensors([])
    ws = torch.empty(twa.twa_grad_norm_workspace_bytes(ts), dtype=torch.uint8, device=DEV)
    twa.twa_grad_norm(ctx, ts, norm, ws)
    assert float(norm) == 0.0
    ok(ctx)
    bad = torch.ones(50000, device=DEV)
    bad[40000] = math.inf
    ts = twa.Tensors([torch.ones(3, device=DEV), bad])
    twa.twa_grad_norm(ctx, ts, norm, ws)
    assert float(norm) == math.inf and twa.twa_get_status(ctx)[0] == twa.TWA_ERR_NONFINITE
    twa.twa_clear_status(ctx)
    bad[40000] = 2.0
    twa.twa_grad_norm(ctx, ts, norm, ws)
    assert abs(float(norm) - math.sqrt(50002 + 4)) < 1e-3
    ok(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size,spread", [(7e18, 1.0), (1.5e19, 1.0), (1e36, 1.0), (1e-22, 1.0), (3e-30, 1.0), (1e-38, 1.0), (1e-16, 1e-4), (1e16, 1e4)])
def test_norm_and_clipping_at_the_ends_of_float32(ctx, dtype, size, spread):
    """Elements whose squares are no float32, alone and beside others that are `spread` times as large."""
    g = gen(9)
    values = size * (1.0 + torch.rand(5003, generator=g, device=DEV, dtype=torch.float64))
    values[::3] = 0.0
    values[1::16] *= spread
    grads = [values[:4001].to(dtype), values[4001:].to(dtype)]
    ts = twa.Tensors(grads)
    ws, norm = torch.empty(twa.twa_grad_norm_workspace_bytes(ts), dtype=torch.uint8, device=DEV), torch.empty(1, device=DEV)
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    # sixteen roundings of a relative U, and half a unit in the last place of a result below 2^-126
    twa.twa_grad_norm(ctx, ts, norm, ws)
    assert abs(float(norm) - want) <= 16 * U * want + 2.0 ** -149
    out = torch.empty(5003, dtype=dtype, device=DEV)
    twa.twa_clip_gather(ctx, ts, 0.5 * want, out, norm, ws, eps=0.0)
    ref = 0.5 * torch.cat([t.double() for t in grads])
    close(out, ref, (20 * U + ROUND[dtype]) * ref.abs() + (2.0 ** -149 if dtype is F32 else 2.0 ** -133))
    ok(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [75, 505, 2840, 9001])
@pytest.mark.parametrize("top", [1, 20])
def test_best_tokens_of_many_short_rows(ctx, dtype, vocab, top):
    # several rows for each of the warps that finish them, while the next rows are being added up
    rows = 4001
    z = (2.5 * torch.randn(rows, vocab, generator=gen(vocab + top), device=DEV)).to(dtype)
    want = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :top]
    t = torch.zeros(rows, dtype=torch.int64, device=DEV)
    for again in range(3):
        lp, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        ids = torch.empty(rows, top, dtype=torch.int32, device=DEV)
        tlp = torch.empty(rows, top, device=DEV)
        twa.twa_token_logprobs(ctx, z, t, lp, lse, top_ids=ids, top_logp=tlp)
        assert torch.equal(ids.long(), want)
    ok(ctx)


def test_logprobs_report_a_wait_that_ran_out(ctx):
    """Rows of equal logits keep the warps that finish rows busy for milliseconds, and the summing warps wait for them: with a
    limit of one millisecond that wait runs out, which has to be reported; with the usual one nothing is wrong."""
    vocab, top = 1 << 21, 4
    rows = 5 * 2 * torch.cuda.get_device_properties(0).multi_processor_count       # five for each resident block
    z = torch.zeros(rows, vocab, dtype=BF16, device=DEV)
    t = torch.zeros(rows, dtype=torch.int64, device=DEV)
    logp, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ids, tlp = torch.empty(rows, top, dtype=torch.int32, device=DEV), torch.empty(rows, top, device=DEV)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_WAIT_LIMIT_MS, 1)
    try:
        twa.twa_token_logprobs(ctx, z, t, logp, lse, top_ids=ids, top_logp=tlp)
        assert twa.twa_get_status(ctx)[0] == twa.TWA_ERR_TIMEOUT
    finally:
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_WAIT_LIMIT_MS, 0)
        twa.twa_clear_status(ctx)
    twa.twa_token_logprobs(ctx, z, t, logp, lse, top_ids=ids, top_logp=tlp)
    assert bool((ids == torch.arange(top, device=DEV)).all())
    want = torch.full((rows,), math.log(vocab), dtype=torch.float64, device=DEV)
    tol, _ = logprob_tolerances(z[:1], vocab)
    close(lse, want, tol + 2 * U * want)
    assert torch.equal(logp, -lse) and torch.equal(tlp, -lse[:, None].expand(rows, top))
    ok(ctx)


# ------------------------------------------------------------------------------------------- streams, graphs, refusals
def test_operators_replay_from_a_graph_on_a_stream_of_their_own(ctx):
    g = gen(21)
    rows, cols, vocab = 64, 128, 1003
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        own = twa.twa_create(0)
        table, ids = randn(g, vocab, cols), torch.randint(0, vocab, (rows,), generator=g, device=DEV)
        x, y, dx = (torch.empty(rows, cols, device=DEV) for _ in range(3))
        w, mean, rstd, dw, db = randn(g, cols), *(torch.empty(n, device=DEV) for n in (rows, rows, cols, cols))
        z, dz, logp, lse = randn(g, rows, vocab), torch.empty(rows, vocab, device=DEV), *(torch.empty(rows, device=DEV) for _ in range(2))
        grad, flat, norm = torch.empty_like(table), torch.empty(vocab * cols + 2 * cols, device=DEV), torch.empty(1, device=DEV)
        ws = torch.empty(max(twa.twa_layer_norm_workspace_bytes(rows, cols), twa.twa_embedding_workspace_bytes(rows, vocab, cols),
                             twa.twa_grad_norm_workspace_bytes(3)), dtype=torch.uint8, device=DEV)
        ts, minus = twa.Tensors([grad, dw, db]), torch.full((rows,), -1.0 / rows, device=DEV)

        def step():
            twa.twa_embedding(own, table, ids, 2.0, x)
            twa.twa_layer_norm(own, x, w, None, 1e-5, y, mean, rstd)
            twa.twa_token_logprobs(own, z, ids, logp, lse)
            twa.twa_token_logprobs_backward(own, z, ids, lse, minus, dz)
            twa.twa_layer_norm_backward(own, y, x, w, mean, rstd, dx, dw, db, ws)
            twa.twa_embedding_backward(own, dx, ids, 2.0, grad, ws)
            twa.twa_clip_gather(own, ts, 1.0, flat, norm, ws)

        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        table.mul_(1.5)
        z.add_(0.25 * randn(g, rows, vocab))
        graph.replay()
        stream.synchronize()
        replayed = [t.clone() for t in (x, y, logp, dz, dx, dw, grad, flat, norm)]
        step()
        stream.synchronize()
        for a, b in zip(replayed, (x, y, logp, dz, dx, dw, grad, flat, norm)):
            assert torch.equal(a, b)
        assert twa.twa_get_status(own)[0] == 0
        twa.twa_destroy(own)


def test_empty_inputs(ctx):
    x = torch.empty(0, 16, device=DEV)
    twa.twa_layer_norm(ctx, x, None, None, 1e-5, x.clone(), torch.empty(0, device=DEV), torch.empty(0, device=DEV))
    dw = torch.full((16,), 4.0, device=DEV)
    ws = torch.empty(max(twa.twa_layer_norm_workspace_bytes(0, 16), twa.twa_embedding_workspace_bytes(0, 5, 16)), dtype=torch.uint8,
                     device=DEV)
    none = torch.empty(0, device=DEV)
    twa.twa_layer_norm_backward(ctx, x, x, None, none, none, x.clone(), dw, None, ws)
    assert bool((dw == 0).all())
    ids = torch.empty(0, dtype=torch.int64, device=DEV)
    grad = torch.full((5, 16), 4.0, device=DEV)
    twa.twa_embedding(ctx, grad, ids, 1.0, x.clone())
    twa.twa_embedding_backward(ctx, x, ids, 1.0, grad, ws, accumulate=True)
    assert bool((grad == 4).all())
    twa.twa_embedding_backward(ctx, x, ids, 1.0, grad, ws)
    assert bool((grad == 0).all())
    twa.twa_token_logprobs(ctx, x, ids, none, none.clone())
    twa.twa_token_logprobs_backward(ctx, x, ids, none, none, x.clone())
    ok(ctx)


def test_pointers_of_empty_arrays_are_not_looked_at(ctx):
    lib, odd = twa.load(), 7                      # on no element's boundary
    ws, out = torch.empty(1 << 16, dtype=torch.uint8, device=DEV), torch.full((4, 16), 3.0, device=DEV)
    dw, norm = torch.full((16,), 3.0, device=DEV), torch.full((1,), 3.0, device=DEV)
    assert lib.twa_layer_norm(ctx, odd, 16, 0, None, None, 0, 0, 16, 1e-5, odd, 16, odd, odd) == 0
    assert lib.twa_layer_norm_backward(ctx, odd, 16, odd, 16, 0, None, 0, odd, odd, 0, 16, odd, 16, dw.data_ptr(), None, 0, 0,
                                       ws.data_ptr(), ws.nbytes) == 0
    assert lib.twa_embedding(ctx, out.data_ptr(), 16, 0, 4, 16, odd, 1, 0, 1.0, odd, 16, 0) == 0
    assert lib.twa_embedding_backward(ctx, odd, 16, 0, odd, 1, 0, 4, 16, 1.0, -1, out.data_ptr(), 16, 0, 0, ws.data_ptr(), ws.nbytes) == 0
    assert lib.twa_token_logprobs(ctx, odd, 8, 0, 0, 8, odd, 1, -100, odd, odd, odd, 4, odd, odd) == 0
    assert lib.twa_token_logprobs_backward(ctx, odd, 8, 0, 0, 8, odd, 1, -100, odd, odd, odd, odd, odd, 8) == 0
    two = (ctypes.c_void_p * 2)(odd, dw.data_ptr()), (ctypes.c_int64 * 2)(0, 16), (ctypes.c_int32 * 2)(0, 0)
    t = twa.twa_tensors(*(ctypes.addressof(a) for a in two), 2)
    assert lib.twa_grad_norm(ctx, ctypes.byref(t), norm.data_ptr(), ws.data_ptr(), ws.nbytes) == 0
    assert bool((dw == 0).all()) and bool((out == 0).all()) and float(norm) == 0.0
    ok(ctx)


def refused(code, call, *args, **kw):
    with pytest.raises(twa.TwaError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_refusals(ctx):
    x, v = torch.zeros(4, 8, device=DEV), torch.zeros(4, device=DEV)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    w, small = torch.zeros(8, device=DEV), torch.empty(8, dtype=torch.uint8, device=DEV)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    refused(twa.TWA_ERR_INVALID_ARG, twa.twa_layer_norm, ctx, x, w, w, -1.0, x)
    refused(twa.TWA_ERR_INVALID_ARG, twa.twa_layer_norm, ctx, x, w, w, math.nan, x)
    refused(twa.TWA_ERR_WORKSPACE, twa.twa_layer_norm_backward, ctx, x, x, w, v, v, x, w, w, small)
    refused(twa.TWA_ERR_WORKSPACE, twa.twa_layer_norm_backward, ctx, x, x, w, v, v, x, w, w, None)
    refused(twa.TWA_ERR_MISALIGNED, twa.twa_layer_norm_backward, ctx, x, x, w, v, v, x, w, w, ws[1:])
    refused(twa.TWA_ERR_WORKSPACE, twa.twa_embedding_backward, ctx, x, ids, 1.0, x, small)
    many = torch.empty(twa.TWA_EMBEDDING_MAX_VOCAB + 1, 1, dtype=BF16, device=DEV)
    refused(twa.TWA_ERR_UNSUPPORTED, twa.twa_embedding, ctx, many, ids, 1.0, x[:, :1])
    refused(twa.TWA_ERR_UNSUPPORTED, twa.twa_embedding_backward, ctx, x[:, :1], ids, 1.0, many, ws)
    del many
    refused(twa.TWA_ERR_INVALID_ARG, twa.twa_token_logprobs, ctx, x, ids, v, v, top_ids=torch.zeros(4, 9, dtype=torch.int32, device=DEV),
            top_logp=torch.zeros(4, 9, device=DEV))
    wide = torch.zeros(4, 64, device=DEV)
    refused(twa.TWA_ERR_UNSUPPORTED, twa.twa_token_logprobs, ctx, wide, ids, v, v,
            top_ids=torch.zeros(4, 33, dtype=torch.int32, device=DEV), top_logp=torch.zeros(4, 33, device=DEV))
    refused(twa.TWA_ERR_INVALID_ARG, twa.twa_token_logprobs_backward, ctx, x, ids, v, v, x, d_entropy=v)
    ts, norm = twa.Tensors([x.view(-1)]), torch.zeros(1, device=DEV)
    refused(twa.TWA_ERR_INVALID_ARG, twa.twa_clip_gather, ctx, ts, 0.0, torch.zeros(32, device=DEV), norm, ws)
    refused(twa.TWA_ERR_INVALID_ARG, twa.twa_clip_gather, ctx, ts, math.nan, torch.zeros(32, device=DEV), norm, ws)
    refused(twa.TWA_ERR_WORKSPACE, twa.twa_grad_norm, ctx, ts, norm, small)
    # what the binding sees for itself
    with pytest.raises(TypeError):
        twa.twa_layer_norm(ctx, x.half(), None, None, 1e-5, x.half())
    with pytest.raises(TypeError):
        twa.twa_embedding(ctx, x, ids.to(torch.int16), 1.0, x)
    with pytest.raises(TypeError):
        twa.Tensors([x.half()])
    for call in (lambda: twa.twa_layer_norm(ctx, x, w[:4], None, 1e-5, x), lambda: twa.twa_layer_norm(ctx, x, w, None, 1e-5, x[:2]),
                 lambda: twa.twa_layer_norm(ctx, x.t(), None, None, 1e-5, x.t()),
                 lambda: twa.twa_embedding(ctx, x, ids, 1.0, x[:, :4]), lambda: twa.twa_token_logprobs(ctx, x, ids[:2], v, v),
                 lambda: twa.twa_token_logprobs(ctx, x, ids, v[:2], v), lambda: twa.Tensors([x.t()]), lambda: twa.Tensors([x.cpu()]),
                 lambda: twa.twa_layer_norm(ctx, x.cpu(), w, None, 1e-5, x), lambda: twa.twa_embedding(ctx, x, ids.cpu(), 1.0, x),
                 lambda: twa.twa_layer_norm_backward(ctx, x, x, w, v, v.cpu(), x, w, w, ws),
                 lambda: twa.twa_clip_gather(ctx, ts, 1.0, torch.zeros(31, device=DEV), norm, ws)):
        with pytest.raises(ValueError):
            call()
    ok(ctx)
