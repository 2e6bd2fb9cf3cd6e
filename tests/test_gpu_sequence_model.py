"""The example that runs the sequence model's operators together: its gradient against automatic differentiation in 64 bits, a short
training run in the subspace of its checkpoints, and generation a token at a time against whole sequences."""

import math

import pytest
import torch

from paper_2205_13104_b200 import language_model as lm
from paper_2205_13104_b200 import sequence_model as sm
from paper_2205_13104_b200 import twa
from philox import dropout_numbers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def float32_products():
    torch.cuda.set_device(0)
    allow = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    yield
    torch.backends.cuda.matmul.allow_tf32 = allow


def reference_loss(model, w, ids, targets, starts, chosen, drop):
    """drop: what the two dropouts multiply by."""
    p = model.split(w)

    def norm(x, number):
        d = x - x.mean(1, keepdim=True)
        return d / torch.sqrt((d * d).mean(1, keepdim=True) + lm.EPS) * p[f"norm{number}_w"] + p[f"norm{number}_b"]

    x0 = p["table"][ids] * math.sqrt(model.dim)
    y1 = norm(x0, 1)
    u, a = y1 @ p["inputs"].T, torch.sigmoid(y1 @ p["gates"].T + p["gates_b"])
    rows, edges = [], starts.tolist()
    for begin, end in zip(edges, edges[1:]):
        h = torch.zeros(model.dim, dtype=w.dtype, device=w.device)
        for t in range(begin, end):
            h = a[t] * h + (1 - a[t]) * u[t]
            rows.append(h)
    x1 = x0 + drop[0] * (torch.stack(rows) @ p["mixed"].T)
    y2 = norm(x1, 2)
    odds = torch.softmax(y2 @ p["router"].T, 1).gather(1, chosen)
    out = 0.0
    for j in range(model.top):
        act = torch.relu(torch.einsum("thd,td->th", p["up"][chosen[:, j]], y2))
        out = out + odds[:, j, None] * torch.einsum("tdh,th->td", p["down"][chosen[:, j]], act)
    x2 = x1 + drop[1] * out
    z = norm(x2, 3) @ p["table"].T
    return -(z.gather(1, targets[:, None])[:, 0] - torch.logsumexp(z, 1)).mean()


@pytest.mark.parametrize("vocab,dim,hidden,experts,top,tokens,sequences", [(50, 16, 24, 4, 2, 60, 5), (301, 33, 20, 7, 3, 129, 2)])
def test_gradient_of_the_sequence_model(vocab, dim, hidden, experts, top, tokens, sequences):
    model = sm.SequenceModel(vocab, dim, hidden, experts, top, tokens, sequences, dropout=0.25, seed=11)
    text = sm.Text(vocab, 3, sequences, 3, DEV)
    w = model.initial(1)
    w += 0.05 * torch.randn(w.shape, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    ids, targets, starts = text.batch(tokens)
    loss = model.gradient(w, ids, targets, starts, 1e6)                # nothing is clipped
    drop = [torch.from_numpy(dropout_numbers(11, 1, site, tokens, dim) >= 16384).to(DEV) / 0.75 for site in (sm.RECURRENCE, sm.EXPERTS)]
    w64 = w.double().requires_grad_()
    want = reference_loss(model, w64, ids, targets, starts, model.chosen.long(), [d.double() for d in drop])
    want.backward()
    want = float(want.detach())
    assert abs(float(loss) - want) <= 1e-5 * abs(want)
    # float32 through some twenty operations, sums of at most a few hundred terms: 1e-4 of the gradient's length leaves room
    error = (model.g.double() - w64.grad).norm() / w64.grad.norm()
    assert float(error) <= 1e-4
    full, step = model.g.clone(), int(model.rng[1])
    model.rng[1] = step - 1                                            # the same dropout once more
    model.gradient(w, ids, targets, starts, 0.5 * float(model.norm))
    assert torch.allclose(model.g, 0.5 * full, rtol=1e-5, atol=0)
    assert twa.twa_get_status(model.ctx)[0] == 0
    model.close()


def test_generation_is_the_whole_sequence():
    """Logits of a sequence that goes on a token a call, its states carried, against those of the sequence at once."""
    vocab, dim, n, count = 40, 24, 6, 20
    model = sm.SequenceModel(vocab, dim, 16, 4, 2, n * (count + 1), n)
    w = model.initial(5)
    first = torch.arange(n, device=DEV)
    said = model.generate(w, first, count)
    assert said.shape == (count, n) and bool(((said >= 0) & (said < vocab)).all())
    ids = torch.cat([first[None], said[:-1].long()]).T.contiguous().view(-1)
    z = model.logits(w, ids, torch.arange(n + 1, device=DEV) * count)
    best = z.view(n, count, vocab).topk(2, -1)
    sure = best.values[..., 0] - best.values[..., 1] > 1e-3            # float32 rounding moves logits of order one by far less
    assert bool((best.indices[..., 0] == said.T)[sure].all()) and float(sure.float().mean()) > 0.5
    assert twa.twa_get_status(model.ctx)[0] == 0
    model.close()


def test_training_in_the_subspace_of_checkpoints():
    said = []
    losses = sm.train(vocab=100, dim=32, hidden=32, experts=4, tokens=1024, sequences=16, checkpoints=6, between=5, steps=10, say=said.append)
    assert all(math.isfinite(v) for v in losses)
    assert len(said) == 7
