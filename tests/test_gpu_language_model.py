"""The example that runs the model's operators together: its gradient against automatic differentiation in 64 bits, and a
short training run in the subspace of its checkpoints."""

import math

import pytest
import torch

from paper_2205_13104_b200 import language_model as lm
from paper_2205_13104_b200 import twa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def reference_loss(model, w, ids, targets):
    p = model.split(w)
    x0 = p["table"][ids] * math.sqrt(model.dim)

    def norm(x, weight, bias):
        d = x - x.mean(1, keepdim=True)
        return d / torch.sqrt((d * d).mean(1, keepdim=True) + lm.EPS) * weight + bias

    y1 = norm(x0, p["norm1_w"], p["norm1_b"])
    x1 = x0 + torch.relu(y1 @ p["up"].T) @ p["down"].T
    z = norm(x1, p["norm2_w"], p["norm2_b"]) @ p["table"].T
    return -(z.gather(1, targets[:, None])[:, 0] - torch.logsumexp(z, 1)).mean()


@pytest.mark.parametrize("vocab,dim,hidden,tokens", [(50, 16, 24, 40), (301, 33, 48, 129)])
def test_gradient_of_the_language_model(vocab, dim, hidden, tokens):
    torch.cuda.set_device(0)
    allow = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        model, text = lm.LanguageModel(vocab, dim, hidden, tokens), lm.Text(vocab, 3, DEV)
        w = model.initial(1)
        w += 0.05 * torch.randn(w.shape, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
        ids, targets = text.batch(tokens)
        loss = model.gradient(w, ids, targets, 1e6)                # nothing is clipped
        w64 = w.double().requires_grad_()
        want = reference_loss(model, w64, ids, targets)
        want.backward()
        want = float(want.detach())
        assert abs(float(loss) - want) <= 1e-5 * abs(want)
        # float32 through some ten operations, sums of at most a few hundred terms: 1e-4 of the gradient's length leaves room
        error = (model.g.double() - w64.grad).norm() / w64.grad.norm()
        assert float(error) <= 1e-4
        assert abs(float(model.norm) / float(w64.grad.norm()) - 1) <= 1e-4
        full = model.g.clone()
        model.gradient(w, ids, targets, 0.5 * float(model.norm))
        assert torch.allclose(model.g, 0.5 * full, rtol=1e-5, atol=0)
        assert twa.twa_get_status(model.ctx)[0] == 0
        model.close()
    finally:
        torch.backends.cuda.matmul.allow_tf32 = allow


def test_training_in_the_subspace_of_checkpoints():
    said = []
    last, mean, found = lm.train(vocab=300, dim=32, hidden=64, tokens=1024, checkpoints=6, between=10, steps=20, say=said.append)
    assert all(math.isfinite(v) for v in (last, mean, found))
    assert found < mean                                            # steps down the gradient of the same text
    assert found < math.log(300)                                   # better than guessing
    assert len(said) == 7
