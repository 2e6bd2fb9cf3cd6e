"""A small language model trained in the subspace of its own checkpoints: every operator between the lifted weights w and
the gradient g that a step takes, as a program runs them together.

    python -m paper_2205_13104_b200.language_model

The model predicts the next token from the present one: embedding (scaled by sqrt(dim)), layer norm, a two-layer
perceptron with a residual connection, layer norm, and an output layer that shares the embedding's table.  Its
parameters are slices of one flat float32 vector, as the lift writes it.  Stage one trains all parameters by gradient descent
and keeps checkpoints; stage two (Algorithm 1 of the paper) trains the coefficients of the checkpoints' basis, 8 bits a
value, from the flat clipped gradient.  Matrix products are torch's; everything else is this library's.
"""

from __future__ import annotations

import argparse
import math

import torch

from . import twa
from .inputs import padded_ld

EPS = 1e-5


class LanguageModel:
    """Buffers and calls of one model of `vocab` tokens, width `dim`, `hidden` units, for batches of `tokens` tokens."""

    def __init__(self, vocab, dim, hidden, tokens, device="cuda:0"):
        self.vocab, self.dim, self.hidden, self.tokens = vocab, dim, hidden, tokens
        self.shapes = [("table", (vocab, dim)), ("norm1_w", (dim,)), ("norm1_b", (dim,)), ("up", (hidden, dim)), ("down", (dim, hidden)),
                       ("norm2_w", (dim,)), ("norm2_b", (dim,))]
        self.D = sum(math.prod(s) for _, s in self.shapes)
        self.device = device
        self.ctx = twa.twa_create(torch.device(device).index or 0)

        def new(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=device)

        self.grads = {name: new(*shape) for name, shape in self.shapes}
        self.tensors = twa.Tensors(self.grads.values())
        self.g, self.norm = new(self.D), new(1)
        self.x0, self.y1, self.x1, self.y2, self.dx = (new(tokens, dim) for _ in range(5))
        self.stats = [new(tokens) for _ in range(4)]              # mean and 1 / deviation of both norms
        self.logp, self.lse, self.entropy = (new(tokens) for _ in range(3))
        self.weight = torch.full((tokens,), -1.0 / tokens, device=device)
        self.ws = new(max(twa.twa_layer_norm_workspace_bytes(tokens, dim), twa.twa_embedding_workspace_bytes(tokens, vocab, dim),
                          twa.twa_grad_norm_workspace_bytes(self.tensors)), dtype=torch.uint8)

    def close(self):
        twa.twa_destroy(self.ctx)

    def split(self, w):
        """The parameters as slices of the flat vector."""
        out, at = {}, 0
        for name, shape in self.shapes:
            n = math.prod(shape)
            out[name] = w[at: at + n].view(shape)
            at += n
        return out

    def initial(self, seed):
        gen = torch.Generator(device=self.device)
        gen.manual_seed(seed)
        w = torch.empty((self.D,), device=self.device)
        p = self.split(w)
        for name in ("table", "up", "down"):
            p[name].copy_(torch.randn(p[name].shape, generator=gen, device=self.device) / math.sqrt(p[name].shape[1]))
        for name in ("norm1", "norm2"):
            p[name + "_w"].fill_(1.0)
            p[name + "_b"].zero_()
        return w

    def logits(self, w, ids):
        p, ctx = self.split(w), self.ctx
        twa.twa_embedding(ctx, p["table"], ids, math.sqrt(self.dim), self.x0)
        twa.twa_layer_norm(ctx, self.x0, p["norm1_w"], p["norm1_b"], EPS, self.y1, self.stats[0], self.stats[1])
        self.act = torch.relu(self.y1 @ p["up"].T)
        torch.add(self.x0, self.act @ p["down"].T, out=self.x1)
        twa.twa_layer_norm(ctx, self.x1, p["norm2_w"], p["norm2_b"], EPS, self.y2, self.stats[2], self.stats[3])
        return self.y2 @ p["table"].T

    def loss(self, w, ids, targets):
        """Mean of -log p of the targets (a device scalar); fills logp, lse and the distributions' entropy."""
        self.z = self.logits(w, ids)
        twa.twa_token_logprobs(self.ctx, self.z, targets, self.logp, self.lse, entropy=self.entropy)
        return -self.logp.mean()

    def gradient(self, w, ids, targets, max_norm):
        """The loss, and its gradient clipped to max_norm as one flat vector in self.g."""
        loss = self.loss(w, ids, targets)
        p, g, ctx = self.split(w), self.grads, self.ctx
        twa.twa_token_logprobs_backward(ctx, self.z, targets, self.lse, self.weight, self.z)            # in place
        torch.mm(self.z.T, self.y2, out=g["table"])
        dy = self.z @ p["table"]
        twa.twa_layer_norm_backward(ctx, dy, self.x1, p["norm2_w"], self.stats[2], self.stats[3], self.dx, g["norm2_w"],
                                    g["norm2_b"], self.ws)
        torch.mm(self.dx.T, self.act, out=g["down"])
        dact = (self.dx @ p["down"]).mul_(self.act > 0)
        torch.mm(dact.T, self.y1, out=g["up"])
        twa.twa_layer_norm_backward(ctx, dact @ p["up"], self.x0, p["norm1_w"], self.stats[0], self.stats[1], dy, g["norm1_w"],
                                    g["norm1_b"], self.ws)
        dy.add_(self.dx)
        # the table is the output layer's too: the lookup's gradient is added to what is there
        twa.twa_embedding_backward(ctx, dy, ids, math.sqrt(self.dim), g["table"], self.ws, accumulate=True)
        twa.twa_clip_gather(ctx, self.tensors, max_norm, self.g, self.norm, self.ws)
        return loss


class Text:
    """Batches of a synthetic text: each token is followed by one of four, often by the first."""

    def __init__(self, vocab, seed, device):
        self.gen = torch.Generator(device=device)
        self.gen.manual_seed(seed)
        self.next = torch.randint(0, vocab, (vocab, 4), generator=self.gen, device=device)
        self.odds = torch.tensor([0.7, 0.15, 0.1, 0.05], device=device)
        self.vocab = vocab

    def batch(self, tokens):
        u = torch.rand((tokens,), generator=self.gen, device=self.next.device)
        ids = (torch.exp(u * math.log(self.vocab + 1)) - 1).long().clamp_(0, self.vocab - 1)            # frequent and rare ones
        which = torch.multinomial(self.odds, tokens, replacement=True, generator=self.gen)
        return ids, self.next[ids, which]


def train(vocab=2000, dim=128, hidden=512, tokens=4096, checkpoints=10, between=20, steps=40, lr=2.0, subspace_lr=2.0, max_norm=1.0,
          seed=0, device="cuda:0", say=print):
    """Stage one and stage two; returns the losses on fresh text of the last checkpoint, of the checkpoints' mean and of the
    weights that the subspace training found."""
    model, text = LanguageModel(vocab, dim, hidden, tokens, device), Text(vocab, seed + 1, device)
    return stages(model, text, checkpoints, between, steps, lr, subspace_lr, max_norm, seed, say)


def stages(model, text, checkpoints, between, steps, lr, subspace_lr, max_norm, seed, say):
    """Both stages for a model and its text; closes the model."""
    device, tokens = model.device, model.tokens
    w = model.initial(seed)
    W = torch.zeros((checkpoints, padded_ld(model.D)), device=device)
    for step in range((checkpoints + 2) * between):
        loss = model.gradient(w, *text.batch(tokens), max_norm)
        w.add_(model.g, alpha=-lr)
        taken = step + 1 - 3 * between                             # checkpoints after a while, every `between` steps
        if taken >= 0 and taken % between == 0 and taken // between < checkpoints:
            W[taken // between, : model.D] = w
            say(f"step {step + 1}: loss {float(loss):.4f}, gradient norm {float(model.norm):.3f}, "
                f"entropy {float(model.entropy.mean()):.3f}")
    held_out = [text.batch(tokens) for _ in range(8)]

    def measure(weights):
        return float(sum(model.loss(weights, *b) for b in held_out)) / len(held_out)

    last = measure(w)
    ws, wbar = twa.new_workspace(device), torch.empty(model.D, device=device)
    _, (P,) = twa.twa_build_quantized(model.ctx, W, model.D, wbar, [8], ws)
    alpha, lifted = torch.zeros(checkpoints, device=device), wbar.clone()
    mean = measure(lifted)
    for _ in range(steps):
        model.gradient(lifted, *text.batch(tokens), max_norm)
        twa.twa_step(model.ctx, P, model.g, subspace_lr, 0.0, alpha, wbar, lifted, ws)
    found = measure(lifted)
    code, detail = twa.twa_get_status(model.ctx)
    if code:
        raise twa.TwaError(code, "stages", f"detail {detail}")
    say(f"loss on fresh text: last checkpoint {last:.4f}, mean of {checkpoints} checkpoints {mean:.4f}, "
        f"after {steps} steps in their subspace {found:.4f}")
    model.close()
    return last, mean, found


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=40, help="steps in the subspace")
    p.add_argument("--checkpoints", type=int, default=10)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    train(checkpoints=a.checkpoints, steps=a.steps, seed=a.seed)


if __name__ == "__main__":
    main()
