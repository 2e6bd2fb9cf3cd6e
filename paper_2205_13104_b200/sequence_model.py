"""A small sequence model trained in the subspace of its own checkpoints, and texts generated from it: the operators of
language_model.py and those that tokens of a sequence need to see each other, with experts and dropout.

    python -m paper_2205_13104_b200.sequence_model

The model predicts the next token from all before it: embedding (scaled by sqrt(dim)); layer norm and a gated linear recurrence
whose inputs and gates are products of the normed tokens; layer norm and a few two-layer perceptrons, the experts, of which each
token is sent to the `top` that a router finds most likely, their results weighted by the router's probabilities; layer norm and an
output layer that shares the embedding's table.  Both blocks have a residual connection and dropout.  A batch is a number of
sequences of different lengths one after another.  Its parameters are slices of one flat float32 vector, as the lift writes it.
Matrix products and the router's gradient are torch's; everything else is this library's.
"""

from __future__ import annotations

import argparse
import math

import torch

from . import language_model as lm
from . import twa

RECURRENCE, EXPERTS = 0, 1                                        # the two dropouts


class SequenceModel:
    """Buffers and calls of one model of `vocab` tokens, width `dim`, `experts` perceptrons of `hidden` units, for batches of
    `tokens` tokens in at most `sequences` sequences."""

    def __init__(self, vocab, dim, hidden, experts, top, tokens, sequences, dropout=0.1, seed=0, device="cuda:0"):
        self.vocab, self.dim, self.hidden, self.experts, self.top = vocab, dim, hidden, experts, top
        self.tokens, self.sequences, self.dropout, self.device = tokens, sequences, dropout, device
        self.shapes = [("table", (vocab, dim)), ("norm1_w", (dim,)), ("norm1_b", (dim,)), ("inputs", (dim, dim)), ("gates", (dim, dim)),
                       ("gates_b", (dim,)), ("mixed", (dim, dim)), ("norm2_w", (dim,)), ("norm2_b", (dim,)), ("router", (experts, dim)),
                       ("up", (experts, hidden, dim)), ("down", (experts, dim, hidden)), ("norm3_w", (dim,)), ("norm3_b", (dim,))]
        self.D = sum(math.prod(s) for _, s in self.shapes)
        self.ctx = twa.twa_create(torch.device(device).index or 0)

        def new(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=device)

        self.grads = {name: new(*shape) for name, shape in self.shapes}
        self.tensors = twa.Tensors(self.grads.values())
        self.g, self.norm = new(self.D), new(1)
        self.rng = torch.tensor([seed, 0], device=device)            # seed and step of the dropouts
        self.x0, self.y1, self.h, self.x1, self.y2, self.x2, self.y3, self.dx, self.dy, self.du, self.df = (new(tokens, dim) for _ in range(11))
        self.stats = [new(tokens) for _ in range(6)]                  # mean and 1 / deviation of the norms
        self.states = new(twa.twa_gated_scan_states_bytes(tokens, sequences, dim), dtype=torch.uint8)
        self.place, self.starts = new(tokens, top, dtype=torch.int32), new(experts + 1, dtype=torch.int32)
        self.rows, self.made, self.drows, self.act = new(tokens * top, dim), new(tokens * top, dim), new(tokens * top, dim), new(tokens * top, hidden)
        self.chosen, self.odds = new(tokens, top, dtype=torch.int32), new(tokens, top)
        self.none = torch.full((tokens,), -100, device=device)        # the router has no targets
        self.logp, self.lse, self.entropy, self.router_logp, self.router_lse = (new(tokens) for _ in range(5))
        self.weight = torch.full((tokens,), -1.0 / tokens, device=device)
        self.ws = new(max(twa.twa_layer_norm_workspace_bytes(tokens, dim), twa.twa_embedding_workspace_bytes(tokens, vocab, dim),
                          twa.twa_grad_norm_workspace_bytes(self.tensors)), dtype=torch.uint8)

    def close(self):
        twa.twa_destroy(self.ctx)

    split = lm.LanguageModel.split

    def initial(self, seed):
        gen = torch.Generator(device=self.device)
        gen.manual_seed(seed)
        w = torch.empty((self.D,), device=self.device)
        for name, p in self.split(w).items():
            if name.startswith("norm") or name == "gates_b":
                p.fill_({"w": 1.0, "b": 0.0}[name[-1]] if name != "gates_b" else 1.5)         # gates that remember a few tokens
            else:
                p.copy_(torch.randn(p.shape, generator=gen, device=self.device) / math.sqrt(p.shape[-1]))
        return w

    def _added(self, x, site, residual, out, train):
        """out = residual + x, with dropout in training."""
        return twa.twa_dropout(self.ctx, x, self.dropout if train else 0.0, self.rng, site, out, residual)

    def _experts(self, p, n):
        """Sends y2's first n tokens to their experts and the results, weighted, back: (tokens, dim)."""
        ctx, place, chosen, odds = self.ctx, self.place[:n], self.chosen[:n], self.odds[:n]
        self.router_z = self.y2[:n] @ p["router"].T
        twa.twa_token_logprobs(ctx, self.router_z, self.none[:n], self.router_logp[:n], self.router_lse[:n], top_ids=chosen, top_logp=odds)
        odds.exp_()
        twa.twa_expert_dispatch(ctx, self.y2[:n], chosen, self.experts, place, self.starts, self.rows)
        self.edges = self.starts.tolist()
        for e, (a, b) in enumerate(zip(self.edges, self.edges[1:])):
            if b > a:
                torch.mm(self.rows[a:b], p["up"][e].T, out=self.act[a:b]).relu_()
                torch.mm(self.act[a:b], p["down"][e].T, out=self.made[a:b])
        return twa.twa_expert_combine(ctx, self.made, place, odds, torch.empty_like(self.y2[:n]))

    def logits(self, w, ids, starts, train=False, state=None):
        """Of every next token.  state: (sequences, dim) recurrence states of sequences that go on, replaced by those after `ids`
        (then starts None: equally many tokens for each)."""
        p, ctx, n = self.split(w), self.ctx, len(ids)
        x0, y1, h, x1, y2, x2, y3 = (t[:n] for t in (self.x0, self.y1, self.h, self.x1, self.y2, self.x2, self.y3))
        s = [t[:n] for t in self.stats]
        twa.twa_embedding(ctx, p["table"], ids, math.sqrt(self.dim), x0)
        twa.twa_layer_norm(ctx, x0, p["norm1_w"], p["norm1_b"], lm.EPS, y1, s[0], s[1])
        self.u, self.f = y1 @ p["inputs"].T, torch.addmm(p["gates_b"], y1, p["gates"].T)
        count = len(state) if starts is None else len(starts) - 1
        twa.twa_gated_scan(ctx, self.u, self.f, h, starts, count, state, state, self.states if train else None)
        self._added(h @ p["mixed"].T, RECURRENCE, x0, x1, train)
        twa.twa_layer_norm(ctx, x1, p["norm2_w"], p["norm2_b"], lm.EPS, y2, s[2], s[3])
        self._added(self._experts(p, n), EXPERTS, x1, x2, train)
        twa.twa_layer_norm(ctx, x2, p["norm3_w"], p["norm3_b"], lm.EPS, y3, s[4], s[5])
        return y3 @ p["table"].T

    def loss(self, w, ids, targets, starts, train=False):
        """Mean of -log p of the targets (a device scalar); fills logp, lse and the distributions' entropy."""
        self.z = self.logits(w, ids, starts, train)
        twa.twa_token_logprobs(self.ctx, self.z, targets, self.logp, self.lse, entropy=self.entropy)
        return -self.logp.mean()

    def gradient(self, w, ids, targets, starts, max_norm):
        """The loss with dropout drawn anew, and its gradient clipped to max_norm as one flat vector in self.g."""
        self.rng[1] += 1
        loss = self.loss(w, ids, targets, starts, train=True)
        p, g, ctx, s, drop = self.split(w), self.grads, self.ctx, self.stats, self.dropout

        def norm_back(dy, x, number, out):
            name = f"norm{number}"
            return twa.twa_layer_norm_backward(ctx, dy, x, p[name + "_w"], s[2 * number - 2], s[2 * number - 1], out, g[name + "_w"],
                                               g[name + "_b"], self.ws)

        twa.twa_token_logprobs_backward(ctx, self.z, targets, self.lse, self.weight, self.z)            # in place
        torch.mm(self.z.T, self.y3, out=g["table"])
        dx = norm_back(self.z @ p["table"], self.x2, 3, self.dx)
        # the experts: through the weights, the perceptrons and the router
        dodds = torch.empty_like(self.odds)
        twa.twa_expert_combine_backward(ctx, twa.twa_dropout_backward(ctx, dx, drop, self.rng, EXPERTS, self.dy), self.made, self.place, self.odds,
                                        self.made, dodds)
        for e, (a, b) in enumerate(zip(self.edges, self.edges[1:])):
            made, act = self.made[a:b], self.act[a:b]
            torch.mm(made.T, act, out=g["down"][e])
            dact = (made @ p["down"][e]).mul_(act > 0)
            torch.mm(dact.T, self.rows[a:b], out=g["up"][e])
            torch.mm(dact, p["up"][e], out=self.drows[a:b])
        share = dodds.mul_(self.odds)                                  # the odds are probabilities of a softmax over all experts
        drouter = (self.router_z - self.router_lse[:, None]).exp_().mul_(-share.sum(1, keepdim=True)).scatter_add_(1, self.chosen.long(), share)
        torch.mm(drouter.T, self.y2, out=g["router"])
        dy2 = twa.twa_expert_combine(ctx, self.drows, self.place, None, self.dy).addmm_(drouter, p["router"])
        dx.add_(norm_back(dy2, self.x1, 2, self.du))
        # the recurrence
        dmixed = twa.twa_dropout_backward(ctx, dx, drop, self.rng, RECURRENCE, self.dy)
        torch.mm(dmixed.T, self.h, out=g["mixed"])
        twa.twa_gated_scan_backward(ctx, dmixed @ p["mixed"], self.u, self.f, self.states, self.du, self.df, starts, len(starts) - 1)
        torch.mm(self.du.T, self.y1, out=g["inputs"])
        torch.mm(self.df.T, self.y1, out=g["gates"])
        torch.sum(self.df, 0, out=g["gates_b"])
        dx.add_(norm_back((self.du @ p["inputs"]).addmm_(self.df, p["gates"]), self.x0, 1, self.dy))
        # the table is the output layer's too: the lookup's gradient is added to what is there
        twa.twa_embedding_backward(ctx, dx, ids, math.sqrt(self.dim), g["table"], self.ws, accumulate=True)
        twa.twa_clip_gather(ctx, self.tensors, max_norm, self.g, self.norm, self.ws)
        return loss

    def generate(self, w, first, count):
        """`count` most likely tokens after each of `first`, (sequences,) ids: (count, sequences), a token of every sequence a call."""
        n = len(first)
        state = torch.zeros((n, self.dim), device=self.device)
        ids, out = first, []
        top, odds = torch.empty((n, 1), dtype=torch.int32, device=self.device), torch.empty((n, 1), device=self.device)
        for _ in range(count):
            z = self.logits(w, ids, None, state=state)
            twa.twa_token_logprobs(self.ctx, z, self.none[:n], self.logp[:n], self.lse[:n], top_ids=top, top_logp=odds)
            ids = top[:, 0].clone()
            out.append(ids)
        return torch.stack(out)


class Text:
    """Batches of a synthetic text: every sequence has a topic, which says what token follows which; it shows in the tokens only."""

    def __init__(self, vocab, topics, sequences, seed, device):
        self.gen = torch.Generator(device=device)
        self.gen.manual_seed(seed)
        self.follows = torch.randint(0, vocab, (topics, vocab), generator=self.gen, device=device)
        self.vocab, self.sequences, self.device = vocab, sequences, device

    def batch(self, tokens):
        """ids, the tokens after them, and where each of the sequences begins."""
        cuts = torch.randint(1, tokens, (self.sequences - 1,), generator=self.gen, device=self.device).sort().values.tolist()
        edges = [0, *cuts, tokens]
        longest = max(b - a for a, b in zip(edges, edges[1:]))
        topic = torch.randint(0, len(self.follows), (self.sequences,), generator=self.gen, device=self.device)
        text = torch.empty((longest + 1, self.sequences), dtype=torch.int64, device=self.device)
        text[0] = torch.randint(0, self.vocab, (self.sequences,), generator=self.gen, device=self.device)
        strange = torch.rand((longest, self.sequences), generator=self.gen, device=self.device) < 0.1
        other = torch.randint(0, self.vocab, (longest, self.sequences), generator=self.gen, device=self.device)
        for t in range(longest):
            text[t + 1] = torch.where(strange[t], other[t], self.follows[topic, text[t]])
        ids = torch.cat([text[: b - a, i] for i, (a, b) in enumerate(zip(edges, edges[1:]))])
        targets = torch.cat([text[1: b - a + 1, i] for i, (a, b) in enumerate(zip(edges, edges[1:]))])
        return ids, targets, torch.tensor(edges, dtype=torch.int32, device=self.device)


def train(vocab=500, dim=128, hidden=128, experts=8, top=2, tokens=4096, sequences=48, topics=4, checkpoints=10, between=20, steps=40, lr=2.0,
          subspace_lr=2.0, max_norm=1.0, dropout=0.1, seed=0, device="cuda:0", say=print):
    """Stage one and stage two as in language_model.py; returns the losses on fresh text of the last checkpoint, of the checkpoints'
    mean and of the weights that the subspace training found."""
    model = SequenceModel(vocab, dim, hidden, experts, top, tokens, sequences, dropout, seed, device)
    return lm.stages(model, Text(vocab, topics, sequences, seed + 1, device), checkpoints, between, steps, lr, subspace_lr, max_norm, seed, say)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=40, help="steps in the subspace")
    p.add_argument("--checkpoints", type=int, default=10)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    train(checkpoints=a.checkpoints, steps=a.steps, seed=a.seed)


if __name__ == "__main__":
    main()
