"""Routing queries by what a small model's answers say, and the routing's bias searched by the loop.

A small model has answered a set of queries (synthetic logits: easy queries have sharp
distributions). On the device, every answer's tokens become log-probabilities and
entropies (boute_token_logprobs), every answer one row of scores (boute_answer_scores),
and a linear router sends each query to a replica of one of the models (boute_route).

  train   the router's weights, by the gradient of the expected error through
          boute_route_grad (and on to the model's logits, through
          boute_answer_scores_grad and boute_token_logprobs_grad)
  search  one bias per model, the decision vector of boute_mobo_run: each evaluation
          routes all queries and returns the slowest replica's time and the mean error

Run: python examples/route_queries.py
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2602_10729_gb300 import boute as bt  # noqa: E402

F32, I32, I64 = torch.float32, torch.int32, torch.int64
WEAKNESS = (1.0, 0.35)  # a model's error on the hardest query
COST = (1.0, 4.0)       # its time per query of one replica


class Answers:
    """A small model's answers to `queries` queries: tokens, logits, offsets, difficulty."""

    def __init__(self, queries=2048, vocabulary=4096, seed=0):
        g = torch.Generator().manual_seed(seed)
        n = (8 + torch.rand(queries, generator=g) * 48).long()
        self.offsets = torch.cat([torch.zeros(1, dtype=I64), n.cumsum(0)]).cuda()
        self.difficulty = torch.rand(queries, generator=g).cuda()
        T = int(n.sum())
        z = torch.randn((T, vocabulary), generator=g).cuda()
        sharp = 9.0 - 6.0 * self.difficulty.repeat_interleave(n.cuda())
        first = torch.randint(0, vocabulary, (T,), generator=g).cuda()
        z[torch.arange(T, device="cuda"), first] += sharp
        self.logits, self.targets = z.to(torch.bfloat16), first

    def scores(self):
        """One row of four scores per answer, with what the backward pass needs."""
        T, Q = self.logits.shape[0], self.offsets.shape[0] - 1
        f = lambda *s: torch.empty(s, device="cuda")
        self.logprob, self.entropy, self.lse = f(T), f(T), f(T)
        top, top_logprob = torch.empty((T, 2), dtype=I64, device="cuda"), f(T, 2)
        bt.boute_token_logprobs(self.logits, self.targets, 1.0, self.logprob, self.entropy,
                                self.lse, top, top_logprob)
        out, counts = f(Q, 4), torch.empty(Q, dtype=I32, device="cuda")
        bt.boute_answer_scores(self.logprob, self.entropy, self.targets, self.offsets, out, counts)
        return out

    def backward(self, g_scores):
        """The gradient of the logits for the gradient of the scores."""
        gl, gh = torch.empty_like(self.logprob), torch.empty_like(self.entropy)
        bt.boute_answer_scores_grad(self.logprob, self.entropy, self.targets, self.offsets,
                                    g_scores, gl, gh)
        dx = torch.empty_like(self.logits)
        bt.boute_token_logprobs_grad(self.logits, self.targets, 1.0, self.lse, self.entropy, gl,
                                     gh, dx)
        return dx


class Router:
    """A linear router over standardised scores: `models` models of `replicas` replicas each."""

    def __init__(self, scores, models=2, replicas=4, seed=1):
        self.models, self.replicas = models, replicas
        self.mean, self.std = scores.mean(0), scores.std(0)
        g = torch.Generator().manual_seed(seed)
        self.W = (torch.randn((5, models * replicas), generator=g) * 0.1).cuda()

    def features(self, scores):
        x = (scores - self.mean) / self.std
        return torch.cat([x, torch.ones_like(x[:, :1])], 1)

    def logits(self, scores):
        return (self.features(scores) @ self.W).contiguous()

    def route(self, x, k, bias=None, mode=bt.BOUTE_ROUTE_SOFTMAX, keep=None):
        Q, E = x.shape
        idx = torch.empty((Q, k), dtype=I32, device="cuda")
        w, load = torch.empty((Q, k), device="cuda"), torch.empty(E, dtype=I32, device="cuda")
        bt.boute_route(x, bias, mode, self.models, keep or self.models, 1, True, 1.0, idx, w, load)
        return idx, w, load


def errors(router, answers, idx):
    """The error of each query at each chosen replica's model."""
    weakness = torch.tensor(WEAKNESS, device="cuda")
    return answers.difficulty[:, None] * weakness[(idx // router.replicas).long()]


def train(router, answers, steps=60, lr=0.5):
    """Gradient descent on the expected error plus the expected time, k = 4 replicas a query."""
    scores = answers.scores()
    feats = router.features(scores)
    cost = 0.05 * torch.tensor(COST, device="cuda")
    losses = []
    for _ in range(steps):
        x = router.logits(scores)
        idx, w, _ = router.route(x, 4)
        loss_of = errors(router, answers, idx) + cost[(idx // router.replicas).long()]
        losses.append(float((w * loss_of).sum(1).mean()))
        dx = torch.empty_like(x)
        bt.boute_route_grad(x, bt.BOUTE_ROUTE_SOFTMAX, True, 1.0, idx,
                            (loss_of / x.shape[0]).contiguous(), dx)
        g_feats = dx @ router.W.t()
        router.W -= lr * feats.t() @ dx
    # the same gradient, on through the scores to the model's own logits
    g_logits = answers.backward((g_feats[:, :4] / router.std).contiguous())
    return losses, g_logits


def search(router, answers, evaluations=20, seed=0):
    """The loop over one bias per model: minimise (slowest replica's time, mean error)."""
    scores = answers.scores()
    x = router.logits(scores)
    cost = np.repeat(np.array(COST), router.replicas)

    def objective(theta):
        bias = torch.tensor(np.repeat(theta - 0.5, router.replicas), dtype=F32, device="cuda")
        idx, _, load = router.route(x, 1, bias, bt.BOUTE_ROUTE_SIGMOID, keep=1)
        slowest = float((load.cpu().numpy() * cost).max())
        return [slowest, float(errors(router, answers, idx).mean())]

    rng = np.random.default_rng(seed)
    X0 = rng.random((6, router.models))
    Y0 = np.array([objective(t) for t in X0])
    m, d = 2, router.models
    out = bt.boute_mobo_run(objective, rng.random((4096, d)), np.full(m, 1.1), np.full((m, d), 0.4),
                            np.ones(m), np.full(m, 1e-3), X0, Y0, max_evals=evaluations,
                            patience=evaluations)
    Y = out["Y"]
    front = [i for i in range(len(Y)) if not any((Y[j] <= Y[i]).all() and (Y[j] < Y[i]).any()
                                                 for j in range(len(Y)))]
    return out, front


def main(queries=2048, vocabulary=4096, steps=60, evaluations=20):
    answers = Answers(queries, vocabulary)
    router = Router(answers.scores())
    losses, g_logits = train(router, answers, steps)
    print(f"training: expected loss {losses[0]:.4f} -> {losses[-1]:.4f}, "
          f"gradient of the logits {float(g_logits.float().norm()):.3g}")
    out, front = search(router, answers, evaluations)
    for i in sorted(front, key=lambda i: out["Y"][i][0]):
        print(f"bias {np.round(out['X'][i] - 0.5, 3)}: slowest replica {out['Y'][i][0]:.0f}, "
              f"error {out['Y'][i][1]:.4f}")
    return dict(losses=losses, g_logits=g_logits, search=out, front=front)


if __name__ == "__main__":
    main()
