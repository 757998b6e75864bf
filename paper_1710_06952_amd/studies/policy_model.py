"""A small language policy trained by AD-PSGD workers with the library's operators of a training step: dense layers
with their epilogues, a policy or preference loss over the vocabulary, and AdamW with 8-bit moments.

Every worker has prompts of its own, each with one right answer token.  For an event the library hands the gradient
function the worker's stale row and the slot that receives a gradient (model "external", adpsgd_run_events_with).  The
function rounds the row to bfloat16 weights, runs

    h = dense(e, W1, b1, residual=e, activation="gelu"),   logits = dense(h, W2, b2)

on a minibatch of prompts, takes the loss with its gradient for the logits, lets autograd run the dense layers'
backward pass, and hands the event the worker's AdamW direction (clipped by the global norm) in the place of a gradient:
the event averages with a neighbour and steps along it.  Moments are the worker's own, as momentum buffers are.

  --loss policy       answers are sampled; reward 1 for the right one, less the batch's mean, and a KL term to the
                      initial model, whose log-probabilities come from token_log_probs
  --loss preference   pairs of answers of one token: the right one is chosen, a random one rejected

    python -m paper_1710_06952_amd.studies.policy_model [--loss policy] [--n 4] [--events 400] [--json]
"""
from __future__ import annotations

import argparse
import json

import numpy as np

from .convergence import ring


class Policy:
    """The network at a flat parameter vector [W1 | b1 | W2 | b2], W1 width x width, W2 vocab x width."""

    def __init__(self, vocab, width, prompts, seed, device):
        import torch
        self.vocab, self.width = vocab, width
        self.shapes = [(width, width), (width,), (vocab, width), (vocab,)]
        self.sizes = [int(np.prod(s)) for s in self.shapes]
        self.d = sum(self.sizes)
        rng = np.random.default_rng(seed)
        self.embeddings = torch.from_numpy(rng.standard_normal((prompts, width)).astype(np.float32)).to(device).bfloat16()

    def initial(self, seed):
        rng = np.random.default_rng(seed + 1)
        parts = [rng.standard_normal(s) / np.sqrt(self.width) if len(s) == 2 else np.zeros(s) for s in self.shapes]
        return np.concatenate([p.reshape(-1) for p in parts]).astype(np.float32)

    def views(self, flat):
        out, at = [], 0
        for shape, size in zip(self.shapes, self.sizes):
            out.append(flat[at:at + size].view(shape))
            at += size
        return out

    def logits(self, weights, prompts):
        import paper_1710_06952_amd as P
        w1, b1, w2, b2 = weights
        e = self.embeddings[prompts]
        h = P.dense(e, w1, b1, residual=e, activation="gelu")
        return P.dense(h, w2, b2)


class Worker:
    """One worker's weights in bfloat16, gradients, direction and AdamW state."""

    def __init__(self, policy, device, weight_decay, seed):
        import torch
        import paper_1710_06952_amd as P
        self.policy = policy
        self.weights = torch.zeros(policy.d, dtype=torch.bfloat16, device=device)
        self.grads = torch.zeros(policy.d, dtype=torch.bfloat16, device=device)
        self.direction = torch.zeros(policy.d, dtype=torch.float32, device=device)
        decay = [weight_decay if len(s) == 2 else 0.0 for s in policy.shapes]
        self.optimizer = P.AdamW(policy.views(self.weights), policy.views(self.grads), out=policy.views(self.direction), weight_decay=decay, state_bits=8,
                                 seed=seed)

    def step_direction(self, logits, weights, dlogits, out):
        import torch
        for g, to in zip(torch.autograd.grad(logits, weights, dlogits), self.policy.views(self.grads)):
            to.copy_(g)
        self.optimizer.step(max_norm=1.0)
        out.copy_(self.direction)


def run_study(loss="policy", n=4, vocab=512, width=128, prompts_each=64, M=128, events=400, T_max=2, gamma=2e-3, weight_decay=0.01, kl=0.01, seed=0,
              device="cuda:0"):
    import torch
    import paper_1710_06952_amd as P
    prompts = n * prompts_each
    policy = Policy(vocab, width, prompts, seed, device)
    right = torch.from_numpy(np.random.default_rng(seed + 2).integers(0, vocab, prompts)).to(device)
    eng = P.Engine(ring(n), policy.d, "external", gamma=gamma, T_max=T_max, device=device)
    x0 = policy.initial(seed)
    eng.set_models(x0)
    frozen = policy.views(torch.from_numpy(x0).to(device).bfloat16())
    workers = [Worker(policy, device, weight_decay, seed + 10 + i) for i in range(n)]
    offsets = torch.arange(2 * M + 1, device=device)      # answers of one token
    losses = torch.zeros(events, device=device)

    def gradient(worker, event, xhat, out):
        w = workers[worker]
        gen = torch.Generator(device=device)
        gen.manual_seed(seed * 1_000_003 + event)
        w.weights.copy_(xhat)
        weights = [v.detach().requires_grad_() for v in policy.views(w.weights)]
        asked = worker * prompts_each + torch.randint(0, prompts_each, (M,), device=device, generator=gen)
        if loss == "policy":
            logits = policy.logits(weights, asked)
            answers = torch.multinomial(torch.softmax(logits.detach().float(), 1), 1, generator=gen)[:, 0]
            reward = (answers == right[asked]).float()
            old, ref = P.token_log_probs(logits, answers), P.token_log_probs(policy.logits(frozen, asked), answers)
            r = P.policy_loss_and_gradient(logits, answers, old, reward - reward.mean(), ref, clip=(0.2, 0.2), kl_coef=kl)
        else:
            twice = torch.cat([asked, asked])
            logits = policy.logits(weights, twice)
            wrong = (right[asked] + torch.randint(1, vocab, (M,), device=device, generator=gen)) % vocab
            answers = torch.cat([right[asked], wrong])
            ref = P.token_log_probs(policy.logits(frozen, twice), answers)
            r = P.preference_loss_and_gradient(logits, answers, offsets, ref, beta=0.5)
        losses[event] = r.loss
        w.step_direction(logits, weights, r.dlogits, out)

    def chance():
        """Mean probability of the right answers under the mean model."""
        mean = torch.from_numpy(eng.get_mean_model()).to(device).bfloat16()
        with torch.no_grad():
            return float(P.token_log_probs(policy.logits(policy.views(mean), torch.arange(prompts, device=device)), right).exp().mean())

    curve = [chance()]
    sched = P.adpsgd_make_schedule(ring(n), events, seed=seed, T_max=T_max)
    eng.run_events_in_pieces(sched, max(1, events // 4), gradient_fn=gradient, between=lambda _events: curve.append(chance()))
    per = max(1, events // 4)
    res = {"loss": loss, "n": n, "d": policy.d, "vocab": vocab, "events": eng.get_stats()["events"], "gamma": gamma, "chance": curve,
           "losses": [float(losses[a:a + per].mean()) for a in range(0, events, per)], "consensus_distance": eng.consensus_distance(),
           "steps": [w.optimizer.steps for w in workers]}
    eng.close()
    return res


def format_table(res):
    lines = ["quarter | mean loss | right answer's probability", "-" * 48, "      0 |           | %.4f" % res["chance"][0]]
    for q, (l, c) in enumerate(zip(res["losses"], res["chance"][1:])):
        lines.append("%7d | %9.5f | %.4f" % (q + 1, l, c))
    lines.append("%d events; consensus distance %.3g" % (res["events"], res["consensus_distance"]))
    return "\n".join(lines)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--loss", choices=("policy", "preference"), default="policy")
    ap.add_argument("--n", type=int, default=4)
    ap.add_argument("--events", type=int, default=400)
    ap.add_argument("--gamma", type=float, default=2e-3)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--json", action="store_true")
    a = ap.parse_args(argv)
    res = run_study(a.loss, a.n, events=a.events, gamma=a.gamma, seed=a.seed)
    print(json.dumps(res) if a.json else format_table(res))


if __name__ == "__main__":
    main()
