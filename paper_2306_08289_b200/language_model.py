"""Decentralised training of a small language model with the engine: a population of asynchronous workers whose rows are
the parameters of

    y_t = E[id_t] sqrt(width),   h_t = y_t + tanh(M y_t),   loss_t = cross entropy of (W h_t) against the next token,

each with its own gradient events on its own text (a seeded Markov chain: the next token is one of a few followers of the last one).
At a gradient event the worker's gradient is evaluated at its stored row (Algorithm 1 of the paper, first loop) and written straight
into its gradient row: E and W through the operators' gradients, M through torch, and M's part is replaced by its orthogonalisation, for
all workers of a batch in one call. The event kernel then applies the mixing and the step.

    python -m paper_2306_08289_b200.language_model [--n 16] [--vocab 512] [--width 128] [--T 60] [--storage f32]

prints, at ten common times, the loss of the workers' mean model on held-out text, the source's entropy (the lowest loss there is) and the
consensus distance.
"""
from __future__ import annotations

import argparse
import math

import numpy as np

from . import binding as B
from . import workload as W
from .consensus_study import closed_loop_batches


class MarkovText:
    """Text whose next token is one of `followers` tokens of the last one, with fixed probabilities."""

    def __init__(self, vocab, followers, seed):
        rng = np.random.Generator(np.random.PCG64(np.random.SeedSequence([seed, 21])))
        self.vocab = vocab
        self.next = np.stack([rng.choice(vocab, followers, replace=False) for _ in range(vocab)])
        p = 1.0 / (1.0 + np.arange(followers))
        self.p = p / p.sum()
        self.entropy = float(-(self.p * np.log(self.p)).sum())

    def draw(self, rng, sequences, length):
        """(ids, targets), int32 [sequences * length]; a sequence's last token has no target (-1)."""
        ids = np.empty((sequences, length), dtype=np.int32)
        ids[:, 0] = rng.integers(0, self.vocab, sequences)
        pick = rng.choice(len(self.p), size=(sequences, length), p=self.p)
        for k in range(1, length):
            ids[:, k] = self.next[ids[:, k - 1], pick[:, k]]
        targets = np.full_like(ids, -1)
        targets[:, :-1] = ids[:, 1:]
        return ids.reshape(-1), targets.reshape(-1)


class Model:
    """Where the three matrices lie inside a row, and the gradient of one batch of tokens."""

    def __init__(self, vocab, width):
        self.vocab, self.width = vocab, width
        self.at = {"E": 0, "M": vocab * width, "W": vocab * width + width * width}
        self.d = 2 * vocab * width + width * width
        self.shape = {"E": (vocab, width), "M": (width, width), "W": (vocab, width)}

    def part(self, rows, name):
        """The matrices `name` of a row [d] or of all rows [n, pitch], as a view."""
        r, c = self.shape[name]
        lo = self.at[name]
        return rows[..., lo:lo + r * c].view(*rows.shape[:-1], r, c)

    def initial_row(self, seed):
        rng = np.random.Generator(np.random.PCG64(np.random.SeedSequence([seed, 22])))
        row = rng.standard_normal(self.d).astype(np.float32) / math.sqrt(self.width)
        return row

    def forward(self, row, ids):
        import torch

        from . import operators as ops

        y = ops.embed(self.part(row, "E"), ids, scale=math.sqrt(self.width))
        a = torch.tanh(y @ self.part(row, "M").T)
        return y, a, y + a

    def loss(self, row, ids, targets):
        """Mean loss over the tokens that have a target."""
        from . import operators as ops

        loss, _ = ops.vocab_loss(self.forward(row, ids)[2], self.part(row, "W"), targets)
        return loss.sum() / (targets >= 0).sum()

    def gradient(self, row, ids, targets, scale, out):
        """The gradient of scale * sum of the losses, written into the row `out`."""
        from . import operators as ops

        y, a, h = self.forward(row, ids)
        _, _, dh, _ = ops.vocab_loss_grad(h, self.part(row, "W"), targets, scale=scale, grad_head=self.part(out, "W"))
        da = dh * (1.0 - a * a)
        self.part(out, "M").copy_(da.T @ y)
        dy = dh + da @ self.part(row, "M")
        ops.embed_grad(dy, ids, self.vocab, scale=math.sqrt(self.width), out=self.part(out, "E"))


def train(n=16, vocab=512, width=128, T=60.0, gamma=0.1, storage="f32", sequences=16, length=32, loss_scale=30.0, update=0.2, seed=3, samples=10,
          device="cuda:0"):
    """Returns the trace [(time, loss of the mean model, consensus distance per worker)] and the text's entropy. loss_scale multiplies the
    mean loss whose gradient E and W follow; `update` scales M's orthogonalised step."""
    import torch

    from . import operators as ops

    text, model = MarkovText(vocab, 4, seed), Model(vocab, width)
    edges = W.make_edges("ring", n)
    rates = W.edge_rates_per_worker(n, edges, 1.0)
    eta, alpha, alpha_t = B.prescribe(*B.graph_chi(n, edges, rates), True)
    n_events = int((n + rates.sum()) * T)
    ev = W.poisson_events(n, edges, rates, n_events, seed=seed)
    eng = B.Engine(n, model.d, eta, alpha, alpha_t, gamma, storage=storage, n_grad_slots=n, device=device)
    row = model.initial_row(seed)
    stored = W.f32_to_bf16_bits(row) if storage == "bf16" else row
    for w in range(n):  # consensus at the start, as in the paper
        eng.fill_row("x", w, stored)
        eng.fill_row("xt", w, stored)
    rng = np.random.Generator(np.random.PCG64(np.random.SeedSequence([seed, 23])))

    def tokens(count):
        return (torch.from_numpy(v).to(device) for v in text.draw(rng, count, length))

    held_ids, held_targets = tokens(64)
    x, g = eng.x[:, : model.d], eng.g[:, : model.d]
    trace = []

    def sample(t):
        mean = x.float().mean(0).to(eng.x.dtype)
        trace.append((t, float(model.loss(mean, held_ids, held_targets)), eng.consensus_distance() / n))

    sample(0.0)
    step = max(1, n_events // samples)
    for k in range(0, n_events, step):
        c = ev.slice(k, k + step)
        plan = eng.plan(c.times, c.wi, c.wj, c.slot, flags=0)
        for b, (_, workers, slots) in enumerate(closed_loop_batches(plan.sched, c)):
            for w, slot in zip(workers, slots):
                ids, targets = tokens(sequences)
                model.gradient(x[w], ids, targets, loss_scale / (sequences * (length - 1)), g[slot])
            if len(workers):
                at = torch.from_numpy(slots).to(device)
                m = model.part(g, "M")
                m[at] = ops.orthogonalize(m[at], scale=update)
            plan.run(b, 1)
        plan.close()
        t = float(c.times[-1])
        eng.flush(t)
        sample(t)
    eng.close()
    return trace, text.entropy


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--n", type=int, default=16)
    ap.add_argument("--vocab", type=int, default=512)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--T", type=float, default=60.0)
    ap.add_argument("--gamma", type=float, default=0.1)
    ap.add_argument("--storage", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    trace, entropy = train(a.n, a.vocab, a.width, a.T, a.gamma, a.storage)
    for t, loss, distance in trace:
        print(f"t={t:7.2f}  loss of the mean model {loss:.4f} (entropy {entropy:.4f})  consensus distance / n {distance:.3e}")


if __name__ == "__main__":
    main()
