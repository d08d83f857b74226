"""Decentralised training of a small language model with the engine: a population of asynchronous workers whose rows are
the parameters of

    y_t = E[id_t] sqrt(width),   h_t = y_t + tanh(M y_t),   loss_t = cross entropy of (W h_t) against the next token,

or, with norms and with experts (`--norm`, `--experts`),

    u_t = norm(y_t) N,   a_t = tanh(M u_t)  or  sum over the chosen experts e of w_te tanh(M_e u_t), w_t from the logits R u_t,
    h_t = norm(y_t + a_t) F,

each with its own gradient events on its own text (a seeded Markov chain: the next token is one of a few followers of the last one).
At a gradient event the worker's gradient is evaluated at its stored row (Algorithm 1 of the paper, first loop) and written straight
into its gradient row: E, W, the norms' weights and the experts' choice through the operators' gradients, M through torch, and M's part is replaced by its
orthogonalisation, for all workers of a batch in one call. With `--clip` every worker's gradient is clipped to a norm of its own, and one that is not finite is left out, before the event
brings it to the others. The event kernel then applies the mixing and the step.

    python -m paper_2306_08289_b200.language_model [--n 16] [--vocab 512] [--width 128] [--T 60] [--storage f32] [--norm] [--experts 8] [--clip 1.0]

prints, at ten common times, the loss of the workers' mean model on held-out text (with norms also with the last hidden states in 8 bits), the source's entropy
(the lowest loss there is) and the consensus distance.
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
    """Where the matrices lie inside a row, and the gradient of one batch of tokens. norm: with the norms' weights N and F; experts: as many matrices M and a
    router R that chooses `chosen` of them for a token."""

    def __init__(self, vocab, width, norm=False, experts=0, chosen=2):
        self.vocab, self.width, self.norm, self.experts, self.chosen = vocab, width, norm, experts, min(chosen, max(experts, 1))
        self.shape = {"E": (vocab, width), "M": (max(experts, 1) * width, width), "W": (vocab, width)}
        if experts:
            self.shape["R"] = (experts, width)
        if norm:
            self.shape.update(N=(1, width), F=(1, width))
        self.at, self.d = {}, 0
        for name, (r, c) in self.shape.items():
            self.at[name] = self.d
            self.d += r * c

    def part(self, rows, name):
        """The matrices `name` of a row [d] or of all rows [n, pitch], as a view."""
        r, c = self.shape[name]
        lo = self.at[name]
        return rows[..., lo:lo + r * c].view(*rows.shape[:-1], r, c)

    def hidden(self, rows):
        """The matrices M of a row, [experts, width, width], or of all rows, [n, experts, width, width], as a view."""
        return self.part(rows, "M").unflatten(-2, (-1, self.width))

    def initial_row(self, seed):
        rng = np.random.Generator(np.random.PCG64(np.random.SeedSequence([seed, 22])))
        row = rng.standard_normal(self.d).astype(np.float32) / math.sqrt(self.width)
        for name in ("N", "F"):
            if name in self.at:
                row[self.at[name]:self.at[name] + self.width] = 1.0
        return row

    def _mix(self, row, u):
        """(a, what the gradient needs of it): the hidden layer on u."""
        import torch

        from . import operators as ops

        if not self.experts:
            a = torch.tanh(u @ self.part(row, "M").T)
            return a, (a,)
        logits = u @ self.part(row, "R").T
        ids, weights, _ = ops.route(logits, self.chosen)
        each = torch.tanh(torch.einsum("ti,eoi->teo", u, self.hidden(row)))  # of all experts: they are few and small here
        picked = each.gather(1, ids.long().clamp(min=0)[:, :, None].expand(-1, -1, self.width))
        a = (weights[:, :, None] * picked.float()).sum(1).to(u.dtype)
        return a, (logits, ids, weights, each, picked)

    def forward(self, row, ids):
        """(y, a, h); of a model with norms or experts (y, u, a, what the gradient needs of the hidden layer, s or None, h)."""
        y, u, a, kept, s, h = self._layers(row, ids)
        return (y, u, a, kept, s, h) if self.norm or self.experts else (y, a, h)

    def _layers(self, row, ids):
        from . import operators as ops

        y = ops.embed(self.part(row, "E"), ids, scale=math.sqrt(self.width))
        u = ops.rms_norm(y, self.part(row, "N")[0]) if self.norm else y
        a, kept = self._mix(row, u)
        if not self.norm:
            return y, u, a, kept, None, y + a
        h, s = ops.rms_norm(a, self.part(row, "F")[0], residual=y)
        return y, u, a, kept, s, h

    def loss(self, row, ids, targets, quantized=False):
        """Mean loss over the tokens that have a target; quantized: with the last hidden states held in 8 bits."""
        from . import operators as ops

        *_, s, h = self._layers(row, ids)
        if quantized:
            h = ops.dequantize(*ops.rms_norm_quantized(s, self.part(row, "F")[0], block=32 if self.width > 32 else 0), h.dtype)
        loss, _ = ops.vocab_loss(h, self.part(row, "W"), targets)
        return loss.sum() / (targets >= 0).sum()

    def gradient(self, row, ids, targets, scale, out):
        """The gradient of scale * sum of the losses, written into the row `out`."""
        import torch

        from . import operators as ops

        y, u, a, kept, s, h = self._layers(row, ids)
        _, _, dh, _ = ops.vocab_loss_grad(h, self.part(row, "W"), targets, scale=scale, grad_head=self.part(out, "W"))
        if self.norm:  # dh of the sum from here on
            dh, _ = ops.rms_norm_grad(dh, s, self.part(row, "F")[0], grad_weight=self.part(out, "F")[0])
        if not self.experts:
            da = dh * (1.0 - a * a)
            self.part(out, "M").copy_(da.T @ u)
            du = da @ self.part(row, "M")
        else:
            logits, chosen, weights, each, picked = kept
            dweights = (picked * dh[:, None]).float().sum(2)
            dlogits = ops.route_grad(logits, chosen, dweights)
            self.part(out, "R").copy_(dlogits.T @ u)
            share = torch.zeros(logits.shape, device=row.device).scatter_add_(1, chosen.long().clamp(min=0), weights).to(u.dtype)
            dz = share[:, :, None] * dh[:, None] * (1.0 - each * each)
            self.hidden(out).copy_(torch.einsum("teo,ti->eoi", dz, u))
            du = torch.einsum("teo,eoi->ti", dz, self.hidden(row)) + dlogits @ self.part(row, "R")
        if self.norm:
            dy, _ = ops.rms_norm_grad(du, y, self.part(row, "N")[0], grad_sum=dh, grad_weight=self.part(out, "N")[0])
        else:
            dy = dh + du
        ops.embed_grad(dy, ids, self.vocab, scale=math.sqrt(self.width), out=self.part(out, "E"))


def train(n=16, vocab=512, width=128, T=60.0, gamma=0.1, storage="f32", sequences=16, length=32, loss_scale=30.0, update=0.2, seed=3, samples=10,
          device="cuda:0", norm=False, experts=0, clip=None):
    """Returns the trace [(time, loss of the mean model, consensus distance per worker)], with norms with the loss in 8 bits behind, and the text's entropy. loss_scale
    multiplies the mean loss whose gradient E and W follow; `update` scales M's orthogonalised step; `clip` is the largest norm of a worker's gradient."""
    import torch

    from . import operators as ops

    text, model = MarkovText(vocab, 4, seed), Model(vocab, width, norm, experts)
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
    fresh = torch.zeros(n, model.d, dtype=eng.x.dtype, device=device)  # gradients of a batch before they are clipped
    trace = []

    def sample(t):
        mean = x.float().mean(0).to(eng.x.dtype)
        bits = (float(model.loss(mean, held_ids, held_targets, quantized=True)),) if norm else ()
        trace.append((t, float(model.loss(mean, held_ids, held_targets)), eng.consensus_distance() / n, *bits))

    sample(0.0)
    step = max(1, n_events // samples)
    for k in range(0, n_events, step):
        c = ev.slice(k, k + step)
        plan = eng.plan(c.times, c.wi, c.wj, c.slot, flags=0)
        for b, (_, workers, slots) in enumerate(closed_loop_batches(plan.sched, c)):
            for k_th, (w, slot) in enumerate(zip(workers, slots)):
                ids, targets = tokens(sequences)
                model.gradient(x[w], ids, targets, loss_scale / (sequences * (length - 1)), g[slot] if clip is None else fresh[k_th])
            if len(workers):
                at = torch.from_numpy(slots).to(device)
                if clip is None and not experts:
                    m = model.part(g, "M")
                    m[at] = ops.orthogonalize(m[at], scale=update)
                else:
                    rows = g[at] if clip is None else fresh[:len(workers)]
                    m = model.hidden(rows)
                    m.copy_(ops.orthogonalize(m.reshape(-1, width, width), scale=update).view(m.shape))
                    if clip is not None:
                        ops.clip_gradients([rows], clip, per_worker=True, zero_nonfinite=True)
                    g[at] = rows
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
    ap.add_argument("--norm", action="store_true", help="with root-mean-square norms")
    ap.add_argument("--experts", type=int, default=0, help="matrices of the hidden layer of which a router chooses two for each token")
    ap.add_argument("--clip", type=float, default=None, help="largest norm of a worker's gradient")
    a = ap.parse_args()
    trace, entropy = train(a.n, a.vocab, a.width, a.T, a.gamma, a.storage, norm=a.norm, experts=a.experts, clip=a.clip)
    for t, loss, distance, *bits in trace:
        in_bits = f", in 8 bits {bits[0]:.4f}" if bits else ""
        print(f"t={t:7.2f}  loss of the mean model {loss:.4f}{in_bits} (entropy {entropy:.4f})  consensus distance / n {distance:.3e}")


if __name__ == "__main__":
    main()
