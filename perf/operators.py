"""Measurement cases for the language-model operators of the package: embedding lookup and its gradient by sorted
tokens, the vocabulary loss (softmax cross entropy over a large vocabulary, with its gradients) and the
orthogonalisation of matrix updates by Newton-Schulz products.

`run` computes an operator in its plain form (elementary torch operations in 32 bits) or, with `own` set, through the
package's public entry points. `exact` gives the same outputs from the definitions in 64 bits."""
import math

import torch

own = False

DEV = "cuda"
COEFFS = (3.4445, -4.7750, 2.0315)  # the quintic of the orthogonalisation, five steps of it
STEPS = 5
EPS = 1e-7


# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one sequence's tokens through a small worker's table: launch latency
        {"name": "embed bf16 short", "op": "embed", "type": "bf16", "tokens": 48, "vocab": 1000, "width": 128},
        # a large micro-batch over a large odd vocabulary: bandwidth
        {"name": "embed f32 large", "op": "embed", "type": "f32", "tokens": 65536, "vocab": 50003, "width": 1024},
        # gradient of an ordinary micro-batch: most table rows get no token and are zeros
        {"name": "embed grad bf16", "op": "embed_grad", "type": "bf16", "tokens": 4096, "vocab": 32000, "width": 512},
        # gradient of a large micro-batch, frequent tokens in thousands of places
        {"name": "embed grad f32 large", "op": "embed_grad", "type": "f32", "tokens": 32768, "vocab": 50003, "width": 1024},
        # loss of a few tokens over a byte vocabulary: launch latency
        {"name": "loss f32 bytes", "op": "loss", "type": "f32", "tokens": 32, "vocab": 257, "width": 64, "grad": False},
        # evaluation of a batch, forward only, odd vocabulary
        {"name": "loss bf16 evaluation", "op": "loss", "type": "bf16", "tokens": 4096, "vocab": 50003, "width": 1024, "grad": False},
        # a gradient event of a small worker, everything odd
        {"name": "loss grad f32 odd", "op": "loss", "type": "f32", "tokens": 333, "vocab": 5003, "width": 201, "grad": True},
        # a gradient event with 32-bit rows over a large vocabulary
        {"name": "loss grad f32", "op": "loss", "type": "f32", "tokens": 2048, "vocab": 32000, "width": 512, "grad": True},
        # the largest gradient event: bf16 rows, long micro-batch, wide model
        {"name": "loss grad bf16 large", "op": "loss", "type": "bf16", "tokens": 8192, "vocab": 65536, "width": 2048, "grad": True},
        # small matrices of a batch of workers: latency
        {"name": "orthogonalize f32 small", "op": "orthogonalize", "type": "f32", "mats": 16, "rows": 64, "cols": 64},
        # one hidden matrix of 16 workers, tall and odd, 32-bit rows
        {"name": "orthogonalize f32", "op": "orthogonalize", "type": "f32", "mats": 16, "rows": 1001, "cols": 512},
        # large hidden matrices, bf16 rows
        {"name": "orthogonalize bf16 large", "op": "orthogonalize", "type": "bf16", "mats": 4, "rows": 2048, "cols": 4096},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "loss", "loss", "loss", "orthogonalize", "orthogonalize"])
    case = {"op": op, "type": rng.choice(["f32", "bf16"])}
    if op in ("embed", "embed_grad"):
        case.update(tokens=_log_int(rng, 1, 65536), vocab=_log_int(rng, 16, 65536), width=_log_int(rng, 8, 2048))
        if op == "embed_grad" and case["tokens"] * case["width"] > 2**25:
            case["tokens"] = 2**25 // case["width"]
        elif case["tokens"] * case["width"] > 2**26:
            case["tokens"] = 2**26 // case["width"]
    elif op == "loss":
        case.update(tokens=_log_int(rng, 1, 8192), vocab=_log_int(rng, 64, 65536), width=_log_int(rng, 16, 2048),
                    grad=rng.random() < 0.7)
    else:
        case.update(mats=_log_int(rng, 1, 64), rows=_log_int(rng, 8, 4096), cols=_log_int(rng, 8, 4096))
        most = _orthogonalize_flops(4, 2048, 4096)
        one = _orthogonalize_flops(1, case["rows"], case["cols"])
        if one > most:
            case["rows"] //= 4
            one = _orthogonalize_flops(1, case["rows"], case["cols"])
        case["mats"] = max(1, min(case["mats"], int(most // one)))
    return case


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["type"] == "bf16" else torch.float32


def _zipf_ids(n, vocab, gen):
    """Token ids with the frequencies of text: the k-th most frequent id about 1 / (k + 2.7) as often, in shuffled order."""
    freq = 1.0 / (torch.arange(vocab, device=DEV, dtype=torch.float64) + 2.7)
    edges = torch.cumsum(freq, 0)
    u = torch.rand(n, device=DEV, dtype=torch.float64, generator=gen) * edges[-1]
    rank = torch.searchsorted(edges, u).clamp_(max=vocab - 1)
    return torch.randperm(vocab, device=DEV, generator=gen)[rank].to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = _dtype(case)
    op = case["op"]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, device=DEV, generator=gen) * std).to(dt)

    if op in ("embed", "embed_grad"):
        t, v, h = case["tokens"], case["vocab"], case["width"]
        ids = _zipf_ids(t, v, gen)
        pad = torch.rand(t, device=DEV, generator=gen) < 0.03  # padding between sequences
        ids = torch.where(pad, torch.full_like(ids, -1), ids)
        state = {"op": op, "ids": ids, "scale": math.sqrt(h), "vocab": v}
        if op == "embed":
            state["table"] = normal(v, h, std=0.02)
        else:
            state["grad_out"] = normal(t, h, std=1e-3)
        return state
    if op == "loss":
        t, v, h = case["tokens"], case["vocab"], case["width"]
        head = normal(v, h, std=1.0 / math.sqrt(h))
        targets = _zipf_ids(t, v, gen)
        # a model in training: the hidden state leans towards its target's row, more for some tokens than for others
        lean = torch.rand(t, 1, device=DEV, generator=gen) * 8.0
        hidden = (torch.randn(t, h, device=DEV, generator=gen) + lean * head[targets.long()].float()).to(dt)
        masked = torch.rand(t, device=DEV, generator=gen) < 0.1  # prompts and padding carry no loss
        targets = torch.where(masked, torch.full_like(targets, -1), targets)
        return {"op": op, "hidden": hidden, "head": head, "targets": targets, "grad": case["grad"], "scale": 1.0 / t}
    b, m, n = case["mats"], case["rows"], case["cols"]
    # momentum of a few correlated gradients over noise, of a different size in each worker
    r = max(1, min(m, n) // 8)
    common = torch.bmm(torch.randn(b, m, r, device=DEV, generator=gen), torch.randn(b, r, n, device=DEV, generator=gen))
    size = torch.exp(torch.randn(b, 1, 1, device=DEV, generator=gen)) * 1e-3
    mats = (common / math.sqrt(r) + torch.randn(b, m, n, device=DEV, generator=gen)) * size
    return {"op": op, "mats": mats.to(dt), "scale": math.sqrt(max(1.0, m / n))}


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    op = state["op"]
    if op == "embed":
        ids, table = state["ids"].long(), state["table"]
        rows = table[ids.clamp(min=0)].float() * state["scale"]
        return (rows * (ids >= 0)[:, None]).to(table.dtype)
    if op == "embed_grad":
        ids, g = state["ids"].long(), state["grad_out"]
        rows = g.float() * (ids >= 0)[:, None]
        out = torch.zeros(state["vocab"], g.shape[1], device=g.device, dtype=torch.float32)
        out.index_add_(0, ids.clamp(min=0), rows)
        return (out * state["scale"]).to(g.dtype)
    if op == "loss":
        hidden, head = state["hidden"].float(), state["head"].float()
        targets = state["targets"].long()
        live = targets >= 0
        at = targets.clamp(min=0)[:, None]
        logits = hidden @ head.T
        top = logits.amax(dim=1, keepdim=True)
        e = torch.exp(logits - top)
        total = e.sum(dim=1, keepdim=True)
        lse = (top + torch.log(total))[:, 0]
        loss = torch.where(live, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
        if not state["grad"]:
            return {"loss": loss, "lse": lse}
        p = e.div_(total)
        p.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
        p.mul_((live * state["scale"])[:, None])
        dt = state["hidden"].dtype
        return {"loss": loss, "lse": lse, "grad_hidden": (p @ head).to(dt), "grad_head": (p.T @ hidden).to(dt)}
    g = state["mats"].float()
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2) if tall else g
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS)
    a, b, c = COEFFS
    for _ in range(STEPS):
        s = x @ x.transpose(1, 2)
        x = a * x + (b * s + c * (s @ s)) @ x
    x = x * state["scale"]
    return (x.transpose(1, 2) if tall else x).to(state["mats"].dtype).contiguous()


def _run_own(state):
    from paper_2306_08289_b200 import operators as ops

    op = state["op"]
    if op == "embed":
        return ops.embed(state["table"], state["ids"], scale=state["scale"])
    if op == "embed_grad":
        return ops.embed_grad(state["grad_out"], state["ids"], state["vocab"], scale=state["scale"])
    if op == "loss":
        if not state["grad"]:
            loss, lse = ops.vocab_loss(state["hidden"], state["head"], state["targets"])
            return {"loss": loss, "lse": lse}
        loss, lse, gh, gw = ops.vocab_loss_grad(state["hidden"], state["head"], state["targets"], scale=state["scale"])
        return {"loss": loss, "lse": lse, "grad_hidden": gh, "grad_head": gw}
    return ops.orthogonalize(state["mats"], steps=STEPS, coeffs=COEFFS, eps=EPS, scale=state["scale"])


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def _orthogonalize_flops(mats, rows, cols):
    m, n = min(rows, cols), max(rows, cols)
    # per step: X X^T and A^2 are symmetric (half of each is enough), B X is not
    return float(STEPS * mats) * (m * m * n + m * m * m + 2 * m * m * n)


def work(case):
    size = 2 if case["type"] == "bf16" else 4
    op = case["op"]
    if op == "embed":
        t, v, h = case["tokens"], case["vocab"], case["width"]
        return {"bytes": (min(t, v) + t) * h * size + 4 * t, "flops": t * h}
    if op == "embed_grad":
        t, v, h = case["tokens"], case["vocab"], case["width"]
        return {"bytes": (t + v) * h * size + 4 * t, "flops": t * h}
    if op == "loss":
        t, v, h = case["tokens"], case["vocab"], case["width"]
        passes = 2 if case["grad"] else 1
        # logits once, and for the gradients two more products; inputs read once, gradients written once
        return {"bytes": passes * (t + v) * h * size + 12 * t, "flops": (6.0 if case["grad"] else 2.0) * t * v * h}
    b, m, n = case["mats"], case["rows"], case["cols"]
    return {"bytes": 2 * b * m * n * size, "flops": _orthogonalize_flops(b, m, n)}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        out = torch.zeros(case["tokens"], case["width"], device=DEV, dtype=torch.float64)
        at = torch.nonzero(state["ids"] >= 0)[:, 0]
        out[at] = torch.index_select(state["table"], 0, state["ids"][at]).double() * state["scale"]
        return out
    if op == "embed_grad":
        ids, g = state["ids"].long(), state["grad_out"]
        order = torch.argsort(ids, stable=True)
        order = order[ids[order] >= 0]
        out = torch.zeros(case["vocab"], case["width"], device=DEV, dtype=torch.float64)
        out.index_add_(0, ids[order], g[order].double() * state["scale"])
        return out
    if op == "loss":
        head, t = state["head"].double(), case["tokens"]
        loss = torch.zeros(t, device=DEV, dtype=torch.float64)
        lse = torch.zeros_like(loss)
        gh = torch.zeros(t, case["width"], device=DEV, dtype=torch.float64)
        gw = torch.zeros_like(head)
        for lo in range(0, t, 512):
            h = state["hidden"][lo:lo + 512].double()
            y = state["targets"][lo:lo + 512].long()
            z = h @ head.T
            lse[lo:lo + 512] = torch.logsumexp(z, dim=1)
            rows = torch.nonzero(y >= 0)[:, 0]
            loss[lo + rows] = lse[lo + rows] - z[rows, y[rows]]
            if case["grad"]:
                p = torch.softmax(z[rows], dim=1)
                p[torch.arange(len(rows), device=DEV), y[rows]] -= 1.0
                p *= state["scale"]
                gh[lo + rows] = p @ head
                gw += p.T @ h[rows]
        out = {"loss": loss, "lse": lse}
        if case["grad"]:
            out.update(grad_hidden=gh, grad_head=gw)
        return out
    # all five steps multiply G by polynomials of its Gram matrix, so the small side alone is iterated
    g = state["mats"].double()
    tall = g.shape[1] > g.shape[2]
    gram = g.transpose(1, 2) @ g if tall else g @ g.transpose(1, 2)
    norm = torch.sqrt(torch.diagonal(gram, dim1=1, dim2=2).sum(1))[:, None, None] + EPS
    s = gram / norm**2
    eye = torch.eye(s.shape[1], device=DEV, dtype=torch.float64)
    total = eye / norm
    a, b, c = COEFFS
    for _ in range(STEPS):
        step = a * eye + b * s + c * (s @ s)
        total = step @ total
        s = step @ s @ step
    out = g @ total if tall else total @ g
    return out * state["scale"]
