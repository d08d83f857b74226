"""Measurement cases for further operators of a language model's gradient event: the root-mean-square norm with the
residual's addition, its output in 8 bits with scales, and its gradient; the routing of tokens to experts and its gradient; the norm of
a gradient over many tensors and its clipping.

`run` computes an operator in its plain form (elementary torch operations in 32 bits; routing's choices in 64) or, with `own` set, through
the package's public entry points. `exact` gives the same outputs from the definitions in 64 bits."""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
E4M3_MAX = 448.0
SCALE_MIN = 2.0**-126  # of a block of zeros
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of a generation step through a wide model: launch latency
        {"name": "norm bf16 one token", "op": "norm", "type": "bf16", "tokens": 1, "width": 2048, "residual": True, "weight": True},
        # a large micro-batch of 32-bit rows, residual stream in and out: bandwidth
        {"name": "norm f32 large", "op": "norm", "type": "f32", "tokens": 16384, "width": 4096, "residual": True, "weight": True},
        # activations for 8-bit products, a scale for every 128 columns
        {"name": "norm e4m3 blocks", "op": "norm8", "type": "bf16", "tokens": 8192, "width": 2048, "residual": True, "weight": True, "block": 128},
        # gradient of an odd small model, 32-bit rows
        {"name": "norm grad f32 odd", "op": "norm_grad", "type": "f32", "tokens": 1001, "width": 201, "residual": False, "weight": True},
        # gradient of an ordinary micro-batch, with the gradient that arrives through the residual stream
        {"name": "norm grad bf16", "op": "norm_grad", "type": "bf16", "tokens": 16384, "width": 2048, "residual": True, "weight": True},
        # a few tokens over few experts: launch latency
        {"name": "route bf16 few", "op": "route", "type": "bf16", "tokens": 16, "experts": 64, "k": 2, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "renormalize": True},
        # a large micro-batch over many experts in groups, balanced by a bias
        {"name": "route f32 groups", "op": "route", "type": "f32", "tokens": 32768, "experts": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "renormalize": True},
        # gradient where every expert's logit has one, odd sizes
        {"name": "route grad f32 dense", "op": "route_grad", "type": "f32", "tokens": 30011, "experts": 161, "k": 6, "score": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "renormalize": False},
        # gradient of renormalised weights: the chosen experts' logits alone have one
        {"name": "route grad bf16", "op": "route_grad", "type": "bf16", "tokens": 8192, "experts": 128, "k": 8, "score": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "renormalize": True},
        # one worker's small model: a list of tensors of both types, copied to the rows that the event reads
        {"name": "clip small", "op": "clip", "workers": 1, "tensors": 12, "elements": 200003, "mixed": True, "clipped": True},
        # all workers of a batch, each with a norm of its own, matrices inside the workers' rows
        {"name": "clip workers", "op": "clip", "workers": 16, "tensors": 3, "elements": 1117184, "mixed": False, "clipped": True},
        # one large gradient
        {"name": "clip large", "op": "clip", "workers": 1, "tensors": 40, "elements": 134217728, "mixed": True, "clipped": True},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm8", "norm_grad", "norm_grad", "route", "route", "route_grad", "route_grad", "clip", "clip"])
    case = {"op": op}
    if op in ("norm", "norm8", "norm_grad"):
        width = _log_int(rng, 8, 16384)
        if rng.random() < 0.5:
            width = max(8, width // 8 * 8)
        most = 2**26 if op == "norm" else 2**25
        case.update(type=rng.choice(["f32", "bf16"]), tokens=min(_log_int(rng, 1, 65536), most // width), width=width, residual=rng.random() < 0.6,
                    weight=rng.random() < 0.9)
        if op == "norm8":
            case["block"] = rng.choice([0, 32, 64, 128])
    elif op in ("route", "route_grad"):
        groups = rng.choice([1, 1, 1, 2, 4, 8])
        experts = max(groups * 4, _log_int(rng, 8, 512) // groups * groups)
        top_groups = rng.randint(1, groups)
        k = min(_log_int(rng, 1, 16), experts // groups * top_groups)
        case.update(type=rng.choice(["f32", "bf16"]), tokens=min(_log_int(rng, 1, 65536), 2**23 // experts), experts=experts, k=k,
                    score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups, top_groups=top_groups,
                    renormalize=k > 1 and rng.random() < 0.6)
    else:
        workers = rng.choice([1, 1, _log_int(rng, 2, 64)])
        elements = _log_int(rng, 100, 2**27 // workers)
        case.update(workers=workers, tensors=min(_log_int(rng, 1, 60), elements), elements=elements, mixed=workers == 1 and rng.random() < 0.5,
                    clipped=rng.random() < 0.8)
    return case


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _parts(tensors, elements):
    """Sizes of a model's tensors: a few large matrices and many small vectors, odd ones among them."""
    shares = [1.0 / (1 + k) ** 1.5 for k in range(tensors)]
    sizes = [max(1, int(elements * s / sum(shares))) for s in shares]
    sizes[0] = max(1, elements - sum(sizes[1:]))
    return sizes


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op = case["op"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device=DEV, generator=gen) * std

    if op in ("norm", "norm8", "norm_grad"):
        n, w, dt = case["tokens"], case["width"], TYPES[case["type"]]
        # a residual stream: tokens of different size, a few columns that stand out
        size = torch.exp(normal(n, 1) * 0.5)
        column = torch.exp(normal(w) * 0.7)
        state = {"op": op, "x": (normal(n, w) * size * column).to(dt), "weight": None, "other": None, "block": case.get("block", 0)}
        if case["weight"]:
            state["weight"] = (1.0 + normal(w, std=0.2)).to(dt)
        if case["residual"]:
            # the stream itself, or for the gradient what arrives through it
            state["other"] = normal(n, w, std=1e-3 if op == "norm_grad" else 1.0).to(dt)
        if op == "norm_grad":
            state["grad_out"] = normal(n, w, std=1e-3).to(dt)
        return state
    if op in ("route", "route_grad"):
        t, e, dt = case["tokens"], case["experts"], TYPES[case["type"]]
        logits = normal(t, e, std=1.2) + normal(e, std=0.5)
        logits.masked_fill_(torch.rand(t, e, device=DEV, generator=gen) < 0.02, -math.inf)  # experts that are full or switched off
        logits.masked_fill_(torch.rand(t, 1, device=DEV, generator=gen) < 0.01, -math.inf)  # padding
        state = {"op": op, "logits": logits.to(dt), "bias": normal(e, std=0.05) if case["bias"] else None, "k": case["k"], "score": case["score"],
                 "groups": case["groups"], "top_groups": case["top_groups"], "group_score": "top2" if case["bias"] else "max",
                 "renormalize": case["renormalize"], "scale": 2.5 if case["score"] == "sigmoid" else 1.0}
        if op == "route_grad":
            state["ids"] = _chosen(state)[0]
            state["grad_weights"] = normal(t, case["k"], std=1e-3)
        return state
    workers, sizes = case["workers"], _parts(case["tensors"], case["elements"])
    state = {"op": op, "workers": workers, "per_worker": workers > 1}
    if workers > 1:  # matrices inside the workers' rows, and the rows that the event kernels read
        pitch = (sum(sizes) + 7) // 8 * 8
        state["rows"], state["out_rows"] = torch.zeros(workers, pitch, device=DEV), torch.zeros(workers, pitch, device=DEV)
        lows = [sum(sizes[:i]) for i in range(len(sizes))]
        worker_size = torch.exp(normal(workers, 1))
        state["tensors"], state["out"] = ([buf[:, lo:lo + size] for lo, size in zip(lows, sizes)] for buf in (state["rows"], state["out_rows"]))
        for part in state["tensors"]:
            part.copy_(normal(workers, part.shape[1]) * worker_size)
    else:
        kinds = [torch.bfloat16 if case["mixed"] and i % 3 != 1 else torch.float32 for i in range(len(sizes))]
        state["tensors"] = [normal(size, std=10.0 ** -(i % 3)).to(dt) for i, (size, dt) in enumerate(zip(sizes, kinds))]
        state["out"] = [torch.empty_like(p) for p in state["tensors"]]
    rms = math.sqrt(case["elements"])
    state["max_norm"] = rms * 1e-3 if case["clipped"] else rms * 1e3
    return state


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def _normalised(state):
    s = state["x"].float()
    if state["other"] is not None:
        s = s + state["other"].float()
    y = s * torch.rsqrt(s.square().mean(dim=1, keepdim=True) + EPS)
    return s, y if state["weight"] is None else y * state["weight"].float()


def _scores(state, x):
    """Scores of the available experts from their logits (zero for the others)."""
    if state["score"] == "sigmoid":
        return torch.sigmoid(x)
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    return e / e.sum(dim=1, keepdim=True).clamp(min=1e-30)


def _chosen(state):
    """(ids int32 [t, k], counts int32 [experts]): the choice, in 64 bits."""
    logits, k, groups = state["logits"], state["k"], state["groups"]
    t, experts = logits.shape
    available = logits > torch.finfo(logits.dtype).min
    x = torch.where(available, logits.double(), torch.full((), -math.inf, device=DEV, dtype=torch.float64))
    ranked = x
    if state["bias"] is not None or state["group_score"] == "top2":
        key = _scores(state, x)
        key = key if state["bias"] is None else key + state["bias"].double()
        key = torch.where(available, key, torch.full_like(key, -math.inf))
        ranked = key if state["bias"] is not None else x
    if groups > 1:
        if state["group_score"] == "top2":
            best = key.view(t, groups, -1).sort(dim=2, descending=True).values[:, :, :2].sum(dim=2)
        else:
            best = ranked.view(t, groups, -1).amax(dim=2)
        order = best.sort(dim=1, descending=True, stable=True).indices[:, :state["top_groups"]]
        open_ = torch.zeros(t, groups, device=DEV, dtype=torch.bool).scatter_(1, order, True)
        ranked = ranked.masked_fill(~open_.repeat_interleave(experts // groups, dim=1), -math.inf)
    values, ids = ranked.sort(dim=1, descending=True, stable=True)
    ids = torch.where(values[:, :k] > -math.inf, ids[:, :k], torch.full((), -1, device=DEV))
    counts = torch.bincount(ids.reshape(-1) + 1, minlength=experts + 1)[1:]
    return ids.to(torch.int32), counts.to(torch.int32)


def _of_chosen(state, ids):
    """(scores of all experts, those of the chosen ones, which are any, sums of the chosen) in 32 bits."""
    logits = state["logits"]
    x = torch.where(logits > torch.finfo(logits.dtype).min, logits.float(), torch.full((), -math.inf, device=DEV))
    s = _scores(state, x)
    live = ids >= 0
    a = s.gather(1, ids.long().clamp(min=0)) * live
    return s, a, live, a.sum(dim=1, keepdim=True).clamp(min=1e-30)


def run(state):
    if own:
        return _run_own(state)
    op = state["op"]
    if op == "norm":
        s, y = _normalised(state)
        dt = state["x"].dtype
        return {"y": y.to(dt)} if state["other"] is None else {"y": y.to(dt), "sum": s.to(dt)}
    if op == "norm8":
        s, y = _normalised(state)
        n, w = y.shape
        block = state["block"] or w
        blocks = -(-w // block)
        y = torch.nn.functional.pad(y, (0, blocks * block - w)).view(n, blocks, block)
        scales = (y.abs().amax(dim=2, keepdim=True) / E4M3_MAX).clamp(min=SCALE_MIN)
        values = (y / scales).to(torch.float8_e4m3fn).float() * scales
        out = {"values": values.view(n, -1)[:, :w].to(torch.bfloat16), "scales": scales[:, :, 0]}
        if state["other"] is not None:
            out["sum"] = s.to(state["x"].dtype)
        return out
    if op == "norm_grad":
        x, g, dt = state["x"].float(), state["grad_out"].float(), state["x"].dtype
        r = torch.rsqrt(x.square().mean(dim=1, keepdim=True) + EPS)
        hat = x * r
        wg = g if state["weight"] is None else g * state["weight"].float()
        dx = r * (wg - hat * (hat * wg).mean(dim=1, keepdim=True))
        if state["other"] is not None:
            dx = dx + state["other"].float()
        out = {"grad_x": dx.to(dt)}
        if state["weight"] is not None:
            out["grad_weight"] = (g * hat).sum(dim=0).to(dt)
        return out
    if op == "route":
        ids, counts = _chosen(state)
        _, a, _, total = _of_chosen(state, ids)
        return {"ids": ids, "weights": (a / total if state["renormalize"] else a) * state["scale"], "counts": counts}
    if op == "route_grad":
        ids = state["ids"]
        s, a, live, total = _of_chosen(state, ids)
        g = state["grad_weights"] * live * state["scale"]
        da = (g - (g * a).sum(dim=1, keepdim=True) / total) / total if state["renormalize"] else g
        ds = torch.zeros_like(s).scatter_add_(1, ids.long().clamp(min=0), da * live)
        dz = ds * s * (1.0 - s) if state["score"] == "sigmoid" else s * (ds - (ds * s).sum(dim=1, keepdim=True))
        return dz.to(state["logits"].dtype)
    if state["per_worker"]:
        norms = torch.sqrt(sum([p.float().square().sum(dim=1) for p in state["tensors"]]))
        factor = (state["max_norm"] / norms).clamp(max=1.0)[:, None]
    else:
        norms = torch.sqrt(sum([p.float().square().sum() for p in state["tensors"]]))
        factor = (state["max_norm"] / norms).clamp(max=1.0)
    _ = [o.copy_((p.float() * factor).to(p.dtype)) for p, o in zip(state["tensors"], state["out"])]
    return {"norms": norms, "out": state["out_rows"] if state["per_worker"] else state["out"]}


def _run_own(state):
    from paper_2306_08289_b200 import operators as ops

    op = state["op"]
    if op == "norm":
        if state["other"] is None:
            return {"y": ops.rms_norm(state["x"], state["weight"], eps=EPS)}
        y, s = ops.rms_norm(state["x"], state["weight"], residual=state["other"], eps=EPS)
        return {"y": y, "sum": s}
    if op == "norm8":
        got = ops.rms_norm_quantized(state["x"], state["weight"], residual=state["other"], eps=EPS, block=state["block"])
        out = {"values": ops.dequantize(got[0], got[1], torch.bfloat16), "scales": got[1]}
        if state["other"] is not None:
            out["sum"] = got[2]
        return out
    if op == "norm_grad":
        gx, gw = ops.rms_norm_grad(state["grad_out"], state["x"], state["weight"], grad_sum=state["other"], eps=EPS)
        return {"grad_x": gx} if gw is None else {"grad_x": gx, "grad_weight": gw}
    if op == "route":
        ids, weights, counts = ops.route(state["logits"], state["k"], score=state["score"], bias=state["bias"], groups=state["groups"],
                                         top_groups=state["top_groups"], group_score=state["group_score"], renormalize=state["renormalize"],
                                         scale=state["scale"])
        return {"ids": ids, "weights": weights, "counts": counts}
    if op == "route_grad":
        return ops.route_grad(state["logits"], state["ids"], state["grad_weights"], score=state["score"], renormalize=state["renormalize"],
                              scale=state["scale"])
    norms = ops.clip_gradients(state["tensors"], state["max_norm"], per_worker=state["per_worker"], out=state["out"])
    return {"norms": norms, "out": state["out_rows"] if state["per_worker"] else state["out"]}


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("norm", "norm8", "norm_grad"):
        n, w, size = case["tokens"], case["width"], 2 if case["type"] == "bf16" else 4
        row, weight = n * w * size, w * size * case["weight"]
        if op == "norm":
            return {"bytes": (4 if case["residual"] else 2) * row + weight, "flops": 5.0 * n * w}
        if op == "norm8":
            scales = 4 * n * (-(-w // case["block"]) if case["block"] else 1)
            # the 8-bit values are written, read back and widened to 16 bits
            return {"bytes": (3 if case["residual"] else 1) * row + weight + n * w * (1 + 1 + 2) + 2 * scales, "flops": 8.0 * n * w}
        return {"bytes": (4 if case["residual"] else 3) * row + 2 * weight, "flops": 10.0 * n * w}
    if op in ("route", "route_grad"):
        t, e, k, size = case["tokens"], case["experts"], case["k"], 2 if case["type"] == "bf16" else 4
        chosen = 8 * t * k
        if op == "route":
            return {"bytes": t * e * size + chosen + 4 * e * (1 + case["bias"]), "flops": 4.0 * t * e}
        read = t * e if case["score"] == "softmax" and not case["renormalize"] else t * k
        return {"bytes": (read + t * e) * size + chosen, "flops": 4.0 * read}
    sizes = _parts(case["tensors"], case["elements"])
    total = sum(size * (2 if case["mixed"] and i % 3 != 1 else 4) for i, size in enumerate(sizes)) * case["workers"]
    return {"bytes": 2 * total + 4 * case["workers"], "flops": 3.0 * sum(sizes) * case["workers"]}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _e4m3(v):
    """The nearest value of 4 exponent and 3 mantissa bits, ties to even, saturating at the largest."""
    _, exponent = torch.frexp(v)
    step = torch.exp2((exponent - 4).clamp(min=-9).double())
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "norm8"):
        s = state["x"].double()
        if state["other"] is not None:
            s += state["other"]
        y = s / torch.sqrt((s * s).sum(1) / case["width"] + EPS)[:, None]
        if state["weight"] is not None:
            y *= state["weight"]
        out = {"y": y}
        if op == "norm8":
            block = case["block"] or case["width"]
            pieces, scales = [], []
            for lo in range(0, case["width"], block):
                piece = y[:, lo:lo + block]
                scale = torch.linalg.vector_norm(piece, math.inf, dim=1, keepdim=True) / E4M3_MAX
                scale = torch.maximum(scale, torch.full_like(scale, SCALE_MIN))
                pieces.append(_e4m3(piece / scale) * scale)
                scales.append(scale)
            out = {"values": torch.cat(pieces, 1), "scales": torch.cat(scales, 1)}
        if state["other"] is not None:
            out["sum"] = s
        return out
    if op == "norm_grad":
        x, g = state["x"].double(), state["grad_out"].double()
        wg = g if state["weight"] is None else g * state["weight"]
        mean = torch.einsum("nw,nw->n", x, x) / case["width"] + EPS
        # d/dx of x_j w_j g_j / sqrt(mean): the direct part, and the one through the mean
        through = torch.einsum("nw,nw->n", x, wg) / case["width"] / mean**1.5
        out = {"grad_x": wg / torch.sqrt(mean)[:, None] - x * through[:, None]}
        if state["other"] is not None:
            out["grad_x"] += state["other"]
        if state["weight"] is not None:
            out["grad_weight"] = torch.einsum("nw,nw,n->w", g, x, mean**-0.5)
        return out
    if op in ("route", "route_grad"):
        logits = state["logits"].double()
        t, e, k = case["tokens"], case["experts"], case["k"]
        masked = torch.isinf(logits)
        if case["score"] == "sigmoid":
            s = torch.where(masked, 0.0, 1.0 / (1.0 + torch.exp(-logits)))
        else:
            s = torch.nan_to_num(torch.softmax(logits, dim=1), nan=0.0)
        rows = torch.arange(t, device=DEV)
        if op == "route":
            key = s + state["bias"].double() if case["bias"] else logits.clone()
            key[masked] = -math.inf
            if case["groups"] > 1:
                # top groups one after the other: the lowest of those with the best score
                size = e // case["groups"]
                g = key.reshape(t, case["groups"], size)
                first = g.amax(2)
                if case["bias"]:
                    at = (g == first[:, :, None]).to(torch.int8).argmax(2, keepdim=True)
                    score = first + g.scatter(2, at, -math.inf).amax(2) if size > 1 else first
                else:
                    score = first
                taken = torch.zeros(t, case["groups"], device=DEV, dtype=torch.bool)
                numbers = torch.arange(case["groups"], device=DEV)
                for _ in range(case["top_groups"]):
                    best = score.masked_fill(taken, -math.inf).amax(1, keepdim=True)
                    here = (score == best) & ~taken
                    taken[rows, torch.where(here, numbers, case["groups"]).amin(1)] = True
                g[~taken] = -math.inf
                key = g.reshape(t, e)
            numbers = torch.arange(e, device=DEV)
            ids = torch.full((t, k), -1, device=DEV, dtype=torch.int64)
            for j in range(k):
                best = key.amax(1, keepdim=True)
                at = torch.where(key == best, numbers, e).amin(1)
                found = best[:, 0] > -math.inf
                ids[:, j] = torch.where(found, at, -1)
                key[rows, at] = -math.inf
        else:
            ids = state["ids"].long()
        live = ids >= 0
        a = torch.where(live, s[rows[:, None], ids.clamp(min=0)], 0.0)
        total = a.sum(1, keepdim=True)
        total[total == 0] = 1.0
        w = a * state["scale"] / (total if case["renormalize"] else 1.0)
        if op == "route":
            counts = torch.zeros(e, device=DEV, dtype=torch.int64)
            counts.index_add_(0, ids[live], torch.ones_like(ids[live]))
            return {"ids": ids.to(torch.int32), "weights": w, "counts": counts.to(torch.int32)}
        # derivatives by the chosen scores' logarithms, then by the logits
        h = torch.where(live, state["grad_weights"].double(), 0.0) * w
        if case["renormalize"]:
            h = h - a / total * h.sum(1, keepdim=True)
        out = torch.zeros(t, e, device=DEV, dtype=torch.float64)
        if case["score"] == "sigmoid":
            h = h * (1.0 - a)
        for j in range(k):
            out[rows, ids[:, j].clamp(min=0)] += h[:, j] * live[:, j]
        if case["score"] == "softmax" and not case["renormalize"]:
            out -= s * h.sum(1, keepdim=True)
        return out
    tensors, max_norm = state["tensors"], state["max_norm"]
    if state["per_worker"]:
        rows = state["rows"].double()
        norms = torch.linalg.vector_norm(rows, dim=1)
        return {"norms": norms, "out": rows * torch.minimum(torch.ones_like(norms), max_norm / norms)[:, None]}
    norms = torch.sqrt(torch.stack([torch.dot(p.double(), p.double()) for p in tensors]).sum())
    factor = min(1.0, max_norm / float(norms))
    return {"norms": norms, "out": [p.double() * factor for p in tensors]}
