"""Norm, routing and clipping where single bits, neighbouring rows or ties decide: beside the bounds of test_gpu_train_operators.py."""
import math

import numpy as np
import pytest
import torch

from paper_2306_08289_b200 import binding as B
from paper_2306_08289_b200 import language_model as LM
from paper_2306_08289_b200 import operators as ops
from tests.test_gpu_operators import DEV, DT, assert_within, gen
from tests.test_gpu_train_operators import TINY, grad_of, reference_loss, route_of

pytestmark = pytest.mark.gpu


def quotients(y, block):
    """(values, scales) of a result in fp32, by the definition: scale = max(largest magnitude / 448, 2^-126), values = result / scale to the nearest of 8 bits, ties to even. Both
    quotients are of two tensors, which torch divides by the IEEE rule (a number it would multiply by its reciprocal)."""
    n, width = y.shape
    b = block or width
    blocks = -(-width // b)
    most = torch.nn.functional.pad(y, (0, blocks * b - width)).view(n, blocks, b).abs().amax(2)
    scales = (most / torch.full_like(most, 448.0)).clamp(min=2.0**-126)
    return (y / scales.repeat_interleave(b, 1)[:, :width]).to(torch.float8_e4m3fn), scales


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("block", [0, 32, 64, 128])
@pytest.mark.parametrize("n,width", [(4096, 2048), (3000, 200), (1, 8192)])
def test_values_in_8_bits_are_the_nearest_of_the_quotients(storage, block, n, width):
    """Bit for bit. Rows are whole numbers up to 15, whose squares' sums fp32 holds exactly in any order, so that the result before the 8 bits is that of `rms_norm` on the
    same rows in fp32; a weight of 24 bits (8 of bf16) spreads the quotients over all fractions. 2^23 of them have some 50 within an approximate reciprocal's error of the middle
    of two values."""
    g, dt = gen(width + block), DT[storage]
    x = torch.randint(-15, 16, (n, width), generator=g, device=DEV).to(dt)
    x[0, : width // 2] = 0
    w = torch.randn(width, generator=g, device=DEV).to(dt)
    w[3] *= 2.0**-12  # results below the 8 bits' normal range
    values, scales = ops.rms_norm_quantized(x, w, block=block)
    y = ops.rms_norm(x.float(), w.float())
    want, want_scales = quotients(y, block)
    assert torch.equal(scales, want_scales)
    assert torch.equal(values.view(torch.uint8), want.view(torch.uint8))


def test_values_in_8_bits_of_extreme_results():
    """Results from the end of fp32's range to its other end, in one block and over several, beside the largest and the smallest scale."""
    g = gen(3)
    x = torch.randint(-15, 16, (64, 256), generator=g, device=DEV).float()
    for low, high in ((-140, -100), (-20, 20), (90, 123)):
        w = torch.randn(256, generator=g, device=DEV) * torch.exp2(torch.randint(low, high + 1, (256,), generator=g, device=DEV).float())
        for block in (0, 32, 128):
            values, scales = ops.rms_norm_quantized(x, w, block=block)
            want, want_scales = quotients(ops.rms_norm(x, w), block)
            assert torch.equal(scales, want_scales)
            assert torch.equal(values.view(torch.uint8), want.view(torch.uint8)), (low, block)


# groups of 2, 4 and 3 warps, 8 warps alone in bf16 and fp32: (type, rows, columns)
@pytest.mark.parametrize("storage,n,width", [("bf16", 16384, 2048), ("f32", 16384, 1024), ("bf16", 9001, 520), ("f32", 9001, 260), ("bf16", 6000, 1030), ("f32", 6000, 2047), ("bf16", 6000, 4096)])
@pytest.mark.parametrize("special", ["nan", "inf", "zeros", "large", "small"])
def test_rows_out_of_range_leave_the_gradient_of_the_others_alone(storage, n, width, special):
    """Every seventh row needs the scaled way; all other rows have the bits that they have without such rows, in every one of many calls, and so has the weight's gradient from call to
    call."""
    g, dt = gen(n + width), DT[storage]
    x, go = (torch.randn(n, width, generator=g, device=DEV).to(dt) for _ in range(2))
    w = (1.0 + 0.3 * torch.randn(width, generator=g, device=DEV)).to(dt)
    want, _ = ops.rms_norm_grad(go, x, w, eps=0.0)
    odd = x.clone()
    rows = odd[3::7]
    if special == "nan":
        rows[:, width // 2] = math.nan
    elif special == "inf":
        rows[:, width - 1] = math.inf
    elif special == "zeros":
        rows.zero_()
    else:
        rows.mul_(2.0**80 if special == "large" else 2.0**-80)
    others = torch.arange(n, device=DEV) % 7 != 3
    first = None
    for _ in range(50):
        gx, gw = ops.rms_norm_grad(go, odd, w, eps=0.0)
        assert torch.equal(gx[others], want[others])
        first = (gx, gw) if first is None else first
        assert torch.equal(gw.view(torch.int8), first[1].view(torch.int8)) and torch.equal(gx.view(torch.int8), first[0].view(torch.int8))
    if special in ("nan", "inf"):
        assert torch.isnan(gx[3::7]).any(1).all()
    elif special == "zeros":
        assert not gx[3::7].any()
    if special in ("zeros", "large", "small"):
        # of the columns: a zero row adds nothing, a scaled one what it adds unscaled. At most 16384 / 148 additions in a slot's column, 2048 in the join, and a term's 2^-17
        keep = others if special == "zeros" else torch.ones_like(others)
        terms = go.double() * x.double() / torch.sqrt((x.double() ** 2).mean(1, keepdim=True))
        terms[~keep] = 0.0
        u = 2.0**-8 if storage == "bf16" else 2.0**-24
        assert_within(gw, terms.sum(0), ((n / 148 + 2048) * 2.0**-24 + 2.0**-17) * terms.abs().sum(0) + u * terms.sum(0).abs())


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("width", [48, 1000, 2048, 9000])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("with_sum", [False, True])
def test_gradients_of_zero_rows_and_of_rows_out_of_range(storage, width, eps, with_sum):
    """A row of zeros without eps has zeros for its own part and adds none to the weight's gradient, one with eps has r w g; rows beyond fp32's squares as the formula says."""
    g, dt = gen(width), DT[storage]
    u = 2.0**-8 if storage == "bf16" else 2.0**-24
    x = torch.randn(40, width, generator=g, device=DEV, dtype=torch.float64)
    x[1::8] *= 2.0**90
    x[2::8] *= 2.0**-90
    x[3::8] = 0.0
    x[5::8] = 0.0
    x[5::8, width - 1] = 2.0**100
    x = x.to(dt)
    go, ds = (torch.randn(40, width, generator=g, device=DEV).to(dt) for _ in range(2))
    w = (1.0 + 0.3 * torch.randn(width, generator=g, device=DEV)).to(dt)
    gx, gw = ops.rms_norm_grad(go, x, w, eps=eps, grad_sum=ds if with_sum else None)
    zero = ~x.any(1)
    assert int(zero.sum()) == 5
    if eps == 0.0:
        assert torch.equal(gx[zero], ds[zero] if with_sum else torch.zeros_like(gx[zero]))
    d, size = grad_of(go.double(), x.double(), w, eps, ds.double() if with_sum else None)
    rows = ~zero if eps == 0.0 else torch.ones_like(zero)
    assert_within(gx[rows], d[rows], 2.0**-16 * size[rows] + u * d[rows].abs() + TINY[storage])  # as in test_rms_norm_grad
    hat = x.double() / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + eps)
    terms = (go.double() * hat).nan_to_num(0.0)
    assert_within(gw, terms.sum(0), (40 * 2.0**-24 + 2.0**-17) * terms.abs().sum(0) + u * terms.sum(0).abs() + TINY[storage])


# ------------------------------------------------------------------------------------------------
# routing
# ------------------------------------------------------------------------------------------------
def tied_tokens(n, experts, k, dt, score, with_bias, g):
    """(logits, bias): k - 1 or k - 2 experts of every token are sure to be chosen; for the places that are left there are some with the same logit and bias, and one or two with a
    slightly larger key that fp32 scores (without a bias: the keys' upper bits) cannot tell from theirs."""
    z = torch.full((n, experts), -45.0, device=DEV)
    bias = torch.zeros(experts, device=DEV) if with_bias else None
    base, more = 30.0, 31.0  # of a sigmoid: 1 - 9e-14 and 1 - 3e-14
    if not with_bias:
        base, more = 1.5, 1.5 + 2.0**-23
    elif score == "softmax":  # beside an expert that has almost all of the sum, and is out by its bias: 1 + 2e-9 and 1 + 3e-9, or less
        base, more = 10.0, 10.5
    for t in range(n):
        order = torch.randperm(experts - 1, generator=g, device=DEV) + 1
        sure = max(0, k - 1 - t % 2)
        equal, larger = 2 + t % 5, 1 + t // 5 % 2
        at = order[: sure + equal + larger].cpu()
        tied = at[sure:].sort().values if t % 3 else at[sure:]  # the larger ones behind the others, or anywhere
        z[t, at[:sure]] = 2.0 if not with_bias else 40.0 + torch.arange(sure, device=DEV) if score == "sigmoid" else 20.0 + 0.5 * torch.arange(sure, device=DEV)
        z[t, tied[:equal]] = base
        z[t, tied[equal:]] = more
    if with_bias and score == "softmax":
        z[:, 0] = 30.0
        bias += 1.0
        bias[0] = -4.0
    return z.to(dt), bias


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("experts,k", [(16, 1), (16, 3), (32, 2), (64, 1), (64, 8), (128, 4), (256, 1), (256, 8), (500, 2), (1024, 8), (1024, 31)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (4, 4), (4, 3)])
def test_route_where_the_last_choice_is_tied_with_one_and_beaten_by_another(storage, experts, k, score, with_bias, groups, top_groups):
    """The tie says nothing about the third expert, which has the larger key."""
    n = 60
    z, bias = tied_tokens(n, experts, k, DT[storage], score, with_bias, gen(experts + k))
    k = min(k, experts // groups * top_groups)
    args = dict(score=score, bias=bias, groups=groups, top_groups=top_groups, group_score="max", renormalize=True, scale=1.0)
    ids = ops.route(z, k, **args)[0].cpu().numpy()
    want = route_of(z, k, **args)[0]
    assert (ids == want).all(), (ids[(ids != want).any(1)][:3], want[(ids != want).any(1)][:3])
    many = ops.route(z.repeat(50, 1), k, **args)[0].view(50, n, k)
    assert (many == many[0]).all() and (many[0].cpu().numpy() == want).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (4, 2)])
def test_route_of_infinite_logits_beside_the_largest_float(score, renormalize, with_bias, groups, top_groups):
    """A logit of +inf counts as the largest float, so the lower expert comes first, whatever is asked for beside the choice."""
    big = torch.finfo(torch.float32).max
    for experts in (8, 64, 256, 1024):
        z = torch.randn(40, experts, generator=gen(experts), device=DEV)
        low, high = experts // 4, experts // 2 - 1  # of one group of two
        low, high = (low, high) if groups == 1 else (experts // 4, experts // 4 + 1)
        z[:, low] = big
        z[:, high] = math.inf
        z[20:, low], z[20:, high] = math.inf, big
        z[30:, experts - 1] = math.inf
        bias = torch.zeros(experts, device=DEV) if with_bias else None
        args = dict(score=score, bias=bias, groups=groups, top_groups=top_groups, group_score="max", renormalize=renormalize, scale=1.0)
        ids, weights, _ = ops.route(z, 2, **args)
        want = torch.tensor([low, high], dtype=torch.int32, device=DEV)
        assert (ids == want).all(), (ids[0], ids[-1])
        share = 0.5 if renormalize or score == "softmax" else 1.0
        assert (weights[:30] == share).all() and torch.isfinite(weights).all()


@pytest.mark.parametrize("experts", [8, 64, 65, 128, 256, 500, 1024])
def test_dense_gradient_of_experts_far_below_the_best(experts):
    """Softmax, not renormalised, one expert chosen that has the whole sum: the others' gradients are -s_e g s. Differences of logits are whole multiples of 2^-8, so no error comes from
    them; the exponential is off by a unit in the last place (2^-23), and there are at most six roundings beside it: 2^-21 in all, however small s_e."""
    g = gen(experts)
    z = -50.0 - torch.randint(0, 37 * 256 + 1, (300, experts), generator=g, device=DEV) / 256.0  # down to e^-87, above the smallest normal float
    best = torch.randint(0, experts, (300, 1), generator=g, device=DEV)
    z.scatter_(1, best, 0.0)
    gw = torch.randn(300, 1, generator=g, device=DEV) * 100.0
    got = ops.route_grad(z, best.to(torch.int32), gw, score="softmax", renormalize=False)
    s = torch.softmax(z.double(), 1)
    chosen = torch.zeros_like(s).scatter_(1, best, 1.0)
    # the chosen expert's own is g s (1 - s), a difference of nearly equal numbers
    want = s * (chosen - s.gather(1, best)) * gw.double()
    assert_within(got, want, 2.0**-21 * (want.abs() + chosen * gw.double().abs()))


# ------------------------------------------------------------------------------------------------
# the example
# ------------------------------------------------------------------------------------------------
def test_forward_of_a_model_without_norms_and_experts_gives_three_tensors():
    model = LM.Model(40, 24)
    row = torch.from_numpy(model.initial_row(5)).to(DEV)
    ids = torch.arange(30, dtype=torch.int32, device=DEV)
    y, a, h = model.forward(row, ids)
    assert y.shape == a.shape == h.shape == (30, 24) and torch.equal(h, y + a)
    assert torch.equal(a, torch.tanh(y @ model.part(row, "M").T))
    for more in (dict(norm=True), dict(experts=4), dict(norm=True, experts=4)):
        model = LM.Model(40, 24, **more)
        assert len(model.forward(torch.from_numpy(model.initial_row(5)).to(DEV), ids)) == 6


@pytest.mark.parametrize("norm,experts", [(False, 0), (True, 0), (False, 5), (True, 8)])
def test_gradients_of_the_example_in_bf16(norm, experts):
    """Against autograd in 64 bits at the same row. Some 16 tensors on the way are rounded to bf16 (2^-8 each), and 1 - a^2 of an ordinary tanh doubles what a was off by: 2^-3 of a part. The
    router's part is a difference of the chosen experts' gradients, whose errors are relative to their magnitudes."""
    text = LM.MarkovText(40, 4, 1)
    model = LM.Model(40, 24, norm=norm, experts=experts)
    row = torch.from_numpy(model.initial_row(5)).to(DEV)
    row = (row + 0.05 * torch.randn(model.d, generator=gen(1), device=DEV)).bfloat16()
    ids, targets = (torch.from_numpy(v).to(DEV) for v in text.draw(np.random.default_rng(2), 6, 11))
    out = torch.full((model.d,), math.nan, device=DEV, dtype=torch.bfloat16)
    model.gradient(row, ids, targets, 0.1, out)
    chosen = model.forward(row, ids)[3][1].long() if experts else None
    wide = row.double().requires_grad_()
    reference_loss(model, wide, ids, targets, 0.1, chosen).backward()
    for name in model.shape:
        got, want = model.part(out, name).double(), model.part(wide.grad, name)
        bound = 2.0**-3 * float(want.norm())
        if name == "R":
            _, u, _, (_, _, weights, _, picked), _, _ = model.forward(row, ids)
            _, _, dh, _ = ops.vocab_loss_grad(model.forward(row, ids)[5], model.part(row, "W"), targets, scale=0.1)
            if norm:
                dh, _ = ops.rms_norm_grad(dh, model.forward(row, ids)[4], model.part(row, "F")[0])
            each = weights.double() * (picked.double() * dh.double()[:, None]).abs().sum(2)
            size = torch.zeros(len(ids), experts, dtype=torch.float64, device=DEV).scatter_add_(1, chosen, each)
            bound = 2.0**-3 * float((size.T @ u.double().abs()).norm())
        assert torch.isfinite(got).all() and float((got - want).norm()) <= bound, name


# ------------------------------------------------------------------------------------------------
# the two ways to the library
# ------------------------------------------------------------------------------------------------
def calls_of_every_kind(storage):
    g, dt = gen(7), DT[storage]
    x, r, go = (torch.randn(70, 200, generator=g, device=DEV).to(dt) for _ in range(3))
    w = torch.randn(200, generator=g, device=DEV).to(dt)
    z, bias = torch.randn(70, 64, generator=g, device=DEV).to(dt), torch.randn(64, generator=g, device=DEV) * 0.1
    inside = torch.randn(70, 211, generator=g, device=DEV).to(dt)[:, 3:203]
    values, scales = ops.rms_norm_quantized(x, w, block=64)
    ids, weights, _ = ops.route(z, 4)
    workers = torch.randn(6, 5000, generator=g, device=DEV).to(dt)
    parts = [workers[:, :3000].view(6, 50, 60), workers[:, 3000:3007], workers[:, 4000:]]
    return {
        "norm": lambda: ops.rms_norm(x, w), "norm, residual": lambda: ops.rms_norm(x, None, residual=r, eps=1e-3), "norm inside rows": lambda: ops.rms_norm(inside, w, residual=x),
        "norm of no rows": lambda: ops.rms_norm(x[:0], w, residual=x[:0]), "norm of one row": lambda: ops.rms_norm(x[3:4], w), "eps whole": lambda: ops.rms_norm(x, w, eps=1),
        "8 bits": lambda: ops.rms_norm_quantized(x, w, block=64), "8 bits a row, residual": lambda: ops.rms_norm_quantized(inside, w, residual=r, block=0),
        "back": lambda: ops.dequantize(values, scales), "back to fp32": lambda: ops.dequantize(values, scales, torch.float32), "back, inside": lambda: ops.dequantize(values[:, :192], scales[:, :3].contiguous()),
        "gradient": lambda: ops.rms_norm_grad(go, x, w), "gradient, sum": lambda: ops.rms_norm_grad(go, inside, w, grad_sum=r), "gradient of rows": lambda: ops.rms_norm_grad(go, x, w, grad_weight=None),
        "gradient of the weight": lambda: ops.rms_norm_grad(go, x, w, grad_x=None), "gradient without a weight": lambda: ops.rms_norm_grad(go, x), "gradient of no rows": lambda: ops.rms_norm_grad(go[:0], x[:0], w),
        "route": lambda: ops.route(z, 4), "route, groups": lambda: ops.route(z, 6, "sigmoid", bias, 8, 3, "top2", False, 2.5), "route of one": lambda: ops.route(z[5:6], 1, renormalize=False),
        "route of none": lambda: ops.route(z[:0], 3), "route gradient": lambda: ops.route_grad(z, ids, weights), "route gradient, sigmoid": lambda: ops.route_grad(z, ids, weights, "sigmoid", False, 2),
        "norms": lambda: ops.gradient_norms([x, w, z]), "norms of workers": lambda: ops.gradient_norms(parts, per_worker=True), "norms of a tuple": lambda: ops.gradient_norms((x, r)),
        "clipped": lambda: [t := [x.clone(), w.clone()], ops.clip_gradients(t, 1.0)], "clipped workers": lambda: [t := workers.clone(), ops.clip_gradients([t[:, 9:3009], t[:, 3100:]], 2.0, per_worker=True, zero_nonfinite=True)],
        "clipped elsewhere": lambda: [o := [torch.empty_like(x), torch.empty_like(w)], ops.clip_gradients([x, w], 0.5, out=o)], "not clipped": lambda: [t := [x.clone()], ops.clip_gradients(t, math.inf)],
    }


def refused_of_every_kind(storage):
    dt = DT[storage]
    x, w = torch.randn(10, 64, device=DEV).to(dt), torch.ones(64, device=DEV).to(dt)
    wide = torch.zeros(2, 32769, device=DEV).to(dt)
    ids, weights, _ = ops.route(x, 2)
    return [lambda: ops.rms_norm(x, eps=-1.0), lambda: ops.rms_norm(x, w[:5]), lambda: ops.rms_norm(wide), lambda: ops.rms_norm(x.T), lambda: ops.rms_norm_quantized(x, block=3), lambda: ops.rms_norm_grad(x, x[:4]),
            lambda: ops.rms_norm_grad(x, x, eps=math.inf), lambda: ops.route(x, 0), lambda: ops.route(x, 65), lambda: ops.route(x, 40), lambda: ops.route(x, 2, groups=7), lambda: ops.route(x, 2, scale=math.inf),
            lambda: ops.route_grad(x, ids.long(), weights), lambda: ops.route_grad(x, ids, weights, scale=math.nan), lambda: ops.clip_gradients([x, x], 1.0), lambda: ops.clip_gradients([x], -1.0),
            lambda: ops.gradient_norms([x.half()]), lambda: ops.gradient_norms([x, w], per_worker=True), lambda: ops.gradient_norms([x[:1].expand(10, 64)])]


def flat(v):
    return [t for x in v for t in flat(x)] if isinstance(v, (list, tuple)) else [v]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_both_ways_to_the_library_give_the_same(storage, monkeypatch):
    """The calls that go to it from C++ and the ones that go from Python: results bit for bit, refusals by their codes."""
    usual = ops._usual()
    assert not isinstance(usual, ops._NoCalls)
    calls, refused = calls_of_every_kind(storage), refused_of_every_kind(storage)

    def code(call):
        with pytest.raises(B.A2Error) as e:
            call()
        return e.value.code

    first, codes = {name: flat(call()) for name, call in calls.items()}, [code(call) for call in refused]
    monkeypatch.setattr(ops, "_calls", ops._NoCalls())
    for name, call in calls.items():
        again = flat(call())
        assert len(again) == len(first[name])
        for a, b in zip(first[name], again):
            if a is None or b is None:
                assert a is b, name
                continue
            assert a.shape == b.shape and a.dtype == b.dtype and a.device == b.device and a.stride() == b.stride(), name
            assert torch.equal(a.contiguous().view(torch.uint8) if a.dim() else a, b.contiguous().view(torch.uint8) if b.dim() else b), name
    assert codes == [code(call) for call in refused]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,width,experts", [(8192, 2048, 256), (300, 129, 64), (1, 2048, 8)])
def test_calls_behind_one_another_have_the_bits_of_a_call_alone(storage, n, width, experts):
    """Passes over two sets of inputs in turn, with nothing waiting between them, so that buffers of one are those of another a moment before."""
    dt = DT[storage]

    def inputs(seed):
        g = gen(seed)
        x, r, go = (torch.randn(n, width, generator=g, device=DEV).to(dt) for _ in range(3))
        return x, r, go, torch.randn(width, generator=g, device=DEV).to(dt), torch.randn(n, experts, generator=g, device=DEV).to(dt), 0.1 * torch.randn(experts, generator=g, device=DEV)

    def one(x, r, go, w, z, bias):
        values, scales, total = ops.rms_norm_quantized(x, w, residual=r, block=128)
        back = ops.dequantize(values, scales, dt)
        gx, gw = ops.rms_norm_grad(go, total, w, grad_sum=r)
        ids, weights, counts = ops.route(z, 2, score="sigmoid", bias=bias, groups=4, top_groups=2, group_score="top2")
        dz = ops.route_grad(z, ids, weights, renormalize=False)
        out = [torch.empty_like(gx), torch.empty_like(gw), torch.empty_like(dz)]
        norms = ops.clip_gradients([gx, gw, dz], 1.0, out=out)
        return [values.view(torch.uint8), scales, total, back, gx, gw, ids, weights, counts, dz, norms, *out]

    sets = [inputs(seed) for seed in (1, 2)]
    want = []
    for s in sets:
        torch.cuda.synchronize()
        want.append([t.clone() for t in one(*s)])
        torch.cuda.synchronize()
    for k in range(60):
        got = one(*sets[k % 2])  # the results of the pass before last are free again
        if k % 7 == 6:
            assert all(torch.equal(a, b) for a, b in zip(got, want[k % 2])), k
