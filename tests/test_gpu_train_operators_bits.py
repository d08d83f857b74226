"""Norm, routing and clipping where single bits, neighbouring rows or ties decide: beside the bounds of test_gpu_train_operators.py."""
import math

import pytest
import torch

from paper_2306_08289_b200 import language_model as LM
from paper_2306_08289_b200 import operators as ops
from tests.test_gpu_operators import DEV, DT, assert_within, gen
from tests.test_gpu_train_operators import route_of

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
