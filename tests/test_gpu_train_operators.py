"""Root-mean-square norm, routing and clipping against plain implementations in 64 bits.

Tolerances are bounds of the arithmetic, written at each test: u = unit roundoff of the storage type (2^-24 fp32, 2^-8 bf16); a sum that a group of
threads takes in fp32 has at most 64 additions in a thread and 10 over the threads, so it is off by at most 75 * 2^-24 < 2^-17 of the
sum of magnitudes."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2306_08289_b200 import binding as B
from paper_2306_08289_b200 import operators as ops
from tests.test_gpu_operators import DEV, DT, SHIFTS, U, assert_within, gen, matrix, outside_untouched, slow

pytestmark = pytest.mark.gpu

TINY = {"f32": 2.0**-149, "bf16": 2.0**-133}  # the storage type's smallest step


# ------------------------------------------------------------------------------------------------
# the norm
# ------------------------------------------------------------------------------------------------
def norm_of(s, weight, eps):
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    return y if weight is None else y * weight.double()


# rows: one, odd, many; widths: one, around vectors, warps and the steps from one kernel's shape to the next, the largest
WIDTHS = [1, 7, 8, 64, 201, 256, 257, 1024, 2047, 2048, 2056, 4100, 8200, 16384, 32768]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("pad,shift", SHIFTS)
@pytest.mark.parametrize("with_residual", [False, True])
def test_rms_norm(storage, width, pad, shift, with_residual):
    n = 37 if width < 5000 else 3
    g, dt, u = gen(width + pad), DT[storage], U[storage]
    x, _ = matrix(n, width, dt, g, pad=pad, shift=shift)
    r = matrix(n, width, dt, g, pad=pad, shift=shift)[0] if with_residual else None
    w = torch.randn(width, generator=g, device=DEV).to(dt) if width % 2 == 0 else None
    out, out_buf = matrix(n, width, dt, g, pad=pad, shift=shift)
    total, total_buf = matrix(n, width, dt, g, pad=pad, shift=shift)
    s = x.double() + (r.double() if with_residual else 0.0)
    got = ops.rms_norm(x, w, residual=r, eps=1e-5, out=out, sum_out=total if with_residual else None)
    y = got[0] if with_residual else got
    assert y is out
    # the sum's relative error halves in the root; a root, a division, two products: below 2^-18 in all
    want = norm_of(s, w, 1e-5)
    assert_within(y, want, (2.0**-18 + u) * want.abs() + TINY[storage])
    outside_untouched(out, out_buf)
    if with_residual:
        assert got[1] is total
        assert_within(total, s, (u if storage == "bf16" else 0.0) * s.abs() + 2.0**-24 * s.abs() * 1.01 + TINY[storage])
        outside_untouched(total, total_buf)
    # rows that do not start alike in memory, and an allocated result
    odd, _ = matrix(n, width, dt, g, pad=pad + 1, shift=shift + 1)
    odd.copy_(x)
    again = ops.rms_norm(odd, w, residual=r, eps=1e-5)
    again = again[0] if with_residual else again
    assert_within(again, want, (2.0**-18 + u) * want.abs() + TINY[storage])


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_rms_norm_in_place_and_empty(storage):
    g, dt = gen(3), DT[storage]
    x, r, w = (torch.randn(*shape, generator=g, device=DEV).to(dt) for shape in ((50, 1000), (50, 1000), (1000,)))
    y, s = ops.rms_norm(x, w, residual=r)
    for out, total in ((0, 1), (1, 0), (0, None), (None, 1)):
        a, b = x.clone(), r.clone()
        pick = lambda i: None if i is None else (a, b)[i]  # noqa: E731
        y2, s2 = ops.rms_norm(a, w, residual=b, out=pick(out), sum_out=pick(total))
        assert torch.equal(y2, y) and torch.equal(s2, s)
    a = x.clone()
    assert torch.equal(ops.rms_norm(a, w, out=a), ops.rms_norm(x, w))
    assert ops.rms_norm(x[:0], w).shape == (0, 1000)
    y, s = ops.rms_norm(x[:0], w, residual=r[:0])
    assert y.shape == s.shape == (0, 1000)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("width", [48, 1000, 9000])
def test_rms_norm_special_rows(storage, width):
    g, dt, u = gen(8), DT[storage], U[storage]
    base = torch.randn(8, width, generator=g, device=DEV, dtype=torch.float64)
    base[1] *= 2.0**100  # squares beyond floats
    base[2] *= 2.0**-100  # and below them
    base[3] = 0.0
    base[6] *= 2.0**60
    x = base.to(dt)
    x[4, 5] = math.nan
    x[5, 7] = math.inf
    x[7] = 0.0
    x[7, width - 1] = 2.0**126
    for eps in (0.0, 1e-6):
        got = ops.rms_norm(x, eps=eps)
        want = norm_of(x.double(), None, eps)
        if eps == 0.0:
            want[3] = 0.0
        for row in (0, 1, 2, 3, 6, 7):
            assert_within(got[row], want[row], (2.0**-18 + u) * want[row].abs() + TINY[storage], (eps, row))
        assert torch.isnan(got[4]).any() and torch.isnan(got[5]).any()
        # gradients of the same rows
        go = torch.randn(8, width, generator=g, device=DEV).to(dt)
        gx, gw = ops.rms_norm_grad(go, x, torch.ones(width, dtype=dt, device=DEV), eps=eps)
        for row in (0, 1, 2, 6, 7):
            d, bound = grad_of(go[row:row + 1].double(), x[row:row + 1].double(), None, eps, None)
            top = torch.finfo(dt).max
            ok = d.abs() < top
            assert_within(gx[row:row + 1][ok], d[ok], 2.0**-16 * bound[ok] + u * d[ok].abs() + TINY[storage], (eps, row))
        assert not torch.isnan(gx[3]).any() or eps == 0.0


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_rms_norm_sum_without_a_residual(storage):
    """The library's own call writes the sum also where nothing is added: a copy of the rows."""
    dt = DT[storage]
    x = torch.randn(5, 72, generator=gen(1), device=DEV).to(dt)
    out, total = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.current_stream().cuda_stream
    assert B.lib().a2cid2_rms_norm(x.data_ptr(), 72, None, 0, None, 5, 72, 1e-6, total.data_ptr(), 72, out.data_ptr(), 72, ops._DTYPES[dt], s) == B.A2_OK
    assert torch.equal(total, x) and torch.equal(out, ops.rms_norm(x))


def test_rms_norm_offsets_past_32_bits():
    """Rows of more than 2^31 elements in all: the last ones against a copy of them."""
    n, width = 67000, 32768
    x = torch.zeros(n, width, dtype=torch.bfloat16, device=DEV)
    x[-3:] = torch.randn(3, width, generator=gen(2), device=DEV).bfloat16()
    w = torch.ones(width, dtype=torch.bfloat16, device=DEV)
    y = ops.rms_norm(x, w)
    assert torch.equal(y[-3:], ops.rms_norm(x[-3:].clone(), w)) and not y[:3].any()
    gx, gw = ops.rms_norm_grad(x, x, w, grad_x=y)
    small = ops.rms_norm_grad(x[-3:].clone(), x[-3:].clone(), w)
    assert torch.equal(gx[-3:], small[0]) and torch.allclose(gw.float(), small[1].float(), rtol=2.0**-7)
    del y, gx
    values, scales = ops.rms_norm_quantized(x, w, block=128)
    small = ops.rms_norm_quantized(x[-3:].clone(), w, block=128)
    assert torch.equal(values[-3:].view(torch.uint8), small[0].view(torch.uint8)) and torch.equal(scales[-3:], small[1])
    assert torch.equal(ops.dequantize(values, scales, out=x)[-3:], ops.dequantize(*small))


E4M3 = [0.0] + sorted({(1 + m / 8) * 2.0**e for e in range(-6, 9) for m in range(8) if (1 + m / 8) * 2.0**e <= 448} | {m * 2.0**-9 for m in range(1, 8)})


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("block", [0, 32, 64, 128])
@pytest.mark.parametrize("n,width", [(1, 1), (5, 31), (33, 128), (40, 200), (17, 1024), (9, 2056), (3, 8195), (2, 32768)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_rms_norm_quantized(storage, block, n, width, pad, shift):
    g, dt = gen(width + block), DT[storage]
    x, _ = matrix(n, width, dt, g, pad=pad, shift=shift)
    r, _ = matrix(n, width, dt, g, pad=pad, shift=shift)
    x[n - 1] = 0.0
    r[n - 1] = 0.0
    w = torch.randn(width, generator=g, device=DEV).to(dt)
    values, scales, total = ops.rms_norm_quantized(x, w, residual=r, eps=1e-5, block=block)
    b = block or width
    blocks = -(-width // b)
    assert values.dtype == torch.float8_e4m3fn and values.shape == (n, width) and scales.shape == (n, blocks)
    y, s = ops.rms_norm(x, w, residual=r, eps=1e-5)
    assert torch.equal(total, s)
    want = norm_of(x.double() + r.double(), w, 1e-5)
    padded = torch.nn.functional.pad(want, (0, blocks * b - width)).view(n, blocks, b)
    scale = (padded.abs().amax(2) / 448.0).clamp(min=2.0**-126)
    assert_within(scales, scale, 2.0**-17 * scale)  # the largest value's 2^-18, and a division
    # a value is off by half a step of its size (at least half the smallest step), and by what it was off before
    wide = scales.double().repeat_interleave(b, 1)[:, :width]
    q = values.double()
    assert_within(q * wide, want, torch.maximum(want.abs() * 2.0**-4, wide * 2.0**-10) * (1 + 2.0**-12) + 2.0**-16 * want.abs())
    assert not q[n - 1].any() and torch.equal(scales[n - 1], torch.full_like(scales[n - 1], 2.0**-126))
    # nearest values: the table's nearest entry, but for what lies within 2^-16 of the middle of two
    table = torch.tensor(E4M3, dtype=torch.float64, device=DEV)
    v = (want / wide).abs().clamp(max=448.0)
    above = torch.searchsorted(table, v.contiguous()).clamp(1, len(E4M3) - 1)
    low, high = table[above - 1], table[above]
    middle = (low + high) / 2
    sure = (v - middle).abs() > 2.0**-15 * v
    assert torch.equal(torch.where(v < middle, low, high)[sure], q.abs()[sure])
    for dtype in (torch.float32, torch.bfloat16):
        back = ops.dequantize(values, scales, dtype)
        assert torch.equal(back, (values.float() * scales.repeat_interleave(b, 1)[:, :width]).to(dtype))


def test_rms_norm_quantized_values_that_are_not_numbers():
    x = torch.randn(6, 300, generator=gen(1), device=DEV)
    x[1, 3], x[2, 250] = math.nan, math.inf
    for block in (0, 64):
        values, _ = ops.rms_norm_quantized(x, block=block)
        got = values.float()
        assert torch.isnan(got[1]).all() and torch.isnan(got[2, 250])
        assert torch.isfinite(got[[0, 3, 4, 5]]).all() and (got[2, :250] == 0).all()


def grad_of(g, x, w, eps, ds):
    """(gradient of the rows, magnitudes that its errors are relative to) in 64 bits."""
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
    h, wg = x * r, g if w is None else g * w.double()
    d = r * (wg - h * (h * wg).mean(1, keepdim=True))
    size = r * (wg.abs() + h.abs() * (h * wg).abs().mean(1, keepdim=True))
    return (d, size) if ds is None else (d + ds, size + ds.abs())


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,width", [(1, 1), (3, 7), (300, 8), (1001, 201), (77, 256), (40, 1000), (2500, 520), (9, 4104), (13, 8200), (30, 9000), (5, 16385),
                                     (3, 32760), (2, 32768)])
@pytest.mark.parametrize("pad,shift", SHIFTS)
@pytest.mark.parametrize("with_sum", [False, True])
def test_rms_norm_grad(storage, n, width, pad, shift, with_sum):
    g, dt, u = gen(n + width), DT[storage], U[storage]
    x, _ = matrix(n, width, dt, g, pad=pad, shift=shift)
    go, _ = matrix(n, width, dt, g, pad=pad, shift=shift)
    ds = matrix(n, width, dt, g, pad=pad, shift=shift)[0] if with_sum else None
    w = None if width % 4 == 0 and with_sum else (1.0 + 0.3 * torch.randn(width, generator=g, device=DEV)).to(dt)
    out, buf = matrix(n, width, dt, g, pad=pad, shift=shift)
    gw = torch.full((width,), math.nan, dtype=dt, device=DEV)
    got, _ = ops.rms_norm_grad(go, x, w, eps=1e-5, grad_sum=ds, grad_x=out, grad_weight=gw)
    d, size = grad_of(go.double(), x.double(), w, 1e-5, None if ds is None else ds.double())
    # c has two sums' errors (2^-17 each, one halved in the root) and five roundings
    assert_within(got, d, 2.0**-16 * size + u * d.abs() + TINY[storage], "rows")
    outside_untouched(out, buf)
    # at most 2500 additions in a column
    xs, gs = x.double(), go.double()
    terms = gs * xs / torch.sqrt((xs * xs).mean(1, keepdim=True) + 1e-5)
    dw, dw_size = terms.sum(0), terms.abs().sum(0)
    assert_within(gw, dw, (2500 * 2.0**-24 + 2.0**-17) * dw_size + u * dw.abs() + TINY[storage], "weight")
    again, gw2 = ops.rms_norm_grad(go, x, w, eps=1e-5, grad_sum=ds, grad_weight=True if w is not None else gw.clone())
    if pad == 0:  # the same call; rows that do not start alike are summed in another order
        assert torch.equal(again, got) and torch.equal(gw2, gw)
    assert_within(again, d, 2.0**-16 * size + u * d.abs() + TINY[storage])
    assert_within(gw2, dw, (2500 * 2.0**-24 + 2.0**-17) * dw_size + u * dw.abs() + TINY[storage])
    # either gradient alone, and in place
    alone = torch.empty_strided(x.shape, x.stride(), dtype=dt, device=DEV) if pad == 0 else matrix(n, width, dt, g, pad=pad, shift=shift)[0]
    assert torch.equal(ops.rms_norm_grad(go, x, w, eps=1e-5, grad_sum=ds, grad_x=alone, grad_weight=None)[0], got)
    assert torch.equal(ops.rms_norm_grad(go, x, w, eps=1e-5, grad_sum=ds, grad_x=None, grad_weight=gw.clone())[1], gw)
    for place in (go, x, ds):
        if place is not None:
            keep = place.clone()
            ops.rms_norm_grad(go, x, w, eps=1e-5, grad_sum=ds, grad_x=place, grad_weight=None)
            assert torch.equal(place, got)
            place.copy_(keep)


def test_rms_norm_grad_without_rows_and_of_many():
    w = torch.ones(100, device=DEV)
    x = torch.randn(0, 100, device=DEV)
    gx, gw = ops.rms_norm_grad(x, x, w)
    assert gx.shape == (0, 100) and not gw.any()
    # more rows than any number of CTAs, odd rows so that each starts elsewhere: 60,000 rows in at least 148 sequences
    g = gen(4)
    x, go = torch.randn(60001, 99, generator=g, device=DEV), torch.randn(60001, 99, generator=g, device=DEV)
    gx, gw = ops.rms_norm_grad(go, x, w[:99])
    d, size = grad_of(go.double(), x.double(), None, 1e-6, None)
    assert_within(gx, d, 2.0**-16 * size + 2.0**-24 * d.abs())
    terms = go.double() * x.double() / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + 1e-6)
    assert_within(gw, terms.sum(0), (60001 / 148 + 2048) * 2.0**-24 * terms.abs().sum(0))


def test_rms_norm_grad_is_the_difference_quotient_of_rms_norm():
    """Differences of the norm in 64 bits along the gradient: the kernels' gradient must predict them."""
    g = gen(11)
    x, r, w = (torch.randn(*shape, generator=g, device=DEV) for shape in ((12, 70), (12, 70), (70,)))
    c = torch.randn(12, 70, generator=g, device=DEV)  # the loss is sum(c * y) + sum(e * s)
    e = torch.randn(12, 70, generator=g, device=DEV)
    _, s = ops.rms_norm(x, w, residual=r)
    gx, gw = ops.rms_norm_grad(c, s, w, grad_sum=e)

    def loss(x, w):
        t = x + r.double()
        return float((c.double() * norm_of(t, w, 1e-6)).sum() + (e.double() * t).sum())

    h = 1e-5
    for dx, dw in ((gx.double(), 0.0 * gw.double()), (0.0 * gx.double(), gw.double()), (torch.randn(12, 70, generator=g, device=DEV).double(), gw.double())):
        want = (loss(x.double() + h * dx, w.double() + h * dw) - loss(x.double() - h * dx, w.double() - h * dw)) / (2 * h)
        got = float((gx.double() * dx).sum() + (gw.double() * dw).sum())
        assert abs(got - want) <= 1e-4 * abs(want) + 1e-6, (got, want)


# ------------------------------------------------------------------------------------------------
# routing
# ------------------------------------------------------------------------------------------------
def scores_of(logits, score):
    """Scores in 64 bits, and which experts are available."""
    z = logits.double().cpu().numpy().copy()
    low = torch.finfo(logits.dtype).min
    with np.errstate(all="ignore"):
        live = z > low
        z = np.where(live, np.minimum(z, torch.finfo(torch.float32).max), -np.inf)
        if score == "sigmoid":
            s = np.where(live, 1.0 / (1.0 + np.exp(-z)), 0.0)
        else:
            top = z.max(1, keepdims=True)
            e = np.where(live, np.exp(z - np.where(np.isfinite(top), top, 0.0)), 0.0)
            s = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
    return z, s, live


def route_of(logits, k, score, bias, groups, top_groups, group_score, renormalize, scale):
    """The definition, a token at a time."""
    z, s, live = scores_of(logits, score)
    b = None if bias is None else bias.double().cpu().numpy()
    n, experts = z.shape
    ids, weights = np.full((n, k), -1, np.int32), np.zeros((n, k))
    size = experts // groups
    for t in range(n):
        can = live[t].copy()
        key = s[t].copy()
        if b is not None:
            key = key + b
            can &= key > -np.inf
        rank = z[t] if b is None else key
        if groups > 1:
            of_groups = key if group_score == "top2" or b is not None else rank
            of_groups = np.where(can, of_groups, -np.inf).reshape(groups, size)
            best = -np.sort(-of_groups, axis=1)
            value = best[:, :2].sum(1) if group_score == "top2" else best[:, 0]
            order = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
            can &= np.isin(np.arange(experts) // size, order)
        order = sorted((e for e in range(experts) if can[e]), key=lambda e: (-rank[e], e))[:k]
        ids[t, : len(order)] = order
        if order:
            a = s[t, order]
            if renormalize and score == "sigmoid" and a.sum() < 1e-280:
                a = np.exp(z[t, order] - z[t, order].max())
            elif renormalize and score == "softmax":
                a = np.exp(z[t, order] - z[t, order].max())
            weights[t, : len(order)] = scale * (a / a.sum() if renormalize else a)
    return ids, weights, np.bincount(ids.ravel() + 1, minlength=experts + 1)[1:]


def logits_of(n, experts, dt, g, masked=True, pad=0, shift=0):
    z, buf = matrix(n, experts, dt, g, std=2.0, pad=pad, shift=shift)
    if masked and n > 2:
        z[torch.rand(n, experts, generator=g, device=DEV) < 0.1] = -math.inf
        z[1] = -math.inf  # nothing is left
        z[2] = torch.finfo(dt).min
        z[2, experts // 2] = 1.0
    return z, buf


ROUTES = [(1, 1, 1, 1, 1), (2, 2, 1, 1, 1), (40, 8, 2, 1, 1), (65, 33, 5, 1, 1), (64, 64, 8, 8, 3), (100, 160, 6, 8, 3), (31, 96, 32, 3, 2), (300, 256, 8, 8, 4), (33, 256, 8, 32, 5),
          (70, 500, 16, 5, 4), (40, 1024, 32, 1, 1), (41, 1023, 7, 31, 30), (20, 1024, 8, 2, 1), (30, 24, 3, 24, 7)]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,experts,k,groups,top_groups", ROUTES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias,group_score", [(False, "max"), (True, "max"), (True, "top2"), (False, "top2")])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route(storage, n, experts, k, groups, top_groups, score, with_bias, group_score, renormalize):
    g, dt = gen(n + experts), DT[storage]
    z, _ = logits_of(n, experts, dt, g, pad=n % 3, shift=n % 2)
    bias = torch.randn(experts, generator=g, device=DEV) * 0.1 if with_bias else None
    args = dict(score=score, bias=bias, groups=groups, top_groups=top_groups, group_score=group_score, renormalize=renormalize, scale=1.5)
    ids, weights, counts = ops.route(z, k, **args)
    want_ids, want_weights, want_counts = route_of(z, k, **args)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    assert np.array_equal(counts.cpu().numpy(), want_counts)
    # the exponent's argument is off by 2^-24 of up to 16, the exponential by two units, sums of up to 42 terms, a division
    want = torch.from_numpy(want_weights).to(DEV)
    assert_within(weights, want, 2.0**-18 * want.abs())


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [50, 3000])
def test_route_of_equal_and_nearly_equal_keys(storage, n):
    """Decisions that fp32 scores cannot make: the lowest expert of equal keys, the better one of keys that differ by less than an fp32 score's error."""
    g, dt = gen(n), DT[storage]
    experts, k = 64, 6
    flat = torch.zeros(n, experts, dtype=dt, device=DEV)
    few = torch.randint(0, 3, (n, experts), generator=g, device=DEV).to(dt)  # three values only
    bias = torch.randint(0, 2, (experts,), generator=g, device=DEV).float() * 0.25
    signed = torch.where(torch.rand(n, experts, generator=g, device=DEV) < 0.5, -0.0, 0.0).to(dt)
    near = torch.randn(n, 1, generator=g, device=DEV).expand(n, experts).contiguous().to(dt)
    tilt = torch.randint(0, 1 << 20, (experts,), generator=g, device=DEV).float() * 2.0**-40  # biases 2^-40 apart: far below a score's last place
    for z, b in ((flat, None), (flat, torch.zeros(experts, device=DEV)), (few, None), (few, bias), (signed, None), (signed, bias * 0), (near, tilt), (few, tilt)):
        for score in ("softmax", "sigmoid"):
            for groups, top_groups in ((1, 1), (8, 3)):
                args = dict(score=score, bias=b, groups=groups, top_groups=top_groups, group_score="top2", renormalize=True, scale=1.0)
                ids, _, counts = ops.route(z, k, **args)
                want = route_of(z[:60], k, **args)[0]
                assert np.array_equal(ids[:60].cpu().numpy(), want), (score, groups)
                assert int(counts.sum()) == n * k


def test_route_choices_are_those_of_64_bits():
    """Many tokens whose keys come close: every choice is that of 64-bit keys, where fp32 keys would take another in some rows."""
    g = gen(21)
    n, experts, k = 20000, 256, 8
    z = torch.randn(n, experts, generator=g, device=DEV) * 0.05
    bias = torch.randn(experts, generator=g, device=DEV) * 0.01
    for score, s in (("sigmoid", torch.sigmoid), ("softmax", lambda v: torch.softmax(v, 1))):
        ids = ops.route(z, k, score=score, bias=bias)[0].long()
        want = (s(z.double()) + bias.double()).sort(dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(ids, want), score
        narrow = (s(z) + bias).sort(dim=1, descending=True, stable=True).indices[:, :k]
        assert score == "softmax" or (narrow != want).any(), "too easy for this test to mean anything"


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_special_values(storage, score):
    dt = DT[storage]
    z = torch.randn(9, 40, generator=gen(5), device=DEV).to(dt)
    z[0, :] = math.nan
    z[1, 3], z[1, 9] = math.nan, math.inf
    z[2, 3], z[2, 9] = math.inf, math.inf
    z[3] = torch.finfo(dt).min
    z[4] = -200.0 + z[4]  # sigmoids below fp32's range
    z[5] = 200.0 + z[5]
    z[6, :38] = -math.inf
    z[7] *= 1e30
    bias = torch.zeros(40, device=DEV)
    bias[1], bias[2], bias[30] = -math.inf, math.nan, math.inf
    for b in (None, bias):
        for renormalize in (False, True):
            for groups, top in ((1, 1), (4, 2)):
                args = dict(score=score, bias=b, groups=groups, top_groups=top, group_score="max", renormalize=renormalize, scale=2.0)
                ids, weights, _ = ops.route(z, 4, **args)
                if b is None and not (score == "sigmoid" and groups > 1):
                    want_ids, want = route_of(z, 4, **args)[:2]
                    assert np.array_equal(ids.cpu().numpy(), want_ids)
                    want = torch.from_numpy(want).to(DEV)
                    assert_within(weights, want, 2.0**-15 * want.abs() + 2.0**-126)
                assert torch.isfinite(weights).all() and (ids[0] == -1).all() and (ids[3] == -1).all() and not weights[0].any()
                if b is not None:
                    assert not ((ids == 1) | (ids == 2)).any() and (ids[8, 0] == 30)
                d = ops.route_grad(z, ids, torch.randn(9, 4, device=DEV), score=score, renormalize=renormalize, scale=2.0)
                assert torch.isfinite(d).all() and not d[0].any() and not d[3].any()


def route_grad_of(logits, ids, g, score, renormalize, scale):
    """(gradient, magnitudes that its errors are relative to), as a chain of derivatives in 64 bits."""
    z, s, live = scores_of(logits, score)
    z, s, live = (torch.from_numpy(v) for v in (z, s, live))
    ids, g = ids.long().cpu(), g.double().cpu()
    n, experts = z.shape
    ok = (ids >= 0) & (ids < experts)
    at = torch.where(ok, ids, 0)
    ok &= live.gather(1, at)
    a = torch.where(ok, s.gather(1, at), 0.0)
    g = torch.where(ok, g, 0.0) * scale
    d, size = torch.zeros(n, experts, dtype=torch.float64), torch.zeros(n, experts, dtype=torch.float64)
    if renormalize:
        total = a.sum(1, keepdim=True)
        p = torch.where(total > 0, a / total.clamp(min=1e-300), 0.0)
        log_d, log_size = p * (g - (p * g).sum(1, keepdim=True)), p * (g.abs() + (p * g).abs().sum(1, keepdim=True))
    else:
        log_d, log_size = a * g, (a * g).abs()
    if score == "sigmoid":
        t = torch.where(ok, 1.0 / (1.0 + torch.exp(z.gather(1, at))), 0.0)
        d.scatter_add_(1, at, log_d * t)
        size.scatter_add_(1, at, log_size * t)
    else:
        d.scatter_add_(1, at, log_d)
        size.scatter_add_(1, at, log_size)
        if not renormalize:
            d -= s * log_d.sum(1, keepdim=True)
            size += s * log_size.sum(1, keepdim=True)
    return d.to(DEV), size.to(DEV)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,experts,k,groups,top_groups", ROUTES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_grad(storage, n, experts, k, groups, top_groups, score, renormalize):
    g, dt, u = gen(n * experts), DT[storage], U[storage]
    z, _ = logits_of(n, experts, dt, g, pad=n % 3, shift=n % 2)
    ids, _, _ = ops.route(z, k, score=score, groups=groups, top_groups=top_groups)
    gw = torch.randn(n, k, generator=g, device=DEV)
    gw[ids < 0] = math.nan  # does not matter
    out, buf = matrix(n, experts, dt, g, pad=n % 3, shift=n % 2)
    got = ops.route_grad(z, ids, gw, score=score, renormalize=renormalize, scale=1.5, out=out)
    assert got is out
    d, size = route_grad_of(z, ids, gw, score, renormalize, 1.5)
    # as the weights' errors, over two factors and a sum of 32 terms
    assert_within(got, d, 2.0**-16 * size + u * d.abs() + TINY[storage])
    outside_untouched(out, buf)
    again, _ = matrix(n, experts, dt, g, pad=n % 3, shift=n % 2)
    assert torch.equal(ops.route_grad(z, ids, gw, score=score, renormalize=renormalize, scale=1.5, out=again), got)
    # logits that do not start alike are summed in another order
    assert_within(ops.route_grad(z.clone(), ids, gw, score=score, renormalize=renormalize, scale=1.5), d, 2.0**-16 * size + u * d.abs() + TINY[storage])
    assert torch.equal(ops.route_grad(z, ids, gw, score=score, renormalize=renormalize, scale=1.5, out=z), got) and torch.equal(z, got)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_grad_of_ids_of_the_callers_own(score, renormalize):
    """Ids out of range have no part, one that a token has twice counts twice."""
    g = gen(2)
    z = torch.randn(5, 50, generator=g, device=DEV)
    ids = torch.tensor([[0, 49, 7], [3, 3, 3], [-5, 50, 1 << 30], [9, -1, 9], [-(1 << 31), (1 << 31) - 1, 2]], dtype=torch.int32, device=DEV)
    gw = torch.randn(5, 3, generator=g, device=DEV)
    got = ops.route_grad(z, ids, gw, score=score, renormalize=renormalize)
    d, size = route_grad_of(z, ids, gw, score, renormalize, 1.0)
    assert_within(got, d, 2.0**-16 * size + 2.0**-24 * d.abs())
    assert not got[2].any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_grad_is_the_difference_quotient_of_its_weights(score, renormalize):
    g = gen(31)
    z = torch.randn(20, 24, generator=g, device=DEV)
    c = torch.randn(20, 5, generator=g, device=DEV)
    ids, _, _ = ops.route(z, 5, score=score, renormalize=renormalize, scale=2.0)
    d = ops.route_grad(z, ids, c, score=score, renormalize=renormalize, scale=2.0).double()

    def loss(v):
        s = torch.softmax(v, 1) if score == "softmax" else torch.sigmoid(v)
        a = s.gather(1, ids.long())
        return float((c.double() * 2.0 * (a / a.sum(1, keepdim=True) if renormalize else a)).sum())

    h = 1e-5
    for along in (d, torch.randn(20, 24, generator=g, device=DEV).double()):
        want = (loss(z.double() + h * along) - loss(z.double() - h * along)) / (2 * h)
        assert abs(float((d * along).sum()) - want) <= 1e-4 * abs(want) + 1e-6


def test_route_without_tokens():
    z = torch.randn(0, 30, device=DEV)
    ids, weights, counts = ops.route(z, 4)
    assert ids.shape == weights.shape == (0, 4) and not counts.any() and counts.shape == (30,)
    assert ops.route_grad(z, ids, weights).shape == (0, 30)


# ------------------------------------------------------------------------------------------------
# norms and clipping
# ------------------------------------------------------------------------------------------------
def check_clip(tensors, max_norm, per_worker=False, in_place=False, out=None):
    """Norms are sums in 64 bits of squares that are fp32 sums of up to 8 (2^-21), rounded to fp32; the factor is rounded once, the product once."""
    keep = [t.double().clone() for t in tensors]
    workers = tensors[0].shape[0] if per_worker else 1
    squares = sum((k.reshape(workers, k.numel() // max(workers, 1)) ** 2).sum(1) for k in keep)
    norms = squares.sqrt() if per_worker else squares.sqrt()[0]
    got = ops.gradient_norms(tensors, per_worker=per_worker)
    assert_within(got, norms, 2.0**-21 * norms)
    if out is None:
        out = tensors if in_place else [torch.full_like(t, math.nan) for t in tensors]
    again = ops.clip_gradients(tensors, max_norm, per_worker=per_worker, out=None if in_place else out)
    assert torch.equal(again, got)
    factor = (max_norm / norms).clamp(max=1.0)
    factor = torch.where(norms <= max_norm, torch.ones_like(factor), factor)
    for t, o, k in zip(tensors, out, keep):
        f = factor.view(-1, *[1] * (k.dim() - 1)) if per_worker else factor
        u = 2.0**-8 if t.dtype == torch.bfloat16 else 2.0**-24
        assert_within(o, k * f, (2.0**-20 + u) * (k * f).abs() + TINY["bf16" if t.dtype == torch.bfloat16 else "f32"])
        if not in_place:
            assert torch.equal(t.double(), k)
        if bool((norms <= max_norm).all()):
            assert torch.equal(o.double(), k)


SHAPES = [[(1,)], [(7,), (3, 5), ()], [(1000,), (0,), (33, 65)], [(200003,), (64, 64), (1,)], [(513, 1025), (4,), (300000,)], [(40000,)] * 70, [(3,)] * 300]


@pytest.mark.parametrize("shapes", range(len(SHAPES)))
@pytest.mark.parametrize("kinds", ["f32", "bf16", "both"])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(shapes, kinds, in_place):
    g = gen(shapes)
    tensors = [torch.randn(s, generator=g, device=DEV).to(DT["f32" if kinds == "f32" or kinds == "both" and i % 2 else "bf16"]) for i, s in enumerate(SHAPES[shapes])]
    for max_norm in (1e9, 0.5, 0.0, math.inf):
        check_clip([t.clone() for t in tensors], max_norm, in_place=in_place)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("workers,rows,cols,off,pad", [(1, 3, 5, 0, 0), (5, 3, 5, 1, 2), (16, 64, 32, 8, 0), (7, 201, 301, 3, 5), (3, 1000, 128, 16, 8), (300, 8, 8, 0, 0), (0, 4, 4, 0, 0)])
def test_clip_of_workers_rows(storage, workers, rows, cols, off, pad):
    """Matrices inside the workers' rows, of a norm for each worker; what lies around them is left alone."""
    g, dt = gen(rows + cols), DT[storage]
    pitch = off + rows * cols + 77 + pad

    def buffer():
        buf = torch.full((workers, pitch), math.nan, dtype=dt, device=DEV)
        return buf, [buf[:, off:off + rows * cols].view(-1, rows, cols), buf[:, off + rows * cols:off + rows * cols + 70]]

    buf, parts = buffer()
    size = torch.exp(torch.randn(workers, generator=g, device=DEV) * 3)
    for p in parts:
        p.copy_((torch.randn(*p.shape, generator=g, device=DEV) * size.view(-1, *[1] * (p.dim() - 1))).to(dt))
    out_buf, out = buffer()
    check_clip(parts, 5.0, per_worker=True, out=out)
    keep = out_buf.clone()
    for p in buffer_parts(keep, off, rows, cols):
        p.fill_(math.nan)
    assert torch.isnan(keep).all()
    check_clip(parts, 5.0, per_worker=True, in_place=True)


def buffer_parts(buf, off, rows, cols):
    return [buf[:, off:off + rows * cols], buf[:, off + rows * cols:off + rows * cols + 70]]


def test_clip_of_other_orders_and_strides():
    g = gen(9)
    base = torch.randn(300, 500, generator=g, device=DEV)
    for make in (lambda t: t.T, lambda t: t[:, 3:203], lambda t: t[:, :200], lambda t: t[::2], lambda t: t[:, 7], lambda t: t[5:6, ::3], lambda t: t[:, :488].view(300, 8, 61)[:, 2],
                 lambda t: t[:, 1:497].view(300, 8, 62).permute(2, 0, 1), lambda t: t.view(3, 100, 500)[1], lambda t: t.view(3, 100, 500).transpose(0, 2)):
        for in_place in (False, True):
            src = base.clone()
            check_clip([make(src), torch.ones(5, device=DEV)], 3.0, in_place=in_place)
            if not in_place:
                dst = torch.zeros_like(base)
                check_clip([make(src)], 3.0, out=[make(dst)])
                rest = dst.clone()
                make(rest).zero_()
                assert not rest.any()
    wide = torch.randn(300, 504, generator=g, device=DEV)[:, :496]  # rows on boundaries to rows on boundaries, and to one row
    check_clip([wide], 3.0, out=[torch.zeros(300, 496, device=DEV)])
    check_clip([wide.bfloat16()], 3.0, out=[torch.zeros(300, 520, dtype=torch.bfloat16, device=DEV)[:, 8:504]])


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [100, 200000])
def test_clip_of_extreme_values(storage, n):
    dt = DT[storage]
    for value in (3e38, 1e30, 1e-30, 1e-38, 0.0):
        t = torch.full((n,), value, device=DEV).to(dt)
        norm = float(t[0].double()) * math.sqrt(n)
        got = float(ops.gradient_norms([t]))
        if norm > 3.4e38:
            assert got == math.inf  # of fp32; the clipping has it in 64 bits
        else:
            assert abs(got - norm) <= 2.0**-21 * norm + 2.0**-149
        if value:
            out = [torch.empty_like(t)]
            ops.clip_gradients([t], norm / 4, out=out)
            assert torch.allclose(out[0].double(), t.double() / 4, rtol=2.0**-8 if storage == "bf16" else 2.0**-20, atol=TINY[storage])
    for bad in (math.nan, math.inf, -math.inf):
        t = torch.randn(3, n, device=DEV).to(dt)
        t[1, n // 2] = bad
        keep = t.clone()
        norms = ops.clip_gradients([t], 0.1, per_worker=True)
        assert torch.equal(t[1].isfinite(), keep[1].isfinite()) and torch.equal(t[1][t[1].isfinite()], keep[1][keep[1].isfinite()]) and not torch.isfinite(norms[1])
        assert torch.isfinite(norms[[0, 2]]).all() and t[0].double().norm() < 0.101
        ops.clip_gradients([t], 0.1, per_worker=True, zero_nonfinite=True)
        assert not t[1].any() and t[2].any()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [100, 200000, 12000000])
def test_what_need_not_be_clipped_keeps_its_bits_in_place(storage, n):
    """Workers within the norm, and such with elements that are not finite, beside one that is clipped: in every form of the scaling."""
    dt, bits = (torch.float32, torch.int32) if storage == "f32" else (torch.bfloat16, torch.int16)
    t = torch.randn(3, n, generator=gen(n), device=DEV).to(dt)
    t[0] *= 1e-3 / math.sqrt(n)
    t[1, 7:9] = math.inf
    t.view(bits)[1, 11] = 0x7f812345 if storage == "f32" else 0x7f91  # a NaN of its own
    keep = t.clone()
    ops.clip_gradients([t], 0.5, per_worker=True)
    assert torch.equal(t[:2].view(bits), keep[:2].view(bits))
    assert abs(float(t[2].double().norm()) - 0.5) < 1e-2
    other = keep.clone()
    apart = torch.empty(3, n + 5, dtype=dt, device=DEV)[:, 5:]
    ops.clip_gradients([other, other.clone()], 0.5, per_worker=True, out=[other, apart])  # one in place, one not
    assert torch.equal(other[:2].view(bits), keep[:2].view(bits)) and torch.equal(apart[0], keep[0])


def test_clip_by_a_factor_below_the_range_of_floats():
    for n in (100, 300000):
        t = torch.full((n,), 2.0**120, device=DEV)
        out = [torch.empty_like(t)]
        ops.clip_gradients([t], 2.0**-30, out=out)
        assert torch.allclose(out[0].double() * math.sqrt(n), torch.full((n,), 2.0**-30, device=DEV, dtype=torch.float64), rtol=2.0**-20)


def test_clip_offsets_past_32_bits():
    """A gradient of more than 2^31 elements, its only large ones at its ends, and workers' rows as far apart."""
    n = (1 << 31) + 12345
    t = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    t[0], t[n - 1], t[1 << 31] = 3.0, 4.0, 12.0
    norm = ops.clip_gradients([t], 6.5)
    assert float(norm) == 13.0 and float(t[0]) == 1.5 and float(t[n - 1]) == 2.0 and float(t[1 << 31]) == 6.0
    rows = t[1:1 + (1 << 31)].view(2, -1)[:, :100]
    rows.fill_(1.0)
    assert torch.equal(ops.clip_gradients([rows], 5.0, per_worker=True), torch.full((2,), 10.0, device=DEV)) and (rows == 0.5).all()


# ------------------------------------------------------------------------------------------------
# streams, graphs, refusals, the operators together
# ------------------------------------------------------------------------------------------------
def step(x, w, head, z):
    """One layer forward and backward, and its gradient's clipping."""
    y, s = ops.rms_norm(x, w, residual=x)
    values, scales = ops.rms_norm_quantized(s, w, block=64)
    ids, weights, counts = ops.route(z, 4, score="sigmoid", bias=head, groups=4, top_groups=2, group_score="top2")
    dz = ops.route_grad(z, ids, weights, score="sigmoid")
    gx, gw = ops.rms_norm_grad(y, s, w, grad_sum=x)
    out = [torch.empty_like(gx), torch.empty_like(gw), torch.empty_like(dz)]
    norms = ops.clip_gradients([gx, gw, dz], 1.0, out=out)
    return [y, s, values.view(torch.uint8), ops.dequantize(values, scales), ids, weights, counts, dz, gx, gw, norms, *out]


def step_inputs(seed):
    g = gen(seed)
    return [torch.randn(*s, generator=g, device=DEV) for s in ((500, 136), (136,), (64,), (500, 64))]


def test_in_a_cuda_graph_and_on_another_stream():
    inputs = step_inputs(1)
    want = step(*inputs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*inputs)
    second = torch.cuda.CUDAGraph()
    others = step_inputs(2)
    with torch.cuda.graph(second):
        got2 = step(*others)
    for _ in range(3):
        graph.replay()
        second.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(got2, step(*others)))
    for old, new in zip(inputs, others):
        old.copy_(new)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, got2))
    # behind a slow producer, on a stream that is given
    inputs = step_inputs(1)
    s = torch.cuda.Stream()
    late = [torch.zeros_like(t) for t in inputs]
    s.wait_stream(torch.cuda.current_stream())
    slow(s)
    with torch.cuda.stream(s):
        for a, b in zip(late, inputs):
            a.copy_(b)
        got = step(*late)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_a_given_stream():
    x, w, bias, z = step_inputs(3)
    want = step(x, w, bias, z)
    s = torch.cuda.Stream()
    late = torch.zeros_like(x)
    late_z = torch.zeros_like(z)
    s.wait_stream(torch.cuda.current_stream())
    slow(s)
    with torch.cuda.stream(s):
        late.copy_(x)
        late_z.copy_(z)
    y, total = ops.rms_norm(late, w, residual=late, stream=s)
    values, scales = ops.rms_norm_quantized(total, w, block=64, stream=s)
    back = ops.dequantize(values, scales, stream=s)
    ids, weights, counts = ops.route(late_z, 4, score="sigmoid", bias=bias, groups=4, top_groups=2, group_score="top2", stream=s)
    dz = ops.route_grad(late_z, ids, weights, score="sigmoid", stream=s)
    gx, gw = ops.rms_norm_grad(y, total, w, grad_sum=late, stream=s)
    norms = ops.gradient_norms([gx, gw, dz], stream=s)
    again = ops.clip_gradients([gx, gw, dz], math.inf, stream=s)
    assert not s.query(), "too little work in front of the calls for this test to mean anything"
    s.synchronize()
    got = [y, total, values.view(torch.uint8), back, ids, weights, counts, dz, gx, gw, norms]
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(again, norms)
    del y, total, values, scales, back, ids, weights, counts, dz, gx, gw, norms, again, got


def test_two_calls_at_once():
    """The same operators on two streams at a time, each with inputs of its own."""
    inputs = [step_inputs(seed) for seed in (11, 12)]
    want = [step(*v) for v in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(step(*inputs[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for result in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(result, want[k]))


def test_route_biases_that_switch_experts_off():
    """-inf, NaN and the lowest value, in choices that fp32 makes and in those that 64 bits have to make (all logits alike)."""
    for dt in (torch.float32, torch.bfloat16):
        z = torch.randn(200, 64, generator=gen(4), device=DEV).to(dt)
        z[100:] = 0.0
        bias = 1e-12 * torch.randn(64, generator=gen(5), device=DEV)
        off = [3, 17, 40]
        bias[off[0]], bias[off[1]], bias[off[2]] = -math.inf, math.nan, torch.finfo(torch.float32).min
        for score in ("softmax", "sigmoid"):
            for groups in (1, 8):
                ids, _, counts = ops.route(z, 8, score=score, bias=bias, groups=groups, top_groups=max(groups // 2, 1), group_score="top2")
                assert not counts[off].any() and (ids >= 0).all() and int(counts.sum()) == 1600
                best = bias.nan_to_num(-1.0).clamp(min=-1.0).sort(descending=True, stable=True).indices[:8].to(torch.int32)
                assert groups > 1 or (ids[100:] == best).all()


def test_refusals_of_the_wrappers():
    x = torch.randn(10, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    v, sc = ops.rms_norm_quantized(x, block=32)
    ids, weights, _ = ops.route(x, 2)
    big = torch.randn(1, 32769, device=DEV)
    bad = [
        lambda: ops.rms_norm(x.cpu()), lambda: ops.rms_norm(x.double()), lambda: ops.rms_norm(x[0]), lambda: ops.rms_norm(x.T), lambda: ops.rms_norm(x, w[:63]),
        lambda: ops.rms_norm(x, w.bfloat16()), lambda: ops.rms_norm(x, w, residual=x[:9]), lambda: ops.rms_norm(x, w, residual=x.bfloat16()), lambda: ops.rms_norm(x, eps=-1.0),
        lambda: ops.rms_norm(x, eps=math.nan), lambda: ops.rms_norm(x, eps=1e300), lambda: ops.rms_norm(x, sum_out=x), lambda: ops.rms_norm(x, residual=x, out=x, sum_out=x),
        lambda: ops.rms_norm(x, out=x[:, :63]), lambda: ops.rms_norm(x[:, :0]), lambda: ops.rms_norm(x.clone().requires_grad_()),
        lambda: ops.rms_norm(x, torch.ones(64, device=DEV, requires_grad=True)), lambda: ops.rms_norm(None), lambda: ops.rms_norm(x[:1].expand(10, 64)),
        lambda: ops.rms_norm_quantized(x, block=16), lambda: ops.rms_norm_quantized(x, block=None), lambda: ops.rms_norm_quantized(x, block=32.0),
        lambda: ops.dequantize(x, sc), lambda: ops.dequantize(v, sc[:, :1].expand(10, 2)), lambda: ops.dequantize(v, sc.repeat(1, 3)), lambda: ops.dequantize(v, sc, torch.float16),
        lambda: ops.dequantize(v, sc, torch.float32, out=x.bfloat16()), lambda: ops.dequantize(v, sc.double()), lambda: ops.dequantize(v, sc[:9]),
        lambda: ops.rms_norm_grad(x, x[:9]), lambda: ops.rms_norm_grad(x, x, w[:3]), lambda: ops.rms_norm_grad(x, x, grad_sum=x[:, :3]), lambda: ops.rms_norm_grad(x, x, grad_x=False),
        lambda: ops.rms_norm_grad(x, x, w, grad_weight=w[:5]), lambda: ops.rms_norm_grad(x, x.bfloat16()),
        lambda: ops.route(x, 0), lambda: ops.route(x, 65), lambda: ops.route(x, 2.0), lambda: ops.route(x, 2, score="tanh"), lambda: ops.route(x, 2, score=None),
        lambda: ops.route(x, 2, group_score="mean"), lambda: ops.route(x, 2, groups=5), lambda: ops.route(x, 2, groups=0), lambda: ops.route(x, 2, groups=4, top_groups=5),
        lambda: ops.route(x, 17, groups=4, top_groups=1), lambda: ops.route(x, 2, bias=w[:5]), lambda: ops.route(x, 2, bias=w.double()), lambda: ops.route(x, 2, scale=math.nan),
        lambda: ops.route(x.half(), 2), lambda: ops.route(x.clone().requires_grad_(), 2),
        lambda: ops.route_grad(x, ids.long(), weights), lambda: ops.route_grad(x, ids, weights.double()), lambda: ops.route_grad(x, ids, weights[:, :1]),
        lambda: ops.route_grad(x, ids[:9], weights[:9]), lambda: ops.route_grad(x, ids.T, weights.T), lambda: ops.route_grad(x, ids[:, :0].contiguous(), weights[:, :0].contiguous()),
        lambda: ops.route_grad(x, ids, weights, out=x[:9]), lambda: ops.route_grad(x, ids, weights, score=3),
        lambda: ops.gradient_norms([]), lambda: ops.gradient_norms(x), lambda: ops.gradient_norms([x.cpu()]), lambda: ops.gradient_norms([x, None]), lambda: ops.gradient_norms([x.half()]),
        lambda: ops.gradient_norms([x[:1].expand(10, 64)]), lambda: ops.gradient_norms([x, w], per_worker=True), lambda: ops.gradient_norms([x[0, 0]], per_worker=True),
        lambda: ops.gradient_norms([x.view(2, 5, 64)[:, 1:4, 2:60].unflatten(2, (2, 29))[:, :, :, ::2]]),
        lambda: ops.clip_gradients([x], None), lambda: ops.clip_gradients([x], -1.0), lambda: ops.clip_gradients([x], math.nan), lambda: ops.clip_gradients([x, x], 1.0),
        lambda: ops.clip_gradients([x], 1.0, out=[x, x]), lambda: ops.clip_gradients([x], 1.0, out=x), lambda: ops.clip_gradients([x], 1.0, out=[x.bfloat16()]),
        lambda: ops.clip_gradients([x], 1.0, out=[x[:, :5]]), lambda: ops.clip_gradients([x.clone().requires_grad_()], 1.0),
        lambda: ops.clip_gradients([torch.zeros(64, 10, device=DEV).T], 1.0, out=[torch.zeros(10, 70, device=DEV)[:, :64]]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(B.A2Error) as e:
            call()
        assert e.value.code == B.A2_EINVAL, (i, str(e.value))
    for call in (lambda: ops.rms_norm(big), lambda: ops.rms_norm_grad(big, big), lambda: ops.route(torch.randn(2, 1025, device=DEV), 2), lambda: ops.route(x, 33),
                 lambda: ops.route(x, 2, groups=64, top_groups=64), lambda: ops.gradient_norms([torch.zeros(65536, 1, device=DEV)], per_worker=True)):
        with pytest.raises(B.A2Error) as e:
            call()
        assert e.value.code == B.A2_ERANGE, str(e.value)
    p = x.clone().requires_grad_()
    with torch.no_grad():
        ops.rms_norm(p)
        ops.clip_gradients([p], 1.0)
    torch.cuda.synchronize()


def test_a_backward_graph_beside_an_eager_one():
    """The gradients captured into a graph while torch has an eager graph of the same leaves alive."""
    leaf = torch.randn(40, 64, device=DEV, requires_grad=True)
    eager = (leaf * 2).sum()
    x = leaf.detach()
    w = torch.ones(64, device=DEV)
    want = ops.rms_norm_grad(x, x, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.rms_norm_grad(x, x, w)
    graph.replay()
    eager.backward()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(leaf.grad, torch.full_like(leaf, 2.0))


def reference_loss(model, row, ids, targets, scale, chosen):
    """The example's loss in torch, whose autograd gives its gradient; `chosen` are the experts that the model has taken."""
    w = model.width
    y = model.part(row, "E")[ids.long()] * math.sqrt(w)
    rms = lambda v, g: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * g  # noqa: E731
    u = rms(y, model.part(row, "N")) if model.norm else y
    if model.experts:
        s = torch.softmax(u @ model.part(row, "R").T, 1).gather(1, chosen)
        s = s / s.sum(1, keepdim=True)
        each = torch.tanh(torch.einsum("ti,eoi->teo", u, model.hidden(row)))
        a = (s[:, :, None] * each.gather(1, chosen[:, :, None].expand(-1, -1, w))).sum(1)
    else:
        a = torch.tanh(u @ model.part(row, "M").T)
    h = rms(y + a, model.part(row, "F")) if model.norm else y + a
    live = targets >= 0
    z = h @ model.part(row, "W").T
    return scale * (torch.logsumexp(z, 1) - z.gather(1, targets.long().clamp(min=0)[:, None])[:, 0])[live].sum()


@pytest.mark.parametrize("norm,experts", [(False, 0), (True, 0), (False, 5), (True, 8)])
def test_gradients_of_the_example(norm, experts):
    """Norm, routing, embedding and loss forward and backward in a model, against autograd in 64 bits."""
    from paper_2306_08289_b200 import language_model as LM

    text = LM.MarkovText(40, 4, 1)
    model = LM.Model(40, 24, norm=norm, experts=experts)
    row = torch.from_numpy(model.initial_row(5)).to(DEV)
    row += 0.05 * torch.randn(model.d, generator=gen(1), device=DEV)
    ids, targets = (torch.from_numpy(v).to(DEV) for v in text.draw(np.random.default_rng(2), 6, 11))
    out = torch.full((model.d,), math.nan, device=DEV)
    model.gradient(row, ids, targets, 0.1, out)
    chosen = None
    if experts:
        *_, kept, _, _ = model.forward(row, ids)
        chosen = kept[1].long()
    wide = row.double().requires_grad_()
    reference_loss(model, wide, ids, targets, 0.1, chosen).backward()
    want = wide.grad
    # a chain of fp32 products of up to 66 terms each: some hundred roundings of a part's own size
    for name in model.shape:
        g, d = model.part(out, name).double(), model.part(want, name)
        assert (g - d).norm() <= 1e-5 * d.norm(), name
    model.gradient(row.bfloat16(), ids, targets, 0.1, out.bfloat16())


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_rows_of_an_engine_train_a_model_with_norms_and_experts(storage):
    """The operators together as a user runs them: norms, experts and clipping in the closed loop."""
    from paper_2306_08289_b200 import language_model

    trace, entropy = language_model.train(n=4, vocab=64, width=32, T=6.0, storage=storage, sequences=4, length=16, samples=2, norm=True, experts=4, clip=1.0)
    assert len(trace) >= 3 and all(len(row) == 4 and all(math.isfinite(v) for v in row) for row in trace)
    trace, _ = language_model.train(n=4, vocab=64, width=32, T=6.0, storage=storage, sequences=4, length=16, samples=2, clip=0.5)
    assert all(len(row) == 3 and all(math.isfinite(v) for v in row) for row in trace)
    ops.check()
