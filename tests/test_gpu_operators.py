"""The language-model operators against plain implementations in 64 bits.

Tolerances are bounds derived from the arithmetic the header promises, written at each test: u = unit roundoff of the
storage type (2^-24 fp32, 2^-8 bf16), sums of k terms in fp32 at most k * 2^-23 of the sum of magnitudes (each addition rounded
or cut), operands of fp32 products kept to 22 bits."""
import ctypes as C
import math

import pytest
import torch

from paper_2306_08289_b200 import binding as B
from paper_2306_08289_b200 import operators as ops

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0**-24, "bf16": 2.0**-8}
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def matrix(rows, cols, dt, g, std=1.0, pad=0, shift=0):
    """A matrix inside a larger row: `pad` columns between rows, starting `shift` elements into the buffer. What lies around it is NaN."""
    buf = torch.full((shift + max(rows, 1) * (cols + pad) + 8,), math.nan, dtype=dt, device=DEV)
    m = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_((torch.randn(rows, cols, generator=g, device=DEV) * std).to(dt))
    return m, buf


def outside_untouched(m, buf):
    """Nothing but the matrix was written: all else in the buffer is still NaN."""
    keep = buf.clone()
    view = torch.as_strided(keep, m.shape, m.stride(), m.storage_offset())
    view.fill_(math.nan)
    assert torch.isnan(keep).all()


def assert_within(got, want, bound, name=""):
    got = got.double()
    assert got.shape == want.shape
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(((got - want).abs() / bound.clamp(min=1e-300)).nan_to_num(1e9).max()))


SHIFTS = [(0, 0), (8, 8), (3, 1)]  # (columns between rows, first element): contiguous, aligned inside a row, odd


# ------------------------------------------------------------------------------------------------
# embedding
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", [(0, 5, 8), (1, 1, 1), (1, 300, 64), (37, 11, 24), (129, 1000, 200), (1000, 257, 33), (70, 50, 2056)])
@pytest.mark.parametrize("pad,shift", SHIFTS)
def test_embed(storage, n, vocab, width, pad, shift):
    g, dt = gen(n + width), DT[storage]
    table, _ = matrix(vocab, width, dt, g, pad=pad, shift=shift)
    ids = torch.randint(-1, vocab + 1, (n,), generator=g, device=DEV, dtype=torch.int32)
    if n > 3:
        ids[0], ids[1], ids[2] = -(2**31), 2**31 - 1, vocab - 1
    out, buf = matrix(n, width, dt, g, pad=pad, shift=shift)
    ops.embed(table, ids, scale=1.7, out=out)
    live = (ids >= 0) & (ids < vocab)
    want = table.double()[ids.long().clamp(0, vocab - 1)] * 1.7 * live[:, None]
    # scale and product each rounded to fp32, the result once to the storage type
    assert_within(out, want, want.abs() * (U[storage] + 3 * 2.0**-24))
    outside_untouched(out, buf)
    assert torch.equal(ops.embed(table, ids, scale=1.7), out)


def grad_reference(dy, ids, vocab, scale):
    live = (ids >= 0) & (ids < vocab)
    at = ids[live].long()
    want = torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device=DEV).index_add_(0, at, dy[live].double())
    mags = torch.zeros_like(want).index_add_(0, at, dy[live].double().abs())
    count = torch.zeros(vocab, dtype=torch.float64, device=DEV).index_add_(0, at, torch.ones(len(at), dtype=torch.float64, device=DEV))
    return want * scale, mags * abs(scale), count


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width,kind", [
    (0, 7, 16, "uniform"), (1, 1, 1, "uniform"), (1, 700, 64, "uniform"), (31, 3, 40, "uniform"), (500, 1, 33, "uniform"),
    (511, 600, 136, "one"), (4096, 513, 64, "skewed"), (4097, 511, 24, "skewed"), (6000, 262145, 8, "skewed"), (9000, 40, 260, "one"),
    (20000, 9000, 72, "skewed"), (20000, 5, 17, "uniform"), (300, 300, 2056, "skewed"), (64, 90, 16, "none"), (8192, 3000, 24, "skewed"), (8000, 70000, 40, "uniform"), (70000, 20000, 20, "skewed"), (4096, 17000, 40, "skewed"), (2000, 257, 136, "skewed")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad(storage, n, vocab, width, kind, accumulate):
    g, dt = gen(n + vocab), DT[storage]
    pad, shift = SHIFTS[(n + width) % 3]
    dy, _ = matrix(n, width, dt, g, pad=pad, shift=shift)
    if kind == "one":
        ids = torch.full((n,), vocab - 1, dtype=torch.int32, device=DEV)
    elif kind == "none":
        ids = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    elif kind == "skewed":
        ids = (torch.rand(n, generator=g, device=DEV) ** 6 * (vocab + 1)).to(torch.int32)
    else:
        ids = torch.randint(-1, vocab + 1, (n,), generator=g, device=DEV, dtype=torch.int32)
    dead = (ids < 0) | (ids >= vocab)
    dy[dead] = math.nan  # rows of padding are not read
    out, buf = matrix(vocab, width, dt, g, pad=pad, shift=shift)
    before = out.double().clone()
    ops.embed_grad(dy, ids, vocab, scale=-0.37, out=out, accumulate=accumulate)
    want, mags, count = grad_reference(dy, ids, vocab, -0.37)
    if accumulate:
        assert torch.equal(out.double()[count == 0], before[count == 0])
        want = want + before
    else:
        assert not out[count == 0].any()
    # c fp32 additions, scale and product (and the addition to what was there) rounded, one rounding to the storage type
    assert_within(out, want, (count[:, None] + 3) * 2.0**-23 * mags + 2.0**-23 * want.abs() + U[storage] * want.abs())
    outside_untouched(out, buf)
    # the same bits again: the order of the sums is fixed
    again = before.to(dt)
    assert torch.equal(ops.embed_grad(dy, ids, vocab, scale=-0.37, out=again, accumulate=accumulate), out)


def test_embed_grad_is_the_difference_quotient_of_embed():
    """The lookup is linear in the table: <dy, embed(E + D) - embed(E)> = <embed_grad(dy), D>."""
    g = gen(5)
    table, step = (torch.randn(90, 40, generator=g, device=DEV) for _ in range(2))
    ids = torch.randint(-1, 91, (700,), generator=g, device=DEV, dtype=torch.int32)
    dy = torch.randn(700, 40, generator=g, device=DEV)
    lhs = (dy.double() * (ops.embed(table + step, ids, 2.5).double() - ops.embed(table, ids, 2.5).double())).sum()
    rhs = (ops.embed_grad(dy, ids, 90, 2.5).double() * step.double()).sum()
    # 28,000 terms of size about 2.5, each side rounded to 2^-22 of its terms
    assert abs(lhs - rhs) <= 28000 * 2.5 * 8 * 2.0**-22


# ------------------------------------------------------------------------------------------------
# vocabulary loss
# ------------------------------------------------------------------------------------------------
def loss_reference(hidden, head, targets, weights, scale):
    h, w = hidden.double(), head.double()
    vocab = w.shape[0]
    live = (targets >= 0) & (targets < vocab)
    y = targets.long().clamp(0, vocab - 1)
    z = h @ w.T
    lse = torch.logsumexp(z, 1)
    loss = torch.where(live, lse - z.gather(1, y[:, None])[:, 0], 0.0)
    p = torch.exp(z - lse[:, None])
    p[torch.arange(len(y), device=DEV), y] -= 1.0
    factor = torch.where(live, scale * (weights.double() if weights is not None else torch.ones_like(lse)), 0.0)
    P = torch.where(live[:, None], factor[:, None] * p, 0.0)
    clean = torch.where(live[:, None], h, 0.0)
    return factor, lse, loss, P, P @ w, P.T @ clean, clean, live


def loss_bounds(hidden, head, targets, g, lse, P, clean, live, storage):
    """Elementwise bounds on loss, lse and both gradients."""
    h, w = clean.abs(), head.double().abs()
    width, vocab, n = h.shape[1], w.shape[0], h.shape[0]
    words = 2.0**-21 if storage == "f32" else 0.0  # two operands of 22 bits
    tz = ((hidden.double().abs() @ w.T).amax(1) * (words + width * 2.0**-23)) if n else lse
    depth = 256 + vocab / 256 + 16  # additions in a row: inside a tile, then over the tiles
    tl = tz + depth * 2.0**-23 + 2.0**-22 * lse.abs()
    loss_tol = tz + tl + 2.0**-22 * (lse.abs() + tz)
    # P: the exponential of a difference known to tz + tl, then one rounding (bf16, or 22 bits with fp32 rows)
    rel = torch.expm1(tz + tl) + 2.0**-20
    at_target = torch.arange(vocab, device=DEV)[None, :] == targets.long()[:, None]
    round_p = 2.0**-8 if storage == "bf16" else 2.0**-21
    grown = torch.where(live[:, None], P.abs() * (rel[:, None] + round_p + words), 0.0)
    # the target's p - 1 cancels: its error is that of p, at most |g| rel
    grown = grown + torch.where(at_target, (g.abs() * rel)[:, None], 0.0)
    ub = U[storage]
    th = grown @ w + (vocab + 64) * 2.0**-23 * (P.abs() @ w) + ub * (P @ head.double()).abs()
    tw = grown.T @ h + (n + 64) * 2.0**-23 * (P.abs().T @ h) + ub * (P.T @ clean).abs()
    return loss_tol, tl, th, tw


SIZES = [(1, 8, 5), (1, 64, 1), (3, 1, 17), (5, 16, 257), (33, 40, 256), (128, 64, 129), (129, 201, 1003), (200, 72, 5003), (260, 328, 511),
         (64, 24, 9000), (700, 520, 1300), (513, 88, 5000)]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,width,vocab", SIZES)
@pytest.mark.parametrize("weighted", [False, True])
def test_vocab_loss_and_gradients(storage, n, width, vocab, weighted):
    g, dt = gen(n * 7 + vocab), DT[storage]
    pad, shift = SHIFTS[(n + vocab) % 3]
    hidden, _ = matrix(n, width, dt, g, pad=pad, shift=shift)
    head, _ = matrix(vocab, width, dt, g, std=2.0 / math.sqrt(width), pad=pad, shift=shift)
    targets = torch.randint(-1, vocab + 1, (n,), generator=g, device=DEV, dtype=torch.int32)
    weights = torch.randn(n, generator=g, device=DEV) if weighted else None
    scale = 0.013
    factor, lse, loss, P, dh, dw, clean, live = loss_reference(hidden, head, targets, weights, scale)
    t_loss, t_lse, t_h, t_w = loss_bounds(hidden, head, targets, factor, lse, P, clean, live, storage)
    got_loss, got_lse = ops.vocab_loss(hidden, head, targets)
    assert_within(got_loss, loss, t_loss, "loss")
    assert_within(got_lse, lse, t_lse, "lse")
    assert not got_loss[~live].any()
    gh, bh = matrix(n, width, dt, g, pad=pad, shift=shift)
    gw, bw = matrix(vocab, width, dt, g, pad=pad, shift=shift)
    l2, s2, _, _ = ops.vocab_loss_grad(hidden, head, targets, weights=weights, scale=scale, grad_hidden=gh, grad_head=gw)
    assert torch.equal(l2, got_loss) and torch.equal(s2, got_lse)
    assert_within(gh, dh, t_h, "grad_hidden")
    assert_within(gw, dw, t_w, "grad_head")
    assert not gh[~live].any()
    outside_untouched(gh, bh)
    outside_untouched(gw, bw)
    # either gradient alone gives the same bits
    _, _, only_h, none = ops.vocab_loss_grad(hidden, head, targets, weights=weights, scale=scale, grad_head=None)
    assert none is None and torch.equal(only_h, gh)
    _, _, none, only_w = ops.vocab_loss_grad(hidden, head, targets, weights=weights, scale=scale, grad_hidden=None)
    assert none is None and torch.equal(only_w, gw)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("storage,n,width,vocab", [("f32", 100, 16, 163841), ("f32", 64, 72, 200064), ("f32", 1, 768, 200064), ("bf16", 25, 264, 327681),
                                                   ("bf16", 16, 64, 400003), ("bf16", 1, 300, 262144)])
def test_few_tokens_of_a_large_vocabulary(storage, n, width, vocab, weighted):
    """Kept logits whose P is longer than a piece of large problems would be."""
    test_vocab_loss_and_gradients(storage, n, width, vocab, weighted)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_vocab_loss_edges(storage):
    g, dt = gen(1), DT[storage]
    head = (torch.randn(300, 48, generator=g, device=DEV)).to(dt)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    loss, lse, gh, gw = ops.vocab_loss_grad(head[:0], head, none)
    assert loss.shape == lse.shape == (0,) and gh.shape == (0, 48) and not gw.any()
    # no token has a target: no loss, no gradient, and what the hidden rows and weights hold does not matter
    hidden = (torch.randn(70, 48, generator=g, device=DEV)).to(dt)
    hidden[3], hidden[4] = math.nan, math.inf
    off = torch.full((70,), -1, dtype=torch.int32, device=DEV)
    weights = torch.full((70,), math.nan, device=DEV)
    loss, lse, gh, gw = ops.vocab_loss_grad(hidden, head, off, weights=weights)
    assert not loss.any() and not gh.any() and not gw.any()
    fine = torch.ones(70, dtype=torch.bool, device=DEV)
    fine[3:5] = False
    want = torch.logsumexp(hidden[fine].double() @ head.double().T, 1)
    assert (lse[fine].double() - want).abs().max() < 1e-3 and not torch.isfinite(lse[~fine]).any()
    # such rows among live ones leave the others alone
    on = torch.randint(0, 300, (70,), generator=g, device=DEV, dtype=torch.int32)
    some = torch.where(fine, on, -1).to(torch.int32)
    a = ops.vocab_loss_grad(hidden, head, some, scale=0.5)
    zeroed = torch.where(fine[:, None], hidden, torch.zeros_like(hidden))
    b = ops.vocab_loss_grad(zeroed, head, some, scale=0.5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,width,vocab", [(70, 48, 300), (700, 264, 2000)])
def test_rows_without_a_target_do_not_weigh_on_the_others(storage, n, width, vocab):
    """Finite garbage of any size in rows without a target: the other rows keep every bit, and the garbage rows have their own lse."""
    g, dt = gen(n), DT[storage]
    hidden = torch.randn(n, width, generator=g, device=DEV).to(dt)
    head = (torch.randn(vocab, width, generator=g, device=DEV) / math.sqrt(width)).to(dt)
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV, dtype=torch.int32)
    off = torch.arange(n, device=DEV) % 5 == 2
    targets[off] = -1
    a = ops.vocab_loss_grad(torch.where(off[:, None], 0.0, hidden).to(dt), head, targets, scale=0.5)
    garbage = hidden * torch.exp2(torch.randint(-60, 90, (n, 1), generator=g, device=DEV).float()).to(dt)
    b = ops.vocab_loss_grad(torch.where(off[:, None], garbage, hidden), head, targets, scale=0.5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and torch.equal(a[3], b[3]) and torch.equal(a[1][~off], b[1][~off])
    z = garbage[off].double() @ head.double().T
    tol = (garbage[off].double().abs() @ head.double().abs().T).amax(1) * (2.0**-21 + width * 2.0**-23) + 2.0**-14
    assert ((b[1][off].double() - torch.logsumexp(z, 1)).abs() <= tol).all()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_vocab_loss_extreme_logits(storage):
    """Logits in the thousands, equal logits, and sizes far from one on either side."""
    dt = DT[storage]
    head = torch.zeros(130, 8, dtype=dt, device=DEV)
    head[:, 0] = torch.arange(130, device=DEV).to(dt)
    hidden = torch.zeros(4, 8, dtype=dt, device=DEV)
    hidden[0, 0], hidden[1, 0], hidden[2, 0] = 64.0, -64.0, 0.0
    hidden[3, 0] = 2.0**-40
    targets = torch.tensor([0, 0, 7, 9], dtype=torch.int32, device=DEV)
    loss, lse, gh, gw = ops.vocab_loss_grad(hidden, head, targets)
    # all products are exact; log(130) and the exponentials are good to a few units
    want = torch.tensor([64.0 * 129, 0.0, math.log(130), math.log(130)], dtype=torch.float64, device=DEV)
    assert ((lse.double() - want).abs() <= 2.0**-22 * (want.abs() + 4)).all()
    z_t = torch.tensor([0.0, 0.0, 0.0, 0.0], dtype=torch.float64, device=DEV)
    assert ((loss.double() - (want - z_t)).abs() <= 2.0**-22 * (want.abs() + 4)).all()
    assert torch.isfinite(gh).all() and torch.isfinite(gw).all()
    # the second token's loss is e^-64 from zero: its gradient is that small too, up to the rounding of P's largest element
    assert float(gh[0, 0]) == 129.0 and float(gh[1].abs().max()) <= 129 * (math.exp(-64) + 2.0**-30)
    # tiny and huge storage values: only their products matter
    g = gen(2)
    h, w = torch.randn(40, 56, generator=g, device=DEV), torch.randn(90, 56, generator=g, device=DEV) / 7
    t = torch.randint(0, 90, (40,), generator=g, device=DEV, dtype=torch.int32)
    a = ops.vocab_loss_grad(h.to(dt), w.to(dt), t)
    b = ops.vocab_loss_grad((h.to(dt) * 2.0**60), (w.to(dt) * 2.0**-60), t)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(a[2], b[2] * 2.0**60) and torch.equal(a[3], b[3] * 2.0**-60)


# A size of every form that the library picks by (tokens, width, vocabulary): without tensor cores; logits kept; kept, with few tiles and a long sum
# over the tokens; made again for a P of the whole vocabulary; made again piece by piece, the last piece shorter
FORMS = {"few": (70, 48, 300), "kept": (700, 264, 2000), "kept, long sums": (5000, 72, 600), "again": (1100, 72, 17003), "pieces": (2600, 136, 32003)}


def loss_case(storage, form, seed=0):
    n, width, vocab = FORMS[form]
    g, dt = gen(n + seed), DT[storage]
    hidden = torch.randn(n, width, generator=g, device=DEV).to(dt)
    head = (torch.randn(vocab, width, generator=g, device=DEV) / math.sqrt(width)).to(dt)
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV, dtype=torch.int32)
    return g, dt, hidden, head, targets


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS)[1:])
@pytest.mark.parametrize("weighted", [False, True])
def test_vocab_loss_and_gradients_of_every_form(storage, form, weighted):
    test_vocab_loss_and_gradients(storage, *FORMS[form], weighted)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
def test_masked_rows_that_are_not_finite(storage, form):
    """NaN and infinity in hidden rows and weights without a target: no loss, no gradient, and every bit of the other tokens as if the rows were zero."""
    g, dt, hidden, head, targets = loss_case(storage, form)
    n = len(hidden)
    off = torch.arange(n, device=DEV) % 7 == 3
    weights = torch.rand(n, generator=g, device=DEV)
    some = torch.where(off, -1, targets).to(torch.int32)
    zeroed = torch.where(off[:, None], torch.zeros_like(hidden), hidden)
    want = ops.vocab_loss_grad(zeroed, head, some, weights=torch.where(off, 0.0, weights), scale=0.5)
    hidden[off, 0] = math.nan
    hidden[off, 5] = math.inf
    hidden[off, 6] = -math.inf
    got = ops.vocab_loss_grad(hidden, head, some, weights=torch.where(off, math.nan, weights), scale=0.5)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])
    assert torch.equal(got[1][~off], want[1][~off]) and not torch.isfinite(got[1][off]).any()
    assert not got[0][off].any() and not got[2][off].any()
    none = torch.full_like(targets, 2**31 - 1)
    loss, lse, gh, gw = ops.vocab_loss_grad(hidden, head, none, weights=torch.full((n,), math.inf, device=DEV))
    assert not loss.any() and not gh.any() and not gw.any()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
def test_tokens_without_a_target_have_zero_rows_whatever_the_head_holds(storage, form):
    _, _, hidden, head, targets = loss_case(storage, form)
    head[11, 3], head[-1, 0] = math.nan, math.inf
    off = torch.arange(len(hidden), device=DEV) % 3 == 1
    loss, lse, gh, gw = ops.vocab_loss_grad(hidden, head, torch.where(off, -5, targets).to(torch.int32))
    assert not loss[off].any() and not gh[off].any()
    assert not torch.isfinite(loss[~off]).any()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
def test_only_the_products_of_sizes_matter(storage, form):
    _, _, hidden, head, targets = loss_case(storage, form)
    a = ops.vocab_loss_grad(hidden, head, targets)
    b = ops.vocab_loss_grad(hidden * 2.0**60, head * 2.0**-60, targets)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(a[2], b[2] * 2.0**60) and torch.equal(a[3], b[3] * 2.0**-60)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
def test_logits_in_the_thousands(storage, form):
    n, width, vocab = FORMS[form]
    dt = DT[storage]
    head = torch.zeros(vocab, width, dtype=dt, device=DEV)
    head[:, 0] = (torch.arange(vocab, device=DEV) % 128).to(dt)
    hidden = torch.zeros(n, width, dtype=dt, device=DEV)
    sizes = torch.tensor([64.0, -64.0, 0.0, 2.0**-40], device=DEV)
    hidden[:, 0] = sizes[torch.arange(n, device=DEV) % 4].to(dt)
    targets = ((torch.arange(n, device=DEV) * 13) % vocab).to(torch.int32)
    loss, lse, gh, gw = ops.vocab_loss_grad(hidden, head, targets, scale=1.0 / n)
    z = hidden[:, :1].double() * head[:, 0].double()[None]
    want = torch.logsumexp(z, 1)
    # products are exact; the logarithm, the exponentials and their sums (of up to `depth` terms in a row) are good to some units
    depth = 256 + vocab / 256 + 16
    tol = depth * 2.0**-23 + 2.0**-22 * (want.abs() + 4)
    assert ((lse.double() - want).abs() <= tol).all()
    at = z.gather(1, targets.long()[:, None])[:, 0]
    assert ((loss.double() - (want - at)).abs() <= tol + 2.0**-23 * (want - at).abs()).all()
    assert torch.isfinite(gh).all() and torch.isfinite(gw).all()
    p = torch.exp(z - want[:, None])
    p[torch.arange(n, device=DEV), targets.long()] -= 1.0
    slope = (p @ head[:, 0].double()) / n
    # of the first column: sums of numbers up to 127 that P's rounding and the exponentials' error (that of lse) leave good to this, and the result's
    # rounding
    rel = 2.0**-8 if storage == "bf16" else 2.0**-18
    mags = (p.abs() @ head[:, 0].double()) / n
    assert ((gh[:, 0].double() - slope).abs() <= (rel + torch.expm1(2 * tol)) * mags + 127 * 2.0**-30 / n + U[storage] * slope.abs()).all()


def test_vocab_loss_gradients_are_difference_quotients():
    """Central differences of the operator's own loss along random directions, 32-bit rows."""
    g = gen(9)
    n, width, vocab = 60, 40, 333
    hidden = torch.randn(n, width, generator=g, device=DEV)
    head = torch.randn(vocab, width, generator=g, device=DEV) / math.sqrt(width)
    targets = torch.randint(-1, vocab, (n,), generator=g, device=DEV, dtype=torch.int32)
    weights = torch.rand(n, generator=g, device=DEV)
    _, _, gh, gw = ops.vocab_loss_grad(hidden, head, targets, weights=weights, scale=0.7)

    def value(h, w):
        return float((0.7 * weights.double() * ops.vocab_loss(h, w, targets)[0].double()).sum())

    for grad, base, other in ((gh, hidden, "h"), (gw, head, "w")):
        d = torch.randn(base.shape, generator=g, device=DEV)
        d /= d.norm()
        eps = 2.0**-3
        f = (lambda x: value(x, head)) if other == "h" else (lambda x: value(hidden, x))
        quotient = (f(base + eps * d) - f(base - eps * d)) / (2 * eps)
        slope = float((grad.double() * d.double()).sum())
        # a unit step moves the logits by at most about |other matrix|; third derivatives of log-sum-exp are below the cube of that move
        move = float(torch.linalg.matrix_norm((head if other == "h" else hidden).double(), 2))
        cut = 0.7 * move**3 * eps**2 / 6
        noise = 60 * 2.0**-20 / eps
        assert abs(quotient - slope) <= cut + noise, (other, quotient, slope, cut, noise)


def check_gradients(hidden, head, targets, weights, scale, storage):
    factor, lse, loss, P, dh, dw, clean, live = loss_reference(hidden, head, targets, weights, scale)
    t_loss, t_lse, t_h, t_w = loss_bounds(hidden, head, targets, factor, lse, P, clean, live, storage)
    got = ops.vocab_loss_grad(hidden, head, targets, weights=weights, scale=scale)
    for name, value, want, tol in zip(("loss", "lse", "grad_hidden", "grad_head"), got, (loss, lse, dh, dw), (t_loss, t_lse, t_h, t_w)):
        assert_within(value, want, tol, name)


@pytest.mark.parametrize("vocab", [1, 3])
def test_long_rows_of_small_losses_are_summed_in_parts(vocab):
    """fp32 rows without tensor cores: 65,536 equal terms, where one chain of additions rounds each to the size of the whole sum. Parts of 128 leave chains
    of 128 and of 512 additions, each good to 2^-24 of the sum."""
    width = 65536
    for h in (0.1, 0.37, 0.713, 1.9):
        hidden = torch.full((2, width), h, device=DEV)
        head = torch.full((vocab, width), 0.1 / 1280, device=DEV) * (1 + torch.arange(vocab, device=DEV)[:, None] / 7)
        lse = ops.vocab_loss(hidden, head, torch.zeros(2, dtype=torch.int32, device=DEV))[1]
        z = hidden.double() @ head.double().T
        tol = (128 + width / 128 + 8) * 2.0**-24 * z.amax() + 2.0**-21
        assert ((lse.double() - torch.logsumexp(z, 1)).abs() <= tol).all()


@pytest.mark.parametrize("n,width,vocab", [(2000, 1753, 356), (2000, 1024, 5003), (300, 512, 300), (256, 1024, 50003), (2500, 768, 9000), (64, 768, 20000)])
def test_the_bf16_loss_is_as_exact_as_fp32(n, width, vocab):
    """Products of bf16 values are exact in fp32, so loss and lse of bf16 rows may be as far from 64 bits as twice what the same logits in fp32 leave (root
    mean square over the tokens; hidden states that lean towards their target, as in training)."""
    g = gen(width)
    head = (torch.randn(vocab, width, generator=g, device=DEV) / math.sqrt(width)).bfloat16()
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV, dtype=torch.int32)
    lean = 8.0 * torch.rand(n, 1, generator=g, device=DEV)
    hidden = (torch.randn(n, width, generator=g, device=DEV) + lean * head[targets.long()].float()).bfloat16()
    got = ops.vocab_loss(hidden, head, targets)

    def form(h, w):
        z = h @ w.T
        lse = torch.logsumexp(z, 1)
        return lse - z.gather(1, targets.long()[:, None])[:, 0], lse

    for name, here, plain, want in zip(("loss", "lse"), got, form(hidden.float(), head.float()), form(hidden.double(), head.double())):
        err, may = (float((x.double() - want).square().mean().sqrt()) for x in (here, plain))
        assert err <= 2.0 * may, (name, err, may)


@pytest.mark.parametrize("form", list(FORMS))
def test_small_probabilities_keep_their_digits(form):
    """A trained model's tokens: what the vocabulary rows that no token names get is a sum of P of 2^-32 and less, to the same relative bound."""
    g, _, hidden, head, targets = loss_case("f32", form, 7)
    hidden = 22.0 * head[targets.long()] / head[targets.long()].square().sum(1, keepdim=True) + 0.3 * hidden
    few = torch.randperm(len(hidden), generator=g, device=DEV)[:8]
    on = torch.full_like(targets, -1)
    on[few] = targets[few]
    check_gradients(hidden, head, on, None, 1.0, "f32")


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("of", ["hidden", "head", "weights"])
def test_a_large_row_leaves_the_others_their_digits(form, of):
    g, _, hidden, head, targets = loss_case("f32", form, 8)
    weights = torch.rand(len(hidden), generator=g, device=DEV) + 0.5
    if of == "hidden":
        hidden[7, -1], head[:, -1] = 2.0**30, 0.0
    elif of == "head":
        head[9, 0], hidden[:, 0] = -(2.0**30), 0.0
    else:
        weights[3::2] *= 2.0**-14
    check_gradients(hidden, head, targets, weights, 1.0, "f32")


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("of", ["hidden", "head"])
def test_gradients_against_differences_along_themselves(form, of):
    """The operator's own loss along the normalised gradient, where its slope is largest: the gradient's norm. Two steps and Richardson's
    extrapolation; what the quotient may be off is a fiftieth of the slope, so a missing or turned gradient cannot pass."""
    g, _, hidden, head, targets = loss_case("f32", form, 3)
    n = len(hidden)
    targets[::9] = -1
    weights = torch.rand(n, generator=g, device=DEV)
    out = ops.vocab_loss_grad(hidden, head, targets, weights=weights, scale=0.7)
    grad, base = (out[2], hidden) if of == "hidden" else (out[3], head)
    slope = float(grad.double().norm())
    d = (grad.double() / slope).float()

    def value(x):
        h, w = (x, head) if of == "hidden" else (hidden, x)
        return float((0.7 * weights.double() * ops.vocab_loss(h, w, targets)[0].double()).sum())

    def quotient(eps):
        return (value(base + eps * d) - value(base - eps * d)) / (2 * eps)

    # a unit step moves token t's logits by at most m_t = |direction's share of it| |the other matrix|; the fifth derivative of its log-sum-exp is
    # below 16 m_t^5 (cumulants of a variable within +-m_t). With steps e and e / 2 the extrapolation leaves e^4 / 480 of it at most.
    eps = 2.0**-3
    if of == "hidden":
        move = d.double().norm(dim=1) * float(head.double().norm(dim=1).max())
    else:
        move = hidden.double().norm(dim=1) * float(d.double().norm(dim=1).max())
    cut = float((0.7 * weights.double() * 16 * move**5).sum()) * eps**4 / 480
    # every loss is good to 2^-20 of the logits' sizes, the errors of the tokens add up at worst
    noise = 0.7 * n * 2.0**-20 / (eps / 2) * 5 / 3
    got = (4 * quotient(eps / 2) - quotient(eps)) / 3
    assert abs(got - slope) <= min(slope / 50, cut + noise), (got, slope, cut, noise)


# ------------------------------------------------------------------------------------------------
# orthogonalisation
# ------------------------------------------------------------------------------------------------
def words(x, storage):
    """What the operator keeps of an intermediate: 22 bits with fp32 rows, 11 with bf16 rows."""
    mantissa, exponent = torch.frexp(x)
    bits = 22 if storage == "f32" else 11
    return torch.ldexp(torch.round(mantissa * 2.0**bits) / 2.0**bits, exponent)


def newton_schulz(g, steps, coeffs, eps, keep=lambda v: v, cut=0.0):
    """In 64 bits; `keep` rounds the intermediates, `cut` is the relative loss of a product's sums."""
    a, b, c = coeffs
    turn = g.shape[1] > g.shape[2]
    x = g.double().transpose(1, 2) if turn else g.double()
    norm = torch.linalg.matrix_norm(x, keepdim=True) + eps
    x = torch.where(norm > 0, x / norm, 0.0)
    for _ in range(steps):
        s = keep((x @ x.transpose(1, 2)) * (1 - cut))
        p = keep(b * s + c * (s @ s) * (1 - cut))
        x = keep(a * x + p @ x * (1 - cut))
    return x.transpose(1, 2) if turn else x


def check_orthogonalize(mats, got, storage, steps=5, coeffs=ops.NEWTON_SCHULZ, eps=1e-7, scale=1.0):
    want = newton_schulz(mats, steps, coeffs, eps) * scale
    k = max(mats.shape[1:])
    # every addition of a sum may be cut instead of rounded: 2^-23 a step of 16 products, at most k / 16 + 16 steps
    model = newton_schulz(mats, steps, coeffs, eps, lambda v: words(v, storage), (k / 16 + 16) * 2.0**-23) * scale
    norm = torch.linalg.matrix_norm(want)
    # four times what the model of the roundings loses, and the storage type's rounding
    tol = 4 * torch.linalg.matrix_norm(model - want) + (U[storage] + 2.0**-22) * norm
    err = torch.linalg.matrix_norm(got.double() - want)
    assert (err <= tol).all(), (err / norm, tol / norm)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("mats,rows,cols", [(1, 1, 1), (2, 1, 40), (2, 40, 1), (3, 8, 8), (2, 17, 33), (5, 64, 64), (2, 100, 65), (2, 128, 128),
                                            (2, 129, 140), (3, 256, 200), (1, 300, 1000), (2, 513, 257), (1, 640, 640), (2, 21, 1030), (3, 2577, 19), (2, 97, 282), (1, 128, 4096),
                                            (2, 4000, 128), (1, 40, 4500), (5, 200, 700)])
def test_orthogonalize(storage, mats, rows, cols):
    g, dt = gen(rows * 3 + cols), DT[storage]
    pad, shift = SHIFTS[(rows + cols) % 3]
    pitch, gap = cols + pad, pad * 5
    stride = rows * pitch + gap
    buf = torch.full((shift + mats * stride,), math.nan, dtype=dt, device=DEV)
    x = torch.as_strided(buf, (mats, rows, cols), (stride, pitch, 1), shift)
    sizes = torch.exp(3 * torch.randn(mats, 1, 1, generator=g, device=DEV))  # workers differ in size
    x.copy_((torch.randn(mats, rows, cols, generator=g, device=DEV) * sizes).to(dt))
    before = buf.clone()
    got = ops.orthogonalize(x, scale=0.7)
    assert torch.equal(buf.view(torch.int16 if storage == "bf16" else torch.int32), before.view(torch.int16 if storage == "bf16" else torch.int32))
    check_orthogonalize(x, got, storage, scale=0.7)
    # in place, inside the rows it came from; nothing around the matrices is written
    ops.orthogonalize(x, scale=0.7, out=x)
    assert torch.equal(x, got)
    x.fill_(math.nan)
    assert torch.isnan(buf).all()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_orthogonalize_steps_coefficients_and_empty(storage):
    g, dt = gen(4), DT[storage]
    x = torch.randn(3, 90, 150, generator=g, device=DEV).to(dt)
    for steps, coeffs in ((0, ops.NEWTON_SCHULZ), (1, (2.0, -1.5, 0.5)), (8, (15 / 8, -10 / 8, 3 / 8))):
        check_orthogonalize(x, ops.orthogonalize(x, steps=steps, coeffs=coeffs), storage, steps, coeffs)
    assert ops.orthogonalize(x[:0]).shape == (0, 90, 150)
    assert torch.equal(ops.orthogonalize(x[1]), ops.orthogonalize(x)[1])


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(40, 40), (300, 200)])
def test_orthogonalize_special_values(storage, rows, cols):
    """Zero matrices, tiny and huge ones (their squares leave fp32), a matrix with a NaN or infinity: each matrix of the batch on its own."""
    g, dt = gen(8), DT[storage]
    base = torch.randn(rows, cols, generator=g, device=DEV).to(dt)
    x = torch.stack([base, torch.zeros_like(base), base * 2.0**-90, base * 2.0**90, base, base])
    x[4, 3, 5] = math.nan
    x[5, 0, 0] = math.inf
    got = ops.orthogonalize(x, eps=0.0)
    assert not got[1].any()
    for k in (0, 2, 3):  # powers of two change nothing
        assert torch.equal(got[k], got[0]), k
    check_orthogonalize(x[:1], got[:1], storage, eps=0.0)
    assert torch.isnan(got[4]).all() and torch.isnan(got[5]).all()
    with_eps = ops.orthogonalize(x[1:3], eps=1e-7)
    assert not with_eps[0].any()
    check_orthogonalize(x[2:3], with_eps[1:2], storage, eps=1e-7)
    # a rank-one matrix has one singular value to push: the polynomial of one, five times
    u, v = torch.randn(rows, 1, generator=g, device=DEV), torch.randn(1, cols, generator=g, device=DEV)
    check_orthogonalize((u @ v)[None].to(dt), ops.orthogonalize((u @ v)[None].to(dt)), storage)


@pytest.mark.parametrize("mats,rows,cols", [(1, 152, 890), (5, 130, 348), (3, 246, 135), (2, 371, 136), (2, 1001, 512)])
def test_orthogonalize_is_as_exact_as_fp32_up_to_the_words(mats, rows, cols):
    """fp32 rows, matrices like momenta (a few common directions over noise): two words an operand have twice fp32's unit roundoff, so the error may be twice
    that of the same products in fp32."""
    g = gen(rows)
    r = min(rows, cols) // 8
    x = torch.randn(mats, rows, r, generator=g, device=DEV) @ torch.randn(mats, r, cols, generator=g, device=DEV) / math.sqrt(r)
    x = x + torch.randn(mats, rows, cols, generator=g, device=DEV)
    want = newton_schulz(x, 5, ops.NEWTON_SCHULZ, 1e-7)
    y = x.transpose(1, 2) if rows > cols else x
    y = y / (torch.linalg.matrix_norm(y, keepdim=True) + 1e-7)
    a, b, c = ops.NEWTON_SCHULZ
    for _ in range(5):
        s = y @ y.transpose(1, 2)
        y = a * y + (b * s + c * (s @ s)) @ y
    y = y.transpose(1, 2) if rows > cols else y
    plain = float((y.double() - want).norm() / want.norm())
    err = float((ops.orthogonalize(x).double() - want).norm() / want.norm())
    assert err <= 2.0 * plain, (err, plain)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(40, 40), (70, 900), (300, 200)])
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_orthogonalize_where_eps_outweighs_the_matrix(storage, rows, cols, steps):
    """X0 = G / (|G| + eps) far below the smallest float: the caller's scale brings the result back, with all its bits."""
    g, dt = gen(12), DT[storage]
    base = torch.randn(2, rows, cols, generator=g, device=DEV)
    base[1] *= 2.0**-30  # another size in the same batch
    x = (base * 2.0**-60).to(dt)
    got = ops.orthogonalize(x, steps=steps, eps=1e30, scale=2.0**110)
    check_orthogonalize(x, got, storage, steps=steps, eps=1e30, scale=2.0**110)
    # without it the result is nothing
    assert not ops.orthogonalize(x, steps=steps, eps=1e38 * 1e60).any()
    # subnormal rows: G (a^steps) to a unit of the smallest float or the words' 2^-20
    x = (base * 2.0**-135).to(dt)
    got = ops.orthogonalize(x, steps=steps, eps=1.0, scale=1.0)
    want = newton_schulz(x, steps, ops.NEWTON_SCHULZ, 1.0)
    rel = 2.0**-20 if storage == "f32" else 2.0**-6
    assert ((got.double() - want).abs() <= rel * want.abs().amax(dim=(1, 2), keepdim=True) + (2.0**-148 if storage == "f32" else 2.0**-132)).all()


# ------------------------------------------------------------------------------------------------
# streams, refusals, the operators together
# ------------------------------------------------------------------------------------------------
def test_operators_on_another_stream():
    """Queued behind a slow producer on the given stream, with the results read there."""
    g = gen(6)
    s = torch.cuda.Stream()
    big = torch.randn(4096, 4096, generator=g, device=DEV)
    table = torch.randn(800, 64, generator=g, device=DEV)
    ids = torch.randint(0, 800, (3000,), generator=g, device=DEV, dtype=torch.int32)
    want_y = ops.embed(table, ids)
    want_e = ops.embed_grad(want_y, ids, 800)
    want_l = ops.vocab_loss_grad(want_y, table, ids)
    want_o = ops.orthogonalize(table)
    late = torch.zeros_like(table)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(20):
            big = big @ big * 1e-4
        late.copy_(table)
    y = ops.embed(late, ids, stream=s)
    e = ops.embed_grad(y, ids, 800, stream=s)
    l = ops.vocab_loss_grad(y, late, ids, stream=s)
    o = ops.orthogonalize(late, stream=s)
    s.synchronize()
    assert torch.equal(y, want_y) and torch.equal(e, want_e) and torch.equal(o, want_o)
    assert all(torch.equal(a, b) for a, b in zip(l, want_l))


def test_refusals_of_arguments_of_another_kind():
    t = torch.randn(10, 8, device=DEV)
    ids = torch.zeros(10, dtype=torch.int32, device=DEV)
    for call, code in ((lambda: ops.embed(t, [0, 1]), B.A2_EINVAL), (lambda: ops.embed(t, None), B.A2_EINVAL), (lambda: ops.embed_grad(t, ids, -1), B.A2_EINVAL),
                       (lambda: ops.embed_grad(t, ids, 10.5), B.A2_EINVAL), (lambda: ops.embed_grad(t, ids, 1 << 40), B.A2_ERANGE),
                       (lambda: ops.vocab_loss_grad(t, t, ids, grad_head=False), B.A2_EINVAL), (lambda: ops.orthogonalize(t, coeffs=(1.0, -0.5)), B.A2_EINVAL),
                       (lambda: ops.orthogonalize(t, out=t.tolist()), B.A2_EINVAL), (lambda: ops.orthogonalize(t, out=t[None]), B.A2_EINVAL)):
        with pytest.raises(B.A2Error) as e:
            call()
        assert e.value.code == code, str(e.value)


def slow(stream):
    with torch.cuda.stream(stream):
        big = torch.ones(4096, 4096, device=DEV)
        for _ in range(40):
            big = big @ big * 1e-4


def test_memory_of_a_call_on_another_stream_is_not_handed_out_too_early():
    """Tensors that the caller drops right after a call on another stream, and results dropped while the caller's own stream still reads them."""
    s = torch.cuda.Stream()
    n, width, vocab = 4099, 136, 701
    ids = torch.randint(0, vocab, (n,), device=DEV, dtype=torch.int32)

    def calls():
        t = torch.randn(vocab, width, device=DEV)
        h = torch.randn(n, width, device=DEV)
        w = torch.rand(n, device=DEV)
        gh, gw, y = torch.empty_like(h), torch.empty_like(t), torch.empty_like(h)
        yield [t, y], lambda: ops.embed(t, ids, out=y, stream=s)
        yield [h, gw], lambda: ops.embed_grad(h, ids, vocab, out=gw, stream=s)
        yield [h, t, w, gh, gw], lambda: ops.vocab_loss_grad(h, t, ids, weights=w, grad_hidden=gh, grad_head=gw, stream=s)
        yield [t], lambda: ops.orthogonalize(t, stream=s)

    slow(s)  # kernels, libraries and pools are set up before what is looked at
    for _, call in calls():
        call()
    for which in range(4):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        made = list(calls())[which]
        sizes, addresses = [x.shape for x in made[0]], {x.data_ptr() for x in made[0]}
        s.wait_stream(torch.cuda.current_stream())
        slow(s)
        made[1]()
        del made
        again = [torch.empty(size, device=DEV) for size in sizes for _ in range(3)]
        assert not s.query(), "too little work in front of the call for this test to mean anything"
        assert not addresses & {x.data_ptr() for x in again}, which
    # results: the caller's stream is the slow one
    t = torch.randn(vocab, width, device=DEV)
    h = torch.randn(n, width, device=DEV)
    for call in (lambda: [ops.embed(t, ids, stream=s)], lambda: [ops.embed_grad(h, ids, vocab, stream=s)], lambda: list(ops.vocab_loss_grad(h, t, ids, stream=s)),
                 lambda: [ops.orthogonalize(t, stream=s)]):
        torch.cuda.synchronize()
        out = call()
        addresses = {x.data_ptr() for x in out}
        torch.cuda.current_stream().wait_stream(s)
        slow(torch.cuda.current_stream())
        for x in out:
            x.add_(1.0)
        del out, x
        s.synchronize()
        with torch.cuda.stream(s):
            again = [torch.empty(size, device=DEV) for size in ((n,), (n,), (n, width), (vocab, width)) for _ in range(3)]
        assert not torch.cuda.current_stream().query()
        assert not addresses & {x.data_ptr() for x in again}
    torch.cuda.synchronize()


def test_tensors_that_require_a_gradient_are_refused_while_torch_records():
    t = torch.randn(10, 8, device=DEV)
    p = t.clone().requires_grad_()
    ids = torch.arange(10, dtype=torch.int32, device=DEV)
    w = torch.ones(10, device=DEV, requires_grad=True)
    calls = (lambda a, v: ops.embed(a, ids), lambda a, v: ops.embed(t, ids, out=a), lambda a, v: ops.embed_grad(a, ids, 10), lambda a, v: ops.vocab_loss(a, t, ids),
             lambda a, v: ops.vocab_loss(t, a, ids), lambda a, v: ops.vocab_loss_grad(t, t, ids, weights=v), lambda a, v: ops.vocab_loss_grad(t, t, ids, grad_head=a),
             lambda a, v: ops.orthogonalize(a))
    for call in calls:
        with pytest.raises(B.A2Error, match="requires a gradient") as e:
            call(p, w)
        assert e.value.code == B.A2_EINVAL
        call(p.detach(), w.detach())
        with torch.no_grad():
            call(p, w)


def test_a_note_of_a_wait_that_ran_out_stops_the_next_call():
    """The note lies in memory that the GPU writes and the host reads without waiting. The lookup writes it here, as a kernel that gives up would."""
    t = torch.ones(1, 1, device=DEV)
    ids = torch.zeros(1, dtype=torch.int32, device=DEV)
    ops.orthogonalize(torch.ones(4, 4, device=DEV))
    find = B.lib()._ZN2a212gave_up_flagEPPi
    note = C.c_void_p()
    find.argtypes = [C.POINTER(C.c_void_p)]
    assert find(C.byref(note)) == 0
    ops.check()
    s = torch.cuda.current_stream().cuda_stream
    assert B.lib().a2cid2_embed(t.data_ptr(), 1, 1, 1, ids.data_ptr(), 1, 1.0, note, 1, B.A2_F32, s) == B.A2_OK
    torch.cuda.synchronize()
    for call in (lambda: ops.embed(t, ids), lambda: ops.embed_grad(t, ids, 1), lambda: ops.vocab_loss(t, t, ids), lambda: ops.orthogonalize(t), ops.check):
        with pytest.raises(B.A2Error, match="incomplete") as e:
            call()
        assert e.value.code == B.A2_ECUDA
    ops.check()
    assert float(ops.embed(t, ids)) == 1.0


def test_operators_in_a_cuda_graph():
    g = gen(16)
    table = torch.randn(700, 136, generator=g, device=DEV)
    ids = torch.randint(-1, 700, (6000,), generator=g, device=DEV, dtype=torch.int32)

    def step():
        y = ops.embed(table, ids)
        loss, lse, gh, gw = ops.vocab_loss_grad(y, table, ids)
        return loss, lse, gh, gw, ops.embed_grad(gh, ids, 700), ops.orthogonalize(gw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    table.mul_(0.7)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_refusals():
    t = torch.randn(10, 8, device=DEV)
    ids = torch.zeros(10, dtype=torch.int32, device=DEV)
    for call in (lambda: ops.embed(t.cpu(), ids), lambda: ops.embed(t.double(), ids), lambda: ops.embed(t[0], ids),
                 lambda: ops.embed(t, ids.long()), lambda: ops.embed(t.T, ids), lambda: ops.embed(t, ids[::2]),
                 lambda: ops.embed(t[:1].expand(10, 8), ids), lambda: ops.embed(t, ids, out=t.bfloat16()),
                 lambda: ops.embed(t, ids, out=torch.empty(9, 8, device=DEV)), lambda: ops.embed(t, ids, scale=math.nan),
                 lambda: ops.embed(t, ids, scale=1e39), lambda: ops.embed(t[:0], ids),
                 lambda: ops.embed_grad(t, ids, 0), lambda: ops.embed_grad(t, ids[:9], 10), lambda: ops.embed_grad(t, ids, 10, accumulate=True),
                 lambda: ops.embed_grad(t[:, :0], ids, 10),
                 lambda: ops.vocab_loss(t, t[:, :7], ids), lambda: ops.vocab_loss(t, t.bfloat16(), ids), lambda: ops.vocab_loss(t, t, ids[:9]),
                 lambda: ops.vocab_loss_grad(t, t, ids, weights=torch.ones(10, device=DEV, dtype=torch.float64)),
                 lambda: ops.vocab_loss_grad(t, t, ids, grad_head=t[:5]), lambda: ops.vocab_loss_grad(t, t, ids, scale=math.inf),
                 lambda: ops.orthogonalize(t, steps=-1), lambda: ops.orthogonalize(t, eps=-1.0), lambda: ops.orthogonalize(t, coeffs=(1, math.nan, 0)),
                 lambda: ops.orthogonalize(t, coeffs=(3.0, 0.0, 0.0)), lambda: ops.orthogonalize(t, coeffs=(1.0, -9.0, 1.0)),
                 lambda: ops.orthogonalize(t[None].expand(3, 10, 8)), lambda: ops.orthogonalize(t[None, None]), lambda: ops.orthogonalize(t.T)):
        with pytest.raises(B.A2Error) as e:
            call()
        assert e.value.code == B.A2_EINVAL, str(e.value)
    # the library's own checks: workspaces and sizes, nothing is queued
    L, s = B.lib(), torch.cuda.current_stream().cuda_stream
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    p, i, w = t.data_ptr(), ids.data_ptr(), ws.data_ptr()
    assert L.a2cid2_embed(p, 10, 8, 8, i, 1 << 31, 1.0, p, 8, B.A2_F32, s) == B.A2_ERANGE
    assert L.a2cid2_embed(p, 10, 1 << 21, 1 << 21, i, 1, 1.0, p, 1 << 21, B.A2_F32, s) == B.A2_ERANGE
    assert L.a2cid2_embed(p + 2, 10, 8, 8, i, 1, 1.0, p, 8, B.A2_F32, s) == B.A2_EINVAL
    assert L.a2cid2_embed_grad(p, 8, i, 9000, 10, 8, 1.0, 0, p, 8, B.A2_F32, w, 16, s) == B.A2_EINVAL and b"needed" in L.a2cid2_last_error(None)
    assert L.a2cid2_embed_grad(p, 8, i, 9000, 10, 8, 1.0, 0, p, 8, B.A2_F32, w + 8, 1 << 30, s) == B.A2_EINVAL
    assert L.a2cid2_vocab_loss(p, 8, p, 8, i, 10, 8, 10, None, 1.0, None, None, None, 0, None, 0, B.A2_F32, w, 1 << 20, s) == B.A2_EINVAL
    assert L.a2cid2_vocab_loss(p, 8, p, 8, i, 10, 8, 10, None, 1.0, p, p, None, 0, None, 0, 5, w, 1 << 20, s) == B.A2_EINVAL
    assert L.a2cid2_orthogonalize(p, 80, 8, 70000, 1, 1, 5, 1.0, 1.0, 1.0, 0.0, 1.0, p, 80, 8, B.A2_F32, w, 1 << 20, s) == B.A2_ERANGE
    torch.cuda.synchronize()


def test_rows_of_an_engine_train_a_language_model():
    """The operators together, as a user runs them: gradients land in the engine's gradient rows and the population learns. The text's
    entropy is 1.24 and a model that has learnt nothing has ln 64 = 4.16."""
    from paper_2306_08289_b200 import language_model

    for storage in ("f32", "bf16"):
        trace, entropy = language_model.train(n=4, vocab=64, width=32, T=40.0, storage=storage, sequences=8, length=16, samples=2)
        assert trace[0][1] > 0.9 * math.log(64) and trace[-1][1] < 0.5 * (entropy + math.log(64)), (trace, entropy)
        assert all(math.isfinite(v) for row in trace for v in row)
    ops.check()
