"""The language-model operators without a GPU: workspace sizes, refusals that come before any device work, and the host side of the
example that trains a language model with them."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2306_08289_b200 import binding as B
from paper_2306_08289_b200 import build as build_mod
from paper_2306_08289_b200 import language_model as LM


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


P = 1 << 20  # an address that is never touched: every call below is refused, or has nothing to do, before any device work


def size(name, *args):
    out = C.c_int64(-1)
    return getattr(B.lib(), name)(*args, C.byref(out)), out.value


def test_workspace_sizes():
    ok, few = size("a2cid2_embed_grad_workspace", 1000, 64, 500)
    assert ok == B.A2_OK and few == 0  # few ids are not sorted
    ok, many = size("a2cid2_embed_grad_workspace", 50003, 1024, 32768)
    assert ok == B.A2_OK and 32768 * 16 <= many <= 32768 * 16 + 32768 // 64 * 2 * 1024 * 4 + (1 << 20)
    ok, forward = size("a2cid2_vocab_loss_workspace", 8192, 2048, 65536, 0, B.A2_BF16)
    ok2, grad = size("a2cid2_vocab_loss_workspace", 8192, 2048, 65536, 1, B.A2_BF16)
    assert ok == ok2 == B.A2_OK and 0 < forward < grad
    assert grad < 8192 * 65536 * 2, "the workspace must not hold the logits of all tokens, not even in 16 bits"
    ok, tiny = size("a2cid2_vocab_loss_workspace", 32, 64, 257, 1, B.A2_F32)
    assert ok == B.A2_OK and 0 < tiny < 1 << 20
    ok, narrow = size("a2cid2_orthogonalize_workspace", 64, 64, 1024, B.A2_F32)
    assert ok == B.A2_OK and narrow == 0
    ok, wide = size("a2cid2_orthogonalize_workspace", 4, 2048, 4096, B.A2_BF16)
    assert ok == B.A2_OK and wide >= 4 * (2 * 2048 * 4096 + 2 * 2048 * 2048) * 2
    for name, args in (("a2cid2_embed_grad_workspace", (0, 8, 8)), ("a2cid2_embed_grad_workspace", (8, 8, -1)),
                       ("a2cid2_vocab_loss_workspace", (8, 8, 8, 1, 9)), ("a2cid2_orthogonalize_workspace", (1, 0, 8, B.A2_F32)),
                       ("a2cid2_orthogonalize_workspace", (-1, 8, 8, B.A2_F32))):
        assert size(name, *args)[0] == B.A2_EINVAL, (name, args)
    for name, args in (("a2cid2_embed_grad_workspace", (1 << 31, 8, 8)), ("a2cid2_embed_grad_workspace", (8, 8, (1 << 26) + 1)), ("a2cid2_embed_grad_workspace", (8, 1 << 21, 8)),
                       ("a2cid2_vocab_loss_workspace", (1 << 30, 1, 1 << 30, 0, B.A2_F32)), ("a2cid2_orthogonalize_workspace", (1 << 17, 8, 8, 0))):
        assert size(name, *args)[0] == B.A2_ERANGE, (name, args)
    assert B.lib().a2cid2_embed_grad_workspace(8, 8, 8, None) == B.A2_EINVAL


@pytest.mark.parametrize("storage,words,most", [(B.A2_F32, 2, 1 << 24), (B.A2_BF16, 1, 1 << 23)])
def test_workspace_holds_the_whole_of_kept_logits_and_P(storage, words, most):
    """Few logits are kept and turned into P at once, so the gradients' part of the workspace holds every column of both, for any vocabulary."""
    seen = 0
    for n in (1, 2, 3, 8, 16, 25, 64, 102, 255, 256, 257, 700, 4000, 16384):
        for vocab in (512, 5003, 65537, 163840, 163841, 200064, 262144, 327680, 327681, 400000, 1 << 20, 1 << 22, (1 << 23) - 1, 1 << 23, 1 << 24):
            if n * vocab > most:
                continue
            for width in ((1 << 27) // (n * vocab) + 1, 257, 768):
                if storage == B.A2_F32 and n * vocab * width <= 1 << 27 or storage == B.A2_BF16 and width <= 256:
                    continue  # the form without tensor cores
                forward, grad = (size("a2cid2_vocab_loss_workspace", n, width, vocab, g, storage)[1] for g in (0, 1))
                assert grad - forward >= n * vocab * (4 + 2 * words), (n, width, vocab)
                seen += 1
    assert seen > 60


EMBED = dict(table=P, vocab=10, width=8, pitch=8, ids=P, n=4, scale=1.0, out=P, out_pitch=8, dtype=B.A2_F32, stream=None)


@pytest.mark.parametrize("change", [dict(table=None), dict(table=P + 2), dict(vocab=0), dict(width=0), dict(pitch=7), dict(ids=None), dict(ids=P + 2),
                                    dict(n=-1), dict(scale=math.nan), dict(scale=1e300), dict(out=None), dict(out_pitch=4), dict(dtype=2)])
def test_embed_refuses(change):
    assert B.lib().a2cid2_embed(*{**EMBED, **change}.values()) == B.A2_EINVAL
    assert len(B.lib().a2cid2_last_error(None)) > 5


GRAD = dict(grad_out=P, grad_pitch=8, ids=P, n=9000, vocab=10, width=8, scale=1.0, accumulate=0, table=P, pitch=8, dtype=B.A2_BF16, ws=P,
            ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(grad_out=None), dict(grad_out=P + 1), dict(ids=None), dict(table=None), dict(pitch=3), dict(grad_pitch=7),
                                    dict(ws=None), dict(ws=P + 128), dict(ws_bytes=100), dict(scale=math.inf)])
def test_embed_grad_refuses(change):
    assert B.lib().a2cid2_embed_grad(*{**GRAD, **change}.values()) == B.A2_EINVAL


LOSS = dict(hidden=P, hidden_pitch=8, head=P, head_pitch=8, targets=P, n=4, width=8, vocab=10, weights=None, scale=1.0, loss=P, lse=P, gh=P, gh_pitch=8,
            gw=P, gw_pitch=8, dtype=B.A2_F32, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(hidden=None), dict(head=None), dict(targets=None), dict(loss=None), dict(lse=None), dict(weights=P + 1),
                                    dict(loss=P + 2), dict(gh_pitch=7), dict(gw_pitch=7), dict(gh=P + 1), dict(head_pitch=1), dict(scale=-math.inf),
                                    dict(ws=None), dict(ws_bytes=8), dict(dtype=-1), dict(n=-2)])
def test_vocab_loss_refuses(change):
    assert B.lib().a2cid2_vocab_loss(*{**LOSS, **change}.values()) == B.A2_EINVAL


ORTH = dict(inp=P, stride=80, pitch=8, mats=3, rows=10, cols=8, steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7, scale=1.0, out=P, out_stride=80,
            out_pitch=8, dtype=B.A2_F32, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(inp=None), dict(out=None), dict(pitch=7), dict(stride=79), dict(out_stride=79), dict(steps=-1), dict(steps=1001),
                                    dict(eps=-1.0), dict(eps=math.nan), dict(a=math.nan), dict(scale=math.inf), dict(out_stride=96), dict(dtype=3),
                                    dict(a=2.0, b=0.0, c=0.0), dict(a=1.0, b=2.95, c=0.0), dict(a=-4.0, b=4.0, c=0.0), dict(a=3.0, b=-8.0, c=1.0)])
def test_orthogonalize_refuses(change):
    """Among them in place with another stride, and coefficients that take singular values past what the intermediates hold."""
    assert B.lib().a2cid2_orthogonalize(*{**ORTH, **change}.values()) == B.A2_EINVAL


def reach(a, b, c, steps):
    """Brute force: the largest singular value, and the largest |a + b s + c s^2|, that the steps meet from [0, 1]."""
    top, poly = 1.0, 0.0
    for _ in range(steps):
        x = np.linspace(0.0, top, 20001)
        p = np.abs(a + b * x**2 + c * x**4)
        poly = max(poly, float(p.max()))
        top = max(top, float((x * p).max()))
        if top > 100.0:
            break
    return top, poly


def test_the_range_of_coefficients_is_what_a_grid_search_finds():
    rng = np.random.default_rng(3)
    accepted = refused = 0
    for _ in range(400):
        a, b, c = rng.uniform(-4.2, 4.2), rng.uniform(-7, 7), rng.uniform(-5, 5)
        steps = int(rng.integers(1, 7))
        top, poly = reach(a, b, c, steps)
        if abs(top - 1.95) < 1e-3 or abs(poly - 3.9) < 1e-3:
            continue
        # no matrices: an accepted call has nothing to do
        got = B.lib().a2cid2_orthogonalize(*{**ORTH, **dict(mats=0, a=a, b=b, c=c, steps=steps)}.values())
        assert (got == B.A2_OK) == (top < 1.95 and poly < 3.9), (a, b, c, steps, top, poly)
        accepted += got == B.A2_OK
        refused += got != B.A2_OK
    assert accepted > 30 and refused > 30


def test_a_stream_of_another_device_is_refused():
    import types

    import torch

    from paper_2306_08289_b200 import operators as ops

    queue = ops._Queue(torch.device("cuda", 0), types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))
    with pytest.raises(B.A2Error, match="cuda:1") as e:
        queue.__enter__()
    assert e.value.code == B.A2_EINVAL


def test_markov_text():
    text = LM.MarkovText(50, 4, seed=1)
    rng = np.random.default_rng(0)
    ids, targets = text.draw(rng, 6, 9)
    assert ids.dtype == targets.dtype == np.int32 and ids.shape == targets.shape == (54,)
    ids, targets = ids.reshape(6, 9), targets.reshape(6, 9)
    assert (targets[:, -1] == -1).all() and np.array_equal(targets[:, :-1], ids[:, 1:])
    for k in range(8):
        assert all(ids[s, k + 1] in text.next[ids[s, k]] for s in range(6))
    p = 1 / np.arange(1, 5)
    p /= p.sum()
    assert abs(text.entropy + (p * np.log(p)).sum()) < 1e-12


def test_model_parts_tile_the_row():
    import torch

    m = LM.Model(12, 5)
    row = torch.arange(m.d)
    e, h, w = (m.part(row, k) for k in "EMW")
    assert e.shape == (12, 5) and h.shape == (5, 5) and w.shape == (12, 5)
    assert torch.equal(torch.cat([e.reshape(-1), h.reshape(-1), w.reshape(-1)]), row)
    rows = torch.zeros(3, m.d + 7)[:, : m.d]
    part = m.part(rows, "M")
    part[1] = 1.0
    assert part.shape == (3, 5, 5) and rows.sum() == 25 and rows[1].sum() == 25  # a view of the rows
