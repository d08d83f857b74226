"""Norm, routing and clipping without a GPU: workspace sizes, refusals that come before any device work, what the host side queues and does when a launch
fails (on a stand-in for the CUDA runtime, fake_cuda.cpp; the kernels do not run), and the host side of the example."""
import array
import ctypes as C
import math
import os
import subprocess

import pytest

from paper_2306_08289_b200 import binding as B
from paper_2306_08289_b200 import build as build_mod
from tests import test_operators_launches_cpu as launches

P = 1 << 20  # an address that is never touched
F32, BF16 = B.A2_F32, B.A2_BF16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def size(name, *args):
    out = C.c_int64(-1)
    return getattr(B.lib(), name)(*args, C.byref(out)), out.value


def test_workspace_sizes():
    ok, few = size("a2cid2_rms_norm_grad_workspace", 40, 1000, 1, F32)
    assert ok == B.A2_OK and few == 0  # one launch
    ok, many = size("a2cid2_rms_norm_grad_workspace", 100000, 1000, 1, BF16)
    assert ok == B.A2_OK and 0 < many < 4 * 1000 * 4096
    assert size("a2cid2_rms_norm_grad_workspace", 100000, 1000, 0, BF16) == (B.A2_OK, 0)
    ok, clip = size("a2cid2_clip_gradients_workspace", 10, 100)
    ok2, table = size("a2cid2_clip_gradients_workspace", 1000, 100)
    assert ok == ok2 == B.A2_OK and 800 < clip < 1 << 16 and clip + 72000 <= table < 1 << 18
    for name, args, code in (("a2cid2_rms_norm_grad_workspace", (-1, 8, 1, F32), B.A2_EINVAL), ("a2cid2_rms_norm_grad_workspace", (8, 0, 1, F32), B.A2_EINVAL),
                             ("a2cid2_rms_norm_grad_workspace", (8, 8, 1, 7), B.A2_EINVAL), ("a2cid2_rms_norm_grad_workspace", (8, 32769, 1, F32), B.A2_ERANGE),
                             ("a2cid2_rms_norm_grad_workspace", (1 << 31, 8, 1, F32), B.A2_ERANGE), ("a2cid2_clip_gradients_workspace", (-1, 1), B.A2_EINVAL),
                             ("a2cid2_clip_gradients_workspace", (1, -1), B.A2_EINVAL), ("a2cid2_clip_gradients_workspace", (65537, 1), B.A2_ERANGE),
                             ("a2cid2_clip_gradients_workspace", (1, 65536), B.A2_ERANGE)):
        assert size(name, *args)[0] == code, (name, args)
    assert B.lib().a2cid2_clip_gradients_workspace(1, 1, None) == B.A2_EINVAL


NORM = dict(x=P, x_pitch=8, residual=P, residual_pitch=8, weight=P, n=4, width=8, eps=1e-6, sum=2 * P, sum_pitch=8, out=P, out_pitch=8, dtype=F32, stream=None)


def refused(call, usual, change, code=B.A2_EINVAL):
    assert getattr(B.lib(), call)(*{**usual, **change}.values()) == code, change
    assert len(B.lib().a2cid2_last_error(None)) > 5


@pytest.mark.parametrize("change", [dict(x=None), dict(x=P + 2), dict(n=-1), dict(width=0), dict(x_pitch=7), dict(residual_pitch=7), dict(residual=P + 1), dict(weight=P + 2),
                                    dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e60), dict(sum=P + 2), dict(sum_pitch=1), dict(out=None), dict(out=P + 3),
                                    dict(out_pitch=7), dict(out_pitch=9), dict(sum=P), dict(sum=P, out=2 * P, sum_pitch=9), dict(dtype=2), dict(dtype=-1)])
def test_rms_norm_refuses(change):
    """Among them in place with another pitch, and a sum and a result in one place."""
    refused("a2cid2_rms_norm", NORM, change)


NORM8 = dict(x=P, x_pitch=8, residual=None, residual_pitch=0, weight=None, n=4, width=8, eps=1e-6, sum=None, sum_pitch=0, block=32, values=P, values_pitch=8, scales=P,
             dtype=BF16, stream=None)


@pytest.mark.parametrize("change", [dict(block=16), dict(block=-32), dict(block=33), dict(block=256), dict(values=None), dict(values_pitch=7), dict(scales=None),
                                    dict(scales=P + 2), dict(x=P + 1), dict(eps=-1.0)])
def test_rms_norm_e4m3_refuses(change):
    refused("a2cid2_rms_norm_e4m3", NORM8, change)


BACK = dict(values=P, values_pitch=8, scales=P, n=4, width=8, block=0, out=P, out_pitch=8, dtype=F32, stream=None)


@pytest.mark.parametrize("change", [dict(values=None), dict(values_pitch=3), dict(scales=None), dict(scales=P + 1), dict(block=7), dict(out=None), dict(out=P + 1), dict(out_pitch=0),
                                    dict(n=-1), dict(width=0), dict(dtype=9)])
def test_dequantize_refuses(change):
    refused("a2cid2_dequantize_e4m3", BACK, change)


GRAD = dict(grad_out=P, grad_out_pitch=8, x=P, x_pitch=8, weight=P, grad_sum=P, grad_sum_pitch=8, n=9000, width=8, eps=1e-6, grad_x=P, grad_x_pitch=8, grad_weight=P,
            dtype=F32, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(grad_out=None), dict(x=None), dict(grad_out=P + 2), dict(x_pitch=1), dict(weight=P + 1), dict(grad_weight=P + 2), dict(grad_sum=P + 2),
                                    dict(grad_sum_pitch=0), dict(grad_x=P + 1), dict(grad_x_pitch=9), dict(eps=math.nan), dict(ws=None), dict(ws=P + 8), dict(ws_bytes=64),
                                    dict(n=-5), dict(dtype=4)])
def test_rms_norm_grad_refuses(change):
    refused("a2cid2_rms_norm_grad", GRAD, change)


ROUTE = dict(logits=P, pitch=64, n=10, experts=64, k=4, score=0, bias=None, groups=8, top_groups=2, group_score=0, renormalize=1, scale=1.0, ids=P, weights=P, counts=P,
             dtype=F32, stream=None)


@pytest.mark.parametrize("change", [dict(logits=None), dict(logits=P + 2), dict(pitch=63), dict(n=-1), dict(experts=0), dict(k=0), dict(k=65), dict(k=17), dict(score=2),
                                    dict(score=-1), dict(bias=P + 1), dict(groups=0), dict(groups=7), dict(groups=-8), dict(top_groups=0), dict(top_groups=9),
                                    dict(group_score=2), dict(scale=math.inf), dict(scale=math.nan), dict(ids=None), dict(ids=P + 1), dict(weights=None), dict(weights=P + 2),
                                    dict(counts=P + 1), dict(dtype=3)])
def test_route_refuses(change):
    refused("a2cid2_route", ROUTE, change)


def test_sizes_out_of_range():
    refused("a2cid2_rms_norm", NORM, dict(width=32769, x_pitch=1 << 20, residual_pitch=1 << 20, sum_pitch=1 << 20, out_pitch=1 << 20), B.A2_ERANGE)
    refused("a2cid2_rms_norm", NORM, dict(n=(1 << 30) + 1), B.A2_ERANGE)
    refused("a2cid2_route", ROUTE, dict(experts=1025, pitch=1025, groups=1, top_groups=1), B.A2_ERANGE)
    refused("a2cid2_route", ROUTE, dict(k=33, groups=1, top_groups=1), B.A2_ERANGE)
    refused("a2cid2_route", ROUTE, dict(groups=64, top_groups=64), B.A2_ERANGE)


ROUTE_GRAD = dict(logits=P, pitch=64, ids=P, grad_weights=P, n=10, experts=64, k=4, score=0, renormalize=1, scale=1.0, out=P, out_pitch=64, dtype=F32, stream=None)


@pytest.mark.parametrize("change", [dict(logits=None), dict(pitch=3), dict(ids=None), dict(ids=P + 2), dict(grad_weights=None), dict(grad_weights=P + 2), dict(k=65), dict(k=0),
                                    dict(score=5), dict(scale=math.nan), dict(out=None), dict(out=P + 1), dict(out_pitch=63), dict(out_pitch=65), dict(dtype=2), dict(n=-1)])
def test_route_grad_refuses(change):
    refused("a2cid2_route_grad", ROUTE_GRAD, change)


TENSOR = dict(inp=P, out=P, stride=100, out_stride=100, rows=10, cols=8, pitch=10, out_pitch=10, dtype=F32)


def clip(tensors, workers=2, max_norm=1.0, zero=0, norms=P, ws=P, ws_bytes=1 << 30, norms_alone=False, lib=None, count=None):
    words = array.array("q", [0 if v is None else v for t in tensors for v in {**TENSOR, **t}.values()])
    L = lib or B.lib()
    table, n = words.buffer_info()[0] if tensors else None, len(tensors) if count is None else count
    if norms_alone:
        return L.a2cid2_gradient_norms(table, n, workers, norms, ws, ws_bytes, None)
    return L.a2cid2_clip_gradients(table, n, workers, max_norm, zero, norms, ws, ws_bytes, None)


def test_clip_refuses():
    for change in (dict(inp=None), dict(out=None), dict(inp=P + 2), dict(out=P + 2), dict(rows=-1), dict(cols=-1), dict(pitch=7), dict(out_pitch=7), dict(stride=97),
                   dict(out_stride=97), dict(dtype=2), dict(out_stride=104), dict(out_pitch=9)):
        assert clip([change]) == B.A2_EINVAL, change
    for kw in (dict(max_norm=-1.0), dict(max_norm=math.nan), dict(norms=None), dict(norms=P + 2), dict(ws=None), dict(ws=P + 16), dict(ws_bytes=100), dict(workers=-1),
               dict(count=-1)):
        assert clip([{}], **kw) == B.A2_EINVAL, kw
    assert clip([{}, dict(inp=3 * P)]) == B.A2_EINVAL and b"same out" in B.lib().a2cid2_last_error(None)
    assert clip([], count=3) == B.A2_EINVAL
    assert clip([dict(rows=1 << 31, cols=1 << 10, pitch=1 << 10, out_pitch=1 << 10, stride=1 << 40, out_stride=1 << 40)], workers=1) == B.A2_ERANGE
    assert clip([{}], workers=65536) == B.A2_ERANGE
    # the norms alone do not look at where clipped ones would go
    assert clip([dict(inp=None, out=None)], norms_alone=True) == B.A2_EINVAL


# ------------------------------------------------------------------------------------------------
# launches
# ------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake"))
    nvcc, sources = build_mod._nvcc(), launches.SOURCES + ["lm_train_api.cu", "rms_norm.cu", "route.cu", "clip.cu"]
    jobs = []
    for source in [os.path.join(build_mod.CSRC, s) for s in sources] + [os.path.join(launches.HERE, "fake_cuda.cpp")]:
        jobs.append((source, subprocess.Popen([nvcc, "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-Xcompiler", "-fPIC", "-I", build_mod.INCLUDE,
                                               "-I", build_mod.CSRC, "-c", "-o", os.path.join(out, os.path.basename(source) + ".o"), source],
                                              stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for source, job in jobs:
        text = job.communicate()[0]
        assert job.returncode == 0, (source, text)
    lib = os.path.join(out, "fake.so")
    wraps = [a for name in launches.FAKED for a in ("-Xlinker", f"--wrap={name}")]
    r = subprocess.run([nvcc, "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=compute_100a", "-o", lib]
                       + [os.path.join(out, os.path.basename(s) + ".o") for s in sources + ["fake_cuda.cpp"]] + wraps, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    L = C.CDLL(lib)
    for name, (restype, argtypes) in B.SIGNATURES.items():
        if hasattr(L, name):
            f = getattr(L, name)
            f.restype, f.argtypes = restype, argtypes
    L.fake_error_text.restype = C.c_char_p
    L.fake_host_memory.restype = C.POINTER(C.c_int)
    return L


BIG = 1 << 50


def norm(L, n, width, dtype, pad=0, shift=0, residual=True):
    p = width + pad
    return L.a2cid2_rms_norm(P + shift, p, P + shift if residual else None, p, P, n, width, 1e-6, None, 0, 3 * P + shift, p, dtype, None)


def norm8(L, n, width, dtype, block, pad=0):
    return L.a2cid2_rms_norm_e4m3(P, width + pad, None, 0, P, n, width, 1e-6, None, 0, block, P, width, P, dtype, None)


def back(L, n, width, block, pad=0):
    return L.a2cid2_dequantize_e4m3(P, width + pad, P, n, width, block, P, width, BF16, None)


def norm_grad(L, n, width, dtype, weight=True, pad=0, shift=0):
    p = width + pad
    return L.a2cid2_rms_norm_grad(P + shift, p, P + shift, p, P, None, 0, n, width, 1e-6, 3 * P + shift, p, P if weight else None, dtype, P, BIG, None)


def route(L, n, experts, k, groups=1, top_groups=1, bias=None, counts=P, dtype=F32):
    return L.a2cid2_route(P, experts, n, experts, k, 1, bias, groups, top_groups, 1, 1, 1.0, P, P, counts, dtype, None)


def route_grad(L, n, experts, k, dtype=F32):
    return L.a2cid2_route_grad(P, experts, P, P, n, experts, k, 0, 0, 1.0, 2 * P, experts, dtype, None)


def clips(L, count, cols, workers=1, **kw):
    return clip([dict(inp=P + (i << 30), out=(P << 20) + (i << 30), rows=1, cols=cols, stride=cols, out_stride=cols) for i in range(count)], workers=workers, lib=L, **kw)


# every form of every operator: (call, arguments, launches)
CALLS = {
    "norm one token": (norm, (1, 2048, BF16), 1), "norm": (norm, (1000, 201, F32), 1), "norm unaligned": (norm, (1000, 201, F32, 3, 4), 1),
    "norm narrow": (norm, (1000, 8, BF16), 1), "norm longest": (norm, (10, 32768, F32), 1), "norm longest bf16": (norm, (10, 32768, BF16, 1), 1),
    "norm of no rows": (norm, (0, 64, F32), 0), "norm without a residual": (norm, (5, 4096, F32, 0, 0, False), 1),
    "8 bits": (norm8, (100, 2048, BF16, 128), 1), "8 bits a row": (norm8, (100, 2048, F32, 0), 1), "8 bits unaligned": (norm8, (100, 1001, F32, 64, 2), 1),
    "back": (back, (100, 2048, 128), 1), "back unaligned": (back, (100, 1001, 0, 5), 1), "back of no rows": (back, (0, 64, 0), 0),
    "gradient of few rows": (norm_grad, (1, 2048, BF16), 1), "gradient of few rows, 16 CTAs": (norm_grad, (500, 200, F32), 1), "gradient": (norm_grad, (5000, 200, F32), 2),
    "gradient unaligned": (norm_grad, (5000, 201, BF16, True, 1, 2), 2), "gradient of rows alone": (norm_grad, (5000, 2048, BF16, False), 1),
    "gradient of long rows": (norm_grad, (50, 16384, BF16), 2), "gradient of the longest rows": (norm_grad, (50, 32768, F32), 2), "gradient of no rows": (norm_grad, (0, 64, F32), 1),
    "gradient of no long rows": (norm_grad, (0, 32768, F32), 2),
    "route few": (route, (16, 64, 2), 1), "route": (route, (1000, 256, 8), 2), "route groups": (route, (1000, 256, 8, 8, 4, P), 2), "route many experts": (route, (20, 1024, 32), 2),
    "route odd groups": (route, (20, 1023, 32, 31, 31), 2), "route without counts": (route, (1000, 100, 3, 1, 1, None, None, BF16), 1), "route no tokens": (route, (0, 64, 2), 1),
    "route no tokens, no counts": (route, (0, 64, 2, 1, 1, None, None), 0),
    "route gradient": (route_grad, (1000, 161, 6), 1), "route gradient few": (route_grad, (3, 8, 2, BF16), 1), "route gradient of no tokens": (route_grad, (0, 8, 2), 0),
    "clip small": (clips, (3, 100), 1), "clip": (clips, (3, 100000), 2), "clip large": (clips, (3, 20000000), 3), "clip many tensors": (clips, (300, 1000), 4),
    "clip workers": (clips, (2, 100000, 64), 3), "clip nothing": (clips, (2, 0, 5), 1), "clip no workers": (clips, (2, 10, 0), 0), "clip no tensors": (clips, (0, 0), 1),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_ends_at_the_first_launch_that_fails(fake, name):
    """So many launches, and A2_ECUDA with a text and nothing queued after a failure, wherever it happens."""
    call, args, count = CALLS[name]
    fake.fake_reset(-1)
    assert call(fake, *args) == B.A2_OK, fake.fake_error_text()
    assert fake.fake_launches() == count
    for k in range(count):
        fake.fake_reset(k)
        assert call(fake, *args) == B.A2_ECUDA, k
        assert fake.fake_launches() == k + 1 and len(fake.fake_error_text()) > 10


def test_norms_alone(fake):
    for count, cols, launched in ((2, 100, 1), (2, 1000000, 2), (60, 1000000, 3)):
        fake.fake_reset(-1)
        assert clips(fake, count, cols, norms_alone=True) == B.A2_OK and fake.fake_launches() == launched


def test_a_wait_that_ran_out_is_reported_before_more_is_queued(fake):
    fake.fake_reset(-1)
    assert launches.loss(fake, 333, 201, 5003, F32) == B.A2_OK
    fake.fake_host_memory()[0] = 1  # as a kernel of the products that gives up does
    fake.fake_reset(-1)
    for call, args, _ in CALLS.values():
        assert call(fake, *args) == B.A2_ECUDA and b"incomplete" in fake.fake_error_text()
    assert fake.fake_launches() == 0 and fake.a2cid2_operators_check(None) == B.A2_ECUDA
    for call, args, _ in CALLS.values():
        assert call(fake, *args) == B.A2_OK


# ------------------------------------------------------------------------------------------------
# the wrappers and the example
# ------------------------------------------------------------------------------------------------
def test_rows_of_a_tensor():
    """How tensors are read as rows at one distance from each other, against what their strides say."""
    import torch

    from paper_2306_08289_b200 import operators as ops

    base = torch.arange(24000).view(20, 30, 40)
    for t in (base, base[:, :, 3:7], base[2:9:2], base.transpose(0, 2), base[:, 5], base[3, :, 7], base[4:5, 6:7], base[:, :, 9], base[0, 0, ::3], base[:, ::2].transpose(0, 1)[:, :1]):
        try:
            rows, cols, pitch, out_pitch = ops._rows_of("t", t.shape, t.stride(), t.stride())
        except B.A2Error:
            continue
        assert rows * cols == t.numel() and pitch == out_pitch and (rows == 1 or pitch >= cols)
        got = torch.as_strided(base, (rows, cols), (pitch, 1), t.storage_offset())
        assert torch.equal(got.flatten().sort().values, t.flatten().sort().values)
    for bad in (base.expand(2, 20, 30, 40), base[:, ::2, ::3], base[::2, :20, :7].transpose(0, 1)):
        with pytest.raises(B.A2Error):
            ops._rows_of("t", bad.shape, bad.stride(), bad.stride())


def test_the_usual_calls_leave_what_is_not_usual():
    """Tensors of the CPU and arguments of another kind go to the wrappers, which say what is wrong."""
    import torch

    from paper_2306_08289_b200 import operators as ops

    t = torch.zeros(4, 8)
    usual = ops._usual()
    for got in (usual.rms_norm(t, None, None, 1e-6), usual.rms_norm(None, None, None, 1e-6), usual.rms_norm_grad(t, t, None, 1e-6, None, True, True),
                usual.rms_norm_quantized(t, None, None, 1e-6, 32), usual.route(t, 2, 0, None, 1, 1, 0, True, 1.0), usual.route_grad(t, t, t, 0, True, 1.0),
                usual.clip([t], None, False, 1.0, False), usual.clip([], None, False, 1.0, False), usual.clip(t, None, False, 1.0, False), usual.dequantize(t, t, 0)):
        assert got is None
    with pytest.raises(TypeError):
        usual.rms_norm(t)
    for call in (lambda: ops.rms_norm(t), lambda: ops.rms_norm_quantized(t), lambda: ops.dequantize(t, t), lambda: ops.rms_norm_grad(t, t), lambda: ops.route(t, 2),
                 lambda: ops.route_grad(t, t, t), lambda: ops.clip_gradients([t], 1.0), lambda: ops.gradient_norms([t])):
        with pytest.raises(B.A2Error) as e:
            call()
        assert e.value.code == B.A2_EINVAL


def test_parts_of_a_model_with_norms_and_experts():
    import torch

    from paper_2306_08289_b200 import language_model as LM

    m = LM.Model(12, 5, norm=True, experts=3)
    row = torch.arange(m.d)
    assert torch.equal(torch.cat([m.part(row, k).reshape(-1) for k in m.shape]), row) and list(m.shape) == ["E", "M", "W", "R", "N", "F"]
    assert m.hidden(row).shape == (3, 5, 5) and torch.equal(m.hidden(row).flatten(), m.part(row, "M").flatten())
    rows = torch.zeros(4, m.d + 3)[:, : m.d]
    m.hidden(rows)[2, 1] = 1.0
    assert m.hidden(rows).shape == (4, 3, 5, 5) and rows.sum() == 25 and rows[2].sum() == 25
    start = torch.from_numpy(m.initial_row(3))
    assert (m.part(start, "N") == 1).all() and (m.part(start, "F") == 1).all()
    assert LM.Model(12, 5).d == 2 * 60 + 25
