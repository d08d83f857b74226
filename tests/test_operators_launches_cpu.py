"""The host side of the language-model operators on a stand-in for the CUDA runtime (fake_cuda.cpp): what they queue, and what they do when
a launch fails. The kernels do not run."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2306_08289_b200 import binding as B
from paper_2306_08289_b200 import build as build_mod

SOURCES = ["lm_api.cu", "embed.cu", "gemm_sm100.cu", "vocab_loss.cu", "vocab_loss_few.cu", "orthogonalize.cu"]
HERE = os.path.dirname(os.path.abspath(__file__))
FAKED = ["cudaLaunchKernelExC", "cudaMemset2DAsync", "cudaGetDevice", "cudaDeviceGetAttribute", "cudaFuncSetAttribute", "cudaHostAlloc", "cudaStreamSynchronize",
         "cudaThreadExchangeStreamCaptureMode", "cudaGetDriverEntryPointByVersion", "cudaGetLastError"]


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake"))
    nvcc = build_mod._nvcc()
    jobs = []
    for source in [os.path.join(build_mod.CSRC, s) for s in SOURCES] + [os.path.join(HERE, "fake_cuda.cpp")]:
        # the kernels are never run: PTX alone builds in seconds
        jobs.append((source, subprocess.Popen([nvcc, "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-Xcompiler", "-fPIC", "-I", build_mod.INCLUDE,
                                               "-I", build_mod.CSRC, "-c", "-o", os.path.join(out, os.path.basename(source) + ".o"), source],
                                              stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for source, job in jobs:
        text = job.communicate()[0]
        assert job.returncode == 0, (source, text)
    lib = os.path.join(out, "fake.so")
    wraps = [a for name in FAKED for a in ("-Xlinker", f"--wrap={name}")]
    r = subprocess.run([nvcc, "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=compute_100a", "-o", lib]
                       + [os.path.join(out, os.path.basename(s) + ".o") for s in SOURCES + ["fake_cuda.cpp"]] + wraps, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    L = C.CDLL(lib)
    for name, (restype, argtypes) in B.SIGNATURES.items():
        if name.startswith(("a2cid2_embed", "a2cid2_vocab", "a2cid2_orthogonalize", "a2cid2_operators")):
            f = getattr(L, name)
            f.restype, f.argtypes = restype, argtypes
    L.fake_error_text.restype = C.c_char_p
    L.fake_host_memory.restype = C.POINTER(C.c_int)
    return L


P = 1 << 20  # addresses: never touched, for no kernel runs
BIG = 1 << 50


def embed(L, n, vocab, width, dtype=B.A2_F32, shift=0):
    return L.a2cid2_embed(P + shift, vocab, width, width, P, n, 1.0, P, width, dtype, None)


def embed_grad(L, n, vocab, width, accumulate=0, dtype=B.A2_F32, shift=0):
    return L.a2cid2_embed_grad(P + shift, width, P, n, vocab, width, 1.0, accumulate, P, width, dtype, P, BIG, None)


def loss(L, n, width, vocab, dtype, grad=(), weights=None, shift=0):
    gh, gw = (P if k in grad else None for k in ("hidden", "head"))
    return L.a2cid2_vocab_loss(P + shift, width, P + shift, width, P, n, width, vocab, weights, 1.0, P, P, gh, width, gw, width, dtype, P, BIG, None)


def orthogonalize(L, mats, rows, cols, dtype, steps=5, shift=0):
    return L.a2cid2_orthogonalize(P + shift, rows * cols, cols, mats, rows, cols, steps, 3.4445, -4.7750, 2.0315, 1e-7, 1.0, P, rows * cols, cols, dtype, P, BIG,
                                  None)


F32, BF16 = B.A2_F32, B.A2_BF16
BOTH = ("hidden", "head")
# every form of every operator
CALLS = {
    "embed": (embed, (100, 50, 64)), "embed unaligned": (embed, (100, 50, 64, BF16, 2)),
    "embed_grad without a sort": (embed_grad, (100, 500, 64)), "embed_grad sorted": (embed_grad, (20000, 9000, 72, 0, BF16)),
    "embed_grad sorted, accumulate": (embed_grad, (20000, 9000, 71, 1)),
    "loss few": (loss, (32, 64, 257, F32)), "loss few, gradients": (loss, (32, 64, 257, F32, BOTH)), "loss few, parts": (loss, (8, 64, 9000, F32, BOTH)),
    "loss few bf16": (loss, (32, 64, 257, BF16, BOTH)),
    "loss kept f32": (loss, (333, 201, 5003, F32)), "loss kept f32, gradients": (loss, (333, 201, 5003, F32, BOTH)),
    "loss kept f32, one gradient": (loss, (333, 201, 5003, F32, ("head",), P)), "loss kept bf16": (loss, (333, 201, 5003, BF16, BOTH, P)),
    "loss large vocabulary": (loss, (64, 512, 200064, F32, BOTH)),
    "loss f32": (loss, (2048, 512, 32000, F32)), "loss f32, gradients in pieces": (loss, (2048, 512, 32000, F32, BOTH, P)),
    "loss bf16 in place": (loss, (4096, 1024, 50003, BF16)), "loss bf16 unaligned": (loss, (4096, 1023, 50003, BF16, (), None, 2)),
    "loss bf16, gradients in pieces": (loss, (8192, 2048, 65536, BF16, BOTH)), "loss bf16, hidden gradient": (loss, (8192, 2048, 65536, BF16, ("hidden",))),
    "loss of no tokens": (loss, (0, 64, 257, F32, BOTH)),
    "orthogonalize narrow": (orthogonalize, (16, 64, 64, F32)), "orthogonalize f32": (orthogonalize, (16, 1001, 512, F32)),
    "orthogonalize bf16": (orthogonalize, (4, 2048, 4096, BF16)), "orthogonalize, parts of K": (orthogonalize, (1, 300, 9000, F32, 3, 4)),
    "orthogonalize, no steps": (orthogonalize, (2, 300, 200, BF16, 0)),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_ends_at_the_first_launch_that_fails(fake, name):
    """A2_ECUDA with a text, and nothing queued after the failure, wherever it happens."""
    call, args = CALLS[name]
    fake.fake_reset(-1)
    assert call(fake, *args) == B.A2_OK, fake.fake_error_text()
    launches = fake.fake_launches()
    assert launches >= 1 and fake.fake_bad_maps() == 0
    for k in range(launches):
        fake.fake_reset(k)
        assert call(fake, *args) == B.A2_ECUDA, (k, launches)
        assert fake.fake_launches() == k + 1 and len(fake.fake_error_text()) > 10


def test_a_wait_that_ran_out_is_reported_before_more_is_queued(fake):
    fake.fake_reset(-1)
    assert loss(fake, 333, 201, 5003, F32) == B.A2_OK and fake.a2cid2_operators_check(None) == B.A2_OK
    fake.fake_host_memory()[0] = 1  # as a kernel that gives up does
    fake.fake_reset(-1)
    for call, args in CALLS.values():
        assert call(fake, *args) == B.A2_ECUDA and b"incomplete" in fake.fake_error_text()
    assert fake.fake_launches() == 0
    assert fake.a2cid2_operators_check(None) == B.A2_ECUDA and b"incomplete" in fake.fake_error_text()
    assert fake.a2cid2_operators_check(None) == B.A2_OK  # reported once
    for call, args in CALLS.values():
        assert call(fake, *args) == B.A2_OK


# Launches without gradients, with grad_head, with grad_hidden, with both. Few: logits, rows; both gradients in one; join. Else fp32 rows take a scan and
# words first, bf16 rows a copy where a gradient needs hidden without its masked rows; then statistics and rows (kept) or finish; P where logits are made again;
# the products of the gradients, in one launch where they do not fill the GPU; joins of split sums; in pieces, P and the products piece by piece.
LAUNCHES = {F32: {"few": [2, 3, 4, 4], "kept": [4, 5, 6, 6], "kept, long sums": [4, 6, 5, 6], "again": [4, 6, 7, 7], "pieces": [4, 10, 11, 14]},
            BF16: {"few": [2, 3, 4, 4], "kept": [2, 4, 5, 5], "kept, long sums": [2, 5, 4, 5], "again": [2, 5, 6, 6], "pieces": [2, 7, 8, 10]}}


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_sizes_of_the_gpu_tests_reach_every_form(fake, dtype):
    from tests.test_gpu_operators import FORMS

    for form, (n, width, vocab) in FORMS.items():
        got = []
        for grad in ((), ("head",), ("hidden",), BOTH):
            fake.fake_reset(-1)
            assert loss(fake, n, width, vocab, dtype, grad) == B.A2_OK
            got.append(fake.fake_launches())
        assert got == LAUNCHES[dtype][form], form
