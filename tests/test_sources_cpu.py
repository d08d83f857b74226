"""What the kernels' sources have to keep to, and no run is sure to show."""
import os
import re

from paper_2306_08289_b200 import build as build_mod


def kernels():
    """(file, name, parameters, body) of every kernel."""
    for file in sorted(os.listdir(build_mod.CSRC)):
        if not file.endswith((".cu", ".cuh", ".h")):
            continue
        with open(os.path.join(build_mod.CSRC, file)) as f:
            text = f.read()
        for m in re.finditer(r"__global__ void(?: __\w+__\((?:[^()]|\([^()]*\))*\))* (\w+)\(", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(text[at], 0)
                at += 1
            body = text[at:text.index("\n}\n", at)]
            yield file, m.group(1), text[m.end():at - 1], body


def test_kernels_that_begin_before_their_predecessor_ends_do_not_promise_the_compiler_constant_inputs():
    """`const T* __restrict__` is read through the read-only cache, and may be read before the wait for the predecessor, which is still writing it then."""
    found = list(kernels())
    chained = [k for k in found if re.search(r"chained\(\)|wait_previous\(\)", k[3])]
    assert len(found) > 40 and len(chained) > 20, "the sources are not read as they should be"
    assert {"k_dequantize", "k_norm_join", "k_route", "k_squares", "k_embed", "k_join", "k_gemm"} <= {k[1] for k in chained}
    for file, name, parameters, _ in chained:
        assert not re.search(r"const [\w:]+\* *__restrict__", parameters), (file, name)
        assert "__ldg" not in _ and "ld.global.nc" not in _, (file, name)


def test_kernels_that_begin_before_their_predecessor_ends_wait_for_it_whatever_their_arguments():
    """What earlier kernels have written is visible behind a kernel's own wait alone, so none is on a condition, and nothing of memory is touched before it."""
    for file, name, _, body in kernels():
        waits = list(re.finditer(r"^.*(?:chained\(\)|wait_previous\(\)).*$", body, re.M))
        if not waits:
            continue
        assert len(waits) == 1, (file, name)
        assert re.fullmatch(r" {4}ptx::(chained|wait_previous)\(\);", waits[0].group()), (file, name)
        before = body[body.index("{") + 1:waits[0].start()]
        assert not re.search(r"\bload|\bstore|atomic|__ld|__st", before), (file, name)
