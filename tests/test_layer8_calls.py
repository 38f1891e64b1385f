"""What calls of the 8-bit layers and of the gated block do where they cannot run, on the host: nothing here needs a GPU."""
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2410_13056_b200 import binding as B
from paper_2410_13056_b200 import build as cuda_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = 4


@pytest.fixture(scope="module")
def L():
    cuda_build.build()
    return B.lib()


# Calls whose arguments are all right, in a process of their own: one that ends by a signal ends alone.
CALLS = r"""
import ctypes
from paper_2410_13056_b200 import binding as B
L = B.lib()
buf = (ctypes.c_char * (1 << 20))()
p = (ctypes.addressof(buf) + 255) // 256 * 256
y, room = p + (1 << 19), 1 << 40
for name, n, d_in, d_ff, d_out in %r:
    w = B.Weight8(p, (max(d_in, d_ff) + 15) // 16 * 16, p, None)
    for word in (None, p):
        if name == "linear":
            s = L.cmpq_linear_i8_fused(p, 0, n, d_in, d_in, None, 0.0, w, d_out, 0, None, 0, y, d_out, word, p, room, None)
        elif name == "matmul":
            s = L.cmpq_matmul_i8(p, w.ld, p, p, w.ld, p, None, 0, n, d_in, d_out, y, d_out, p, room, None)
        else:
            s = L.cmpq_gated_i8(p, 0, n, d_in, d_in, None, 0.0, w, w, w, d_ff, d_out, 2, None, 0, y, d_out, word, p, p, room, None)
        print(name, n, d_in, d_ff, d_out, word is not None, s, flush=True)
"""


def test_without_a_device_calls_answer_an_error(L):
    if torch.cuda.is_available():
        pytest.skip("the addresses are no GPU's")
    calls = [("linear", 1, 20, 0, 5), ("linear", 4, 4096, 0, 500), ("linear", 9, 20, 0, 5), ("linear", 300, 9000, 0, 500), ("matmul", 2, 9000, 0, 500),
             ("gated", 1, 20, 30, 5), ("gated", 2, 8192, 8192, 8192), ("gated", 9, 20, 30, 5)]
    run = subprocess.run([sys.executable, "-c", CALLS % calls], cwd=ROOT, capture_output=True, text=True, timeout=200)
    want = ["%s %d %d %d %d %s %d" % (*c, word, CUDA) for c in calls for word in (False, True)]
    assert run.returncode == 0 and run.stdout.splitlines() == want, (run.returncode, run.stdout, run.stderr)


def _body(source, head):
    """The text of the function whose declaration contains `head`, braces matched."""
    at = source.index(head)
    at = source.index("{", at)
    depth, end = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(source[end], 0)
        end += 1
        if depth == 0:
            return source[at:end]


def test_residuals_are_not_read_as_memory_that_nobody_writes():
    """A residual may be the output, so the kernel that reads it writes it: neither load8, whose wide loads go through the
    read-only path, nor __ldg may read one.  On the chip the difference cannot be seen as long as a thread reads its own entries."""
    read_only = re.compile(r"\b(load8|__ldg)\(")
    for name in sorted(os.listdir(cuda_build.CSRC)):
        for line in open(os.path.join(cuda_build.CSRC, name)):
            for call in read_only.finditer(line):
                assert not re.match(r"[^;]*\bresidual\b", line[call.end():].split(")")[0]), (name, line)
    product = open(os.path.join(cuda_build.CSRC, "product_i8.cuh")).read()
    for head in ("void load16(", "void store_finished(", "void store_eight("):
        body = _body(product, head)
        assert not read_only.search(body), (head, body)
    assert "load16<DT>(residual" in _body(product, "void store_finished(")


ASKED = r"""
#include <cstdio>
#include <initializer_list>
#include "asked.h"

int main() {
    cmpq::AskedOnce fails, works;
    int asked = 0, answers = 0;
    for (int i = 0; i < 3; ++i)
        for (int device : {0, 63}) answers += fails.get(device, [&] { return ++asked, 0; });
    printf("%d %d ", answers, asked);  // no answer is kept as one
    asked = answers = 0;
    for (int i = 0; i < 3; ++i)
        for (int device : {0, 5, 63}) answers += works.get(device, [&] { return ++asked, 7; });
    printf("%d %d ", answers, asked);
    asked = answers = 0;
    for (int device : {-1, 64, 64}) answers += works.get(device, [&] { return ++asked, 9; });  // devices without a place
    printf("%d %d\n", answers, asked);
}
"""


def test_a_number_that_cannot_be_had_is_asked_for_once(tmp_path):
    src, exe = tmp_path / "asked.cpp", str(tmp_path / "asked")
    src.write_text(ASKED)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", cuda_build.CSRC, str(src), "-o", exe], check=True)
    assert subprocess.run([exe], capture_output=True, text=True, timeout=20).stdout.split() == ["0", "2", "63", "3", "27", "3"]


def test_a_failed_query_leaves_no_error_behind():
    """The launch behind it asks for the last error."""
    source = open(os.path.join(cuda_build.CSRC, "linear_i8.cu")).read()
    body = _body(source, "static int cluster_slots(")
    failing = body[body.index("cudaOccupancyMaxActiveClusters"):]
    assert re.match(r"[^;]*== cudaSuccess\) return n;\s*cudaGetLastError\(\);", failing), body
    assert re.search(r"cudaGetDevice\(&dev\) != cudaSuccess\) return cudaGetLastError\(\), 0;", body)


# ---- the wrappers of the C calls --------------------------------------------------------------------------------

F16, BF16, F32, I8, U8, I32 = torch.float16, torch.bfloat16, torch.float32, torch.int8, torch.uint8, torch.int32
N, D, FF, O = 3, 32, 48, 16
ELSEWHERE = "meta"


def _new(dtype, *shape, device="cpu"):
    return torch.zeros(shape, dtype=dtype, device=device)


def _halves(dtype, n):
    """Every second of 2 n entries."""
    return _new(dtype, 2 * n)[::2]


def _matrices(n, d, dtype=F16):
    return [_new(dtype, n - 1, d), _new(dtype, n + 1, d), _new(dtype, n, d - 1), _new(F32, n, d), _new(BF16, n, d), _new(dtype, n * d), _new(dtype, d, n).t(),
            _new(dtype, n, d, device=ELSEWHERE)]


def _vectors(n, dtype):
    return [_new(dtype, n - 1), _new(dtype, n + 1), _halves(dtype, n), _new(dtype, n, 1), _new(torch.float64, n), _new(dtype, n, device=ELSEWHERE)]


WORDS = [_new(torch.int64, 1), _new(I32, 0), _new(I32, 1, device=ELSEWHERE)]


def _refused(call, good, bad):
    """Every bad argument in the place of its good one; the good ones reach the library, which is not called here."""
    for name, values in bad.items():
        for value in values:
            with pytest.raises((ValueError, TypeError)):
                call(**{**good, name: value})


@pytest.fixture
def untouched(L, monkeypatch):
    """The library, where every call of these says that it was made."""
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(B, "lib", lambda: Library())
    monkeypatch.setattr(B, "_on", lambda t: 0)
    return made


def test_norm_quantize_wrapper_refuses_what_does_not_fit(untouched):
    good = dict(X=_new(F16, N, D), norm=_new(F16, D), eps=1e-6, codes=_new(I8, N, D), scale=_new(F32, N), nonfinite=_new(I32, 1))
    codes = [_new(I8, N - 1, D), _new(I8, N + 1, D), _new(I8, N, D - 16), _new(I8, N, D + 16), _new(U8, N, D), _new(I8, N * D), _new(I8, N, D, device=ELSEWHERE)]
    _refused(B.cmpq_norm_quantize_tokens, good, dict(norm=_vectors(D, F16) + [_new(BF16, D)], codes=codes, scale=_vectors(N, F32) + [_new(F16, N)], nonfinite=WORDS))
    assert not untouched
    B.cmpq_norm_quantize_tokens(**good)
    assert untouched == ["cmpq_norm_quantize_tokens"]


def _weights(d_out, d_in, bias=F16):
    return B.weight8(_new(I8, d_out, d_in), _new(F32, d_out), None if bias is None else _new(bias, d_out))


def test_linear_wrapper_refuses_what_does_not_fit(untouched):
    good = dict(X=_new(F16, N, D), weight=_weights(O, D), d_out=O, y=_new(F16, N, O), ws=_new(U8, 4096), norm=_new(F16, D), eps=1e-6, act="silu",
                residual=_new(F16, N, O), nonfinite=_new(I32, 1))
    _refused(B.cmpq_linear_i8_fused, good, dict(weight=[_weights(O + 1, D), _weights(O - 1, D), _weights(O, D + 16), _weights(O, D, BF16)], d_out=[O + 1, O - 1],
                                                y=_matrices(N, O), ws=[_new(U8, 4096)[::2], _new(U8, 4096, device=ELSEWHERE)], norm=_vectors(D, F16) + [_new(BF16, D)],
                                                act=["tanh", "", 2], residual=_matrices(N, O), nonfinite=WORDS, X=[_new(F32, N, D), _new(F16, N, D + 1)]))
    assert not untouched
    for more in ({}, dict(norm=None, residual=None, nonfinite=None, act=None, weight=_weights(O, D, None)), dict(y=_new(F16, N, O + 8)[:, :O])):
        B.cmpq_linear_i8_fused(**{**good, **more})
    assert len(untouched) == 3


def test_gated_wrapper_refuses_what_does_not_fit(untouched):
    good = dict(X=_new(F16, N, D), gate=_weights(FF, D), up=_weights(FF, D), down=_weights(O, FF), d_ff=FF, d_out=O, y=_new(F16, N, O),
                state=_new(U8, B.GATED_STATE_BYTES), ws=_new(U8, 4096), norm=_new(F16, D), eps=1e-6, act="gelu", residual=_new(F16, N, O), word=_new(I32, 1))
    _refused(B.cmpq_gated_i8, good, dict(gate=[_weights(FF - 1, D), _weights(FF, D + 1)], up=[_weights(FF + 1, D)], down=[_weights(O, FF + 16), _weights(O + 1, FF), _weights(O, FF, BF16)],
                                         d_ff=[FF - 1, FF + 1], d_out=[O + 1], y=_matrices(N, O), ws=[_new(U8, 4096, device=ELSEWHERE)], norm=_vectors(D, F16),
                                         state=[_new(U8, B.GATED_STATE_BYTES - 1), _new(U8, 0), _new(U8, 256, device=ELSEWHERE), _new(I32, 128)[::2]],
                                         act=["swish"], residual=_matrices(N, O), word=WORDS, X=[_new(F16, N, D + 1), _new(torch.int8, N, D)]))
    assert not untouched
    for more in ({}, dict(state=_new(I32, 64)), dict(norm=None, residual=None, word=None)):
        B.cmpq_gated_i8(**{**good, **more})
    assert len(untouched) == 3


def test_weights_refuse_what_does_not_fit_and_keep_their_tensors():
    good = dict(codes=_new(I8, O, D), scale=_new(F32, O), bias=_new(F16, O))
    _refused(B.weight8, good, dict(codes=[_new(U8, O, D), _new(I8, D, O).t(), _new(I8, O * D), _new(I8, O + 1, D), _new(I8, O, D, device=ELSEWHERE)],
                                   scale=_vectors(O, F32), bias=[_new(F16, O - 1), _halves(F16, O), _new(F16, O, device=ELSEWHERE)]))
    w = B.weight8(*(t.clone() for t in good.values()))
    assert (w.codes, w.ld, w.scale, w.bias) == (w.tensors[0].data_ptr(), D, w.tensors[1].data_ptr(), w.tensors[2].data_ptr())
