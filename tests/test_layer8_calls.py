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
