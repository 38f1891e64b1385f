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


def test_attention_that_zeroes_rows_takes_its_arguments_as_it_did(L):
    import ctypes

    buf = (ctypes.c_char * 8192)()
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    zero = 0x100
    cache = B.Cache(k_codes=p, k_scale=p, v_codes=p, v_scale=p, n_pages=4, n_kv_heads=2, head_dim=64, page_tokens=16)

    def attention(n_seq=2, n_tok=3, causal=1, window=0, out=p, q=p):
        batch = B.Batch(tok_off=p, lens=p, table=p, ld_table=2, n_seq=n_seq, n_tok=n_tok)
        return L.cmpq_cache_attention(cache, batch, q, 256, 0, 4, 2, 32, 0.1, causal, window, out, 256, None, None, None, 0, None)

    invalid, workspace = 1, 3
    for causal in (0, 1, zero, zero + 1):                  # all that comes next is the work space
        assert attention(causal=causal) == workspace
        assert attention(causal=causal, window=4) == (workspace if causal & 1 else invalid)
        assert attention(causal=causal, out=None) == invalid
        assert attention(causal=causal, n_tok=0, out=None) == 0
        assert attention(causal=causal, n_seq=0, out=None) == (invalid if causal & zero else 0)


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


def test_tensors_of_the_host_are_refused(monkeypatch):
    """Before an address of theirs gets to a kernel."""
    from paper_2410_13056_b200 import serving

    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(B, "lib", lambda: Library())
    with pytest.raises(ValueError, match="GPU"):
        serving.quantize_tokens(_new(F16, N, D))
    with pytest.raises(ValueError, match="GPU"):
        serving.quantize_tokens(_new(F16, N, D), _new(F16, D))
    with pytest.raises(ValueError, match="GPU"):
        B.cmpq_linear_i8_fused(_new(F16, N, D), _weights(O, D), O, _new(F16, N, O), _new(U8, 4096))
    with pytest.raises(ValueError, match="GPU"):
        B.cmpq_gated_i8(_new(F16, N, D), _weights(FF, D), _weights(FF, D), _weights(O, FF), FF, O, _new(F16, N, O), _new(U8, 256), _new(U8, 4096))
    with pytest.raises(ValueError, match="GPU"):
        B.cmpq_quantize_tokens(_new(F16, N, D), _new(I8, N, D), _new(F32, N))
    assert not made


def test_tokens_are_quantized_on_their_own_device(untouched, monkeypatch):
    from paper_2410_13056_b200 import serving

    at = []

    class DeviceOf:
        def __init__(self, t):
            self.t = t

        def __enter__(self):
            at.append(self.t)

        def __exit__(self, *_):
            assert untouched == ["cmpq_norm_quantize_tokens"]
            at.append("left")

    monkeypatch.setattr(torch.cuda, "device_of", DeviceOf)
    x = _new(F16, N, D)
    serving.quantize_tokens(x)
    assert at[0] is x and at[1:] == ["left"]


# ---- how products are covered -------------------------------------------------------------------------------------

PLAN = r"""
#include <cstdio>
#include "plan_i8.h"

int main() {
    long long n, d_in, cols, sms, two, four;
    while (scanf("%lld %lld %lld %lld %lld %lld", &n, &d_in, &cols, &sms, &two, &four) == 6) {
        const auto a = cmpq::plan_product({n, cols, cmpq::ceil_div(d_in, 128), sms}, [&](int parts) { return (int)(parts == 2 ? two : four); });
        printf("%d %d %d %d %d %d\n", a.pair, a.bn, a.rows, a.parts, a.slices, a.per_stage);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan([(tokens, entries of the sum, rows of weights, SMs, clusters of two, of four at once) ..]) -> [dict ..]"""
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(PLAN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", cuda_build.CSRC, str(at / "plan.cpp"), "-o", str(at / "plan")], check=True)

    def run(sizes):
        out = subprocess.run([str(at / "plan")], input="".join("%d %d %d %d %d %d\n" % s for s in sizes), capture_output=True, text=True, timeout=300).stdout
        plans = [dict(zip(("pair", "bn", "rows", "parts", "slices", "per_stage"), map(int, line.split()))) for line in out.splitlines()]
        assert len(plans) == len(sizes)
        return plans

    return run


B200 = (148, 74, 33)  # SMs; clusters of two and of four blocks that run at once
SUMS = [64, 512, 1000, 2049, 4096, 5461, 8192, 11008, 13824, 14336, 18944, 28672, 131072]
CHANNELS = [1, 33, 512, 1024, 2049, 3584, 4096, 5120, 8192, 11008, 22016, 28672, 57344]
TOKENS = [1, 5, 8, 9, 31, 32, 33, 64, 65, 100, 128, 129, 192, 256, 257, 400, 512, 513, 576, 640, 768, 900, 1024, 1152, 1280, 1408, 1600, 1792, 2048, 2560, 3000, 3328, 4000, 4200,
          4400, 10000, 1 << 20]


def test_clusters_do_not_take_the_place_of_pairs_past_their_fit(plan):
    sizes = [(n, d, o) for n in TOKENS for d in SUMS for o in CHANNELS]
    with_clusters, without = plan([s + B200 for s in sizes]), plan([s + (148, 0, 0) for s in sizes])
    taken = [s for s, a, b in zip(sizes, with_clusters, without) if a["parts"] > 1 and b["pair"]]
    assert taken and max(n for n, *_ in taken) <= 512, [s for s in taken if s[0] > 512][:10]
    assert all(a == b for s, a, b in zip(sizes, with_clusters, without) if a["parts"] == 1)
    # what clusters are for: a few wide tiles with long sums
    assert all(p["parts"] > 1 for p in plan([(128, 28672, 1024) + B200, (100, 11008, 4096) + B200, (256, 28672, 8192) + B200]))


def test_plans_fit_the_kernels(plan):
    """Shared memory, rows of an instruction, and whole groups of channels, over all sizes and on devices with few SMs."""
    smem, most_stages = 208 << 10, 40
    sizes = [(n, d, o) + device for device in (B200, (148, 0, 0), (20, 10, 4), (2, 1, 0), (1, 0, 0)) for n in TOKENS for d in SUMS for o in CHANNELS]
    for s, p in zip(sizes, plan(sizes)):
        n, d, _ = s[:3]
        rows, bn, parts, slices = p["rows"], p["bn"], p["parts"], p["slices"]
        assert bn % 16 == 0 and 32 <= bn <= 256 and rows % 8 == 0 and 1 <= rows <= 128, (s, p)
        if p["pair"]:
            assert n > 128 and rows == 128 and parts == slices == 1 and bn >= 128 and bn % 32 == 0, (s, p)
            continue
        assert rows == min(128, -(-n // 8) * 8) and parts in (1, 2, 4) and slices in (1, 2, 4) and min(parts, slices) == 1, (s, p)
        assert bn % (16 * parts) == 0 and slices * rows <= 128 and slices * bn <= 256 and (slices == 1 or n <= 64), (s, p)
        block = slices * (rows + bn) * 128
        slack = (128 - slices * rows) * 128 + 1024
        assert 1 <= p["per_stage"] <= -(-(-(-d // 128)) // (parts * slices)), (s, p)
        stages = min((smem - slack) // (p["per_stage"] * block), most_stages)
        assert stages >= 1 and stages * p["per_stage"] * block + slack <= smem, (s, p)
        assert (parts - 1) * 128 * (bn // parts + 4) * 4 + 1024 <= smem, (s, p)


def test_stages_and_clusters_where_they_were_measured(plan):
    """Tokens, entries of the sum, channels: stages of one block, of several, and clusters, each where the others took longer."""
    one = [(320, 4096, 4096), (576, 4096, 4096), (128, 4096, 11008), (80, 8192, 8192), (192, 8192, 8192), (512, 11008, 4096), (640, 12288, 2304), (900, 2048, 2048),
           (320, 11008, 4096), (384, 11008, 4096), (384, 13824, 5120), (1200, 8192, 1024), (129, 512, 1408)]
    for s, p in zip(one, plan([s + B200 for s in one])):
        assert p["parts"] == p["slices"] == p["per_stage"] == 1 and not p["pair"], (s, p)
    several = [(5, 13824, 5120), (33, 13824, 5120), (16, 28672, 8192), (16, 2048, 2048), (80, 4096, 1024), (100, 4096, 4096), (512, 4096, 1024)]
    for s, p in zip(several, plan([s + B200 for s in several])):
        assert p["parts"] == p["slices"] == 1 and p["per_stage"] > 1 and not p["pair"], (s, p)
    clusters = [(256, 11008, 4096), (128, 13824, 5120), (384, 28672, 4096), (400, 18944, 3584), (256, 5461, 2049), (640, 8192, 1024), (256, 28672, 8192)]
    for s, p in zip(clusters, plan([s + B200 for s in clusters])):
        assert p["parts"] > 1, (s, p)


def test_narrow_pairs_take_the_place_of_tiles_where_they_gain(plan):
    """Tokens, entries of the sum, channels.  Measured in tiles and in narrow pairs: 29.5 and 32.1 us, 30.6 and 32.6, 27.7 and 29.2, 30.0 and
    31.8, 21.0 and 22.1; then 68.7 and 67.0, 55.6 and 55.0, 138.6 and 134.9; and beside wide pairs, 52.4 and 51.3, 75.8 and 73.5."""
    tiles = [(900, 12288, 2304), (1024, 12288, 2304), (2560, 8192, 1024), (2900, 8192, 1024), (3328, 4096, 1024)]
    assert not any(p["pair"] for p in plan([s + (148, 0, 0) for s in tiles]))
    narrow = [(1200, 14336, 4096), (1200, 11008, 4096), (1280, 28672, 4096), (900, 8192, 8192), (1408, 8192, 8192)]
    assert all(p["pair"] and p["bn"] < 256 for p in plan([s + B200 for s in narrow]))
    wide = [(4096, 8192, 28672), (2048, 4096, 11008), (4096, 4096, 4096)]
    assert all(p["pair"] and p["bn"] == 256 for p in plan([s + B200 for s in wide]))


# ---- activations ----------------------------------------------------------------------------------------------------

def test_the_stated_error_of_the_normal_distribution():
    """The polynomial of by_normal with the coefficients as they stand in the source, against the function that it is fitted to."""
    np, special = pytest.importorskip("numpy"), pytest.importorskip("scipy.special")
    source = open(os.path.join(cuda_build.CSRC, "epilogue.cuh")).read()
    comment, body = source[source.index("// z Phi(z)."):source.index("float by_normal(")], _body(source, "float by_normal(")
    number = lambda text: float(np.float32(text))
    root = number(re.search(r"__fmaf_rn\(([\d.]+)f, t, 1\.0f\)", body)[1])
    coefficients = [number(re.search(r"float p = (-?[\d.]+)f", body)[1])] + [number(c) for c in re.findall(r"p = __fmaf_rn\(p, s, (-?[\d.]+)f\)", body)]
    assert len(coefficients) == 9 and abs(root * 8 ** 0.5 - 1) < 2 ** -23
    exact, rounded = (float(v) for v in re.search(r"off by ([\d.]+e-\d+) of its value, and with the roundings of float32 ([\d.]+e-\d+)", comment.replace("\n// ", " ")).groups())
    t = np.linspace(0, 14, 400001, dtype=np.float32).astype(np.float64)
    want = 0.5 * special.erfcx(t / np.sqrt(2))
    s, p = 1 / (1 + root * t), np.zeros_like(t)
    for c in coefficients:
        p = p * s + c
    worst = np.abs(s * p / want - 1).max()
    assert 0.95 * exact < worst < exact
    single = lambda v: v.astype(np.float32).astype(np.float64)
    s, p = single(1 / single(root * t + 1)), np.zeros_like(t)
    for c in coefficients:
        p = single(p * s + c)
    assert 0.9 * rounded < np.abs(single(p * s) / want - 1).max() < 1.1 * rounded
    assert 1.1 * rounded < 5 * 2.0 ** -22 / 2              # less than half of what the header allows where t is small
