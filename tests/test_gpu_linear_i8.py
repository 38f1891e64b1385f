"""8-bit linear layers against the plain statement.  Codes and scales are compared bit for bit.  The product is
exact in int32; what follows is the conversion of the sum, two scalings and a bias, four float32 roundings of values
no larger than |sum| s u + |b|, and one rounding to 16 bits:
    |y - ref| <= 4 * 2^-24 * mag + half an ulp,   the half ulp taken at |ref| (1 + 2^-7) to cover binade edges."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2410_13056_b200 import binding as B
from paper_2410_13056_b200 import serving

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]


def _tokens(n, d, dtype, seed):
    g = np.random.default_rng(seed)
    x = g.normal(size=(n, d)) * np.exp(0.5 * g.normal(size=d))
    x[:, g.integers(0, d)] *= 30.0
    return torch.from_numpy(x).to(dtype)


def _weights(d_out, d_in, seed, pad=0):
    g = np.random.default_rng(seed)
    ld = (d_in + 15) // 16 * 16 + pad
    store = torch.from_numpy(g.integers(-127, 128, size=(d_out, ld)).astype(np.int8))  # the padding is not zero
    scale = torch.from_numpy((0.001 * np.exp(g.normal(size=d_out))).astype(np.float32))
    return store.cuda()[:, :d_in], scale.cuda()


def _check_product(y, codes, scale, wc, ws, bias, dtype):
    want, mag = ref.linear(codes, scale, wc.cpu().numpy(), ws.cpu().numpy(), None if bias is None else bias.float().cpu().numpy())
    got = y.float().cpu().numpy().astype(np.float64)
    tol = 4 * 2.0 ** -24 * mag + ref.half_ulp(np.abs(want) * (1 + 2.0 ** -7), dtype)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (2, 16), (5, 511), (33, 4096), (2, 16384), (3, 20001), (1, 131072)])
def test_quantize_tokens_bit_exact(n, d, dtype):
    x = _tokens(n, d, dtype, 3 * n + d)
    x[0] = 0 if n > 1 else x[0]                       # a row of zeros
    if n > 2:
        x[2] = (x[2].float() * 2.0 ** -12).to(dtype)
    ld = (d + 15) // 16 * 16 + 16
    codes = torch.full((n, ld), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((n,), -1.0, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cmpq_quantize_tokens(x.cuda(), codes[:, :d], scale, word)
    c, s = ref.quantize_tokens(x.float().numpy())
    assert np.array_equal(codes[:, :d].cpu().numpy(), c)
    assert np.array_equal(scale.cpu().numpy(), s)
    assert torch.all(codes[:, d: (d + 15) // 16 * 16] == 0) and torch.all(codes[:, (d + 15) // 16 * 16:] == 99)
    assert int(word) == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_tokens_strides_tiny_rows_and_nonfinite(dtype):
    big = _tokens(6, 107, dtype, 5).cuda()
    for view in (big[:, 3:104], big[::2, 1:], big[1:, :96]):   # rows that start on odd addresses, row strides
        n, d = view.shape
        codes = torch.zeros(n, (d + 15) // 16 * 16, dtype=torch.int8, device="cuda")
        scale = torch.zeros(n, device="cuda")
        B.cmpq_quantize_tokens(view, codes[:, :d], scale)
        c, s = ref.quantize_tokens(view.float().cpu().numpy())
        assert np.array_equal(codes[:, :d].cpu().numpy(), c) and np.array_equal(scale.cpu().numpy(), s)
    if dtype == torch.bfloat16:                        # below the smallest magnitude that gets a scale, and at it
        x = torch.tensor([[2.0 ** -121] * 8, [2.0 ** -120] * 8], dtype=dtype, device="cuda")
        codes, scale = torch.ones(2, 16, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda")
        B.cmpq_quantize_tokens(x, codes[:, :8], scale)
        assert float(scale[0]) == 0 and torch.all(codes[0] == 0) and torch.all(codes[1, :8] == 127)
    for value in (float("nan"), float("inf"), float("-inf")):
        x = _tokens(4, 40, dtype, 6)
        x[2, 39] = value
        word = torch.zeros(1, dtype=torch.int32, device="cuda")
        codes, scale = torch.zeros(4, 48, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
        B.cmpq_quantize_tokens(x.cuda(), codes[:, :40], scale, word)
        assert int(word) == 1
        c, s = ref.quantize_tokens(x[:2].float().numpy())  # the other rows are not touched by it
        assert np.array_equal(codes[:2, :40].cpu().numpy(), c) and np.array_equal(scale[:2].cpu().numpy(), s)


SIZES = [(1, 1, 1), (1, 16, 16), (1, 4096, 129), (2, 100, 33), (3, 257, 1000), (7, 1000, 64), (8, 64, 4096), (9, 130, 257),
         (16, 4096, 640), (17, 512, 128), (31, 33, 31), (33, 2049, 300), (64, 128, 128), (65, 300, 513), (100, 4096, 1024),
         (127, 96, 255), (128, 128, 256), (129, 1025, 257), (200, 513, 1030), (257, 256, 511), (300, 4097, 770),
         (513, 64, 129), (700, 640, 2049), (1025, 272, 384)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_linear_against_the_plain_product(n, d_in, d_out, dtype):
    x = _tokens(n, d_in, dtype, n + d_in)
    wc, ws = _weights(d_out, d_in, d_out, pad=16 * (n % 3))
    bias = None if n % 2 else torch.from_numpy(np.random.default_rng(n).normal(size=d_out)).to(dtype).cuda()
    layer = serving.Int8Linear(wc, ws, bias)
    room = torch.full((n + 1, d_out + 3), 7.0, dtype=dtype, device="cuda")   # a guard around the output
    y = layer(x.cuda(), out=room[:n, :d_out])
    assert torch.all(room[n:] == 7.0) and torch.all(room[:, d_out:] == 7.0)
    codes, scale = ref.quantize_tokens(x.float().numpy())
    _check_product(y, codes, scale, wc, ws, bias, dtype)
    assert torch.equal(layer(x.cuda()), y)             # the same bytes in a plain output, on a second call


def test_matmul_takes_codes_with_any_padding():
    n, d_in, d_out = 21, 333, 190
    g = np.random.default_rng(8)
    xc = torch.from_numpy(g.integers(-127, 128, size=(n, 352)).astype(np.int8)).cuda()
    xs = torch.from_numpy(np.abs(g.normal(size=n)).astype(np.float32)).cuda()
    wc, ws = _weights(d_out, d_in, 9, pad=32)
    ws_buf = torch.empty(B.cmpq_linear_i8_ws_bytes(n, d_in, d_out), dtype=torch.uint8, device="cuda")
    y = torch.empty(n, d_out, dtype=torch.bfloat16, device="cuda")
    B.cmpq_matmul_i8(xc[:, :d_in], xs, wc, ws, None, y, ws_buf)
    _check_product(y, xc[:, :d_in].cpu().numpy(), xs.cpu().numpy(), wc, ws, None, torch.bfloat16)


@pytest.mark.parametrize("n", [1, 20, 200])
def test_largest_sums_are_exact(n):
    """All codes at +-127 over a long row: the sum passes 2^24 by far and has to stay exact."""
    d_in, d_out = 16384, 160
    x = torch.ones(n, d_in, dtype=torch.bfloat16)
    x[:, 1::3] = -1
    wc = torch.full((d_out, d_in), 127, dtype=torch.int8, device="cuda")
    wc[1::2] = -127
    wc[:, 5] = 1
    ws = torch.full((d_out,), 2.0 ** -20, device="cuda")
    layer = serving.Int8Linear(wc, ws)
    y = layer(x.cuda())
    codes, scale = ref.quantize_tokens(x.float().numpy())
    _check_product(y, codes, scale, wc, ws, None, torch.bfloat16)
    wc.fill_(127)
    y = layer(torch.ones(n, d_in, dtype=torch.bfloat16, device="cuda"))
    _check_product(y, np.full((n, d_in), 127, np.int8), scale, wc, ws, None, torch.bfloat16)


def test_long_rows():
    n, d_in, d_out = 5, 131072, 48
    x = _tokens(n, d_in, torch.float16, 1)
    wc, ws = _weights(d_out, d_in, 2)
    y = serving.Int8Linear(wc, ws * 0.01)(x.cuda())
    codes, scale = ref.quantize_tokens(x.float().numpy())
    _check_product(y, codes, scale, wc, ws * 0.01, None, torch.float16)


def test_no_tokens_and_other_streams():
    wc, ws = _weights(100, 64, 3)
    layer = serving.Int8Linear(wc, ws)
    assert layer(torch.empty(0, 64, dtype=torch.float16, device="cuda")).shape == (0, 100)
    x = [_tokens(70 + i, 64, torch.float16, i).cuda() for i in range(4)]
    want = [layer(t) for t in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = []
    for t, s in zip(x, streams):
        with torch.cuda.stream(s):
            got.append([layer(t) for _ in range(20)])
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        assert all(torch.equal(w, y) for y in many)


def test_from_weight_and_refusals():
    g = torch.Generator().manual_seed(1)
    w = (torch.randn(70, 130, generator=g) * 0.02).to(torch.bfloat16).cuda()
    x = torch.randn(12, 130, generator=g).to(torch.bfloat16).cuda()
    layer = serving.Int8Linear.from_weight(w)
    want = x.double() @ w.double().t()
    got = layer(x).double()
    # quantization error: each of the 130 products is off by at most (1/254 + 1/254) of the two largest magnitudes
    assert torch.all((got - want).abs() <= 130 * (2 / 254) * x.double().abs().amax(1, True) * w.double().abs().amax(1) + 0.01)
    assert (got - want).norm() < 0.02 * want.norm()
    with pytest.raises(ValueError):
        layer(x[:, :129])
    with pytest.raises(ValueError):
        serving.Int8Linear(layer.w_codes[:, 1:], layer.w_scale)
    with pytest.raises(TypeError):
        layer(x.float())
    y = torch.full((12, 70), 3.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.CmpqError) as e:
        B.cmpq_linear_i8(x, layer.w_codes, layer.w_scale, None, y, torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    with pytest.raises(B.CmpqError) as e:
        B.cmpq_linear_i8(x, layer.w_codes[:, :120], layer.w_scale, None, y, torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert torch.all(y == 3.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", [(1900, 520, 4400), (2500, 129, 6001), (300, 1040, 18950)])
def test_many_tiles(n, d_in, d_out, dtype):
    """More tiles than SMs, so that blocks walk over several; sums of integers below 2^53 are exact in float64."""
    x = _tokens(n, d_in, dtype, 7)
    wc, ws = _weights(d_out, d_in, 8)
    bias = torch.from_numpy(np.random.default_rng(9).normal(size=d_out)).to(dtype).cuda()
    y = serving.Int8Linear(wc, ws, bias)(x.cuda())
    codes, scale = ref.quantize_tokens(x.float().numpy())
    acc = codes.astype(np.float64) @ wc.cpu().numpy().astype(np.float64).T
    want = acc * scale[:, None].astype(np.float64) * ws.cpu().numpy().astype(np.float64)
    b = bias.float().cpu().numpy().astype(np.float64)
    tol = 4 * 2.0 ** -24 * (np.abs(want) + np.abs(b)) + ref.half_ulp(np.abs(want + b) * (1 + 2.0 ** -7), dtype)
    bad = np.abs(y.float().cpu().numpy().astype(np.float64) - (want + b)) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5])


@pytest.mark.parametrize("n", [1, 37, 300])
def test_calls_one_behind_the_other_see_their_own_scales(n):
    """The product starts while its tokens are quantized, in the work space of the call before: inputs whose scales are
    2^12 apart take turns, in a stream of calls that is never waited for."""
    wc, ws = _weights(1500, 640, 4)
    layer = serving.Int8Linear(wc, ws)
    x = [(_tokens(n, 640, torch.bfloat16, 1).float() * f).bfloat16().cuda() for f in (1.0, 2.0 ** 12, 2.0 ** -12)]
    want = [layer(t) for t in x]
    torch.cuda.synchronize()
    got = [layer(x[i % 3]) for i in range(600)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 3]) for i, y in enumerate(got))
    codes, scale = ref.quantize_tokens(x[1].float().cpu().numpy())
    _check_product(want[1], codes, scale, wc, ws, None, torch.bfloat16)


@pytest.mark.parametrize("n", [1, 300])
def test_mark_in_the_work_space_starts_from_zero(n):
    """Calls without a word keep the mark of a kernel that gave up in the work space, whose contents are undefined before
    the call: it reads 0 after a product that ended well, and the caller's word is used where there is one."""
    d_in, d_out = 256, 512
    wc, ws = _weights(d_out, d_in, 4)
    x = _tokens(n, d_in, torch.float16, 2).cuda()
    xc, xs = torch.empty(n, d_in, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    B.cmpq_quantize_tokens(x, xc, xs)
    size = B.cmpq_linear_i8_ws_bytes(n, d_in, d_out)
    want = serving.Int8Linear(wc, ws)(x)
    for call in ("matmul", "linear", "word"):
        buf = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        mark = buf[size - 256: size - 252].view(torch.int32)
        y, word = torch.empty_like(want), torch.zeros(1, dtype=torch.int32, device="cuda")
        if call == "matmul":
            B.cmpq_matmul_i8(xc, xs, wc, ws, None, y, buf)
        else:
            B.cmpq_linear_i8(x, wc, ws, None, y, buf, word if call == "word" else None)
        assert int(mark if call != "word" else word) == 0 and torch.equal(y, want), call
        B.cmpq_check_cache(mark if call != "word" else word)
