"""The norm on the way into 8 bits, the linear layer with its epilogue, the gated feed-forward block and the decoder layer of
them.  Codes are compared bit for bit, the rest within the bounds that layer_ref derives."""
import numpy as np
import pytest
import torch

import layer_ref as ref
from paper_2410_13056_b200 import binding as B
from paper_2410_13056_b200 import serving

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]
ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]
EPS = 1e-5


def _tokens(n, d, dtype, seed):
    g = np.random.default_rng(seed)
    x = g.normal(size=(n, d)) * np.exp(0.5 * g.normal(size=d))
    x[:, g.integers(0, d)] *= 30.0
    return torch.from_numpy(x).to(dtype).cuda()


def _norm(d, dtype, seed):
    g = torch.from_numpy(1 + 0.3 * np.random.default_rng(seed).normal(size=d)).to(dtype)
    g[:: 7] *= -1
    return g.cuda()


def _weights(d_out, d_in, dtype, seed, bias=False, pad=0):
    """A layer whose outputs are of the size of its inputs' root mean square."""
    g = np.random.default_rng(seed)
    ld = (d_in + 15) // 16 * 16 + pad
    store = torch.from_numpy(g.integers(-127, 128, size=(d_out, ld)).astype(np.int8)).cuda()  # the padding is not zero
    scale = torch.from_numpy((np.exp(0.3 * g.normal(size=d_out)) / (73 * np.sqrt(d_in))).astype(np.float32)).cuda()
    b = torch.from_numpy(0.3 * g.normal(size=d_out)).to(dtype).cuda() if bias else None
    return serving.Int8Linear(store[:, :d_in], scale, b)


def _np(t):
    return None if t is None else t.float().cpu().numpy()


def _parts(layer):
    return layer.w_codes.cpu().numpy(), layer.w_scale.cpu().numpy(), _np(layer.bias)


def _compare(y, want, tol):
    got = y.float().cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])


# ---- norm ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (2, 16), (5, 511), (33, 4096), (4, 4100), (3, 8192), (2, 16384), (3, 20001), (1, 131072)])
def test_norm_quantize_codes_bit_exact(n, d, dtype):
    x, g = _tokens(n, d, dtype, n + d), _norm(d, dtype, d)
    if n > 1:
        x[0] = 0
    ld = (d + 15) // 16 * 16 + 16
    codes, scale = torch.full((n, ld), 99, dtype=torch.int8, device="cuda"), torch.full((n,), -1.0, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cmpq_norm_quantize_tokens(x, g, EPS, codes[:, :d], scale, word)
    c, s, rel = ref.norm_quantize(_np(x), _np(g), EPS)
    assert np.array_equal(codes[:, :d].cpu().numpy(), c)
    assert np.all(np.abs(scale.cpu().numpy() - s) <= rel * s)
    assert torch.all(codes[:, d: (d + 15) // 16 * 16] == 0) and torch.all(codes[:, (d + 15) // 16 * 16:] == 99)
    assert int(word) == 0
    again = serving.quantize_tokens(x, g, EPS)
    assert torch.equal(again[0], codes[:, :d]) and torch.equal(again[1], scale)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_of_rows_whose_squares_pass_float32(dtype):
    """In one kernel, in the kernels of their own, and beside rows of ordinary size."""
    d, ff = 1024, 6000
    block, g = _block(1, d, ff, d, dtype, "silu", False), _norm(d, dtype, 8)
    x = _tokens(5, d, dtype, 7)
    want = block(x, norm=g, eps=2.0 ** -60)
    if dtype == torch.bfloat16:                            # powers of two that the norm takes out again
        for row, p in ((0, 90), (2, -20), (3, 100)):
            x[row] = (x[row].float() * 2.0 ** p).to(dtype)
    for n in (5, 4):
        assert torch.equal(block(x[:n], norm=g, eps=2.0 ** -60), want[:n])
    block.check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_quantize_strides_and_extremes(dtype):
    big, gs = _tokens(6, 107, dtype, 5), _norm(108, dtype, 6)
    for view, g in ((big[:, 3:104], gs[1:102]), (big[::2, 1:], gs[2:]), (big[1:, :96], gs[:96]), (big[:, 8:104], gs[3:99])):
        codes, scale = serving.quantize_tokens(view, g.contiguous() if g.storage_offset() % 2 else g, EPS)
        c, s, rel = ref.norm_quantize(_np(view), _np(g), EPS)
        assert np.array_equal(codes.cpu().numpy(), c) and np.all(np.abs(scale.cpu().numpy() - s) <= rel * s)
    for d in (64, 20000):  # rows that stay in registers, and rows that are read again
        x, g = _tokens(8, d, dtype, 7).float(), _norm(d, dtype, 8)
        powers = [0, -13, -20, 8, -2, 3, 5, -9] if dtype == torch.float16 else [0, -40, -70, 60, 66, 90, 118, -100]
        for i, p in enumerate(powers):
            x[i] *= 2.0 ** p
        x[3, 1:] *= 2.0 ** -6
        x = x.clamp(-torch.finfo(dtype).max / 8, torch.finfo(dtype).max / 8).to(dtype)
        for eps in (EPS, 2.0 ** -126, 1.0):
            codes, scale = serving.quantize_tokens(x, g, eps)
            c, s, rel = ref.norm_quantize(_np(x), _np(g), eps)
            assert np.array_equal(codes.cpu().numpy(), c)
            # scales at the end of float32's range lose bits: half a unit of the smallest
            assert np.all(np.abs(scale.cpu().numpy() - s) <= rel * s + 2.0 ** -149), (eps, scale, s)
    g = _norm(40, dtype, 9)
    for value in (float("nan"), float("inf"), float("-inf")):
        for zero in (False, True):
            x, w = _tokens(4, 40, dtype, 6), g.clone()
            x[2, 39] = value
            w[39] = 0.0 if zero else w[39]
            word = torch.zeros(1, dtype=torch.int32, device="cuda")
            codes, scale = torch.zeros(4, 48, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
            B.cmpq_norm_quantize_tokens(x, w, EPS, codes[:, :40], scale, word)
            assert int(word) == 1
            c, s, rel = ref.norm_quantize(_np(x[:2]), _np(w), EPS)
            assert np.array_equal(codes[:2, :40].cpu().numpy(), c) and np.all(np.abs(scale[:2].cpu().numpy() - s) <= rel * s)
    x = _tokens(5, 200, dtype, 3)
    codes, scale = torch.zeros(5, 208, dtype=torch.int8, device="cuda"), torch.zeros(5, device="cuda")
    B.cmpq_quantize_tokens(x, codes[:, :200], scale)
    same = serving.quantize_tokens(x)
    assert torch.equal(same[0], codes[:, :200]) and torch.equal(same[1], scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", [(1024, 1), (1025, 4096), (1031, 511), (1500, 4104), (1100, 8192), (1027, 5003), (1025, 16384), (1030, 12801), (1024, 16400)])
def test_many_rows_have_the_bytes_of_few(n, d, dtype):
    x, g = _tokens(n, d, dtype, n), _norm(d, dtype, d)
    x[7] = 0
    if dtype == torch.bfloat16:
        x[9] = (x[9].float() * 2.0 ** 100).to(dtype)
        x[11] = (x[11].float() * 2.0 ** -60).to(dtype)
    for view, w in ((x, g), (x[:, 1:], g[1:].clone())) if d > 1 else ((x, g),):
        codes, scale = serving.quantize_tokens(view, w, EPS)
        for lo in (0, n - 500):
            c, s = serving.quantize_tokens(view[lo: lo + 500], w, EPS)
            assert torch.equal(codes[lo: lo + 500], c) and torch.equal(scale[lo: lo + 500], s)
    c, s, rel = ref.norm_quantize(_np(x[:20]), _np(g), EPS)
    codes, scale = serving.quantize_tokens(x, g, EPS)
    assert np.array_equal(codes[:20].cpu().numpy(), c) and np.all(np.abs(scale[:20].cpu().numpy() - s) <= rel * s)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    x[n - 1, d - 1] = float("nan")
    room = torch.full((n, (d + 15) // 16 * 16 + 16), 99, dtype=torch.int8, device="cuda")
    B.cmpq_norm_quantize_tokens(x, g, EPS, room[:, :d], scale, word)
    assert int(word) == 1 and torch.equal(room[: n - 1, :d], codes[: n - 1])
    pad = (d + 15) // 16 * 16
    assert torch.all(room[: n - 1, d: pad] == 0) and torch.all(room[:, pad:] == 99)


# ---- linear layer ----------------------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 512, 129), (2, 100, 33), (4, 4097, 1000), (3, 12800, 300), (1, 12801, 96), (4, 64, 40000), (1, 4096, 19000), (7, 1000, 64), (9, 130, 257), (31, 33, 31), (65, 300, 513), (128, 128, 256), (129, 1025, 257),
         (300, 4097, 770), (513, 64, 129), (700, 640, 2049), (1900, 520, 4400)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_linear_with_its_epilogue(n, d_in, d_out, dtype):
    x = _tokens(n, d_in, dtype, n + d_in)
    layer = _weights(d_out, d_in, dtype, d_out, bias=n % 2 == 0, pad=16 * (n % 3))
    res = _tokens(n + 1, d_out + 3, dtype, 2)
    parts = _parts(layer)
    for i, act in enumerate(ACTS):
        g = _norm(d_in, dtype, 4) if i % 2 == 0 or n == 65 else None
        r = (res[:n, :d_out], res[1:, 3:], None)[i % 3]                       # rows on 16 bytes or not
        room = torch.full((n + 1, d_out + 5), 7.0, dtype=dtype, device="cuda")  # a guard around the output
        y = layer(x, out=room[:n, :d_out], activation=act, residual=r, norm=g, eps=EPS)
        assert torch.all(room[n:] == 7.0) and torch.all(room[:, d_out:] == 7.0)
        z, err = ref.linear(*ref.norm_quantize(_np(x), None if g is None else _np(g), EPS), *parts)
        _compare(y, *ref.finish(z, err, act, _np(r), dtype))
        assert torch.equal(layer(x, activation=act, residual=r, norm=g, eps=EPS), y)
        if r is not None:
            into = r.clone()
            assert torch.equal(layer(x, out=into, activation=act, residual=into, norm=g, eps=EPS), y)   # in place
    layer.check()


@pytest.mark.parametrize("n", [1, 4, 5, 200])
def test_linear_in_place(n):
    """out may be x, or overlap it."""
    d, dtype = 4096, torch.bfloat16
    layer, g, x = _weights(d, d, dtype, 1, True), _norm(d, dtype, 2), _tokens(n, d, dtype, 3)
    want = layer(x, activation="silu", norm=g, residual=x)
    for _ in range(20):
        into = x.clone()
        assert torch.equal(layer(into, out=into, activation="silu", norm=g, residual=into), want)
    room = torch.zeros(n, 2 * d + 7, dtype=dtype, device="cuda")
    for _ in range(20):
        room[:, :d] = x
        y = layer(room[:, :d], out=room[:, 7: d + 7], activation="silu", norm=g)
    assert torch.equal(y, layer(x, activation="silu", norm=g))


def test_activations_over_their_whole_range():
    """One input channel and one output channel per argument: z runs over every size of either sign."""
    args = np.concatenate([np.linspace(-30, 30, 4001), -np.logspace(-30, 4, 200), np.logspace(-30, 4, 200), [-88.5, -89.0, -104.0, 0.0]])
    for dtype in DTYPES:
        scale = torch.from_numpy(np.abs(args).astype(np.float32)).cuda()
        codes = torch.zeros(len(args), 16, dtype=torch.int8, device="cuda")
        codes[:, 0] = torch.from_numpy(np.where(args < 0, -1, 1).astype(np.int8)).cuda()
        layer = serving.Int8Linear(codes[:, :1], scale)
        x = torch.ones(1, 1, dtype=dtype, device="cuda")
        z, err = ref.linear(*ref.norm_quantize(_np(x), None, 0), *_parts(layer))
        for act in ACTS[1:]:
            y, tol = ref.finish(z, err, act, None, dtype)
            if dtype == torch.float16:
                keep = np.abs(y) < 65000
                y, tol, got = y[:, keep[0]], tol[:, keep[0]], layer(x, activation=act)[:, torch.from_numpy(keep[0]).cuda()]
            else:
                got = layer(x, activation=act)
            _compare(got, y, tol)
        assert torch.equal(layer(x, activation="none"), layer(x))
    # sums that pass float32
    codes = torch.zeros(2, 16, dtype=torch.int8, device="cuda")
    codes[0, 0], codes[1, 0] = -127, 127
    layer = serving.Int8Linear(codes[:, :1], torch.full((2,), 3e38, device="cuda"))
    assert torch.equal(layer(x), torch.tensor([[-np.inf, np.inf]], dtype=dtype, device="cuda"))
    for act, low in (("relu", 0.0), ("gelu", 0.0), ("silu", np.nan), ("gelu_tanh", np.nan)):
        y = layer(x, activation=act)[0].float().cpu().numpy()
        assert y[1] == np.inf and (y[0] == low or np.isnan(y[0]) and np.isnan(low)), (act, y)


# ---- gated block -----------------------------------------------------------------------------------------------

GATED = [(1, 1, 1, 1), (1, 16, 8, 16), (1, 512, 1408, 512), (2, 100, 37, 33), (3, 4096, 130, 64), (5, 130, 2590, 65), (8, 256, 1024, 256), (9, 257, 1500, 129),
         (16, 640, 300, 1000), (17, 33, 511, 2000), (33, 512, 700, 512), (64, 128, 1200, 384), (65, 300, 513, 77), (100, 1024, 640, 1024), (128, 512, 512, 512),
         (129, 255, 257, 300), (300, 384, 1000, 520), (513, 200, 640, 200), (1500, 130, 1100, 260)]


# one kernel does all of these: large layers, a few tokens; long and short sums, many tiles and parts for a block, sizes that
# fill nothing
FEW = [(1, 2050, 5461, 2049), (2, 4096, 2001, 4097), (3, 130, 80000, 65), (4, 12800, 700, 300), (1, 64, 131072, 64), (4, 8, 1000, 20000), (2, 16, 64, 262144),
       (4, 1024, 6000, 1024), (3, 8192, 1000, 8192), (1, 1536, 4096, 1536), (4, 13000, 700, 300), (4, 4097, 1500, 4100), (1, 24, 5000, 50000), (2, 100, 9000, 30000)]


def _block(n, d_in, d_ff, d_out, dtype, act, bias):
    gate, up = (_weights(d_ff, d_in, dtype, s, bias, pad=16 * (n % 2)) for s in (1, 2))
    return serving.GatedMLP8(gate, up, _weights(d_out, d_ff, dtype, 3, bias), act)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_ff,d_out", GATED + FEW)
def test_gated_block(n, d_in, d_ff, d_out, dtype):
    x = _tokens(n, d_in, dtype, n + d_in)
    res = _tokens(n + 1, d_out + 3, dtype, 2)
    for i, act in enumerate(ACTS if n < 500 and (n, d_in, d_ff, d_out) not in FEW else ["silu", "gelu"]):
        block = _block(n, d_in, d_ff, d_out, dtype, act, i % 2 == 1)
        g = _norm(d_in, dtype, 4) if i % 3 != 1 else None
        r = (res[:n, :d_out], None, res[1:, 3:])[i % 3]
        room = torch.full((n + 1, d_out + 5), 7.0, dtype=dtype, device="cuda")
        y = block(x, out=room[:n, :d_out], residual=r, norm=g, eps=EPS)
        assert torch.all(room[n:] == 7.0) and torch.all(room[:, d_out:] == 7.0)
        want, tol = ref.gated(_np(x), None if g is None else _np(g), EPS, *map(_parts, (block.gate, block.up, block.down)), act, _np(r), dtype)
        _compare(y, want, tol)
        assert torch.equal(block(x, residual=r, norm=g, eps=EPS), y)
        if d_in == d_out:
            into = x.clone()
            want = block(x, residual=x, norm=g, eps=EPS)
            assert torch.equal(block(into, out=into, residual=into, norm=g, eps=EPS), want)
        block.check()


@pytest.mark.parametrize("d,ff", [(384, 1500), (1024, 6000)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_token_has_the_same_bytes_in_every_batch(dtype, d, ff):
    """Kernels are chosen by the number of tokens; what a token gets does not depend on it."""
    block, x, g = _block(1, d, ff, d, dtype, "silu", True), _tokens(600, d, dtype, 1), _norm(d, dtype, 2)
    layer = block.down
    h = _tokens(600, ff, dtype, 3)
    y = block(x, residual=x, norm=g)
    z = layer(h, activation="gelu", residual=x)
    for n in (1, 2, 3, 4, 5, 8, 9, 32, 64, 65, 128, 129, 300):
        for at in (0, 600 - n):
            part = slice(at, at + n)
            assert torch.equal(block(x[part], residual=x[part], norm=g), y[part]), n
            assert torch.equal(layer(h[part], activation="gelu", residual=x[part]), z[part]), n


# a few tokens and long sums: tiles whose sums are cut into slices, with slices that end early or hold one block fewer
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", [(5, 2049, 500), (9, 4097, 1000), (16, 2500, 2049), (25, 2177, 130), (32, 11000, 515), (33, 4225, 770), (40, 4097, 97),
                                          (57, 5000, 2051), (64, 8200, 1001)])
def test_long_sums_of_a_few_tokens(n, d_in, d_out, dtype):
    test_linear_with_its_epilogue(n, d_in, d_out, dtype)
    test_gated_block(n, d_in, d_out, d_out, dtype)
    for i, layer in enumerate((_weights(d_out, d_in, dtype, d_out, True), _weights(d_out, d_in, dtype, d_out, False, pad=16))):
        x = _tokens(n, d_in, dtype, i)
        y = layer(x)
        _compare(y, *ref.finish(*ref.linear(*ref.norm_quantize(_np(x), None, EPS), *_parts(layer)), "none", None, dtype))


# tiles whose sums two or four blocks share: parts that end early, one or more tiles of tokens, channels that fill no part, both
# halves of a gated tile
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", [(5, 28672, 600), (20, 13000, 1100), (33, 5641, 1024), (64, 11000, 515), (100, 11008, 2050), (127, 8192, 1000), (128, 20480, 33),
                                          (129, 11008, 450), (200, 28672, 1030), (300, 9000, 520), (512, 8193, 257)])
def test_long_sums_over_a_cluster(n, d_in, d_out, dtype):
    test_long_sums_of_a_few_tokens(n, d_in, d_out, dtype)


@pytest.mark.parametrize("n", [1, 20, 300])
def test_largest_sums_are_exact(n):
    """All codes at +-127 over long rows, in both of the block's products."""
    d, ff = 16384, 8192
    one = lambda d_out, d_in, s: serving.Int8Linear(torch.full((d_out, d_in), 127, dtype=torch.int8, device="cuda"), torch.full((d_out,), s, device="cuda"))
    gate, up, down = one(ff, d, 2.0 ** -21), one(ff, d, -2.0 ** -21), one(160, ff, 2.0 ** -20)
    gate.w_codes[3::2] = -127
    x = torch.ones(n, d, dtype=torch.bfloat16, device="cuda")
    y = serving.GatedMLP8(gate, up, down, "none")(x)
    want, tol = ref.gated(_np(x[:1]), None, 0, *map(_parts, (gate, up, down)), "none", None, torch.bfloat16)
    _compare(y[:1], want, tol)
    assert torch.equal(y, y[:1].expand_as(y))


def test_layer_of_a_workload_size():
    """4096 -> 11008 -> 4096 on the few tokens whose reference stays quick."""
    for n, dtype in ((1, torch.bfloat16), (6, torch.float16)):
        block, x, g = _block(n, 4096, 11008, 4096, dtype, "silu", False), _tokens(n, 4096, dtype, 5), _norm(4096, dtype, 6)
        want, tol = ref.gated(_np(x), _np(g), EPS, *map(_parts, (block.gate, block.up, block.down)), "silu", _np(x), dtype)
        _compare(block(x, residual=x, norm=g, eps=EPS), want, tol)


def test_reports():
    d, ff = 64, 200
    for n in (1, 40, 400):
        block = _block(n, d, ff, d, torch.float16, "relu", False)
        x = _tokens(n, d, torch.float16, 1).clamp(-4, 4)
        block(x)
        block.check()
        bad = x.clone()
        bad[-1, 5] = float("nan")
        block(bad)
        with pytest.raises(B.CmpqError) as e:
            block.check()
        assert e.value.status == 6
        y = block(x)
        block.check()
        huge = x.clone()
        huge[0] *= 4000                                   # h of this token passes fp16
        z = block(huge)
        with pytest.raises(B.CmpqError) as e:
            block.check()
        assert e.value.status == 6 and torch.equal(z[1:], y[1:])
        block.word.fill_(8)
        with pytest.raises(B.CmpqError) as e:
            block.check()
        assert e.value.status == 5
        assert torch.equal(block(x), y)
        block.check()
        for part in (block.gate, block.up, block.down):
            part.check()                                  # the block's reports are its own
        layer = block.gate
        layer(bad, norm=_norm(d, torch.float16, 1), activation="silu")
        with pytest.raises(B.CmpqError) as e:
            layer.check()
        assert e.value.status == 6


@pytest.mark.parametrize("n", [1, 4])
def test_reports_of_the_one_kernel(n):
    d, ff = 1024, 6000
    block, x = _block(n, d, ff, d, torch.float16, "silu", True), _tokens(n, d, torch.float16, 1)
    y = block(x)
    block.check()
    for value, at in ((float("nan"), n - 1), (float("inf"), 0)):
        bad = x.clone()
        bad[at, 1000] = value
        z = block(bad)
        with pytest.raises(B.CmpqError) as e:
            block.check()
        keep = [i for i in range(n) if i != at]
        assert e.value.status == 6 and torch.equal(z[keep], y[keep])
    huge = x.clone()
    huge[0] *= 1000                                       # its h passes fp16
    z = block(huge)
    with pytest.raises(B.CmpqError) as e:
        block.check()
    assert e.value.status == 6 and torch.equal(z[1:], y[1:])
    assert torch.equal(block(x), y)
    block.check()


@pytest.mark.parametrize("d,ff", [(64, 200), (1024, 6000)])
@pytest.mark.parametrize("n", [1, 3, 20, 300])
def test_rows_of_zeros(n, d, ff):
    """A token of zeros, and an h of zeros: what is left is the bias, activated where there is an activation, and the residual."""
    dtype = torch.bfloat16
    x = _tokens(n, d, dtype, 2)
    x[0] = 0
    block, g = _block(n, d, ff, d, dtype, "relu", False), _norm(d, dtype, 1)
    y = block(x, residual=x, norm=g)
    assert torch.all(y[0] == 0)
    assert torch.all(block.gate(x, activation="gelu", norm=g)[0] == 0)
    b = torch.linspace(-3, 3, ff).to(dtype).cuda()
    layer = serving.Int8Linear(block.gate.w_codes, block.gate.w_scale, b)
    assert torch.equal(layer(x, activation="relu", norm=g)[0], b.clamp(min=0))
    dead = serving.Int8Linear(block.gate.w_codes, block.gate.w_scale * 0, torch.full((ff,), -1.0, dtype=dtype, device="cuda"))
    down = serving.Int8Linear(block.down.w_codes, block.down.w_scale, b[:d].clone() if d <= ff else None)
    y = serving.GatedMLP8(dead, block.up, down, "relu")(x, residual=x)
    assert torch.equal(y, (x.float() + down.bias.float()).to(dtype))
    block.check()


def test_no_tokens_and_refusals():
    dtype = torch.float16
    block = _block(1, 64, 100, 48, dtype, "silu", True)
    layer = block.down
    assert block(torch.empty(0, 64, dtype=dtype, device="cuda")).shape == (0, 48)
    assert layer(torch.empty(0, 100, dtype=dtype, device="cuda"), activation="silu").shape == (0, 48)
    x, h, g = _tokens(3, 64, dtype, 1), _tokens(3, 100, dtype, 1), _norm(64, dtype, 1)
    r = _tokens(3, 48, dtype, 1)
    for bad in (dict(residual=r[:, :47]), dict(residual=r[:2]), dict(residual=r.bfloat16()), dict(residual=r.cpu()), dict(norm=g[:63]), dict(norm=g.bfloat16()),
                dict(norm=g.cpu()), dict(norm=g[None]), dict(out=r.float()), dict(norm=torch.cat((g, g))[::2]), dict(residual=_tokens(48, 3, dtype, 1).t())):
        with pytest.raises(ValueError):
            block(x, **bad)
        with pytest.raises(ValueError):
            layer(h, **bad)
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        with pytest.raises(B.CmpqError) as e:
            block(x, norm=g, eps=eps)
        assert e.value.status == 1
        with pytest.raises(B.CmpqError):
            block.gate(x, norm=g, eps=eps)
        block(x, eps=eps)                                 # not looked at without a norm
    with pytest.raises(ValueError, match="activation"):
        layer(h, activation="tanh")
    with pytest.raises(ValueError, match="activation"):
        serving.GatedMLP8(block.gate, block.up, block.down, "swish")
    with pytest.raises(ValueError, match="fit"):
        serving.GatedMLP8(block.gate, block.down, block.down)
    with pytest.raises(ValueError, match="fit"):
        serving.GatedMLP8(block.gate, block.up, block.up)
    with pytest.raises(TypeError):
        block(x.bfloat16())                               # biases are fp16
    with pytest.raises(TypeError):
        block(x.float())
    with pytest.raises(ValueError):
        block(h)
    with pytest.raises(TypeError):
        layer(h, None, "silu")                            # options go by name
    block.check(), layer.check()


def test_c_calls_through_the_binding():
    n, d, ff, dtype = 4, 1024, 6000, torch.bfloat16
    block, x, g = _block(n, d, ff, d, dtype, "gelu", True), _tokens(n, d, dtype, 1), _norm(d, dtype, 2)
    w = [B.weight8(p.w_codes, p.w_scale, p.bias) for p in (block.gate, block.up, block.down)]
    y, word = torch.empty_like(x), torch.zeros(1, dtype=torch.int32, device="cuda")
    size = B.cmpq_gated_i8_ws_bytes(n, d, ff, d)
    state = torch.zeros(B.GATED_STATE_BYTES, dtype=torch.uint8, device="cuda")
    for word_or_none in (word, None):
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        for _ in range(3):
            y.zero_()
            B.cmpq_gated_i8(x, *w, ff, d, y, state, ws, g, EPS, "gelu", x, word_or_none)
            assert torch.equal(y, block(x, residual=x, norm=g, eps=EPS)) and int(word) == 0 and not state.any()
    with pytest.raises(B.CmpqError) as e:
        B.cmpq_gated_i8(x, *w, ff, d, y, state, ws[: size - 256], g, EPS, "gelu", x, word)
    assert e.value.status == 3
    state[-4] = 8                                         # the mark of a kernel that gave up
    B.cmpq_gated_i8(x[:1], *w, ff, d, torch.empty_like(x[:1]), state, ws, word=word)
    assert int(word) == 8
    word.zero_()
    ws = torch.empty(B.cmpq_linear_i8_ws_bytes(n, d, ff), dtype=torch.uint8, device="cuda")
    z = torch.empty(n, ff, dtype=dtype, device="cuda")
    B.cmpq_linear_i8_fused(x, w[0], ff, z, ws, g, EPS, "silu", None, word)
    assert torch.equal(z, block.gate(x, norm=g, eps=EPS, activation="silu")) and int(word) == 0


# ---- together ----------------------------------------------------------------------------------------------------

def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


H, KV, D, WIDTH, FF, PAGE = 8, 2, 64, 512, 1300, 16


def _decoder(dtype, pages):
    g = torch.Generator().manual_seed(2)
    w = lambda o, i: (torch.randn(o, i, generator=g) / i ** 0.5).to(dtype).cuda()
    weights = [w((H + 2 * KV) * D, WIDTH), w(WIDTH, H * D), w(FF, WIDTH), w(FF, WIDTH), w(WIDTH, FF)]
    qkv, out, gate, up, down = map(serving.Int8Linear.from_weight, weights)
    cache = serving.PagedCache8.empty(pages, KV, D, PAGE)
    angle = torch.arange(512, device="cuda")[:, None] * 0.01 * torch.arange(1, D // 2 + 1, device="cuda")
    cos, sin = angle.cos().contiguous(), angle.sin().contiguous()
    norms = [_norm(WIDTH, dtype, s) for s in (1, 2)]
    layer = serving.DecoderLayer8(serving.AttentionLayer8(qkv, out, cache, H, cos, sin), serving.GatedMLP8(gate, up, down), *norms, EPS)
    return layer, weights, norms, cos, sin


@pytest.mark.parametrize("dtype", DTYPES)
def test_decoder_layer(dtype):
    """Prompts and then single tokens through a whole layer: the bytes of the separate calls, and near the layer in 64 bits."""
    new = [37, 1, 90]
    off, lens = i32(np.cumsum([0] + new)), i32(new)
    table = torch.arange(3 * 7, device="cuda", dtype=torch.int32).view(3, 7)
    layer, weights, norms, cos, sin = _decoder(dtype, 21)
    x = torch.randn(sum(new), WIDTH, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    y = layer(x, off, lens, table, max_new=90, max_len=90)
    # the same steps one by one, on a cache of their own
    other, *_ = _decoder(dtype, 21)
    a, c = other.attention, other.attention.cache

    def steps(x, off, lens, max_new):
        qkv = a.qkv(x, norm=norms[0], eps=EPS)
        q, k, v = (qkv[:, lo * D: hi * D].unflatten(1, (hi - lo, D)) for lo, hi in ((0, H), (H, H + KV), (H + KV, H + 2 * KV)))
        q = c.append(k, v, off, lens, table, q=q, cos=cos, sin=sin)
        x = a.out(c.attend(q, off, lens, table, max_new, 100).flatten(1), residual=x)
        return x, other.mlp(x, residual=x, norm=norms[1], eps=EPS)

    mid, want = steps(x, off, lens, 90)
    assert torch.equal(y, want)
    for _ in range(3):
        lens = lens + 1
        token = y[:3].contiguous()
        y = layer(token, i32([0, 1, 2, 3]), lens, table, max_new=1, max_len=100)
        assert torch.equal(y, steps(token, i32([0, 1, 2, 3]), lens, 1)[1])
    layer.check()

    # The first prompt in 64 bits from the 16-bit weights.  A code is off by up to half a step, 1/sqrt(12) of it on average: at a
    # largest entry of 3.5 standard deviations 0.8 % of the rows' norm, for normal tokens and weights alike, 1.1 % a product; for h,
    # whose largest entry is some 12 times its root mean square, 2.7 %.  A handful of those, added as squares, is below 5 % for
    # either block; 8 % is allowed.  A norm, activation or residual that is wrong or missing is off by far more.
    X = x[:37].double()
    rms = lambda t, g: t / (t.square().mean(1, True) + EPS).sqrt() * g.double()
    W = [w.double() for w in weights]
    qkv = rms(X, norms[0]) @ W[0].T
    q, k, v = (qkv[:, lo * D: hi * D].unflatten(1, (hi - lo, D)) for lo, hi in ((0, H), (H, H + KV), (H + KV, H + 2 * KV)))

    def turn(t):
        lo, hi = t[..., : D // 2], t[..., D // 2:]
        co, si = cos[:37, None].double(), sin[:37, None].double()
        return torch.cat((lo * co - hi * si, hi * co + lo * si), -1)

    q, k, v = turn(q).transpose(0, 1), turn(k).repeat_interleave(H // KV, 1).transpose(0, 1), v.repeat_interleave(H // KV, 1).transpose(0, 1)
    p = (q @ k.transpose(1, 2) / D ** 0.5).masked_fill(torch.ones(37, 37, device="cuda", dtype=torch.bool).triu(1), -np.inf).softmax(-1)
    added = (p @ v).transpose(0, 1).flatten(1) @ W[1].T
    assert (mid[:37].double() - X - added).norm() < 0.08 * added.norm()
    M = mid[:37].double()
    n = rms(M, norms[1])
    added = (torch.nn.functional.silu(n @ W[2].T) * (n @ W[3].T)) @ W[4].T
    assert (want[:37].double() - M - added).norm() < 0.08 * added.norm()


def test_decoder_layer_refuses_parts_that_do_not_fit():
    layer, *_ = _decoder(torch.float16, 3)
    mlp = layer.mlp
    wrong = serving.GatedMLP8(mlp.gate, mlp.up, serving.Int8Linear.from_weight(torch.zeros(64, FF, dtype=torch.float16, device="cuda")))
    with pytest.raises(ValueError, match="fit"):
        serving.DecoderLayer8(layer.attention, wrong, layer.attention_norm, layer.mlp_norm)


SERVED = (1, 4, 64, 400)


def test_more_captured_calls_than_a_block_has_states_for():
    d, ff, dtype = 1024, 6000, torch.float16
    block, x, g = _block(1, d, ff, d, dtype, "silu", False), _tokens(2, d, dtype, 1), _norm(d, dtype, 2)
    want = [x]
    for _ in range(75):
        want.append(block(want[-1], norm=g))
    graphs, out, at = [], [], x
    for part in range(3):                                 # each graph goes on from the one before it
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(25):
                at = block(at, norm=g)
        graphs.append(graph), out.append(at)
    for _ in range(4):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[i], want[25 * i + 25]) for i in range(3))
        for t in out:
            t.zero_()
    block.check()


@pytest.mark.parametrize("d,ff", [(256, 1000), (1024, 6000)])
def test_graphs_streams_and_eager_calls_together(d, ff):
    """Blocks and layers of several batch sizes, captured, replayed in any order and on several streams, with eager calls
    between: every result has the bytes of a call that ran alone."""
    dtype = torch.bfloat16
    block, layer = _block(1, d, ff, d, dtype, "silu", False), _weights(700, d, dtype, 9, True)
    g = _norm(d, dtype, 1)
    xs = {n: _tokens(n, d, dtype, n) for n in SERVED}
    call = lambda n: (block(xs[n], residual=xs[n], norm=g), layer(xs[n], norm=g, activation="gelu"))
    stream, graphs, out = torch.cuda.Stream(), {}, {}
    for n in SERVED:                                      # the first calls of all are captured ones
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n], stream=stream):
            out[n] = call(n)
    want = {n: call(n) for n in SERVED}
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in SERVED]
    for turn in range(12):
        for i, n in enumerate(SERVED):
            with torch.cuda.stream(streams[(turn + i) % 4] if turn % 2 else stream):
                graphs[n].replay()
        got = []
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got += [(n, call(n)) for n in SERVED]
        torch.cuda.synchronize()
        for n, pair in got + list(out.items()):
            assert all(map(torch.equal, pair, want[n])), (turn, n)
        for n in SERVED:
            for t in out[n]:
                t.zero_()
        torch.cuda.synchronize()
    block.check(), layer.check()
