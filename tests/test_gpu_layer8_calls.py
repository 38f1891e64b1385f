"""Calls of the 8-bit layers that their documentation allows: padded batches, a whole layer in a graph, outputs over inputs,
token counts past those that the choice of kernels was fitted to."""
import numpy as np
import pytest
import torch

import layer_ref as ref
import test_gpu_layer8 as base
from paper_2410_13056_b200 import binding as B
from paper_2410_13056_b200 import serving
from test_gpu_layer8 import DTYPES, EPS, H, KV, D, PAGE, WIDTH, i32

pytestmark = pytest.mark.gpu


# past 512 tokens: two and four blocks to a tile in place of tiles, and pairs where a cluster was chosen once
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", [(600, 4097, 257), (640, 8193, 1001), (700, 12288, 2301), (1280, 11008, 2050)])
def test_long_sums_of_many_tokens(n, d_in, d_out, dtype):
    for act, norm, residual in (("silu", True, True), (None, False, False)):
        x = base._tokens(n, d_in, dtype, n + d_in)
        layer = base._weights(d_out, d_in, dtype, d_out, bias=residual)
        g = base._norm(d_in, dtype, 4) if norm else None
        r = base._tokens(n, d_out, dtype, 2) if residual else None
        y = layer(x, activation=act, residual=r, norm=g, eps=EPS)
        rows = np.r_[0:3, 127:130, 255:258, n - 3:n]   # a token's value does not depend on the others'
        z, err = ref.linear(*ref.norm_quantize(base._np(x[rows]), base._np(g), EPS), *base._parts(layer))
        base._compare(y[rows], *ref.finish(z, err, act, None if r is None else base._np(r[rows]), dtype))
        for lo in range(0, n, 128):                    # and neither do its bytes: another kernel's are the same
            part = slice(lo, lo + 128)
            assert torch.equal(layer(x[part], activation=act, residual=None if r is None else r[part], norm=g, eps=EPS), y[part])
        layer.check()


@pytest.mark.parametrize("n", [1, 4, 5, 40, 200])
def test_every_output_over_its_input_is_right(n):
    d, dtype = 4096, torch.bfloat16
    layer, g, x = base._weights(d, d, dtype, 1, True), base._norm(d, dtype, 2), base._tokens(n, d, dtype, 3)
    want = layer(x, activation="silu", norm=g)
    for by in (7, 8, 4095):                            # rows that begin on 16 bytes and not, and that share one entry
        room = torch.zeros(n, 2 * d + 7, dtype=dtype, device="cuda")
        for at, to in ((0, by), (by, 0)):
            for _ in range(10):
                room[:, at: at + d] = x
                assert torch.equal(layer(room[:, at: at + d], out=room[:, to: to + d], activation="silu", norm=g), want), (by, at, to)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [1, 7, 128, 1000, 2048, 4096])
def test_the_few_token_kernel_quantizes_as_the_quantization_does(d, dtype):
    """A layer whose weight is the identity, scaled by 1, returns a token's codes times its scale: for up to four tokens those of
    the kernel that quantizes its own tokens, else those of the kernels that quantize_tokens starts."""
    eye = torch.zeros(d, (d + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    eye[torch.arange(d), torch.arange(d)] = 1
    layer = serving.Int8Linear(eye[:, :d], torch.ones(d, device="cuda"))
    x, g = base._tokens(64, d, dtype, d), base._norm(d, dtype, 1)
    x[3] = 0
    if dtype == torch.bfloat16:
        for row, p in ((5, 60), (6, 100), (9, -60), (10, -100)):   # squares that pass float32, or vanish beside eps
            x[row] = (x[row].float() * 2.0 ** p).to(dtype)
    for norm in (None, g):
        codes, scale = serving.quantize_tokens(x, norm, EPS)
        want = (codes.float() * scale[:, None]).to(dtype)
        for n in (1, 2, 3, 4):
            for at in range(0, 64, n):
                assert torch.equal(layer(x[at: at + n], norm=norm, eps=EPS), want[at: at + n])


def _nans(like, count=24):
    """Leaves NaN in the memory that tensors of this size get next."""
    blocks = [torch.full_like(like, float("nan")) for _ in range(count)]
    del blocks


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_behind_the_last_sequence(dtype):
    """A batch in a larger array, as a program with captured batch sizes has it: nothing of the rows behind the last sequence is
    reported, and the tokens before them get the bytes that they get alone."""
    layer, *_ = base._decoder(dtype, 21)
    alone, *_ = base._decoder(dtype, 21)
    x = torch.randn(64, WIDTH, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    table = torch.arange(3 * 7, device="cuda", dtype=torch.int32).view(3, 7)
    lens = i32([0, 0, 0])
    for new, rows in (([20, 0, 13], 64), ([1, 1, 1], 8), ([1, 0, 1], 3), ([0, 0, 0], 2), ([2, 3, 0], 5), ([0, 1, 1], 33)):
        lens = lens + i32(new)
        off, n = i32(np.cumsum([0] + new)), sum(new)
        want = alone(x[:n], off, lens, table, max(new), 100) if n else x[:0]
        _nans(torch.empty(rows, H * D, dtype=dtype, device="cuda"))
        y = layer(x[:rows], off, lens, table, max_new=max(1, *new), max_len=100)
        assert torch.equal(y[:n], want) and torch.isfinite(y).all()
        layer.check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_decoder_layer_in_graphs(dtype):
    """Single tokens through captured layers, the lengths advanced on the device: the bytes of eager calls, for more than one batch
    size on one cache, with eager calls between, and with padded rows."""
    layer, *_ = base._decoder(dtype, 42)
    eager, *_ = base._decoder(dtype, 42)
    table = torch.arange(6 * 7, device="cuda", dtype=torch.int32).view(6, 7)
    prompt = torch.randn(6 * 5, WIDTH, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    off, lens = i32(np.arange(7) * 5), i32([5] * 6)
    for one in (layer, eager):
        one(prompt, off, lens, table, 5, 100)

    class Batch:
        """The sequences [lo, hi) of the table in an array of `rows` rows."""

        def __init__(self, lo, hi, rows):
            self.x = torch.zeros(rows, WIDTH, dtype=dtype, device="cuda")
            self.off, self.lens, self.table, self.count = i32(np.arange(hi - lo + 1)), i32([5] * (hi - lo)), table[lo:hi], hi - lo
            self.graph = torch.cuda.CUDAGraph()
            stream = torch.cuda.Stream()
            with torch.cuda.graph(self.graph, stream=stream):
                self.lens += 1
                self.y = layer(self.x, self.off, self.lens, self.table, 1, 100)
                self.x[: self.count] = self.y[: self.count]

    batches = [Batch(0, 1, 1), Batch(1, 4, 3), Batch(4, 6, 8)]
    want = []
    for i, b in enumerate(batches):
        b.x[: b.count] = prompt[i: i + b.count]
        want.append([b.x[: b.count].clone(), i32([5] * b.count)])
    torch.cuda.synchronize()
    for step in range(40):
        for b, state in zip(batches if step % 2 else batches[::-1], want if step % 2 else want[::-1]):
            b.graph.replay()
            state[1] += 1
            state[0] = eager(state[0], b.off, state[1], b.table, 1, 100)
            assert torch.equal(b.y[: b.count], state[0]) and torch.equal(b.x[: b.count], state[0]) and torch.equal(b.lens, state[1])
    layer.check(), eager.check()
    a, b = layer.attention.cache, eager.attention.cache
    assert torch.equal(a.k_codes, b.k_codes) and torch.equal(a.v_codes, b.v_codes)


def test_captured_calls_take_a_state_only_where_blocks_meet_in_it():
    """A program that captures a graph for every batch size has its states left for the calls that need them."""
    d, ff, dtype = 1024, 6000, torch.bfloat16
    block, x, g = base._block(1, d, ff, d, dtype, "silu", False), base._tokens(300, d, dtype, 1), base._norm(d, dtype, 2)
    sizes = [5, 6, 8, 33, 64, 100, 128, 129, 200, 300] * 8 + [1, 2, 3, 4]
    want = {n: block(x[:n], residual=x[:n], norm=g) for n in set(sizes)}
    assert block._impl.captured_states == 0
    graph, out = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        for n in sizes:
            out.append(block(x[:n], residual=x[:n], norm=g))
    assert block._impl.captured_states == 4
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, want[n]) for n, y in zip(sizes, out))
        for y in out:
            y.zero_()
    block.check()


# the kernel for few rows and the one for prompts, whose blocks share out the keys or not; outputs on 16 bytes and not
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,lens,heads,kv,d,page", [([1, 1, 1], [40, 300, 7], 8, 2, 64, 16), ([3, 0, 2], [90, 5, 64], 4, 4, 128, 64), ([0, 1], [9, 20], 6, 2, 256, 32),
                                                      ([0, 0], [9, 0], 8, 2, 64, 16), ([200, 70], [500, 90], 8, 2, 64, 16), ([130, 0], [130, 40], 16, 1, 128, 64),
                                                      ([0, 0, 300], [4, 4, 2000], 2, 2, 128, 128), ([300, 1], [300, 1], 64, 8, 64, 64)])
def test_rows_behind_are_zeroed_where_that_is_asked_for(new, lens, heads, kv, d, page, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    pages = -(-max(lens) // page)
    c = serving.PagedCache8.empty(len(lens) * pages, kv, d, page)
    for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)):
        codes.random_(-127, 128, generator=g), scale.uniform_(0.005, 0.02, generator=g)
    table = torch.arange(len(lens) * pages, dtype=torch.int32, device="cuda").view(-1, pages)
    n = sum(new)
    off, lengths = i32(np.cumsum([0] + new)), i32(lens)
    for rows in (n, n + 1, n + 37, n + 700):
        q = torch.randn(rows, heads, d, device="cuda", generator=g).to(dtype)
        for spare in (0, 3):                           # entries between the rows of the output
            room = torch.full((rows + 1, heads * d + spare), 7.0, dtype=dtype, device="cuda")
            out = room[:rows, : heads * d].unflatten(1, (heads, d))
            for max_new in (max(1, *new), 700):        # the bound chooses the kernel
                args = dict(max_new=max_new, max_len=max(lens), window=0)
                want, lse = c.attend(q, off, lengths, table, out=out, return_lse=True, **args)
                want = want[:n].clone()
                assert torch.all(out[n:] == 7.0)       # left alone
                got, again = c.attend(q, off, lengths, table, out=out, return_lse=True, zero_behind=True, **args)
                assert torch.equal(got[:n], want) and torch.equal(again[:n], lse[:n]) and not got[n:].any()
                assert torch.all(room[rows:] == 7.0) and torch.all(room[:, heads * d:] == 7.0)
                room[:] = 7.0
    c.check()


def test_rows_behind_without_any_sequence():
    c = serving.PagedCache8.empty(2, 2, 64, 16)
    q, none = torch.ones(5, 4, 64, dtype=torch.float16, device="cuda"), i32([])
    room = torch.full((6, 256 + 8), 7.0, dtype=torch.float16, device="cuda")
    out = room[:5, :256].unflatten(1, (4, 64))
    args = (i32([0]), none, torch.empty(0, 1, dtype=torch.int32, device="cuda"), 1, 16)
    c.attend(q, *args, out=out)
    assert torch.all(room == 7.0)
    c.attend(q, *args, out=out, zero_behind=True)
    assert not out.any() and torch.all(room[5:] == 7.0) and torch.all(room[:, 256:] == 7.0)
    c.check()


def test_offsets_that_do_not_fit_zero_nothing_out_of_range():
    """What the host cannot see: the rows of a wrong batch are unspecified, nothing behind the array is written."""
    c = serving.PagedCache8.empty(4, 2, 64, 16)
    q = torch.ones(6, 4, 64, dtype=torch.float16, device="cuda")
    room = torch.full((8, 256), 7.0, dtype=torch.float16, device="cuda")
    for last in (7, 1 << 30, -1, -(1 << 31)):
        c.attend(q, i32([0, last]), i32([3]), i32([[0, 1]]), 1, 16, out=room[:6].unflatten(1, (4, 64)), zero_behind=True)
        with pytest.raises(B.CmpqError) as e:
            c.check()
        assert e.value.status == 1 and torch.all(room[6:] == 7.0)
