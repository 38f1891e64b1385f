"""Serving calls in CUDA graphs and on several streams: the same bytes as eager calls on one stream, whatever order graphs
are replayed in, on whatever streams, and whatever eager calls come between."""
import itertools

import numpy as np
import pytest
import torch

from paper_2410_13056_b200 import binding as B
from paper_2410_13056_b200 import serving

pytestmark = pytest.mark.gpu
H, D, P, HEADS, WIDTH = 2, 64, 16, 8, 256
SIZES = (8, 64, 1)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _layer(pages):
    g = torch.Generator().manual_seed(2)
    w = (torch.randn((HEADS + 2 * H) * D, WIDTH, generator=g) * 0.05).half().cuda()
    wo = (torch.randn(WIDTH, HEADS * D, generator=g) * 0.05).half().cuda()
    cache = serving.PagedCache8.empty(pages, H, D, P)
    fill = torch.Generator(device="cuda").manual_seed(5)
    for codes in (cache.k_codes, cache.v_codes):
        codes.copy_(torch.randint(-127, 128, codes.shape, generator=fill, device="cuda", dtype=torch.int8))
    cache.k_scale.fill_(0.01), cache.v_scale.fill_(0.02)
    angle = torch.arange(4096, device="cuda")[:, None] * 0.01 * torch.arange(1, D // 2 + 1, device="cuda")
    return serving.AttentionLayer8(serving.Int8Linear.from_weight(w), serving.Int8Linear.from_weight(wo), cache, HEADS,
                                   angle.cos().contiguous(), angle.sin().contiguous())


def _step(n, first_page):
    """A token each of n sequences with caches of very different lengths, on pages of their own."""
    g = np.random.default_rng(n)
    lens = g.integers(1, 900, size=n)
    lens[0] = 3000
    per = -(-lens // P)
    table = np.full((n, per.max()), -1)
    for s, p in enumerate(per):
        table[s, :p] = first_page + np.arange(p)
        first_page += p
    x = torch.from_numpy(g.normal(size=(n, WIDTH))).half().cuda()
    return dict(x=x, tok_off=i32(np.arange(n + 1)), lens=i32(lens), table=i32(table), max_new=1, max_len=3000), first_page


def test_graphs_of_several_batch_sizes():
    steps, page = {}, 0
    for n in SIZES + (300,):
        steps[n], page = _step(n, page)
    layer = _layer(page)
    want = {n: layer(**steps[n]) for n in steps}
    want = {n: layer(**steps[n]) for n in steps}           # appended once more: now a step changes nothing
    layer.cache.check()
    stream, graphs, out = torch.cuda.Stream(), {}, {}
    torch.cuda.synchronize()
    for n in SIZES:
        with torch.cuda.stream(stream):
            layer(**steps[n])                              # warm-up on the stream that is captured
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n], stream=stream):
            out[n] = layer(**steps[n])
    for order in itertools.permutations(SIZES):
        with torch.cuda.stream(stream):
            big = layer(**steps[300])                      # larger than anything before it on this stream
            junk = [torch.full((1 << k,), 255, dtype=torch.uint8, device="cuda") for k in range(9, 24)]
        torch.cuda.synchronize()
        for n in order:
            graphs[n].replay()
        torch.cuda.synchronize()
        assert torch.equal(big, want[300]) and all(int(j.min()) == 255 for j in junk)
        for n in SIZES:
            assert torch.equal(out[n], want[n]), (order, n)
            out[n].zero_()
    # each graph on a stream of its own, and eager calls beside them
    streams = [torch.cuda.Stream() for _ in SIZES]
    torch.cuda.synchronize()
    for _ in range(20):
        for n, s in zip(SIZES, streams):
            with torch.cuda.stream(s):
                graphs[n].replay()
        again = layer(**steps[300])
    torch.cuda.synchronize()
    assert torch.equal(again, want[300])
    for n in SIZES:
        assert torch.equal(out[n], want[n]), n
    layer.cache.check()


def test_attention_first_called_in_a_capture():
    """No call before the capture, two graphs on one stream, the second replayed first."""
    (a, page), (b, _) = _step(1, 0), _step(64, 0)
    layer = _layer(_step(64, 0)[1])
    q = {n: torch.randn(n, HEADS, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).half() for n in (1, 64)}
    args = {n: [q[n], s["tok_off"], s["lens"], s["table"], 1, 3000] for n, s in ((1, a), (64, b))}
    stream, graphs, out = torch.cuda.Stream(), {}, {}
    for n in (1, 64):
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n], stream=stream):
            out[n] = layer.cache.attend(*args[n])
    for n in (64, 1, 1, 64):
        graphs[n].replay()
    torch.cuda.synchronize()
    for n in (1, 64):
        assert torch.equal(out[n], layer.cache.attend(*args[n])), n
    layer.cache.check()


def test_attend_on_four_streams_at_once():
    steps, page = [], 0
    for n in (1, 5, 64, 30):
        s, page = _step(n, page)
        steps.append((n, s))
    cache = _layer(page).cache
    other = _layer(page).cache                             # two caches share a stream's work space
    q = [torch.randn(n, HEADS, D, device="cuda").bfloat16() for n, _ in steps]
    run = lambda c, i: c.attend(q[i], steps[i][1]["tok_off"], steps[i][1]["lens"], steps[i][1]["table"], 1, 3000)
    want = [run(cache, i) for i in range(4)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(4)], []
    for _ in range(25):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got += [(i, run(cache, i)), (i, run(other, i))]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i, y in got)
    cache.check(), other.check()


@pytest.mark.parametrize("new", [1, 200])
def test_a_work_space_that_a_kernel_gave_up_on_is_reported_by_later_calls(new):
    cache = _layer(20).cache
    q = torch.randn(new, HEADS, D, device="cuda").half()
    off, lens, table = i32([0, new]), i32([300]), i32([np.arange(19)])
    batch = B.Batch(off.data_ptr(), lens.data_ptr(), table.data_ptr(), 19, 1, new)
    c = B.Cache(cache.k_codes.data_ptr(), cache.k_scale.data_ptr(), cache.v_codes.data_ptr(), cache.v_scale.data_ptr(), 20, H, D, P)
    ws = torch.zeros(B.cmpq_cache_attention_ws_bytes(1, new, new, 300, HEADS, H, D), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(new, HEADS, device="cuda")
    for mark in (0, 1):
        word = i32([0])
        ws[4092:4096].view(torch.int32).fill_(mark)
        B.cmpq_cache_attention(c, batch, q, new, 300, 0.125, True, 0, out, lse, ws, word)
        assert int(word) == 8 * mark
        assert torch.equal(out, cache.attend(q, off, lens, table, new, 300))
    with pytest.raises(B.CmpqError) as e:
        B.cmpq_check_cache(word)
    assert e.value.status == 5


def test_layer_reports_what_its_calls_met():
    """NaN and infinity in the activations reach the user through check(), once; so does the mark of a kernel that gave up."""
    step, page = _step(3, 0)
    layer = _layer(page)
    layer(**step)
    layer.check()
    step["x"][1, 7] = float("nan")
    layer(**step)
    for part in (layer.qkv, layer):                        # the projection's report, then the cache's and the output's
        with pytest.raises(B.CmpqError) as e:
            part.check()
        assert e.value.status == 6
    layer.check()
    linear = layer.out
    x = torch.zeros(2, HEADS * D, dtype=torch.float16, device="cuda")
    x[1, 3] = float("inf")
    linear(x)
    with pytest.raises(B.CmpqError) as e:
        linear.check()
    assert e.value.status == 6
    linear(x[:1])
    linear.check()
    linear.nonfinite.fill_(8)
    with pytest.raises(B.CmpqError) as e:
        linear.check()
    assert e.value.status == 5
    linear.check()
