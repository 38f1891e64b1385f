"""The paged 8-bit cache against the plain statements: append and read back bit for bit (every step is one float32
operation), attention against float64.

Tolerance of the attention, for a row with weights p (sum 1), values v, D entries, L visible keys:
  score  products of a 16-bit query (in fp16 after a power-of-two scaling: exact up to 2^-24 of the row's largest
         entry) with exact codes, summed in fp32, then scaled: |ds| <= (D + 8) 2^-23 T,  T = scale max_j sum |q k|
  p      relative 2 ds + 2^-20 (exponential, running sum, fp32 accumulation over L <= 2^13 keys in tiles) and
         2^-11 for the rounding to fp16, or 2^-25 absolute (against a largest weight of 1) where that is subnormal
  out    sum_j |dp_j| |v_j| + half an ulp of the 16-bit type
so |out - ref| <= (2^-10 + 4 ds) sum p|v| + 2^-24 L max|v| + half ulp, and |lse - ref| <= 2 ds + 2^-20 (1 + |lse|)."""
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2410_13056_b200 import binding as B
from paper_2410_13056_b200 import serving

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def make(lens, H, d, P, seed, garbage=True):
    """A cache that holds `lens` tokens per sequence on shuffled pages; what no sequence owns is garbage: scales NaN
    in free pages, arbitrary codes past a sequence's end, table entries that are no pages past the last."""
    g = np.random.default_rng(seed)
    per = [-(-max(0, n) // P) for n in lens]
    n_pages = sum(per) + 2
    ids = g.permutation(n_pages)
    width = max(per + [1]) + 1
    table = np.full((len(lens), width), -1, np.int64)
    table[:, 1::2] = 10 ** 9 if garbage else -1
    cache = {}
    for x in "kv":
        cache[x + "_codes"] = np.clip(np.rint(g.normal(size=(n_pages, H, P, d)) * 40), -127, 127).astype(np.int8)
        cache[x + "_scale"] = (0.02 * np.exp(0.5 * g.normal(size=(n_pages, H)))).astype(np.float32)
    at = 0
    for s, p in enumerate(per):
        table[s, :p] = ids[at: at + p]
        at += p
    if garbage:
        for x in "kv":
            cache[x + "_scale"][ids[at:]] = np.nan
    return cache, table


def up(cache):
    return serving.PagedCache8(*(torch.from_numpy(cache[x].copy()).cuda() for x in ("k_codes", "k_scale", "v_codes", "v_scale")))


def tokens(n, h, d, dtype, seed, spread=1.0):
    x = np.random.default_rng(seed).normal(size=(n, h, d)) * spread
    return torch.from_numpy(x).to(dtype)


def rope(n_pos, rot):
    a = np.arange(n_pos)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


APPENDS = [  # lens after the call, new tokens, heads, head_dim, page, rot, interleaved
    ([1], [1], 1, 64, 16, 64, False),
    ([17, 16, 15, 33], [1, 1, 1, 1], 2, 128, 16, 128, False),
    ([40, 5, 64, 0, 70], [40, 0, 3, 0, 41], 3, 128, 32, 64, True),
    ([129, 128, 127], [129, 64, 2], 2, 128, 64, 128, False),
    ([300, 7], [170, 7], 1, 256, 128, 96, False),
    ([300, 20], [299, 13], 2, 256, 64, 20, False),
    ([200], [200], 4, 64, 128, 0, False),
    ([90, 90], [33, 50], 2, 64, 32, 2, True),
    ([50] * 300, [1] * 300, 1, 64, 16, 64, False),
    ([77], [60], 2, 128, 64, 6, False),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,new,H,d,P,rot,inter", APPENDS)
def test_append_and_read_bit_exact(lens, new, H, d, P, rot, inter, dtype):
    cache, table = make(lens, H, d, P, len(lens) + d, garbage=False)
    for x in "kv":                                     # some pages have to be scaled anew, some not
        cache[x + "_scale"] *= np.where(np.arange(len(cache[x + "_scale"])) % 2, 0.05, 4.0).astype(np.float32)[:, None]
    off = np.concatenate(([0], np.cumsum(new)))
    n, heads = int(off[-1]), 2 * H + 1
    # columns of one projection's output: row strides, and an odd start that leaves no alignment for the last case
    odd = 1 if lens == [77] else 0
    qkv = tokens(n, 1, (heads + 2 * H) * d + odd, dtype, 3).cuda()[:, 0, odd:]
    q, k, v = (qkv[:, a * d: b * d].unflatten(1, (b - a, d)) for a, b in ((0, heads), (heads, heads + H), (heads + H, heads + 2 * H)))
    k[: n // 2] *= 3
    cos, sin = rope(max(lens) + 1, rot) if rot else (None, None)
    t = {} if not rot else {"cos": torch.from_numpy(cos).cuda(), "sin": torch.from_numpy(sin).cuda()}
    c = up(cache)
    out = c.append(k, v, i32(off), i32(lens), i32(table), q=q, interleaved=inter, **t)
    ref.append(cache, off, lens, table, k.float().cpu().numpy(), v.float().cpu().numpy(), cos, sin, inter)
    c.check()
    used = np.concatenate([table[s][: -(-m // P)] for s, m in enumerate(lens)]).astype(int)
    for x in "kv":
        got, want = getattr(c, x + "_scale").cpu().numpy(), cache[x + "_scale"]
        assert np.array_equal(got, want), x
        codes = getattr(c, x + "_codes").cpu().numpy()
        assert np.array_equal(codes, cache[x + "_codes"]), x       # free pages and the slots past the end too
    pos = np.concatenate([np.arange(m - w, m) for m, w in zip(lens, new)]).astype(int)
    want = q.float().cpu().numpy()
    want = torch.from_numpy(ref.rotate(want, pos, cos, sin, inter) if rot else want).to(dtype)
    assert torch.equal(out.cpu(), want)
    # in place
    c2 = up(cache)
    same = q.clone()
    c2.append(k, v, i32(off), i32(lens), i32(table), q=same, q_out=same, interleaved=inter, **t)
    assert torch.equal(same, out)
    # read back all tokens of every sequence, more than were appended
    all_off = np.concatenate(([0], np.cumsum(lens)))
    kk, vv = c.read(i32(all_off), i32(lens), i32(table), int(all_off[-1]), dtype)
    for x, got in (("k", kk), ("v", vv)):
        vals = cache[x + "_codes"].astype(np.float32) * cache[x + "_scale"][..., None, None]
        rows = [vals[table[s][p // P], :, p % P] for s, m in enumerate(lens) for p in range(m)]
        assert torch.equal(got.cpu(), torch.from_numpy(np.stack(rows)).to(dtype)), x
    c.check()
    assert used.size


def test_append_grows_page_by_page_like_one_call():
    """Token by token the scale can only grow, and the codes of a page end within the roundings of its growth."""
    H, d, P, n = 2, 64, 16, 40
    k, v = tokens(n, H, d, torch.float16, 1).cuda(), tokens(n, H, d, torch.float16, 2).cuda()
    table = i32([[2, 0, 1]])
    one = serving.PagedCache8.empty(3, H, d, P)
    one.append(k, v, i32([0, n]), i32([n]), table)
    steps = serving.PagedCache8.empty(3, H, d, P)
    for i in range(n):
        steps.append(k[i: i + 1], v[i: i + 1], i32([0, 1]), i32([i + 1]), table)
    one.check(), steps.check()
    assert torch.equal(one.k_scale, steps.k_scale) and torch.equal(one.v_scale, steps.v_scale)
    # at most 16 roundings of half a code, each later shrunk with the growth that follows it
    assert (one.k_codes.int() - steps.k_codes.int()).abs().max() <= 8


@pytest.mark.parametrize("P,d", [(16, 64), (64, 128)])
def test_append_and_read_many_tokens(P, d):
    """Prompts of thousands of tokens, some sequences without any, and all of them read back in one call."""
    lens, new, H = [5000, 0, 3301, 77, 1], [4990, 0, 3301, 20, 1], 2
    cache, table = make(lens, H, d, P, 4, garbage=False)
    off = np.concatenate(([0], np.cumsum(new)))
    k, v = (tokens(int(off[-1]), H, d, torch.bfloat16, s).cuda() for s in (1, 2))
    cos, sin = rope(5000, d)
    c = up(cache)
    q = tokens(int(off[-1]), 3, d, torch.bfloat16, 3).cuda()
    out = c.append(k, v, i32(off), i32(lens), i32(table), q=q, cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda())
    ref.append(cache, off, lens, table, k.float().cpu().numpy(), v.float().cpu().numpy(), cos, sin)
    pos = np.concatenate([np.arange(m - w, m) for m, w in zip(lens, new)]).astype(int)
    assert torch.equal(out.cpu(), torch.from_numpy(ref.rotate(q.float().cpu().numpy(), pos, cos, sin, False)).bfloat16())
    for x in "kv":
        assert np.array_equal(getattr(c, x + "_scale").cpu().numpy(), cache[x + "_scale"]), x
        assert np.array_equal(getattr(c, x + "_codes").cpu().numpy(), cache[x + "_codes"]), x
    all_off = np.concatenate(([0], np.cumsum(lens)))
    got = c.read(i32(all_off), i32(lens), i32(table), int(all_off[-1]), torch.float16)
    for x, t in zip("kv", got):
        vals = cache[x + "_codes"].astype(np.float32) * cache[x + "_scale"][..., None, None]
        rows = [vals[table[s][p // P], :, p % P] for s, m in enumerate(lens) for p in range(m)]
        assert torch.equal(t.cpu(), torch.from_numpy(np.stack(rows)).half()), x
    c.check()


def test_append_extremes():
    """Zeros take the smallest scale, huge values the largest, NaN and infinity are reported; no fault, no spill."""
    H, d, P = 1, 64, 16
    c = serving.PagedCache8.empty(4, H, d, P)
    zeros = torch.zeros(3, H, d, dtype=torch.bfloat16, device="cuda")
    c.append(zeros, zeros, i32([0, 3]), i32([3]), i32([[0]]))
    assert float(c.k_scale[0]) == 2.0 ** -60 and torch.all(c.k_codes[0] == 0)
    huge = torch.full((1, H, d), 3e38, dtype=torch.bfloat16, device="cuda")
    c.append(huge, -huge, i32([0, 1]), i32([1]), i32([[1]]))
    assert float(c.k_scale[1]) == 2.0 ** 60 and torch.all(c.k_codes[1, :, 0] == 127) and torch.all(c.v_codes[1, :, 0] == -127)
    c.check()
    bad = torch.ones(2, H, d, dtype=torch.bfloat16, device="cuda")
    bad[1, 0, 5] = float("nan")
    c.append(zeros[:2], bad, i32([0, 2]), i32([2]), i32([[2]]))
    with pytest.raises(B.CmpqError) as e:
        c.check()
    assert e.value.status == 6
    c.check()                                          # forgotten


def test_what_does_not_fit_is_left_out_and_reported():
    H, d, P = 2, 64, 16
    k = tokens(6, H, d, torch.float16, 1).cuda()
    cos, sin = (torch.from_numpy(x).cuda() for x in rope(20, d))
    good = dict(tok_off=[0, 3, 6], lens=[3, 20], table=[[0, 1], [2, 3]])
    for change in (dict(lens=[2, 20]), dict(lens=[-1, 20]), dict(table=[[0, 1], [2, 4]]), dict(table=[[-1, 1], [2, 3]]),
                   dict(lens=[3, 40]), dict(tok_off=[0, 3, 9]), dict(lens=[3, 21])):
        b = {**good, **change}
        c = serving.PagedCache8.empty(4, H, d, P)
        args = (i32(b["tok_off"]), i32(b["lens"]), i32(b["table"]))
        c.append(k, k, *args, q=k, cos=cos, sin=sin)
        with pytest.raises(B.CmpqError) as e:
            c.check()
        assert e.value.status == 1
        if "tok_off" not in change and change != dict(lens=[3, 21]) and b["lens"][0] == 3 and b["table"][0][0] == 0:
            # the sequence that fits is as it would be alone
            c2 = serving.PagedCache8.empty(4, H, d, P)
            c2.append(k[:3], k[:3], i32([0, 3]), i32([3]), i32([[0, 1]]), cos=cos, sin=sin)
            assert torch.equal(c.k_codes[0], c2.k_codes[0]) and torch.equal(c.k_scale[0], c2.k_scale[0])
    c = serving.PagedCache8.empty(4, H, d, P)
    c.append(k, k, i32([0, 3, 6]), i32([3, 20]), i32([[0, 1], [2, 3]]), q=k, cos=cos, sin=sin)
    c.check()
    for change in (dict(lens=[3, 40]), dict(lens=[-2, 20]), dict(table=[[0, 1], [2, 9]]), dict(lens=[3, 33])):
        b = {**good, **change}
        out = c.attend(k, i32(b["tok_off"]), i32(b["lens"]), i32(b["table"]), max_new=3, max_len=32)
        with pytest.raises(B.CmpqError) as e:
            c.check()
        assert e.value.status == 1
        if b["lens"][0] == 3:
            alone = c.attend(k[:3], i32([0, 3]), i32([3]), i32([[0, 1]]), max_new=3, max_len=32)
            assert torch.equal(out[:3], alone)
    c.attend(k, i32([0, 3, 6]), i32([3, 20]), i32([[0, 1], [2, 3]]), max_new=2, max_len=32)
    with pytest.raises(B.CmpqError):
        c.check()


ATTENDS = [  # lens, new, query heads, cached heads, head_dim, page, window, causal
    ([1], [1], 1, 1, 64, 16, 0, True),
    ([0, 1, 16, 17], [0, 1, 1, 1], 4, 2, 64, 16, 0, True),
    ([31, 64, 65, 129], [1, 1, 1, 1], 8, 1, 128, 64, 0, True),
    ([700, 3, 255], [1, 1, 1], 8, 8, 128, 64, 0, True),
    ([1500], [1], 16, 1, 128, 128, 0, True),
    ([333, 120], [1, 1], 14, 2, 128, 32, 0, True),
    ([90, 256], [1, 1], 6, 2, 256, 64, 0, True),
    ([5, 0, 2], [7, 2, 2], 4, 2, 64, 16, 0, True),                 # rows before the first token: nothing to see
    ([50, 200, 1000], [3, 5, 8], 8, 2, 64, 16, 0, True),
    ([400, 77], [4, 4], 16, 2, 128, 64, 33, True),
    ([400, 77], [4, 1], 16, 4, 128, 64, 1, True),
    ([600], [16], 3, 3, 128, 32, 5000, True),
    ([130, 70], [130, 70], 4, 2, 128, 64, 0, True),
    ([300, 40, 257], [150, 0, 257], 4, 1, 64, 32, 0, True),
    ([513], [257], 8, 2, 128, 128, 100, True),
    ([140, 300], [140, 129], 2, 1, 256, 16, 0, True),
    ([100, 390], [30, 200], 2, 2, 128, 64, 0, False),
    ([0, 45], [3, 1], 2, 1, 64, 16, 0, False),
    ([1100], [400], 8, 8, 64, 16, 0, True),
]


def check_attend(cache, off, lens, table, q, scale, causal, window, out, lse, dtype):
    want, wlse, weight, span, terms = ref.attend(cache, off, lens, table, q.float().cpu().numpy(), scale, causal, window)
    d = q.shape[2]
    ds = (d + 8) * 2.0 ** -23 * terms
    got = out.float().cpu().numpy().astype(np.float64)
    tol = (2.0 ** -10 + 4 * ds[..., None]) * weight + 2.0 ** -24 * span + ref.half_ulp(np.abs(want) + 2.0 ** -9 * weight, dtype)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])
    empty = np.isneginf(wlse)
    assert np.all(got[empty] == 0)
    if lse is not None:
        l = lse.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isneginf(l), empty)
        assert np.all(np.abs(l[~empty] - wlse[~empty]) <= (2 * ds + 2.0 ** -20 * (1 + np.abs(wlse)))[~empty])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,new,heads,H,d,P,window,causal", ATTENDS)
def test_attend_against_float64(lens, new, heads, H, d, P, window, causal, dtype):
    cache, table = make(lens, H, d, P, sum(lens) + heads)
    off = np.concatenate(([0], np.cumsum(new)))
    n = int(off[-1])
    wide = tokens(n + 2, heads + 1, d, dtype, 4).cuda()
    q = wide[:n, :heads] if heads == 1 else wide.flatten(1)[:n, : heads * d].unflatten(1, (heads, d))  # a row stride
    scale = 1.0 / math.sqrt(d)
    c = up(cache)
    room = torch.full((n + 1, heads, d), 7.0, dtype=dtype, device="cuda")
    out, lse = c.attend(q, i32(off), i32(lens), i32(table), max_new=max(new), max_len=max(lens), window=window,
                        causal=causal, out=room[:n], return_lse=True)
    assert torch.all(room[n] == 7.0)
    c.check()
    check_attend(cache, off, lens, table, q, scale, causal, window, out, lse, dtype)
    # looser bounds may choose another kernel and split, not another answer beyond the tolerance; twice the same bytes
    for bounds in (dict(max_new=max(new) + 40, max_len=max(lens) + 5000), dict(max_new=max(new))):
        a = c.attend(q, i32(off), i32(lens), i32(table), window=window, causal=causal, **bounds)
        b = c.attend(q, i32(off), i32(lens), i32(table), window=window, causal=causal, **bounds)
        assert torch.equal(a, b)
        check_attend(cache, off, lens, table, q, scale, causal, window, a, None, dtype)
    c.check()


@pytest.mark.parametrize("new", [1, 5, 140])
def test_attend_sharp_rows_and_small_scales(new):
    """Rows that see one key only in effect, rows of zeros, queries far outside fp16's range, pages whose value
    scales differ by 2^20, zero scales."""
    H, d, P, heads, lens = 2, 128, 32, 8, [500]
    cache, table = make(lens, H, d, P, 5, garbage=False)
    cache["v_scale"][table[0][::3][:5]] *= np.float32(2.0 ** -20)
    cache["v_scale"][table[0][4], 0] = 0
    cache["v_codes"][table[0][4], 0] = 0
    q = tokens(new, heads, d, torch.bfloat16, 6)
    q[:, 0] *= 1e4
    q[:, 1] = 0
    q[:, 2] *= 1e-30
    q[:, 3] *= 300
    q = q.cuda()
    c = up(cache)
    out, lse = c.attend(q, i32([0, new]), i32(lens), i32(table), max_new=new, max_len=500, return_lse=True)
    check_attend(cache, [0, new], lens, table, q, 1 / math.sqrt(d), True, 0, out, lse, torch.bfloat16)


def test_attend_many_sequences_and_a_long_one():
    """Lengths from 0 to thousands in one call: the work is shared out, no sequence is forgotten."""
    g = np.random.default_rng(0)
    lens = [int(x) for x in np.exp(g.uniform(0, np.log(300), 150))] + [6000, 0, 1]
    new = [1] * 153
    H, d, P, heads = 1, 64, 16, 4
    cache, table = make(lens, H, d, P, 9)
    off = np.arange(154)
    q = tokens(153, heads, d, torch.float16, 1).cuda()
    c = up(cache)
    out, lse = c.attend(q, i32(off), i32(lens), i32(table), max_new=1, max_len=6000, return_lse=True)
    c.check()
    check_attend(cache, off, lens, table, q, 1 / 8.0, True, 0, out, lse, torch.float16)


def test_attend_past_32_bit_offsets():
    """Pages whose codes lie more than 2^31 bytes from the start."""
    H, d, P, n_pages = 8, 128, 128, 16500                   # 2.16 GB of codes each for keys and values
    c = serving.PagedCache8.empty(n_pages, H, d, P)
    g = torch.Generator(device="cuda").manual_seed(1)
    last = [n_pages - 1, n_pages - 7]
    for t in (c.k_codes, c.v_codes):
        t[last] = torch.randint(-127, 128, (2, H, P, d), generator=g, device="cuda", dtype=torch.int8)
    for t in (c.k_scale, c.v_scale):
        t[last] = 0.01
    small = serving.PagedCache8.empty(2, H, d, P)
    for a, b in ((c.k_codes, small.k_codes), (c.v_codes, small.v_codes), (c.k_scale, small.k_scale), (c.v_scale, small.v_scale)):
        b.copy_(a[last])
    for new in (1, 130):
        q = tokens(new, 8, d, torch.bfloat16, 2).cuda()
        args = dict(max_new=new, max_len=200)
        far = c.attend(q, i32([0, new]), i32([200]), i32([last]), **args)
        near = small.attend(q, i32([0, new]), i32([200]), i32([[0, 1]]), **args)
        assert torch.equal(far, near)
        k = tokens(new, H, d, torch.bfloat16, 3).cuda()
        c.append(k, k, i32([0, new]), i32([200 + new]), i32([last + [5]]))
        small2 = serving.PagedCache8.empty(3, H, d, P)
        for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
            getattr(small2, name)[:2].copy_(getattr(small, name))
        small2.append(k, k, i32([0, new]), i32([200 + new]), i32([[0, 1, 2]]))
        assert torch.equal(c.k_codes[last], small2.k_codes[:2])
        kk, _ = c.read(i32([0, 50]), i32([200 + new]), i32([last + [5]]), 50)
        k2, _ = small2.read(i32([0, 50]), i32([200 + new]), i32([[0, 1, 2]]), 50)
        assert torch.equal(kk, k2)
        for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
            getattr(small, name).copy_(getattr(c, name)[last])


def test_refusals():
    with pytest.raises(B.CmpqError) as e:
        c = serving.PagedCache8.empty(2, 1, 80, 16)
        c.read(i32([0, 1]), i32([1]), i32([[0]]), 1)
    assert e.value.status == 2
    c = serving.PagedCache8.empty(2, 2, 64, 16)
    q = torch.zeros(1, 3, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError):
        c.attend(q, i32([0, 1]), i32([1]), i32([[0]]), max_new=1)
    q = torch.zeros(1, 4, 64, dtype=torch.float16, device="cuda")
    for bad in (dict(scale=0.0), dict(scale=float("nan")), dict(window=-1), dict(window=3, causal=False), dict(max_len=-1)):
        with pytest.raises(B.CmpqError) as e:
            c.attend(q, i32([0, 1]), i32([1]), i32([[0]]), max_new=1, **bad)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        c.attend(q, i32([0, 1]).long(), i32([1]), i32([[0]]), max_new=1)
    with pytest.raises(ValueError):
        c.attend(q.transpose(1, 2).contiguous().transpose(1, 2), i32([0, 1]), i32([1]), i32([[0]]), max_new=1)
    with pytest.raises(ValueError):
        c.append(q[:, :1], q[:, :1], i32([0, 1]), i32([1]), i32([[0]]))
    with pytest.raises(TypeError):
        c.append(q[:, :2].float(), q[:, :2].float(), i32([0, 1]), i32([1]), i32([[0]]))
    empty = torch.zeros(0, 2, 64, dtype=torch.float16, device="cuda")
    c.append(empty, empty, i32([0]), torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 1, dtype=torch.int32, device="cuda"))
    assert c.attend(torch.zeros(0, 4, 64, dtype=torch.float16, device="cuda"), i32([0, 0]), i32([5]), i32([[0]]), max_new=0).shape[0] == 0
    c.check()


def test_layer_runs_them_together():
    """Projections, append, attention and output of the block against the same steps on 64-bit values of what the
    block stored: a prompt, then token by token."""
    d_model, heads, H, d, P = 192, 4, 2, 64, 16
    g = torch.Generator().manual_seed(3)
    w = (torch.randn((heads + 2 * H) * d, d_model, generator=g) * 0.05).to(torch.bfloat16).cuda()
    wo = (torch.randn(d_model, heads * d, generator=g) * 0.05).to(torch.bfloat16).cuda()
    cos, sin = (torch.from_numpy(x).cuda() for x in rope(64, d))
    cache = serving.PagedCache8.empty(8, H, d, P)
    layer = serving.AttentionLayer8(serving.Int8Linear.from_weight(w), serving.Int8Linear.from_weight(wo), cache, heads, cos, sin)
    lens, table = np.array([20, 33]), i32([[0, 1, 2], [3, 4, 5]])
    new = lens.copy()
    for step in range(4):
        off = np.concatenate(([0], np.cumsum(new)))
        x = torch.randn(int(off[-1]), d_model, generator=g).to(torch.bfloat16).cuda()
        y = layer(x, i32(off), i32(lens), table, max_new=int(new.max()), max_len=48)
        qkv = layer.qkv(x)
        pos = np.concatenate([np.arange(m - n, m) for m, n in zip(lens, new)])
        q = ref.rotate(qkv[:, : heads * d].unflatten(1, (heads, d)).float().cpu().numpy(), pos, cos.cpu().numpy(), sin.cpu().numpy(), False)
        held = {n: getattr(cache, n).cpu().numpy() for n in ("k_codes", "k_scale", "v_codes", "v_scale")}
        a = ref.attend(held, off, lens, table.cpu().numpy(), torch.from_numpy(q).bfloat16().float().numpy(), 1 / 8.0)[0]
        want = layer.out(torch.from_numpy(a).bfloat16().flatten(1).cuda())
        # the attention's roundings may turn an activation code by one: 2 / 127 of the row's largest for few entries
        assert (y.double() - want.double()).norm() <= 0.02 * want.double().norm()
        lens, new = lens + 1, np.array([1, 1])
    cache.check()


@pytest.mark.parametrize("new", [1, 5, 140])
def test_attend_queries_at_the_ends_of_bf16(new):
    """Rows of subnormals with zeros between, down to the smallest, and rows that reach 2^127: `scale` and the keys'
    scales bring their scores to ordinary size, so the tolerance stays as sharp as elsewhere."""
    H, d, P, heads, lens = 2, 128, 32, 4, [300]
    g = np.random.default_rng(11)
    cache, table = make(lens, H, d, P, 6, garbage=False)
    for exponents, scale, keys in (((-133, -131, -129, -126), 2.0 ** 100, 2.0 ** 28), ((127, 126, 127, 125), 2.0 ** -90, 2.0 ** -34)):
        x = np.zeros((new, heads, d))
        for h, e in enumerate(exponents):
            steps = g.integers(-3, 4, size=(new, d)) * (g.random((new, d)) < 0.6)
            steps[:, 0] = 1                                # no row is zero, none is larger than 1.75 * 2^e
            x[:, h] = steps * 2.0 ** e * (1.0 if e == -133 else 0.5)
        q = torch.from_numpy(x).to(torch.bfloat16)
        assert np.array_equal(q.double().numpy(), x)       # bf16 holds them
        c = {**cache, "k_scale": (cache["k_scale"] * np.float32(keys)).astype(np.float32)}
        held = up(c)
        out, lse = held.attend(q.cuda(), i32([0, new]), i32(lens), i32(table), max_new=new, max_len=300, scale=scale, return_lse=True)
        held.check()
        check_attend(c, [0, new], lens, table, q, scale, True, 0, out, lse, torch.bfloat16)


def check_weights(cache, pages, q, scale, got, lse, length, window=0):
    """One sequence, against float64, with nothing in the tolerance that is relative to values a row hardly weighs.  Weights
    times value scales are rounded to fp16 with the largest of a row, w, at 2^7 or above: relative 2^-11, or 2^-25 absolute,
    which is 2^-32 w.  So |out - ref| <= (2^-10 + 4 ds) sum p|v| + L 2^-32 * 127 w + half ulp."""
    n, heads, d = q.shape
    H, P = cache["k_codes"].shape[1], cache["k_codes"].shape[2]
    kc, vc = (cache[x][pages].transpose(0, 2, 1, 3).reshape(-1, H, d)[:length].astype(np.float64) for x in ("k_codes", "v_codes"))
    ks, vs = (np.repeat(cache[x][pages].astype(np.float64), P, 0)[:length] for x in ("k_scale", "v_scale"))
    x, y = q.double().cpu().numpy(), got.double().cpu().numpy()
    for h in range(heads):
        kh = h // (heads // H)
        k, S = kc[:, kh] * ks[:, kh, None], vs[:, kh]
        s = scale * (x[:, h] @ k.T)
        pos, key = np.arange(length - n, length)[:, None], np.arange(length)
        s[(key > pos) | ((key <= pos - window) if window else False)] = -np.inf
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1, keepdims=True)
        p /= total
        ds = (d + 8) * 2.0 ** -23 * scale * (np.abs(x[:, h]) @ np.abs(k).T * np.isfinite(s)).max(1)
        want, size = (p * S) @ vc[:, kh], (p * S) @ np.abs(vc[:, kh])
        floor = length * 2.0 ** -32 * 127 * (p * S).max(1)
        tol = (2.0 ** -10 + 4 * ds)[:, None] * size + floor[:, None] + ref.half_ulp(np.abs(want) + 2.0 ** -9 * size, got.dtype)
        bad = ~(np.abs(y[:, h] - want) <= tol)
        assert not bad.any(), (h, int(bad.sum()), np.argwhere(bad)[:4], y[:, h][bad][:4], want[bad][:4])
        l = (top + np.log(total))[:, 0]
        assert np.all(np.abs(lse[:, h].double().cpu().numpy() - l) <= 2 * ds + 2.0 ** -20 * (1 + np.abs(l)))


@pytest.mark.parametrize("ratio", [2.0 ** -16, 2.0 ** -27, 2.0 ** -60])
@pytest.mark.parametrize("new,d,P,window", [(1, 64, 16, 0), (1, 128, 64, 0), (1, 256, 32, 0), (7, 128, 16, 0), (7, 128, 128, 150), (140, 64, 32, 0),
                                            (300, 128, 16, 0), (300, 128, 64, 64), (300, 256, 128, 0), (513, 64, 128, 0)])
def test_attend_value_scales_of_pages_that_a_row_does_not_weigh(new, d, P, window, ratio):
    """Value scales that are far apart.  Head 0: small ones on the early pages, large ones on the pages that only later rows
    see.  Head 1: small ones on every other page, and all of a row's weight there.  Head 2: the large ones on the first page,
    far behind a window or hardly weighed."""
    H, L = 3, 700
    g = np.random.default_rng(d + P)
    cache, table = make([L], H, d, P, 2, garbage=False)
    pages = table[0][: -(-L // P)].astype(int)
    sign = g.choice([-1, 1], size=(2, d)).astype(np.int8)
    small = np.zeros((len(pages), H), bool)
    small[: max(1, len(pages) // 2), 0] = True
    small[::2, 1] = True
    small[1:, 2] = True
    cache["k_scale"][:] = np.float32(0.01)
    cache["v_scale"][pages] *= np.where(small, np.float32(ratio), np.float32(1))
    turn = g.integers(1, 60, size=(len(pages), P, d)).astype(np.int8) * sign[0]
    cache["k_codes"][pages, 1] = np.where(small[:, 1, None, None], turn, -turn)
    cache["k_codes"][pages, 2] = np.where(small[:, 2, None, None], turn, -turn)
    q = tokens(new, H, d, torch.float16, 3).float().numpy()
    q[:, 1:] = np.abs(q[:, 1:]) * sign[0] * (0.5 + 4.0 / np.sqrt(d))
    q = torch.from_numpy(q).half().cuda()
    c = up(cache)
    scale = 12 / math.sqrt(d)                              # heads 1 and 2: the large pages lie some e^-40 behind
    out, lse = c.attend(q, i32([0, new]), i32([L]), i32(table), max_new=new, max_len=L, scale=scale, window=window, return_lse=True)
    c.check()
    check_weights(cache, pages, q, scale, out, lse, L, window)
    low = c.attend(q.bfloat16(), i32([0, new]), i32([L]), i32(table), max_new=new, max_len=L, scale=scale, window=window, return_lse=True)
    check_weights(cache, pages, q.bfloat16(), scale, *low, L, window)


@pytest.mark.parametrize("new", [1, 65])
def test_attend_many_keys_of_small_weight(new):
    """131072 keys, one of them with 2^25.5 times the weight of each other one and values of zero: all of the output comes
    from weights that plain fp16 would round to nothing."""
    H, d, P, L = 1, 64, 128, 131072
    cache, table = make([L], H, d, P, 3, garbage=False)
    pages = table[0][: L // P].astype(int)
    cache["k_codes"][:] = 0
    cache["k_scale"][:] = np.float32(0.125)
    cache["k_codes"][pages[7], 0, 5] = 64
    cache["v_codes"][:] = np.abs(cache["v_codes"])
    cache["v_codes"][pages[7], 0, 5] = 0
    cache["v_scale"][:] = np.float32(0.02)
    q = torch.full((new, 2, d), 0.5, dtype=torch.bfloat16, device="cuda")
    scale = 25.5 * math.log(2) / (64 * 0.125 * 0.5 * d)
    c = up(cache)
    out, lse = c.attend(q, i32([0, new]), i32([L]), i32(table), max_new=new, max_len=L, scale=scale, return_lse=True)
    c.check()
    check_weights(cache, pages, q, scale, out, lse, L)


@pytest.mark.parametrize("lens,new,d", [([2, 5, 40], [6, 7, 40], 64), ([3, 1], [9, 260], 128), ([3, 200], [300, 140], 128), ([2, 30], [9, 30], 256)])
def test_attend_windows_that_reach_everything(lens, new, d):
    """`No limit` written as the largest integer, with rows before the first token: the same bytes as no window.  A bound of
    the lengths that is nearly as large keeps the window, and the answer."""
    H, P, heads = 2, 16, 4
    cache, table = make(lens, H, d, P, 3)
    off = np.concatenate(([0], np.cumsum(new)))
    q = tokens(int(off[-1]), heads, d, torch.bfloat16, 5).cuda()
    c = up(cache)
    run = lambda **kw: c.attend(q, i32(off), i32(lens), i32(table), max_new=max(new), return_lse=True, **kw)
    out, lse = run(max_len=max(lens))
    check_attend(cache, off, lens, table, q, 1 / math.sqrt(d), True, 0, out, lse, torch.bfloat16)
    for window in (2 ** 31 - 1, 2 ** 31 - 3, 2 ** 40):
        o, l = run(max_len=max(lens), window=window)
        assert torch.equal(o, out) and torch.equal(l, lse)
    o, l = run(max_len=2 ** 31 - 257, window=2 ** 31 - 258)
    check_attend(cache, off, lens, table, q, 1 / math.sqrt(d), True, 0, o, l, torch.bfloat16)
    c.check()


@pytest.mark.parametrize("d", [64, 256])
def test_attend_with_a_loose_bound_of_the_new_tokens(d):
    """max_new is a bound: the largest integer gives the answer that the exact one gives, in the same bytes where that
    bound names as many tokens as there are."""
    lens, H, P, heads = [30] * 200, 2, 16, 4
    cache, table = make(lens, H, d, P, 3)
    q = tokens(200, heads, d, torch.float16, 5).cuda()
    c, off = up(cache), np.arange(201)
    a = c.attend(q, i32(off), i32(lens), i32(table), max_new=2 ** 31 - 1, max_len=30)
    assert torch.equal(a, c.attend(q, i32(off), i32(lens), i32(table), max_new=200, max_len=30))
    check_attend(cache, off, lens, table, q, 1 / math.sqrt(d), True, 0, a, None, torch.float16)
    c.check()


@pytest.mark.parametrize("row", [0, 2], ids=["first", "last"])
def test_a_table_that_is_part_of_a_wider_one_ends_with_its_columns(row):
    """Lengths that need more pages than the columns of the table given: reported, and nothing beyond the columns is used,
    though the wider table has pages there (and memory ends behind its last row)."""
    H, d, P = 2, 64, 16
    wide = i32(np.arange(18).reshape(3, 6))
    table = wide[:, 3:5]                                   # two pages a sequence, row stride 6
    lens = [20, 20, 20]
    k = tokens(3, H, d, torch.float16, 1).cuda()
    c = serving.PagedCache8.empty(18, H, d, P)
    args = (i32([0, 1, 2, 3]), i32(lens), table)
    c.append(k, k, *args)
    c.check()
    same = serving.PagedCache8.empty(18, H, d, P)
    same.append(k, k, args[0], args[1], table.contiguous())
    assert torch.equal(c.k_codes, same.k_codes) and torch.equal(c.attend(k, *args, 1), same.attend(k, *args[:2], table.contiguous(), 1))
    lens[row] = 33
    for new in (1, 70):                                    # few rows; many, in the kernel for prompts
        before = [t.clone() for t in (c.k_codes, c.k_scale, c.v_codes, c.v_scale)]
        off = np.arange(4) if new == 1 else np.concatenate(([0], np.cumsum([new if s == row else 0 for s in range(3)])))
        lens[row] = 33 if new == 1 else 100
        x = tokens(int(off[-1]), H, d, torch.float16, 2).cuda()
        q = tokens(int(off[-1]), 4 * H, d, torch.float16, 3).cuda()
        for call in (lambda: c.append(x, x, i32(off), i32(lens), table), lambda: c.read(i32(off), i32(lens), table, int(off[-1])),
                     lambda: c.attend(q, i32(off), i32(lens), table, new, 200)):
            call()
            with pytest.raises(B.CmpqError) as e:
                c.check()
            assert e.value.status == 1
        others = [p for p in range(18) if p not in wide[:, 3:5].flatten().tolist()]
        for t, was in zip((c.k_codes, c.k_scale, c.v_codes, c.v_scale), before):
            assert torch.equal(t[others], was[others])


def test_binding_of_the_c_calls():
    """The ctypes wrappers make the calls that the extension makes: same bytes, same errors."""
    H, d, P, heads, lens = 2, 64, 16, 4, [40, 17]
    k, v, q = tokens(20, H, d, torch.float16, 1).cuda(), tokens(20, H, d, torch.float16, 2).cuda(), tokens(20, heads, d, torch.float16, 3).cuda()
    cos, sin = (torch.from_numpy(x).cuda() for x in rope(64, d))
    off, length, table = i32([0, 3, 20]), i32(lens), i32([[0, 1, 2], [4, 5, 6]])
    one, two = (up(make(lens, H, d, P, 8, garbage=False)[0]) for _ in range(2))
    assert one.n_pages >= 7
    want_q = one.append(k, v, off, length, table, q=q, cos=cos, sin=sin)
    want_k, want_v = one.read(off, length, table, 20, torch.float16)
    want, want_lse = one.attend(want_q, off, length, table, 17, 48, return_lse=True)
    c = B.Cache(*(t.data_ptr() for t in (two.k_codes, two.k_scale, two.v_codes, two.v_scale)), two.n_pages, H, d, P)
    b = B.Batch(off.data_ptr(), length.data_ptr(), table.data_ptr(), 3, 2, 20, 3)
    got_q, got_k, got_v, out, word = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(q), i32([0])
    lse = torch.empty(20, heads, device="cuda")
    B.cmpq_cache_append(c, b, k, v, cos, sin, False, q, got_q, word)
    B.cmpq_cache_read(c, b, got_k, got_v, word)
    ws = torch.zeros(B.cmpq_cache_attention_ws_bytes(2, 20, 17, 48, heads, H, d), dtype=torch.uint8, device="cuda")
    B.cmpq_cache_attention(c, b, got_q, 17, 48, 1 / math.sqrt(d), True, 0, out, lse, ws, word)
    B.cmpq_check_cache(word)
    for x, y in ((got_q, want_q), (got_k, want_k), (got_v, want_v), (out, want), (lse, want_lse), (two.k_codes, one.k_codes), (two.v_scale, one.v_scale)):
        assert torch.equal(x, y)
    length[1] = 49                                         # past the table
    B.cmpq_cache_read(c, b, got_k, got_v, word)
    with pytest.raises(B.CmpqError) as e:
        B.cmpq_check_cache(word)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        B.cmpq_cache_read(c, b, got_k, got_v[:, :, :32], word)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,d,P", [(1, 64, 16), (1, 128, 64), (3, 256, 32), (9, 128, 16), (40, 64, 64), (200, 128, 32), (300, 64, 16)])
def test_attend_rows_that_see_one_key_return_its_value(new, d, P, dtype):
    """With a window of one a row's output is its own token's value: the largest weight times scale is a power of two in
    fp16, so nothing but the fp32 division (2^-20 of the value) and the last rounding is between them."""
    H, heads, L = 2, 4, 310
    cache, table = make([L], H, d, P, 7, garbage=False)
    q = tokens(new, heads, d, dtype, 3).cuda()
    c = up(cache)
    out, lse = c.attend(q, i32([0, new]), i32([L]), i32(table), max_new=new, max_len=L, window=1, return_lse=True)
    c.check()
    pages = table[0][: -(-L // P)].astype(int)
    v, k = ((cache[x + "_codes"][pages].astype(np.float64) * cache[x + "_scale"][pages].astype(np.float64)[..., None, None])
            .transpose(0, 2, 1, 3).reshape(-1, H, d)[L - new: L].repeat(heads // H, 1) for x in "vk")
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - v) <= 2.0 ** -20 * np.abs(v) + ref.half_ulp(np.abs(v) * (1 + 2.0 ** -20), dtype))
    x = q.double().cpu().numpy()
    s, ds = (x * k).sum(2) / math.sqrt(d), (d + 8) * 2.0 ** -23 * (np.abs(x) * np.abs(k)).sum(2) / math.sqrt(d)
    assert np.all(np.abs(lse.double().cpu().numpy() - s) <= 2 * ds + 2.0 ** -20 * (1 + np.abs(s)))
