"""Cases, plain forms and 64-bit definitions of the 8-bit serving operators.

Three operators serve a layer whose activations and cache are held in 8 bits: the linear layer (tokens are
quantized to 8-bit integers, multiplied with 8-bit weights, scaled per token and output channel), the append to
the paged cache (rotation by position, one scale per page and head, read back afterwards) and the attention over
that cache.  `run` computes them with elementary torch operations in 32 bits while `own` is false and through
paper_2410_13056_b200.serving while it is true.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
_SCALE_LO, _SCALE_HI = 2.0 ** -60, 2.0 ** 60


# ---- cases ---------------------------------------------------------------------------------------------------

def _linear(name, n, d_in, d_out, dtype, bias):
    return {"name": name, "op": "linear", "n": n, "d_in": d_in, "d_out": d_out, "dtype": dtype, "bias": bias}


def _cache(name, op, seqs, new, length, hq, hkv, d, page, dtype, shape_seed, **more):
    c = {"name": name, "op": op, "seqs": seqs, "new": new, "len": length, "hq": hq, "hkv": hkv, "d": d, "page": page,
         "dtype": dtype, "shape_seed": shape_seed}
    c.update(more)
    return c


def listed():
    return [
        # one generated token through an attention projection: the time of the call itself counts
        _linear("linear one token", 1, 4096, 4096, "bf16", False),
        # a decoding batch through an up projection, with a bias and a token count that fills no tile
        _linear("linear batch 37", 37, 4096, 11008, "fp16", True),
        # a chunk of a prompt through a down projection, neither size a multiple of a tile
        _linear("linear chunk 1000", 1000, 11008, 4096, "bf16", False),
        # whole prompts through the largest layer of the largest workload
        _linear("linear prompts 4096", 4096, 8192, 28672, "bf16", False),
        # one stream generating: one token joins a page that already holds others
        _cache("append one token", "append", 1, 1, 1025, 32, 32, 128, 64, "bf16", 1, rot=128, interleaved=False),
        # a batch of generating streams, grouped heads
        _cache("append batch 64", "append", 64, 1, 4001, 64, 8, 128, 64, "fp16", 2, rot=128, interleaved=False),
        # prompts of uneven lengths, some continuing a half-filled page; half of each head is rotated, in pairs
        _cache("append prompts", "append", 5, 4096, 5000, 64, 8, 128, 32, "bf16", 3, rot=64, interleaved=True),
        # one stream generating, every query head with its own keys
        _cache("attend one token", "attend", 1, 1, 2049, 32, 32, 128, 64, "bf16", 4, window=0),
        # a batch of generating streams of very different lengths
        _cache("attend batch 64", "attend", 64, 1, 8191, 64, 8, 128, 64, "bf16", 5, window=0),
        # two streams with very long caches: few rows, a long axis
        _cache("attend long", "attend", 2, 1, 131072, 64, 8, 128, 128, "fp16", 6, window=0),
        # a few drafted tokens per stream, small heads, a sliding window
        _cache("attend drafts", "attend", 16, 5, 4093, 64, 8, 64, 16, "fp16", 7, window=1024),
        # prompts that continue a cached prefix
        _cache("attend prompts", "attend", 2, 2048, 6145, 32, 32, 128, 64, "bf16", 8, window=0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "append", "attend", "attend"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "linear":
        while True:
            n, d_in, d_out = _log_int(rng, 1, 4096), _log_int(rng, 512, 11008), _log_int(rng, 512, 28672)
            if rng.random() < 0.6:  # most layers have round sizes
                d_in, d_out = (d_in + 127) // 128 * 128, (d_out + 127) // 128 * 128
            if 3072 not in (n, d_in, d_out) and n * d_in * d_out <= 4096 * 8192 * 28672:
                break
        c = _linear("", n, d_in, d_out, dtype, rng.random() < 0.5)
    else:
        d, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
        while True:
            hkv = rng.choice([1, 4, 8, 32])
            hq = hkv * rng.choice([1, 2, 4, 8] if hkv <= 8 else [1, 2])
            if (hq + 2 * hkv) * d != 3072:
                break
        shape_seed = rng.randrange(1 << 20)
        if op == "append":
            while True:
                if rng.random() < 0.5:
                    seqs, new = _log_int(rng, 1, 128), 1
                else:
                    seqs, new = rng.randint(1, 6), _log_int(rng, 2, 4096)
                length = new + _log_int(rng, 1, 5000)
                if 3072 not in (new, length) and seqs * new * (hq + 4 * hkv) * d <= 5 * 4096 * 96 * 128:
                    break
            c = _cache("", op, seqs, new, length, hq, hkv, d, page, dtype, shape_seed, rot=rng.choice([d, d // 2]),
                       interleaved=rng.random() < 0.3)
        else:
            while True:
                kind = rng.random()
                seqs = _log_int(rng, 1, 64)
                new = 1 if kind < 0.5 else rng.randint(2, 8) if kind < 0.75 else _log_int(rng, 16, 2048)
                seqs = seqs if new <= 8 else min(seqs, 4)
                length = new + _log_int(rng, 16, 131072 if new <= 8 else 6144)
                if (3072 not in (new, length) and seqs * length * hkv * d <= 64 * 8192 * 8 * 128 and seqs * new * length * hq * d <= 2 * 2048 * 6145 * 32 * 128
                        and seqs * new * length * hq <= 1 << 30):
                    break
            c = _cache("", op, seqs, new, length, hq, hkv, d, page, dtype, shape_seed,
                       window=rng.choice([0, 0, 0, _log_int(rng, 1, length)]))
    del c["name"]
    return c


def _lengths(case):
    """Tokens in the cache after the call and new tokens of each sequence; the first has the most of both."""
    r = random.Random(case["shape_seed"])
    new, lens = [], []
    for s in range(case["seqs"]):
        if s == 0:
            n, length = case["new"], case["len"]
        else:
            n = 1 if case["new"] == 1 else r.randint(0 if s % 4 == 3 else 1, case["new"])
            length = max(n, r.randint(max(1, case["len"] // 8), case["len"]))
        new.append(n)
        lens.append(length)
    return new, lens


def _visible(case):
    """Pairs of a query and a key that it sees, and cached tokens that any query of their sequence sees."""
    pairs = tokens = 0
    for n, length in zip(*_lengths(case)):
        w = case["window"] or length
        first = length - n  # tokens before the first query
        pairs += sum(min(first + i + 1, w) for i in range(n))
        tokens += length - max(0, first + 1 - w) if n else 0
    return pairs, tokens


# ---- inputs --------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _prepare_linear(case, seed):
    g, dt = _gen(seed), _DT[case["dtype"]]
    n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
    # channels of very different size, one in a hundred far out: what 8-bit activations meet
    sigma = torch.exp(0.5 * _randn(g, d_in))
    sigma[torch.randperm(d_in, generator=g, device="cuda")[: max(1, d_in // 100)]] *= 8.0
    x = (_randn(g, n, d_in) * sigma).to(dt)
    w = _randn(g, d_out, d_in) * 0.02
    scale = w.abs().amax(1) * (1.0 / 127.0)
    ld = (d_in + 15) // 16 * 16  # rows of the weight codes start on 16 bytes
    codes = torch.zeros(d_out, ld, dtype=torch.int8, device="cuda")
    codes[:, :d_in] = torch.round(w / scale[:, None]).to(torch.int8)
    bias = (0.1 * _randn(g, d_out)).to(dt) if case["bias"] else None
    return {"x": x, "w_codes": codes[:, :d_in], "w_scale": scale, "bias": bias}


def _prepare_cache(case, seed):
    """A paged cache that holds each sequence's tokens (before the call's, for the append), pages in random order."""
    g, dt = _gen(seed), _DT[case["dtype"]]
    new, lens = _lengths(case)
    page, hkv, d, hq = case["page"], case["hkv"], case["d"], case["hq"]
    per = [-(-length // page) for length in lens]
    n_pages = sum(per) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(per)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, p in enumerate(per):
        table[s, :p] = order[at: at + p]
        at += p
    st = {"table": table, "lens": _ints(lens), "page": page, "max_new": max(new),
          "tok_off": _ints([sum(new[:s]) for s in range(len(new) + 1)])}
    sigma = torch.exp(0.4 * _randn(g, 1, hkv, 1, d))
    for name, spread in (("k", sigma), ("v", 0.7)):
        values = _randn(g, n_pages, hkv, page, d) * spread * torch.exp(0.2 * _randn(g, n_pages, hkv, 1, 1))
        scale = values.abs().amax((2, 3)) * (1.0 / 127.0)
        st[name + "_scale"] = scale
        st[name + "_codes"] = torch.round(values / scale[:, :, None, None]).to(torch.int8)
        del values
    # queries, keys and values are columns of one projection's output, as a fused projection leaves them
    n_tok = sum(new)
    qkv = _randn(g, n_tok, (hq + 2 * hkv) * d)
    qkv[:, hq * d: (hq + hkv) * d] *= sigma.reshape(1, -1)
    qkv = qkv.to(dt)
    st["q"] = qkv[:, : hq * d].unflatten(1, (hq, d))
    st["k"] = qkv[:, hq * d: (hq + hkv) * d].unflatten(1, (hkv, d))
    st["v"] = qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d))
    return st, new, lens


def _prepare_append(case, seed):
    st, new, lens = _prepare_cache(case, seed)
    page, rot = case["page"], case["rot"]
    # the cache starts a little smaller than the new tokens, so that some pages have to be scaled anew
    st["k_scale"] *= 0.8
    st["v_scale"] *= 0.8
    angle = (torch.arange(case["len"], device="cuda", dtype=torch.float64)[:, None]
             * torch.pow(10000.0, -torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot))
    st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
    st["interleaved"] = case["interleaved"]
    # what is read back: every token of the pages that the new tokens touch
    back = [0 if n == 0 else n + (length - n) % page for n, length in zip(new, lens)]
    st["read_off"] = _ints([sum(back[:s]) for s in range(len(back) + 1)])
    st["n_read"] = sum(back)
    table = st["table"].tolist()
    st["touched"] = _ints([table[s][p] for s, (n, length) in enumerate(zip(new, lens)) if n
                           for p in range((length - n) // page, -(-length // page))], torch.int64)
    return st


def _prepare_attend(case, seed):
    st, _, _ = _prepare_cache(case, seed)
    st["softmax_scale"] = 1.0 / math.sqrt(case["d"])
    st["window"] = case["window"]
    st["max_len"] = case["len"]
    return st


def prepare(case, seed):
    st = {"linear": _prepare_linear, "append": _prepare_append, "attend": _prepare_attend}[case["op"]](case, seed)
    st["op"] = case["op"]
    return st


# ---- plain forms ---------------------------------------------------------------------------------------------

def _plain_linear(st):
    x = st["x"].float()
    scale = x.abs().amax(1, keepdim=True) * (1.0 / 127.0)
    inv = torch.where(scale > 0, torch.reciprocal(scale), torch.zeros_like(scale))
    codes = torch.round(x * inv).clamp(-127, 127)
    y = (codes @ st["w_codes"].float().t()) * scale * st["w_scale"]
    if st["bias"] is not None:
        y = y + st["bias"].float()
    return {"y": y.to(st["x"].dtype)}


def _token_places(off, lens, n):
    """Sequence and position of each of n tokens, of which off[s]..off[s+1] are the last ones of sequence s."""
    t = torch.arange(n, device=off.device, dtype=torch.int32)
    s = torch.searchsorted(off, t, right=True) - 1
    return s, lens[s] - off[s + 1] + t


def _rotate(x, cos, sin, interleaved):
    rot = 2 * cos.shape[1]
    c, s = cos[:, None, :], sin[:, None, :]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_append(st):
    n, P = st["q"].shape[0], st["page"]
    s, pos = _token_places(st["tok_off"], st["lens"], n)
    cos, sin = st["cos"][pos], st["sin"][pos]
    q = _rotate(st["q"].float(), cos, sin, st["interleaved"]).to(st["q"].dtype)
    page, slot = st["table"][s, pos // P].long(), (pos % P).long()
    n_pages, hkv = st["k_scale"].shape
    touched = st["touched"]
    first = torch.full((n_pages,), P, device=q.device, dtype=torch.int64).scatter_reduce(0, page, slot, "amin")[touched]
    old = torch.arange(P, device=q.device) < first[:, None]
    for name, x in (("k", _rotate(st["k"].float(), cos, sin, st["interleaved"])), ("v", st["v"].float())):
        codes, scale = st[name + "_codes"], st[name + "_scale"]
        amax = torch.zeros(n_pages, hkv, device=q.device).index_reduce_(0, page, x.abs().amax(-1), "amax")[touched]
        before = torch.where(first[:, None] > 0, scale[touched], torch.zeros_like(amax))
        after = torch.maximum(before, (amax * (1.0 / 127.0)).clamp(_SCALE_LO, _SCALE_HI))
        inv = torch.reciprocal(after)
        held = codes[touched]
        again = torch.round(held.float() * (before * inv)[:, :, None, None]).clamp(-127, 127).to(torch.int8)
        grew = (after > before)[:, :, None, None] & old[:, None, :, None]
        codes[touched] = torch.where(grew, again, held)
        scale[touched] = after
        codes[page, :, slot] = torch.round(x * torch.reciprocal(scale[page])[:, :, None]).clamp(-127, 127).to(torch.int8)
    s, pos = _token_places(st["read_off"], st["lens"], st["n_read"])
    page, slot = st["table"][s, pos // P].long(), (pos % P).long()
    back = [(st[x + "_codes"][page, :, slot].float() * st[x + "_scale"][page][:, :, None]).to(q.dtype) for x in "kv"]
    return {"q": q, "k": back[0], "v": back[1], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _plain_attend(st):
    q, P, table, lens, off = st["q"], st["page"], st["table"].long().clamp(min=0), st["lens"], st["tok_off"].long()
    n, hq, d = q.shape
    B, hkv, m = table.shape[0], st["k_scale"].shape[1], st["max_new"]

    def held(name):  # [B][hkv][tokens][d], in 32 bits
        x = st[name + "_codes"][table].float() * st[name + "_scale"][table][..., None, None]
        return x.transpose(1, 2).reshape(B, hkv, -1, d)

    # queries of a sequence in rows of their own, the short ones filled up
    row = off[:-1, None] + torch.arange(m, device=q.device)
    real = row < off[1:, None]
    qs = q.float()[row.clamp(max=n - 1)]
    qs = qs.unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, d)
    score = (qs @ held("k").transpose(2, 3)).mul_(st["softmax_scale"]).unflatten(2, (-1, m))
    pos = (lens[:, None] - (off[1:, None] - row))[:, :, None]
    key = torch.arange(score.shape[-1], device=q.device)
    seen = (key <= pos) & real[:, :, None]
    if st["window"]:
        seen &= key > pos - st["window"]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ held("v")).unflatten(2, (-1, m)) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, m, hq, d)
    lse = lse.permute(0, 3, 1, 2).reshape(B, m, hq)
    s, _ = _token_places(st["tok_off"], lens, n)
    at = torch.arange(n, device=q.device) - off[s]
    return {"out": out[s, at].to(q.dtype), "lse": lse[s, at]}


# ---- the framework's operators -------------------------------------------------------------------------------

def _own(st):
    from paper_2410_13056_b200 import serving

    op = st["op"]
    if "handle" not in st:  # what a program makes once and keeps
        if op == "linear":
            st["handle"] = serving.Int8Linear(st["w_codes"], st["w_scale"], st["bias"])
        else:
            st["handle"] = serving.PagedCache8(st["k_codes"], st["k_scale"], st["v_codes"], st["v_scale"])
    h = st["handle"]
    if op == "linear":
        return {"y": h(st["x"])}
    if op == "append":
        q = h.append(st["k"], st["v"], st["tok_off"], st["lens"], st["table"], q=st["q"], cos=st["cos"], sin=st["sin"],
                     interleaved=st["interleaved"])
        k, v = h.read(st["read_off"], st["lens"], st["table"], st["n_read"], dtype=q.dtype)
        return {"q": q, "k": k, "v": v, "k_scale": h.k_scale, "v_scale": h.v_scale}
    out, lse = h.attend(st["q"], st["tok_off"], st["lens"], st["table"], max_new=st["max_new"], max_len=st["max_len"],
                        scale=st["softmax_scale"], window=st["window"], return_lse=True)
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "append": _plain_append, "attend": _plain_attend}[state["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    if case["op"] == "linear":
        n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
        return {"bytes": 2 * n * d_in + d_in * d_out + 4 * d_out + 2 * n * d_out + (2 * d_out if case["bias"] else 0),
                "flops": 2 * n * d_in * d_out}
    new, lens = _lengths(case)
    hq, hkv, d, page, n = case["hq"], case["hkv"], case["d"], case["page"], sum(new)
    if case["op"] == "append":
        back = sum(0 if m == 0 else m + (length - m) % page for m, length in zip(new, lens))
        pages = sum(-(-length // page) - (length - m) // page for m, length in zip(new, lens) if m)
        # rotated queries in and out, keys and values in, their codes out; then the pages' codes in, values out
        # (the whole arrays of scales come back as they stand: only the touched ones are read and written)
        return {"bytes": 4 * n * hq * d + 2 * n * hkv * d * (2 + 1) + 4 * n * case["rot"] + 2 * back * hkv * d * (1 + 2)
                + 4 * pages * hkv * 4,
                "flops": 3 * n * (hq + hkv) * case["rot"] + 4 * n * hkv * d + 2 * back * hkv * d}
    pairs, tokens = _visible(case)
    return {"bytes": 2 * tokens * hkv * d + 8 * (tokens // page + 1) * hkv + 4 * n * hq * d + 4 * n * hq,
            "flops": 4 * pairs * hq * d}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------

def _exact_linear(st):
    x = st["x"].double()
    top = x.abs().max(dim=1).values
    step = top / 127
    codes = torch.where(top[:, None] > 0, torch.round(x / step[:, None].clamp(min=1e-300)), torch.zeros_like(x))
    y = torch.matmul(codes, st["w_codes"].double().T) * torch.outer(step, st["w_scale"].double())
    return {"y": y if st["bias"] is None else y + st["bias"].double()}


def _turn64(x, pos, st):
    cos, sin = st["cos"].double()[pos], st["sin"].double()[pos]
    rot = 2 * cos.shape[1]
    i = torch.arange(rot // 2, device=x.device)
    lo, hi = (2 * i, 2 * i + 1) if st["interleaved"] else (i, i + rot // 2)
    y = x.clone()
    y[..., lo] = x[..., lo] * cos[:, None] - x[..., hi] * sin[:, None]
    y[..., hi] = x[..., hi] * cos[:, None] + x[..., lo] * sin[:, None]
    return y


def _exact_append(st):
    P, off, lens, table = st["page"], st["tok_off"].tolist(), st["lens"].tolist(), st["table"].tolist()
    codes = {x: st[x + "_codes"] for x in "kv"}
    scale = {x: st[x + "_scale"].double() for x in "kv"}
    q_out, back = [], {"k": [], "v": []}
    for s, length in enumerate(lens):
        n = off[s + 1] - off[s]
        if n == 0:
            continue
        start = length - n
        pos = torch.arange(start, length, device="cuda")
        q_out.append(_turn64(st["q"][off[s]: off[s + 1]].double(), pos, st))
        rows = {"k": _turn64(st["k"][off[s]: off[s + 1]].double(), pos, st), "v": st["v"][off[s]: off[s + 1]].double()}
        for p in range(start // P, -(-length // P)):
            lo, hi, at = max(start, p * P), min(length, (p + 1) * P), table[s][p]
            for x in "kv":
                fresh = rows[x][lo - start: hi - start].transpose(0, 1)  # [hkv][tokens][d]
                step = (fresh.abs().amax((1, 2)) / 127).clamp(_SCALE_LO, _SCALE_HI)
                held = codes[x][at][:, : lo - p * P].double()
                if lo > p * P:
                    was = scale[x][at].clone()
                    step = torch.maximum(step, was)
                    held = torch.round(held * (was / step)[:, None, None])
                scale[x][at] = step
                fresh = torch.round(fresh / step[:, None, None]).clamp(-127, 127)
                back[x].append((torch.cat((held, fresh), 1) * step[:, None, None]).transpose(0, 1))
    return {"q": torch.cat(q_out), "k": torch.cat(back["k"]), "v": torch.cat(back["v"]), "k_scale": scale["k"],
            "v_scale": scale["v"]}


def _exact_attend(st):
    off, lens, table, P = st["tok_off"].tolist(), st["lens"].tolist(), st["table"], st["page"]
    n, hq, d = st["q"].shape
    out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
    for s, length in enumerate(lens):
        m = off[s + 1] - off[s]
        if m == 0:
            continue
        ids = table[s, : -(-length // P)].long()
        i = torch.arange(length - m, length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")[None]
        hide = (j > i) if not st["window"] else (j > i) | (j <= i - st["window"])
        for h in range(st["k_scale"].shape[1]):
            k, v = ((st[x + "_codes"][ids, h].double() * st[x + "_scale"][ids, h].double()[:, None, None]).reshape(-1, d)[:length]
                    for x in "kv")
            g = hq // st["k_scale"].shape[1]
            q = st["q"][off[s]: off[s + 1], h * g: (h + 1) * g].double()
            a = torch.einsum("mgd,ld->gml", q, k) * st["softmax_scale"]
            a = a.masked_fill(hide[None], -math.inf)
            lse[off[s]: off[s + 1], h * g: (h + 1) * g] = torch.logsumexp(a, -1).T
            out[off[s]: off[s + 1], h * g: (h + 1) * g] = torch.einsum("gml,ld->mgd", torch.softmax(a, -1), v)
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    return {"linear": _exact_linear, "append": _exact_append, "attend": _exact_attend}[case["op"]](st)
