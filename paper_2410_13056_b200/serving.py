"""Serving with 8-bit activations and an 8-bit cache: what holds the buffers of those C-ABI calls.

`Int8Linear` is a linear layer with 8-bit weight codes, `PagedCache8` a paged cache of keys and values with a scale
per page and head (append, read back, attend), `AttentionLayer8` the attention block that runs them together: the
projections, the append with the rotation on the way, the attention over the cache and the output projection.
Everything is enqueued on the current torch stream; nothing is computed here.  The calls of the first two are
marshalled in C++ (csrc/serving_ext.cpp, built next to the library): wrong shapes and types raise ValueError and
TypeError, a status of the library CmpqError.

Work spaces: eager calls share one per device and stream, whatever layer or cache makes them.  All calls can be captured in
CUDA graphs; a captured call takes its work space from its graph, so graphs may be replayed in any order and on any stream.
"""
import torch

from . import binding as B
from . import build as _build


def _ext():
    """The extension module; raises if it was not built (run paper_2410_13056_b200/build.py)."""
    B.lib()
    try:
        from . import _serving
    except ImportError as e:
        raise RuntimeError("extension %s is missing or does not load: build it with `python -m paper_2410_13056_b200.build`"
                           % _build.EXT_PATH) from e
    return _serving


class Int8Linear:
    """y = x W^T + b with 8-bit codes on both sides.  w_codes: int8 [d_out][d_in], rows on multiples of 16 bytes;
    w_scale: fp32 [d_out]; bias: fp16/bf16 [d_out] or None (its dtype is then the activations')."""

    def __init__(self, w_codes, w_scale, bias=None):
        self._impl = _ext().Linear(w_codes, w_scale, bias)
        self.w_codes, self.w_scale, self.bias = w_codes, self._impl.w_scale, self._impl.bias
        self.d_out, self.d_in = w_codes.shape
        self.nonfinite = self._impl.nonfinite  # what check() looks at: bit 0 a NaN or an infinity, bit 3 a kernel gave up waiting

    @classmethod
    def from_weight(cls, weight, bias=None):
        """weight: fp16/bf16 [d_out][d_in]; every output channel gets its largest magnitude over 127 as scale."""
        d_out, d_in = weight.shape
        codes = torch.empty(d_out, (d_in + 15) // 16 * 16, dtype=torch.int8, device=weight.device)[:, :d_in]
        scale = torch.empty(d_out, dtype=torch.float32, device=weight.device)
        B.cmpq_quantize_tokens(weight, codes, scale)
        return cls(codes, scale, bias)

    def __call__(self, x, out=None):
        """x: fp16/bf16 [n][d_in].  Returns out [n][d_out] of x's dtype."""
        return self._impl(x, out)

    def check(self):
        """Waits for the current stream and raises CmpqError if a token of a call so far held a NaN or an infinity (status
        6) or a kernel gave up waiting, its output unspecified (status 5); forgets what it reported."""
        self._impl.check()


class PagedCache8:
    """Paged cache of keys and values in 8 bits.  codes: int8 [n_pages][n_kv][page_tokens][head_dim], scales: fp32
    [n_pages][n_kv].  The calls take a batch of sequences: tok_off int32 [n_seq + 1] (where a sequence's rows begin
    in the token arrays), lens int32 [n_seq] (its cached tokens after the call, the call's among them), table int32
    [n_seq][max pages] (its pages in order); all on the GPU.  What a call finds wrong with them it leaves out and
    reports through check()."""

    def __init__(self, k_codes, k_scale, v_codes, v_scale):
        self._impl = _ext().Cache(k_codes, k_scale, v_codes, v_scale)
        self.k_codes, self.k_scale, self.v_codes, self.v_scale = k_codes, k_scale, v_codes, v_scale
        self.n_pages, self.n_kv, self.page_tokens, self.head_dim = k_codes.shape
        self.word = self._impl.word

    @classmethod
    def empty(cls, n_pages, n_kv, head_dim, page_tokens=64, device="cuda"):
        codes = [torch.zeros(n_pages, n_kv, page_tokens, head_dim, dtype=torch.int8, device=device) for _ in range(2)]
        scale = [torch.zeros(n_pages, n_kv, dtype=torch.float32, device=device) for _ in range(2)]
        return cls(codes[0], scale[0], codes[1], scale[1])

    def append(self, k, v, tok_off, lens, table, q=None, cos=None, sin=None, interleaved=False, q_out=None):
        """Writes new tokens' keys (rotated by cos, sin: fp32 [positions][rot_dim / 2]) and values ([n_tok][n_kv][head_dim])
        into their pages; returns the rotated queries ([n_tok][heads][head_dim]) where q is given."""
        return self._impl.append(k, v, tok_off, lens, table, q, cos, sin, interleaved, q_out)

    def read(self, tok_off, lens, table, n_tok, dtype=torch.bfloat16):
        """The last tok_off[s+1] - tok_off[s] tokens of every sequence as 16-bit values: k, v [n_tok][n_kv][head_dim]."""
        if dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("expected float16 or bfloat16, got %s" % dtype)
        return self._impl.read(tok_off, lens, table, n_tok, dtype is torch.bfloat16)

    def attend(self, q, tok_off, lens, table, max_new, max_len=None, scale=None, causal=True, window=0, out=None,
               return_lse=False):
        """Attention of q [n_tok][heads][head_dim] over the cached tokens.  max_new, max_len: bounds of the new and of
        the cached tokens of a sequence (max_len defaults to what the table can hold)."""
        result = self._impl.attend(q, tok_off, lens, table, max_new, max_len, scale, causal, window, out, return_lse)
        return result if return_lse else result[0]

    def check(self):
        """Waits for the current stream and raises CmpqError if a call so far met a NaN or an infinity (status 6) or
        lengths and tables that do not fit (status 1), or if a kernel gave up waiting (status 5); forgets what it reported."""
        self._impl.check()


class AttentionLayer8:
    """The attention block of a served layer in 8 bits: one Int8Linear for queries, keys and values (rows of its
    weight in that order), the paged cache, and one Int8Linear for the output."""

    def __init__(self, qkv, out, cache, n_heads, cos, sin, interleaved=False):
        d = cache.head_dim
        if qkv.d_out != (n_heads + 2 * cache.n_kv) * d or out.d_in != n_heads * d:
            raise ValueError("the projections do not fit %d query heads, %d cached heads of %d entries"
                             % (n_heads, cache.n_kv, d))
        self.qkv, self.out, self.cache, self.n_heads = qkv, out, cache, n_heads
        self.cos, self.sin, self.interleaved = cos, sin, interleaved

    def __call__(self, x, tok_off, lens, table, max_new, max_len=None, window=0):
        """x: fp16/bf16 [n_tok][d_model], the new tokens of a batch (see PagedCache8).  Returns [n_tok][out.d_out]."""
        h, kv, d = self.n_heads, self.cache.n_kv, self.cache.head_dim
        y = self.qkv(x)
        q, k, v = (y[:, a * d: b * d].unflatten(1, (b - a, d)) for a, b in ((0, h), (h, h + kv), (h + kv, h + 2 * kv)))
        self.cache.append(k, v, tok_off, lens, table, q=q, cos=self.cos, sin=self.sin, interleaved=self.interleaved, q_out=q)
        a = self.cache.attend(q, tok_off, lens, table, max_new, max_len, window=window)
        return self.out(a.flatten(1))

    def check(self):
        """check() of both projections and of the cache; raises the first of their errors, and all forget theirs."""
        errors = []
        for part in (self.qkv, self.cache, self.out):
            try:
                part.check()
            except B.CmpqError as e:
                errors.append(e)
        if errors:
            raise errors[0]
