"""Serving with 8-bit activations and an 8-bit cache: what holds the buffers of those C-ABI calls.

`Int8Linear` is a linear layer with 8-bit weight codes, `PagedCache8` a paged cache of keys and values with a scale
per page and head (append, read back, attend), `AttentionLayer8` the attention block that runs them together: the
projections, the append with the rotation on the way, the attention over the cache and the output projection.
Everything is enqueued on the current torch stream; nothing is computed here.
"""
import math

import torch

from . import binding as B


def _need(t, dtype, name, dims):
    if not t.is_cuda or t.dtype != dtype or t.dim() != dims:
        raise ValueError("%s needs a %d-dimensional CUDA tensor of %s, got %s %s on %s"
                         % (name, dims, dtype, tuple(t.shape), t.dtype, t.device))


class Int8Linear:
    """y = x W^T + b with 8-bit codes on both sides.  w_codes: int8 [d_out][d_in], rows on multiples of 16 bytes;
    w_scale: fp32 [d_out]; bias: fp16/bf16 [d_out] or None (its dtype is then the activations')."""

    def __init__(self, w_codes, w_scale, bias=None):
        _need(w_codes, torch.int8, "w_codes", 2)
        _need(w_scale, torch.float32, "w_scale", 1)
        if w_codes.stride(1) != 1 or w_codes.stride(0) % 16 or w_codes.data_ptr() % 16:
            raise ValueError("w_codes needs rows that start on multiples of 16 bytes")
        if w_scale.shape[0] != w_codes.shape[0] or (bias is not None and tuple(bias.shape) != (w_codes.shape[0],)):
            raise ValueError("w_scale and bias need one entry per row of w_codes")
        self.w_codes, self.w_scale, self.bias = w_codes, w_scale.contiguous(), None if bias is None else bias.contiguous()
        self.d_out, self.d_in = w_codes.shape
        self.nonfinite = torch.zeros(1, dtype=torch.int32, device=w_codes.device)
        self._ws = {}

    @classmethod
    def from_weight(cls, weight, bias=None):
        """weight: fp16/bf16 [d_out][d_in]; every output channel gets its largest magnitude over 127 as scale."""
        d_out, d_in = weight.shape
        codes = torch.empty(d_out, (d_in + 15) // 16 * 16, dtype=torch.int8, device=weight.device)[:, :d_in]
        scale = torch.empty(d_out, dtype=torch.float32, device=weight.device)
        B.cmpq_quantize_tokens(weight, codes, scale)
        return cls(codes, scale, bias)

    def _workspace(self, n):
        # one per stream: calls on different streams may overlap
        ws = self._ws[B._on(self.w_codes)] = (n, torch.empty(B.cmpq_linear_i8_ws_bytes(n, self.d_in, self.d_out),
                                                             dtype=torch.uint8, device=self.w_codes.device))
        return ws

    def __call__(self, x, out=None):
        """x: fp16/bf16 [n][d_in].  Returns out [n][d_out] of x's dtype."""
        if x.dim() != 2 or x.shape[1] != self.d_in or not x.is_cuda:
            raise ValueError("x needs shape [n][%d] on the GPU, got %s on %s" % (self.d_in, tuple(x.shape), x.device))
        if self.bias is not None and self.bias.dtype != x.dtype:
            raise TypeError("bias is %s, x is %s" % (self.bias.dtype, x.dtype))
        n = x.shape[0]
        if out is None:
            out = x.new_empty((n, self.d_out))
        elif out.dtype != x.dtype or tuple(out.shape) != (n, self.d_out):
            raise ValueError("out needs shape [n][%d] and x's dtype" % self.d_out)
        if n:
            ws = self._ws.get(B._on(x))
            if ws is None or ws[0] < n:
                ws = self._workspace(n)
            B.cmpq_linear_i8(x, self.w_codes, self.w_scale, self.bias, out, ws[1], self.nonfinite)
        return out


class PagedCache8:
    """Paged cache of keys and values in 8 bits.  codes: int8 [n_pages][n_kv][page_tokens][head_dim], scales: fp32
    [n_pages][n_kv].  The calls take a batch of sequences: tok_off int32 [n_seq + 1] (where a sequence's rows begin
    in the token arrays), lens int32 [n_seq] (its cached tokens after the call, the call's among them), table int32
    [n_seq][max pages] (its pages in order); all on the GPU.  What a call finds wrong with them it leaves out and
    reports through check()."""

    def __init__(self, k_codes, k_scale, v_codes, v_scale):
        for name, t in (("k_codes", k_codes), ("v_codes", v_codes)):
            _need(t, torch.int8, name, 4)
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            _need(t, torch.float32, name, 2)
        if k_codes.shape != v_codes.shape or k_scale.shape != k_codes.shape[:2] or v_scale.shape != k_scale.shape:
            raise ValueError("codes need shape [n_pages][n_kv][page_tokens][head_dim] and scales [n_pages][n_kv]")
        if not all(t.is_contiguous() for t in (k_codes, k_scale, v_codes, v_scale)):
            raise ValueError("the cache's tensors need to be contiguous")
        self.k_codes, self.k_scale, self.v_codes, self.v_scale = k_codes, k_scale, v_codes, v_scale
        self.n_pages, self.n_kv, self.page_tokens, self.head_dim = k_codes.shape
        self.device = k_codes.device
        self.word = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._c = B.Cache(k_codes.data_ptr(), k_scale.data_ptr(), v_codes.data_ptr(), v_scale.data_ptr(), self.n_pages,
                          self.n_kv, self.head_dim, self.page_tokens)
        self._ws, self._need = {}, {}

    @classmethod
    def empty(cls, n_pages, n_kv, head_dim, page_tokens=64, device="cuda"):
        codes = [torch.zeros(n_pages, n_kv, page_tokens, head_dim, dtype=torch.int8, device=device) for _ in range(2)]
        scale = [torch.zeros(n_pages, n_kv, dtype=torch.float32, device=device) for _ in range(2)]
        return cls(codes[0], scale[0], codes[1], scale[1])

    def _batch(self, tok_off, lens, table, n_tok):
        n_seq, width = table.shape
        stride = table.stride()
        if (tok_off.dtype is not torch.int32 or lens.dtype is not torch.int32 or table.dtype is not torch.int32
                or tok_off.shape != (n_seq + 1,) or lens.shape != (n_seq,)):
            raise ValueError("tok_off [n_seq + 1], lens [n_seq] and table [n_seq][pages] need to be int32 tensors, got %s, "
                             "%s, %s" % tuple((t.dtype, tuple(t.shape)) for t in (tok_off, lens, table)))
        if not (tok_off.is_cuda and lens.is_cuda and table.is_cuda and tok_off.is_contiguous() and lens.is_contiguous()
                and (stride[1] == 1 or width <= 1)):
            raise ValueError("tok_off, lens and table need contiguous rows on the GPU")
        return B.Batch(tok_off.data_ptr(), lens.data_ptr(), table.data_ptr(), stride[0] if n_seq > 1 else width, n_seq, n_tok)

    def _heads(self, t, name, heads=None):
        shape = t.shape
        if len(shape) != 3 or shape[2] != self.head_dim or (heads and shape[1] != heads) or not t.is_cuda:
            raise ValueError("%s needs shape [n_tok][%s][%d] on the GPU, got %s"
                             % (name, heads or "heads", self.head_dim, tuple(shape)))

    def append(self, k, v, tok_off, lens, table, q=None, cos=None, sin=None, interleaved=False, q_out=None):
        """Writes new tokens' keys (rotated by cos, sin: fp32 [positions][rot_dim / 2]) and values into their pages;
        returns the rotated queries where q is given."""
        self._heads(k, "k", self.n_kv)
        self._heads(v, "v", self.n_kv)
        if v.dtype != k.dtype or v.shape[0] != k.shape[0]:
            raise ValueError("k and v need one dtype and token count")
        if (cos is None) != (sin is None) or (cos is not None and (cos.shape != sin.shape or not cos.is_contiguous()
                                                                   or not sin.is_contiguous()
                                                                   or cos.dtype != torch.float32 or sin.dtype != torch.float32)):
            raise ValueError("cos and sin need to be contiguous fp32 tensors of one shape")
        if q is not None:
            self._heads(q, "q")
            if q.dtype != k.dtype or q.shape[0] != k.shape[0]:
                raise ValueError("q needs k's dtype and token count")
            if q_out is None:
                q_out = q.new_empty(q.shape)
            elif q_out.shape != q.shape or q_out.dtype != q.dtype:
                raise ValueError("q_out needs q's shape and dtype")
        B.cmpq_cache_append(self._c, self._batch(tok_off, lens, table, k.shape[0]), k, v, cos, sin, interleaved, q, q_out,
                            self.word)
        return q_out

    def read(self, tok_off, lens, table, n_tok, dtype=torch.bfloat16):
        """The last tok_off[s+1] - tok_off[s] tokens of every sequence as 16-bit values: k, v [n_tok][n_kv][head_dim]."""
        k, v = torch.empty((2, n_tok, self.n_kv, self.head_dim), dtype=dtype, device=self.device).unbind(0)
        B.cmpq_cache_read(self._c, self._batch(tok_off, lens, table, n_tok), k, v, self.word)
        return k, v

    def attend(self, q, tok_off, lens, table, max_new, max_len=None, scale=None, causal=True, window=0, out=None,
               return_lse=False):
        """Attention of q [n_tok][heads][head_dim] over the cached tokens.  max_new, max_len: bounds of the new and of
        the cached tokens of a sequence (max_len defaults to what the table can hold)."""
        self._heads(q, "q")
        n, heads, d = q.shape
        if heads % self.n_kv:
            raise ValueError("%d query heads are no multiple of the cache's %d heads" % (heads, self.n_kv))
        if max_len is None:
            max_len = table.shape[1] * self.page_tokens
        if out is None:
            out = q.new_empty(q.shape)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out needs q's shape and dtype")
        lse = self.k_scale.new_empty((n, heads)) if return_lse else None
        batch = self._batch(tok_off, lens, table, n)
        size, stream = (lens.shape[0], n, max_new, max_len, heads), B._on(q)
        need = self._need.get(size)
        if need is None:
            if len(self._need) > 1000:
                self._need.clear()
            need = self._need[size] = B.cmpq_cache_attention_ws_bytes(*size, self.n_kv, d)
        ws = self._ws.get(stream)  # one work space per stream: calls on different streams may overlap
        if ws is None or ws.numel() < need:
            ws = self._ws[stream] = torch.zeros(need, dtype=torch.uint8, device=q.device)  # its counters start at 0
        B.cmpq_cache_attention(self._c, batch, q, max_new, max_len, 1.0 / math.sqrt(d) if scale is None else scale,
                               causal, window, out, lse, ws, self.word)
        return (out, lse) if return_lse else out

    def check(self):
        """Waits for the current stream and raises CmpqError if a call so far met a NaN or an infinity (status 6) or
        lengths and tables that do not fit (status 1); forgets what it reported."""
        try:
            B.cmpq_check_cache(self.word)
        finally:
            self.word.zero_()


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
