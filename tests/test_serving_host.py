"""Host-side checks of the 8-bit serving calls that need no GPU: bad arguments are refused before any launch."""
import ctypes

import pytest

from paper_2410_13056_b200 import binding as B
from paper_2410_13056_b200 import build as cuda_build

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def L():
    cuda_build.build()
    return B.lib()


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_char * 8192)()
    keep = ctypes.cast(buf, ctypes.c_void_p)
    yield ctypes.c_void_p((keep.value + 255) // 256 * 256)
    del buf


def _off(p, by):
    return ctypes.c_void_p(p.value + by)


def test_quantize_tokens(L, p):
    q = lambda X=p, dt=0, n=2, d=20, ldx=20, codes=p, ldc=32, scale=p: L.cmpq_quantize_tokens(X, dt, n, d, ldx, codes, ldc, scale, None, None)
    for bad in (dict(X=None), dict(codes=None), dict(scale=None), dict(dt=2), dict(n=-1), dict(d=0), dict(d=262145, ldx=262145, ldc=262160),
                dict(ldx=19), dict(ldc=16), dict(ldc=30), dict(codes=_off(p, 8)), dict(X=_off(p, 1)), dict(n=1 << 31)):
        assert q(**bad) == INVALID, bad
    assert q(n=0, X=None) == 0


def test_products(L, p):
    m = lambda xc=p, ldxc=32, xs=p, wc=p, ldwc=32, ws=p, bias=None, dt=0, n=2, d_in=20, d_out=5, y=p, ldy=5, w=p, wb=1 << 30: \
        L.cmpq_matmul_i8(xc, ldxc, xs, wc, ldwc, ws, bias, dt, n, d_in, d_out, y, ldy, w, wb, None)
    for bad in (dict(xc=None), dict(xs=None), dict(wc=None), dict(ws=None), dict(y=None), dict(dt=3), dict(n=-1), dict(d_in=0),
                dict(d_out=0), dict(d_out=262145, ldy=262145), dict(d_in=131073, ldxc=131088, ldwc=131088), dict(ldxc=16),
                dict(ldxc=33), dict(ldwc=24), dict(ldy=4), dict(xc=_off(p, 4)), dict(wc=_off(p, 8)), dict(y=_off(p, 1)), dict(bias=_off(p, 1))):
        assert m(**bad) == INVALID, bad
    assert m(w=None) == WORKSPACE and m(wb=16) == WORKSPACE and m(w=_off(p, 16)) == WORKSPACE
    assert m(n=0, xc=None, w=None) == 0
    l = lambda X=p, dt=0, n=2, d_in=20, ldx=20, wc=p, ldwc=32, ws=p, bias=None, d_out=5, y=p, ldy=5, w=p, wb=1 << 30: \
        L.cmpq_linear_i8(X, dt, n, d_in, ldx, wc, ldwc, ws, bias, d_out, y, ldy, None, w, wb, None)
    for bad in (dict(X=None), dict(wc=None), dict(ws=None), dict(y=None), dict(dt=-1), dict(ldx=19), dict(ldwc=17), dict(ldy=1),
                dict(X=_off(p, 1))):
        assert l(**bad) == INVALID, bad
    assert l(w=None) == WORKSPACE and l(wb=16) == WORKSPACE
    assert B.cmpq_linear_i8_ws_bytes(3, 0, 4) == 0 and B.cmpq_linear_i8_ws_bytes(-1, 4, 4) == 0
    assert B.cmpq_linear_i8_ws_bytes(7, 33, 9) >= 7 * 48 + 7 * 4


def _cache(p, **more):
    v = dict(k_codes=p.value, k_scale=p.value, v_codes=p.value, v_scale=p.value, n_pages=4, n_kv_heads=2, head_dim=64, page_tokens=16)
    v.update(more)
    return B.Cache(**v)


def _batch(p, **more):
    v = dict(tok_off=p.value, lens=p.value, table=p.value, ld_table=2, n_seq=2, n_tok=3)
    v.update(more)
    return B.Batch(**v)


BAD_CACHES = [(dict(k_codes=None), INVALID), (dict(v_scale=None), INVALID), (dict(n_pages=0), INVALID), (dict(n_kv_heads=0), INVALID),
              (dict(head_dim=96), UNSUPPORTED), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED)]
BAD_BATCHES = [dict(tok_off=None), dict(lens=None), dict(table=None), dict(ld_table=0), dict(n_seq=-1), dict(n_seq=65537), dict(n_tok=-1),
               dict(n_tok=1 << 31)]


def test_append_and_read(L, p):
    def a(cache=None, batch=None, k=p, ldk=128, v=p, ldv=128, dt=0, cos=p, sin=p, n_pos=9, rot=64, inter=0, q=p, ldq=256, heads=4, qo=p, ldqo=256):
        return L.cmpq_cache_append(cache or _cache(p), batch or _batch(p), k, ldk, v, ldv, dt, cos, sin, n_pos, rot, inter, q, ldq, heads, qo, ldqo, None, None)

    def r(cache=None, batch=None, dt=0, k=p, v=p, ldo=128):
        return L.cmpq_cache_read(cache or _cache(p), batch or _batch(p), dt, k, v, ldo, None, None)

    for more, why in BAD_CACHES:
        assert a(cache=_cache(p, **more)) == why and r(cache=_cache(p, **more)) == why, more
    for more in BAD_BATCHES:
        assert a(batch=_batch(p, **more)) == INVALID and r(batch=_batch(p, **more)) == INVALID, more
    for bad in (dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=1), dict(dt=2), dict(rot=63), dict(rot=66), dict(rot=-2), dict(cos=None),
                dict(sin=None), dict(n_pos=-1), dict(ldq=255), dict(ldqo=9), dict(qo=None), dict(heads=0), dict(k=_off(p, 1)), dict(q=_off(p, 1))):
        assert a(**bad) == INVALID, bad
    for bad in (dict(k=None), dict(v=None), dict(ldo=100), dict(dt=5), dict(v=_off(p, 1))):
        assert r(**bad) == INVALID, bad
    assert a(batch=_batch(p, n_seq=0)) == 0 and r(batch=_batch(p, n_tok=0)) == 0
    assert L.cmpq_cache_append(None, _batch(p), p, 128, p, 128, 0, p, p, 9, 64, 0, None, 0, 0, None, 0, None, None) == INVALID
    assert L.cmpq_check_cache(None, None) == INVALID


def test_attention(L, p):
    def a(cache=None, batch=None, q=p, ldq=256, dt=0, heads=4, max_new=2, max_len=32, scale=0.1, causal=1, window=0, out=p, ldo=256, lse=None, ws=p, wb=1 << 40):
        return L.cmpq_cache_attention(cache or _cache(p), batch or _batch(p), q, ldq, dt, heads, max_new, max_len, scale, causal, window, out, ldo, lse, None, ws, wb, None)

    for more, why in BAD_CACHES:
        assert a(cache=_cache(p, **more)) == why, more
    for more in BAD_BATCHES:
        assert a(batch=_batch(p, **more)) == INVALID, more
    for bad in (dict(q=None), dict(out=None), dict(ldq=255), dict(ldo=2), dict(dt=4), dict(heads=3), dict(heads=0), dict(max_new=-1),
                dict(max_len=-1), dict(max_len=1 << 31), dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=-1.0),
                dict(window=-1), dict(window=4, causal=0), dict(q=_off(p, 1)), dict(out=_off(p, 1)), dict(lse=_off(p, 2))):
        assert a(**bad) == INVALID, bad
    assert a(ws=None) == WORKSPACE and a(wb=0) == WORKSPACE and a(ws=_off(p, 64)) == WORKSPACE
    assert a(batch=_batch(p, n_tok=0)) == 0
    size = B.cmpq_cache_attention_ws_bytes
    assert size(2, 3, 1, 100, 4, 3, 64) == 0 and size(-1, 3, 1, 100, 4, 2, 64) == 0 and size(2, 3, 1, 100, 4, 2, 0) == 0
    assert size(2, 3, 1, 100, 4, 2, 64) >= 256


def test_extension_is_built_and_refuses_what_is_not_on_the_gpu(L, monkeypatch):
    import torch

    from paper_2410_13056_b200 import serving

    assert serving._ext().__file__ == cuda_build.EXT_PATH
    codes, scale = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    with pytest.raises(ValueError, match="CUDA"):
        serving.Int8Linear(codes, scale)
    pages, scales = torch.zeros(2, 1, 16, 64, dtype=torch.int8), torch.zeros(2, 1)
    with pytest.raises(ValueError, match="CUDA"):
        serving.PagedCache8(pages, scales, pages, scales)
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(B, "_LIB_PATH", "/nonexistent/libcmpq.so")
    with pytest.raises(RuntimeError, match="missing"):
        serving.Int8Linear(codes, scale)


def test_codes_need_room_for_their_padding():
    """Rows of codes are filled up to 16 bytes when they are written: a row without that room is refused, a single one too."""
    import torch

    zeros = lambda *shape: torch.zeros(*shape, dtype=torch.int8)
    for good, ld in ((zeros(1, 16)[:, :5], 16), (zeros(1, 32), 32), (zeros(4, 48)[:, :33], 48), (zeros(6, 16)[5:, :1], 16), (zeros(3, 16), 16),
                     (zeros(64)[16:].view(3, 16)[:, :9], 16), (zeros(0, 5), 5)):
        assert B._code_room(good) == ld, good.shape
    for bad in (zeros(1, 5), zeros(8, 5)[3:4], zeros(2, 20), zeros(64)[59:].view(1, 5), zeros(37).as_strided((2, 5), (32, 1))):
        with pytest.raises(ValueError, match="room"):
            B._code_room(bad)


def test_token_counts_that_tiles_would_carry_past_32_bits(L, p):
    for n in ((1 << 31) - 1, (1 << 31) - 256):
        assert B.cmpq_linear_i8_ws_bytes(n, 16, 1) == 0
        assert L.cmpq_linear_i8(p, 0, n, 16, 16, p, 16, p, None, 1, p, 1, None, p, 1 << 60, None) == INVALID
        assert L.cmpq_matmul_i8(p, 16, p, p, 16, p, None, 0, n, 16, 1, p, 1, p, 1 << 60, None) == INVALID
    assert B.cmpq_linear_i8_ws_bytes((1 << 31) - 257, 16, 1) > 0
