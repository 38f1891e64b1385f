"""Host-side checks of the linear layer with its epilogue and of the gated block that need no GPU."""
import ctypes

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

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


def _w(p, **more):
    v = dict(codes=p.value, ld=32, scale=p.value, bias=None)
    v.update(more)
    return B.Weight8(**v)


BAD_WEIGHTS = [dict(codes=None), dict(scale=None), dict(ld=16), dict(ld=33), "codes", "scale", "bias"]


def _bad(p, what):
    return _w(p, **what) if isinstance(what, dict) else _w(p, **{what: p.value + 1})


def test_norm_quantize(L, p):
    q = lambda X=p, dt=0, n=2, d=20, ldx=20, norm=p, eps=1e-6, codes=p, ldc=32, scale=p: \
        L.cmpq_norm_quantize_tokens(X, dt, n, d, ldx, norm, eps, codes, ldc, scale, None, None)
    for bad in (dict(X=None), dict(codes=None), dict(scale=None), dict(dt=2), dict(n=-1), dict(d=0), dict(ldx=19), dict(ldc=16), dict(norm=_off(p, 1)),
                dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-40), dict(codes=_off(p, 8))):
        assert q(**bad) == INVALID, bad
    assert q(n=0, X=None) == 0 and q(n=0, norm=None, eps=0.0) == 0


def test_linear(L, p):
    def l(X=p, dt=0, n=2, d_in=20, ldx=20, norm=p, eps=1e-6, weight="", d_out=5, act=2, res=p, ldr=5, y=p, ldy=5, ws=p, wb=1 << 30):
        return L.cmpq_linear_i8_fused(X, dt, n, d_in, ldx, norm, eps, _w(p) if weight == "" else weight, d_out, act, res, ldr, y, ldy, None, ws, wb, None)

    for bad in (dict(X=None), dict(y=None), dict(dt=-1), dict(n=-1), dict(d_in=0), dict(d_out=0), dict(d_in=131073, ldx=131073), dict(ldx=19), dict(ldy=4),
                dict(act=-1), dict(act=5), dict(ldr=4), dict(res=_off(p, 1)), dict(norm=_off(p, 1)), dict(eps=0.0), dict(weight=None), dict(X=_off(p, 1)),
                dict(y=_off(p, 1)), dict(n=(1 << 31) - 1)):
        assert l(**bad) == INVALID, bad
    for what in BAD_WEIGHTS:
        assert l(weight=_bad(p, what)) == INVALID, what
    assert l(ws=None) == WORKSPACE and l(wb=16) == WORKSPACE and l(ws=_off(p, 16)) == WORKSPACE
    assert l(n=0, X=None, ws=None) == 0 and l(ws=None, norm=None, eps=0.0, res=None, ldr=0) == WORKSPACE


def test_gated(L, p):
    def g(X=p, dt=0, n=2, d_in=20, ldx=20, norm=p, eps=1e-6, gate="", up="", down="", d_ff=30, d_out=5, act=2, res=p, ldr=5, y=p, ldy=5, state=p, ws=p, wb=1 << 40):
        w = [_w(p) if x == "" else x for x in (gate, up, down)]
        return L.cmpq_gated_i8(X, dt, n, d_in, ldx, norm, eps, *w, d_ff, d_out, act, res, ldr, y, ldy, None, state, ws, wb, None)

    for bad in (dict(state=None), dict(state=_off(p, 8)), dict(X=None), dict(y=None), dict(dt=2), dict(n=-1), dict(d_in=0), dict(d_ff=0), dict(d_out=0), dict(d_in=131073, ldx=131073), dict(d_ff=131073),
                dict(d_out=262145, ldy=262145, ldr=262145), dict(ldx=19), dict(ldy=4), dict(act=7), dict(ldr=4), dict(res=_off(p, 1)), dict(norm=_off(p, 1)),
                dict(eps=float("nan")), dict(gate=None), dict(up=None), dict(down=None), dict(X=_off(p, 1)), dict(y=_off(p, 1)), dict(n=(1 << 31) - 256)):
        assert g(**bad) == INVALID, bad
    for what in BAD_WEIGHTS:
        for part in ("gate", "up", "down"):
            assert g(**{part: _bad(p, what)}) == INVALID, (part, what)
    assert g(ws=None) == WORKSPACE and g(wb=256) == WORKSPACE and g(ws=_off(p, 64)) == WORKSPACE
    assert g(n=0, X=None, ws=None) == 0
    size = B.cmpq_gated_i8_ws_bytes
    assert size(-1, 4, 4, 4) == size(1, 0, 4, 4) == size(1, 4, 0, 4) == size(1, 4, 4, 0) == size(1, 4, 131073, 4) == 0
    assert size(7, 33, 100, 9) >= 7 * (2 * 100 + 112 + 8)
    # rows of h and codes whose bytes pass 32 bits are counted in 64
    assert size(1 << 20, 4096, 131072, 4096) >= (1 << 20) * 131072 * 3


HERE, THERE = "cuda:0", "cuda:1"


@pytest.mark.filterwarnings("ignore::UserWarning")
def test_other_devices_are_refused(L):
    from paper_2410_13056_b200 import serving

    if torch.cuda.is_available():
        pytest.skip("stand-ins for GPUs want a machine without one")
    ext = serving._ext()
    new = lambda device, dtype, *shape: torch.empty(shape, dtype=dtype, device=device)
    f16 = torch.float16
    with FakeTensorMode():
        layer = lambda d, o, i: ext.Linear(new(d, torch.int8, o, i), new(d, torch.float32, o), None)
        shapes = dict(x=(f16, 3, 16), out=(f16, 3, 32), residual=(f16, 3, 32), norm=(f16, 16))
        linear = layer(HERE, 32, 16)
        for wrong in shapes:
            with pytest.raises(ValueError, match=wrong + " is on cuda:1"):
                linear(**{k: new(THERE if k == wrong else HERE, *s) for k, s in shapes.items()})
        for at, name in ((1, "up"), (2, "down")):
            d = [THERE if i == at else HERE for i in range(3)]
            with pytest.raises(ValueError, match=name + " is on cuda:1"):
                ext.Gated(layer(d[0], 48, 16), layer(d[1], 48, 16), layer(d[2], 32, 48), "silu")
        block = ext.Gated(layer(HERE, 48, 16), layer(HERE, 48, 16), layer(HERE, 32, 48), "silu")
        for wrong in shapes:
            with pytest.raises(ValueError, match=wrong + " is on cuda:1"):
                block(**{k: new(THERE if k == wrong else HERE, *s) for k, s in shapes.items()})
        with pytest.raises(ValueError, match="norm needs 16"):
            block(**{k: new(HERE, *(s if k != "norm" else (f16, 17))) for k, s in shapes.items()})


def test_binding_refuses_what_does_not_fit(L):
    x = torch.zeros(3, 16, dtype=torch.float16)
    for norm in (torch.zeros(15, dtype=torch.float16), torch.zeros(16), torch.zeros(16, 1, dtype=torch.float16), torch.zeros(32, dtype=torch.float16)[::2]):
        with pytest.raises(ValueError, match="norm"):
            B.cmpq_norm_quantize_tokens(x, norm, 1e-6, torch.zeros(3, 16, dtype=torch.int8), torch.zeros(3))
    for res in (torch.zeros(3, 7, dtype=torch.float16), torch.zeros(2, 8, dtype=torch.float16), torch.zeros(3, 8), torch.zeros(8, 3, dtype=torch.float16).t()):
        with pytest.raises(ValueError):
            B._residual(res, 3, 8, x)
    assert B._residual(None, 3, 8, x) == (None, 0)
