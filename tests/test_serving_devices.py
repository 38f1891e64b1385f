"""Tensors of one serving call lie on one device: refused before anything is launched.  Tensors without storage that say
that they are on some GPU stand in for two of them."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2410_13056_b200 import build as cuda_build

HERE, THERE = "cuda:0", "cuda:1"


@pytest.fixture(scope="module")
def ext():
    cuda_build.build()
    from paper_2410_13056_b200 import serving

    if torch.cuda.is_available():
        pytest.skip("stand-ins for GPUs want a machine without one")
    return serving._ext()


@pytest.mark.filterwarnings("ignore::UserWarning")
def test_other_devices_are_refused(ext):
    new = lambda device, dtype, *shape: torch.empty(shape, dtype=dtype, device=device)
    i8, i32, f32, f16 = torch.int8, torch.int32, torch.float32, torch.float16
    with FakeTensorMode():
        codes, scale, bias = lambda d: new(d, i8, 4, 16), lambda d: new(d, f32, 4), lambda d: new(d, f16, 4)
        for s, b, name in ((THERE, HERE, "w_scale"), (HERE, THERE, "bias")):
            with pytest.raises(ValueError, match=name + " is on cuda:1, the rest on cuda:0"):
                ext.Linear(codes(HERE), scale(s), bias(b))
        linear = ext.Linear(codes(HERE), scale(HERE), bias(HERE))
        with pytest.raises(ValueError, match="x is on cuda:1"):
            linear(new(THERE, f16, 3, 16))
        with pytest.raises(ValueError, match="out is on cuda:1"):
            linear(new(HERE, f16, 3, 16), new(THERE, f16, 3, 4))

        pages, scales = lambda d: new(d, i8, 3, 2, 16, 64), lambda d: new(d, f32, 3, 2)
        for at, name in ((1, "k_scale"), (2, "v_codes"), (3, "v_scale")):
            d = [THERE if i == at else HERE for i in range(4)]
            with pytest.raises(ValueError, match=name + " is on cuda:1"):
                ext.Cache(pages(d[0]), scales(d[1]), pages(d[2]), scales(d[3]))
        cache = ext.Cache(pages(HERE), scales(HERE), pages(HERE), scales(HERE))
        shapes = dict(k=(f16, 5, 2, 64), v=(f16, 5, 2, 64), tok_off=(i32, 2), lens=(i32, 1), table=(i32, 1, 2), q=(f16, 5, 4, 64), cos=(f32, 9, 32),
                      sin=(f32, 9, 32), q_out=(f16, 5, 4, 64))
        for wrong in shapes:
            with pytest.raises(ValueError, match=wrong + " is on cuda:1"):
                cache.append(**{x: new(THERE if x == wrong else HERE, *shape) for x, shape in shapes.items()})
        for wrong in ("q", "tok_off", "lens", "table", "out"):
            t = {x: new(THERE if x == wrong else HERE, *shapes.get(x, shapes["q"])) for x in ("q", "tok_off", "lens", "table", "out")}
            with pytest.raises(ValueError, match=wrong + " is on cuda:1"):
                cache.attend(t["q"], t["tok_off"], t["lens"], t["table"], 5, 32, None, True, 0, t["out"], False)
        for wrong in ("tok_off", "lens", "table"):
            t = [new(THERE if x == wrong else HERE, *shapes[x]) for x in ("tok_off", "lens", "table")]
            with pytest.raises(ValueError, match=wrong + " is on cuda:1"):
                cache.read(*t, 5, True)
