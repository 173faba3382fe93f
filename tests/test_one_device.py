"""The check that a call's tensors are on one GPU, whatever place a stray one is in: of
the two passes over arguments that use it, with stand-ins for tensors of two GPUs and of
the host."""
import types

import pytest
import torch

from paper_2410_17954_amd import ops


class Stand:
    def __init__(self, device, packed=True):
        self.device, self.packed = device, packed
        self.dtype, self.shape = torch.float32, torch.Size((2, 3))

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.packed


@pytest.fixture(autouse=True)
def two_gpus(monkeypatch):
    cuda = types.SimpleNamespace(current_device=lambda: 0, device=lambda d: ("device", d),
                                 stream=lambda s: ("stream", s))
    monkeypatch.setattr(ops, "_torch", lambda: types.SimpleNamespace(cuda=cuda))


def _plain(ts, stream=None):
    return ops._one_device(stream, *ts)


def _specs(ts, stream=None, strided=0):
    return ops._checked(stream, [t for t in ts[:strided] if t is not None],
                        *(("x", t, (2, 3), torch.float32) for t in ts[strided:]))


CALLS = [_plain, _specs, lambda ts, stream=None: _specs(ts, stream, 1),
         lambda ts, stream=None: _specs(ts, stream, 3)]


@pytest.mark.parametrize("call", CALLS)
def test_a_stray_tensor_in_every_place(call):
    good = [Stand(0), None, Stand(0), Stand(0), None, Stand(0)]
    assert call(good) is ops._CURRENT
    assert call([t and Stand(1) for t in good]) == ("device", 1)
    for i in range(len(good)):
        with pytest.raises(ValueError, match="on the GPU"):
            call(good[:i] + [Stand(-1)] + good[i + 1:])
        with pytest.raises(ValueError, match="the same GPU"):
            call(good[:i] + [Stand(1)] + good[i + 1:])
    with pytest.raises(ValueError, match="on the GPU"):
        call([Stand(-1)] * 4)


@pytest.mark.parametrize("call", CALLS)
def test_streams_and_layouts(call):
    ts = [Stand(1)] * 4
    stream = types.SimpleNamespace(device=types.SimpleNamespace(index=1))
    assert call(ts, stream) == ("stream", stream)
    stream.device.index = 0
    with pytest.raises(ValueError, match="stream"):
        call(ts, stream)
    with pytest.raises(ValueError, match="contiguous"):
        call(ts[:3] + [Stand(1, packed=False)])


def test_shapes_and_types():
    for shape, dtype in (((2, 4), torch.float32), ((2, 3), torch.bfloat16)):
        with pytest.raises(ValueError, match="x must be"):
            ops._checked(None, (), ("x", Stand(0), shape, dtype))
    assert ops._checked(None, (), ("x", Stand(0), None, None)) is ops._CURRENT
