"""What `DeviceModel.layer_forward_cached` refuses before the library sees it: operands that are not where the model is.
(Stand-ins for tensors, so that it runs without a GPU; nothing is launched.)"""
import contextlib
import types

import pytest
import torch

from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D


class Tensor:
    """As much of a tensor on GPU `dev` (-1: the host) as the call asks for."""

    dtype = torch.float32

    def __init__(self, dev, shape=(4, 8), contiguous=True):
        self.dev, self.shape, self.contiguous = dev, shape, contiguous
        self.device, self.is_cuda, self.nbytes = f"cuda:{dev}", dev >= 0, 4096

    def get_device(self):
        return self.dev

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 4096

    def numel(self):
        return self.nbytes // 4


@pytest.fixture
def call(monkeypatch):
    """The call on GPU 0 but for what is given; returns the arguments that the library got, and the device."""
    got, current = [], [0]

    @contextlib.contextmanager
    def on(device):
        was, current[0] = current[0], int(str(device).split(":")[1])
        yield
        current[0] = was

    monkeypatch.setattr(D, "_current_device", lambda: current[0])
    monkeypatch.setattr(D, "stream_handle", lambda: 100 + current[0])
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(L, "mebp_layer_forward_cached", lambda *a: got.append(a))

    def go(gpu=0, **kw):
        t = dict(dict.fromkeys(("x_in", "x_out", "pages", "past", "table", "ws", "model"), gpu), **kw)
        t = {k: v if isinstance(v, Tensor) else Tensor(v) for k, v in t.items()}
        model = types.SimpleNamespace(ws=t["model"], cfg=types.SimpleNamespace(hidden=8), ccfg=None, base=[None], lora=[None])
        model.layer_forward_cached = types.MethodType(D.DeviceModel.layer_forward_cached, model)
        model.layer_forward_cached(0, t["x_in"], t["x_out"], types.SimpleNamespace(pages=t["pages"], struct=None),
                                   types.SimpleNamespace(past=t["past"], struct=None), types.SimpleNamespace(table=t["table"], struct=None), t["ws"])
        return got.pop()

    return go


@pytest.mark.parametrize("what", ["x_in", "x_out", "pages", "past", "table", "ws"])
@pytest.mark.parametrize("dev", [-1, 1])
def test_operands_that_are_not_on_the_models_device(call, what, dev):
    with pytest.raises(ValueError):
        call(**{what: dev})


def test_workspaces(call):
    with pytest.raises(ValueError):
        call(ws=Tensor(0, contiguous=False))
    assert call()[-2] == 4096  # its bytes, whatever its type


def test_a_model_on_another_device_than_the_current_one(call):
    assert call()[-1] == 100
    assert call(gpu=1)[-1] == 101  # that device's stream
