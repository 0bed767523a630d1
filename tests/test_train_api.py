"""What the Python classes of the training step hold on to and refuse, on the host: the library's calls are replaced and the
tensors are stand-ins, so nothing is launched."""

import types

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import ScarError, api  # noqa: E402

HERE, OTHER = torch.device("cuda", 0), torch.device("cuda", 1)


class Stand:
    """A CUDA tensor as far as the classes look at one."""

    def __init__(self, *shape, dtype=torch.float32, device=HERE):
        self.shape, self.dtype, self.device, self.is_cuda = shape, dtype, device, device.type == "cuda"

    def data_ptr(self):
        return 0x1000

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def dim(self):
        return len(self.shape)

    def stride(self, i):
        return self.shape[1] if i == 0 else 1

    def is_contiguous(self):
        return True



def handle(cls, **fields):
    op = object.__new__(cls)
    stream = types.SimpleNamespace(cuda_stream=7)
    fake = types.SimpleNamespace(empty=lambda shape, dtype=None, device=None: Stand(*(shape if isinstance(shape, tuple) else () if shape == () else (shape,)), dtype=dtype, device=device),
                                 int64=torch.int64, float32=torch.float32)
    op.__dict__.update(_device=HERE, _stream=stream, _torch=fake, _here=lambda index: 7, op=0, **fields)  # nothing to destroy
    return op


@pytest.fixture
def calls(monkeypatch):
    """The names of the library's calls in order; ``refuse`` lists those that answer with SCAR_ERR_LAYOUT."""
    got, refuse = [], set()
    for name in ("scar_gnorm_init", "scar_gnorm_bind", "scar_gnorm_norm", "scar_gnorm_clip", "scar_gnorm_destroy", "scar_xent_loss", "scar_xent_loss_grad", "scar_xent_destroy"):
        def call(*args, name=name, **kw):
            got.append(name)
            if name in refuse:
                raise ScarError(-2, name)
            return 5
        monkeypatch.setattr(api, name, call)
    return types.SimpleNamespace(got=got, refuse=refuse)


def test_a_refused_bind_keeps_the_registered_tensors(calls):
    """The handle goes on with the old addresses: their tensors must stay alive."""
    op = handle(api.GradientNorm)
    first, out = [Stand(8), Stand(3)], [Stand(8), Stand(3)]
    op.bind(first, out)
    calls.refuse.add("scar_gnorm_bind")
    with pytest.raises(ScarError):
        op.bind([Stand(9)], None)
    assert op._tensors == first and op._out == out
    calls.refuse.clear()
    second = [Stand(8), Stand(3)]
    op.bind(second)
    assert op._tensors == second and op._out == [None, None]
    assert calls.got == ["scar_gnorm_bind"] * 3
    with pytest.raises(ValueError):
        op.bind([Stand(8), Stand(3)], [Stand(8)])
    assert op._tensors == second and len(calls.got) == 3
    op.close()


def test_tensors_of_another_device_are_refused_before_anything_is_launched(calls):
    op = handle(api.LinearCrossEntropy, max_tokens=4, n_classes=6, dim=8, dtype=torch.float32)
    y = lambda **kw: Stand(4, dtype=torch.int64, **kw)  # noqa: E731
    h, w, row = Stand(4, 8), Stand(6, 8), Stand(4)
    op.loss(h, w, y(), row_loss=row)
    op.loss_and_grad(h, w, y(), row_loss=row, dh=Stand(4, 8), dw=Stand(6, 8))
    assert calls.got == ["scar_xent_loss", "scar_xent_loss_grad"]
    for there in (OTHER, torch.device("cpu")):
        def far(*shape):
            return Stand(*shape, device=there)
        for args, kw in (((far(4, 8), w, y()), {}), ((h, far(6, 8), y()), {}), ((h, w, y(device=there)), {}), ((h, w, y()), dict(row_loss=far(4)))):
            with pytest.raises((TypeError, ValueError)):
                op.loss(*args, **kw)
            with pytest.raises((TypeError, ValueError)):
                op.loss_and_grad(*args, **kw)
        for kw in (dict(dh=far(4, 8)), dict(dw=far(6, 8))):
            with pytest.raises((TypeError, ValueError)):
                op.loss_and_grad(h, w, y(), **kw)
    assert len(calls.got) == 2
    norm = handle(api.GradientNorm)
    norm.bind([Stand(8)])
    for ts, out in (([Stand(8, device=OTHER)], None), ([Stand(8)], [Stand(8, device=OTHER)]), ([Stand(8, device=torch.device("cpu"))], None)):
        with pytest.raises(ValueError):
            norm.bind(ts, out)
    assert len(calls.got) == 3
