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
    op.__dict__.update(_device=HERE, _stream=stream, _torch=fake, _here=lambda index: 7, op=5, **fields)
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
