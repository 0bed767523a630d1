"""Refusals of the hidden layer's operators on the host: the library's before any CUDA work, the Python classes' before any call
of the library (stand-ins for tensors, so nothing is launched)."""

import ctypes as C
import types

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import _build, api  # noqa: E402

HERE, OTHER, HOST = torch.device("cuda", 0), torch.device("cuda", 1), torch.device("cpu")
INVALID, ALLOC, CUDA, STATE, CAPACITY = -1, -3, -4, -5, -7


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return api.load_library()


def drop(p=0.5, d_offset=None):
    return api.scar_dropout(p, 1, 2, d_offset)


def test_dropout_refuses_before_anything_is_enqueued(lib):
    def call(rule=drop(), dtype=api.SCAR_F32, x=0x1000, xp=64, r=None, rp=0, y=0x2000, yp=64, rows=8, cols=64):
        return lib.scar_dropout_apply(rule, dtype, x, xp, r, rp, y, yp, rows, cols, None)

    for p in (-0.1, 1.5, float("nan"), float("inf")):
        assert call(rule=drop(p)) == INVALID
    assert call(rule=None) == INVALID and call(rule=drop(0.5, 0x1004)) == INVALID
    for dtype in (api.SCAR_I32, 9, -1):
        assert call(dtype=dtype) == INVALID
    assert call(x=None) == call(y=None) == INVALID
    assert call(x=0x1002) == call(y=0x2001) == call(r=0x3003, rp=64) == INVALID
    assert call(dtype=api.SCAR_BF16, x=0x1001) == INVALID
    assert call(xp=63) == call(yp=63) == call(r=0x3000, rp=10) == INVALID
    assert call(xp=1 << 41, rows=2) == INVALID
    assert call(rows=1 << 31) == call(cols=1 << 31) == CAPACITY
    assert call(rows=0, x=None, y=None) == call(cols=0, x=None, y=None) == 0


@pytest.mark.parametrize("change", [dict(dtype=api.SCAR_I32), dict(dtype=7), dict(activation=-1), dict(activation=4), dict(in_features=0), dict(out_features=0),
                                    dict(in_features=1 << 31), dict(out_features=1 << 31), dict(max_rows=1 << 31)])
def test_linear_refuses_configurations(lib, change):
    cfg = api.scar_linear_config(**{**dict(max_rows=8, in_features=16, out_features=16, dtype=api.SCAR_BF16, activation=0, forward_only=0), **change})
    op = C.c_void_p(5)
    assert lib.scar_linear_init(C.byref(op), C.byref(cfg), None) == INVALID and op.value is None


@pytest.mark.parametrize("change,code", [(dict(dtype=api.SCAR_I32), INVALID), (dict(kind=2), INVALID), (dict(kind=-1), INVALID), (dict(dim=0), INVALID), (dict(eps=-1e-6), INVALID),
                                         (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(max_rows=1 << 31), INVALID), (dict(dim=16385), CAPACITY)])
def test_resnorm_refuses_configurations(lib, change, code):
    cfg = api.scar_resnorm_config(**{**dict(max_rows=8, dim=16, eps=1e-6, dtype=api.SCAR_F32, kind=0, forward_only=0), **change})
    op = C.c_void_p(5)
    assert lib.scar_resnorm_init(C.byref(op), C.byref(cfg), None) == code and op.value is None


def test_null_handles(lib):
    for name in ("scar_linear", "scar_resnorm"):
        assert getattr(lib, f"{name}_init")(None, None, None) == INVALID
        op = C.c_void_p(5)
        assert getattr(lib, f"{name}_init")(C.byref(op), None, None) == INVALID and op.value is None
        for call in ("status", "selftest_arm_timeout", "destroy"):
            assert getattr(lib, f"{name}_{call}")(None) == INVALID
        assert getattr(lib, f"{name}_launch_count")(None) == 0
    block = api.scar_resnorm_block()
    assert lib.scar_linear_forward(None, *[None, 0] * 2, None, None, 0, None, 0, None, 0, None) == INVALID
    assert lib.scar_linear_backward(None, *[None, 0] * 3, None, None, 0, *[None, 0] * 2, None) == INVALID
    assert lib.scar_resnorm_forward(None, C.byref(block), *[None, 0] * 2, 0, *[None, 0] * 2) == INVALID
    assert lib.scar_resnorm_backward(None, C.byref(block), *[None, 0] * 4, 0, *[None, 0] * 3, *[None] * 4) == INVALID
    assert lib.scar_linear_slope_bytes(None, 3) == lib.scar_linear_workspace_bytes(None) == 0


class Stand:
    """A CUDA tensor as far as the classes look at one."""

    def __init__(self, *shape, dtype=torch.float32, device=HERE, stride=None):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, device
        self._stride = stride or tuple(int(torch.Size(shape[i + 1:]).numel()) for i in range(len(shape)))
        self._whole = stride is None

    def __len__(self):
        return self.shape[0]

    def data_ptr(self):
        return 0x1000

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self._stride if i is None else self._stride[i]

    def is_contiguous(self):
        return self._whole

    def new_empty(self, shape, dtype=None):
        return Stand(*shape, dtype=dtype or self.dtype, device=self.device)

    def view(self, *shape):
        raise RuntimeError("not viewable")


def handle(cls, **fields):
    op = object.__new__(cls)
    fake = types.SimpleNamespace(empty_like=lambda t: Stand(*t.shape, dtype=t.dtype, device=t.device), int64=torch.int64, float32=torch.float32, float16=torch.float16, bfloat16=torch.bfloat16,
                                 cuda=types.SimpleNamespace(current_device=lambda: 0))
    op.__dict__.update(_device=HERE, _stream=types.SimpleNamespace(cuda_stream=7), _torch=fake, _here=lambda index: 7, op=0, **fields)
    return op


@pytest.fixture
def calls(monkeypatch):
    got = []
    for name in ("scar_dropout_apply", "scar_linear_forward", "scar_linear_backward", "scar_resnorm_forward", "scar_resnorm_backward"):
        monkeypatch.setattr(api, name, lambda *a, name=name, **kw: got.append(name))
    return got


def refused(call, *args, **kw):
    with pytest.raises((TypeError, ValueError)):
        call(*args, **kw)


def test_layers_refuse_other_shapes_types_and_devices(calls):
    layer = handle(api.LinearLayer, max_rows=4, in_features=6, out_features=10, dtype=torch.float32, activation="gelu")
    x, w, b, res, dy, slope = Stand(4, 6), Stand(10, 6), Stand(10), Stand(4, 10), Stand(4, 10), Stand(4, 16)
    layer.forward(x, w, b, res)
    assert layer.forward_train(x, w)[1].shape == (4, 16)
    layer.backward(dy, x, w, slope)
    good = ["scar_linear_forward"] * 2 + ["scar_linear_backward"]
    assert calls == good
    half = torch.bfloat16
    for bad in (Stand(4, 7), Stand(6), Stand(4, 6, dtype=half), Stand(4, 6, device=OTHER), Stand(4, 6, device=HOST), Stand(4, 6, stride=(1, 4)), Stand(4, 6, stride=(5, 1))):
        refused(layer.forward, bad, w)
        refused(layer.backward, dy, bad, w, slope)
        refused(layer.backward, dy, x, w, slope, dx=bad)
    for bad in (Stand(9, 6), Stand(10, 6, device=OTHER)):
        refused(layer.forward, x, bad)
        refused(layer.backward, dy, x, bad, slope)
        refused(layer.backward, dy, x, w, slope, dw=bad)
    for bad in (Stand(9), Stand(10, device=HOST), Stand(10, dtype=half), Stand(10, stride=(2,))):
        refused(layer.forward, x, w, bad)
        refused(layer.backward, dy, x, w, slope, dbias=bad)
    for bad in (Stand(4, 9), Stand(3, 10), Stand(4, 10, device=OTHER)):
        refused(layer.forward, x, w, b, bad)
        refused(layer.forward, x, w, b, res, out=bad)
        refused(layer.backward, bad, x, w, slope)
    for bad in (Stand(4, 10), Stand(4, 16, dtype=torch.float16), Stand(4, 16, device=OTHER), None):
        refused(layer.backward, dy, x, w, bad)
    offset = Stand(1, dtype=torch.int64, device=OTHER)
    refused(layer.forward, x, w, dropout=api.DropoutMask(drop(), offset))
    identity = handle(api.LinearLayer, max_rows=4, in_features=6, out_features=10, dtype=torch.float32, activation="identity")
    refused(identity.backward, dy, x, w, slope)
    assert calls == good


def test_dropout_refuses_other_shapes_types_and_devices(calls):
    d = handle(api.Dropout, p=0.5, seed=3)
    x = Stand(4, 6)
    d.forward(x, 1, residual=Stand(4, 6), out=Stand(4, 6))
    d.forward(Stand(4, 6, stride=(9, 1)))
    assert calls == ["scar_dropout_apply"] * 2
    for bad in (Stand(4, 5), Stand(24), Stand(4, 6, dtype=torch.float16), Stand(4, 6, device=OTHER), Stand(4, 6, stride=(1, 4)), Stand(4, 6, stride=(3, 1))):
        refused(d.forward, x, residual=bad)
        refused(d.forward, x, out=bad)
    for bad in (Stand(4, 6, device=HOST), Stand(4, 6, dtype=torch.int32), Stand(2, 3, 4, stride=(1, 2, 6))):
        refused(d.forward, bad)
    for bad in (Stand(1), Stand(2, dtype=torch.int64), Stand(1, dtype=torch.int64, device=HOST)):
        refused(d.forward, x, bad)
        refused(d.mask, bad)
    for p in (-0.1, 1.1, float("nan")):
        refused(api.Dropout, p)
    assert len(calls) == 2


def test_norms_refuse_other_shapes_types_and_devices(calls):
    n = handle(api.ResidualNorm, max_rows=4, dim=6, dtype=torch.float32, kind="layer")
    x, f, w, gate = Stand(4, 6), Stand(4, 6), Stand(6), Stand(2, 6)
    kw = dict(gate=gate, rows_per_gate=2, w_post=w, b_post=w, w_pre=w, b_pre=w)
    n.forward(x, f, **kw)
    assert set(n.backward(x, x, x, f, **kw)) == {"dx", "df", "dgate", "dw_post", "db_post", "dw_pre", "db_pre"}
    good = ["scar_resnorm_forward", "scar_resnorm_backward"]
    assert calls == good
    bad_rows = (Stand(4, 5), Stand(5, 6), Stand(4, 6, dtype=torch.float16), Stand(4, 6, device=OTHER), Stand(4, 6, stride=(4, 1)))
    for bad in bad_rows:
        refused(n.forward, x, bad)
        refused(n.forward, x, f, y=bad)
        refused(n.forward, x, f, n=bad)
        refused(n.backward, x, bad, x, f)
        refused(n.backward, x, x, bad, f)
        refused(n.backward, x, x, x, bad)
        refused(n.backward, x, x, x, f, out={"df": bad})
    for bad in (Stand(5), Stand(6, device=HOST), Stand(6, stride=(2,))):
        for k in ("w_post", "b_post", "w_pre", "b_pre"):
            refused(n.forward, x, f, **{k: bad})
    refused(n.forward, x, f, gate=gate)           # a row for each is wanted
    refused(n.forward, x, f, gate=Stand(3, 6), rows_per_gate=2)
    refused(n.forward, x, f, gate=gate, rows_per_gate=0)
    assert calls == good
