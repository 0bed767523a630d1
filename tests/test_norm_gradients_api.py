"""What ResidualNorm.backward refuses before the library is called: gradients that the call does not have."""

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import api  # noqa: E402
from test_hidden_api import Stand, calls, handle  # noqa: E402, F401


def test_a_call_without_gradients_or_with_some_it_does_not_have(calls):  # noqa: F811
    norm = handle(api.ResidualNorm, max_rows=4, dim=6, dtype=torch.float32, kind="layer")
    x, f, w, gate = Stand(4, 6), Stand(4, 6), Stand(6), Stand(2, 6)
    for args, kw in (((None, None, x), {}), ((None, None, x, f), dict(pre=False)), ((x, x, x, f), dict(pre=False)),
                     ((x, x, x, f), dict(out={"dw_post": w})), ((x, x, x, f), dict(out={"dgate": gate})), ((x, x, x), dict(out={"df": x}, w_pre=w)),
                     ((x, x, x, f), dict(out={"dy": x})), ((x, None, None, f), dict(pre=False, w_pre=w, out={"dw_pre": w}))):
        with pytest.raises(ValueError):
            norm.backward(*args, **kw)
    assert not calls
    got = norm.backward(x, x, x, f, w_post=w, w_pre=w, gate=gate, rows_per_gate=2, out={"dw_post": w, "dgate": gate, "dx": x, "df": None})
    assert got["dw_post"] is w and got["dgate"] is gate and got["dx"] is x and got["df"] is None and got["dw_pre"] is not None
    assert norm.backward(x, None, None, f, pre=False)["df"] is not None
    # one call's gradients are the next one's tensors, None where there was none
    first = norm.backward(x, x, x, f, w_pre=w)
    assert first["dgate"] is None and norm.backward(x, x, x, f, w_pre=w, out=first) == first
    assert calls == ["scar_resnorm_backward"] * 4
