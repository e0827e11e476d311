"""The native marshalling of the language-model calls: what it leaves to the general path, and a module that does not load."""
import sys
import warnings

import pytest
import torch

from paper_1908_05033_amd import binding as B

CALLS = {"rms_norm": 10, "rms_norm_bwd": 9, "linear_w4": 9, "linear_w4a8": 10}


def test_init_takes_seven_addresses():
    m = B.load_marshal()
    for args in ((), (1,) * 6, (1,) * 8):
        with pytest.raises(TypeError):
            m.init_lm(*args)
    with pytest.raises(TypeError):
        m.init_lm(*["x"] * 7)


@pytest.mark.parametrize("name", CALLS)
def test_other_forms_are_left_alone(name):
    f, n = getattr(B.load_marshal(), name), CALLS[name]
    cpu = torch.zeros(4, 64)
    for args in ([None] * n, [cpu] * n, [cpu] + [None] * (n - 1), [0x1000] * n, [1.0] * n, [object()] * n, [torch.zeros(4, 64, device="meta")] * n):
        assert f(*args) is None
    assert f() is None and f(*[None] * (n + 1)) is None and f(*[None] * (n - 1)) is None


def test_module_that_does_not_load(monkeypatch):
    import paper_1908_05033_amd as package
    monkeypatch.setattr(B, "_marshal", None)
    monkeypatch.delattr(package, "_marshal", raising=False)
    monkeypatch.setitem(sys.modules, "paper_1908_05033_amd._marshal", None)
    x, u8 = torch.zeros(4, 64), torch.zeros(64, dtype=torch.uint8)
    with pytest.warns(RuntimeWarning, match="_marshal"):
        with pytest.raises(TypeError):
            B.dsq_rms_norm(x, None, None, 1e-6, None, x, None, None, None)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with pytest.raises(TypeError):
            B.dsq_rms_norm_bwd(x, None, x, x, None, x, None, None)
        with pytest.raises(TypeError):
            B.dsq_linear_w4(x, u8, u8, 16, 64, 64, None, x)
        with pytest.raises(TypeError):
            B.dsq_linear_w4a8(u8, x, u8, u8, 16, 64, 64, None, x)
