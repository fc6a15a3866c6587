"""Host-side checks of the dropout entry points (CPU only, no kernel launches): bad arguments get the documented
status before anything is launched."""
import ctypes

import pytest
import torch

# addresses that are never dereferenced (validation fails first)
A = 0x10000000
MB = 1 << 20
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def B():
    from paper_1807_01702_amd import bnr
    return bnr


BAD = [
    (dict(m=0), "BNR_ERR_SHAPE"), (dict(m=-1), "BNR_ERR_SHAPE"), (dict(m=(1 << 31) + 1), "BNR_ERR_SHAPE"),
    (dict(c=0), "BNR_ERR_SHAPE"), (dict(dtype=7), "BNR_ERR_DTYPE"), (dict(x=None), "BNR_ERR_NULL"),
    (dict(y=None), "BNR_ERR_NULL"), (dict(d=False), "BNR_ERR_NULL"), (dict(p=-0.1), "BNR_ERR_SHAPE"),
    (dict(p=1.5), "BNR_ERR_SHAPE"), (dict(p=float("nan")), "BNR_ERR_SHAPE"), (dict(step_dev=A + 2), "BNR_ERR_ALIGN"),
    (dict(x=A + 1), "BNR_ERR_ALIGN"), (dict(y=A + MB + 1), "BNR_ERR_ALIGN"), (dict(dtype=F32, x=A + 2), "BNR_ERR_ALIGN"),
    (dict(x_ldc=23), "BNR_ERR_SHAPE"), (dict(y_ldc=1), "BNR_ERR_SHAPE"), (dict(add=A + 2 * MB, add_ldc=20), "BNR_ERR_SHAPE"),
    (dict(add=A + 2 * MB + 1, add_ldc=24), "BNR_ERR_ALIGN"),
    (dict(y=A + 48), "BNR_ERR_ALIAS"),                                   # a row later: not the same view
    (dict(y=A, y_ldc=32), "BNR_ERR_ALIAS"),                              # the same start, another stride
    (dict(add=A + MB + 2, add_ldc=24), "BNR_ERR_ALIAS"), (dict(step_dev=A + MB + 32), "BNR_ERR_ALIAS"),
    (dict(m=1 << 31, c=1 << 20, x_ldc=1 << 20, y=A + (1 << 53), y_ldc=1 << 20), "BNR_ERR_UNSUPPORTED"),
]


@pytest.mark.parametrize("kw,status", BAD)
@pytest.mark.parametrize("name", ["bnr_dropout_fwd", "bnr_dropout_bwd"])
def test_dropout_refuses(B, name, kw, status):
    a = dict(m=10, c=24, dtype=BF16, x=A, x_ldc=24, add=None, add_ldc=0, y=A + MB, y_ldc=24, p=0.1, step_dev=None, d=True)
    a.update(kw)
    d = B.DropoutStruct(a["p"], 1, 2, 3, a["step_dev"])
    ref = ctypes.byref(d) if a["d"] else None
    f = B._lib_fns[name]
    mid = (a["add"], a["add_ldc"], ref) if name == "bnr_dropout_fwd" else (ref, a["add"], a["add_ldc"])
    got = f(a["m"], a["c"], a["dtype"], a["x"], a["x_ldc"], *mid, a["y"], a["y_ldc"], None)
    assert B.STATUS[got] == status, B._lib_fns["bnr_last_error"]()


def test_dropout_binding_refuses(B):
    for kw in (dict(seed=-1), dict(seed=1 << 64), dict(seed=0, site=1 << 32), dict(seed=0, site=-1)):
        with pytest.raises(ValueError):
            B.Dropout(0.1, **kw)
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):                       # not a GPU's
        B.bnr_dropout_fwd(x, B.Dropout(0.1, 1), torch.zeros(4, 8))
    with pytest.raises(ValueError):                       # another shape, another type
        B.bnr_dropout_fwd(x, B.Dropout(0.1, 1), torch.zeros(4, 9))
    with pytest.raises(ValueError):
        B.bnr_dropout_bwd(x, B.Dropout(0.1, 1), torch.zeros(4, 8, dtype=torch.bfloat16))
    for step in (-1, 1 << 32, torch.zeros(1), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            B.Dropout(0.1, 1, step=step).struct()


@pytest.mark.parametrize("name", ["bnr_dropout_fwd", "bnr_dropout_bwd"])
def test_largest_call(B, name):
    """2^39 blocks of eight channels are the first too many."""
    d = B.DropoutStruct(0.1, 1, 2, 3, None)
    mid = (None, 0, ctypes.byref(d)) if name == "bnr_dropout_fwd" else (ctypes.byref(d), None, 0)
    for m, c, ldc in ((1 << 31, 2041, 2048), (1 << 31, 2048, 2048), (1 << 28, 1 << 14, 1 << 14)):
        got = B._lib_fns[name](m, c, BF16, A, ldc, *mid, A + (1 << 53), ldc, None)
        assert B.STATUS[got] == "BNR_ERR_UNSUPPORTED"
