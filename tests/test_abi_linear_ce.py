"""Host-side checks of the linear cross-entropy entry points (CPU only, no kernel launches): bad arguments get the
documented status before anything is launched."""
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


BASE = dict(m=10, c=64, classes=100, dtype=BF16, h=A, h_ld=64, w=A + MB, w_ld=64, bias=A + 2 * MB, labels=A + 3 * MB,
            ignore=-1, smoothing=0.0, z=0.0, lse=A + 4 * MB, ce=True, ws=A + 100 * MB, ws_bytes=1 << 40)
BAD = [
    (dict(m=0), "BNR_ERR_SHAPE"), (dict(m=-2), "BNR_ERR_SHAPE"), (dict(m=(1 << 24) + 1), "BNR_ERR_SHAPE"),
    (dict(c=0), "BNR_ERR_SHAPE"), (dict(classes=0), "BNR_ERR_SHAPE"), (dict(classes=-5), "BNR_ERR_SHAPE"),
    (dict(classes=(1 << 30) + 1), "BNR_ERR_UNSUPPORTED"),
    (dict(dtype=2), "BNR_ERR_DTYPE"), (dict(m=1 << 24, classes=1 << 30), "BNR_ERR_UNSUPPORTED"),
    (dict(m=1 << 24, c=(1 << 16) + 8, h_ld=1 << 17, w_ld=1 << 17), "BNR_ERR_UNSUPPORTED"),
    (dict(h=None), "BNR_ERR_NULL"), (dict(w=None), "BNR_ERR_NULL"), (dict(ce=False), "BNR_ERR_NULL"),
    (dict(labels=None), "BNR_ERR_NULL"), (dict(lse=None), "BNR_ERR_NULL"),
    (dict(h=A + 2), "BNR_ERR_ALIGN"), (dict(w=A + MB + 8), "BNR_ERR_ALIGN"), (dict(c=60), "BNR_ERR_ALIGN"),
    (dict(h_ld=68), "BNR_ERR_ALIGN"), (dict(w_ld=66), "BNR_ERR_ALIGN"), (dict(dtype=F32, c=62), "BNR_ERR_ALIGN"),
    (dict(labels=A + 3 * MB + 2), "BNR_ERR_ALIGN"), (dict(bias=A + 2 * MB + 1), "BNR_ERR_ALIGN"),
    (dict(lse=A + 4 * MB + 2), "BNR_ERR_ALIGN"), (dict(h_ld=56), "BNR_ERR_SHAPE"), (dict(w_ld=32), "BNR_ERR_SHAPE"),
    (dict(w_ld=(1 << 20) + 8), "BNR_ERR_UNSUPPORTED"), (dict(smoothing=1.0), "BNR_ERR_SHAPE"),
    (dict(smoothing=-0.1), "BNR_ERR_SHAPE"), (dict(smoothing=float("nan")), "BNR_ERR_SHAPE"),
    (dict(z=-1.0), "BNR_ERR_SHAPE"), (dict(z=float("inf")), "BNR_ERR_SHAPE"), (dict(z=float("nan")), "BNR_ERR_SHAPE"),
    (dict(ws=None), "BNR_ERR_WORKSPACE"), (dict(ws_bytes=100), "BNR_ERR_WORKSPACE"), (dict(ws=A + 100 * MB + 16), "BNR_ERR_ALIGN"),
]


def _ce(B, a):
    s = B.CEStruct(a["bias"], a["labels"], a["ignore"], a["smoothing"], a["z"], a["lse"])
    return s, (ctypes.byref(s) if a["ce"] else None)


def _fwd(B, **kw):
    a = dict(BASE, loss=A + 5 * MB)
    a.update(kw)
    s, ref = _ce(B, a)
    return B.STATUS[B._lib_fns["bnr_linear_ce_fwd"](a["m"], a["c"], a["classes"], a["dtype"], a["h"], a["h_ld"], a["w"],
                                                    a["w_ld"], ref, a["loss"], a["ws"], a["ws_bytes"], None)]


def _bwd(B, **kw):
    a = dict(BASE, dloss=None, dh=A + 6 * MB, dh_ld=64, dw=A + 7 * MB, dw_ld=64, dw_dtype=BF16, dbias=A + 8 * MB)
    a.update(kw)
    s, ref = _ce(B, a)
    return B.STATUS[B._lib_fns["bnr_linear_ce_bwd"](a["m"], a["c"], a["classes"], a["dtype"], a["h"], a["h_ld"], a["w"],
                                                    a["w_ld"], ref, a["dloss"], a["dh"], a["dh_ld"], a["dw"], a["dw_ld"],
                                                    a["dw_dtype"], a["dbias"], a["ws"], a["ws_bytes"], None)]


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(loss=None), "BNR_ERR_NULL"), (dict(loss=A + 5 * MB + 1), "BNR_ERR_ALIGN"),
    (dict(loss=A + 4 * MB + 40), "BNR_ERR_ALIAS"), (dict(loss=A + 64), "BNR_ERR_ALIAS"),
    (dict(loss=A + MB + 64), "BNR_ERR_ALIAS"), (dict(loss=A + 2 * MB + 4), "BNR_ERR_ALIAS"),
    (dict(lse=A + 3 * MB), "BNR_ERR_ALIAS"),
])
def test_forward_refuses(B, kw, status):
    assert _fwd(B, **kw) == status, B._lib_fns["bnr_last_error"]()


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(dh=None, dw=None, dbias=None), "BNR_ERR_NULL"), (dict(dw_dtype=5), "BNR_ERR_DTYPE"),
    (dict(dh=A + 6 * MB + 2), "BNR_ERR_ALIGN"), (dict(dw=A + 7 * MB + 4), "BNR_ERR_ALIGN"),
    (dict(dbias=A + 8 * MB + 2), "BNR_ERR_ALIGN"), (dict(dloss=A + 9 * MB + 1), "BNR_ERR_ALIGN"),
    (dict(dh_ld=60), "BNR_ERR_SHAPE"), (dict(dw_ld=68), "BNR_ERR_ALIGN"), (dict(dw_dtype=F32, dw_ld=66), "BNR_ERR_ALIGN"),
    (dict(dh=A), "BNR_ERR_ALIAS"), (dict(dw=A + MB), "BNR_ERR_ALIAS"), (dict(dh=A + 7 * MB - 64), "BNR_ERR_ALIAS"),
    (dict(dbias=A + 7 * MB + 64), "BNR_ERR_ALIAS"), (dict(dbias=A + 4 * MB), "BNR_ERR_ALIAS"),
    (dict(dbias=A + 2 * MB), "BNR_ERR_ALIAS"), (dict(dloss=A + 8 * MB), "BNR_ERR_ALIAS"), (dict(dh=A + 3 * MB), "BNR_ERR_ALIAS"),
])
def test_backward_refuses(B, kw, status):
    assert _bwd(B, **kw) == status, B._lib_fns["bnr_last_error"]()


def test_slices_of_one_buffer_are_apart(B):
    """dh may be another channel slice of h's buffer (here the call goes on to the next refusal), not one that shares
    channels."""
    assert _bwd(B, h_ld=192, dh=A + 128, dh_ld=192, ws=None) == "BNR_ERR_WORKSPACE"
    assert _bwd(B, h_ld=192, dh=A + 64, dh_ld=192, ws=None) == "BNR_ERR_ALIAS"


def test_workspace_size(B):
    f = B._lib_fns["bnr_linear_ce_workspace_size"]
    for back in (0, 1):
        assert f(1, 8, 1, BF16, back) > 0 and f(8192, 4096, 131072, BF16, back) > 0 and f(100, 4, 7, F32, back) > 0
        for m, c, v, t in ((0, 8, 8, BF16), (4, 0, 8, BF16), (4, 8, 0, BF16), (4, 8, 8, 3), (4, 12, 8, BF16), (4, 6, 8, F32)):
            assert f(m, c, v, t, back) == 0
    # never all gradients of the logits at once
    assert f(8192, 4096, 131072, BF16, 1) < 8192 * 131072 * 2
    assert f(1 << 16, 1024, 131072, BF16, 1) < 4 << 30


def test_binding_refuses(B):
    h, w, labels = torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int32)
    loss = torch.zeros(5)
    ce = B.CE(labels)
    assert ce.lse.shape == (5,)
    with pytest.raises(ValueError):                       # not a GPU's
        B.bnr_linear_ce_fwd(h, w, ce, loss)
    for bad in (dict(h=torch.zeros(4, 16)), dict(w=torch.zeros(5, 8, dtype=torch.bfloat16)), dict(loss=torch.zeros(4)),
                dict(ce=B.CE(labels.long())), dict(ce=B.CE(labels[:3])), dict(ce=B.CE(labels, bias=torch.zeros(4))),
                dict(ce=B.CE(labels, lse=torch.zeros(4))), dict(w=torch.zeros(2, 5, 8)), dict(ce=B.CE(labels, ignore=1 << 40))):
        a = dict(h=h, w=w, ce=ce, loss=loss)
        a.update(bad)
        with pytest.raises(ValueError):
            B.bnr_linear_ce_fwd(**a)
    for bad in (dict(dh=torch.zeros(3, 8)), dict(dw=torch.zeros(5, 9)), dict(dbias=torch.zeros(6)), dict(dloss=torch.zeros(4))):
        with pytest.raises(ValueError):
            B.bnr_linear_ce_bwd(h, w, ce, **bad)


@pytest.mark.parametrize("m,c,v,t", [(1 << 16, 1024, 131072, BF16), (1 << 18, 64, 131072, F32), (1 << 20, 64, 131072, BF16)])
def test_backward_keeps_nothing_of_all_classes(B, m, c, v, t):
    """The rows' copy, float32 sums of dh, a piece's g (256 MiB, or 512 classes) and 1/16 as much for dbias, whatever the
    number of classes."""
    es = 2 if t == BF16 else 4
    most = m * c * (es + 4) + max(256 << 20, m * 512 * es) * 17 // 16 + m * 64 + (64 << 20)
    assert B._lib_fns["bnr_linear_ce_workspace_size"](m, c, v, t, 1) < most
