"""Host-side refusals of the norm, the products by expert and the row form in 8 bits: checked before
any HIP call, with the documented status and a sentence that names the argument."""
import os
from ctypes import byref, c_void_p

import pytest

from paper_2606_00395_amd import binding as B

pytestmark = [
    pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libpr2.so not built"),
    # the calls that pass the checks name addresses that no kernel may be given
    pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="runs on machines without a GPU"),
]

READY = ("PR2_ERR_DEVICE", "PR2_OK")
FAR = 1 << 40


def name(st):
    msg = B.lib().pr2_last_error().decode()
    if st:
        assert msg
    return B.STATUS[st]


def ptrs(args):
    return [c_void_p(v) if v else None for v in args.values()]


def places(names):
    """An address for each tensor, far apart, never dereferenced."""
    return {n: FAR * (i + 1) for i, n in enumerate(names.split())}


MM = {"pr2_grouped_mm": "x W offsets route out", "pr2_grouped_mm_backward": "dy W offsets dx",
      "pr2_grouped_mm_quant": "q row_scale Wq w_scale offsets route out", "pr2_weight_grad": "dy x offsets route dW ws"}
NEED = {"pr2_grouped_mm": "x W out", "pr2_grouped_mm_backward": "dy W dx",
        "pr2_grouped_mm_quant": "q row_scale Wq w_scale out", "pr2_weight_grad": "dy x dW ws"}


def mm(fn, ptr=None, ws_bytes=None, **kw):
    base = dict(R=64, Rx=32, n_out=48, n_in=40, N=4, k=2, act_dtype=B.PR2_BF16)
    base.update(kw)
    d = B.WgradDesc(*(base[f] for f in ("R", "Rx", "n_out", "n_in", "N", "k", "act_dtype")))
    args = dict(places(MM[fn]), **(ptr or {}))
    tail = []
    if fn == "pr2_weight_grad":
        tail = [B.lib().pr2_weight_grad_workspace_bytes(byref(d)) if ws_bytes is None else ws_bytes]
    return name(getattr(B.lib(), fn)(byref(d), *ptrs(args), *tail, None))


@pytest.mark.parametrize("fn", MM)
def test_products(fn):
    assert mm(fn) in READY
    assert mm(fn, R=0) in READY
    for kw in (dict(R=-1), dict(n_out=0), dict(n_in=0), dict(N=0)):
        assert mm(fn, **kw) == "PR2_ERR_SHAPE", kw
    for kw in (dict(N=1025), dict(R=2 ** 31), dict(n_out=(1 << 20) + 1), dict(n_in=(1 << 20) + 1),
               dict(N=1024, n_out=1 << 14, n_in=1 << 13)):
        assert mm(fn, **kw) == "PR2_ERR_UNSUPPORTED", kw
    assert mm(fn, act_dtype=2) == "PR2_ERR_DTYPE"
    if fn != "pr2_grouped_mm_backward":
        for kw in (dict(Rx=-1), dict(k=0)):
            assert mm(fn, **kw) == "PR2_ERR_SHAPE", kw
        assert mm(fn, ptr=dict(route=0)) == "PR2_ERR_SHAPE"             # R > Rx
        assert mm(fn, ptr=dict(route=0), Rx=64) in READY
        assert mm(fn, Rx=2 ** 31) == "PR2_ERR_UNSUPPORTED"
    for n in NEED[fn].split():
        assert mm(fn, ptr={n: 0}) == "PR2_ERR_NULL", n
        if n != "ws":
            assert mm(fn, ptr={n: FAR + 2}) == "PR2_ERR_ALIGN", n
    assert mm(fn, ptr=dict(offsets=0)) == "PR2_ERR_NULL"
    assert mm(fn, ptr=dict(offsets=0), N=1) in READY
    assert mm(fn, ptr=dict(offsets=FAR + 2)) == "PR2_ERR_ALIGN"
    d = getattr(B.lib(), fn)(None, *ptrs(places(MM[fn])), *([0] if "ws" in MM[fn] else []), None)
    assert name(d) == "PR2_ERR_NULL"


@pytest.mark.parametrize("fn,out,ins", [("pr2_grouped_mm", "out", "x W"), ("pr2_grouped_mm_backward", "dx", "dy W"),
                                        ("pr2_grouped_mm_quant", "out", "q Wq")])
def test_products_refuse_overlap(fn, out, ins):
    for n in ins.split():
        assert mm(fn, ptr={out: places(MM[fn])[n]}) == "PR2_ERR_SHAPE", n
        assert mm(fn, ptr={out: places(MM[fn])[n] + 16}) == "PR2_ERR_SHAPE", n


def test_eight_bit_sums_stay_in_range():
    assert mm("pr2_grouped_mm_quant", n_in=(1 << 17) - 1) in READY
    assert mm("pr2_grouped_mm_quant", n_in=1 << 17) == "PR2_ERR_UNSUPPORTED"
    assert mm("pr2_grouped_mm", n_in=1 << 17) in READY


def test_weight_grad_workspace():
    assert mm("pr2_weight_grad", ws_bytes=10) == "PR2_ERR_WORKSPACE"
    d = B.WgradDesc(64, 32, 48, 40, 4, 2, B.PR2_BF16)
    assert mm("pr2_weight_grad", ws_bytes=B.lib().pr2_weight_grad_workspace_bytes(byref(d)) - 1) == "PR2_ERR_WORKSPACE"


def quant(fn, R=4, C=64, dt=B.PR2_BF16, **kw):
    return name(getattr(B.lib(), fn)(R, C, dt, *ptrs(dict(places("x q row_scale"), **kw)), None))


@pytest.mark.parametrize("fn", ["pr2_act_quant", "pr2_swiglu_quant"])
def test_rows_in_8_bits(fn):
    assert quant(fn) in READY and quant(fn, R=0, x=0, q=0, row_scale=0) in READY
    assert quant(fn, R=-1) == "PR2_ERR_SHAPE" and quant(fn, C=0) == "PR2_ERR_SHAPE"
    assert quant(fn, dt=3) == "PR2_ERR_DTYPE"
    assert quant(fn, R=2 ** 31) == "PR2_ERR_UNSUPPORTED" and quant(fn, C=(1 << 28) + 1) == "PR2_ERR_UNSUPPORTED"
    for n in "x q row_scale".split():
        assert quant(fn, **{n: 0}) == "PR2_ERR_NULL"
        assert quant(fn, **{n: FAR + 2}) == "PR2_ERR_ALIGN"
    assert quant(fn, q=FAR) == "PR2_ERR_SHAPE"


NORM = "x residual weight h_out y rstd_out q scale row_scale"


def norm(T=4, d=64, dt=B.PR2_BF16, eps=1e-6, **kw):
    args = dict(places(NORM), row_scale=0)
    args.update(kw)
    return name(B.lib().pr2_rms_norm(T, d, dt, eps, *ptrs(args), None))


def test_norm():
    assert norm() in READY and norm(scale=0, row_scale=FAR * 20) in READY
    assert norm(T=0, x=0, weight=0) in READY
    assert norm(T=-1) == "PR2_ERR_SHAPE" and norm(d=0) == "PR2_ERR_SHAPE" and norm(dt=5) == "PR2_ERR_DTYPE"
    assert norm(d=32769) == "PR2_ERR_UNSUPPORTED" and norm(T=2 ** 31) == "PR2_ERR_UNSUPPORTED"
    for eps in (-1e-9, float("nan"), float("inf")):
        assert norm(eps=eps) == "PR2_ERR_SHAPE"
    for n in ("x", "weight"):
        assert norm(**{n: 0}) == "PR2_ERR_NULL"
    assert norm(residual=0, h_out=0, y=0, rstd_out=0) in READY
    assert norm(h_out=0, y=0, rstd_out=0, q=0, scale=0) == "PR2_ERR_NULL"
    assert norm(q=0) == "PR2_ERR_NULL" and norm(scale=0) == "PR2_ERR_NULL"
    assert norm(row_scale=FAR * 20) == "PR2_ERR_SHAPE"
    for n in ("x", "residual", "h_out", "y", "q", "scale", "weight", "rstd_out"):
        assert norm(**{n: FAR * 30 + 2}) == "PR2_ERR_ALIGN", n
    p = places(NORM)
    # in place is allowed, half in place is not
    for n in ("x", "residual"):
        assert norm(h_out=p[n]) in READY and norm(y=p[n]) in READY
        assert norm(h_out=p[n] + 16) == "PR2_ERR_SHAPE" and norm(y=p[n] + 16) == "PR2_ERR_SHAPE"
        assert norm(q=p[n]) == "PR2_ERR_SHAPE" and norm(scale=p[n]) == "PR2_ERR_SHAPE"
    assert norm(y=p["h_out"]) == "PR2_ERR_SHAPE" and norm(h_out=p["x"], y=p["x"]) == "PR2_ERR_SHAPE"
    assert norm(h_out=p["x"], y=p["residual"]) in READY


BACK = "dy dh h rstd weight dx dweight ws"


def norm_backward(T=4, d=64, dt=B.PR2_BF16, ws_bytes=None, **kw):
    need = B.lib().pr2_rms_norm_workspace_bytes(T, d) if ws_bytes is None else ws_bytes
    return name(B.lib().pr2_rms_norm_backward(T, d, dt, *ptrs(dict(places(BACK), **kw)), need, None))


def test_norm_backward():
    assert norm_backward() in READY and norm_backward(dh=0) in READY
    assert norm_backward(dweight=0, ws=0, ws_bytes=0) in READY
    assert norm_backward(T=0, dy=0, h=0, rstd=0, dx=0, ws=0, ws_bytes=0) in READY
    for kw in (dict(T=-1), dict(d=0)):
        assert norm_backward(ws_bytes=1, **kw) == "PR2_ERR_SHAPE"
    assert norm_backward(d=32769, ws_bytes=1) == "PR2_ERR_UNSUPPORTED" and norm_backward(dt=5) == "PR2_ERR_DTYPE"
    for n in ("dy", "h", "rstd", "weight", "dx", "ws"):
        assert norm_backward(**{n: 0}) == "PR2_ERR_NULL", n
    for n in ("dy", "dh", "h", "rstd", "weight", "dx", "dweight"):
        assert norm_backward(**{n: FAR * 30 + 2}) == "PR2_ERR_ALIGN", n
    need = B.lib().pr2_rms_norm_workspace_bytes(4, 64)
    assert norm_backward(ws_bytes=need - 1) == "PR2_ERR_WORKSPACE"
    p = places(BACK)
    for n in ("dy", "dh", "h"):
        assert norm_backward(dx=p[n]) in READY
        assert norm_backward(dx=p[n] + 16) == "PR2_ERR_SHAPE"


def test_norm_workspace():
    size = B.lib().pr2_rms_norm_workspace_bytes
    for d in (1, 300, 2048, 2049, 9000, 32768):
        sizes = [size(T, d) for T in (1, 7, 8, 9, 300, 2047, 5000, 10 ** 6)]
        assert sizes == sorted(sizes) and sizes[0] >= 4 * d
    assert size(-1, 4) == 0 and size(4, 0) == 0 and size(4, 32769) == 0 and size(2 ** 31, 4) == 0
