"""Host-side refusals of the operators around the layer: checked before any HIP call,
with the documented status and a sentence that names the argument."""
import ctypes
import os
from ctypes import byref, c_void_p

import pytest

from paper_2606_00395_amd import binding as B

pytestmark = [
    pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libpr2.so not built"),
    # the calls that pass the checks name addresses that no kernel may be given
    pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="runs on machines without a GPU"),
]

P1, P2, P3 = 0x10000, 0x200000000, 0x400000000     # far apart, never dereferenced
READY = ("PR2_ERR_DEVICE", "PR2_OK")


def name(st):
    msg = B.lib().pr2_last_error().decode()
    if st:
        assert msg
    return B.STATUS[st]


def policy_desc(**kw):
    base = dict(T=4, ldl=100, ldd=100, V=100, act_dtype=B.PR2_BF16, token_dtype=B.PR2_I64,
                inv_temp=1.0, clip_low=0.2, clip_high=0.28, kl_coef=0.0)
    base.update(kw)
    return B.PolicyDesc(**base)


def ptrs(args, **kw):
    args = dict(args, **kw)
    return [c_void_p(v) if v else None for v in args.values()]


def loss(d, ws_bytes=None, **kw):
    a = dict(logits=P1, token=P2, old=P2, ref=0, adv=P2, weight=0, sums=P2, logp=0, lse=0, ent=0,
             coef=0, dlogits=P3, ws=P2)
    need = B.lib().pr2_policy_workspace_bytes(byref(d)) if ws_bytes is None else ws_bytes
    return name(B.lib().pr2_policy_loss(byref(d), *ptrs(a, **kw), need, None))


def logprob(d, ws_bytes=None, **kw):
    a = dict(logits=P1, token=P2, logp=P2, lse=0, ent=0, ws=P2)
    need = B.lib().pr2_policy_workspace_bytes(byref(d)) if ws_bytes is None else ws_bytes
    return name(B.lib().pr2_token_logprob(byref(d), *ptrs(a, **kw), need, None))


def loss_backward(d, **kw):
    a = dict(logits=P1, token=P2, lse=P2, coef=P2, grad=0, dlogits=P3)
    return name(B.lib().pr2_policy_loss_backward(byref(d), *ptrs(a, **kw), None))


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "PR2_ERR_SHAPE"), (dict(V=0), "PR2_ERR_SHAPE"), (dict(ldl=99), "PR2_ERR_SHAPE"),
    (dict(act_dtype=9), "PR2_ERR_DTYPE"), (dict(token_dtype=B.PR2_I16), "PR2_ERR_DTYPE"),
    (dict(inv_temp=0.0), "PR2_ERR_SHAPE"), (dict(inv_temp=-1.0), "PR2_ERR_SHAPE"),
    (dict(inv_temp=float("nan")), "PR2_ERR_SHAPE"), (dict(inv_temp=float("inf")), "PR2_ERR_SHAPE"),
    (dict(T=1 << 40), "PR2_ERR_UNSUPPORTED"), (dict(ldl=1 << 40), "PR2_ERR_UNSUPPORTED"), (dict(V=2 ** 31 - 1, ldl=2 ** 31), "PR2_ERR_UNSUPPORTED"),
])
def test_policy_descriptor(kw, status):
    d = policy_desc(**kw)
    if "V" in kw:
        d.ldd = max(d.ldd, d.ldl)
    for fn in (loss, logprob, loss_backward):
        assert fn(d) == status


def test_policy_arguments():
    d = policy_desc()
    for kw in (dict(clip_low=-0.1), dict(clip_high=float("nan")), dict(kl_coef=float("inf"))):
        assert loss(policy_desc(**kw)) == "PR2_ERR_SHAPE"
        assert logprob(policy_desc(**kw)) in READY          # not read there
    for n in ("logits", "token", "old", "adv", "sums", "ws"):
        assert loss(d, **{n: 0}) == "PR2_ERR_NULL", n
    for n in ("logits", "token", "logp", "ws"):
        assert logprob(d, **{n: 0}) == "PR2_ERR_NULL", n
    for n in ("logits", "token", "lse", "coef", "dlogits"):
        assert loss_backward(d, **{n: 0}) == "PR2_ERR_NULL", n
    assert loss(policy_desc(ldd=99)) == "PR2_ERR_SHAPE"
    assert loss(policy_desc(ldd=0), dlogits=0) in READY      # not read without a gradient
    assert loss(d, logits=P1 + 1) == "PR2_ERR_ALIGN"
    assert loss(d, logits=P1 + 2) in READY                   # bf16 rows start anywhere
    assert loss(policy_desc(act_dtype=B.PR2_F32), logits=P1 + 2) == "PR2_ERR_ALIGN"
    assert loss(d, token=P2 + 4) == "PR2_ERR_ALIGN"
    assert loss(d, coef=P2 + 2) == "PR2_ERR_ALIGN"
    need = B.lib().pr2_policy_workspace_bytes(byref(d))
    assert loss(d, ws_bytes=need - 1) == "PR2_ERR_WORKSPACE"
    assert logprob(d, ws_bytes=need - 1) == "PR2_ERR_WORKSPACE"
    assert B.lib().pr2_policy_workspace_bytes(byref(policy_desc(T=5000))) >= need
    assert B.lib().pr2_policy_workspace_bytes(byref(policy_desc(T=1 << 60))) == 0
    # in place is the same rows or nothing
    assert loss(d, dlogits=P1) in READY
    assert loss(policy_desc(ldd=104), dlogits=P1) == "PR2_ERR_SHAPE"
    assert loss(d, dlogits=P1 + 2) == "PR2_ERR_SHAPE"
    assert loss_backward(d, dlogits=P1 + 2 * 399) == "PR2_ERR_SHAPE"
    assert loss_backward(d, dlogits=P1 + 2 * 400) in READY
    assert logprob(policy_desc(T=0), logits=0, token=0, logp=0, ws=0) == "PR2_OK"


def rows(fn, d, **kw):
    order = {"pr2_dispatch": dict(x=P1, off=P2, row=P2, xs=P3),
             "pr2_dispatch_backward": dict(dxs=P1, row=P2, dx=P3),
             "pr2_combine": dict(o=P1, row=P2, gate=P2, y=P3),
             "pr2_combine_backward": dict(dy=P2, o=P1, off=P2, row=P2, gate=P2, d_o=P3, dgate=P2)}
    return name(getattr(B.lib(), fn)(byref(d), *ptrs(order[fn], **kw), None))


ROW_ARGS = {"pr2_dispatch": ("x", "off", "row", "xs"), "pr2_dispatch_backward": ("dxs", "row", "dx"),
            "pr2_combine": ("o", "row", "gate", "y"),
            "pr2_combine_backward": ("dy", "o", "off", "row", "gate", "d_o", "dgate")}


@pytest.mark.parametrize("fn", ROW_ARGS)
def test_row_calls(fn):
    ok = B.make_desc(8, 64, 4, 2)
    assert rows(fn, ok) in READY
    for a in ROW_ARGS[fn]:
        assert rows(fn, ok, **{a: 0}) == "PR2_ERR_NULL", a
        base = {"row": P2, "off": P2, "gate": P2, "dgate": P2}.get(a)
        if base:
            assert rows(fn, ok, **{a: base + 2}) == "PR2_ERR_ALIGN", a
    for a in ("x", "xs", "dxs", "dx", "o", "y", "dy", "d_o"):
        if a in ROW_ARGS[fn]:
            assert rows(fn, ok, **{a: P1 + 0x100000 + 8}) == "PR2_ERR_ALIGN", a
    assert rows(fn, B.make_desc(8, 0, 4, 2)) == "PR2_ERR_SHAPE"
    assert rows(fn, B.make_desc(8, 64, 4, 5)) == "PR2_ERR_SHAPE"
    assert rows(fn, B.make_desc(8, 64, 4, 2, act=3)) == "PR2_ERR_DTYPE"
    assert rows(fn, B.make_desc(2 ** 31, 64, 4, 2)) == "PR2_ERR_UNSUPPORTED"
    assert rows(fn, B.make_desc(0, 64, 4, 2), **{a: 0 for a in ROW_ARGS[fn]}) == "PR2_OK"


def test_row_calls_refuse_overlap():
    d = B.make_desc(8, 64, 4, 2)
    assert rows("pr2_dispatch", d, xs=P1 + 512) == "PR2_ERR_SHAPE"
    assert rows("pr2_dispatch_backward", d, dx=P1) == "PR2_ERR_SHAPE"
    assert rows("pr2_combine", d, y=P1 + 1024) == "PR2_ERR_SHAPE"
    assert rows("pr2_combine_backward", d, d_o=P1) in READY
    assert rows("pr2_combine_backward", d, d_o=P1 + 16) == "PR2_ERR_SHAPE"
    assert rows("pr2_combine_backward", d, d_o=P2) == "PR2_ERR_SHAPE"


def test_plan_arguments():
    L = B.lib()

    def plan(d, ldi=2, ws_bytes=None, **kw):
        a = dict(off=P2, row=P2, route=P3, ws=P2)
        idx = kw.pop("idx", P1)
        need = B.workspace_bytes(d, B.OP_DISPATCH_PLAN) if ws_bytes is None else ws_bytes
        return name(L.pr2_dispatch_plan(byref(d), c_void_p(idx) if idx else None, ldi, *ptrs(a, **kw), need, None))

    d = B.make_desc(8, 64, 4, 2)
    assert plan(d) in READY
    assert plan(d, ldi=1) == "PR2_ERR_SHAPE"
    for a in ("idx", "off", "row", "route", "ws"):
        assert plan(d, **{a: 0}) == "PR2_ERR_NULL", a
    assert plan(d, idx=P1 + 2) == "PR2_ERR_ALIGN"
    assert plan(B.make_desc(8, 64, 4, 2, idx=B.PR2_I16), idx=P1 + 2) in READY
    assert plan(B.make_desc(8, 64, 4, 2, idx=B.PR2_I64)) == "PR2_ERR_DTYPE"
    need = B.workspace_bytes(d, B.OP_DISPATCH_PLAN)
    assert need > 0 and plan(d, ws_bytes=need - 1) == "PR2_ERR_WORKSPACE"
    sizes = [B.workspace_bytes(B.make_desc(T, 1, 128, 8), B.OP_DISPATCH_PLAN) for T in (0, 1, 100, 5000, 40000)]
    assert sizes == sorted(sizes)


def pack(fn, R=4, C=64, dt=B.PR2_BF16, **kw):
    order = {"pr2_act_pack": dict(x=P1, q=P2, e=P3), "pr2_act_unpack": dict(q=P1, e=P2, x=P3),
             "pr2_swiglu_pack": dict(au=P1, h=P2, q=P3, e=P2),
             "pr2_swiglu_backward_packed": dict(q=P1, e=P2, dh=P2, dau=P3, h=0)}
    return name(getattr(B.lib(), fn)(R, C, dt, *ptrs(order[fn], **kw), None))


@pytest.mark.parametrize("fn,need", [("pr2_act_pack", "x q e"), ("pr2_act_unpack", "q e x"),
                                     ("pr2_swiglu_pack", "au h q e"),
                                     ("pr2_swiglu_backward_packed", "q e dh dau")])
def test_packed_calls(fn, need):
    assert pack(fn) in READY
    for a in need.split():
        assert pack(fn, **{a: 0}) == "PR2_ERR_NULL", a
        assert pack(fn, **{a: P1 + 8}) == "PR2_ERR_ALIGN", a
    assert pack(fn, R=-1) == "PR2_ERR_SHAPE"
    assert pack(fn, C=0) == "PR2_ERR_SHAPE"
    assert pack(fn, dt=2) == "PR2_ERR_DTYPE"
    assert pack(fn, R=2 ** 31) == "PR2_ERR_UNSUPPORTED"
    assert pack(fn, C=2 ** 30) == "PR2_ERR_UNSUPPORTED"
    assert pack(fn, R=0, **{a: 0 for a in need.split()}) == "PR2_OK"
    if fn == "pr2_swiglu_backward_packed":
        assert pack(fn, h=P1 + 8) == "PR2_ERR_ALIGN"


def test_weight_grad_arguments():
    def wg(ws_bytes=None, ptr=None, **kw):
        base = dict(R=16, Rx=16, n_out=64, n_in=64, N=2, k=1, act_dtype=B.PR2_BF16)
        base.update(kw)
        d = B.WgradDesc(**base)
        a = dict(dy=P1, q=P2, e=P2, off=P2, route=0, dW=P3, ws=P2)
        need = B.lib().pr2_weight_grad_workspace_bytes(byref(d)) if ws_bytes is None else ws_bytes
        return name(B.lib().pr2_weight_grad_packed(byref(d), *ptrs(a, **(ptr or {})), need, None))

    assert wg() in READY
    for a in ("dy", "q", "e", "off", "dW"):
        assert wg(ptr={a: 0}) == "PR2_ERR_NULL", a
    assert wg(N=1, ptr={"off": 0}) in READY
    for a, base in (("dy", P1), ("q", P2), ("e", P2), ("dW", P3)):
        assert wg(ptr={a: base + 8}) == "PR2_ERR_ALIGN", a
    assert wg(ptr={"route": P2 + 2}) == "PR2_ERR_ALIGN"
    for kw in (dict(R=-1), dict(Rx=-1), dict(n_out=0), dict(n_in=0), dict(N=0), dict(k=0), dict(R=17)):
        assert wg(**kw) == "PR2_ERR_SHAPE", kw
    assert wg(R=17, ptr={"route": P2}) in READY
    assert wg(act_dtype=5) == "PR2_ERR_DTYPE"
    for kw in (dict(N=1025), dict(R=2 ** 31, Rx=2 ** 31), dict(n_in=2 ** 21)):
        assert wg(**kw) == "PR2_ERR_UNSUPPORTED", kw
    assert wg(R=0, Rx=0, ptr=dict(dy=0, q=0, e=0, off=0)) in READY      # zeros are still written
    # few tiles and many rows: the workspace holds the slices' partial sums
    long = dict(R=8192, Rx=8192, n_out=2048, n_in=2048, N=1)
    need = B.lib().pr2_weight_grad_workspace_bytes(byref(B.WgradDesc(k=1, act_dtype=B.PR2_BF16, **long)))
    assert need > 2 * 4 * 2048 * 2048
    assert wg(ptr={"off": 0}, **long) in READY
    assert wg(ptr={"off": 0}, ws_bytes=need - 1, **long) == "PR2_ERR_WORKSPACE"
    assert wg(ptr={"off": 0, "ws": 0}, **long) == "PR2_ERR_NULL"


def test_null_descriptors():
    L = B.lib()
    for fn in ("pr2_policy_workspace_bytes", "pr2_weight_grad_workspace_bytes"):
        assert getattr(L, fn)(None) == 0
    assert name(L.pr2_policy_loss(None, *[None] * 13, 0, None)) == "PR2_ERR_NULL"
    assert name(L.pr2_combine(None, *[None] * 5)) == "PR2_ERR_NULL"
    assert name(L.pr2_weight_grad_packed(None, *[None] * 7, 0, None)) == "PR2_ERR_NULL"


def test_host_checks_under_the_sanitizers():
    """These checks against the library's host code built with AddressSanitizer and
    UndefinedBehaviorSanitizer."""
    import shutil
    import subprocess
    import sys
    if os.environ.get("PR2_LIBRARY"):
        pytest.skip("already running against a named build")
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not available")
    try:
        from paper_2606_00395_amd import build_sanitized as S
    except ImportError:
        pytest.skip("the sanitizer build is not part of this tree")
    env = dict(os.environ, LD_PRELOAD=S.runtime_preload(), PR2_LIBRARY=S.build(), HIP_VISIBLE_DEVICES="",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-s",
                        "-p", "no:cacheprovider"], env=env, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0 and "runtime error" not in r.stdout, r.stdout[-2000:]


@pytest.mark.parametrize("n_out,n_in,N,dt", [(512, 512, 1, B.PR2_BF16), (2048, 2048, 1, B.PR2_BF16), (64, 128, 1, B.PR2_BF16),
                                             (64, 128, 9, B.PR2_F32), (33, 50, 20, B.PR2_F32), (135, 203, 7, B.PR2_BF16)])
def test_weight_grad_workspace_does_not_decrease_with_the_rows(n_out, n_in, N, dt):
    def need(R):
        d = B.WgradDesc(R=R, Rx=R, n_out=n_out, n_in=n_in, N=N, k=1, act_dtype=dt)
        return B.lib().pr2_weight_grad_workspace_bytes(byref(d))

    sizes = [need(R) for R in [*range(6000), *range(6000, 70000, 371), 2 ** 24, 2 ** 30]]
    assert sizes[0] > 0 and sizes == sorted(sizes)


def test_rows_of_logits_and_gradient_between_each_other():
    """Column parts of one buffer do not overlap; parts that share columns do."""
    d = policy_desc(ldl=250, ldd=250)
    for start, status in ((200, None), (300, None), (302, "PR2_ERR_SHAPE"), (198, "PR2_ERR_SHAPE"), (700, None),
                          (-300, None), (-200, None), (-198, "PR2_ERR_SHAPE"), (500, "PR2_ERR_SHAPE"), (2000, None)):
        for fn in (loss, loss_backward):
            got = fn(d, dlogits=P1 + start)
            assert got in READY if status is None else got == status, start
    assert loss(policy_desc(ldl=250, ldd=251), dlogits=P1 + 200) == "PR2_ERR_SHAPE"
    assert loss(policy_desc(ldl=250, ldd=250, T=1), dlogits=P1 + 200) in READY
