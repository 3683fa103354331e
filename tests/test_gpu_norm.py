"""The norm in front of the layer and the row form in 8 bits, against the float64 definitions.

Tolerances, set before any run.  h is compared bit for bit.  A sum of d squares or products over
a piece, the lanes and the pieces has at most 55 roundings of 2^-24 in a row (8 elements, a tree of 6 over the
lanes, one of 7 over 128 pieces, and the products').  r takes half of that (a root) and four more roundings: 32 2^-24; y two more;
so y is within 36 2^-24 relatively, and within 2^-8 more as bf16.  dx = dh + r (g - n mean(g n)),
n = h r: every factor of its terms adds a rounding, so dx is within 70 2^-24 of r (|g| + |n| mean|g n|)
and 2 2^-24 of |dh|, and 2^-8 of itself as bf16.  dweight over T rows is within (T + 4) 2^-24 of the
sum of its terms' magnitudes.  The row form: the step is the rounded product bit for bit and q
the quotient's rounding (of fp32(h w) for the norm) exactly; the norm's scale is within 36 2^-24.
silu(a) u is within 1e-6 (1 + |a|) in bf16 and within 8 2^-24 (1 + |a| / 8) in fp32 (an exponential
of 2 2^-24 and the rounding of nothing else in its argument, a sum, a quotient, two products).
"""
import numpy as np
import pytest

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8
TYPES = pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])


def act(a, bf16):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if bf16 else t


def host(t):
    return t.double().cpu().numpy()


def stream_rows(T, d, seed):
    """Rows of different sizes with a few large columns, a row of zeros among them."""
    g = np.random.default_rng([T, d, seed])
    x = g.standard_normal((T, d)) * np.exp(g.normal(0, 3, (T, 1)))
    x[:, ::97] *= 20
    if T > 2:
        x[1] = 0
    return x


SHAPES = [(1, 1), (3, 3), (2, 7), (5, 8), (4, 9), (7, 31), (9, 33), (6, 511), (5, 512), (5, 513), (70, 333),
          (8, 1021), (5, 1025), (33, 2048), (3, 2049), (17, 4096), (4, 4100), (3, 8192), (2, 8200), (2, 16384),
          (2, 16388), (2, 32767), (3, 32768), (2500, 40), (9000, 1), (2100, 2056)]
IDS = [f"{T}x{d}" for T, d in SHAPES]


def forward(T, d, bf16, residual=True, weight=None, eps=1e-6, place=None):
    """All outputs of both 8-bit forms, and the inputs."""
    import torch
    from paper_2606_00395_amd import binding as B
    x = act(stream_rows(T, d, 0), bf16)
    res = act(stream_rows(T, d, 1), bf16) if residual else None
    g = np.random.default_rng(d)
    w = torch.from_numpy((1 + 0.3 * g.standard_normal(d)).astype(np.float32)).cuda() if weight is None else weight
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    y, h = (torch.full_like(x, float("nan")) for _ in range(2))
    q, q8 = (torch.full((T, d), 99, dtype=torch.int8, device="cuda") for _ in range(2))
    e = torch.full((T, -(-d // 32)), 77, dtype=torch.uint8, device="cuda")
    rstd, rs = nan(T), nan(T)
    B.rms_norm(x, w, y, residual=res, h_out=h, rstd_out=rstd, q=q, scale=e, eps=eps)
    B.rms_norm(x, w, residual=res, q=q8, row_scale=rs, eps=eps)
    return dict(x=x, res=res, w=w, y=y, h=h, q=q, e=e, q8=q8, rs=rs, rstd=rstd)


def check_forward(s, bf16, eps=1e-6):
    import torch
    from paper_2606_00395_amd import binding as B
    want_h = s["x"] if s["res"] is None else (s["x"].float() + s["res"].float()).to(s["x"].dtype)
    assert torch.equal(s["h"], want_h)
    h, w = host(want_h), host(s["w"])
    y, rstd = O.rms_norm(h, w, eps)
    assert np.all(np.abs(host(s["rstd"]) - rstd) <= 32 * U * rstd)
    assert np.all(np.abs(host(s["y"]) - y) <= (36 * U + (BF if bf16 else 0)) * np.abs(y) + 2.0 ** -133)
    # the packed form is act_pack's of the y that was written
    q, e = torch.empty_like(s["q"]), torch.empty_like(s["e"])
    B.act_pack(s["y"], q, e)
    assert torch.equal(s["q"], q) and torch.equal(s["e"], e)
    # the row form is that of h w
    v = (h.astype(np.float32) * w.astype(np.float32)).astype(np.float64)
    step = O.row_scale(v)
    assert np.array_equal(host(s["q8"]), np.rint(v / step[:, None]))
    assert np.all(np.abs(host(s["rs"]) - step * rstd) <= 36 * U * step * rstd)


@TYPES
@pytest.mark.parametrize("T,d", SHAPES, ids=IDS)
def test_forward(T, d, bf16):
    for residual in (True, False):
        check_forward(forward(T, d, bf16, residual), bf16)


@TYPES
def test_forward_with_large_eps_and_zero_weights(bf16):
    import torch
    w = torch.zeros(96, device="cuda")
    w[3] = -2.5
    check_forward(forward(6, 96, bf16, weight=w, eps=3.0), bf16, eps=3.0)
    check_forward(forward(2, 96, bf16, weight=torch.zeros(96, device="cuda")), bf16)


def test_forward_of_tiny_and_huge_rows_without_eps():
    """Rows whose norm is near the ends of fp32's range, and one of zeros with a positive eps."""
    import torch
    from paper_2606_00395_amd import binding as B
    g = np.random.default_rng(8)
    x = g.standard_normal((4, 100)) * np.array([1e-17, 1e-19, 1e17, 1.0])[:, None]
    w = np.full(100, 1e15)
    w[0] = 1e-20
    xt, wt = act(x, False), act(w, False)
    y, r = torch.empty_like(xt), torch.empty(4, device="cuda")
    B.rms_norm(xt, wt, y, rstd_out=r, eps=0.0)
    want, rstd = O.rms_norm(host(xt), host(wt), 0.0)
    assert np.all(np.abs(host(r) - rstd) <= 32 * U * rstd)
    assert np.all(np.abs(host(y) - want) <= 36 * U * np.abs(want) + 2.0 ** -126)
    B.rms_norm(torch.zeros_like(xt), wt, y, rstd_out=r, eps=1e-6)
    assert not y.any() and np.all(np.abs(host(r) - 1e3) <= 1e3 * 32 * U)


@TYPES
@pytest.mark.parametrize("T,d", [(6, 64), (5, 333), (3, 4100), (3, 9001)])
def test_forward_in_place(T, d, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    s = forward(T, d, bf16)
    for h_on, y_on in (("x", "res"), ("res", "x"), ("x", None), (None, "x"), (None, "res")):
        x, res = s["x"].clone(), s["res"].clone()
        at = dict(x=x, res=res)
        h = at.get(h_on, torch.empty_like(x))
        y = at.get(y_on, torch.empty_like(x))
        B.rms_norm(x, s["w"], y, residual=res, h_out=h)
        assert torch.equal(h, s["h"]) and torch.equal(y, s["y"]), (h_on, y_on)


@TYPES
@pytest.mark.parametrize("d", [40, 333, 4100])
def test_values_that_are_no_numbers_stay_in_their_rows(d, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    s = forward(6, d, bf16, residual=False)
    x = s["x"].clone()
    x[2, d - 1], x[4, 0] = float("nan"), float("inf")
    y, q, e = torch.empty_like(x), torch.empty_like(s["q"]), torch.empty_like(s["e"])
    q8, rs = torch.empty_like(q), torch.empty(6, device="cuda")
    B.rms_norm(x, s["w"], y, q=q, scale=e)
    B.rms_norm(x, s["w"], q=q8, row_scale=rs)
    ok = torch.tensor([0, 1, 3, 5], device="cuda")
    for a, b in ((y, s["y"]), (q, s["q"]), (e, s["e"]), (q8, s["q8"]), (rs, s["rs"])):
        assert torch.equal(a[ok], b[ok])
    assert torch.isnan(y[2]).all() and torch.isnan(y[4, 0]) and torch.isnan(rs[2]) and torch.isnan(rs[4])
    assert not q8[2].any() and not q8[4].any() and torch.all(e[2] == 255)


def backward_inputs(T, d, bf16):
    g = np.random.default_rng([T, d])
    h = act(stream_rows(T, d, 3), bf16)
    return (act(g.standard_normal((T, d)), bf16), h, act(g.standard_normal((T, d)), bf16),
            np.asarray(1 + 0.3 * g.standard_normal(d), dtype=np.float32))


@TYPES
@pytest.mark.parametrize("T,d", SHAPES, ids=IDS)
def test_backward(T, d, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    dy, h, dh, w = backward_inputs(T, d, bf16)
    eps = 1e-3
    rstd64 = O.rms_norm(host(h), w, eps)[1]
    rstd = torch.from_numpy(rstd64.astype(np.float32)).cuda()
    wt = torch.from_numpy(w).cuda()
    r = host(rstd)
    n = host(h) * r[:, None]
    gw = host(dy) * w
    for extra in (dh, None):
        dx, dw = torch.full_like(dy, float("nan")), torch.full((d,), float("nan"), device="cuda")
        B.rms_norm_backward(dy, h, rstd, wt, dx, dh=extra, dweight=dw)
        want, want_w = O.rms_norm_backward(host(dy), host(h), r, w, None if extra is None else host(dh))
        tol = 70 * U * r[:, None] * (np.abs(gw) + np.abs(n) * np.mean(np.abs(gw * n), axis=1, keepdims=True))
        tol += 2 * U * (0 if extra is None else np.abs(host(dh)))
        tol += (BF if bf16 else 0) * np.abs(want) + 2.0 ** -133
        assert np.all(np.abs(host(dx) - want) <= (1 + BF) * tol)
        assert np.all(np.abs(host(dw) - want_w) <= (T + 4) * U * np.sum(np.abs(host(dy) * n), axis=0))
        # without the weight's gradient, and in place: the same bits
        for on in range(3):
            a, b, c = dy.clone(), h.clone(), None if extra is None else extra.clone()
            to = (a, b, c)[on]
            if to is None:
                continue
            B.rms_norm_backward(a, b, rstd, wt, to, dh=c)
            assert torch.equal(to, dx), on


@TYPES
@pytest.mark.parametrize("T,d", [(9, 40), (70, 333), (700, 2049), (300, 2055), (600, 4099), (300, 8191), (520, 8193), (40, 16387)])
def test_backward_in_place(T, d, bf16):
    """dx on each of its inputs, also where a row's last piece is moved back over another wavefront's."""
    import torch
    from paper_2606_00395_amd import binding as B
    g = torch.Generator(device="cuda").manual_seed(T)
    D = torch.bfloat16 if bf16 else torch.float32
    at = {n: torch.randn((T, d), generator=g, device="cuda").to(D) for n in ("dy", "h", "dh")}
    w, r = torch.rand(d, generator=g, device="cuda"), torch.rand(T, generator=g, device="cuda")
    want, dw = torch.empty_like(at["h"]), torch.empty(d, device="cuda")
    B.rms_norm_backward(at["dy"], at["h"], r, w, want, at["dh"], dw)
    for n in at:
        now = {k: v.clone() for k, v in at.items()}
        dw2 = torch.empty(d, device="cuda")
        B.rms_norm_backward(now["dy"], now["h"], r, w, now[n], now["dh"], dw2)
        assert torch.equal(now[n], want) and torch.equal(dw, dw2), n


def test_backward_against_differences():
    import torch
    from paper_2606_00395_amd import binding as B
    T, d, eps = 3, 24, 0.05
    g = np.random.default_rng(5)
    x, dy = g.standard_normal((T, d)), g.standard_normal((T, d))
    w = 1 + 0.3 * g.standard_normal(d)
    xt, dyt, wt = act(x, False), act(dy, False), act(w, False)
    y, rstd, dx, dw = torch.empty_like(xt), torch.empty(T, device="cuda"), torch.empty_like(xt), torch.empty_like(wt)
    B.rms_norm(xt, wt, y, rstd_out=rstd, eps=eps)
    B.rms_norm_backward(dyt, xt, rstd, wt, dx, dweight=dw)
    x, dy, w = host(xt), host(dyt), host(wt)
    loss = lambda x, w: np.sum(dy * O.rms_norm(x, w, eps)[0])
    step = 1e-5
    for i in np.ndindex(T, d):
        e = np.zeros((T, d))
        e[i] = step
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - host(dx)[i]) < 1e-5
    for i in range(d):
        e = np.zeros(d)
        e[i] = step
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * step) - host(dw)[i]) < 1e-5


@TYPES
@pytest.mark.parametrize("d", [300, 600, 1500, 2048, 3000, 5000, 8192])
def test_a_row_has_the_same_bits_in_any_batch(d, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    T = 2600
    s = forward(T, d, bf16)
    g = torch.Generator(device="cuda").manual_seed(d)
    dy = torch.randn((T, d), generator=g, device="cuda").to(s["x"].dtype)
    dx, a8, b8 = torch.empty_like(dy), torch.empty_like(s["q"]), torch.empty(T, device="cuda")
    B.rms_norm_backward(dy, s["h"], s["rstd"], s["w"], dx)
    B.act_quant(s["y"], a8, b8)
    for n in (1, 7, 300):
        c = {k: v[-n:].clone() for k, v in s.items() if k not in ("w",)}
        B.rms_norm(c["x"], s["w"], c["y"].zero_(), residual=c["res"], h_out=c["h"].zero_(), rstd_out=c["rstd"].zero_(),
                   q=c["q"].zero_(), scale=c["e"].zero_())
        B.rms_norm(c["x"], s["w"], residual=c["res"], q=c["q8"].zero_(), row_scale=c["rs"].zero_())
        for k in ("y", "h", "rstd", "q", "e", "q8", "rs"):
            assert torch.equal(c[k], s[k][-n:]), (n, k)
        part, q, rs = torch.empty_like(dx[-n:]), torch.empty_like(a8[-n:]), torch.empty(n, device="cuda")
        B.rms_norm_backward(dy[-n:].clone(), c["h"], c["rstd"], s["w"], part)
        B.act_quant(c["y"], q, rs)
        assert torch.equal(part, dx[-n:]) and torch.equal(q, a8[-n:]) and torch.equal(rs, b8[-n:])


def test_no_rows():
    import torch
    from paper_2606_00395_amd import binding as B
    x, w = torch.empty((0, 48), device="cuda"), torch.ones(48, device="cuda")
    dw = torch.full((48,), 9.0, device="cuda")
    B.rms_norm(x, w, torch.empty_like(x))
    B.rms_norm_backward(x, x, torch.empty(0, device="cuda"), w, torch.empty_like(x), dweight=dw)
    assert not dw.any()
    B.act_quant(x, torch.empty((0, 48), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"))


def test_one_workspace_for_batches_up_to_the_largest():
    import torch
    from paper_2606_00395_amd import binding as B
    dy, h, _, w = backward_inputs(5000, 257, True)
    ws = B.rms_norm_workspace(dy)
    rstd, w = torch.rand(5000, device="cuda"), torch.from_numpy(w).cuda()
    for T in (5000, 2047, 8, 1):
        dx, a, b = torch.empty_like(dy[:T]), torch.empty_like(w), torch.empty_like(w)
        B.rms_norm_backward(dy[:T], h[:T], rstd[:T], w, dx, dweight=a, ws=ws)
        B.rms_norm_backward(dy[:T], h[:T], rstd[:T], w, dx, dweight=b)
        assert torch.equal(a, b)


QUANT = [(1, 1), (4, 3), (3, 8), (5, 17), (7, 100), (6, 512), (5, 777), (4, 1025), (9, 2048), (3, 2051), (3, 8192),
         (2, 8197), (2, 32768), (2, 32771), (2, 100003), (5000, 24)]


@TYPES
@pytest.mark.parametrize("R,C", QUANT, ids=[f"{R}x{C}" for R, C in QUANT])
def test_row_form(R, C, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    x = stream_rows(R, C, 7)
    if R > 3:
        x[3] *= 1e-35
        x[0] *= 3e38 / np.abs(x[0]).max()
    x = act(x, bf16)
    q, s = torch.full((R, C), 99, dtype=torch.int8, device="cuda"), torch.full((R,), float("nan"), device="cuda")
    B.act_quant(x, q, s)
    v = host(x)
    step = O.row_scale(v)
    assert np.array_equal(host(s), step)
    assert np.array_equal(host(q), np.rint(v / step[:, None]))
    if R > 3:
        # rows that are no numbers
        x[2, C // 2], x[3, C - 1] = float("inf"), float("nan")
        q2, s2 = torch.empty_like(q), torch.empty_like(s)
        B.act_quant(x, q2, s2)
        assert torch.isnan(s2[2:4]).all() and not q2[2:4].any()
        keep = [r for r in range(R) if r not in (2, 3)]
        assert torch.equal(q2[keep], q[keep]) and torch.equal(s2[keep], s[keep])


@TYPES
@pytest.mark.parametrize("R,m", QUANT, ids=[f"{R}x{m}" for R, m in QUANT])
def test_row_form_of_swiglu(R, m, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    g = np.random.default_rng([R, m])
    au = act(g.normal(0, 2, (R, 2 * m)), bf16)
    q, s = torch.full((R, m), 99, dtype=torch.int8, device="cuda"), torch.full((R,), float("nan"), device="cuda")
    B.swiglu_quant(au, q, s)
    a, u = host(au)[:, :m], host(au)[:, m:]
    v = O.swiglu(a, u)
    off = (1e-6 * (1 + np.abs(a)) if bf16 else U * (8 + np.abs(a))) * np.abs(v)      # of each value
    step = O.row_scale(v)
    most = off.max(1) / (127 * step)                    # of the row's largest, relatively
    assert np.all(np.abs(host(s) - step) <= (3 * U + most) * step)
    assert np.all(np.abs(host(q) - v / step[:, None]) <= 0.5 + 127 * 2 * U + (off / step[:, None] + 127 * most[:, None]))


@TYPES
def test_row_form_next_to_a_half(bf16):
    """Every odd multiple of half a step and its neighbours, at steps of many mantissas: rounded as
    exact arithmetic rounds them, ties to even."""
    import torch
    from paper_2606_00395_amd import binding as B
    g = np.random.default_rng(2)
    top = np.concatenate([[127.0, 254.0, 63.5, 127 * 2.0 ** 60], g.uniform(1, 1000, 400)]).astype(np.float32)
    step = (top * np.float32(1 / 127)).astype(np.float32)
    halves = np.arange(-126.5, 127)
    near = np.stack([step[:, None].astype(np.float64) * halves * (1 + f * U) for f in (-3, -2, -1, 0, 1, 2, 3)], 2)
    x = np.concatenate([top[:, None].astype(np.float64), near.reshape(len(top), -1)], 1)
    x = np.clip(x, -top[:, None], top[:, None])
    x = act(x, bf16)
    q, s = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(len(top), device="cuda")
    B.act_quant(x, q, s)
    v = host(x)
    step = O.row_scale(v)
    assert np.array_equal(host(s), step)
    assert np.array_equal(host(q), np.rint(v / step[:, None]))


def test_more_rows_than_workgroups_and_large_offsets():
    """More than 2^31 elements: the first and last rows as alone."""
    import torch
    from paper_2606_00395_amd import binding as B
    T, d, n = 1_100_000, 2048, 64
    x = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    for sl in (slice(0, n), slice(T - n, T)):
        x[sl] = torch.randn((n, d), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(d, generator=g, device="cuda")
    y, q, s = torch.empty_like(x), torch.empty((T, d), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    rstd = torch.empty(T, device="cuda")
    B.rms_norm(x, w, y, rstd_out=rstd, q=q, row_scale=s)
    for sl in (slice(0, n), slice(T - n, T)):
        y2, q2, s2 = torch.empty_like(y[sl]), torch.empty_like(q[sl]), torch.empty_like(s[sl])
        B.rms_norm(x[sl].clone(), w, y2, q=q2, row_scale=s2)
        assert torch.equal(y[sl], y2) and torch.equal(q[sl], q2) and torch.equal(s[sl], s2)
    assert not y[n:T - n].any() and not q[n:T - n].any()
    B.act_quant(y, q, s)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    B.rms_norm_backward(y, x, rstd, w, dx, dweight=dw)
    for sl in (slice(0, n), slice(T - n, T)):
        q2, s2, dx2 = torch.empty_like(q[sl]), torch.empty_like(s[sl]), torch.empty_like(dx[sl])
        B.act_quant(y[sl].clone(), q2, s2)
        B.rms_norm_backward(y[sl].clone(), x[sl].clone(), rstd[sl].clone(), w, dx2)
        assert torch.equal(q[sl], q2) and torch.equal(s[sl], s2) and torch.equal(dx[sl], dx2)


def test_refusals_of_the_binding():
    import torch
    from paper_2606_00395_amd import binding as B
    x, w = torch.zeros((4, 64), device="cuda"), torch.ones(64, device="cuda")
    y = torch.empty_like(x)
    q, s = torch.empty((4, 64), dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    with pytest.raises(TypeError):
        B.rms_norm(x.half(), w, y)
    with pytest.raises(ValueError):
        B.rms_norm(x, w[:32], y)
    with pytest.raises(ValueError):
        B.rms_norm(x[:, ::2], w[::2], y)
    with pytest.raises(B.Pr2Error):
        B.rms_norm(x, w)
    with pytest.raises(B.Pr2Error):
        B.rms_norm(x, w, y, q=q)
    with pytest.raises(TypeError):
        B.rms_norm(x, w, y, residual=x.to(torch.bfloat16))
    with pytest.raises(ValueError):
        B.rms_norm(x.cpu(), w, y)
    with pytest.raises(TypeError):
        B.act_quant(x, q.to(torch.uint8), s)
    with pytest.raises(ValueError):
        B.swiglu_quant(torch.zeros((4, 63), device="cuda"), q, s)
    with pytest.raises(ValueError):
        B.rms_norm_backward(x, x, s[:3], w, y)
    with pytest.raises(ValueError):
        B.rms_norm_backward(x, None, s, w, y)
