"""Activations in 8 bits and what is computed from them, against the float64 definitions.

The packed form is compared bit for bit.  Tolerances of the rest, set before any run: the
sigmoid takes one fast exponential (relative error 2^-22 + 2^-23 |a|), one addition and one
fast reciprocal (2^-22), so silu(a) u is within 1e-6 (1 + |a|) relatively and the slope of
silu, at most 1.1 in magnitude, within 1e-6 (1 + |a|)^2; a weight gradient over K rows is
within (K + 2) 2^-23 of the sum of its terms' magnitudes; bf16 outputs add 2^-8 of the value.
"""
import numpy as np
import pytest

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu


def act(a, bf16):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if bf16 else t


def host(t):
    return t.double().cpu().numpy()


def packed_like(R, C):
    import torch
    return (torch.full((R, C), 99, dtype=torch.int8, device="cuda"),
            torch.full((R, -(-C // 32)), 77, dtype=torch.uint8, device="cuda"))


def do_pack(x):
    from paper_2606_00395_amd import binding as B
    q, e = packed_like(*x.shape)
    B.act_pack(x, q, e)
    return q, e


def values(R, C, seed=0):
    """Rows of very different sizes, zeros, subnormals and the largest numbers among them."""
    g = np.random.default_rng([seed, R, C])
    x = g.standard_normal((R, C)) * np.exp(g.normal(0, 8, (R, 1)))
    x[g.random((R, C)) < 0.05] = 0.0
    if R > 4:
        x[0] = 0.0
        x[1] *= 1e-40 / max(1e-30, np.abs(x[1]).max())
        x[2] *= 3.3e38 / max(1e-30, np.abs(x[2]).max())
        x[3] = np.where(np.arange(C) % 3 == 0, 1.999, 0.5 / 127)
    return x


SHAPES = [(1, 1), (3, 5), (7, 16), (6, 31), (9, 32), (5, 33), (8, 48), (70, 100), (4, 2049), (33, 2048),
          (2, 70003), (1030, 15), (513, 512)]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,C", SHAPES, ids=[f"{R}x{C}" for R, C in SHAPES])
def test_packed_form_bit_for_bit(R, C, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    x = act(values(R, C), bf16)
    q, e = do_pack(x)
    rq, re = O.pack(x.float().cpu().numpy())
    assert np.array_equal(e.cpu().numpy(), re)
    assert np.array_equal(q.cpu().numpy(), rq)
    back = torch.full_like(x, float("nan"))
    B.act_unpack(q, e, back)
    assert np.array_equal(host(back), O.unpack(rq, re))


def test_groups_that_are_not_finite():
    import torch
    from paper_2606_00395_amd import binding as B
    for bf16 in (True, False):
        x = act(values(9, 200, 1), bf16)
        x[5, 40], x[6, 199], x[7, 0] = float("nan"), float("inf"), float("-inf")
        q, e = do_pack(x)
        rq, re = O.pack(x.float().cpu().numpy())
        assert np.array_equal(e.cpu().numpy(), re) and np.array_equal(q.cpu().numpy(), rq)
        back = torch.empty_like(x)
        B.act_unpack(q, e, back)
        bad = np.isnan(host(back))
        assert bad[5, 32:64].all() and bad[6, 192:].all() and bad[7, :32].all() and bad.sum() == 32 + 8 + 32


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,m", [(1, 1), (3, 7), (5, 16), (4, 32), (130, 48), (65, 96), (17, 333), (9, 1408),
                                 (300, 768), (2, 40001)])
def test_swiglu_and_its_backward(R, m, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    g = np.random.default_rng([R, m])
    au = act(np.concatenate([g.normal(0, 4, (R, m)), g.normal(0, 1, (R, m))], 1), bf16)
    au[0, 0] = -100.0 if m > 1 else 2.0
    dh = act(g.standard_normal((R, m)), bf16)
    h, hb, dau = torch.full_like(dh, float("nan")), torch.full_like(dh, float("nan")), torch.full_like(au, float("nan"))
    q, e = packed_like(R, 2 * m)
    B.swiglu_pack(au, h, q, e)
    rq, re = O.pack(au.float().cpu().numpy())
    assert np.array_equal(e.cpu().numpy(), re) and np.array_equal(q.cpu().numpy(), rq)
    half = 2.0 ** -8 if bf16 else 0.0
    a, u, d = host(au)[:, :m], host(au)[:, m:], host(dh)
    want = O.swiglu(a, u)
    assert np.all(np.abs(host(h) - want) <= (1e-6 * (1 + np.abs(a)) + half) * np.abs(want) + 1e-37)

    B.swiglu_backward_packed(q, e, dh, dau, hb)
    v = O.unpack(rq, re)
    a, u = v[:, :m], v[:, m:]
    da, du, want = O.swiglu_backward(a, u, d)
    got = host(dau)
    s = 1e-6 * (1 + np.abs(a))
    assert np.all(np.abs(host(hb) - want) <= (s + half) * np.abs(want) + 1e-37)
    assert np.all(np.abs(got[:, m:] - du) <= (s + half) * np.abs(du) + 1e-37)
    assert np.all(np.abs(got[:, :m] - da) <= s * (1 + np.abs(a)) * np.abs(d * u) + half * np.abs(da) + 1e-37)
    again = torch.full_like(dau, float("nan"))
    B.swiglu_backward_packed(q, e, dh, again)           # without h
    assert torch.equal(again, dau)


def check_wgrad(dy, x, offsets=None, route=None, k=1, N=1):
    import torch
    from paper_2606_00395_amd import binding as B
    q, e = do_pack(x)
    dW = torch.full((N, dy.shape[1], x.shape[1]), float("nan"), device="cuda")
    B.weight_grad_packed(dy, q, e, dW, offsets=offsets, route_of_row=route, k=k)
    v = O.unpack(*O.pack(x.float().cpu().numpy()))
    off = None if offsets is None else offsets.cpu().numpy()
    want, mag = O.weight_grad(host(dy), v, off, None if route is None else route.cpu().numpy(), k)
    rows = dy.shape[0] if off is None else int(max(np.diff(off)))
    err = np.abs(host(dW) - want)
    assert np.all(err <= (rows + 2) * 2.0 ** -23 * mag + 1e-37), (err - (rows + 2) * 2.0 ** -23 * mag).max()
    return dW


LINEAR = [(1, 1, 1), (2, 8, 16), (3, 70, 33), (31, 256, 256), (32, 264, 272), (33, 8, 512), (100, 135, 203),
          (257, 520, 48), (1000, 256, 512), (2049, 64, 96), (130, 1032, 1040), (5000, 300, 260), (640, 2048, 64)]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,n_out,n_in", LINEAR, ids=["x".join(map(str, c)) for c in LINEAR])
def test_weight_gradient_of_one_layer(R, n_out, n_in, bf16):
    g = np.random.default_rng([R, n_out, n_in])
    check_wgrad(act(g.standard_normal((R, n_out)), bf16), act(g.standard_normal((R, n_in)), bf16))


# T, N, k, n_out, n_in, dropped: experts without rows, with one row, with several hundred
EXPERTS = [(1, 4, 1, 16, 32, 0.0), (5, 40, 3, 256, 256, 0.3), (40, 3, 2, 64, 96, 0.0), (300, 5, 2, 520, 272, 0.1),
           (700, 8, 4, 264, 512, 0.0), (500, 1, 1, 512, 288, 0.0), (64, 60, 4, 1536, 256, 0.0), (333, 7, 3, 135, 203, 0.2)]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", EXPERTS, ids=["x".join(map(str, c)) for c in EXPERTS])
def test_weight_gradients_of_experts(case, bf16):
    import torch
    T, N, k, n_out, n_in, drop = case
    g = np.random.default_rng(case[:5])
    # a load as uneven as a hot expert makes it
    w = np.exp(g.normal(0, 1.5, N))
    idx = np.stack([g.choice(N, k, replace=False, p=w / w.sum()) for _ in range(T)])
    idx = np.where(g.random((T, k)) < drop, -1, idx)
    off, _, route = O.dispatch_plan(idx, N)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    dy = g.standard_normal((T * k, n_out))
    dy[off[-1]:] = np.nan                               # rows of no expert are not read
    dW = check_wgrad(act(dy, bf16), act(g.standard_normal((T, n_in)), bf16), i32(off), i32(route), k, N)
    empty = np.nonzero(np.diff(off) == 0)[0]
    assert torch.all(dW[torch.from_numpy(empty).cuda()] == 0)


def test_many_experts_and_long_ones():
    """1024 experts in 6144 tiles (two column tiles per workgroup), one expert with more rows
    than a workgroup holds the indexes of, one with none; sampled experts against float64."""
    import torch
    from paper_2606_00395_amd import binding as B
    N, n_out, n_in, T = 1024, 264, 528, 1500
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = torch.randint(0, 6, (N,), generator=g, device="cuda")
    rows[7], rows[8], rows[1023] = 17000, 0, 33
    R = int(rows.sum())
    off = torch.cat([rows.new_zeros(1), rows.cumsum(0)]).to(torch.int32)
    route = torch.randint(0, 2 * T, (R,), generator=g, device="cuda", dtype=torch.int32)
    dy = torch.randn((R, n_out), generator=g, device="cuda").to(torch.bfloat16)
    x = torch.randn((T, n_in), generator=g, device="cuda").to(torch.bfloat16)
    q, e = do_pack(x)
    dW = torch.full((N, n_out, n_in), float("nan"), device="cuda")
    B.weight_grad_packed(dy, q, e, dW, offsets=off, route_of_row=route, k=2)
    v = torch.empty_like(x)
    B.act_unpack(q, e, v)
    ends = off.tolist()
    for i in [0, 1, 2, 6, 7, 8, 9, 500, 1022, 1023]:
        a = dy[ends[i]:ends[i + 1]].double()
        b = v[(route[ends[i]:ends[i + 1]] // 2).long()].double()
        want, mag = a.T @ b, a.abs().T @ b.abs()
        assert torch.all((dW[i].double() - want).abs() <= (len(a) + 2) * 2.0 ** -23 * mag + 1e-37), i
    assert torch.isfinite(dW).all() and torch.all(dW[8] == 0)
    again = torch.empty_like(dW)
    B.weight_grad_packed(dy, q, e, again, offsets=off, route_of_row=route, k=2)
    assert torch.equal(again, dW)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_weight_gradient_over_many_rows(bf16):
    """Slices of the rows, each in several parts, and their join; an odd number of outputs."""
    import torch
    from paper_2606_00395_amd import binding as B
    for R, n_out, n_in in ((70001, 248, 240), (20011, 77, 35)):
        g = torch.Generator(device="cuda").manual_seed(R)
        dt = torch.bfloat16 if bf16 else torch.float32
        dy = torch.randn((R, n_out), generator=g, device="cuda").to(dt)
        x = torch.randn((R, n_in), generator=g, device="cuda").to(dt)
        q, e = do_pack(x)
        v = torch.empty_like(x)
        B.act_unpack(q, e, v)
        dW = torch.full((1, n_out, n_in), float("nan"), device="cuda")
        B.weight_grad_packed(dy, q, e, dW)
        want, mag = dy.double().T @ v.double(), dy.double().abs().T @ v.double().abs()
        # (sums of slices: the longest chain is shorter than R)
        assert torch.all((dW[0].double() - want).abs() <= 2.0 ** -23 * 2000 * mag)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_rows_without_a_source_add_nothing(bf16):
    import torch
    g = np.random.default_rng(3)
    R, T, k = 100, 50, 2
    route = g.integers(0, T * k, R)
    route[10], route[40], route[99], route[5] = -1, T * k, 2 ** 31 - 1, -2 ** 31
    dy = g.standard_normal((R, 264))
    dy[[10, 40, 99, 5]] = np.inf
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    from paper_2606_00395_amd import binding as B
    x = act(g.standard_normal((T, 288)), bf16)
    q, e = do_pack(x)
    dW = torch.empty((1, 264, 288), device="cuda")
    B.weight_grad_packed(act(dy, bf16), q, e, dW, offsets=i32([0, R]), route_of_row=i32(route), k=k)
    keep = np.ones(R, bool)
    keep[[10, 40, 99, 5]] = False
    dyh = host(act(dy, bf16))
    v = O.unpack(*O.pack(x.float().cpu().numpy()))
    want, mag = O.weight_grad(dyh[keep], v, [0, keep.sum()], route[keep], k)
    assert np.all(np.abs(host(dW) - want) <= (R + 2) * 2.0 ** -23 * mag)


def test_infinite_gradients_stay_in_their_rows_and_columns():
    """An infinity in one row and column of dy reaches that output row alone, with the
    sign of its products; padding of tiles and of the last step adds no NaN."""
    import torch
    from paper_2606_00395_amd import binding as B
    for bf16 in (True, False):
        g = np.random.default_rng(4)
        dy = act(g.standard_normal((77, 272)), bf16)
        dy[76, 271] = float("inf")
        x = act(np.abs(g.standard_normal((77, 304))) + 0.1, bf16)
        q, e = do_pack(x)
        dW = torch.empty((1, 272, 304), device="cuda")
        B.weight_grad_packed(dy, q, e, dW)
        assert torch.isinf(dW[0, 271]).all() and torch.isfinite(dW[0, :271]).all()


def test_no_rows_give_zeros():
    import torch
    from paper_2606_00395_amd import binding as B
    dW = torch.full((3, 8, 64), 5.0, device="cuda")
    dy = torch.empty((0, 8), dtype=torch.bfloat16, device="cuda")
    q, e = packed_like(0, 64)
    B.weight_grad_packed(dy, q, e, dW, offsets=torch.zeros(4, dtype=torch.int32, device="cuda"),
                         route_of_row=torch.empty(0, dtype=torch.int32, device="cuda"), k=2)
    assert torch.all(dW == 0)
    B.act_pack(torch.empty((0, 64), device="cuda"), q, e)


def test_offsets_past_two_to_the_31():
    """Packed and unpacked elements at indexes above 2^31, weight gradients of rows there."""
    import torch
    from paper_2606_00395_amd import binding as B
    R, C = 2 ** 20 + 77, 2080
    assert R * C > 2 ** 31
    x = torch.zeros((R, C), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    tail = torch.randn((64, C), generator=g, device="cuda").to(torch.bfloat16)
    x[-64:] = tail
    q, e = do_pack(x)
    tq, te = do_pack(tail)
    assert torch.equal(q[-64:], tq) and torch.equal(e[-64:], te) and not q[:-64].any()
    B.act_unpack(q, e, x)
    small = torch.empty_like(tail)
    B.act_unpack(tq, te, small)
    assert torch.equal(x[-64:], small)
    # the last rows alone have an expert
    dy = torch.randn((64, 72), generator=g, device="cuda").to(torch.bfloat16)
    route = torch.arange(R - 64, R, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    a, b = torch.empty((1, 72, C), device="cuda"), torch.empty((1, 72, C), device="cuda")
    B.weight_grad_packed(dy, q, e, a, offsets=off, route_of_row=route)
    B.weight_grad_packed(dy, tq, te, b)
    assert torch.equal(a, b)


def test_another_stream_and_graph_replays():
    import torch
    from paper_2606_00395_amd import binding as B
    T, N, k, d, m = 400, 6, 2, 256, 128
    g = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.topk(torch.randn((T, N), generator=g, device="cuda"), k).indices.to(torch.int32).contiguous()
    off, _, route = (torch.from_numpy(a.astype(np.int32)).cuda() for a in O.dispatch_plan(ids.cpu().numpy(), N))
    x, au, dh = rnd(T, d), rnd(T * k, 2 * m), rnd(T * k, m)
    q, e = packed_like(T, d)
    qa, ea = packed_like(T * k, 2 * m)
    h, dau, hb = torch.empty_like(dh), torch.empty_like(au), torch.empty_like(dh)
    dW = torch.empty((N, 2 * m, d), device="cuda")
    outs = (q, e, qa, ea, h, dau, hb, dW)

    def step(st=None):
        B.act_pack(x, q, e, stream=st)
        B.swiglu_pack(au, h, qa, ea, stream=st)
        B.swiglu_backward_packed(qa, ea, dh, dau, hb, stream=st)
        B.weight_grad_packed(dau, q, e, dW, offsets=off, route_of_row=route, k=k, stream=st)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), rep
        B.act_pack(torch.roll(x, 1, 0), *packed_like(T, d))
        torch.cuda.synchronize()


def test_refusals_of_the_binding():
    import torch
    from paper_2606_00395_amd import binding as B
    x = torch.zeros((4, 64), device="cuda")
    q, e = packed_like(4, 64)
    with pytest.raises(TypeError):
        B.act_pack(x.half(), q, e)
    with pytest.raises(ValueError):
        B.act_pack(x, q, e[:, :1])
    with pytest.raises(TypeError):
        B.act_pack(x, q.to(torch.uint8), e)
    with pytest.raises(ValueError):
        B.act_pack(x[:, ::2], *packed_like(4, 32))
    with pytest.raises(ValueError):
        B.swiglu_pack(torch.zeros((4, 63), device="cuda"), x, q, e)
    with pytest.raises(ValueError):
        B.weight_grad_packed(x, q, e, torch.zeros((2, 64, 64), device="cuda"))
    with pytest.raises(B.Pr2Error, match="R = 8"):
        B.weight_grad_packed(torch.zeros((8, 4), device="cuda"), q, e, torch.zeros((1, 4, 64), device="cuda"))


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_out,n_in", [(3, 5), (63, 7), (65, 8), (9, 9), (1, 15), (71, 33), (8, 66), (130, 71)])
def test_weight_gradients_at_the_edges_of_narrow_tiles(n_out, n_in, bf16):
    """Rows shorter than a thread's piece, pieces that end outside the row, dropped routes and
    rows past the last expert's."""
    import torch
    T, N, k = 90, 3, 2
    g = np.random.default_rng([n_out, n_in])
    idx = np.sort(np.stack([g.choice(N, k, replace=False) for _ in range(T)]), 1)
    idx[g.random((T, k)) < 0.2] = -1
    from paper_2606_00395_amd import binding as B
    i32 = dict(dtype=torch.int32, device="cuda")
    offsets, row, route = torch.empty(N + 1, **i32), torch.empty((T, k), **i32), torch.empty(T * k, **i32)
    B.dispatch_plan(torch.from_numpy(idx.astype(np.int32)).cuda(), N, offsets, row, route)
    assert int(offsets[N]) < T * k
    check_wgrad(act(g.standard_normal((T * k, n_out)), bf16), act(g.standard_normal((T, n_in)), bf16),
                offsets, route, k, N)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,n_out,n_in,N", [(20000, 8, 16, 1), (9973, 24, 48, 1), (6001, 40, 32, 5), (900, 520, 272, 2),
                                            (300, 264, 512, 9)])
def test_weight_gradients_in_many_slices_and_of_few_experts(R, n_out, n_in, N, bf16):
    """Small outputs over many rows, the rows of an expert in up to 64 slices (some empty where
    another expert has most of the rows), and experts whose tiles go to all XCDs."""
    import torch
    g = np.random.default_rng([R, n_out, N])
    offsets = None
    if N > 1:
        cuts = np.sort(g.integers(0, R // 3, N - 1))        # the last one has most
        offsets = torch.from_numpy(np.concatenate([[0], cuts, [R]]).astype(np.int32)).cuda()
    check_wgrad(act(g.standard_normal((R, n_out)), bf16), act(g.standard_normal((R, n_in)), bf16), offsets, N=N)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,n_out,n_in", [(70, 264, 272), (70, 135, 203), (300, 8, 64)])
@pytest.mark.parametrize("top,slope", [(3.3e38, 1e-30), (1e-38, 1e30)], ids=["largest", "smallest"])
def test_weight_gradients_of_the_largest_and_smallest_groups(top, slope, R, n_out, n_in, bf16):
    """Groups at both ends of the scale's range, zeros among their values: every value is a
    finite number, and the sums of products that are finite stay so, at every width."""
    g = np.random.default_rng([R, n_out, n_in])
    x = g.uniform(-1, 1, (R, n_in)) * top
    x[g.random((R, n_in)) < 0.3] = 0.0
    scale = O.pack(act(x, bf16).float().cpu().numpy())[1]
    assert np.any(scale == (248 if top > 1 else 1))
    check_wgrad(act(g.standard_normal((R, n_out)) * slope, bf16), act(x, bf16))


def test_as_many_rows_as_are_allowed():
    """2^31 - 1 rows: the first and last ones as packed alone, the others zeros."""
    import torch
    from paper_2606_00395_amd import binding as B
    R, n = 2 ** 31 - 1, 700
    x = torch.zeros((R, 1), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    for sl in (slice(0, n), slice(R - n, R)):
        x[sl] = torch.randn((n, 1), generator=g, device="cuda").to(torch.bfloat16)
    q = torch.full((R, 1), 99, dtype=torch.int8, device="cuda")
    e = torch.full((R, 1), 77, dtype=torch.uint8, device="cuda")
    B.act_pack(x, q, e)
    for sl in (slice(0, n), slice(R - n, R)):
        sq, se = do_pack(x[sl].clone())
        assert torch.equal(q[sl], sq) and torch.equal(e[sl], se)
    for r in range(n, R - n, 2 ** 28):      # (in parts: the comparisons take memory too)
        sl = slice(r, min(r + 2 ** 28, R - n))
        assert not q[sl].any() and torch.all(e[sl] == 1)
    x.fill_(float("nan"))
    B.act_unpack(q, e, x)
    for sl in (slice(0, n), slice(R - n, R)):
        back = torch.full((n, 1), float("nan"), dtype=torch.bfloat16, device="cuda")
        B.act_unpack(q[sl].clone(), e[sl].clone(), back)
        assert torch.equal(x[sl], back)
    for r in range(n, R - n, 2 ** 28):
        assert not x[r:min(r + 2 ** 28, R - n)].any()


def test_one_workspace_for_batches_up_to_the_largest():
    """A workspace made for 5000 rows serves every smaller batch, also those in more slices."""
    import torch
    from paper_2606_00395_amd import binding as B
    g = np.random.default_rng(9)
    dy, x = act(g.standard_normal((5000, 512)), True), act(g.standard_normal((5000, 512)), True)
    q, e = do_pack(x)
    ws = B.weight_grad_workspace(dy, q)
    for R in (5000, 2000, 480, 479, 448, 30, 1):
        a, b = (torch.full((1, 512, 512), float("nan"), device="cuda") for _ in range(2))
        B.weight_grad_packed(dy[:R], q[:R], e[:R], a, ws=ws)
        B.weight_grad_packed(dy[:R], q[:R], e[:R], b)
        assert torch.equal(a, b) and torch.isfinite(a).all(), R


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_distance_of_the_packed_values(bf16):
    """Half a step of 1/128 to 1/64 of the group's largest magnitude, which is not exact itself;
    a whole one for fp32 magnitudes that are cut."""
    import torch
    from paper_2606_00395_amd import binding as B
    g = np.random.default_rng(10)
    x = g.uniform(-1, 1, (200, 96)) * np.exp(g.normal(0, 20, (200, 1)))
    for r, v in enumerate((1.0078125, 1.9921875, 1.9999, 1.0)):       # every 8-bit and a 24-bit mantissa's ends
        x[r] = np.where(np.arange(96) % 32 == r, v, v / 3)
    x[4] = 2.0 ** -127
    x = act(x, bf16)
    q, e = do_pack(x)
    back = torch.empty_like(x)
    B.act_unpack(q, e, back)
    v, step = host(x), np.repeat(np.exp2(e.double().cpu().numpy() - 127), 32, axis=1)
    top = np.repeat(np.abs(v).reshape(200, 3, 32).max(2), 32, axis=1)
    assert np.all((step >= top / 128) & ((step <= top / 64) | (step == 2.0 ** -126)))
    off = np.abs(host(back) - v) / step
    cut = np.abs(v) > 127.5 * step
    assert np.all(off[~cut] <= 0.5) and np.all(off[cut] < 1) and (not bf16 or not cut.any())
    assert host(back)[0, 0] == 1.0 and host(back)[1, 1] == 1.984375
