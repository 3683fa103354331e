"""Every form of the products by expert at sizes that take it (the launches' names say so), with ragged
experts, rows behind the last one, routes that are none and edges inside its tiles, against the same in
64 bits.  Tolerances as in test_gpu_grouped.py, set before any run: (K + 2) 2^-23 of the sum of the terms'
magnitudes, 2^-8 of the value as bf16, exact sums and three roundings in 8 bits."""
import pytest

pytestmark = pytest.mark.gpu

BF = 2.0 ** -8


def ragged(N, mean, seed):
    """Offsets of experts of 0, 1 and uneven numbers of rows, about `mean` on average."""
    import torch
    g = torch.Generator().manual_seed(seed)
    n = (torch.rand(N, generator=g) * 2 * mean).long()
    n[0] = 0
    if N > 2:
        n[2] = 1
    if N == 1:
        n[0] = mean
    return torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(n, 0)]).to(torch.int32).cuda()


def names(fn):
    """The library's launches during fn."""
    from paper_2606_00395_amd import binding as B
    B.profile_reset()
    B.profile_enable(True)
    fn()
    got = set(B.profile_collect())
    B.profile_enable(False)
    return got


def wanted(x, W, off, src, R):
    """out and the sums of magnitudes in 64 bits."""
    import torch
    out = torch.zeros((R, W.shape[1]), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(out)
    ends = off.tolist()
    for e in range(W.shape[0]):
        r = slice(ends[e], ends[e + 1])
        rows = x[src[r].clamp(min=0)].double() * (src[r] >= 0).unsqueeze(1)
        out[r] = rows @ W[e].double().T
        mag[r] = rows.abs() @ W[e].double().abs().T
    return out, mag


def setup(N, mean, C, K, dt, seed=0, k=3):
    """Tokens read through routes, a few of them none, and seven rows of no expert."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    off = ragged(N, mean, seed)
    R = int(off[-1]) + 7
    T = -(-R // k)
    route = torch.randperm(T * k, generator=g, device="cuda")[:R].to(torch.int32)
    route[::11] = -1
    route[5::97] = T * k
    src = torch.where((route >= 0) & (route < T * k), route // k, -1).long()
    if dt == "q8":
        x = torch.randint(-127, 128, (T, K), generator=g, device="cuda", dtype=torch.int8)
        W = torch.randint(-127, 128, (N, C, K), generator=g, device="cuda", dtype=torch.int8)
    else:
        x = torch.randn((T, K), generator=g, device="cuda").to(dt)
        W = torch.randn((N, C, K), generator=g, device="cuda").to(dt)
    return off, R, route, src, x, W, k


PRODUCTS = [
    # name, type, N, mean rows, C, K
    ("mm_thin", "bf16", 3, 30, 130, 136), ("mm_thin", "bf16", 1, 77, 1001, 1032), ("mm_thin", "bf16", 5, 40, 333, 131),
    ("mm_tile", "bf16", 16, 200, 515, 517), ("mm_tile", "bf16", 8, 500, 333, 130), ("mm_thin", "bf16", 5, 900, 135, 1001),
    ("mm_few", "bf16", 64, 40, 520, 200), ("mm_few", "bf16", 64, 45, 1001, 1032), ("mm_few", "bf16", 9, 300, 1000, 136),
    ("mm_mid", "bf16", 64, 200, 1000, 520), ("mm_mid", "bf16", 64, 210, 901, 200),
    ("mm_wide", "bf16", 16, 700, 1400, 136), ("mm_wide", "bf16", 16, 650, 1303, 520), ("mm_wide", "bf16", 3, 5000, 2000, 1032),
    # (more than 128 MiB of outputs, written past the caches)
    ("mm_wide", "bf16", 8, 4200, 2100, 72), ("mm_wide", "bf16", 8, 4200, 2101, 72),
    ("mm_thin", "f32", 3, 40, 135, 203), ("mm_tile", "f32", 8, 900, 333, 150), ("mm_tile", "f32", 1, 2100, 401, 131),
]


@pytest.mark.parametrize("gather", [True, False], ids=["plan", "sorted"])
@pytest.mark.parametrize("name,dt,N,mean,C,K", PRODUCTS, ids=["-".join(map(str, p)) for p in PRODUCTS])
def test_product(name, dt, N, mean, C, K, gather):
    import torch
    from paper_2606_00395_amd import binding as B
    D = torch.bfloat16 if dt == "bf16" else torch.float32
    off, R, route, src, x, W, k = setup(N, mean, C, K, D)
    if not gather:
        x = x[src.clamp(min=0)].contiguous()
        src = torch.arange(R, device="cuda")
    out = torch.full((R + 2, C), 9.0, dtype=D, device="cuda")
    got = names(lambda: B.grouped_mm(x, W, out[:R], offsets=off, route_of_row=route if gather else None, k=k))
    assert got == {name}
    want, mag = wanted(x, W, off, src, R)
    err = (out[:R].double() - want).abs() - (K + 2) * 2.0 ** -23 * mag
    assert (err <= (BF if dt == "bf16" else 0) * want.abs()).all()
    assert torch.all(out[R:] == 9) and not out[int(off[-1]):R].any()


QUANT = [
    ("mm_thin", 3, 30, 130, 256), ("mm_thin", 2, 41, 333, 131), ("mm_thin", 2, 20, 1001, 1032),
    ("mm_few", 64, 40, 520, 208), ("mm_few", 33, 50, 1001, 1040),
    ("mm_mid", 64, 200, 1000, 1040), ("mm_mid", 64, 210, 901, 144),
    ("mm_wide", 16, 700, 1400, 1040), ("mm_wide", 16, 900, 1303, 528), ("mm_wide", 8, 4200, 2100, 144),
    ("mm_tile", 16, 300, 700, 333), ("mm_tile", 1, 2100, 801, 1030),
]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("name,N,mean,C,K", QUANT, ids=["-".join(map(str, p)) for p in QUANT])
def test_product_in_8_bits(name, N, mean, C, K, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    off, R, route, src, x, W, k = setup(N, mean, C, K, "q8")
    g = torch.Generator(device="cuda").manual_seed(1)
    rs = torch.rand(x.shape[0], generator=g, device="cuda") + 0.1
    ws = torch.rand((N, C), generator=g, device="cuda") + 0.1
    out = torch.full((R + 2, C), 9.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    got = names(lambda: B.grouped_mm_quant(x, rs, W, ws, out[:R], offsets=off, route_of_row=route, k=k))
    assert got == {name}
    want, _ = wanted(x, W, off, src, R)
    ends = off.tolist()
    for e in range(N):
        r = slice(ends[e], ends[e + 1])
        want[r] *= rs[src[r].clamp(min=0)].double().unsqueeze(1) * ws[e].double()
    tol = (3.01 * 2.0 ** -24 + (BF if bf16 else 0)) * want.abs()
    assert ((out[:R].double() - want).abs() <= tol).all()
    assert torch.all(out[R:] == 9) and not out[int(off[-1]):R].any()


BACK = [
    ("mm_back_thin2", "bf16", 2, 8, 136, 264), ("mm_back_tile", "bf16", 4, 20, 333, 131), ("mm_back_thin", "bf16", 4, 6, 1000, 136),
    ("mm_back_thin2", "bf16", 8, 300, 520, 1000), ("mm_back_tile", "bf16", 2, 60, 333, 517),
    ("mm_back_tile", "bf16", 16, 700, 333, 517), ("mm_back_tile", "bf16", 5, 900, 1001, 135), ("mm_back_tile", "bf16", 3, 2000, 66, 1004),
   
    ("mm_back_wide", "bf16", 64, 500, 520, 1000), ("mm_back_wide", "bf16", 16, 2000, 72, 520),
    ("mm_back_wide", "bf16", 40, 900, 1048, 776),
    ("mm_back_thin", "f32", 7, 90, 135, 203), ("mm_back_tile", "f32", 16, 900, 250, 333),
]


@pytest.mark.parametrize("name,dt,N,mean,n_out,n_in", BACK, ids=["-".join(map(str, p)) for p in BACK])
def test_row_gradients(name, dt, N, mean, n_out, n_in):
    import torch
    from paper_2606_00395_amd import binding as B
    D = torch.bfloat16 if dt == "bf16" else torch.float32
    off = ragged(N, mean, 3)
    R = int(off[-1]) + 7
    g = torch.Generator(device="cuda").manual_seed(2)
    W = torch.randn((N, n_out, n_in), generator=g, device="cuda").to(D)
    dy = torch.randn((R, n_out), generator=g, device="cuda").to(D)
    dx = torch.full((R + 2, n_in), 9.0, dtype=D, device="cuda")
    got = names(lambda: B.grouped_mm_backward(dy, W, dx[:R], offsets=off))
    assert got == {name}
    want, mag = wanted(dy, W.transpose(1, 2), off, torch.arange(R, device="cuda"), R)
    err = (dx[:R].double() - want).abs() - (n_out + 2) * 2.0 ** -23 * mag
    assert (err <= (BF if dt == "bf16" else 0) * want.abs()).all()
    assert torch.all(dx[R:] == 9) and not dx[int(off[-1]):R].any()


WGRAD = [
    ({"wgrad_mfma"}, "bf16", 4, 60, 264, 136), ({"wgrad_mfma", "wgrad_join"}, "bf16", 1, 6000, 136, 264),
    ({"wgrad_mfma", "expert_order"}, "bf16", 70, 90, 520, 1000), ({"wgrad_mfma"}, "bf16", 2, 9000, 2048, 2056),
    ({"wgrad_thin"}, "f32", 7, 170, 135, 203), ({"wgrad_thin"}, "bf16", 5, 100, 133, 131),
    ({"wgrad_thin"}, "f32", 8, 700, 301, 403), ({"wgrad_tile", "wgrad_join"}, "f32", 1, 6000, 70, 130),
    ({"wgrad_tile"}, "f32", 3, 900, 901, 1003), ({"wgrad_tile"}, "bf16", 3, 900, 901, 1003),
]


@pytest.mark.parametrize("name,dt,N,mean,n_out,n_in", WGRAD, ids=["-".join(map(str, (sorted(p[0])[-1],) + p[1:])) for p in WGRAD])
def test_weight_gradients(name, dt, N, mean, n_out, n_in):
    import torch
    from paper_2606_00395_amd import binding as B
    D = torch.bfloat16 if dt == "bf16" else torch.float32
    off, R, route, src, x, _, k = setup(N, mean, 1, n_in, D, seed=4)
    g = torch.Generator(device="cuda").manual_seed(2)
    dy = torch.randn((R, n_out), generator=g, device="cuda").to(D)
    dy[int(off[-1]):] = float("nan")            # rows of no expert
    dW = torch.full((N, n_out, n_in), 9.0, device="cuda")
    got = names(lambda: B.weight_grad(dy, x, dW, offsets=off, route_of_row=route, k=k))
    assert got == name
    ends = off.tolist()
    for e in range(N):
        r = slice(ends[e], ends[e + 1])
        on = src[r] >= 0
        y, xr = dy[r][on].double(), x[src[r][on]].double()
        want, mag = y.T @ xr, y.abs().T @ xr.abs()
        assert ((dW[e].double() - want).abs() <= (y.shape[0] + 2) * 2.0 ** -23 * mag).all()


@pytest.mark.parametrize("name,dt,N,mean,C,K", [p for p in PRODUCTS if p[0] != "mm_thin"][:-4] + PRODUCTS[-2:],
                         ids=lambda v: str(v))
def test_no_number_reaches_another_row_or_column(name, dt, N, mean, C, K):
    """A NaN in two rows of x, an infinity in one row of an expert's weights, both at their first and last K, and
    rows without a source beside them."""
    import torch
    from paper_2606_00395_amd import binding as B
    D = torch.bfloat16 if dt == "bf16" else torch.float32
    off, R, route, src, x, W, k = setup(N, mean, C, K, D)
    dy = torch.randn((R, C), device="cuda").to(D)
    clean, back = torch.empty((R, C), dtype=D, device="cuda"), torch.empty((R, K), dtype=D, device="cuda")
    B.grouped_mm(x, W, clean, offsets=off, route_of_row=route, k=k)
    B.grouped_mm_backward(dy, W, back, offsets=off)
    e = N - 1
    own = torch.zeros(R, dtype=torch.bool, device="cuda")
    own[int(off[e]):int(off[e + 1])] = True
    bad_tokens = [int(src[src >= 0][0]), int(src[src >= 0][-1])]
    x[bad_tokens[0], K - 1] = x[bad_tokens[1], 0] = float("nan")
    W[e, C // 2, K - 1] = float("inf")
    W[e, C // 2, 0] = float("inf")
    rows = (src == bad_tokens[0]) | (src == bad_tokens[1])
    rows[int(off[-1]):] = False
    column = torch.zeros(C, dtype=torch.bool, device="cuda")
    column[C // 2] = True
    out = torch.empty_like(clean)
    B.grouped_mm(x, W, out, offsets=off, route_of_row=route, k=k)
    may = rows.unsqueeze(1) | (own & (src >= 0)).unsqueeze(1) & column
    assert torch.equal(out[~may], clean[~may]) and torch.isnan(out[rows]).all()
    # the rows' gradients: of those weights, columns 0 and K - 1 of the expert's rows; a NaN of dy its row
    dy[3 if N == 1 else int(off[1]) + 3, C - 1] = float("nan")
    dx = torch.empty_like(back)
    B.grouped_mm_backward(dy, W, dx, offsets=off)
    may = torch.zeros((R, K), dtype=torch.bool, device="cuda")
    may[own, 0] = may[own, K - 1] = True
    may[3 if N == 1 else int(off[1]) + 3] = True
    assert torch.equal(dx[~may], back[~may])


@pytest.mark.parametrize("C,K,mean", [(1400, 136, 700), (901, 200, 210), (333, 131, 900)], ids=["wide", "mid", "tile"])
def test_offsets_that_fall_or_overrun(C, K, mean):
    """Any offsets: no fault, nothing behind the outputs."""
    import torch
    from paper_2606_00395_amd import binding as B
    N = 16
    off, R, route, src, x, W, k = setup(N, mean, C, K, torch.bfloat16)
    dy = torch.randn((R, C), device="cuda").to(torch.bfloat16)
    g = torch.Generator().manual_seed(0)
    for t in range(4):
        o = torch.randint(-3 * R, 3 * R, (N + 1,), generator=g).to(torch.int32).cuda()
        if t == 3:
            o[::2], o[1::2] = 0, R
        out = torch.full((R + 300, C), 9.0, dtype=torch.bfloat16, device="cuda")
        dx = torch.full((R + 300, K), 9.0, dtype=torch.bfloat16, device="cuda")
        B.grouped_mm(x, W, out[:R], offsets=o, route_of_row=route, k=k)
        B.grouped_mm_backward(dy, W, dx[:R], offsets=o)
        assert torch.all(out[R:] == 9) and torch.all(dx[R:] == 9)
