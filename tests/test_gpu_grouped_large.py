"""Tokens of more than 4 GiB read through the plan by the tiles that take them (rows of any alignment, 64-bit
addresses), and the weight gradient from the same tokens: as from the rows gathered before."""
import pytest

from tests.test_gpu_grouped_forms import names, ragged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,mean,C", [("mm_tile", 400, 512), ("mm_thin", 2, 96)])
@pytest.mark.parametrize("dt", ["bf16", "q8"])
def test_gathered_rows_past_4_gib(name, mean, C, dt):
    import torch
    from paper_2606_00395_amd import binding as B
    N, K, k = 8, 2048, 2
    T = (2 ** 32 + 2 ** 27) // (K * (1 if dt == "q8" else 2))
    g = torch.Generator(device="cuda").manual_seed(0)
    off = ragged(N, mean, 1)
    R = int(off[-1]) + 5
    tokens = torch.cat([torch.tensor([0, T - 1, T - 2], device="cuda"),
                        torch.randint(0, T, (R - 3,), generator=g, device="cuda")])
    route = (tokens * k + torch.randint(0, k, (R,), generator=g, device="cuda")).int()
    if dt == "q8":
        x = torch.zeros((T, K), dtype=torch.int8, device="cuda")
        x[tokens] = torch.randint(-127, 128, (R, K), generator=g, device="cuda", dtype=torch.int8)
        W = torch.randint(-127, 128, (N, C, K), generator=g, device="cuda", dtype=torch.int8)
        sx, sw = torch.rand(T, generator=g, device="cuda"), torch.rand((N, C), generator=g, device="cuda")
        product = lambda x, sx, out, **kw: B.grouped_mm_quant(x, sx, W, sw, out, offsets=off, **kw)
    else:
        x = torch.zeros((T, K), dtype=torch.bfloat16, device="cuda")
        x[tokens] = torch.randn((R, K), generator=g, device="cuda").bfloat16()
        W = torch.randn((N, C, K), generator=g, device="cuda").bfloat16()
        sx = torch.empty(T, device="cuda")
        product = lambda x, sx, out, **kw: B.grouped_mm(x, W, out, offsets=off, **kw)
    out, want = (torch.full((R, C), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert names(lambda: product(x, sx, out, route_of_row=route, k=k)) == {name}
    sorted_x = x[tokens]
    product(sorted_x, sx[tokens], want)
    if dt == "q8":
        assert torch.equal(out, want)           # (exact sums)
        return
    # (another order of the same exact products: 2 K 2^-24 of the sum of their magnitudes, and two roundings to bf16)
    for e in range(N):
        r = slice(int(off[e]), int(off[e + 1]))
        mag = sorted_x[r].float().abs() @ W[e].float().abs().T
        diff = (out[r].float() - want[r].float()).abs()
        assert (diff <= 2 * K * 2.0 ** -24 * mag + 2 * 2.0 ** -8 * want[r].float().abs() * (1 + 2.0 ** -8)).all()
    assert not out[int(off[-1]):].any()
    dy = torch.randn((R, C), generator=g, device="cuda").bfloat16()
    a, b = (torch.empty((N, C, K), device="cuda") for _ in range(2))
    B.weight_grad(dy, x, a, offsets=off, route_of_row=route, k=k)
    B.weight_grad(dy, sorted_x, b, offsets=off)
    assert torch.equal(a, b)
