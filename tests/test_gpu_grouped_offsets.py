"""Offsets that fall or overrun in the tiles of few rows and in 8 bits: no fault, and nothing behind the outputs is
written."""
import pytest

from tests.test_gpu_grouped_forms import names, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,dt,N,mean,C,K", [("mm_few", "bf16", 64, 40, 520, 200), ("mm_few", "q8", 64, 40, 520, 400),
                                                ("mm_mid", "q8", 64, 200, 1000, 1040), ("mm_thin", "bf16", 3, 30, 130, 136)])
def test_offsets_that_fall_or_overrun(name, dt, N, mean, C, K):
    import torch
    from paper_2606_00395_amd import binding as B
    off, R, route, src, x, W, k = setup(N, mean, C, K, "q8" if dt == "q8" else torch.bfloat16)
    sx, sw = torch.rand(len(x), device="cuda"), torch.rand((N, C), device="cuda")
    g = torch.Generator().manual_seed(0)
    for t in range(5):
        o = torch.randint(-3 * R, 3 * R, (N + 1,), generator=g).to(torch.int32)
        if t >= 3:
            o[::2], o[1::2] = 0, R
        if t == 4:
            o[1] = 1
        o = o.cuda()
        out = torch.full((R + 300, C), 9.0, dtype=torch.bfloat16, device="cuda")

        def call():
            if dt == "q8":
                B.grouped_mm_quant(x, sx, W, sw, out[:R], offsets=o, route_of_row=route, k=k)
            else:
                B.grouped_mm(x, W, out[:R], offsets=o, route_of_row=route, k=k)
        assert names(call) == {name}
        assert torch.all(out[R:] == 9)
