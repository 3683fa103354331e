"""The norm under weights of any size, against y = round(h r w) in 64 bits.

Tolerance, set before any run: that of test_gpu_norm.py, 36 2^-24 of y and 2^-8 as bf16, where y is a number of fp32;
an infinity of y's sign above its range, and what h r w is in 64 bits where a weight is infinite.
"""
import numpy as np
import pytest

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(5, 29), (5, 300), (5, 2048), (2050, 1500), (5, 5000)])
def test_weights_of_any_size(T, d, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    g = np.random.default_rng(d)
    size = np.resize([1e-17, 1e17, 1.0, 3e-10, 3e10], T)
    x = torch.from_numpy((g.standard_normal((T, d)) * size[:, None]).astype(np.float32)).cuda()
    x = x.to(torch.bfloat16) if bf16 else x
    x[2, 0] = x[3, 7] = 0
    w = np.asarray(1 + 0.3 * g.standard_normal(d), dtype=np.float32)
    w[:16] = [np.inf, -np.inf, 1e22, -1e25, 1e30, 2e35, -1e-25, 1e-30, 1e-22, 1e-20, -1e-37, 0, 1e38, 1e15, 1e-15, np.inf]
    y, wt = torch.empty_like(x), torch.from_numpy(w).cuda()
    B.rms_norm(x, wt, y, eps=0.0)
    got = y.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want, _ = O.rms_norm(x.double().cpu().numpy(), w.astype(np.float64), 0.0)
        edge = (np.abs(want) > 3.3e38) & (np.abs(want) < 3.5e38)
        want = np.where(np.abs(want) >= 3.5e38, np.sign(want) * np.inf, want)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        number = np.isfinite(want) & ~edge
        off = np.abs(got - want) - (36 * U + (BF if bf16 else 0)) * np.abs(want) - 2.0 ** -133
        assert np.all(off[number] <= 0)
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
