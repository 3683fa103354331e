"""The row form of silu(a) u: the values themselves, read from rows of one element, whose scale is
fp32(|v| fp32(1 / 127)).

Tolerance, set before any run: v = a / (1 + exp(-a)) u.  The exponential is within one last place (2 2^-24 relatively) and
its share of 1 + exp(-a) is below 1; the sum, the quotient, the product with u and the one with fp32(1 / 127) are
one rounding of 2^-24 each: 6 2^-24, and 2^-46 for their products.  Nothing in it grows with |a|.
"""
import numpy as np
import pytest

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("lo,hi", [(-1, 1), (-8, 8), (-40, -8), (-80, -40), (8, 300)])
def test_values(lo, hi, bf16):
    import torch
    from paper_2606_00395_amd import binding as B
    R = 50000
    g = np.random.default_rng([lo + 100, hi + 100])
    au = np.stack([g.uniform(lo, hi, R), g.choice([-1, 1], R) * g.uniform(1, 2, R) * 2.0 ** g.integers(0, 30, R)], 1)
    au = torch.from_numpy(au.astype(np.float32)).cuda()
    au = au.to(torch.bfloat16) if bf16 else au
    q, s = torch.full((R, 1), 99, dtype=torch.int8, device="cuda"), torch.empty(R, device="cuda")
    B.swiglu_quant(au, q, s)
    a, u = au[:, 0].double().cpu().numpy(), au[:, 1].double().cpu().numpy()
    v = O.swiglu(a, u)
    seen = np.abs(v) > 2.0 ** -99           # (smaller rows have the least scale)
    want = np.abs(v) * np.float64(np.float32(1) / np.float32(127))
    got = s.double().cpu().numpy()
    assert np.all(np.abs(got - want)[seen] <= (6 * U + 2.0 ** -46) * want[seen])
    assert np.array_equal(q.cpu().numpy()[seen, 0], 127 * np.sign(v[seen]))
