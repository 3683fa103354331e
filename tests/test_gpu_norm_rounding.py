"""y and rstd of the norm are the values of the definition, rounded: no sum or product before the last
rounding is off by as much as a step of fp32, at any row length and in every form.

Window, set before any run.  Squares of fp32 values are exact in 64 bits, a row's sum of them has at most 55 roundings of
2^-53 in a row, the mean, eps and the root a few more (halved by the root), the two products one each: below 2^-47
relatively, and the reference in 64 bits the same again.  So the result is the rounding to fp32 (then to bf16) of
a value within 2^-46 of the reference's.
"""
import numpy as np
import pytest

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu

W = 2.0 ** -46
SHAPES = [(1, 1), (3, 3), (8, 33), (70, 333), (5, 1021), (8, 2048), (300, 2048), (2600, 513), (2600, 2048), (4200, 2048),
          (17, 4096), (2100, 4100), (6, 8200), (3, 16388), (2, 32767), (2, 32768)]


def between(got, want, bf16):
    """Whether got is the rounding of a value within W of want."""
    import torch

    def rounded(v):
        with np.errstate(over="ignore"):
            t = torch.from_numpy(v.astype(np.float32))
        return (t.to(torch.bfloat16) if bf16 else t).double().numpy()
    a, b = rounded(want * (1 - W)), rounded(want * (1 + W))
    return (got == a) | (got == b)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES, ids=[f"{T}x{d}" for T, d in SHAPES])
def test_rounded_once(T, d, bf16):
    check(T, d, bf16, 1.0)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(5, 40), (5, 2048), (2600, 300), (5, 9000)])
@pytest.mark.parametrize("size", [2.0 ** 80, 2.0 ** -90])
def test_rows_whose_squares_pass_fp32s_range(T, d, size, bf16):
    check(T, d, bf16, size, 1e-50)


def check(T, d, bf16, most, eps=1e-6):
    """One row of them `most` times as large as the others."""
    import torch
    from paper_2606_00395_amd import binding as B
    dt = torch.bfloat16 if bf16 else torch.float32
    g = np.random.default_rng([T, d])

    def rows(s):
        x = g.standard_normal((T, d)) * s
        x[:, ::97] *= 20
        return torch.from_numpy(x.astype(np.float32)).cuda().to(dt)
    size = np.exp(g.normal(0, 3, (T, 1)))
    size[T // 2] *= most
    x, res = rows(size), rows(np.where(size < 2.0 ** -60, 0.0, 1.0))
    w = (1 + 0.3 * g.standard_normal(d)).astype(np.float32)
    wt = torch.from_numpy(w).cuda()
    for residual in (res, None):
        y, h, r = torch.empty_like(x), torch.empty_like(x), torch.empty(T, device="cuda")
        q, e = torch.empty((T, d), dtype=torch.int8, device="cuda"), torch.empty((T, -(-d // 32)), dtype=torch.uint8, device="cuda")
        B.rms_norm(x, wt, y, residual=residual, h_out=h, rstd_out=r, q=q, scale=e, eps=eps)
        h64 = h.double().cpu().numpy()
        want, rstd = O.rms_norm(h64, w.astype(np.float64), np.float64(np.float32(eps)))
        ok = between(y.double().cpu().numpy(), want, bf16)
        assert ok.all(), f"{np.count_nonzero(~ok)} of {ok.size} are not the rounded value"
        assert between(r.double().cpu().numpy(), rstd, False).all()
        # and the packed form that of the rounded value
        a, b = torch.empty_like(q), torch.empty_like(e)
        B.act_pack(y, a, b)
        assert torch.equal(a, q) and torch.equal(b, e)
