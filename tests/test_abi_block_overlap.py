"""pr2_weight_grad refuses weight gradients that share memory with what they are formed from, as the products by expert
refuse their outputs; host checks, before any HIP call."""
import pytest

from paper_2606_00395_amd import binding as B
from tests.test_abi_block import FAR, READY, mm, pytestmark  # noqa: F401

# mm()'s sizes: dy [64, 48], x [32, 40], dW [4, 48, 40]
DW = 4 * 4 * 48 * 40


@pytest.mark.parametrize("dt,a", [(B.PR2_BF16, 2), (B.PR2_F32, 4)], ids=["bf16", "f32"])
@pytest.mark.parametrize("other,elements", [("dy", 64 * 48), ("x", 32 * 40)])
def test_weight_grad_refuses_overlap(other, elements, dt, a):
    at = 9 * FAR
    for dW in (at, at + a * elements - 16, at - DW + 16):
        assert mm("pr2_weight_grad", ptr={other: at, "dW": dW}, act_dtype=dt) == "PR2_ERR_SHAPE", dW - at
    for dW in (at + a * elements, at - DW):
        assert mm("pr2_weight_grad", ptr={other: at, "dW": dW}, act_dtype=dt) in READY, dW - at
