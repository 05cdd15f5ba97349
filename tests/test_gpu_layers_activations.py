"""Activations of the hidden layers on the GPU: infinite arguments, and how exact GELU is in float32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_35099_b200 as e3j

pytestmark = pytest.mark.gpu
SILU, TANH, GELU = e3j.E3J_ACT_SILU, e3j.E3J_ACT_TANH, e3j.E3J_ACT_GELU
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act,low,high", [(0, -INF, INF), (SILU, NAN, INF), (TANH, -1.0, 1.0), (GELU, NAN, INF)])
def test_infinite_arguments(act, low, high, dtype):
    """z = infinity by way of the bias: what the formulas give (silu and gelu of -infinity are -infinity times 0)."""
    want = torch.tensor([high, low, NAN], device="cuda")
    for n in (3, 64, 200):
        b = torch.zeros(n, dtype=dtype, device="cuda")
        b[:3] = torch.tensor([INF, -INF, NAN], device="cuda")
        x, W = torch.randn(300, 16, device="cuda").to(dtype), torch.randn(16, n, device="cuda").to(dtype)
        for y in (e3j.e3j_linear_fwd(x, W, b, act=act), e3j.e3j_layer_norm_fwd(torch.randn(300, n, device="cuda").to(dtype), None, b, act=act)):
            assert torch.equal(y[:, :3].float().nan_to_num(nan=7.0), want.expand(300, 3).nan_to_num(nan=7.0)), (n, y[0, :3])
            assert torch.isfinite(y[:, 3:].float()).all()
