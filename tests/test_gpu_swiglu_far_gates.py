"""adagc_swiglu_backward at gates far below 0, with factors whose product leaves fp32's range before the gate brings it back."""
import math

import pytest
import torch

from paper_2502_11034_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("up, d", [(2.0 ** 100, 2.0 ** 100), (-2.0 ** 80, 2.0 ** 120), (2.0 ** 120, 1.0), (2.0 ** 120, 2.0 ** -20), (2.0 ** -20, 2.0 ** 120)])
def test_gradient_of_the_gate(dtype, up, d):
    rows, cols = 3, 64
    gate = torch.tensor([-96.0, -104.0, -112.0], dtype=torch.float64)               # a checkpoint holds these as they are
    g, u, d_out = (torch.empty(rows, cols, dtype=dtype, device=DEV) for _ in range(3))
    g.copy_(gate[:, None])
    u.fill_(up)
    d_out.fill_(d)
    kept = [torch.empty(B.adagc_act8_bytes(rows, cols), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for values, ckpt in zip((g, u), kept):
        B.adagc_act8_pack(values, ckpt)
    d_gate, d_up = torch.empty_like(g), torch.empty_like(g)
    B.adagc_swiglu_backward(d_out, *kept, d_gate, d_up)
    t = torch.sigmoid(gate)
    # the sigmoid is off by 8 half steps, with bf16 2 |g| more, and six roundings; bf16's own
    off = (14 + (0 if dtype == torch.float32 else 2 * 112)) * 2.0 ** -24 + (0 if dtype == torch.float32 else 2.0 ** -8)
    for got, want in ((d_gate, d * up * t * (1 + gate)), (d_up, d * gate * t)):
        assert (want.abs() < 2.0 ** 120).all() and math.isfinite(float(want.abs().max()))
        error = (got.double().cpu() - want[:, None]).abs()
        assert (error <= off * want.abs()[:, None] + 2.0 ** -126).all()
