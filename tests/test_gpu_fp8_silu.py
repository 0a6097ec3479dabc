"""SiLU(gate) * up in 32 bits: the block's scale shows it without the rounding to e4m3."""
import pytest
import torch

import rows_util as R
from paper_2603_09983_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("up", [1.0, -3.0, 1e15])
def test_silu_in_32_bits_over_the_range(up):
    """Gates from -87 to 87, one to a block, whose scale times 448 is then |silu(gate) * up|.  Off by: the
    exponential's four roundings of 2^-24, that of 1 + e, two of its reciprocal, those of the two products and of the scale's quotient: ten."""
    n = 4096
    gate = torch.linspace(-87.0, 87.0, n)
    gate = torch.where(gate.abs() < 1e-3, torch.full_like(gate, 0.5), gate)
    x = torch.zeros(n, 256)
    x[:, 5], x[:, 128 + 5] = gate, up
    q, scale = torch.empty(n, 128, dtype=torch.uint8, device="cuda"), torch.empty(n, 1, device="cuda")
    B.moe_swiglu_fp8(x.cuda(), False, None, n, 128, q, scale)
    want = (gate.double() * torch.sigmoid(gate.double()) * torch.tensor(up).double()).abs().clamp(min=2.0 ** -100)
    off = ((scale.cpu().double()[:, 0] * 448 - want).abs() / want)
    assert float(off.max()) <= 10 * R.U * (1 + 2.0 ** -20), float(off.max()) / R.U


def test_gates_beyond_the_range():
    """Infinite gates and those whose exponential is 0 or infinite: silu(g) is g, or 0; a NaN marks its block."""
    inf = float("inf")
    for gate, want in ((inf, inf), (1e30, 1e30), (200.0, 200.0), (-200.0, 2.0 ** -100), (-1e30, 2.0 ** -100), (float("nan"), float("nan"))):
        x = torch.zeros(1, 256)
        x[0, 7], x[0, 128 + 7] = gate, 1.0
        q, scale = torch.empty(1, 128, dtype=torch.uint8, device="cuda"), torch.empty(1, 1, device="cuda")
        B.moe_swiglu_fp8(x.cuda(), False, None, 1, 128, q, scale)
        assert torch.equal(scale.cpu(), torch.tensor([[want]]) / 448.0) or (gate != gate and bool(torch.isnan(scale).all())), gate
