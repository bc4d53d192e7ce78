"""silu and its derivative at gates far from zero, through products that are exact."""
import pytest
import torch

import expert_ref as ref
from test_gpu_experts import Ffn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("up", [1.0, 2.0 ** 100])
def test_silu_of_far_gates(up):
    """A row (1, 0, ...) takes gates and ups from the first column of the weights as they are; the gradient (1, 0, ...) does the same for d act = 1.
    silu(g) u is a normal number of bfloat16 for all of them with the larger u.  Bound: the rounding to the type, (2 + 1.16 |g|) 2^-23 and two more steps of the
    fast exponential and division, a step of 2^-149 of exp(g) where it is subnormal."""
    gates = torch.tensor([0.0, 1.0, -1.0, 20.0, -20.0, 60.0, -60.0, 86.0, -86.0, -87.0, -87.5, 88.0, -88.0, -88.5, -89.0, -90.0, -92.0, -93.0, 100.0, 1000.0, 32768.0,
                          -0.0078125, 0.0078125, -5.0], dtype=torch.float64, device="cuda")
    f = Ffn([2], 8, gates.numel(), "bf16", seed=1)
    f.xs.view.zero_(), f.d_ys.view.zero_(), f.blocks.zero_()
    f.xs.view[:, 0], f.d_ys.view[:, 0] = 1.0, 1.0
    f.blocks[0, :, 0, 0], f.blocks[0, :, 1, 0], f.blocks[0, :, 2, 0] = gates.bfloat16(), up, 1.0
    assert torch.equal(f.blocks[0, :, 0, 0].double(), gates)
    f.forward(), f.backward()
    e = torch.exp(-gates.abs())
    s = torch.where(gates < 0, e, torch.ones_like(e)) / (1 + e)
    off = (4 + 1.16 * gates.abs()) * 2.0 ** -23 + 2.0 ** -149 / torch.exp(gates.clamp(max=0))
    close = lambda got, want, size, what: [ref.close(row, want, ref.half(torch.bfloat16) * want.abs() + off * size + ref.tiny(torch.bfloat16), what) for row in got]
    act = gates * s * up
    close(f.act, act, act.abs(), "act")
    slope = s * (1 + gates * (1 - s))
    close(f.work[0], slope * up, s * (1 + gates.abs() * (1 - s)) * up, "d gate")
    close(f.work[1], gates * s, (gates * s).abs(), "d up")
    close(f.work[2], act, act.abs(), "a")
