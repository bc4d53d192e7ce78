"""Bounded waits of the experts' products: long launches do not run into them, and what one that does run out leaves behind."""
import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import expert_ref as ref
from test_gpu_experts import ok, stream

pytestmark = pytest.mark.gpu


def test_gradient_of_blocks_behind_an_expert_of_very_many_rows():
    """The role that clears rows behind an expert's last has nothing to do for 2^28 rows and so arrives at the next expert that this pair of SMs takes
    (38 experts of two tiles for 74 pairs: the last one's belong to the first one's pairs) more than a second ahead of the products."""
    many, few, H, I, N = 1 << 28, 5, 8, 8, 38
    R = many + few
    zeros = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    xs, d_ys, gate_up, work = zeros(R, H), zeros(R, H), zeros(2, R, I), torch.empty(3, R, I, dtype=torch.bfloat16, device="cuda")
    # all rows of the first expert are zeros (which add nothing) but for some at its start, in its middle and at its end
    live = torch.cat([torch.arange(0, 40), torch.arange(many // 2 - 3, many // 2 + 30), torch.arange(many - 20, many), torch.arange(many, R)]).cuda()
    xs[live], d_ys[live] = rand(live.numel(), H), rand(live.numel(), H)
    for j in (0, 1):
        gate_up[j, live] = rand(live.numel(), I)
    offsets = torch.tensor([0] + [many] * (N - 1) + [R], dtype=torch.int32, device="cuda")
    blocks = rand(N, I, 3, H)
    d_blocks = torch.full_like(blocks, 55.0)
    ok(rb.remoe_expert_ffn_backward(R, N, H, I, rb.REMOE_BF16, xs, H, offsets, blocks, 3 * I * H, gate_up, d_ys, H, work, None, 0, d_blocks, 3 * I * H, stream()))
    torch.cuda.synchronize()
    n = live.numel()
    short = torch.tensor([0] + [n - few] * (N - 1) + [n], dtype=torch.int32, device="cuda")
    want = ref.ffn_backward(xs[live], short, blocks, gate_up[:, live], d_ys[live])["d_blocks"]
    ref.close(d_blocks, *want, "d_blocks")
