"""Bounded waits of the experts' products: long launches do not run into them, and what one that does run out leaves behind."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import expert_ref as ref
from test_gpu_experts import Ffn, ok, stream

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


def lost_copies(counts, H, I, dtype):
    """In a process with REMOE_FAULT_INJECT=lost_product_copy: of four calls the first waits for a copy of an operand that does not come, in each of its
    launches, and the third for one of kept values.  They return, and what they leave is NaN or right; the calls behind them are right."""
    f = Ffn(counts, H, I, dtype, seed=H + I)

    def four(call, outputs):
        got = []
        for _ in range(4):
            for t in outputs + [f.work]:
                t.fill_(55.0)
            call()
            got.append([t.clone() for t in outputs])
        for lost in (0, 2):
            for a, b in zip(got[lost], got[1]):
                assert bool((torch.isnan(a) | (a == b)).all())
        assert all(torch.equal(a, b) for a, b in zip(got[1], got[3]))
        return [[bool(torch.isnan(t).any()) for t in g] for g in got]

    nan = four(f.forward, [f.ys.view, f.act, f.gate_up])
    assert nan[0] == [True] * 3 and nan[1] == [False] * 3
    want = ref.ffn(f.xs.view, f.offsets, f.blocks)
    ref.close(f.ys.view, *want["ys"], "ys")
    nan = four(f.backward, [f.d_xs.view, f.d_blocks])
    assert nan[0] == [True] * 2 and nan[2] == [True] * 2 and nan[1] == [False] * 2
    want = ref.ffn_backward(f.xs.view, f.offsets, f.blocks, f.gate_up, f.d_ys.view)
    ref.close(f.d_xs.view, *want["d_xs"], "d_xs")
    ref.close(f.d_blocks, *want["d_blocks"], "d_blocks")


# more tiles than pairs of SMs hold results of, rows to clear in the first expert; none to clear there; tiles shared by clusters
LOST = [([300] * 8, 64, 4096, "bf16"), ([320, 7, 512], 136, 264, "f16"), ([40], 2048, 1544, "bf16")]


def test_a_wait_that_runs_out_leaves_nan_and_the_next_call_is_right():
    here = os.path.dirname(os.path.abspath(__file__))
    code = "import test_gpu_experts_waits as t\nfor case in t.LOST: t.lost_copies(*case)\nprint('as it should be')"
    env = dict(os.environ, REMOE_FAULT_INJECT="lost_product_copy", PYTHONPATH=os.pathsep.join([here, os.path.dirname(here)]))
    res = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "as it should be" in res.stdout, res.stdout + res.stderr[-3000:]
