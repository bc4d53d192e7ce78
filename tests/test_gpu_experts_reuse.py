"""Operators on tokens sorted by expert over memory that is used again: lists sorted in place, buffers overwritten between calls."""
import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import expert_ref as ref
from test_gpu_experts import ok, route, run_sort, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,N", [(45001, 3, 50), (130000, 2, 7), (33, 4, 9)])
def test_sort_in_place_of_lists_that_start_anywhere(T, K, N):
    """From 131072 selections on the ids are read a second time, when rows of the same buffer are being written; lines of it belong to two warps where it
    does not start on a line."""
    ids = route(T, K, N, 3, drop=0.2)
    want, offsets = run_sort(ids, N)
    for offset in (0, 1, 13):
        flat = torch.full((offset + T * K + 32,), -9, dtype=torch.int32, device="cuda")
        mine = flat[offset:offset + T * K].view(T, K)
        mine.copy_(ids)
        again = torch.full_like(offsets, -7)
        ok(rb.remoe_expert_sort(T, K, N, mine, mine, again, stream()))
        torch.cuda.synchronize()
        assert torch.equal(mine, want) and torch.equal(again, offsets)
        assert bool((flat[:offset] == -9).all()) and bool((flat[offset + T * K:] == -9).all())
    assert torch.equal(want.cpu(), ref.sort(ids, N)[0])


@pytest.mark.parametrize("n_rows", [2, 3, 1 << 20])
def test_strides_up_to_the_limit(n_rows):
    """Rows as far apart as the header allows; no expert has any, so that none is touched."""
    far, H, I, N = (1 << 38) - 8, 64, 24, 3
    new = lambda *s: torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")
    xs, ys, d_ys, d_xs, blocks, d_blocks = new(1, H), new(1, H), new(1, H), new(1, H), new(N, I, 3, H), new(N, I, 3, H)
    act, gate_up, work = new(n_rows, I), new(2, n_rows, I), new(3, n_rows, I)
    offsets = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    ok(rb.remoe_expert_ffn(n_rows, N, H, I, rb.REMOE_BF16, xs, far, offsets, blocks, 3 * I * H, gate_up, act, ys, far, stream()))
    ok(rb.remoe_expert_ffn_backward(n_rows, N, H, I, rb.REMOE_BF16, xs, far, offsets, blocks, 3 * I * H, gate_up, d_ys, far, work, d_xs, far, d_blocks, 3 * I * H,
                                    stream()))
    torch.cuda.synchronize()
    assert not d_blocks.any() and all(bool((t == 7).all()) for t in (ys, d_xs, act, gate_up, work))
