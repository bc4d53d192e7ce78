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
