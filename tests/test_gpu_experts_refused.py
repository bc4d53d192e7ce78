"""Memory of the host is refused whichever buffer it stands for.  (Pinned memory, which a kernel could read: a check that is not there shows as a wrong
status.)"""
import pytest
import torch

from paper_2605_27081_b200 import binding as rb
from test_gpu_experts import ok, stream

pytestmark = pytest.mark.gpu

F32, BF16 = rb.REMOE_F32, rb.REMOE_BF16


def calls(b):
    """name: (call, arguments, which of them are buffers) with buffer b() for each"""
    return {
        "sort": (rb.remoe_expert_sort, [2, 2, 4, b(), b(), b()], [3, 4, 5]),
        "dispatch": (rb.remoe_expert_dispatch, [2, 2, 8, F32, b(), 8, b(), 4, b(), 8], [4, 6, 8]),
        "combine": (rb.remoe_expert_combine, [2, 2, 8, F32, 4, b(), 8, b(), b(), b(), 8, b(), 8], [5, 7, 8, 9, 11]),
        "combine_backward": (rb.remoe_expert_combine_backward, [2, 2, 8, F32, b(), 8, 4, b(), 8, b(), b(), b(), 8, b()], [4, 7, 9, 10, 11, 13]),
        "ffn": (rb.remoe_expert_ffn, [2, 1, 8, 8, BF16, b(), 8, b(), b(), 192, b(), b(), b(), 8], [5, 7, 8, 10, 11, 12]),
        "ffn_backward": (rb.remoe_expert_ffn_backward, [2, 1, 8, 8, BF16, b(), 8, b(), b(), 192, b(), b(), 8, b(), b(), 8, b(), 192], [5, 7, 8, 10, 11, 13, 14, 16]),
    }


@pytest.mark.parametrize("name", ["sort", "dispatch", "combine", "combine_backward", "ffn", "ffn_backward"])
def test_host_memory_is_refused_in_every_place(name):
    call, args, buffers = calls(lambda: torch.zeros(4096, dtype=torch.int32, device="cuda"))[name]
    host = torch.zeros(4096, dtype=torch.int32).pin_memory()
    assert buffers == [i for i, x in enumerate(args) if torch.is_tensor(x)]
    ok(call(*args, stream()))
    torch.cuda.synchronize()
    for i in buffers:
        assert call(*args[:i], host, *args[i + 1:], stream()) == rb.REMOE_E_ARG, i
    torch.cuda.synchronize()
    assert not host.any()


def test_buffers_that_a_call_does_not_look_at_may_be_anything():
    host = torch.zeros(4096, dtype=torch.int32).pin_memory()
    d = lambda: torch.zeros(4096, dtype=torch.int32, device="cuda")
    ok(rb.remoe_expert_sort(0, 2, 4, host, host, d(), stream()))
    ok(rb.remoe_expert_dispatch(2, 2, 8, F32, d(), 8, d(), 0, host, 8, stream()))
    ok(rb.remoe_expert_combine(2, 2, 8, F32, 0, host, 8, d(), None, None, 0, d(), 8, stream()))
    ok(rb.remoe_expert_combine_backward(2, 2, 8, F32, d(), 8, 4, host, 8, d(), None, d(), 8, None, stream()))
    ok(rb.remoe_expert_ffn_backward(0, 1, 8, 8, BF16, host, 8, d(), d(), 192, host, host, 8, host, host[2048:], 8, d(), 192, stream()))
    ok(rb.remoe_expert_ffn_backward(2, 1, 8, 8, BF16, host, 8, d(), d(), 192, d(), d(), 8, d(), d(), 8, None, 0, stream()))
    torch.cuda.synchronize()
    assert not host.any()


@pytest.mark.parametrize("name", ["sort", "dispatch", "combine", "combine_backward", "ffn", "ffn_backward"])
def test_calls_from_a_thread_that_has_not_used_the_gpu(name):
    import threading
    call, args, buffers = calls(lambda: torch.zeros(4096, dtype=torch.int32, device="cuda"))[name]
    host = torch.zeros(4096, dtype=torch.int32).pin_memory()
    places = [args] + [args[:i] + [host] + args[i + 1:] for i in buffers]
    torch.cuda.synchronize()
    got = []
    for a in places:                                     # a thread for each: the first call that it makes
        t = threading.Thread(target=lambda: got.append(call(*a, None)))
        t.start()
        t.join()
    torch.cuda.synchronize()
    assert got == [0] + [rb.REMOE_E_ARG] * len(buffers)
