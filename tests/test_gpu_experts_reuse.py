"""Operators on tokens sorted by expert over memory that is used again: lists sorted in place, buffers overwritten between calls."""
import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import expert_ref as ref
from test_gpu_experts import NAN, ok, route, run_sort, stream
from test_gpu_experts_layer import Layer

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


def poison(m):
    """Whatever a layer's calls write: NaN in matrices, -7 in lists."""
    for t in (m.ln_gates, m.d_gates, m.xs, m.ys, m.d_ys, m.d_xs, m.act, m.gate_up, m.work, m.out, m.d_x, m.d_blocks):
        t.fill_(NAN)
    for t in (m.ids, m.rows, m.offsets):
        t.fill_(-7)


def results(m):
    return m.outputs() + [t.clone() for t in (m.ids, m.rows, m.offsets, m.ln_gates)]


def test_two_streams_at_once_over_overwritten_buffers():
    layers = [Layer(500, 6, 20, 512, 264, seed=3, skew=1.0), Layer(300, 2, 3, 1024, 136, "f16", seed=4, drop=0.1)]
    want = []
    for m in layers:
        m.run(), m.back()
        torch.cuda.synchronize()
        want.append(results(m))
        assert not any(bool(torch.isnan(t).any()) for t in want[-1])
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for m in layers:
            poison(m)
        torch.cuda.synchronize()
        for m, s in zip(layers, streams):
            with torch.cuda.stream(s):
                m.run(), m.back()
        torch.cuda.synchronize()
        for m, w in zip(layers, want):
            assert all(torch.equal(a, b) for a, b in zip(results(m), w))


def test_two_graphs_at_once_over_overwritten_buffers():
    layers = [Layer(200, 4, 12, 256, 136, seed=1), Layer(90, 2, 5, 328, 72, "f16", seed=2, drop=0.2)]
    graphs, gates = [], []
    for m in layers:
        m.run(), m.back()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.run(), m.back()
        graphs.append(g)
        gates.append(m.gates)                            # the graph's own
    streams = [torch.cuda.Stream() for _ in graphs]
    for seed in (7, 8):
        want = []
        for m in layers:
            g = torch.Generator(device="cuda").manual_seed(seed)
            for t in (m.x, m.base, m.d_out, m.logits):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
            m.run(), m.back()
            torch.cuda.synchronize()
            want.append(results(m))
        for _ in range(3):
            for m, g in zip(layers, gates):
                poison(m)
                g.fill_(NAN)
            torch.cuda.synchronize()
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
            torch.cuda.synchronize()
            for m, w in zip(layers, want):
                assert all(torch.equal(a, b) for a, b in zip(results(m), w))
