"""A run of the operators on tokens sorted by expert together, as a layer uses them, forward and backward: against 64-bit autograd and
differences, against a decode step of a stack, captured and replayed, on two streams, at the largest sizes and offsets, and
with rows and blocks that hold NaN."""
import numpy as np
import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import expert_ref as ref
from test_gpu_experts import DT, NAN, Ffn, Rows, generator, ok, route, run_sort, stream

pytestmark = pytest.mark.gpu


class Layer:
    """Buffers of a layer's forward and backward pass over T tokens; run() and back() are the calls a program makes."""

    def __init__(self, T, K, N, H, I, dtype="bf16", seed=0, drop=0.0, skew=0.5):
        self.T, self.K, self.N, self.H, self.I = T, K, N, H, I
        self.dt, self.code = DT[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.x = rand(T, H).to(self.dt)
        self.base = rand(T, H).to(self.dt)
        self.d_out = rand(T, H).to(self.dt)
        self.blocks = (rand(N, I, 3, H) * (2.0 / H) ** 0.5).to(self.dt)
        self.logits = rand(T, N) + skew * rand(1, N)
        self.left_out = torch.rand(T, generator=g, device="cuda") < drop
        R = T * K
        new = lambda *s: torch.zeros(*s, dtype=self.dt, device="cuda")
        self.ids, self.rows = (torch.empty(T, K, dtype=torch.int32, device="cuda") for _ in range(2))
        self.ln_gates, self.d_gates = (torch.empty(T, K, device="cuda") for _ in range(2))
        self.offsets = torch.empty(N + 1, dtype=torch.int32, device="cuda")
        self.xs, self.ys, self.d_ys, self.d_xs = (new(R, H) for _ in range(4))
        self.act, self.gate_up, self.work = new(R, I), new(2, R, I), new(3, R, I)
        self.out, self.d_x, self.d_blocks = new(T, H), new(T, H), torch.zeros_like(self.blocks)

    def run(self):
        T, K, N, H, I, code, s = self.T, self.K, self.N, self.H, self.I, self.code, stream()
        ok(rb.remoe_token_logprobs(T, N, rb.REMOE_F32, self.logits, N, 1.0, None, K, None, None, self.ids, self.ln_gates, None, s))
        self.gates = self.ln_gates.exp()
        self.ids.masked_fill_(self.left_out.unsqueeze(1), -1)
        ok(rb.remoe_expert_sort(T, K, N, self.ids, self.rows, self.offsets, s))
        ok(rb.remoe_expert_dispatch(T, K, H, code, self.x, H, self.rows, T * K, self.xs, H, s))
        ok(rb.remoe_expert_ffn(T * K, N, H, I, code, self.xs, H, self.offsets, self.blocks, 3 * H * I, self.gate_up, self.act, self.ys, H, s))
        ok(rb.remoe_expert_combine(T, K, H, code, T * K, self.ys, H, self.rows, self.gates, self.base, H, self.out, H, s))

    def back(self):
        T, K, N, H, I, code, s = self.T, self.K, self.N, self.H, self.I, self.code, stream()
        ok(rb.remoe_expert_combine_backward(T, K, H, code, self.d_out, H, T * K, self.ys, H, self.rows, self.gates, self.d_ys, H, self.d_gates, s))
        ok(rb.remoe_expert_ffn_backward(T * K, N, H, I, code, self.xs, H, self.offsets, self.blocks, 3 * H * I, self.gate_up, self.d_ys, H, self.work,
                                        self.d_xs, H, self.d_blocks, 3 * H * I, s))
        ok(rb.remoe_expert_combine(T, K, H, code, T * K, self.d_xs, H, self.rows, None, None, 0, self.d_x, H, s))

    def outputs(self):
        return [t.clone() for t in (self.out, self.d_x, self.d_gates, self.d_blocks)]

    def loss64(self, x, gates, blocks):
        """sum of d_out * out in 64 bits, straight from the definition, token by token and expert by expert"""
        out = self.base.double()
        for e in range(self.N):
            t, k = (self.ids == e).nonzero(as_tuple=True)
            if t.numel():
                wg, wu, wd = blocks[e].unbind(1)
                out = out.index_add(0, t, (ref.silu(x[t] @ wg.T) * (x[t] @ wu.T)) @ wd * gates[t, k].unsqueeze(1))
        return (out * self.d_out.double()).sum(), out

    def gate_terms64(self):
        """[T, K]: root of the sum of squares of the terms whose roundings reach a gate's gradient <y, d out>: the products y_h d_h (y is rounded) and,
        act having been rounded before it, a_i <W_down[i], d out>."""
        size = torch.zeros(self.T, self.K, dtype=torch.float64, device="cuda")
        x, d = self.x.double(), self.d_out.double()
        for e in range(self.N):
            t, k = (self.ids == e).nonzero(as_tuple=True)
            if t.numel():
                wg, wu, wd = self.blocks[e].double().unbind(1)
                a = ref.silu(x[t] @ wg.T) * (x[t] @ wu.T)
                size[t, k] = (((a @ wd) * d[t]).pow(2).sum(1) + (a * (d[t] @ wd.T)).pow(2).sum(1)).sqrt()
        return size


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,K,N,H,I", [(1, 1, 1, 64, 32), (1, 6, 64, 256, 96), (33, 4, 9, 264, 136), (300, 6, 16, 512, 192), (700, 1, 1, 256, 520)])
def test_layer_against_autograd_and_differences(T, K, N, H, I, dtype):
    a = Layer(T, K, N, H, I, dtype, seed=T, drop=0.15 if T > 1 else 0.0)
    a.run()
    a.back()
    torch.cuda.synchronize()
    x, gates, blocks = (v.double().requires_grad_(True) for v in (a.x, a.gates, a.blocks))
    loss, out = a.loss64(x, gates, blocks)
    loss.backward()
    live = (a.ids >= 0).double()
    # Roundings on the way: out: act, ys, out; d_x: gate and up, d ys, d g and d u, d xs, d x; d_blocks: x's or d ys's partner and the
    # result.  n independent ones of at most half / sqrt(3) each stay below half * sqrt(n / 3); the slope of silu may add as much for kept gates.
    ref.rms_close(a.out, out.detach(), a.dt, "out", times=1.5)
    ref.rms_close(a.d_x, x.grad, a.dt, "d_x", times=2.0)
    # A gate's gradient is one sum, whose terms may cancel: its error is a sum of independent roundings of those, each at most half a step, with a
    # standard deviation of half / sqrt(3) times the root of their squares' sum.  Seven of them:
    gate_error = 4 * ref.half(a.dt) * a.gate_terms64()
    ref.close(a.d_gates * live, gates.grad * live, gate_error, "d_gates")
    ref.rms_close(a.d_blocks, blocks.grad, a.dt, "d_blocks", times=2.0)
    # and with differences of the 64-bit loss in random directions: what the kernel's gradient says of them is off by its error's norm at most
    g = torch.Generator(device="cuda").manual_seed(5)
    eps = 1e-5
    norm = lambda grad: 2.0 * ref.half(a.dt) * float(grad.double().norm())
    for theta, grad, error in ((0, a.d_x, norm(a.d_x)), (1, a.d_gates * live, float(gate_error.norm())), (2, a.d_blocks, norm(a.d_blocks))):
        base = [a.x.double(), a.gates.double(), a.blocks.double()]
        v = torch.randn(base[theta].shape, generator=g, device="cuda", dtype=torch.float64)
        if theta == 1:
            v = v * live
        up, down = list(base), list(base)
        up[theta], down[theta] = base[theta] + eps * v, base[theta] - eps * v
        with torch.no_grad():
            slope = (a.loss64(*up)[0] - a.loss64(*down)[0]) / (2 * eps)
        assert abs(float((grad.double() * v).sum() - slope)) <= error * float(v.norm()) + 1e-6 * abs(float(slope))


def test_layer_gives_what_a_decode_step_gives():
    import synth
    from paper_2605_27081_b200.loader import LoadedWorkload
    shape = synth.Shape(1, 512, 32, 4, 96, 1, 64, 0, 1, 1, 1)
    wl = LoadedWorkload(shape, 8, seed=3)
    try:
        bits = lambda a, *s: torch.from_numpy(np.ascontiguousarray(a).view(np.int16).copy()).view(torch.bfloat16).view(*s).cuda()
        blocks = torch.stack([bits(wl.expert_block(0, e), 96, 3, 512) for e in range(32)])
        shared = bits(wl.shared[0][0], 64, 3, 512)
        T = 12
        x = torch.randn(T, 512, generator=generator(1)).to(torch.bfloat16).cuda()
        want, ids, gates = torch.empty(T, 512, device="cuda"), torch.empty(T, 4, dtype=torch.int32, device="cuda"), torch.empty(T, 4, device="cuda")
        for t in range(T):
            wl.stack.decode_step(x[t].float().contiguous(), want[t], ids[t], gates[t])
        torch.cuda.synchronize()
        s = stream()
        rows, offsets = run_sort(ids, 32)
        new = lambda *sh: torch.empty(*sh, dtype=torch.bfloat16, device="cuda")
        xs, ys, act, base, out = new(T * 4, 512), new(T * 4, 512), new(T * 4, 96), new(T, 512), new(T, 512)
        every = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        ok(rb.remoe_expert_ffn(T, 1, 512, 64, rb.REMOE_BF16, x, 512, every, shared, 3 * 64 * 512, None, new(T, 64), base, 512, s))
        ok(rb.remoe_expert_dispatch(T, 4, 512, rb.REMOE_BF16, x, 512, rows, T * 4, xs, 512, s))
        ok(rb.remoe_expert_ffn(T * 4, 32, 512, 96, rb.REMOE_BF16, xs, 512, offsets, blocks, 3 * 96 * 512, None, act, ys, 512, s))
        ok(rb.remoe_expert_combine(T, 4, 512, rb.REMOE_BF16, T * 4, ys, 512, rows, gates, base, 512, out, 512, s))
        torch.cuda.synchronize()
        ref.rms_close(out, want, torch.bfloat16, "layer against decode step", times=2.0)      # act, ys, base, out: four roundings
    finally:
        wl.close()


def test_captured_and_replayed_on_new_inputs_two_graphs_at_once():
    a, b = Layer(200, 4, 12, 256, 136, seed=1), Layer(90, 2, 5, 328, 72, "f16", seed=2, drop=0.2)
    graphs = []
    for m in (a, b):
        m.run(), m.back()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.run(), m.back()
        graphs.append(g)
    for seed in (7, 8):
        want = []
        for m in (a, b):
            g = torch.Generator(device="cuda").manual_seed(seed)
            for t in (m.x, m.base, m.d_out, m.logits):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
            m.run(), m.back()
            torch.cuda.synchronize()
            want.append(m.outputs())
            for t in (m.out, m.d_x, m.d_blocks, m.xs, m.ys, m.act, m.work, m.gate_up):
                t.fill_(NAN)
        streams = [torch.cuda.Stream() for _ in graphs]
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for m, w in zip((a, b), want):
            assert all(torch.equal(x, y) for x, y in zip(m.outputs(), w))


def test_two_streams_at_once_and_the_same_bits_every_time():
    layers = [Layer(500, 6, 20, 512, 264, seed=3, skew=1.0), Layer(300, 2, 3, 1024, 136, seed=4)]
    want = []
    for m in layers:
        m.run(), m.back()
        torch.cuda.synchronize()
        want.append(m.outputs())
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for m, s in zip(layers, streams):
            with torch.cuda.stream(s):
                m.run(), m.back()
        torch.cuda.synchronize()
        for m, w in zip(layers, want):
            assert all(torch.equal(x, y) for x, y in zip(m.outputs(), w))


def test_nan_and_infinity_reach_what_they_take_part_in_and_nothing_else():
    for value in (NAN, float("inf")):
        f = Ffn([70, 3, 40, 17], 136, 72, "bf16", seed=9)
        f.forward(), f.backward()
        clean = f.ys.view.clone(), f.d_xs.view.clone(), f.d_blocks.clone()
        x_was = f.xs.view[71].clone()
        f.xs.view[71] = value                           # a row of the second expert
        f.forward()
        others = torch.arange(f.R, device="cuda") != 71
        assert torch.equal(f.ys.view[others], clean[0][others]) and not bool(torch.isfinite(f.ys.view[71]).any())
        f.backward()
        assert torch.equal(f.d_xs.view[others], clean[1][others])
        assert all(torch.equal(f.d_blocks[e], clean[2][e]) for e in (0, 2, 3)) and bool(torch.isnan(f.d_blocks[1, :, 0]).all())
        f.xs.view[71] = x_was
        was = f.blocks[2].clone()
        f.blocks[2] = value                              # an expert's weights
        f.forward()
        live = torch.cat([torch.arange(0, 73), torch.arange(113, 130)]).cuda()
        assert torch.equal(f.ys.view[live], clean[0][live]) and not bool(torch.isfinite(f.ys.view[73:113]).any())
        f.blocks[2] = was
        f.forward(), f.backward()
        assert torch.equal(f.ys.view, clean[0]) and torch.equal(f.d_blocks, clean[2])


@pytest.mark.parametrize("given,held", [([5, 2, 900, 3], [5, 5, 60, 60]), ([-7, 10, 10, 2 ** 31 - 1], [0, 10, 10, 60]), ([60, 0, 0, 0], [60, 60, 60, 60])])
def test_offsets_are_held_to_the_rows(given, held):
    f = Ffn([20, 20, 20], 72, 40, "bf16", seed=2)
    f.offsets.copy_(torch.tensor(held, dtype=torch.int32))
    f.forward(), f.backward()
    want = f.ys.view.clone(), f.d_xs.view.clone(), f.d_blocks.clone()
    for t in (f.ys.view, f.d_xs.view, f.d_blocks):
        t.fill_(55.0)
    f.offsets.copy_(torch.tensor(given, dtype=torch.int32))
    f.forward(), f.backward()
    rows = slice(held[0], held[3])
    assert torch.equal(f.ys.view[rows], want[0][rows]) and torch.equal(f.d_xs.view[rows], want[1][rows]) and torch.equal(f.d_blocks, want[2])
    assert bool((f.ys.view[:held[0]] == 55).all())


@pytest.mark.parametrize("counts,H,I", [([3], 65536, 8), ([5, 1], 8, 65536), ([1] * 1024, 16, 8), ([0] * 1023 + [300], 64, 24), ([4000], 64, 64)])
def test_largest_widths_and_numbers_of_experts(counts, H, I):
    f = Ffn(counts, H, I, "bf16", seed=1)
    f.check_forward(rms=False)
    f.check_backward(rms=False)


def test_no_rows_at_all():
    f = Ffn([0, 0, 0], 64, 24, "bf16")
    ok(rb.remoe_expert_ffn(0, 3, 64, 24, f.code, None, 64, f.offsets, f.blocks, f.block, None, None, None, 64, stream()))
    ok(rb.remoe_expert_ffn_backward(0, 3, 64, 24, f.code, None, 64, f.offsets, f.blocks, f.block, None, None, 64, None, None, 64, f.d_blocks, f.block, stream()))
    torch.cuda.synchronize()
    assert bool((f.d_blocks == 0).all())


def test_gradient_over_the_gradient_of_the_rows():
    """frozen experts: d_xs in the place of d_ys"""
    f = Ffn([40, 0, 33, 300], 136, 72, "f16", seed=6, pad=8)
    f.forward(), f.backward(blocks=False)
    want = f.d_xs.view.clone()
    ok(rb.remoe_expert_ffn_backward(f.R, f.N, f.H, f.I, f.code, None, 0, f.offsets, f.blocks, f.block, f.gate_up, f.d_ys.view, f.d_ys.stride, f.work,
                                    f.d_ys.view, f.d_ys.stride, None, 0, stream()))
    torch.cuda.synchronize()
    assert torch.equal(f.d_ys.view, want)


def test_offsets_that_pass_32_bits():
    """rows and buffers of more than 2^31 elements: the last rows, and blocks of experts whose addresses lie far apart"""
    R, H, I = 1_100_000, 2048, 2048
    big = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
    xs, ys, act = big(R, H), big(R, H), big(R, I)
    gate_up, work, d_xs = big(2, R, I), big(3, R, I), big(R, H)
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 7
    x, d = (torch.randn(n, H, generator=g, device="cuda").bfloat16() for _ in range(2))
    xs[-n:] = x
    d_ys = ys                                            # (the forward pass is over when it is filled)
    far = 2 ** 31 + 8
    flat = torch.empty(far + 3 * I * H, dtype=torch.bfloat16, device="cuda")
    blocks = torch.as_strided(flat, (2, I, 3, H), (far, 3 * H, H, 1))
    blocks[:] = (torch.randn(2, I, 3, H, generator=g, device="cuda") * 0.02).bfloat16()
    offsets = torch.tensor([R - n, R - 3, R], dtype=torch.int32, device="cuda")
    ok(rb.remoe_expert_ffn(R, 2, H, I, rb.REMOE_BF16, xs, H, offsets, blocks, far, gate_up, act, ys, H, stream()))
    small = torch.tensor([0, n - 3, n], dtype=torch.int32, device="cuda")
    want = ref.ffn(x, small, blocks)
    ref.close(ys[-n:], want["ys"][0], want["ys"][1], "ys")
    ref.close(gate_up[1, -n:], want["up"][0], want["up"][1], "up")
    d_ys[-n:] = d
    d_blocks = torch.empty_like(flat)
    ok(rb.remoe_expert_ffn_backward(R, 2, H, I, rb.REMOE_BF16, xs, H, offsets, blocks, far, gate_up, d_ys, H, work, d_xs, H, d_blocks, far, stream()))
    back = ref.ffn_backward(x, small, blocks, gate_up[:, -n:], d)
    ref.close(d_xs[-n:], back["d_xs"][0], back["d_xs"][1], "d_xs")
    ref.close(torch.as_strided(d_blocks, (2, I, 3, H), (far, 3 * H, H, 1)), back["d_blocks"][0], back["d_blocks"][1], "d_blocks")
    # rows out and back
    rows = torch.tensor([[R - 1], [R - 4], [R - 2]], dtype=torch.int32, device="cuda")
    tok, out = torch.randn(3, H, generator=g, device="cuda").bfloat16(), big(3, H)
    ok(rb.remoe_expert_dispatch(3, 1, H, rb.REMOE_BF16, tok, H, rows, R, xs, H, stream()))
    ok(rb.remoe_expert_combine(3, 1, H, rb.REMOE_BF16, R, xs, H, rows, None, None, 0, out, H, stream()))
    d_gates = torch.empty(3, 1, device="cuda")
    ok(rb.remoe_expert_combine_backward(3, 1, H, rb.REMOE_BF16, tok, H, R, xs, H, rows, None, d_xs, H, d_gates, stream()))
    torch.cuda.synchronize()
    assert torch.equal(out, tok) and torch.equal(d_xs[R - 4], tok[1])
    ref.close(d_gates.squeeze(1), (tok.double() ** 2).sum(1), (H / 32 + 16) * ref.U * (tok.double() ** 2).sum(1), "d_gates")


# rows that are not whole numbers of accesses, more items than fit at once, more than 32 selections a token, every width of an access
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,K,H,pad,offset", [(5, 40, 33, 0, 0), (600, 9, 2050, 6, 0), (4000, 3, 96, 0, 8), (4000, 11, 60, 4, 0), (3700, 2, 7, 1, 0), (700, 8, 1021, 3, 0),
                                               (900, 33, 520, 0, 4), (1500, 1, 1000, 2, 2), (460, 5, 9001, 7, 0)])
def test_rows_of_every_layout(T, K, H, pad, offset, dtype):
    dt, code = DT[dtype]
    g = generator(T + K)
    N = 50
    ids = torch.randint(-1, N, (T, K), generator=g).int().cuda()
    rows, offsets = run_sort(ids, N)
    used = int(offsets[-1])
    x, base = (Rows(torch.randn(T, H, generator=g).to(dt), pad, offset) for _ in range(2))
    xs = Rows(torch.full((T * K, H), NAN, dtype=dt), pad, offset)
    ok(rb.remoe_expert_dispatch(T, K, H, code, x.view, x.stride, rows, T * K, xs.view, xs.stride, stream()))
    there = rows >= 0
    picked = x.view.double().unsqueeze(1).expand(T, K, H)[there]
    assert torch.equal(xs.view[rows[there].long()].double(), picked)
    xs.others_untouched(slice(0, used))
    gates = torch.rand(T, K, generator=g).cuda()
    out = Rows(torch.full((T, H), 55.0, dtype=dt), pad, offset)
    ok(rb.remoe_expert_combine(T, K, H, code, T * K, xs.view, xs.stride, rows, gates, base.view, base.stride, out.view, out.stride, stream()))
    weight = (gates.double() * there).sum(1, keepdim=True)
    want = weight * x.view.double() + base.view.double()
    bound = (K + 2) * ref.U * (weight * x.view.double().abs() + base.view.double().abs()) + ref.half(dt) * want.abs() + ref.tiny(dt)
    ref.close(out.view, want, bound, "combine")
    out.others_untouched()
    d_ys, d_gates = Rows(torch.full((T * K, H), 55.0, dtype=dt), pad, offset), torch.empty(T, K, device="cuda")
    ok(rb.remoe_expert_combine_backward(T, K, H, code, base.view, base.stride, T * K, xs.view, xs.stride, rows, gates, d_ys.view, d_ys.stride, d_gates, stream()))
    dot = x.view.double() * base.view.double()
    ref.close(d_gates, dot.sum(1, keepdim=True) * there, (H / 32 + 16) * ref.U * dot.abs().sum(1, keepdim=True), "d_gates")
    w = (gates.double().unsqueeze(2) * base.view.double().unsqueeze(1))[there]
    ref.close(d_ys.view[rows[there].long()], w, (ref.half(dt) + 2 * ref.U) * w.abs() + ref.tiny(dt), "d_ys")
    d_ys.others_untouched(slice(0, used))


def test_memory_of_the_host_is_refused():
    host = torch.zeros(4096).pin_memory()
    d = torch.zeros(4096, dtype=torch.int32, device="cuda")
    assert rb.remoe_expert_sort(2, 2, 4, d, d, host, stream()) == rb.REMOE_E_ARG
    assert rb.remoe_expert_dispatch(2, 2, 8, rb.REMOE_F32, host, 8, d, 4, d, 8, stream()) == rb.REMOE_E_ARG
    assert rb.remoe_expert_combine(2, 2, 8, rb.REMOE_F32, 4, d, 8, d, None, None, 0, host, 8, stream()) == rb.REMOE_E_ARG
    assert rb.remoe_expert_combine_backward(2, 2, 8, rb.REMOE_F32, host, 8, 4, d, 8, d, None, d, 8, None, stream()) == rb.REMOE_E_ARG
    assert rb.remoe_expert_ffn(2, 1, 8, 8, rb.REMOE_BF16, d, 8, d, host, 192, None, d, d, 8, stream()) == rb.REMOE_E_ARG
    assert rb.remoe_expert_ffn_backward(2, 1, 8, 8, rb.REMOE_BF16, d, 8, d, host, 192, d, d, 8, d, d, 8, None, 0, stream()) == rb.REMOE_E_ARG
    torch.cuda.synchronize()
