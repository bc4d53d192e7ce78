"""Operators on tokens sorted by expert against their 64-bit values (expert_ref), at the sizes, counts and layouts where they can
go wrong, through the C entry points."""
import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import expert_ref as ref

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, rb.REMOE_F32), "bf16": (torch.bfloat16, rb.REMOE_BF16), "f16": (torch.float16, rb.REMOE_F16)}
NAN = float("nan")


def stream():
    return torch.cuda.current_stream().cuda_stream


def ok(rc):
    assert rc == 0, rb.strerror(rc)


class Rows:
    """A matrix on the GPU with `pad` elements between its rows, `offset` elements behind an aligned address, canaries around."""

    def __init__(self, x, pad=0, offset=0):
        n, w = x.shape
        self.flat = torch.full((offset + n * (w + pad) + 16,), 777.0, dtype=x.dtype, device="cuda")
        self.view = self.flat[offset:offset + n * (w + pad)].view(n, w + pad)[:, :w]
        self.view.copy_(x)
        self.before = self.flat.clone()
        self.stride = w + pad

    def others_untouched(self, rows=None):
        """Nothing outside the matrix (outside the given rows of it) has changed."""
        now, was = self.flat.clone(), self.before.clone()
        n, w = self.view.shape
        for f in (now, was):
            v = f[self.view.storage_offset():][:n * self.stride].view(n, self.stride)[:, :w]
            if rows is None:
                v.zero_()
            else:
                v[rows] = 0
        assert torch.equal(now.nan_to_num(-5.0), was.nan_to_num(-5.0))


def generator(seed):
    return torch.Generator().manual_seed(seed)


def route(T, K, N, seed, drop=0.0, skew=0.0):
    g = generator(seed)
    logits = torch.randn(T, N, generator=g) + skew * torch.randn(1, N, generator=g)
    ids = logits.topk(K, 1).indices.int()
    ids[torch.rand(T, generator=g) < drop] = -1
    return ids.cuda()


def run_sort(ids, N):
    T, K = ids.shape
    rows = torch.full((T, K), -7, dtype=torch.int32, device="cuda")
    offsets = torch.full((N + 3,), -7, dtype=torch.int32, device="cuda")
    ok(rb.remoe_expert_sort(T, K, N, ids, rows, offsets, stream()))
    torch.cuda.synchronize()
    assert offsets[N + 1:].tolist() == [-7, -7]
    return rows, offsets[:N + 1]


# ------------------------------------------------------------------------------------------------------------- sort

@pytest.mark.parametrize("T,K,N", [(0, 1, 1), (1, 1, 1), (1, 6, 64), (5, 3, 7), (32, 8, 128), (33, 1, 2), (100, 4, 60), (257, 6, 64), (1000, 5, 33),
                                   (4096, 6, 64), (8191, 8, 128), (3000, 2, 1024), (20000, 8, 1000), (70001, 3, 17), (300000, 1, 5)])
def test_sort(T, K, N):
    for seed in range(3):
        g = generator(seed)
        ids = torch.randint(-1 if seed else 0, N + (2 if seed == 2 else 0), (T, K), generator=g).int()
        if seed == 2 and T > 2:
            ids[1, 0], ids[2, 0] = 2 ** 31 - 1, -2 ** 31
        rows, offsets = run_sort(ids.cuda(), N)
        want_rows, want_offsets, _ = ref.sort(ids, N)
        assert torch.equal(offsets.cpu(), want_offsets) and torch.equal(rows.cpu(), want_rows)


@pytest.mark.parametrize("T,K,N", [(1, 1, 3), (500, 4, 9), (9000, 7, 300)])
def test_sort_one_expert_takes_all_or_none(T, K, N):
    for e in (0, N - 1, -1, N):
        ids = torch.full((T, K), e, dtype=torch.int32, device="cuda")
        rows, offsets = run_sort(ids, N)
        want_rows, want_offsets, _ = ref.sort(ids, N)
        assert torch.equal(offsets.cpu(), want_offsets) and torch.equal(rows.cpu(), want_rows)


def test_sort_in_place():
    ids = route(3001, 5, 50, 3, drop=0.2)
    want, offsets = run_sort(ids, 50)
    ok(rb.remoe_expert_sort(3001, 5, 50, ids, ids, offsets, stream()))
    torch.cuda.synchronize()
    assert torch.equal(ids, want)


# ------------------------------------------------------------------------------------ dispatch, combine and its backward

SHAPES = [(1, 1, 1, 1), (1, 6, 64, 2048), (3, 2, 5, 7), (32, 8, 128, 2048), (65, 3, 20, 1021), (200, 17, 40, 264), (1000, 4, 60, 96), (50, 2, 3, 9000),
          (7, 9, 9, 40)]
LAYOUTS = [(0, 0), (1, 3), (8, 8), (4, 4)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,K,N,H", SHAPES)
def test_dispatch(T, K, N, H, dtype):
    dt, code = DT[dtype]
    for pad, offset in LAYOUTS:
        ids = route(T, K, N, T + pad, drop=0.2 if pad else 0.0)
        rows, offsets = run_sort(ids, N)
        used = int(offsets[-1])
        x = Rows(torch.randn(T, H, generator=generator(H)).to(dt), pad, offset)
        x.view[0, 0] = NAN
        xs = Rows(torch.full((T * K, H), 55.0, dtype=dt), pad, offset)
        ok(rb.remoe_expert_dispatch(T, K, H, code, x.view, x.stride, rows, T * K, xs.view, xs.stride, stream()))
        torch.cuda.synchronize()
        want = torch.full((T * K, H), 55.0, dtype=dt, device="cuda")
        there = rows.flatten() >= 0
        want[rows.flatten()[there].long()] = x.view.repeat_interleave(K, 0)[there]
        assert torch.equal(xs.view.nan_to_num(-3.0), want.nan_to_num(-3.0))
        xs.others_untouched(slice(0, used))


def test_dispatch_and_combine_leave_out_rows_that_are_not_there():
    rows = torch.tensor([[0, 9], [-5, 3], [4, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    x, xs = torch.randn(3, 16, device="cuda"), torch.full((4, 16), 5.0, device="cuda")
    ok(rb.remoe_expert_dispatch(3, 2, 16, rb.REMOE_F32, x, 16, rows, 4, xs, 16, stream()))
    assert torch.equal(xs[0], x[0]) and torch.equal(xs[3], x[1]) and bool((xs[1:3] == 5).all())
    out = torch.empty(3, 16, device="cuda")
    gates = torch.full((3, 2), 2.0, device="cuda")
    gates[0, 1] = NAN
    ok(rb.remoe_expert_combine(3, 2, 16, rb.REMOE_F32, 4, xs, 16, rows, gates, None, 0, out, 16, stream()))
    assert torch.equal(out[0], 2 * x[0]) and torch.equal(out[1], 2 * x[1]) and bool((out[2] == 0).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,K,N,H", SHAPES)
def test_combine(T, K, N, H, dtype):
    dt, code = DT[dtype]
    for i, (pad, offset) in enumerate(LAYOUTS):
        ids = route(T, K, N, T + pad, drop=0.2 if pad else 0.0)
        rows, offsets = run_sort(ids, N)
        used, g = int(offsets[-1]), generator(H + i)
        ys = Rows(torch.randn(T * K, H, generator=g).to(dt), pad, offset)
        ys.view[used:] = NAN
        gates = torch.rand(T, K, generator=g).cuda() if i != 1 else None
        base = Rows(torch.randn(T, H, generator=g).to(dt), pad, offset) if i % 2 else None
        out = Rows(torch.full((T, H), 55.0, dtype=dt), pad, offset)
        picked = ys.view[rows.clamp(min=0).long()].double().masked_fill((rows < 0).unsqueeze(2), 0.0)
        terms = picked * (1.0 if gates is None else gates.double().unsqueeze(2))
        want = terms.sum(1) + (base.view.double() if base else 0)
        bound = (K + 2) * ref.U * (terms.abs().sum(1) + (base.view.double().abs() if base else 0)) + ref.half(dt) * want.abs() + ref.tiny(dt)
        ok(rb.remoe_expert_combine(T, K, H, code, T * K, ys.view, ys.stride, rows, gates, base.view if base else None, base.stride if base else 0,
                                   out.view, out.stride, stream()))
        torch.cuda.synchronize()
        ref.close(out.view, want, bound, "combine")
        out.others_untouched()
        if base:                                       # onto the base itself
            ok(rb.remoe_expert_combine(T, K, H, code, T * K, ys.view, ys.stride, rows, gates, base.view, base.stride, base.view, base.stride, stream()))
            torch.cuda.synchronize()
            assert torch.equal(base.view, out.view)
            base.others_untouched()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,K,N,H", SHAPES)
def test_combine_backward(T, K, N, H, dtype):
    dt, code = DT[dtype]
    for i, (pad, offset) in enumerate(LAYOUTS):
        ids = route(T, K, N, T + pad, drop=0.2 if pad else 0.0)
        rows, offsets = run_sort(ids, N)
        used, g = int(offsets[-1]), generator(H + i)
        ys = Rows(torch.randn(T * K, H, generator=g).to(dt), pad, offset)
        ys.view[used:] = NAN
        d_out = Rows(torch.randn(T, H, generator=g).to(dt), pad, offset)
        gates = torch.rand(T, K, generator=g).cuda() if i != 1 else None
        d_ys = Rows(torch.full((T * K, H), 55.0, dtype=dt), pad, offset)
        d_gates = torch.full((T, K), 55.0, device="cuda")
        there = rows >= 0
        picked = ys.view[rows.clamp(min=0).long()].double().masked_fill(~there.unsqueeze(2), 0.0)
        terms = picked * d_out.view.double().unsqueeze(1)
        want_rows = (d_out.view.double().unsqueeze(1) * (1.0 if gates is None else gates.double().unsqueeze(2)).expand(T, K, H) if gates is not None
                     else d_out.view.double().unsqueeze(1).expand(T, K, H))
        call = lambda a, b: ok(rb.remoe_expert_combine_backward(T, K, H, code, d_out.view, d_out.stride, T * K, ys.view, ys.stride, rows, gates,
                                                                a, d_ys.stride if a is not None else 0, b, stream()))
        call(d_ys.view, d_gates)
        torch.cuda.synchronize()
        ref.close(d_gates, terms.sum(2), (H / 32 + 16) * ref.U * terms.abs().sum(2), "d_gates")
        got = d_ys.view[rows[there].long()]
        ref.close(got, want_rows[there], (ref.half(dt) + 2 * ref.U) * want_rows[there].abs() + ref.tiny(dt), "d_ys")
        d_ys.others_untouched(slice(0, used))
        both = d_ys.view.clone(), d_gates.clone()
        d_ys.view.fill_(1.0)
        call(d_ys.view, None)                           # each alone, and over the rows themselves
        call(None, d_gates.fill_(9.0))
        torch.cuda.synchronize()
        assert torch.equal(d_ys.view[:used], both[0][:used]) and torch.equal(d_gates, both[1])
        ok(rb.remoe_expert_combine_backward(T, K, H, code, d_out.view, d_out.stride, T * K, ys.view, ys.stride, rows, gates, ys.view, ys.stride,
                                            d_gates.fill_(9.0), stream()))
        torch.cuda.synchronize()
        assert torch.equal(ys.view[:used], both[0][:used]) and torch.equal(d_gates, both[1])


# More tokens than fit on the card at once: every number of rows a group may have, rows of one and of several parts, whole accesses and ragged ones.
MANY = [(2000, 1, 8, 64), (1800, 2, 8, 4104), (1500, 3, 9, 2056), (2100, 4, 12, 1028), (900, 5, 12, 1030), (1200, 6, 64, 2048), (800, 7, 16, 520), (700, 8, 16, 2568),
        (5000, 9, 20, 136), (600, 33, 40, 1032), (1300, 4, 6, 1021)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,K,N,H", MANY)
def test_rows_of_many_tokens(T, K, N, H, dtype):
    test_dispatch(T, K, N, H, dtype)
    test_combine(T, K, N, H, dtype)
    test_combine_backward(T, K, N, H, dtype)


# ---------------------------------------------------------------------------------------------------- the experts' products

class Ffn:
    """Rows, blocks and buffers of a call; rows that belong to no expert and what lies between rows hold NaN."""

    def __init__(self, counts, H, I, dtype, seed=0, pad=0, behind=0, block_pad=0, first=0):
        self.dt, self.code = DT[dtype]
        self.N, self.H, self.I = len(counts), H, I
        self.used, self.R = sum(counts), first + sum(counts) + behind
        self.offsets = torch.tensor([first] + list(torch.tensor(counts).cumsum(0) + first), dtype=torch.int32, device="cuda")
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows = lambda scale: Rows(torch.randn(self.R, H, generator=g, device="cuda").mul_(scale).to(self.dt), pad)
        self.live = slice(first, first + self.used)
        self.xs, self.d_ys = rows(1.0), rows(0.5)
        for m in (self.xs, self.d_ys):
            m.flat[m.flat == 777.0] = NAN
            dead = torch.ones(self.R, dtype=torch.bool, device="cuda")
            dead[self.live] = False
            m.view[dead] = NAN
        self.block = 3 * I * H + block_pad
        flat = torch.full((self.N * self.block,), NAN, dtype=self.dt, device="cuda")
        self.blocks = flat.view(self.N, self.block)[:, :3 * I * H].unflatten(1, (I, 3, H))
        self.blocks.copy_(torch.randn(self.N, I, 3, H, generator=g, device="cuda") * (2.0 / H) ** 0.5)
        self.ys, self.d_xs = (Rows(torch.full((self.R, H), 55.0, dtype=self.dt), pad) for _ in range(2))
        self.act = torch.full((self.R, I), 55.0, dtype=self.dt, device="cuda")
        self.gate_up = torch.full((2, self.R, I), 55.0, dtype=self.dt, device="cuda")
        self.work = torch.full((3, self.R, I), 55.0, dtype=self.dt, device="cuda")
        self.d_flat = torch.full((self.N * self.block + 8,), 55.0, dtype=self.dt, device="cuda")
        self.d_blocks = self.d_flat[:self.N * self.block].view(self.N, self.block)[:, :3 * I * H].unflatten(1, (I, 3, H))

    def forward(self, keep=True):
        ok(rb.remoe_expert_ffn(self.R, self.N, self.H, self.I, self.code, self.xs.view, self.xs.stride, self.offsets, self.blocks, self.block,
                               self.gate_up if keep else None, self.act, self.ys.view, self.ys.stride, stream()))
        torch.cuda.synchronize()

    def backward(self, rows=True, blocks=True):
        ok(rb.remoe_expert_ffn_backward(self.R, self.N, self.H, self.I, self.code, self.xs.view if blocks else None, self.xs.stride, self.offsets,
                                        self.blocks, self.block, self.gate_up, self.d_ys.view, self.d_ys.stride, self.work,
                                        self.d_xs.view if rows else None, self.d_xs.stride, self.d_blocks if blocks else None, self.block, stream()))
        torch.cuda.synchronize()

    def check_forward(self, rms=True):
        self.forward()
        want, live = ref.ffn(self.xs.view, self.offsets, self.blocks), self.live
        for name, got in (("gate", self.gate_up[0]), ("up", self.gate_up[1]), ("act", self.act), ("ys", self.ys.view)):
            ref.close(got[live], want[name][0][live], want[name][1][live], name)
            dead = torch.ones(self.R, dtype=torch.bool, device="cuda")
            dead[live] = False
            assert bool((got[dead] == 55.0).all()), name
        if rms and self.used:
            ref.rms_close(self.ys.view[live], want["ys"][0][live], self.dt, "ys")
        self.ys.others_untouched(live)
        first, act = self.ys.view.clone(), self.act.clone()
        self.act.fill_(1.0)
        self.forward(keep=False)
        assert torch.equal(self.ys.view[live], first[live]) and torch.equal(self.act[live], act[live])

    def check_backward(self, rms=True):
        live = self.live
        want = ref.ffn_backward(self.xs.view, self.offsets, self.blocks, self.gate_up, self.d_ys.view)
        self.backward()
        ref.close(self.d_xs.view[live], want["d_xs"][0][live], want["d_xs"][1][live], "d_xs")
        ref.close(self.d_blocks, *want["d_blocks"], "d_blocks")
        if rms and self.used:
            ref.rms_close(self.d_xs.view[live], want["d_xs"][0][live], self.dt, "d_xs")
            ref.rms_close(self.d_blocks, want["d_blocks"][0], self.dt, "d_blocks")
        self.d_xs.others_untouched(live)
        between = self.d_flat[:self.N * self.block].view(self.N, self.block)[:, 3 * self.I * self.H:]
        assert bool((between == 55.0).all()) and bool((self.d_flat[self.N * self.block:] == 55.0).all())
        kept = self.d_xs.view.clone(), self.d_blocks.clone()
        self.d_xs.view[live] = 1.0
        self.backward(blocks=False)                     # frozen experts, then the blocks alone
        assert torch.equal(self.d_xs.view[live], kept[0][live])
        self.d_blocks.fill_(3.0)
        self.backward(rows=False)
        assert torch.equal(self.d_blocks, kept[1])


# tile of rows: 256, in steps of 32; stages of 64; boxes of 16, 64, 128 rows
EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 0, 0, 127, 128, 129, 160, 255, 256, 257, 300, 511, 512, 513, 1]
FFN = [([1], 8, 8), ([1], 64, 64), ([3, 0, 2], 72, 40), ([1] * 6 + [0] * 3, 256, 128), (EDGES, 136, 72), ([300], 8, 1408), ([70, 1], 2048, 8), ([40, 400], 320, 1032),
       ([17] * 9, 512, 264), ([0, 0, 5], 1000, 200), ([1300], 264, 136), ([2] * 300, 64, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts,H,I", FFN)
def test_ffn(counts, H, I, dtype):
    for pad, behind, block_pad, first in [(0, 0, 0, 0), (8, 5, 64, 3)]:
        f = Ffn(counts, H, I, dtype, seed=H + I, pad=pad, behind=behind, block_pad=block_pad, first=first)
        f.check_forward(rms=f.used * H > 5000)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts,H,I", FFN)
def test_ffn_backward(counts, H, I, dtype):
    for pad, behind, block_pad, first in [(0, 0, 0, 0), (8, 5, 64, 3)]:
        f = Ffn(counts, H, I, dtype, seed=H + I, pad=pad, behind=behind, block_pad=block_pad, first=first)
        f.forward()
        f.check_backward(rms=f.used * H > 5000)


# Few tiles of a long k: two and four pairs of SMs share a tile's k.  Some calls have room for more tiles than the rows turn out to need.
FEW = [([1], 1544, 1544), ([15], 2048, 1400), ([33], 1536, 760), ([64, 0, 3], 1600, 520), ([129], 264, 5632), ([200], 4104, 264), ([256], 1992, 2056), ([257], 512, 1928),
       ([2, 90, 31, 128], 1672, 128), ([5, 1], 4096, 3080), ([0, 0], 2048, 1544)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts,H,I", FEW)
def test_ffn_of_few_tiles(counts, H, I, dtype):
    for pad, behind, block_pad, first in [(0, 0, 0, 0), (8, 5, 64, 3)]:
        f = Ffn(counts, H, I, dtype, seed=H + I, pad=pad, behind=behind, block_pad=block_pad, first=first)
        f.check_forward()
        f.check_backward()


@pytest.mark.parametrize("counts,H,I", [([0, 2], 8, 40), ([0, 3, 0], 264, 72), ([0, 0, 1, 0], 24, 136), ([5, 0], 1304, 264), ([0], 544, 8)])
def test_experts_without_rows_have_no_gradient(counts, H, I):
    """The last tile of columns is narrow: 8 to 32 of them."""
    f = Ffn(counts, H, I, "bf16", seed=3, behind=2, block_pad=8)
    f.forward()
    f.check_backward(rms=False)
    assert not f.d_blocks[[e for e, n in enumerate(counts) if n == 0]].any()


def test_ffn_of_few_tiles_captured():
    f = Ffn([40], 2048, 1544, "bf16", seed=2)
    f.forward()
    f.backward()
    want = f.ys.view.clone(), f.d_xs.view.clone(), f.d_blocks.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ok(rb.remoe_expert_ffn(f.R, f.N, f.H, f.I, f.code, f.xs.view, f.xs.stride, f.offsets, f.blocks, f.block, f.gate_up, f.act, f.ys.view, f.ys.stride, stream()))
        ok(rb.remoe_expert_ffn_backward(f.R, f.N, f.H, f.I, f.code, f.xs.view, f.xs.stride, f.offsets, f.blocks, f.block, f.gate_up, f.d_ys.view, f.d_ys.stride, f.work,
                                        f.d_xs.view, f.d_xs.stride, f.d_blocks, f.block, stream()))
    for _ in range(3):
        for t in (f.ys.view, f.d_xs.view, f.d_blocks, f.gate_up):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((f.ys.view, f.d_xs.view, f.d_blocks), want))


# ---------------------------------------------------------------------------------------------------- as many selections as a call may have

MOST = 2**31 - 1


def test_sort_of_the_most_selections():
    N, piece = 3, 1 << 27
    ids = torch.empty(MOST, dtype=torch.int32, device="cuda")
    rows = torch.full((MOST,), -7, dtype=torch.int32, device="cuda")
    offsets = torch.full((N + 1,), -7, dtype=torch.int32, device="cuda")
    for s in range(0, MOST, piece):                 # expert s % 3, but for every eighth, which has none
        at = torch.arange(s, min(s + piece, MOST), dtype=torch.int64, device="cuda")
        ids[s:s + piece] = torch.where(at % 8 == 7, -1, at // 8 % N).int()
    ok(rb.remoe_expert_sort(MOST, 1, N, ids, rows, offsets, stream()))
    torch.cuda.synchronize()
    # eights 0, 1, 2, ...: seven selections of expert 0, seven of expert 1, ...; the last eight has no eighth
    eights = (MOST + 1) // 8
    counts = [7 * ((eights - e + N - 1) // N) for e in range(N)]
    first = [0, counts[0], counts[0] + counts[1], sum(counts)]
    assert offsets.tolist() == first
    start = torch.tensor(first[:N], device="cuda")
    for s in range(0, MOST, piece):
        at = torch.arange(s, min(s + piece, MOST), dtype=torch.int64, device="cuda")
        want = torch.where(at % 8 == 7, -1, start[at // 8 % N] + at // 8 // N * 7 + at % 8)
        assert torch.equal(rows[s:s + piece].long(), want)


def test_combine_backward_of_the_most_tokens():
    n_rows, piece = 5, 1 << 27
    d_out = torch.empty(MOST, 1, dtype=torch.bfloat16, device="cuda")
    rows = torch.empty(MOST, dtype=torch.int32, device="cuda")
    ys = torch.tensor([[0.5], [-1.0], [2.0], [3.0], [-0.25]], dtype=torch.bfloat16, device="cuda")
    d_gates = torch.full((MOST,), 9.0, device="cuda")
    for s in range(0, MOST, piece):                 # values of a few bits: the products are exact
        at = torch.arange(s, min(s + piece, MOST), device="cuda")
        rows[s:s + piece] = (at % 6).int()
        d_out[s:s + piece, 0] = (at % 17 - 8).bfloat16()
    ok(rb.remoe_expert_combine_backward(MOST, 1, 1, rb.REMOE_BF16, d_out, 1, n_rows, ys, 1, rows, None, None, 0, d_gates, stream()))
    torch.cuda.synchronize()
    value = torch.cat([ys[:, 0].float(), torch.zeros(1, device="cuda")])
    for s in range(0, MOST, piece):
        at = torch.arange(s, min(s + piece, MOST), device="cuda")
        assert torch.equal(d_gates[s:s + piece], value[at % 6] * (at % 17 - 8))


def test_two_streams_at_once():
    """Calls that share tiles over clusters and calls that do not, next to one another."""
    calls = [Ffn([40], 2048, 1544, "bf16", seed=4), Ffn([300, 7, 0, 129], 1544, 264, "f16", seed=5), Ffn([3, 1], 4096, 1544, "bf16", seed=6)]
    want = []
    for f in calls:
        f.forward()
        f.backward()
        want.append((f.ys.view.clone(), f.d_xs.view.clone(), f.d_blocks.clone()))
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for f in calls:
            for t in (f.ys.view, f.d_xs.view, f.d_blocks, f.gate_up, f.act, f.work):
                t.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(8):
            for f, s in zip(calls, streams):
                ok(rb.remoe_expert_ffn(f.R, f.N, f.H, f.I, f.code, f.xs.view, f.xs.stride, f.offsets, f.blocks, f.block, f.gate_up, f.act, f.ys.view, f.ys.stride,
                                       s.cuda_stream))
                ok(rb.remoe_expert_ffn_backward(f.R, f.N, f.H, f.I, f.code, f.xs.view, f.xs.stride, f.offsets, f.blocks, f.block, f.gate_up, f.d_ys.view,
                                                f.d_ys.stride, f.work, f.d_xs.view, f.d_xs.stride, f.d_blocks, f.block, s.cuda_stream))
        torch.cuda.synchronize()
        for f, w in zip(calls, want):
            assert all(torch.equal(a, b) for a, b in zip((f.ys.view, f.d_xs.view, f.d_blocks), w))
