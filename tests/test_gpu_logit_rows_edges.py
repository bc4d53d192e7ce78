"""Operators on rows of logits where their arithmetic turns: lists whose probabilities do not sum to one, sums that change their
reference, the ends of the ranges that are allowed.  Against 64-bit values, through the C entry points."""
import math

import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import logit_rows_ref as ref
import test_gpu_logit_rows as rows_of

pytestmark = pytest.mark.gpu

DT, NINF, NAN, INF = rows_of.DT, rows_of.NINF, rows_of.NAN, rows_of.INF
stream, place, logprobs, run_distill = rows_of.stream, rows_of.place, rows_of.logprobs, rows_of.run_distill
CODE = {torch.float32: rb.REMOE_F32, torch.bfloat16: rb.REMOE_BF16, torch.float16: rb.REMOE_F16}


# ---- lists whose probabilities do not sum to one --------------------------------------------------------------------

def loss64(x, s, ids, y, tail):
    """The loss by its definition, entry by entry, [T] in 64 bits; differentiable in x."""
    ln_p = torch.log_softmax(x * s, 1)
    out = []
    for t in range(x.shape[0]):
        i, v = ids[t].long(), y[t].double()
        i, v = i[v > NINF], v[v > NINF]
        if not tail:
            v = v - v.logsumexp(0)
        loss = (v.exp() * (v - ln_p[t, i])).sum()
        outside = torch.ones(x.shape[1], dtype=torch.bool, device=x.device)
        outside[ids[t].long()] = False
        outside &= x[t].detach() > NINF
        q_rest = max(0.0, 1.0 - float(v.exp().sum()))
        if tail and q_rest > 0 and bool(outside.any()):
            loss = loss + q_rest * (math.log(q_rest) - ln_p[t, outside].logsumexp(0))
        out.append(loss)
    return torch.stack(out)


def uneven_lists(T, V, K, s, dtype, pad=0, offset=0, seed=3):
    """Rows with lists of K ids whose q sum to 0.6 with nothing alive outside (every fourth row from 0), to 1.7 (from 1), to 1.7
    with an id that stands there three times (from 2), and to 0.6 with others outside (from 3, where Q is 1)."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, V, generator=g) * 2
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).int()
    y = torch.log_softmax(torch.randn(T, K, generator=g), 1)
    kind = torch.arange(T) % 4
    y = (y + torch.where((kind == 0) | (kind == 3), math.log(0.6), math.log(1.7)).unsqueeze(1)).float()
    alone = torch.full((T, V), NINF).scatter_(1, ids.long(), 0.0)
    x = torch.where((kind == 0).unsqueeze(1), x + alone, x)
    if K > 2:
        twice = ids.clone()
        twice[:, 1] = twice[:, 2] = ids[:, 0]
        ids = torch.where((kind == 2).unsqueeze(1), twice, ids)
    view, _ = place(x.to(DT[dtype][0]), pad, offset)
    return view, ids.contiguous().cuda(), y.contiguous().cuda()


def three_gradients(view, s, ids, y, tail, w):
    """By the call with the loss, in place, and apart."""
    T, V = view.shape
    out, out2 = torch.full_like(view, 3.0), torch.full_like(view, 3.0)
    loss, st = run_distill(view, s, ids, y, tail, w, out, stats=True)
    assert rb.remoe_distill_topk_backward(T, V, CODE[view.dtype], view, view.stride(0), s, ids.shape[1], ids, y, st, w, out2, out2.stride(0), stream()) == 0
    same = view.clone()
    run_distill(same, s, ids, y, tail, w, same)
    return loss, {"with the loss": out, "apart": out2, "in place": same}


def close_to_loss(got, want, view, s, ids, y, tail, w):
    size = ref.distill(view, s, ids, y, tail, w)["size"]          # of the terms that the loss is made of
    ref.close(got, want, size * (ref.rel(view.shape[1]) + 4 * ref.U) + ref.U * want.abs(), "loss")


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("V,K", [(29, 4), (64, 7), (120, 12), (250, 9), (300, 5), (1000, 40)])
def test_distill_gradient_is_the_loss_s(V, K, tail):
    T, s = 8, 0.8
    view, ids, y = uneven_lists(T, V, K, s, "f32")
    w = torch.tensor([1.0, 0.5, -2.0, 1.0, 1.5, 1.0, 1.0, 0.3]).cuda()
    loss, got = three_gradients(view, s, ids, y, tail, w)
    x, h = view.double(), 1e-5
    want = torch.zeros(T, V, dtype=torch.float64, device="cuda")
    # differences along the live elements (a masked one stays masked): those of the list and some of the others
    for v in sorted(set(ids.flatten().tolist()) | set(range(0, V, max(1, V // 16)))):
        e = torch.zeros_like(x)
        e[:, v] = h
        d = (loss64(x + e, s, ids, y, tail) - loss64(x - e, s, ids, y, tail)) * w / (2 * h)
        want[:, v] = torch.where(x[:, v] > NINF, d, torch.zeros_like(d))
        # third derivatives (at most 1.7 * 2 here) times h^2 and the loss's own rounding (1e-15 * 10) over h; the float32 work on terms
        # of at most (Q p + q) s w <= 2 * 1.7 * 0.8 * 2 = 5.5, as in check_grad
        tol = 4e-9 + 5.5 * (2 * ref.rel(V) + 40 * ref.U)
        for what, o in got.items():
            alive = x[:, v] > NINF
            err = (o[:, v].double() - want[:, v])[alive].abs()
            assert bool((err <= tol).all()), (what, v, float(err.max()))
    close_to_loss(loss, loss64(x, s, ids, y, tail), view, s, ids, y, tail, w)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V,K", [(4, 3, 3), (36, 64, 8), (9, 130, 130), (6, 256, 20), (8, 257, 31), (8, 9001, 256), (5, 40007, 64), (160, 12000, 24)])
def test_distill_gradient_of_uneven_lists(T, V, K, dtype, tail):
    for pad, offset, s in [(0, 0, 1.0), (3, 1, 0.7)]:
        view, ids, y = uneven_lists(T, V, K, s, dtype, pad, offset, seed=V)
        w = (torch.rand(T, generator=torch.Generator().manual_seed(2)) + 0.5).cuda()
        loss, got = three_gradients(view, s, ids, y, tail, w)
        x = view.double().requires_grad_()
        want = loss64(x, s, ids, y, tail)
        (want * w.double()).sum().backward()
        grad = x.grad.nan_to_num(0.0).masked_fill(view == NINF, 0.0)
        size = ref.distill(view, s, ids, y, tail, w)["grad_size"]
        for what, o in got.items():
            ref.check_grad(o.masked_fill(view == NINF, 0.0), grad, size, V, what, s * 1.5)
        close_to_loss(loss, want.detach(), view, s, ids, y, tail, w)


# ---- sums that change their reference ------------------------------------------------------------------------------
# A thread's sum is kept relative to a reference that moves when an element lies 40 powers of two above it, in one of two ways to the
# exponent.  Rows in which each thread sees three levels in turn: a first one, many elements just under 40 powers of two above it
# (they do not move the reference and have nearly all of the mass), and some just over 40 above it, which do, across a boundary between
# the two ways: |m c| = 2^20, or (fp16, bf16) 160 powers of two above the type's lowest value or -2^60.

LEVELS = {  # type, inverse temperature, first level, its step from row to row, second, third (differences)
    "f32 up": ("f32", 1.0, 726802.0, 0.0625, 27.5, 28.0),
    "f32 down": ("f32", 1.0, -726830.0, 0.0625, 27.5, 28.0),
    "f32 cold": ("f32", 40.0, 18170.0, 1 / 512, 0.6875, 0.697265625),
    "f32 colder": ("f32", 1e4, 72.68, 2.0 ** -17, 0.00275, 0.00279),
    "f16": ("f16", 1 / 727, 0.0, 1.0, 20096.0, 20288.0),
    "bf16": ("bf16", 7.8e-17, 0.0, 2.0 ** 52, 3.52e17, 3.58e17),
}


def level_rows(kind, T, V, first, last):
    """[T, V]: `first` elements of the first level, the third level in the last `last` elements."""
    dtype, s, base, step, second, third = LEVELS[kind]
    x = torch.empty(T, V, dtype=torch.float64)
    low = (base + step * (torch.arange(T) % 16).double()).unsqueeze(1)
    x[:] = low + second
    x[:, :first] = low
    x[:, V - last:] = low + third
    x[:, torch.arange(V) % 7 == 3] = low
    return x.to(DT[dtype][0]).cuda(), s


def sums_tolerance(V):
    # as in rel(); and each term's exponent is taken from the reference, up to 41 powers of two away: 41 ln 2 u for its rounding, as much
    # again for the factor from the reference to the maximum
    return ref.rel(V) + 2 * 41 * ref.U


@pytest.mark.parametrize("kind", list(LEVELS))
@pytest.mark.parametrize("T,V,top", [(300, 1536, 0), (300, 6144, 5), (300, 12288, 1), (300, 18432, 0), (160, 8192, 0), (160, 36864, 3), (150, 49152, 0),
                                     (40, 24576, 7), (1, 98304, 2)])
def test_sums_across_the_two_ways(kind, T, V, top):
    half = V // 3
    for first, last in [(half, half), (half, 64), (max(64, V - 2 * 6144), 6144), (2048, 2048), (V // 4, V // 2)]:
        if first + last >= V:
            continue
        x, s = level_rows(kind, T, V, first, last)
        tok = torch.arange(T, dtype=torch.int32, device="cuda") * 37 % V
        got = logprobs(x, s, tok, top)
        want = {k: v.cpu() for k, v in ref.logprobs(x, s, tok, top).items()}
        tz, lnv = sums_tolerance(V), math.log(V + 1)
        ref.close(got["row_stats"][:, 1], want["ln_z"], tz + ref.U * 2 * lnv, "ln Z")
        ref.close(got["logprob"], want["logprob"], tz + ref.U * (8 * want["logprob"].abs() + 2 * lnv), "logprob")
        # the mean of |d| is taken from sums relative to the reference, up to 41 ln 2 = 28.4 nats away
        ref.close(got["entropy"], want["entropy"], (1 + 2 * lnv + 2 * 28.4) * tz + ref.U * 4 * lnv, "entropy")


@pytest.mark.parametrize("kind", list(LEVELS))
@pytest.mark.parametrize("T,V", [(300, 1536), (300, 6144), (300, 18432), (150, 49152), (300, 24576), (40, 24576), (1, 98304)])
def test_distill_sums_across_the_two_ways(kind, T, V):
    half = V // 3
    for first, last in [(half, half), (half, 64), (2048, 2048), (V // 4, V // 2), (max(64, V - 2 * 8192), 8192)]:
        if first + last >= V:
            continue
        x, s = level_rows(kind, T, V, first, last)
        ids = (torch.arange(4).unsqueeze(0) * (V // 4) + torch.arange(T).unsqueeze(1) % 50).int().cuda()
        y = torch.log(torch.tensor([0.4, 0.1, 0.2, 0.1])).expand(T, 4).contiguous().cuda()
        w = torch.ones(T, device="cuda")
        want = ref.distill(x, s, ids, y, 1, w)
        tol = want["size"] * (sums_tolerance(V) + 4 * ref.U) + ref.U * want["loss"].abs()
        loss, _ = run_distill(x, s, ids, y, 1, w)
        ref.close(loss, want["loss"], tol, "loss")
        out = torch.empty_like(x)
        loss, st = run_distill(x, s, ids, y, 1, w, out, stats=True)
        ref.close(loss, want["loss"], tol, "loss with the gradient")
        # by the gradient's bound, with the wider one of the sums
        fi = torch.finfo(x.dtype)
        tol = want["grad"].abs() * (fi.eps / 2) + want["grad_size"] * (2 * sums_tolerance(V) + 40 * ref.U) + fi.smallest_normal * fi.eps / 2 + 2.0 ** -126
        assert bool(((out.double() - want["grad"]).abs() <= tol).all())


# ---- the ends of what is allowed -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [40, 700, 9000])
@pytest.mark.parametrize("s", [2.0 ** -100, 2.0 ** 100])
def test_least_and_largest_inverse_temperature(V, dtype, s):
    T = 4
    view, _ = rows_of.rows(T, V, dtype, seed=V)
    view[1] = 2.0                                # uniform at any temperature
    view[2, 7] = view[2].max()                   # two largest elements share the mass of a cold row
    tok = view.argmax(1).int()
    rows_of.check_logprobs(view, s, tok, 5)
    ids, y = rows_of.teacher(view.cpu(), 5, 1.0)
    w = torch.ones(T, device="cuda")
    want = ref.distill(view, s, ids.cuda(), y.cuda(), 0, w)
    loss, _ = run_distill(view, s, ids.cuda(), y.cuda(), 0, w)
    ref.close(loss, want["loss"], want["size"] * (ref.rel(V) + 4 * ref.U) + ref.U * want["loss"].abs(), "loss")


@pytest.mark.parametrize("V", [50, 700, 20001])
def test_entropy_gradient_beside_a_bad_token(V):
    """A token outside the vocabulary has no log probability (NaN); the entropy's gradient does not look at it."""
    T = 6
    view, _ = rows_of.rows(T, V, "f32", seed=V, pad=1)
    tok = torch.tensor([V, -2, 2 ** 31 - 1, -2 ** 31, V + 3, 3], dtype=torch.int32, device="cuda")
    st = logprobs(view, 0.9, tok, 0)["row_stats"].cuda()
    g_ent = torch.tensor([1.0, 0.5, -1.0, 2.0, 1.0, 1.0], device="cuda")
    want, size = ref.logprobs_grad(view, 0.9, torch.full_like(tok, -1), None, g_ent)
    for g_lp in (None, torch.zeros(T, device="cuda")):
        out = torch.full((T, V), 3.0, device="cuda")
        assert rb.remoe_token_logprobs_backward(T, V, rb.REMOE_F32, view, view.stride(0), 0.9, tok, st, g_lp, g_ent, out, V, stream()) == 0
        ref.check_grad(out, want, size, V)
    g_lp = torch.ones(T, device="cuda")
    assert rb.remoe_token_logprobs_backward(T, V, rb.REMOE_F32, view, view.stride(0), 0.9, tok, st, g_lp, g_ent, out, V, stream()) == 0
    assert bool(torch.isnan(out[:5]).all()) and bool(torch.isfinite(out[5]).all())


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("V", [20, 64, 100, 256, 300, 20000])
def test_faint_probabilities_of_the_teacher(V, tail):
    """q below float32's least normal value is a probability all the same: a student that masks its token has an infinite loss, and
    one that gives the token the type's lowest value a large one."""
    T = 6
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(V)).cuda()
    ids = torch.arange(3, dtype=torch.int32).expand(T, 3).contiguous().cuda()
    y = torch.tensor([[0.4, 0.3, 0.0]]).log().expand(T, 3).clone()
    y[:, 2] = torch.tensor([-90.0, -90.0, -700.0, -88.0, -800.0, NINF])
    x[0, 2], x[2, 2], x[4, 2], x[5, 2] = NINF, NINF, NINF, NINF
    x[3, 2] = torch.finfo(torch.float32).min
    w, y = torch.ones(T, device="cuda"), y.cuda()
    want = ref.distill(x, 1.0, ids, y, tail, w)
    assert bool(torch.isinf(want["loss"][[0, 2]]).all()) and bool(torch.isfinite(want["loss"][[1, 3, 4, 5]]).all()) and want["loss"][3] > 2
    out = torch.empty_like(x)
    for o in (None, out):
        loss, _ = run_distill(x, 1.0, ids, y, tail, w, o)
        ref.close(loss, want["loss"], want["size"].nan_to_num(0, posinf=0) * (ref.rel(V) + 4 * ref.U), "loss")
    ref.check_grad(out, want["grad"], want["grad_size"], V)


def test_a_failed_allocation_is_not_the_next_call_s():
    """A stack too large for the device is refused; calls after it report their own outcome."""
    T = 3
    for V, K in [(40, 4), (700, 4), (9000, 4)]:
        x, _ = rows_of.rows(T, V, "bf16")
        tok = torch.zeros(T, dtype=torch.int32, device="cuda")
        lp, one = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")
        st, ds, d = torch.zeros(T, 4, device="cuda"), torch.zeros(T, 8, device="cuda"), torch.zeros_like(x)
        ids, y = torch.zeros(T, K, dtype=torch.int32, device="cuda"), torch.zeros(T, K, device="cuda")
        code = rb.REMOE_BF16
        calls = [
            lambda: rb.remoe_token_logprobs(T, V, code, x, V, 1.0, tok, K, lp, None, ids, y, st, stream()),
            lambda: rb.remoe_token_logprobs_backward(T, V, code, x, V, 1.0, tok, st, one, None, d, V, stream()),
            lambda: rb.remoe_distill_topk(T, V, code, x, V, 1.0, K, ids, y, 1, None, lp, ds, None, 0, stream()),
            lambda: rb.remoe_distill_topk(T, V, code, x, V, 1.0, K, ids, y, 1, None, lp, ds, d, V, stream()),
            lambda: rb.remoe_distill_topk_backward(T, V, code, x, V, 1.0, K, ids, y, ds, one, d, V, stream()),
        ]
        shape = dict(n_layers=64, hidden=1024, n_routed=256, top_k=4, inter_routed=8192, n_shared=0, inter_shared=0, shared_gate=0,
                     renorm_topk=0, weight_dtype=rb.REMOE_F32, batch=1)
        for call in calls:
            assert rb.remoe_stack_create(shape, 256)[0] == rb.REMOE_E_NOMEM      # 1.6 TB of slots
            assert call() == rb.REMOE_OK
        torch.cuda.synchronize()


@pytest.mark.parametrize("V", [40, 700, 33000])
def test_log_probabilities_of_far_apart_logits(V):
    """Two finite logits whose difference is beyond float32 have a log probability that is not."""
    T, s = 160, 0.25
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(V))
    x[:, 3] = 3e38
    x[:, 5] = -3e38
    view, _ = place(x)
    tok = torch.full((T,), 5, dtype=torch.int32, device="cuda")
    for n in (T, 2):
        got = rows_of.check_logprobs(view[:n], s, tok[:n], min(V, 40))
        assert bool((got["logprob"] < -1.49e38).all()) and bool(torch.isfinite(got["logprob"]).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V,K", [(5, 61, 6), (4, 250, 20), (3, 2033, 31), (3, 20001, 64), (150, 9001, 16)])
def test_distill_in_place_leaves_the_gaps(T, V, K, dtype):
    view, flat = rows_of.rows(T, V, dtype, seed=V, pad=5, offset=3)
    ids, y = rows_of.teacher(view.cpu(), K, 0.9)
    ids, y, w = ids.cuda(), y.cuda(), torch.ones(T, device="cuda")
    before = flat.clone()
    out = torch.empty(T, V, dtype=view.dtype, device="cuda")
    _, st = run_distill(view, 0.9, ids, y, 1, w, out, stats=True)
    assert torch.equal(flat, before)
    run_distill(view, 0.9, ids, y, 1, w, view)
    rows_of.untouched(view, flat, before)
    view.copy_(before[3:3 + T * (V + 5)].view(T, V + 5)[:, :V])
    assert rb.remoe_distill_topk_backward(T, V, CODE[view.dtype], view, view.stride(0), 0.9, K, ids, y, st, w, view, view.stride(0), stream()) == 0
    rows_of.untouched(view, flat, before)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T", [1, 149])
def test_the_longest_rows(T, dtype):
    V, K, s = rb.REMOE_ROWS_MAX_VOCAB, rb.REMOE_ROWS_MAX_TOP, 0.9
    g = torch.Generator(device="cuda").manual_seed(T)
    flat = torch.full((3 + T * (V + 1) + 16,), 777.0, dtype=DT[dtype][0], device="cuda")
    view = flat[3:3 + T * (V + 1)].view(T, V + 1)[:, :V]
    for t in range(T):
        view[t] = torch.randn(V, generator=g, device="cuda") * 3
    tok = torch.arange(T, dtype=torch.int32, device="cuda") * 2609 % V
    tok[0] = V - 1
    code, before = DT[dtype][1], flat.clone()
    few = [0] if T == 1 else [0, 1, T // 2, T - 1]          # rows that are compared
    part, ptok = view[few], tok[few]
    tz, lnv = ref.rel(V), math.log(V + 1)
    want = {k: v.cpu() for k, v in ref.logprobs(part, s, ptok, K).items()}
    for top in (K, 0):
        got = logprobs(view, s, tok, top)
        ref.close(got["logprob"][few], want["logprob"], tz + ref.U * (8 * want["logprob"].abs() + 2 * lnv), "logprob")
        ref.close(got["entropy"][few], want["entropy"], (1 + 2 * lnv) * tz + ref.U * 4 * lnv, "entropy")
        if top:
            assert torch.equal(got["top_ids"][few], want["top_ids"])
            ids, y = got["top_ids"].cuda(), got["top_logprobs"].cuda()
    g_lp, g_ent = torch.ones(T, device="cuda"), torch.full((T,), 0.5, device="cuda")
    out = torch.full((T, V), 3.0, dtype=view.dtype, device="cuda")
    stats = got["row_stats"].cuda()
    assert rb.remoe_token_logprobs_backward(T, V, code, view, view.stride(0), s, tok, stats, g_lp, g_ent, out, V, stream()) == 0
    dx, size = ref.logprobs_grad(part, s, ptok, g_lp[few], g_ent[few])
    ref.check_grad(out[few], dx, size, V, "log probabilities")
    # a teacher: the rows' own records, a little flatter, so that there is a divergence
    y = (y * 0.9 - 0.5).contiguous()
    w = torch.ones(T, device="cuda")
    want = ref.distill(part, s, ids[few], y[few], 1, w[few])
    tol = want["size"] * (ref.rel(V) + 4 * ref.U) + ref.U * want["loss"].abs()
    loss, _ = run_distill(view, s, ids, y, 1, w)
    ref.close(loss[few], want["loss"], tol, "loss")
    loss, st = run_distill(view, s, ids, y, 1, w, out, stats=True)
    ref.close(loss[few], want["loss"], tol, "loss with the gradient")
    ref.check_grad(out[few], want["grad"], want["grad_size"], V, "gradient with the loss", s)
    assert rb.remoe_distill_topk_backward(T, V, code, view, view.stride(0), s, K, ids, y, st, w, out, V, stream()) == 0
    ref.check_grad(out[few], want["grad"], want["grad_size"], V, "gradient apart", s)
    assert torch.equal(flat, before)
    run_distill(view, s, ids, y, 1, w, view)
    rows_of.untouched(view, flat, before)


# ---- precision as it is, beside the worst case ---------------------------------------------------------------------

@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("T,V,K", [(512, 64, 64), (512, 64, 16), (300, 250, 32), (64, 1021, 32), (64, 32003, 64), (256, 151936, 64)])
def test_root_mean_square_errors(T, V, K, tail):
    """The worst case of rel() adds up what in earnest averages out.  What does not: the exponential's own error (at most 4 u, one
    sign at worst), that of log2(e) / temperature (1.2 u on a mean distance of about 5), and a rounding or two of a logarithm: 4 + 6 + 3 u.
    Sixteen u for ln Z, and for the divergence from a teacher so near that the true one is of that size itself."""
    g = torch.Generator().manual_seed(V + K)
    x = (torch.randn(T, V, generator=g) * 2.5 + torch.randn(T, 1, generator=g) * 4).cuda()
    tok = x.argmax(1).int()
    got, want = logprobs(x, 0.9, tok, 0), ref.logprobs(x, 0.9, tok, 0)

    def rms(a, b):
        return float((a.double().cpu() - b.cpu()).square().mean().sqrt())

    assert rms(got["row_stats"][:, 1], want["ln_z"]) <= 16 * ref.U
    t = torch.log_softmax((x + torch.randn(T, V, generator=g).cuda() * 1e-4).double() * 0.9, 1).topk(K, 1)
    ids, y, w = t.indices.int(), t.values.float(), torch.ones(T, device="cuda")
    want = ref.distill(x, 0.9, ids, y, tail, w)["loss"]
    assert rms(run_distill(x, 0.9, ids, y, tail, w)[0], want) <= 16 * ref.U
    assert rms(run_distill(x, 0.9, ids, y, tail, w, torch.empty_like(x))[0], want) <= 16 * ref.U
