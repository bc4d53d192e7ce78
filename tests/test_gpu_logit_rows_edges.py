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
