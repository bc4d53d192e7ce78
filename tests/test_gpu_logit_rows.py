"""Operators on rows of logits against their 64-bit values (logit_rows_ref), at the sizes, layouts and masks where they
can go wrong, through the C entry points."""
import math

import pytest
import torch

from paper_2605_27081_b200 import binding as rb
import logit_rows_ref as ref

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, rb.REMOE_F32), "bf16": (torch.bfloat16, rb.REMOE_BF16), "f16": (torch.float16, rb.REMOE_F16)}
NINF, NAN, INF = float("-inf"), float("nan"), float("inf")


def stream():
    return torch.cuda.current_stream().cuda_stream


def rows(T, V, dtype, seed=0, pad=0, offset=0, scale=3.0):
    """Rows on the GPU, `pad` elements between them, the first `offset` elements behind an aligned address; canaries around."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, V, generator=g) * scale).to(DT[dtype][0])
    return place(x, pad, offset)


def place(x, pad=0, offset=0):
    T, V = x.shape
    flat = torch.full((offset + T * (V + pad) + 16,), 777.0, dtype=x.dtype, device="cuda")
    view = flat[offset:offset + T * (V + pad)].view(T, V + pad)[:, :V]
    view.copy_(x)
    return view, flat


def untouched(view, flat, before):
    """Nothing of `flat` outside `view` has changed."""
    mask = torch.ones_like(flat, dtype=torch.bool)
    T, V = view.shape
    off = view.storage_offset()
    idx = off + torch.arange(T, device="cuda").unsqueeze(1) * view.stride(0) + torch.arange(V, device="cuda")
    mask[idx.flatten()] = False
    assert torch.equal(flat[mask], before[mask])


def logprobs(view, s, tokens, top, stats=True):
    T, V = view.shape
    code = {torch.float32: rb.REMOE_F32, torch.bfloat16: rb.REMOE_BF16, torch.float16: rb.REMOE_F16}[view.dtype]
    out = dict(logprob=torch.full((T,), 55.0, device="cuda"), entropy=torch.full((T,), 55.0, device="cuda"),
               row_stats=torch.full((T, 4), 55.0, device="cuda") if stats else None,
               top_ids=torch.full((T, top), -7, dtype=torch.int32, device="cuda") if top else None,
               top_logprobs=torch.full((T, top), 55.0, device="cuda") if top else None)
    rc = rb.remoe_token_logprobs(T, V, code, view, view.stride(0), s, tokens, top, out["logprob"], out["entropy"], out["top_ids"],
                                 out["top_logprobs"], out["row_stats"], stream())
    assert rc == 0, rb.strerror(rc)
    torch.cuda.synchronize()
    return {k: v.cpu() if v is not None else None for k, v in out.items()}


def check_logprobs(view, s, tokens, top):
    V = view.shape[1]
    got, want = logprobs(view, s, tokens, top), {k: v.cpu() for k, v in ref.logprobs(view, s, tokens, top).items()}
    tz, lnv = ref.rel(V), math.log(V + 1)
    ref.close(got["logprob"], want["logprob"], tz + ref.U * (8 * want["logprob"].abs() + 2 * lnv), "logprob")
    ref.close(got["entropy"], want["entropy"], (1 + 2 * lnv) * tz + ref.U * 4 * lnv, "entropy")
    st = got["row_stats"]
    whole = ~want["broken"]
    ref.close(st[whole][:, 0], want["max"][whole], 0.0, "max")
    ref.close(st[whole][:, 1], want["ln_z"][whole], tz + ref.U * 2 * lnv, "ln Z")
    assert torch.equal(st[:, 2].nan_to_num(9.0), got["entropy"].nan_to_num(9.0)) and torch.equal(st[:, 3].nan_to_num(9.0), got["logprob"].nan_to_num(9.0))
    if top:
        assert torch.equal(got["top_ids"], want["top_ids"])
        ref.close(got["top_logprobs"], want["top_logprobs"], tz + ref.U * (8 * want["top_logprobs"].abs().nan_to_num(0, posinf=0) + 2 * lnv), "top")
    return got


def tokens_for(T, V, seed=1, skip=0.2):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (T,), generator=g)
    return torch.where(torch.rand(T, generator=g) < skip, torch.full_like(t, -1), t).int().cuda()


# lengths: one element, within one unit, group of 8 lanes, of 32, one block of 128 threads, of 512, several parts of a row
SIZES = [(1, 1), (3, 2), (5, 7), (33, 64), (7, 65), (37, 128), (18, 129), (9, 255), (9, 256), (3, 257),
         (5, 1000), (2, 1021), (4, 4099), (3, 8192), (2, 12345), (1, 40007), (5, 33001), (300, 300)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V", SIZES)
def test_logprobs_sizes(T, V, dtype):
    for pad, offset, s in [(0, 0, 1.0), (1, 3, 0.7), (8, 8, 2.0)]:
        view, _ = rows(T, V, dtype, seed=V, pad=pad, offset=offset)
        top = min(V, 1 + (T * 7 + V) % 23)
        check_logprobs(view, s, tokens_for(T, V), top)
        check_logprobs(view, s, tokens_for(T, V), 0)


# rows enough for the persistent blocks: fewer rows than blocks, more, several a block; rows shorter than the ring, longer
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V,top", [(148, 8192, 0), (150, 9001, 1), (297, 12288, 256), (700, 8199, 30), (160, 33001, 64), (310, 65536, 20), (149, 150001, 100), (150, 40009, 256), (148, 131072, 255)])
def test_logprobs_many_rows(T, V, top, dtype):
    for pad, offset, s in [(0, 0, 1.0), (1, 3, 0.7)]:
        view, _ = rows(T, V, dtype, seed=V, pad=pad, offset=offset)
        sp = special_rows(V, view.dtype)
        view[5:5 + sp.shape[0]] = sp.cuda()
        view[-sp.shape[0]:] = sp.cuda()
        view[30, 7] = NAN
        view[31, V - 1] = INF
        view[32, (torch.arange(V, device="cuda") // 8) % 512 < 200] += 40
        check_logprobs(view, s, tokens_for(T, V), top)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V,top", [(1, 8192, 32), (200, 16001, 32), (200, 16001, 33), (3, 32767, 32), (700, 9001, 1), (160, 26700, 20)])
def test_few_alternatives_of_middling_rows(T, V, top, dtype):
    view, _ = rows(T, V, dtype, seed=T + top, pad=1)
    check_logprobs(view, 0.8, tokens_for(T, V), top)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V,top", [(64, 64), (200, 200), (256, 256), (300, 256), (1500, 65), (2000, 256), (5000, 64), (9001, 256), (70000, 256), (70000, 1)])
def test_many_alternatives(V, top, dtype):
    for T in (1, 4):
        view, _ = rows(T, V, dtype, seed=top, pad=5)
        check_logprobs(view, 1.0, tokens_for(T, V), top)


def special_rows(V, dtype, seed=3):
    """Rows whose masks leave nothing, one or few elements; the type's lowest value; equal elements; sorted rows."""
    g = torch.Generator().manual_seed(seed)
    low = torch.finfo(dtype).min
    x = torch.randn(14, V, generator=g) * 3
    x[0] = NINF
    x[1] = low
    x[2] = 0.0
    x[3] = NINF
    x[3, V - 1] = -5.0
    x[4] = NINF
    x[4, [V // 3, V // 2, 1]] = torch.tensor([1.0, 2.0, 2.0])
    x[5, torch.rand(V, generator=g) < 0.9] = low
    x[6, torch.rand(V, generator=g) < 0.5] = NINF
    x[7] = torch.arange(V) / V * 20
    x[8] = -torch.arange(V) / V * 20
    x[9] = (torch.arange(V) % 3).float()
    x[10] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    x[11, V // 2] = 60.0                      # nearly all of the mass on one
    x[12] = NINF
    x[12, : V // 2] = low
    x[13] = torch.finfo(dtype).max / 2
    return x.to(dtype)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [17, 64, 250, 1025, 9000, 40003])
def test_masked_and_equal_rows(V, dtype):
    x = special_rows(V, DT[dtype][0])
    view, _ = place(x, pad=1)
    tok = torch.full((x.shape[0],), V // 2, dtype=torch.int32, device="cuda")
    check_logprobs(view, 1.0, tok, min(V, 16))
    check_logprobs(view, 1.5, tok, min(V, 200))
    for r in range(x.shape[0]):               # each row alone: split over several blocks where it is long
        check_logprobs(view[r:r + 1], 0.5, tok[:1], min(V, 9))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [4096 * 3, 4096 * 9])
def test_large_elements_in_few_threads(V, dtype):
    # every 4096th group of eight holds the row's large elements: the threads' maxima say little, the exact scan decides
    x = torch.randn(2, V, generator=torch.Generator().manual_seed(1))
    x[:, (torch.arange(V) // 8) % 512 < 200] += 40
    x[1] = x[1].round()
    view, _ = place(x.to(DT[dtype][0]))
    check_logprobs(view, 0.1, tokens_for(2, V, skip=0), 256)
    check_logprobs(view[:1], 0.1, tokens_for(1, V, skip=0), 201)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [50, 700, 20000])
def test_nan_inf_and_bad_tokens(V, dtype):
    x, _ = rows(6, V, dtype)
    x = x.cpu().clone()
    x[0, V // 2] = NAN
    x[1, 3] = INF
    x[2, V - 1] = INF
    x[2, 0] = INF
    x[3, V - 1] = NAN
    view, _ = place(x, pad=3)
    got = check_logprobs(view, 1.0, torch.tensor([1, 3, 0, 1, V, -2], dtype=torch.int32).cuda(), 4)
    assert torch.isnan(got["logprob"]).all() and not torch.isnan(got["entropy"][4:]).any()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [60, 33000])
def test_confident_rows(V, dtype):
    # p of the token from 1 - 1e-12 to 1 - 1e-2: its log probability is -(1 - p) and has to keep its digits
    gap = torch.linspace(5, 30, 16) + math.log(V)
    x = torch.zeros(16, V)
    x[:, 5] = gap
    x = x.to(DT[dtype][0])
    view, _ = place(x)
    tok = torch.full((16,), 5, dtype=torch.int32, device="cuda")
    got = logprobs(view, 1.0, tok, 0)
    lp = -torch.log1p((V - 1) * (-(x[:, 5].double())).exp())
    # relative: the exponentials and the sum of equal terms, as in rel(); |d| is up to 41 here
    tol = lp.abs() * (ref.rel(V) + 3 * 41 * ref.U + 4 * ref.U)
    assert bool(((got["logprob"].double() - lp).abs() <= tol).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [100, 3001, 20000])
@pytest.mark.parametrize("s", [1e-30, 1e-4, 2e-3, 40.0, 1e5, 1e25])
def test_temperatures(V, dtype, s):
    x, _ = rows(4, V, dtype, scale=5.0)
    x[0, ::3] = NINF
    x[1] = torch.finfo(x.dtype).min               # lowest values beside masked ones
    x[1, ::2] = NINF
    x[1, :2000] = NINF
    x[1, V - 1] = torch.finfo(x.dtype).min
    x[2, ::2] *= 1000
    check_logprobs(x, s, tokens_for(4, V, skip=0), 9)
    for r in range(4):
        check_logprobs(x[r:r + 1], s, tokens_for(1, V, skip=0), 9)


GRAD_SIZES = [(1, 1), (4, 2), (3, 9), (40, 64), (6, 130), (5, 256), (5, 257), (3, 2033), (3, 2041), (2, 8200), (2, 20001)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V", GRAD_SIZES)
@pytest.mark.parametrize("which", ["both", "logprob", "entropy"])
def test_logprobs_backward(T, V, dtype, which):
    for pad, offset, dpad, doff, s in [(0, 0, 0, 0, 1.0), (3, 1, 3, 1, 0.7), (0, 0, 5, 2, 1.4), (1, 0, 1, 1, 1.0)]:
        view, flat = rows(T, V, dtype, seed=T + V, pad=pad, offset=offset)
        if V > 8:
            view[:, 4] = NINF
        out, oflat = place(torch.zeros(T, V, dtype=view.dtype), dpad, doff)
        tok = tokens_for(T, V)
        g = torch.Generator().manual_seed(9)
        g_lp = torch.randn(T, generator=g).cuda() if which != "entropy" else None
        g_ent = torch.randn(T, generator=g).cuda() if which != "logprob" else None
        stats = logprobs(view, s, tok, 0)["row_stats"].cuda()
        before, obefore = flat.clone(), oflat.clone()
        args = (T, V, DT[dtype][1], view, view.stride(0), s, tok, stats, g_lp, g_ent)
        assert rb.remoe_token_logprobs_backward(*args, out, out.stride(0), stream()) == 0
        want, size = ref.logprobs_grad(view.cpu(), s, tok.cpu(), None if g_lp is None else g_lp.cpu(), None if g_ent is None else g_ent.cpu())
        ref.check_grad(out.cpu(), want, size, V, (pad, offset, dpad, doff))
        assert torch.equal(flat, before)
        untouched(out, oflat, obefore)
        assert rb.remoe_token_logprobs_backward(*args, view, view.stride(0), stream()) == 0     # in place
        assert torch.equal(view, out)
        untouched(view, flat, before)


def test_logprobs_gradient_against_differences():
    T, V, s = 4, 37, 0.8
    x, _ = rows(T, V, "f32", scale=1.0)
    tok = tokens_for(T, V, skip=0)
    g_lp, g_ent = torch.randn(T).cuda(), torch.randn(T).cuda()
    stats = logprobs(x, s, tok, 0)["row_stats"].cuda()
    dx = torch.empty_like(x)
    assert rb.remoe_token_logprobs_backward(T, V, rb.REMOE_F32, x, x.stride(0), s, tok, stats, g_lp, g_ent, dx, V, stream()) == 0

    def objective(y):
        r = ref.logprobs(y, s, tok.cpu(), 0)
        return (r["logprob"] * g_lp.cpu().double() + r["entropy"] * g_ent.cpu().double())

    h, x64 = 1e-5, x.cpu().double()
    for v in range(V):
        e = torch.zeros_like(x64)
        e[:, v] = h
        diff = (objective(x64 + e) - objective(x64 - e)) / (2 * h)
        # the difference's own error: third derivatives (of order 10 |g|) times h^2, and 1e-15 * 10 / h
        assert bool(((dx[:, v].cpu().double() - diff).abs() <= 2e-8 + 1e-6).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [17, 250, 1025, 9000])
def test_backward_of_masked_rows(V, dtype):
    x = special_rows(V, DT[dtype][0])
    view, _ = place(x)
    T = x.shape[0]
    tok = torch.full((T,), V // 2, dtype=torch.int32, device="cuda")
    g_lp, g_ent = torch.ones(T, device="cuda"), torch.full((T,), 0.5, device="cuda")
    stats = logprobs(view, 1.0, tok, 0)["row_stats"].cuda()
    out = torch.full_like(view, 3.0)
    assert rb.remoe_token_logprobs_backward(T, V, DT[dtype][1], view, view.stride(0), 1.0, tok, stats, g_lp, g_ent, out, out.stride(0), stream()) == 0
    want, size = ref.logprobs_grad(x, 1.0, tok.cpu(), g_lp.cpu(), g_ent.cpu())
    # rows whose token has no probability at all (masked): ln p = -inf has the gradient of the formula all the same
    ref.check_grad(out.cpu(), want, size, V)


def test_backward_leaves_out_and_poisons():
    T, V = 5, 600
    x, _ = rows(T, V, "bf16")
    x[0, 7] = NAN                              # left out by its token, no entropy gradient: zeros all the same
    x[3, 5] = NAN
    tok = torch.tensor([-1, 4, V, 2, -2], dtype=torch.int32).cuda()
    stats = logprobs(x, 1.0, tok, 0)["row_stats"].cuda()
    out = torch.full_like(x, 3.0)
    g = torch.ones(T, device="cuda")
    assert rb.remoe_token_logprobs_backward(T, V, rb.REMOE_BF16, x, V, 1.0, tok, stats, g, None, out, V, stream()) == 0
    assert bool((out[0] == 0).all()) and bool(torch.isfinite(out[1]).all())
    assert bool(torch.isnan(out[2:]).all())


# ---- distillation ---------------------------------------------------------------------------------------------------

def teacher(x, K, s, seed=5, kind="near"):
    """ids [T, K] and log probabilities of a teacher near the student, on the CPU."""
    g = torch.Generator().manual_seed(seed)
    t = torch.log_softmax((x.cuda().double() + torch.randn(x.shape, generator=g).cuda().double()) * s, 1)
    v, i = t.topk(K, 1)
    return i.int().cpu().contiguous(), v.float().cpu().contiguous()


def run_distill(view, s, ids, y, tail, weight, out=None, stats=False):
    T, V = view.shape
    code = {torch.float32: rb.REMOE_F32, torch.bfloat16: rb.REMOE_BF16, torch.float16: rb.REMOE_F16}[view.dtype]
    loss = torch.full((T,), 55.0, device="cuda")
    st = torch.full((T, 8), 55.0, device="cuda") if stats else None
    rc = rb.remoe_distill_topk(T, V, code, view, view.stride(0), s, ids.shape[1], ids, y, tail, weight, loss, st, out,
                               out.stride(0) if out is not None else 0, stream())
    assert rc == 0, rb.strerror(rc)
    return loss, st


def check_distill(view, s, ids, y, tail, weight, oplace=(0, 0)):
    T, V = view.shape
    ids, y, weight = ids.cuda(), y.cuda(), weight.cuda()
    want = ref.distill(view, s, ids, y, tail, weight)
    factor = s * float(weight.abs().max())
    code = {torch.float32: rb.REMOE_F32, torch.bfloat16: rb.REMOE_BF16, torch.float16: rb.REMOE_F16}[view.dtype]
    tol = want["size"].nan_to_num(0, posinf=0) * (ref.rel(V) + 4 * ref.U) + ref.U * want["loss"].abs().nan_to_num(0, posinf=0)
    loss, _ = run_distill(view, s, ids, y, tail, weight)
    ref.close(loss, want["loss"], tol, "loss")
    out, flat = place(torch.zeros(T, V, dtype=view.dtype), *oplace)
    before = flat.clone()
    loss2, st = run_distill(view, s, ids, y, tail, weight, out, stats=True)
    ref.close(loss2, want["loss"], tol, "loss with the gradient")      # summed in another order than without: not the same bits
    ref.check_grad(out, want["grad"], want["grad_size"], V, "gradient with the loss", factor)
    untouched(out, flat, before)
    out2, flat2 = place(torch.zeros(T, V, dtype=view.dtype), *oplace)
    assert rb.remoe_distill_topk_backward(T, V, code, view, view.stride(0), s, ids.shape[1], ids, y, st, weight, out2, out2.stride(0), stream()) == 0
    ref.check_grad(out2, want["grad"], want["grad_size"], V, "gradient apart", factor)
    untouched(out2, flat2, before)
    for apart in (False, True):                    # in place
        again = view.clone(memory_format=torch.preserve_format)
        big, bflat = place(view.cpu(), view.stride(0) - V if T > 1 else 0, view.storage_offset())
        if apart:
            assert rb.remoe_distill_topk_backward(T, V, code, big, big.stride(0), s, ids.shape[1], ids, y, st, weight, big, big.stride(0), stream()) == 0
            assert torch.equal(big, out2)
        else:
            run_distill(big, s, ids, y, tail, weight, big)
            assert torch.equal(big, out)
        assert torch.equal(again, view)
    return loss.cpu(), out


DISTILL_SIZES = [(1, 1, 1), (3, 2, 1), (2, 9, 9), (40, 64, 64), (33, 64, 6), (6, 65, 65), (37, 128, 20), (6, 130, 8),
                 (5, 256, 256), (5, 257, 256), (3, 1021, 31), (2, 4099, 64), (2, 9000, 256), (1, 40007, 100), (3, 33001, 20)]


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V,K", DISTILL_SIZES)
def test_distill_sizes(T, V, K, dtype, tail):
    for pad, offset, oplace, s in [(0, 0, (0, 0), 1.0), (1, 3, (1, 3), 0.7), (5, 0, (2, 1), 1.5)]:
        view, _ = rows(T, V, dtype, seed=V + K, pad=pad, offset=offset)
        ids, y = teacher(view.cpu(), K, s)
        weight = torch.rand(T, generator=torch.Generator().manual_seed(2)) + 0.5
        weight[::3] *= -1 if T > 2 else 1
        if T > 1:
            weight[1] = 0.0
        check_distill(view, s, ids, y, tail, weight, oplace)


# rows enough for the persistent blocks: rows of one chunk, of fewer chunks than the ring has, of more; several rows a block
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,V,K", [(148, 8192, 1), (150, 9001, 256), (700, 8199, 30), (1300, 8192, 5), (160, 33001, 64), (310, 65536, 20), (149, 150001, 100), (900, 20011, 33)])
def test_distill_many_rows(T, V, K, dtype, tail):
    for pad, offset, oplace, s in [(0, 0, (0, 0), 1.0), (1, 3, (1, 3), 0.7), (5, 0, (2, 1), 1.5)]:
        view, _ = rows(T, V, dtype, seed=V + K, pad=pad, offset=offset)
        sp = special_rows(V, view.dtype)
        g = torch.Generator().manual_seed(6)
        ids, y = teacher(view.cpu(), K, s)
        weight = torch.rand(T, generator=g) + 0.5
        weight[torch.rand(T, generator=g) < 0.3] = 0.0
        weight[::7] *= -1
        view[3:3 + sp.shape[0]] = sp.cuda()
        view[-sp.shape[0]:] = sp.cuda()
        ids[20, 0] = V - 1                              # the ends of a row
        ids[21:25, K - 1] = 0
        if K > 4:
            ids[30:60, 1] = -1
            ids[40:70, 3] = ids[40:70, 2]               # an id twice
            ids[50] = -1
        check_distill(view, s, ids, y, tail, weight, oplace)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [17, 64, 250, 1025, 9000, 40003])
def test_distill_masks_and_lists(V, dtype, tail):
    """Masked students, lists with unused entries, an id twice, values of -inf, in any order."""
    x = special_rows(V, DT[dtype][0])
    T, K = x.shape[0], 8
    view, _ = place(x, pad=1)
    g = torch.Generator().manual_seed(4)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).int()
    y = torch.log_softmax(torch.randn(T, K + 1, generator=g), 1)[:, :K].float().contiguous()
    ids[:, 2] = -1                                  # unused entries, anything for a value
    y[:, 2] = 3.0
    ids[5:, 6] = ids[5:, 0]                         # an id twice, and three times
    ids[8:, 7] = ids[8:, 0]
    y[6, 3] = NINF                                  # a token that the teacher rules out
    ids[9] = -1                                     # no list at all
    y[10] = NINF
    w = torch.ones(T)
    # a list's token that the student masks gives an infinite loss and a finite gradient
    loss, _ = check_distill(view, 1.0, ids, y, tail, w)
    assert loss[9] == 0 and loss[10] == 0 and loss[0] == 0
    for r in range(T):
        check_distill(view[r:r + 1], 1.0, ids[r:r + 1].contiguous(), y[r:r + 1].contiguous(), tail, w[:1])


@pytest.mark.parametrize("V", [64, 700, 20000])
def test_distill_where_little_is_left_outside(V):
    # the student has all but 1e-9 .. 1e-3 of its mass on the list, the teacher leaves 1 % outside
    x = torch.randn(6, V, generator=torch.Generator().manual_seed(1))
    x[:, :4] += torch.linspace(8, 22, 6).unsqueeze(1) + math.log(V)
    ids = torch.arange(4, dtype=torch.int32).expand(6, 4).contiguous()
    y = torch.full((6, 4), math.log(0.99 / 4))
    view, _ = place(x)
    check_distill(view, 1.0, ids, y, 1, torch.ones(6))


@pytest.mark.parametrize("dtype", list(DT))
def test_distill_poison_many_rows(dtype):
    T, V = 400, 12000
    x, _ = rows(T, V, dtype, pad=1)
    ids = torch.randint(0, V, (T, 4), generator=torch.Generator().manual_seed(2)).int()
    y = torch.log(torch.full((T, 4), 0.2))
    x[10, 9] = NAN
    x[11, ids[11, 0].item()] = NAN
    x[12, V - 1] = INF
    x[13, ids[13, 2].item()] = INF
    ids[14, 1] = V
    ids[15, 0] = -5
    y[16, 3] = NAN
    y[17, 3] = INF
    w = torch.ones(T)
    x[300:310, 7] = NAN
    w[300:310] = 0.0
    ids, y, w = ids.cuda(), y.cuda(), w.cuda()
    out = torch.full((T, V), 3.0, dtype=x.dtype, device="cuda")
    for o in (None, out):
        loss, st = run_distill(x, 1.0, ids, y, 1, w, o, stats=True)
        assert bool(torch.isnan(loss[10:18]).all()) and bool((loss[300:310] == 0).all())
        fine = torch.ones(T, dtype=torch.bool, device="cuda")
        fine[10:18] = False
        assert bool(torch.isfinite(loss[fine]).all())
    out2 = torch.full_like(out, 3.0)
    assert rb.remoe_distill_topk_backward(T, V, DT[dtype][1], x, x.stride(0), 1.0, 4, ids, y, st, w, out2, V, stream()) == 0
    for o in (out, out2):
        assert bool(torch.isnan(o[10:18]).all()) and bool((o[300:310] == 0).all()) and bool(torch.isfinite(o[fine]).all())


@pytest.mark.parametrize("V", [40, 600, 20000])
def test_distill_poison(V):
    x, _ = rows(7, V, "f32")
    x[0, 9] = NAN
    x[1, 3] = INF
    x[5, 9] = NAN
    ids = torch.tensor([[1, 2]] * 7, dtype=torch.int32)
    y = torch.log(torch.tensor([[0.5, 0.25]] * 7))
    ids[2, 1] = V
    ids[3, 0] = -2
    y[4, 0] = NAN
    w = torch.ones(7)
    w[5] = 0.0                                      # left out: its NaN is not looked at
    out = torch.full_like(x, 3.0)
    ids, y, w = ids.cuda(), y.cuda(), w.cuda()
    loss, st = run_distill(x, 1.0, ids, y, 1, w, out, stats=True)
    out2 = torch.full_like(x, 3.0)
    assert rb.remoe_distill_topk_backward(7, V, rb.REMOE_F32, x, V, 1.0, 2, ids, y, st, w, out2, V, stream()) == 0
    for o in (out, out2):
        assert bool(torch.isnan(o[:5]).all()) and bool((o[5] == 0).all()) and bool(torch.isfinite(o[6]).all())
    assert bool(torch.isnan(loss[:5]).all()) and loss[5] == 0 and math.isfinite(loss[6])


@pytest.mark.parametrize("tail", [0, 1])
def test_distill_gradient_against_differences(tail):
    T, V, s = 3, 29, 0.8
    x, _ = rows(T, V, "f32", scale=1.0)
    ids, y = teacher(x.cpu(), 5, s)
    w = torch.tensor([1.0, 0.5, -2.0])
    dx = torch.empty_like(x)
    run_distill(x, s, ids.cuda(), y.cuda(), tail, w.cuda(), dx)
    h, x64 = 1e-5, x.cpu().double()
    for v in range(V):
        e = torch.zeros_like(x64)
        e[:, v] = h
        diff = (ref.distill(x64 + e, s, ids, y, tail, w)["loss"] - ref.distill(x64 - e, s, ids, y, tail, w)["loss"]) * w / (2 * h)
        # third derivatives (of order one) times h^2 and 1e-15 * 10 / h; the kernel's own float32 error
        assert bool(((dx[:, v].cpu().double() - diff).abs() <= 2e-8 + 1e-6).all())


# ---- calls as programs make them ----------------------------------------------------------------------------------

def test_teacher_to_student():
    """A teacher's alternatives recorded by one operator are the list of the other; a student equal to its teacher has no
    divergence and no gradient, and steps along the gradient bring another one nearer."""
    T, V, K = 24, 5003, 32
    t, _ = rows(T, V, "bf16", seed=1)
    tok = tokens_for(T, V, skip=0)
    rec = logprobs(t, 0.9, tok, K)
    ids, y, w = rec["top_ids"].cuda(), rec["top_logprobs"].cuda(), torch.ones(T, device="cuda")
    d = torch.empty_like(t)
    loss, _ = run_distill(t, 0.9, ids, y, 1, w, d)
    # the recorded values are float32: each q is off by |y| u relative, the loss by the square of that and the sums' own error
    assert float(loss.abs().max()) <= 40 * ref.rel(V) and float(d.float().abs().max()) <= 40 * ref.rel(V)
    x = torch.randn(T, V, device="cuda")
    d = torch.empty_like(x)
    first, _ = run_distill(x, 0.9, ids, y, 1, w, d)
    want = ref.distill(x.cpu(), 0.9, ids.cpu(), y.cpu(), 1, w.cpu())
    ref.check_grad(d.cpu(), want["grad"], want["grad_size"], V)
    second, _ = run_distill(x - 0.01 * d / d.norm(dim=1, keepdim=True), 0.9, ids, y, 1, w)
    assert bool((second < first).all())


def test_on_another_stream_and_captured():
    T, V, K = 8, 30000, 16
    x, _ = rows(T, V, "bf16")
    tok, w = tokens_for(T, V), torch.ones(T, device="cuda")
    eager = logprobs(x, 1.0, tok, K)
    ids, y = eager["top_ids"].cuda(), eager["top_logprobs"].cuda()
    side = torch.cuda.Stream()
    lp, ent = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    st, loss = torch.zeros(T, 4, device="cuda"), torch.zeros(T, device="cuda")
    oi, ol = torch.zeros(T, K, dtype=torch.int32, device="cuda"), torch.zeros(T, K, device="cuda")
    d1, d2 = torch.zeros_like(x), torch.zeros_like(x)
    torch.cuda.synchronize()

    def all_four(s):
        assert rb.remoe_token_logprobs(T, V, rb.REMOE_BF16, x, V, 1.0, tok, K, lp, ent, oi, ol, st, s) == 0
        assert rb.remoe_token_logprobs_backward(T, V, rb.REMOE_BF16, x, V, 1.0, tok, st, w, w, d1, V, s) == 0
        assert rb.remoe_distill_topk(T, V, rb.REMOE_BF16, x, V, 1.0, K, oi, ol, 1, w, loss, None, d2, V, s) == 0

    all_four(side.cuda_stream)
    side.synchronize()
    first = [t.clone() for t in (lp, ent, oi, ol, st, loss, d1, d2)]
    assert torch.equal(oi.cpu(), eager["top_ids"]) and torch.equal(lp.cpu(), eager["logprob"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_four(torch.cuda.current_stream().cuda_stream)
    for _ in range(2):
        for t in (lp, ent, oi, ol, st, loss, d1, d2):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((lp, ent, oi, ol, st, loss, d1, d2), first):
            assert torch.equal(a, b)
    x.mul_(0.5)                                       # new inputs in the same place
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(lp.cpu(), logprobs(x, 1.0, tok, K)["logprob"])


def test_two_calls_at_once_do_not_share_anything():
    T, V, K = 4, 60000, 64
    a, _ = rows(T, V, "bf16", seed=1)
    b, _ = rows(T, V, "bf16", seed=2)
    tok = tokens_for(T, V)
    alone = [logprobs(t, 1.0, tok, K) for t in (a, b)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    out = [[torch.zeros(T, device="cuda"), torch.zeros(T, K, dtype=torch.int32, device="cuda"), torch.zeros(T, K, device="cuda")] for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for t, s, o in ((a, s1, out[0]), (b, s2, out[1])):
            assert rb.remoe_token_logprobs(T, V, rb.REMOE_BF16, t, V, 1.0, tok, K, o[0], None, o[1], o[2], None, s.cuda_stream) == 0
    torch.cuda.synchronize()
    for o, w in zip(out, alone):
        assert torch.equal(o[0].cpu(), w["logprob"]) and torch.equal(o[1].cpu(), w["top_ids"]) and torch.equal(o[2].cpu(), w["top_logprobs"])


def test_rows_far_apart():
    # offsets beyond 2^31 elements
    V, stride = 1000, (1 << 30) + 8
    flat = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(flat, (3, V), (stride, 1))
    src, _ = rows(3, V, "bf16", seed=8)
    x.copy_(src)
    tok = tokens_for(3, V, skip=0)
    got, want = logprobs(x, 1.0, tok, 5), logprobs(src, 1.0, tok, 5)
    assert torch.equal(got["logprob"], want["logprob"]) and torch.equal(got["top_ids"], want["top_ids"])
    w = torch.ones(3, device="cuda")
    ids, y = got["top_ids"].cuda(), got["top_logprobs"].cuda()
    d = torch.empty(3, V, dtype=torch.bfloat16, device="cuda")
    run_distill(src, 1.0, ids, y, 1, w, d)
    run_distill(x, 1.0, ids, y, 1, w, x)
    assert torch.equal(x, d)


def test_optional_outputs():
    T, V = 3, 3000
    x, _ = rows(T, V, "f32")
    tok = tokens_for(T, V)
    want = logprobs(x, 1.0, tok, 3)
    ent = torch.zeros(T, device="cuda")
    assert rb.remoe_token_logprobs(T, V, rb.REMOE_F32, x, V, 1.0, None, 0, None, ent, None, None, None, stream()) == 0
    assert torch.equal(ent.cpu(), want["entropy"])
    st = torch.zeros(T, 4, device="cuda")
    assert rb.remoe_token_logprobs(T, V, rb.REMOE_F32, x, V, 1.0, None, 0, None, None, None, None, st, stream()) == 0
    assert torch.equal(st[:, :3].cpu(), want["row_stats"][:, :3]) and bool((st[:, 3] == 0).all())
    ids = torch.zeros(T, 3, dtype=torch.int32, device="cuda")
    lps = torch.zeros(T, 3, device="cuda")
    assert rb.remoe_token_logprobs(T, V, rb.REMOE_F32, x, V, 1.0, None, 3, None, None, ids, lps, None, stream()) == 0
    assert torch.equal(ids.cpu(), want["top_ids"]) and torch.equal(lps.cpu(), want["top_logprobs"])
    d, d0 = torch.zeros_like(x), torch.zeros_like(x)
    one = torch.ones(T, device="cuda")
    assert rb.remoe_distill_topk(T, V, rb.REMOE_F32, x, V, 1.0, 3, ids, lps, 0, None, None, None, d, V, stream()) == 0
    run_distill(x, 1.0, ids, lps, 0, one, d0)
    assert torch.equal(d, d0)


def test_host_rows_are_refused():
    x = torch.zeros(2, 64)
    out = torch.zeros(2, device="cuda")
    assert rb.remoe_token_logprobs(2, 64, rb.REMOE_F32, x, 64, 1.0, None, 0, None, out, None, None, None, stream()) == rb.REMOE_E_ARG
    pinned = x.pin_memory()
    assert rb.remoe_token_logprobs(2, 64, rb.REMOE_F32, pinned, 64, 1.0, None, 0, None, out, None, None, None, stream()) == rb.REMOE_E_ARG


def test_drift_of_a_rerouted_stack():
    """What the operators are for here: a chained stack with the cache-aware rerouting bonus, its answers against those
    of the stack without it.  (The head that turns hidden states into logits is the caller's: a matrix product.)"""
    import synth
    from paper_2605_27081_b200.loader import LoadedWorkload
    H, V, T, K = 512, 4097, 24, 32
    shape = synth.Shape(3, H, 32, 4, 96, 1, 64, 1, 0, 1, 1)
    head = torch.randn(V, H, generator=torch.Generator().manual_seed(3)).cuda() / math.sqrt(H) * 3
    rng = torch.Generator().manual_seed(4)
    inputs = torch.randn(T, 1, H, generator=rng).cuda()

    def answers(beta):
        wl = LoadedWorkload(shape, 6, seed=0)
        try:
            if beta:
                wl.stack.set_reroute_beta(beta)
            out = torch.empty(T, 1, H, device="cuda")
            ids, gates = torch.empty(3, 1, 4, dtype=torch.int32, device="cuda"), torch.empty(3, 1, 4, device="cuda")
            for t in range(T):
                wl.stack.decode_step_chained(inputs[t], out[t], None, ids, gates)
            torch.cuda.synchronize()
            return (out.view(T, H) @ head.T).contiguous()
        finally:
            wl.close()

    plain, same, moved = answers(0.0), answers(0.0), answers(4.0)
    tok = plain.argmax(1).int()
    rec = logprobs(plain, 1.0, tok, K)
    ids, y, w = rec["top_ids"].cuda(), rec["top_logprobs"].cuda(), torch.ones(T, device="cuda")
    assert torch.equal(rec["top_ids"][:, 0], tok.cpu())
    none, _ = run_distill(same, 1.0, ids, y, 1, w)
    some, _ = run_distill(moved, 1.0, ids, y, 1, w)
    want = ref.distill(moved, 1.0, ids, y, 1, w)
    ref.close(some, want["loss"], want["size"] * (ref.rel(V) + 4 * ref.U) + ref.U * want["loss"].abs(), "drift")
    assert float(none.abs().max()) <= 40 * ref.rel(V) and float(some.max()) > 1e-4
