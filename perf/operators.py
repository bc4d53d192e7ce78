"""Cases of the operators on rows of logits: log probabilities of given tokens with entropy and top alternatives,
and distillation from a teacher's top logits.  Plain forms in elementary torch operations, the same cases through
the library's entry points (`own`), and their values in 64 bits.

Rows of 64 classes are router distributions (one row per layer and token); the longer ones are vocabularies.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NINF = float("-inf")


def _case(name, op, dtype, rows, vocab, top, pad=0, inv_temperature=1.0, mask="none", skip=0.0, tail=False):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "vocab": vocab, "top": top, "pad": pad,
            "inv_temperature": inv_temperature, "mask": mask, "skip": skip, "tail": tail}


def listed():
    return [
        # one sequence's next token with its alternatives: the latency of an answer
        _case("answer_one_token", "logprobs", "bf16", 1, 102400, 20, inv_temperature=1 / 0.7),
        # a batch of 32 decoded together, float32 logits, a tenth of the vocabulary banned
        _case("answer_batch_32", "logprobs", "f32", 32, 151936, 8, mask="some"),
        # constrained decoding: a handful of tokens allowed, odd vocabulary and so unaligned rows
        _case("answer_constrained", "logprobs", "f16", 257, 50257, 5, mask="few"),
        # teacher-forced scoring of a text: token log probabilities and entropy only
        _case("score_text", "logprobs", "bf16", 4096, 102400, 0, skip=0.05),
        # a teacher's top logits recorded for distillation
        _case("record_teacher", "logprobs", "bf16", 2048, 131072, 64),
        # cross-entropy with an entropy bonus, padded batch
        _case("score_backward", "logprobs_backward", "bf16", 4096, 102400, 0, skip=0.2),
        # the same in float32 with an odd vocabulary
        _case("score_backward_odd", "logprobs_backward", "f32", 509, 32003, 0, mask="some"),
        # how far a stack with a lossy expert store has moved from the full one: the divergence alone
        _case("drift_of_store", "distill", "bf16", 1024, 151936, 64, tail=True),
        # routers of 26 layers x 512 tokens held to the frozen router's distribution
        _case("router_anchor", "distill_grad", "f32", 13312, 64, 64),
        # a student's training step
        _case("distill_step", "distill_grad", "bf16", 4096, 102400, 64, tail=True, skip=0.1),
        # the same with masked logits, odd vocabulary and a softened distribution
        _case("distill_step_odd", "distill_grad", "f16", 511, 50257, 31, inv_temperature=0.5, mask="some"),
        # the gradient alone, behind a loss whose weight is known only after the forward pass
        _case("distill_backward", "distill_backward", "bf16", 2048, 131072, 128, pad=64, tail=True),
    ]


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs_backward", "distill", "distill_grad", "distill_backward"])
    vocab = int(math.exp(rng.uniform(math.log(16), math.log(262144))))
    if rng.random() < 0.5:
        vocab = max(16, vocab // 8 * 8)
    rows = int(math.exp(rng.uniform(0, math.log(16384))))
    rows = max(1, min(rows, 400_000_000 // vocab))
    top = int(math.exp(rng.uniform(0, math.log(min(256, vocab)))))
    if op == "logprobs_backward" or (op == "logprobs" and rng.random() < 0.3):
        top = 0
    return _case("", op, rng.choice(["f32", "bf16", "bf16", "f16"]), rows, vocab, top, pad=rng.choice([0, 0, 1, 8, 64, 37]),
                 inv_temperature=rng.choice([1.0, 1.0, 0.5, 1 / 0.7]), mask=rng.choice(["none", "none", "some", "few", "lowest", "rows"]),
                 skip=rng.choice([0.0, 0.0, 0.1, 0.5]), tail=rng.random() < 0.5)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, vocab, dtype, s = case["rows"], case["vocab"], DTYPES[case["dtype"]], case["inv_temperature"]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    # a language model's logits: a broad bulk, and a common shift of each row that its softmax does not see
    x = randn(rows, vocab).mul_(2.5).add_(randn(rows, 1) * 4)
    # the token that was said: likely ones more often (the largest of a few), so that log probabilities differ widely
    guess = torch.randint(0, vocab, (rows, 8), generator=g, device="cuda")
    token = guess.gather(1, x.gather(1, guess).argmax(1, keepdim=True)).squeeze(1).int()
    x.scatter_add_(1, token.long().unsqueeze(1), rand(rows, 1) * 16)
    dead = None
    if case["mask"] in ("some", "lowest"):
        dead = rand(rows, vocab) < 0.1
    elif case["mask"] == "few":
        dead = torch.ones(rows, vocab, dtype=torch.bool, device="cuda").scatter_(1, guess[:, :3], False)
    elif case["mask"] == "rows":
        dead = (rand(rows, 1) < 0.2).expand(rows, vocab)
    low = torch.finfo(dtype).min if case["mask"] == "lowest" else NINF
    if dead is not None:
        if case["mask"] != "rows":
            dead = dead.scatter(1, token.long().unsqueeze(1), False)
        x.masked_fill_(dead, low)
    logits = torch.zeros(rows, vocab + case["pad"], dtype=dtype, device="cuda")[:, :vocab]
    logits.copy_(x)
    left_out = rand(rows) < case["skip"]
    state = {"case": case, "logits": logits, "s": s}

    if case["op"].startswith("logprobs"):
        state["token"] = torch.where(left_out, torch.full_like(token, -1), token)
        if case["op"] == "logprobs":
            state["logprob"], state["entropy"] = (torch.empty(rows, device="cuda") for _ in range(2))
            if case["top"]:
                state["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
                state["top_logprobs"] = torch.empty(rows, case["top"], device="cuda")
            return state
        # what the forward pass of a training step kept of each row: largest logit, log of the sum, entropy
        del x, dead
        m, ln_z, ent, _ = _softmax(logits, s)
        state["row_stats"] = torch.stack([m, ln_z.float(), ent, torch.zeros_like(m)], 1)
        state["grad_logprob"] = -rand(rows)
        state["grad_entropy"] = randn(rows) * 0.01
        state["d_logits"] = torch.empty(rows, vocab + case["pad"], dtype=dtype, device="cuda")[:, :vocab]
        return state

    # the teacher: the student's logits moved a little, under the same masks; its top log probabilities are on record
    t = randn(rows, vocab).mul_(0.7).add_(logits)
    if case["mask"] == "lowest":
        t = t.masked_fill_(dead, NINF)
    del x
    t = torch.log_softmax(t * s, 1)
    t = torch.nan_to_num(t, nan=NINF, neginf=NINF)
    top = t.topk(case["top"], 1)
    state["teacher_ids"], state["teacher_logprobs"] = top.indices.int(), top.values.contiguous()
    del t, top
    state["row_weight"] = torch.where(left_out, torch.zeros(rows, device="cuda"), 0.5 + rand(rows))
    state["loss"] = torch.empty(rows, device="cuda")
    if case["op"] != "distill":
        state["d_logits"] = torch.empty(rows, vocab + case["pad"], dtype=dtype, device="cuda")[:, :vocab]
    if case["op"] == "distill_backward":
        # what the forward pass kept of each row
        r = _distill_rows(state)
        zero = torch.zeros(rows, device="cuda")
        state["row_stats"] = torch.stack([r["m"], r["ln_z"].float(), r["m_rest"], r["ln_z_rest"].float(), r["c_rest"].float(), r["ln_q"].float(),
                                          r["takes_part"].float(), zero], 1)
    return state


# ---- plain forms -------------------------------------------------------------------------------------------------

def _softmax(logits, s):
    """Largest logit, log of the sum, entropy and s (x - max) of each row; a row without a live logit: -inf, -inf, 0.
    The sum over a row is taken in 64 bits: where one token has nearly all the mass, the logarithm is what is left of it."""
    x = logits.float()
    m = x.amax(1)
    empty = m == NINF
    d = (x - m.masked_fill(empty, 0.0).unsqueeze(1)) * s
    e = d.exp()
    z = e.sum(1, dtype=torch.float64)
    ln_z = z.log()
    ent = ln_z - e.mul(d).masked_fill_(e == 0, 0.0).sum(1) / z
    return m, ln_z, ent.masked_fill(empty, 0.0).float(), d


def _order(x):
    """Whole numbers in the order of (value, lowest index first): all distinct, so that ties are settled."""
    b = (x + 0.0).view(torch.int32)
    b = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long()
    return b.mul_(1 << 32).add_((1 << 32) - 1 - torch.arange(x.shape[1], device=x.device))


def _logprobs(st):
    s, k = st["s"], st["case"]["top"]
    _, ln_z, ent, d = _softmax(st["logits"], s)
    token = st["token"].long()
    empty = (ln_z == NINF).unsqueeze(1)
    given = (d.gather(1, token.clamp(min=0).unsqueeze(1)) - ln_z.unsqueeze(1)).masked_fill(empty, NINF).squeeze(1)
    out = {"logprob": given.masked_fill(token < 0, 0.0).float(), "entropy": ent}
    if k:
        ids = _order(st["logits"].float()).topk(k, 1).indices
        out["top_ids"] = ids.int()
        out["top_logprobs"] = (d.gather(1, ids) - ln_z.unsqueeze(1)).masked_fill(empty, NINF).float()
    return out


def _logprobs_backward(st):
    s, token = st["s"], st["token"].long()
    m, ln_z, ent, d = _softmax(st["logits"], s)
    g = st["grad_logprob"].masked_fill(token < 0, 0.0).unsqueeze(1)
    lp = d - ln_z.float().unsqueeze(1)
    p = lp.exp()
    dx = p * (-g - st["grad_entropy"].unsqueeze(1) * (lp.masked_fill_(p == 0, 0.0) + ent.unsqueeze(1)))
    dx.scatter_add_(1, token.clamp(min=0).unsqueeze(1), g)
    return {"d_logits": (dx * s).masked_fill_((m == NINF).unsqueeze(1), 0.0).to(st["logits"].dtype)}


def _distill_rows(st):
    """The quantities of each row that its loss and gradient share.  The teacher's side, a few numbers a row, in 64 bits:
    what is left of its mass is a difference of numbers near one."""
    s, tail = st["s"], st["case"]["tail"]
    ids, y = st["teacher_ids"].long(), st["teacher_logprobs"].double()
    some = (y > NINF).any(1)
    ln_q = torch.zeros_like(y[:, 0]) if tail else y.logsumexp(1).masked_fill(~some, 0.0)
    y = y - ln_q.unsqueeze(1)
    q = y.exp()
    q_rest = (1 - q.sum(1)).clamp(min=0.0) if tail else torch.zeros_like(ln_q)
    x = st["logits"].float()
    m = x.amax(1)
    d = (x - m.masked_fill(m == NINF, 0.0).unsqueeze(1)) * s
    ln_z = d.exp().sum(1, dtype=torch.float64).log()
    others = x.scatter(1, ids, NINF)
    m_rest = others.amax(1)
    ln_z_rest = ((others - m_rest.masked_fill(m_rest == NINF, 0.0).unsqueeze(1)) * s).exp().sum(1, dtype=torch.float64).log()
    rest = m_rest > NINF
    ln_p = d.gather(1, ids).double() - ln_z.unsqueeze(1)
    ln_p_rest = ((m_rest.double() - m) * s + ln_z_rest - ln_z).masked_fill(~rest, 0.0)
    q_rest = q_rest.masked_fill(~rest, 0.0)
    return {"m": m, "ln_z": ln_z, "m_rest": m_rest, "ln_z_rest": ln_z_rest, "rest": rest, "q": q, "y": y, "ln_p": ln_p, "q_rest": q_rest,
            "ln_p_rest": ln_p_rest, "c_rest": (ln_p_rest.exp() - q_rest).masked_fill(~rest, 0.0), "ln_q": ln_q,
            "takes_part": some & (st["row_weight"] != 0) & (m > NINF), "d": d, "others": others}


def _distill(st, r):
    terms = (r["q"] * (r["y"] - r["ln_p"])).masked_fill(r["q"] == 0, 0.0).sum(1)
    rest = (r["q_rest"] * (r["q_rest"].log() - r["ln_p_rest"])).masked_fill(r["q_rest"] == 0, 0.0)
    return (terms + rest).masked_fill(~r["takes_part"], 0.0).float()


def _distill_gradient(st, r):
    s, ids = st["s"], st["teacher_ids"].long()
    rest = (r["others"] - r["m_rest"].masked_fill(~r["rest"], 0.0).unsqueeze(1)) * s
    dx = (rest - r["ln_z_rest"].float().masked_fill(~r["rest"], 0.0).unsqueeze(1)).exp() * r["c_rest"].float().unsqueeze(1)
    dx.scatter_(1, ids, (r["ln_p"].exp() - r["q"]).float())
    dx = dx * (s * st["row_weight"]).unsqueeze(1)
    return dx.masked_fill_(~r["takes_part"].unsqueeze(1), 0.0).to(st["logits"].dtype)


# ---- the library's calls -----------------------------------------------------------------------------------------

def _own(st):
    from paper_2605_27081_b200 import binding as rb
    case, logits = st["case"], st["logits"]
    rows, vocab, stride, s, top = case["rows"], case["vocab"], logits.stride(0), st["s"], case["top"]
    dtype = {"f32": rb.REMOE_F32, "bf16": rb.REMOE_BF16, "f16": rb.REMOE_F16}[case["dtype"]]
    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "logprobs":
        rc = rb.remoe_token_logprobs(rows, vocab, dtype, logits, stride, s, st["token"], top, st["logprob"], st["entropy"],
                                     st.get("top_ids"), st.get("top_logprobs"), None, stream)
        keys = ("logprob", "entropy", "top_ids", "top_logprobs") if top else ("logprob", "entropy")
    elif case["op"] == "logprobs_backward":
        rc = rb.remoe_token_logprobs_backward(rows, vocab, dtype, logits, stride, s, st["token"], st["row_stats"], st["grad_logprob"],
                                              st["grad_entropy"], st["d_logits"], st["d_logits"].stride(0), stream)
        keys = ("d_logits",)
    elif case["op"] == "distill_backward":
        rc = rb.remoe_distill_topk_backward(rows, vocab, dtype, logits, stride, s, top, st["teacher_ids"], st["teacher_logprobs"],
                                            st["row_stats"], st["row_weight"], st["d_logits"], st["d_logits"].stride(0), stream)
        keys = ("d_logits",)
    else:
        d = st.get("d_logits")
        rc = rb.remoe_distill_topk(rows, vocab, dtype, logits, stride, s, top, st["teacher_ids"], st["teacher_logprobs"], case["tail"],
                                   st["row_weight"], st["loss"], None, d, d.stride(0) if d is not None else 0, stream)
        keys = ("loss", "d_logits") if d is not None else ("loss",)
    if rc:
        raise rb.RemoeError(rc, case["op"])
    return {k: st[k] for k in keys}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "logprobs":
        return _logprobs(state)
    if op == "logprobs_backward":
        return _logprobs_backward(state)
    r = _distill_rows(state)
    if op == "distill":
        return {"loss": _distill(state, r)}
    if op == "distill_backward":
        return {"d_logits": _distill_gradient(state, r)}
    return {"loss": _distill(state, r), "d_logits": _distill_gradient(state, r)}


def work(case):
    """Bytes: the rows' logits in, the gradient out where there is one, and the few numbers a row.  Operations: per element
    a difference, a scaling, an exponential, a sum and, where they are asked for, a comparison, a product or two more."""
    rows, vocab, top, size = case["rows"], case["vocab"], case["top"], DTYPES[case["dtype"]].itemsize
    n = rows * vocab
    few = rows * {"logprobs": 12 + 8 * top, "logprobs_backward": 28, "distill": 8 + 8 * top, "distill_grad": 8 + 8 * top,
                  "distill_backward": 36 + 8 * top}[case["op"]]
    per = {"logprobs": 7, "logprobs_backward": 6, "distill": 6, "distill_grad": 10, "distill_backward": 4}[case["op"]]
    twice = case["op"] not in ("logprobs", "distill")
    return {"bytes": n * size * (2 if twice else 1) + few, "flops": n * per}


# ---- values in 64 bits, from the definitions ---------------------------------------------------------------------

def exact(case, seed):
    if case["rows"] * case["vocab"] > 1_000_000_000:
        return None
    st = prepare(case, seed)
    step = max(1, 30_000_000 // case["vocab"])
    parts = [_exact_rows(case, {k: v[i:i + step] if torch.is_tensor(v) else v for k, v in st.items()}) for i in range(0, case["rows"], step)]
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_rows(case, st):
    x = st["logits"].double()
    alive = (x > NINF).any(1)
    x = torch.where(alive.unsqueeze(1), x, torch.zeros_like(x)).requires_grad_(case["op"] not in ("logprobs", "distill"))
    ln_p = torch.log_softmax(x * st["s"], 1)
    if case["op"].startswith("logprobs"):
        token = st["token"].long()
        lp = ln_p.gather(1, token.clamp(min=0).unsqueeze(1)).squeeze(1)
        if case["op"] == "logprobs":
            lp = torch.where(alive, lp, torch.full_like(lp, NINF)).masked_fill(token < 0, 0.0)
            ent = torch.where(alive, -torch.xlogy(ln_p.exp(), ln_p.exp()).sum(1), torch.zeros_like(lp))
            out = {"logprob": lp, "entropy": ent}
            if case["top"]:
                ids = st["logits"].double().sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]
                top = ln_p.gather(1, ids)
                out["top_ids"] = ids.int()
                out["top_logprobs"] = torch.where(alive.unsqueeze(1), top, torch.full_like(top, NINF))
            return out
        p = ln_p.exp()
        ent = -(p * ln_p.masked_fill(p == 0, 0.0)).sum(1)
        g = st["grad_logprob"].double().masked_fill(token < 0, 0.0)
        objective = (g * lp.masked_fill(token < 0, 0.0) + st["grad_entropy"].double() * ent)[alive].sum()
        objective.backward()
        return {"d_logits": x.grad.nan_to_num_(0.0)}
    ids, y = st["teacher_ids"].long(), st["teacher_logprobs"].double()
    listed_ = torch.zeros_like(x, dtype=torch.bool).scatter_(1, ids, True)
    has = (y > NINF).any(1)
    q = y.exp()
    if not case["tail"]:
        q = q / q.sum(1, keepdim=True).masked_fill(~has.unsqueeze(1), 1.0)
    each = torch.where(q > 0, q.clamp(min=1e-320).log() - ln_p.gather(1, ids), torch.zeros_like(q)) * q
    loss = each.sum(1)
    if case["tail"]:
        q_rest = 1 - q.sum(1)
        there = (~listed_ & (st["logits"] > NINF)).any(1) & (q_rest > 0)
        p_rest = torch.where(there.unsqueeze(1), ln_p.masked_fill(listed_, NINF), torch.zeros_like(ln_p)).logsumexp(1)
        loss = loss + torch.where(there, q_rest * (q_rest.clamp(min=1e-320).log() - p_rest), torch.zeros_like(q_rest))
    takes_part = has & alive & (st["row_weight"] != 0)
    loss = torch.where(takes_part, loss, torch.zeros_like(loss))
    out = {} if case["op"] == "distill_backward" else {"loss": loss.detach()}
    if case["op"] != "distill":
        (loss * st["row_weight"].double()).sum().backward()
        out["d_logits"] = torch.where(takes_part.unsqueeze(1), x.grad, torch.zeros_like(x))
    return out
