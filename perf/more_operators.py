"""Cases of the operators on tokens sorted by expert: sorting and dispatch, the experts' SwiGLU products, the weighted
combine, and the backward passes.  Plain forms in elementary torch operations, the same cases through the library's entry
points (`own`), and their values in 64 bits.

A token's K selections become K of the T * K rows; the rows of one expert lie together, in the order of the selections.  An
expert's block holds, for each of its `inter` channels, the rows W_gate[i], W_up[i], W_down[:, i]: [experts, inter, 3, hidden].
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, dtype, tokens, top_k, experts, hidden, inter=0, pad=0, skip=0.0, skew=0.5, base=False, train=False, frozen=False):
    return {"name": name, "op": op, "dtype": dtype, "tokens": tokens, "top_k": top_k, "experts": experts, "hidden": hidden, "inter": inter,
            "pad": pad, "skip": skip, "skew": skew, "base": base, "train": train, "frozen": frozen}


def listed():
    return [
        # 32 sequences decoded together: the latency of getting their rows in order
        _case("dispatch_answers", "dispatch", "bf16", 32, 6, 64, 2048),
        # a prompt (or several, padded to one length) of 8192 tokens
        _case("dispatch_prompt", "dispatch", "bf16", 8192, 8, 128, 2048, skip=0.1),
        # one token's experts added onto the residual stream, float32 as the decode step keeps it
        _case("combine_one_token", "combine", "f32", 1, 4, 60, 2048, base=True),
        # the same for a prompt
        _case("combine_prompt", "combine", "bf16", 4096, 6, 64, 2048, base=True),
        # a router's gradient through the gates: a small odd batch in float32
        _case("combine_backward_odd", "combine_backward", "f32", 509, 4, 60, 1021, pad=3, skip=0.1),
        # a training batch
        _case("combine_backward_batch", "combine_backward", "bf16", 8192, 8, 128, 2048, skip=0.1),
        # one token through its six experts: reads each weight once
        _case("experts_one_token", "experts", "bf16", 1, 6, 64, 2048, 1408),
        # 32 sequences decoded together, nearly every expert in use with two or three rows
        _case("experts_answers", "experts", "f16", 32, 8, 128, 2048, 768),
        # a prompt of 4096 tokens
        _case("experts_prompt", "experts", "bf16", 4096, 6, 64, 2048, 1408),
        # one wide shared expert over a training batch: a single expert that takes every token, gate and up kept
        _case("experts_shared_train", "experts", "bf16", 4096, 1, 1, 2048, 5632, train=True),
        # a training step of a prompt's length
        _case("experts_backward_batch", "experts_backward", "bf16", 4096, 6, 64, 2048, 1408),
        # a short padded batch with uneven routing: experts with no row, one row, hundreds
        _case("experts_backward_ragged", "experts_backward", "f16", 777, 4, 60, 2048, 1408, skip=0.2, skew=2.0),
    ]


def draw(rng):
    op = rng.choice(["dispatch", "combine", "combine_backward", "experts", "experts", "experts_backward"])

    def log_range(low, high):
        return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))

    experts = log_range(1, 160)
    top_k = rng.randint(1, min(8, experts))
    tokens = log_range(1, 8192)
    case = dict(skip=rng.choice([0.0, 0.0, 0.1, 0.5]), skew=rng.choice([0.0, 0.5, 2.0]), pad=rng.choice([0, 0, 8, 64]))
    if not op.startswith("experts"):
        hidden = log_range(16, 4096)
        if rng.random() < 0.6:
            hidden = max(8, hidden // 8 * 8)
        case["pad"] = rng.choice([0, 0, 1, 8, 64, 37])
        return _case("", op, rng.choice(["f32", "bf16", "bf16", "f16"]), min(tokens, 130_000_000 // (hidden * top_k)), top_k, experts, hidden,
                     base=op == "combine" and rng.random() < 0.5, **case)
    hidden, inter = log_range(8, 512) * 8, log_range(2, 704) * 8
    hidden = min(hidden, 2048) if experts > 64 else hidden
    inter = max(8, min(inter, 500_000_000 // (experts * 3 * hidden) // 8 * 8))
    tokens = max(1, min(tokens, 70_000_000_000 // (hidden * inter * top_k)))
    return _case("", op, rng.choice(["bf16", "bf16", "f16"]), tokens, top_k, experts, hidden, inter,
                 train=op == "experts" and rng.random() < 0.5, frozen=op == "experts_backward" and rng.random() < 0.3, **case)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, K, N, H, I, dtype = case["tokens"], case["top_k"], case["experts"], case["hidden"], case["inter"], DTYPES[case["dtype"]]
    R = T * K

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def matrix(rows, scale, used=None, stray=0.0):
        """[rows, H], `pad` elements between rows; those behind the first `used` hold what was in the memory."""
        m = torch.zeros(max(1, rows), H + case["pad"], dtype=dtype, device="cuda")[:rows, :H]
        m.copy_(randn(rows, H) * scale)
        if used is not None:
            m[used:] = stray
        return m

    # what a router hands on: the top K of its logits, some experts liked better than others, padding tokens without experts
    logits = randn(T, N) + case["skew"] * randn(1, N)
    gates, ids = torch.softmax(logits, 1).topk(K, 1)
    left_out = torch.rand(T, generator=g, device="cuda") < case["skip"]
    ids = torch.where(left_out.unsqueeze(1), torch.full_like(ids, -1), ids).int().contiguous()
    gates = gates.contiguous()
    state = {"case": case}
    if case["op"] == "dispatch":
        state.update(ids=ids, x=matrix(T, 1.0), rows=torch.empty(T, K, dtype=torch.int32, device="cuda"),
                     offsets=torch.empty(N + 1, dtype=torch.int32, device="cuda"), xs=matrix(R, 0.0))
        return state
    offsets, rows = _sort(ids, N)
    # how many rows each expert has, as a program that calls its experts one by one would keep it
    counts = (offsets[1:] - offsets[:-1]).tolist()
    used = sum(counts)
    state.update(rows=rows, offsets=offsets, gates=gates, counts=counts)
    if case["op"] == "combine":
        state.update(ys=matrix(R, 0.3, used, float("nan")), base=matrix(T, 1.0) if case["base"] else None, out=matrix(T, 0.0))
        return state
    if case["op"] == "combine_backward":
        state.update(ys=matrix(R, 0.3, used, float("nan")), d_out=matrix(T, 1e-2), d_ys=matrix(R, 0.0),
                     d_gates=torch.empty(T, K, device="cuda"))
        return state
    state["blocks"] = torch.empty(N, I, 3, H, dtype=dtype, device="cuda")
    for e in range(N):
        state["blocks"][e] = randn(I, 3, H) * 0.02
    state["xs"] = matrix(R, 1.0, used, float("nan"))
    if case["op"] == "experts":
        state.update(ys=matrix(R, 0.0), act=torch.zeros(R, I, dtype=dtype, device="cuda"),
                     gate_up=torch.zeros(2, R, I, dtype=dtype, device="cuda") if case["train"] else None)
        return state
    # what the forward pass kept
    state["gate_up"] = torch.zeros(2, R, I, dtype=dtype, device="cuda")
    for e, a, b in _runs(state):
        w = state["blocks"][e].float()
        x = state["xs"][a:b].float()
        state["gate_up"][0, a:b] = (x @ w[:, 0].T).to(dtype)
        state["gate_up"][1, a:b] = (x @ w[:, 1].T).to(dtype)
    state.update(d_ys=matrix(R, 1e-2, used, float("nan")), work=torch.zeros(3, R, I, dtype=dtype, device="cuda"), d_xs=matrix(R, 0.0),
                 d_blocks=None if case["frozen"] else torch.zeros(N, I, 3, H, dtype=dtype, device="cuda"))
    return state


# ---- plain forms -------------------------------------------------------------------------------------------------

def _sort(ids, experts):
    flat = ids.flatten().long()
    key = torch.where((flat < 0) | (flat >= experts), torch.full_like(flat, experts), flat)
    order = torch.sort(key, stable=True).indices
    rows = torch.empty_like(flat)
    rows[order] = torch.arange(flat.numel(), device=ids.device)
    rows = torch.where(key == experts, torch.full_like(rows, -1), rows)
    counts = (key.unsqueeze(0) == torch.arange(experts, device=ids.device).unsqueeze(1)).sum(1)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=ids.device)
    offsets[1:] = counts.cumsum(0)
    return offsets, rows.int().view(ids.shape)


def _runs(st):
    """(expert, first row, end) of the experts that have rows."""
    a = 0
    for e, n in enumerate(st["counts"]):
        if n:
            yield e, a, a + n
        a += n


def _dispatch(st):
    offsets, rows = _sort(st["ids"], st["case"]["experts"])
    K, flat = st["case"]["top_k"], rows.flatten().long()
    # the selections that have no row write behind the last one
    end = flat.numel()
    xs = torch.zeros(end + 1, st["x"].shape[1], dtype=st["x"].dtype, device="cuda")
    xs[torch.where(flat < 0, torch.full_like(flat, end), flat)] = st["x"].repeat_interleave(K, 0)
    xs[end] = 0
    return {"rows": rows, "offsets": offsets, "xs": xs[:end]}


def _picked(st):
    """[T, K, H] rows of each token in 32 bits, zeros where there is none."""
    rows = st["rows"].long()
    return st["ys"][rows.clamp(min=0)].float().masked_fill((rows < 0).unsqueeze(2), 0.0)


def _combine(st):
    out = (_picked(st) * st["gates"].unsqueeze(2)).sum(1)
    if st["base"] is not None:
        out = out + st["base"].float()
    return {"out": out.to(st["ys"].dtype)}


def _combine_backward(st):
    rows, d = st["rows"].long(), st["d_out"].float().unsqueeze(1)
    end = rows.numel()
    d_gates = (_picked(st) * d).sum(2)
    d_ys = torch.zeros(end + 1, d.shape[2], dtype=st["ys"].dtype, device="cuda")
    d_ys[torch.where(rows < 0, torch.full_like(rows, end), rows).flatten()] = (d * st["gates"].unsqueeze(2)).to(d_ys.dtype).flatten(0, 1)
    return {"d_ys": d_ys[:end], "d_gates": d_gates}


def _experts(st):
    xs, (N, I, _, H) = st["xs"], st["blocks"].shape
    ys = torch.zeros(xs.shape[0], H, dtype=xs.dtype, device="cuda")
    kept = torch.zeros(2, xs.shape[0], I, dtype=xs.dtype, device="cuda") if st["case"]["train"] else None
    for e, a, b in _runs(st):
        w, x = st["blocks"][e].float(), xs[a:b].float()
        g, u = x @ w[:, 0].T, x @ w[:, 1].T
        ys[a:b] = ((g * torch.sigmoid(g) * u) @ w[:, 2]).to(xs.dtype)
        if kept is not None:
            kept[0, a:b] = g.to(xs.dtype)
            kept[1, a:b] = u.to(xs.dtype)
    return {"ys": ys} if kept is None else {"ys": ys, "gate_up": kept}


def _experts_backward(st):
    xs, frozen = st["xs"], st["case"]["frozen"]
    d_xs = torch.zeros(xs.shape, dtype=xs.dtype, device="cuda")
    d_blocks = None if frozen else torch.zeros_like(st["blocks"])
    for e, a, b in _runs(st):
        w, x, d = st["blocks"][e].float(), xs[a:b].float(), st["d_ys"][a:b].float()
        g, u = st["gate_up"][0, a:b].float(), st["gate_up"][1, a:b].float()
        s = torch.sigmoid(g)
        d_act = d @ w[:, 2].T
        d_g, d_u = d_act * u * s * (1 + g * (1 - s)), d_act * g * s
        d_xs[a:b] = (d_g @ w[:, 0] + d_u @ w[:, 1]).to(xs.dtype)
        if not frozen:
            d_blocks[e, :, 0] = (d_g.T @ x).to(xs.dtype)
            d_blocks[e, :, 1] = (d_u.T @ x).to(xs.dtype)
            d_blocks[e, :, 2] = ((g * s * u).T @ d).to(xs.dtype)
    return {"d_xs": d_xs} if frozen else {"d_xs": d_xs, "d_blocks": d_blocks}


# ---- the library's calls -----------------------------------------------------------------------------------------

def _own(st):
    from paper_2605_27081_b200 import binding as rb
    case = st["case"]
    T, K, N, H, I, op = (case[k] for k in ("tokens", "top_k", "experts", "hidden", "inter", "op"))
    dtype = {"f32": rb.REMOE_F32, "bf16": rb.REMOE_BF16, "f16": rb.REMOE_F16}[case["dtype"]]
    stream, R = torch.cuda.current_stream().cuda_stream, T * K
    if op == "dispatch":
        rc = rb.remoe_expert_sort(T, K, N, st["ids"], st["rows"], st["offsets"], stream)
        if not rc:
            rc = rb.remoe_expert_dispatch(T, K, H, dtype, st["x"], st["x"].stride(0), st["rows"], R, st["xs"], st["xs"].stride(0), stream)
        keys = ("rows", "offsets", "xs")
    elif op == "combine":
        base = st["base"]
        rc = rb.remoe_expert_combine(T, K, H, dtype, R, st["ys"], st["ys"].stride(0), st["rows"], st["gates"], base,
                                     0 if base is None else base.stride(0), st["out"], st["out"].stride(0), stream)
        keys = ("out",)
    elif op == "combine_backward":
        rc = rb.remoe_expert_combine_backward(T, K, H, dtype, st["d_out"], st["d_out"].stride(0), R, st["ys"], st["ys"].stride(0),
                                              st["rows"], st["gates"], st["d_ys"], st["d_ys"].stride(0), st["d_gates"], stream)
        keys = ("d_ys", "d_gates")
    elif op == "experts":
        rc = rb.remoe_expert_ffn(R, N, H, I, dtype, st["xs"], st["xs"].stride(0), st["offsets"], st["blocks"], st["blocks"].stride(0),
                                 st["gate_up"], st["act"], st["ys"], st["ys"].stride(0), stream)
        keys = ("ys", "gate_up") if case["train"] else ("ys",)
    else:
        rc = rb.remoe_expert_ffn_backward(R, N, H, I, dtype, st["xs"], st["xs"].stride(0), st["offsets"], st["blocks"],
                                          st["blocks"].stride(0), st["gate_up"], st["d_ys"], st["d_ys"].stride(0), st["work"], st["d_xs"],
                                          st["d_xs"].stride(0), st["d_blocks"], st["blocks"].stride(0), stream)
        keys = ("d_xs",) if case["frozen"] else ("d_xs", "d_blocks")
    if rc:
        raise rb.RemoeError(rc, op)
    return {k: st[k] for k in keys}


def run(state):
    if own:
        return _own(state)
    return {"dispatch": _dispatch, "combine": _combine, "combine_backward": _combine_backward, "experts": _experts,
            "experts_backward": _experts_backward}[state["case"]["op"]](state)


def work(case):
    """Bytes: every row, list and block that takes part once in or once out.  The number of experts in use is that of even
    routing; padding tokens have no rows."""
    T, K, N, H, I, op = (case[k] for k in ("tokens", "top_k", "experts", "hidden", "inter", "op"))
    w = DTYPES[case["dtype"]].itemsize
    live = T * (1 - case["skip"])
    R = live * K
    if op == "dispatch":
        return {"bytes": int(8 * T * K + 4 * (N + 1) + (live + R) * H * w), "flops": T * K}
    if op == "combine":
        return {"bytes": int(8 * T * K + (R + T * (2 if case["base"] else 1)) * H * w), "flops": int(2 * R * H)}
    if op == "combine_backward":
        return {"bytes": int(12 * T * K + (live + 2 * R) * H * w), "flops": int(3 * R * H)}
    in_use = N * (1 - (1 - K / N) ** live)
    block = 3 * I * H * w
    if op == "experts":
        return {"bytes": int(in_use * block + 2 * R * H * w + (2 * R * I * w if case["train"] else 0)), "flops": int(6 * R * H * I)}
    # the gradient of an expert without rows is written, too
    return {"bytes": int(in_use * block + (0 if case["frozen"] else N * block) + (2 if case["frozen"] else 3) * R * H * w + 2 * R * I * w),
            "flops": int((6 if case["frozen"] else 12) * R * H * I)}


# ---- values in 64 bits, from the definitions ---------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    T, K, N, H, I, op = (case[k] for k in ("tokens", "top_k", "experts", "hidden", "inter", "op"))
    if op == "dispatch":
        ids = st["ids"].cpu().tolist()
        lists = [[] for _ in range(N)]
        for t in range(T):
            for k in range(K):
                if 0 <= ids[t][k] < N:
                    lists[ids[t][k]].append(t * K + k)
        order = [s for one in lists for s in one]
        offsets = [0]
        for one in lists:
            offsets.append(offsets[-1] + len(one))
        order = torch.tensor(order, dtype=torch.long, device="cuda")
        rows = torch.full((T * K,), -1, dtype=torch.int32, device="cuda")
        rows[order] = torch.arange(order.numel(), dtype=torch.int32, device="cuda")
        xs = torch.zeros(T * K, H, dtype=torch.float64, device="cuda")
        xs[:order.numel()] = st["x"].double()[order // K]
        return {"rows": rows.view(T, K), "offsets": torch.tensor(offsets, dtype=torch.int32, device="cuda"), "xs": xs}
    rows = st["rows"].long()
    if op.startswith("combine"):
        out = torch.zeros(T, H, dtype=torch.float64, device="cuda")
        gates = st["gates"].double().requires_grad_(True)
        ys = st["ys"].double()
        ys[st["offsets"][-1]:] = 0
        ys.requires_grad_(True)
        for k in range(K):
            there = (rows[:, k] >= 0).nonzero().squeeze(1)
            out = out.index_add(0, there, ys[rows[there, k]] * gates[there, k].unsqueeze(1))
        if op == "combine":
            return {"out": (out + st["base"].double() if case["base"] else out).detach()}
        d_ys, d_gates = torch.autograd.grad(out, (ys, gates), st["d_out"].double())
        return {"d_ys": d_ys, "d_gates": d_gates}
    silu = torch.nn.functional.silu
    R, off = T * K, st["offsets"].tolist()
    if op == "experts":
        ys = torch.zeros(R, H, dtype=torch.float64, device="cuda")
        kept = torch.zeros(2, R, I, dtype=torch.float64, device="cuda")
        for e in range(N):
            mine = slice(off[e], off[e + 1])
            gate, up, down = st["blocks"][e].double().unbind(1)
            kept[0, mine] = torch.einsum("rh,ih->ri", st["xs"][mine].double(), gate)
            kept[1, mine] = torch.einsum("rh,ih->ri", st["xs"][mine].double(), up)
            ys[mine] = torch.einsum("ri,ih->rh", silu(kept[0, mine]) * kept[1, mine], down)
        return {"ys": ys, "gate_up": kept} if case["train"] else {"ys": ys}
    d_xs = torch.zeros(R, H, dtype=torch.float64, device="cuda")
    d_blocks = None if case["frozen"] else torch.zeros(N, I, 3, H, dtype=torch.float64, device="cuda")
    for e in range(N):
        mine = slice(off[e], off[e + 1])
        gate, up, down = st["blocks"][e].double().unbind(1)
        x, d = st["xs"][mine].double(), st["d_ys"][mine].double()
        g, u = (st["gate_up"][j, mine].double().requires_grad_(True) for j in (0, 1))
        act = silu(g) * u
        d_g, d_u = torch.autograd.grad(act, (g, u), torch.einsum("rh,ih->ri", d, down))
        d_xs[mine] = torch.einsum("ri,ih->rh", d_g, gate) + torch.einsum("ri,ih->rh", d_u, up)
        if d_blocks is not None:
            d_blocks[e] = torch.stack([torch.einsum("ri,rh->ih", one, rows_) for one, rows_ in ((d_g, x), (d_u, x), (act.detach(), d))], 1)
    return {"d_xs": d_xs} if d_blocks is None else {"d_xs": d_xs, "d_blocks": d_blocks}
