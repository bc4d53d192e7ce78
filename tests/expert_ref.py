"""Plain 64-bit reference of the operators on tokens sorted by expert, and how far a kernel may be from it.

Bounds, from the arithmetic.  half = finfo(type).eps / 2 is a rounding to the matrices' type, u = 2^-24 one to float32, `tiny` the
type's smallest step.  A float32 sum of n products on the tensor cores is off by at most acc(n) = (n / 8 + 8) 2^-23 of the sum of
the products' absolute values: every eighth product at worst starts a new addition, which loses one step of the running
sum.  Bounds are carried through the formulas element by element with absolute values (matrix products of them):
  g, u              acc(H) |x||W|; kept ones are rounded once more: half |g| + tiny
  a = silu(g) u     1.1 |u| err(g) + |silu(g)| err(u) + (half + 2^-19 (1 + |g|)) |silu(g) u| + tiny: |silu'| <= 1.1, and the fast exponential
                    and division of the sigmoid lose a few steps, more for a larger exponent
  y                 err(a) |W| + acc(I) |a||W| + half |y| + tiny
  d a               acc(H) |d y||W|
  d g, d u          the same with the factors u silu'(g) (|silu'| taken as the sum of its terms' absolute values) and silu(g)
  d x, d W          products of the rounded d g, d u, a
Beside these worst cases, roundings to the type are independent of one another, so that the root mean square of the error
of a whole matrix stays below half times that of the matrix: two roundings on its way, each of at most half / sqrt(3).
"""
import torch

U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def acc(n):
    return (n / 8 + 8) * 2.0 ** -23


def sort(ids, n_experts):
    """rows, offsets, counts from the definition, on the host."""
    T, K = ids.shape
    flat = ids.cpu().flatten().tolist()
    lists = [[] for _ in range(n_experts)]
    for s, e in enumerate(flat):
        if 0 <= e < n_experts:
            lists[e].append(s)
    rows = torch.full((T * K,), -1, dtype=torch.int32)
    offsets, r = [0], 0
    for one in lists:
        for s in one:
            rows[s] = r
            r += 1
        offsets.append(r)
    return rows.view(T, K), torch.tensor(offsets, dtype=torch.int32), [len(o) for o in lists]


def silu(g):
    return g * torch.sigmoid(g)


def slopes(g):
    """silu'(g) and the sum of its terms' absolute values"""
    s = torch.sigmoid(g)
    return s * (1 + g * (1 - s)), s * (1 + g.abs() * (1 - s))


def act_error(g, u, eg, eu, dtype):
    a = silu(g) * u
    return 1.1 * u.abs() * eg + silu(g).abs() * eu + (half(dtype) + 2.0 ** -19 * (1 + g.abs())) * a.abs() + tiny(dtype)


def ffn(xs, offsets, blocks):
    """dict of (value, bound) for ys, gate, up, act, over the rows that belong to experts; 64 bits."""
    N, I, _, H = blocks.shape
    dt, off = xs.dtype, offsets.tolist()
    out = {k: (torch.zeros(xs.shape[0], w, dtype=torch.float64, device=xs.device), torch.zeros(xs.shape[0], w, dtype=torch.float64, device=xs.device))
           for k, w in (("ys", H), ("gate", I), ("up", I), ("act", I))}
    for e in range(N):
        r = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            continue
        x, (wg, wu, wd) = xs[r].double(), blocks[e].double().unbind(1)
        g, u = x @ wg.T, x @ wu.T
        eg, eu = acc(H) * (x.abs() @ wg.abs().T), acc(H) * (x.abs() @ wu.abs().T)
        a, ea = silu(g) * u, act_error(g, u, eg, eu, dt)
        y = a @ wd
        ey = ea @ wd.abs() + acc(I) * (a.abs() @ wd.abs()) + half(dt) * y.abs() + tiny(dt)
        for k, v, b in (("ys", y, ey), ("act", a, ea), ("gate", g, eg + half(dt) * g.abs() + tiny(dt)), ("up", u, eu + half(dt) * u.abs() + tiny(dt))):
            out[k][0][r], out[k][1][r] = v, b
    return out


def ffn_backward(xs, offsets, blocks, gate_up, d_ys):
    """dict of (value, bound) for d_xs, d_blocks."""
    N, I, _, H = blocks.shape
    dt, off = xs.dtype, offsets.tolist()
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64, device=xs.device)
    out = {"d_xs": (zero(xs.shape[0], H), zero(xs.shape[0], H)), "d_blocks": (zero(N, I, 3, H), zero(N, I, 3, H))}
    for e in range(N):
        r = slice(off[e], off[e + 1])
        n = off[e + 1] - off[e]
        if n == 0:
            continue
        x, d, (wg, wu, wd) = xs[r].double(), d_ys[r].double(), blocks[e].double().unbind(1)
        g, u = gate_up[0, r].double(), gate_up[1, r].double()
        da, eda = d @ wd.T, acc(H) * (d.abs() @ wd.abs().T)
        slope, slope_abs = slopes(g)
        few = 2.0 ** -19 * (1 + g.abs())
        dg, du, a = da * u * slope, da * silu(g), silu(g) * u
        edg = eda * (u * slope_abs).abs() + few * (da * u).abs() * slope_abs + half(dt) * dg.abs() + tiny(dt)
        edu = eda * silu(g).abs() + few * du.abs() + half(dt) * du.abs() + tiny(dt)
        ea = (half(dt) + few) * a.abs() + tiny(dt)
        dx = dg @ wg + du @ wu
        edx = edg @ wg.abs() + edu @ wu.abs() + acc(2 * I) * (dg.abs() @ wg.abs() + du.abs() @ wu.abs())
        out["d_xs"][0][r], out["d_xs"][1][r] = dx, edx + half(dt) * dx.abs() + tiny(dt)
        for j, (m, em, side) in enumerate(((dg, edg, x), (du, edu, x), (a, ea, d))):
            w = m.T @ side
            out["d_blocks"][0][e, :, j] = w
            out["d_blocks"][1][e, :, j] = em.T @ side.abs() + acc(n) * (m.abs().T @ side.abs()) + half(dt) * w.abs() + tiny(dt)
    return out


def close(got, want, bound, what=""):
    got, want = got.double(), want.double()
    same = (torch.isnan(got) & torch.isnan(want)) | (got == want)
    bad = ~same & ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), [(tuple(i), float(got[tuple(i)]), float(want[tuple(i)])) for i in bad.nonzero()[:4].tolist()])


def rms_close(got, want, dtype, what="", times=1.0):
    got, want = got.double(), want.double()
    err, size = (got - want).pow(2).mean().sqrt(), want.pow(2).mean().sqrt()
    assert err <= times * half(dtype) * size, (what, float(err), float(size))
