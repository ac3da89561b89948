"""The dense operators' definitions in fp64 (torch on the CPU), and the bounds that their tests hold the kernels to.

Bounds are elementwise and derived from the roundings that the operators state, with u = 2^-8 (bf16) or 2^-11 (fp16) the
half unit of a rounding to 16 bits:
* a sum of n products in fp32 is off by at most n * 2^-23 times the sum of their magnitudes (each of its at most n
  additions may truncate instead of round);
* an activation's value or slope is off by 2^-18 of its own magnitude plus 2^-21 of |z| (fast exponential, erf to 1.5e-7)
  and passes an error of its argument on with a slope of at most 1.13 (gelu; 1.1 silu, 1 relu), its slope with at most 1;
* a value that is rounded to 16 bits as an operand of a further product is off by u of itself.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # significands of 8 and 11 bits
TINY = 2.0 ** -24  # the smallest fp16 number: results below fp16's normal range are rounded absolutely


def act(z, name):
    if name == "relu":
        return torch.clamp_min(z, 0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def hidden(x, w, b, name, gated):
    """(h, its bound, z, z's bound) of one linear unit; x [T, D], w [rows, D]."""
    z = x @ w.t()
    ez = (x.shape[1] + 2) * 2.0 ** -23 * (x.abs() @ w.abs().t() + (0 if b is None else b.abs()))
    if b is not None:
        z = z + b
    own = lambda v: 2.0 ** -18 * act(v, name).abs() + 2.0 ** -21 * v.abs()  # noqa: E731
    if not gated:
        return act(z, name), (1.13 * ez + own(z)) * (name != "none") + ez * (name == "none"), z, ez
    n = z.shape[1] // 2
    a, o = z[:, :n], z[:, n:]
    ea = 1.13 * ez[:, :n] + own(a)
    return act(a, name) * o, ea * (o.abs() + ez[:, n:]) + act(a, name).abs() * ez[:, n:], z, ez


def hidden_grad(z, ez, dh, edh, name, gated):
    """(dz, its bound before any rounding) for a gradient dh (bound edh) of the hidden values."""
    own = lambda v: 2.0 ** -18 * slope(v, name).abs() + 2.0 ** -21 * (1 + v.abs())  # noqa: E731
    # relu's slope jumps: an argument within its bound of zero may fall on either side
    jump = lambda v, e: (v.abs() <= e).double() if name == "relu" else 0.0  # noqa: E731
    if not gated:
        es = (e_s := (1.0 * ez + own(z) + jump(z, ez))) if name != "none" else torch.zeros_like(z)
        return dh * slope(z, name), dh.abs() * es + edh * (slope(z, name).abs() + es)
    n = z.shape[1] // 2
    a, o, ea, eo = z[:, :n], z[:, n:], ez[:, :n], ez[:, n:]
    es = ea + own(a) + jump(a, ea) if name != "none" else torch.zeros_like(a)
    s = slope(a, name)
    ga, ega = dh * o * s, dh.abs() * (eo * (s.abs() + es) + o.abs() * es) + edh * (o.abs() + eo) * (s.abs() + es)
    va = act(a, name)
    eva = 1.13 * ea + 2.0 ** -18 * va.abs() + 2.0 ** -21 * a.abs() if name != "none" else ea
    return torch.cat([ga, dh * va], 1), torch.cat([ega, dh.abs() * eva + edh * (va.abs() + eva)], 1)


def product(a, ea, b, eb):
    """a @ b and its bound, summed in fp32, from operands that are off by ea and eb."""
    n = a.shape[1]
    return a @ b, n * 2.0 ** -23 * (a.abs() @ b.abs()) + ea @ (b.abs() + eb) + a.abs() @ eb


def close(got, want, bound, what):
    """Every element within bound, rounded once to got's type; non-finite ones equal."""
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d off, worst %g where %g is allowed" % (
        what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound.expand_as(off)[bad][off[bad].argmax()]))


def rounded(want, bound, dtype):
    """The bound of a value rounded to dtype at the end."""
    if dtype == torch.float32:
        return bound + 2.0 ** -23 * want.abs()
    return bound * (1 + U[dtype]) + U[dtype] * want.abs() + (TINY if dtype == torch.float16 else 0)


def route(logits, k, score, bias, groups, top_groups, group_best, renorm, scale):
    """(weights fp64, indices, counts, all scores fp64), row by row."""
    T, E = logits.shape
    z = logits.double()
    weights, indices = torch.zeros(T, k, dtype=torch.float64), torch.full((T, k), -1, dtype=torch.int64)
    scores = torch.zeros(T, E, dtype=torch.float64)
    for t in range(T):
        live = [i for i in range(E) if z[t, i] > -math.inf]
        if score == "sigmoid":
            for i in live:
                scores[t, i] = 1 / (1 + math.exp(-z[t, i])) if z[t, i] > -700 else 0.0
        elif live:
            top = max(float(z[t, i]) for i in live)
            e = {i: 1.0 if float(z[t, i]) == top else math.exp(float(z[t, i]) - top) for i in live}
            for i in live:
                scores[t, i] = e[i] / sum(e.values())
        if bias is None and (groups == 1 or group_best == 1):
            key = {i: float(z[t, i]) for i in live}
        else:
            s32 = scores[t].float()
            key = {i: float(s32[i] + bias[i]) if bias is not None else float(s32[i]) for i in live}
        size = E // groups
        rank = []
        for g in range(groups):
            best = sorted((key[i] for i in live if i // size == g), reverse=True)[:group_best]
            rank.append((-float(torch.tensor(best).sum()) if best else math.inf, g))
        kept = {g for _, g in sorted(rank)[:top_groups]}
        chosen = sorted((i for i in live if i // size in kept), key=lambda i: (-key[i], i))[:k]
        total = sum(float(scores[t, i]) for i in chosen) if renorm else 1.0
        for j, i in enumerate(chosen):
            indices[t, j] = i
            weights[t, j] = scale * float(scores[t, i]) / total if total > 0 else 0.0
    counts = torch.bincount(indices[indices >= 0], minlength=E)
    return weights, indices, counts, scores


def experts(x, indices, weights, w1, w2, b1, b2, residual, name, gated, dtype):
    """(y, its bound) in fp64; the weighted hidden values are rounded to dtype once."""
    y = torch.zeros_like(x) if residual is None else residual.clone()
    bound = torch.zeros_like(y)
    for e in range(w1.shape[0]):
        t, j = (indices == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        wt = weights[t, j][:, None]
        h, eh, _, _ = hidden(x[t], w1[e], None if b1 is None else b1[e], name, gated)
        hw = h * wt
        o, eo = product(hw, rounded(hw, eh * wt.abs() + 2.0 ** -23 * hw.abs(), dtype), w2[e].t(), torch.zeros_like(w2[e].t()))
        if b2 is not None:
            o, eo = o + wt * b2[e], eo + 2.0 ** -22 * (wt * b2[e]).abs()
        y.index_add_(0, t, o)
        bound.index_add_(0, t, eo + 2.0 ** -21 * o.abs())
    return y, rounded(y, bound + (0 if residual is None else 2.0 ** -21 * residual.abs()), dtype)


def experts_backward(x, indices, weights, w1, w2, b1, b2, dy, name, gated, dtype):
    """{name: (value, bound)} of every gradient."""
    T, k = indices.shape
    E, rows, D = w1.shape
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    dx, edx, dwt, edwt = zero(T, D), zero(T, D), zero(T, k), zero(T, k)
    out = {n: (zero(*s), zero(*s)) for n, s in (("dw1", w1.shape), ("dw2", w2.shape), ("db1", (E, rows)), ("db2", (E, D)))}
    for e in range(E):
        t, j = (indices == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        xe, g_y, wt = x[t], dy[t], weights[t, j][:, None]
        h, eh, z, ez = hidden(xe, w1[e], None if b1 is None else b1[e], name, gated)
        g, eg = product(g_y, torch.zeros_like(g_y), w2[e], torch.zeros_like(w2[e]))
        d = (h * g).sum(1)
        ed = (eh * (g.abs() + eg) + h.abs() * eg).sum(1) + h.shape[1] * 2.0 ** -23 * (h * g).abs().sum(1)
        if b2 is not None:
            d, ed = d + g_y @ b2[e], ed + (D + 2) * 2.0 ** -23 * (g_y.abs() @ b2[e].abs())
        dwt[t, j], edwt[t, j] = d, ed
        hw, ehw = h * wt, eh * wt.abs()
        dz, edz = hidden_grad(z, ez, g * wt, (eg + 2.0 ** -22 * g.abs()) * wt.abs(), name, gated)
        zz = rounded(dz, edz + 2.0 ** -21 * dz.abs(), dtype)
        px, epx = product(dz, zz, w1[e], torch.zeros_like(w1[e]))
        dx.index_add_(0, t, px)
        edx.index_add_(0, t, epx + 2.0 ** -21 * px.abs())
        for n, (v, ev) in (("dw1", product(dz.t(), zz.t(), xe, torch.zeros_like(xe))),
                           ("dw2", product(g_y.t(), torch.zeros_like(g_y.t()), hw, rounded(hw, ehw + 2.0 ** -22 * hw.abs(), dtype))),
                           ("db1", (dz.sum(0), zz.sum(0) + len(t) * 2.0 ** -23 * dz.abs().sum(0))),
                           ("db2", ((g_y * wt).sum(0), len(t) * 2.0 ** -23 * (g_y * wt).abs().sum(0)))):
            out[n][0][e], out[n][1][e] = v, ev
    res = {"dx": (dx, rounded(dx, edx, dtype)), "dweights": (dwt, edwt)}
    for n, (v, ev) in out.items():
        res[n] = (v, rounded(v, ev, dtype))
    return res
