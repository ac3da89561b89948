"""Cases of the dense operators (`paper_2608_24067_b200.layers`), their plain forms and their definitions in 64 bits.

Three operators, each with its gradient:

* linear   y = act(x W^T + b) + r, the activation optionally gated (first half of W's rows gates the second half);
* route    scores of a token's logits, an optional bias for balance, an optional choice of groups, the k best experts
           (ties to the lowest index), their weights and the number of tokens of every expert;
* experts  y_t = r_t + sum_j w_tj (W2_e act(W1_e x_t + b1_e) + b2_e), e = indices[t, j]; an index of -1 is no expert.

`own = False` computes them with elementary torch operations in fp32; `own = True` calls the library.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_handle = None


def _layers():
    """The library's handle, made once as a user's program keeps it."""
    global _handle
    if _handle is None:
        from paper_2608_24067_b200 import layers
        _handle = layers.Layers()
    return _handle


# ---- cases ----------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token through a gated projection: decoding, where the weights' bytes and the launch are all there is
        {"name": "linear_step", "op": "linear", "T": 1, "D": 4096, "F": 4096, "act": "silu", "gated": True, "bias": False, "residual": False, "type": "bf16"},
        # the router's own product over a long prompt: many rows, few columns
        {"name": "linear_logits", "op": "linear", "T": 8192, "D": 2048, "F": 256, "act": "none", "gated": False, "bias": False, "residual": False, "type": "fp16"},
        # a block's projection over a prompt with everything in its epilogue
        {"name": "linear_prompt", "op": "linear", "T": 4096, "D": 4096, "F": 4096, "act": "gelu", "gated": False, "bias": True, "residual": True, "type": "bf16"},
        # a training step of a projection, odd number of tokens
        {"name": "linear_train", "op": "linear_backward", "T": 4093, "D": 2048, "F": 4096, "act": "gelu", "gated": False, "bias": True, "type": "bf16"},
        # one token's routing: launch latency
        {"name": "route_step", "op": "route", "T": 1, "E": 64, "k": 8, "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "group_best": 1, "renorm": True, "masked": False, "type": "fp32"},
        # a prompt's routing over many experts with groups and a balance bias
        {"name": "route_prompt", "op": "route", "T": 16384, "E": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "group_best": 2, "renorm": True, "masked": False, "type": "fp32"},
        # the gradient of routing, odd sizes, masked experts and padding tokens (rows whose mask leaves nothing)
        {"name": "route_train", "op": "route_backward", "T": 16381, "E": 100, "k": 6, "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "group_best": 1, "renorm": False, "masked": True, "type": "bf16"},
        # one token through its eight experts
        {"name": "experts_step", "op": "experts", "T": 1, "E": 64, "k": 8, "D": 2048, "I": 1024, "act": "silu", "gated": True, "bias": False, "residual": False, "pad": 0.0, "type": "bf16"},
        # a batch of single tokens from many requests: nearly every expert has a few tokens
        {"name": "experts_batch", "op": "experts", "T": 96, "E": 64, "k": 6, "D": 2048, "I": 1024, "act": "silu", "gated": True, "bias": True, "residual": True, "pad": 0.0, "type": "fp16"},
        # a prompt
        {"name": "experts_prompt", "op": "experts", "T": 4096, "E": 64, "k": 8, "D": 2048, "I": 1024, "act": "silu", "gated": True, "bias": False, "residual": True, "pad": 0.0, "type": "bf16"},
        # a training step
        {"name": "experts_train", "op": "experts_backward", "T": 4096, "E": 32, "k": 4, "D": 2048, "I": 1024, "act": "silu", "gated": True, "bias": False, "pad": 0.0, "type": "bf16"},
        # a small training step with ragged sizes, biases and padding tokens that have no expert
        {"name": "experts_train_odd", "op": "experts_backward", "T": 777, "E": 12, "k": 2, "D": 1000, "I": 712, "act": "gelu", "gated": False, "bias": True, "pad": 0.1, "type": "fp16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges that the listed ones stand for, no larger than the largest of them."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["linear", "linear", "linear_backward", "route", "route", "route_backward", "experts", "experts", "experts_backward"])
        if op in ("linear", "linear_backward"):
            c = {"op": op, "T": _log(rng, 1, 8192), "D": 8 * _log(rng, 8, 512), "F": 8 * _log(rng, 8, 512), "act": rng.choice(["none", "relu", "gelu", "silu"]),
                 "gated": rng.random() < 0.4, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5, "type": rng.choice(["bf16", "fp16"])}
            if op == "linear_backward":
                del c["residual"]
        elif op in ("route", "route_backward"):
            groups = rng.choice([1, 1, 2, 4, 8])
            E = groups * _log(rng, 4, 512 // groups)
            top = rng.randint(1, groups)
            c = {"op": op, "T": _log(rng, 1, 16384), "E": E, "k": min(rng.randint(2, 12), top * E // groups), "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5,
                 "groups": groups, "top_groups": top, "group_best": rng.choice([1, 2]), "renorm": rng.random() < 0.6, "masked": rng.random() < 0.3, "type": rng.choice(["fp32", "bf16", "fp16"])}
        else:
            E = _log(rng, 4, 96)
            c = {"op": op, "T": _log(rng, 1, 4096), "E": E, "k": rng.randint(1, min(E, 8)), "D": 8 * _log(rng, 32, 256), "I": 8 * _log(rng, 16, 192), "act": rng.choice(["relu", "gelu", "silu"]),
                 "gated": rng.random() < 0.6, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5, "pad": rng.choice([0.0, 0.0, 0.1]), "type": rng.choice(["bf16", "fp16"])}
            if op == "experts_backward":
                del c["residual"]
        if _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def work(case):
    """Bytes and operations that a pass cannot do without."""
    T, s = case["T"], 4 if case["type"] == "fp32" else 2
    if case["op"] in ("route", "route_backward"):
        E, k = case["E"], case["k"]
        if case["op"] == "route":
            return {"bytes": T * E * s + T * k * 8 + E * 4 * (2 if case["bias"] else 1), "flops": 4 * T * E}
        whole = case["score"] == "softmax" and not case["renorm"]  # (else only the chosen experts' logits matter)
        return {"bytes": T * (E if whole else k) * s + T * k * 8 + T * E * s, "flops": 4 * T * E}
    D = case["D"]
    if case["op"] in ("linear", "linear_backward"):
        F = case["F"]
        rows = F * (2 if case["gated"] else 1)
        if case["op"] == "linear":
            return {"bytes": s * (T * D + rows * D + T * F * (2 if case["residual"] else 1) + (rows if case["bias"] else 0)), "flops": 2 * T * D * rows}
        again = 0 if case["act"] == "none" and not case["gated"] else 1  # the pre-activation
        return {"bytes": s * (2 * T * D + 2 * rows * D + T * F + (2 * rows if case["bias"] else 0)), "flops": 2 * T * D * rows * (2 + again)}
    E, k, I = case["E"], case["k"], case["I"]
    rows = I * (2 if case["gated"] else 1)
    active = E * (1 - (1 - k / E) ** T)  # experts that get a token, expected
    each = rows * D + I * D + (rows + D if case["bias"] else 0)
    slots = T * k
    if case["op"] == "experts":
        return {"bytes": s * (active * each + T * D * (3 if case["residual"] else 2)) + slots * 8, "flops": 2 * slots * D * (rows + I)}
    return {"bytes": s * (active * each + E * each + 3 * T * D) + slots * 8, "flops": 2 * slots * D * (3 * rows + 2 * I)}


# ---- inputs ---------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = TYPES[case["type"]]
    T = case["T"]

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    s = {"case": case}
    if case["op"] in ("linear", "linear_backward"):
        D, F = case["D"], case["F"]
        rows = F * (2 if case["gated"] else 1)
        s["x"] = normal(T, D)
        s["weight"] = normal(rows, D, scale=D ** -0.5)
        s["bias"] = normal(rows, scale=0.1) if case["bias"] else None
        s["residual"] = normal(T, F) if case.get("residual") else None
        if case["op"] == "linear_backward":
            s["dy"] = normal(T, F)
    elif case["op"] in ("route", "route_backward"):
        E, k = case["E"], case["k"]
        liked = torch.randn(E, generator=g, device=DEV)  # some experts are popular
        z = torch.randn(T, E, generator=g, device=DEV) * 1.5 + liked
        if case["masked"]:
            z = z.masked_fill(torch.rand(E, generator=g, device=DEV) < 0.05, -math.inf)
            z = z.masked_fill(torch.rand(T, 1, generator=g, device=DEV) < 0.05, -math.inf)
        s["logits"] = z.to(t)
        s["bias"] = torch.randn(E, generator=g, device=DEV) * 0.05 if case["bias"] else None
        if case["op"] == "route_backward":
            s["indices"] = _choose(s["logits"], s["bias"], case)
            s["dweights"] = torch.randn(T, k, generator=g, device=DEV)
    else:
        E, k, D, I = case["E"], case["k"], case["D"], case["I"]
        rows = I * (2 if case["gated"] else 1)
        s["x"] = normal(T, D)
        z = torch.randn(T, E, generator=g, device=DEV) + 0.5 * torch.randn(E, generator=g, device=DEV)
        best, at = z.topk(k, dim=1)
        weights = best.softmax(1)
        none = torch.rand(T, 1, generator=g, device=DEV) < case["pad"]
        s["indices"] = torch.where(none, -1, at).int().contiguous()
        # a training step keeps the weights in the tokens' type, serving in fp32 as the router gives them
        s["weights"] = weights.masked_fill(none, 0.0).to(t if case["op"] == "experts_backward" else torch.float32).contiguous()
        s["w1"] = normal(E, rows, D, scale=D ** -0.5)
        s["w2"] = normal(E, D, I, scale=I ** -0.5)
        s["b1"] = normal(E, rows, scale=0.1) if case["bias"] else None
        s["b2"] = normal(E, D, scale=0.1) if case["bias"] else None
        s["residual"] = normal(T, D) if case.get("residual") else None
        if case["op"] == "experts_backward":
            s["dy"] = normal(T, D)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        L = _layers()
        if c["op"] == "linear":
            return L.linear(s["x"], s["weight"], s["bias"], s["residual"], act=c["act"], gated=c["gated"])
        if c["op"] == "linear_backward":
            return L.linear_backward(s["x"], s["weight"], s["dy"], s["bias"], act=c["act"], gated=c["gated"])
        if c["op"] == "route":
            return L.route(s["logits"], c["k"], score=c["score"], bias=s["bias"], groups=c["groups"], top_groups=c["top_groups"],
                           group_best=c["group_best"], renorm=c["renorm"], scale=1.0)
        if c["op"] == "route_backward":
            return L.route_backward(s["logits"], s["indices"], s["dweights"], score=c["score"], renorm=c["renorm"], scale=1.0)
        if c["op"] == "experts":
            return L.experts(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], s["b1"], s["b2"], s["residual"], act=c["act"], gated=c["gated"])
        return L.experts_backward(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], s["dy"], s["b1"], s["b2"], act=c["act"], gated=c["gated"])
    return {"linear": _linear, "linear_backward": _linear_backward, "route": _route, "route_backward": _route_backward,
            "experts": _experts, "experts_backward": _experts_backward}[c["op"]](s, c)


def _act(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _activate(z, act, gated):
    if not gated:
        return _act(z, act)
    a, b = z.chunk(2, dim=-1)
    return _act(a, act) * b


def _activate_grad(z, dh, act, gated):
    if not gated:
        return dh * _act_grad(z, act)
    a, b = z.chunk(2, dim=-1)
    return torch.cat([dh * b * _act_grad(a, act), dh * _act(a, act)], dim=-1)


def _linear(s, c):
    z = s["x"].float() @ s["weight"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _activate(z, c["act"], c["gated"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _linear_backward(s, c):
    x, w, dy = s["x"].float(), s["weight"].float(), s["dy"].float()
    dz = dy
    if c["act"] != "none" or c["gated"]:
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        dz = _activate_grad(z, dy, c["act"], c["gated"])
    t = s["x"].dtype
    out = {"dx": (dz @ w).to(t), "dweight": (dz.t() @ x).to(t)}
    if s["bias"] is not None:
        out["dbias"] = dz.sum(0).to(t)
    return out


def _scores(logits, score):
    # A score is rounded to fp32 from 64 bits, so that which of two near scores is the larger does not hang on one library's exp.
    z = logits.double()
    if score == "sigmoid":
        return torch.sigmoid(z).float()
    e = torch.exp(z - z.amax(1, keepdim=True).clamp_min(-1e300))
    return (e / e.sum(1, keepdim=True).clamp_min(1e-300)).float()


def _choose(logits, bias, c):
    """Indices of the k experts with the largest keys, best first, ties to the lowest index; -1 where none is left."""
    z = logits.float()
    T, E = z.shape
    G = c["groups"]
    if bias is None and (G == 1 or c["group_best"] == 1):
        keys = z  # scores grow with the logits
    else:
        keys = _scores(logits, c["score"])
        keys = (keys if bias is None else keys + bias).masked_fill(z == -math.inf, -math.inf)
    if G > 1:
        best = keys.view(T, G, E // G).topk(min(c["group_best"], E // G), dim=2).values
        some = best[..., :1] > -math.inf
        group = best.masked_fill(best == -math.inf, 0.0).sum(2, keepdim=True).masked_fill(~some, -math.inf).squeeze(2)
        order = torch.sort(group, dim=1, descending=True, stable=True).indices
        kept = torch.zeros(T, G, dtype=torch.bool, device=z.device).scatter_(1, order[:, :c["top_groups"]], True)
        keys = keys.masked_fill(~kept.repeat_interleave(E // G, dim=1), -math.inf)
    best, at = torch.sort(keys, dim=1, descending=True, stable=True)
    return torch.where(best[:, :c["k"]] > -math.inf, at[:, :c["k"]], -1).int()


def _route(s, c):
    at = _choose(s["logits"], s["bias"], c)
    none = at < 0
    w = _scores(s["logits"], c["score"]).gather(1, at.clamp_min(0).long()).masked_fill(none, 0.0)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1.2e-38)
    counts = torch.zeros(c["E"] + 1, dtype=torch.int32, device=at.device)
    counts = counts.index_add_(0, torch.where(none, c["E"], at).reshape(-1), torch.ones_like(at).reshape(-1))
    return {"weights": w, "indices": at, "counts": counts[:c["E"]]}


def _route_backward(s, c):
    z, at, dw = s["logits"], s["indices"], s["dweights"]
    none = at < 0
    to = at.clamp_min(0).long()
    p = _scores(z, c["score"])
    q = p.gather(1, to).masked_fill(none, 0.0)
    d = dw.masked_fill(none, 0.0)
    if c["renorm"]:
        total = q.sum(1, keepdim=True).clamp_min(1.2e-38)
        d = ((d - (d * q).sum(1, keepdim=True) / total) / total).masked_fill(none, 0.0)
    ds = torch.zeros_like(p).scatter_add_(1, to, d)
    if c["score"] == "sigmoid":
        return (ds * p * (1 - p)).to(z.dtype)
    return (p * (ds - (p * ds).sum(1, keepdim=True))).to(z.dtype)


def _pack(at, E):
    """The slots (token, place) with an expert, in the experts' order: slot, expert and place among the expert's own; the most that one has."""
    flat = at.reshape(-1).long()
    key, order = torch.sort(torch.where(flat < 0, E, flat), stable=True)
    counts = torch.bincount(key, minlength=E + 1)
    place = torch.arange(len(flat), device=at.device) - (counts.cumsum(0) - counts)[key]
    some = int(counts[:E].sum())
    return order[:some], key[:some], place[:some], int(counts[:E].max())


def _products(s, c):
    """Each slot's rows and weights as batches of products: (rows in, rows out, W1, W2, b1, b2), one batch an expert, or a slot where there are few."""
    at, E = s["indices"], c["E"]
    slot, e, place, most = _pack(at, E)
    w1, w2, b1, b2 = s["w1"], s["w2"], s["b1"], s["b2"]
    if len(slot) <= E:  # few slots: only their experts' weights
        w1, w2, b1, b2 = w1[e], w2[e], b1[e] if b1 is not None else None, b2[e] if b2 is not None else None
        batch, place, n, most = torch.arange(len(slot), device=at.device), torch.zeros_like(place), len(slot), 1
    else:
        batch, n = e, E
    wide = [v.float() if v is not None else None for v in (w1, w2, b1, b2)]

    def fill(v):
        return torch.zeros(n, most, v.shape[1], device=v.device).index_put_((batch, place), v)

    return slot, e, fill, lambda v: v[batch, place], wide


def _experts(s, c):
    T, k = s["indices"].shape
    slot, e, fill, take, (w1, w2, b1, b2) = _products(s, c)
    z = fill(s["x"].float()[slot // k]) @ w1.transpose(1, 2)
    if b1 is not None:
        z = z + b1[:, None]
    o = _activate(z, c["act"], c["gated"]) @ w2.transpose(1, 2)
    if b2 is not None:
        o = o + b2[:, None]
    o = take(o) * s["weights"].float().reshape(-1)[slot, None]
    y = torch.zeros(T * k, o.shape[1], device=o.device).index_copy_(0, slot, o).view(T, k, -1).sum(1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _experts_backward(s, c):
    T, k = s["indices"].shape
    E, t = c["E"], s["x"].dtype
    slot, e, fill, take, (w1, w2, b1, b2) = _products(s, c)
    wt = s["weights"].float().reshape(-1)[slot, None]
    x, dy = fill(s["x"].float()[slot // k]), s["dy"].float()[slot // k]
    z = x @ w1.transpose(1, 2)
    if b1 is not None:
        z = z + b1[:, None]
    h = _activate(z, c["act"], c["gated"])
    o = h @ w2.transpose(1, 2)
    if b2 is not None:
        o = o + b2[:, None]
    dweights = torch.zeros(T * k, device=x.device).index_copy_(0, slot, (take(o) * dy).sum(1))
    do = fill(dy * wt)
    dz = _activate_grad(z, do @ w2, c["act"], c["gated"])
    dx = torch.zeros(T * k, x.shape[2], device=x.device).index_copy_(0, slot, take(dz @ w1)).view(T, k, -1).sum(1)

    def whole(v, like):  # the gradient of every expert's weights from that of the batches
        return v if v.shape[0] == E and len(slot) > E else torch.zeros(E, *like.shape[1:], device=v.device).index_add_(0, e, v)

    out = {"dx": dx.to(t), "dweights": dweights.view(T, k).to(s["weights"].dtype),
           "dw1": whole(dz.transpose(1, 2) @ x, s["w1"]).to(t), "dw2": whole(do.transpose(1, 2) @ h, s["w2"]).to(t)}
    if b1 is not None:
        out["db1"] = whole(dz.sum(1), s["b1"]).to(t)
        out["db2"] = whole(do.sum(1), s["b2"]).to(t)
    return out


# ---- the definitions in 64 bits -------------------------------------------------------------------------------

_F = {"none": lambda v: v, "relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


def _unit(x, w, b, act, gated):
    z = torch.nn.functional.linear(x, w, b)
    if gated:
        n = z.shape[-1] // 2
        return _F[act](z[..., :n]) * z[..., n:]
    return _F[act](z)


def _exact_route(s, c):
    z = s["logits"].double().cpu().numpy()
    T, E = z.shape
    G, k = c["groups"], c["k"]
    live = z > -np.inf
    if c["score"] == "sigmoid":
        p = 1 / (1 + np.exp(-z))
    else:
        top = np.where(live.any(1), z.max(1), 0.0)[:, None]
        p = np.exp(z - top)
        p = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
    if s["bias"] is None and (G == 1 or c["group_best"] == 1):
        keys = z.copy()
    else:
        keys = p.astype(np.float32)
        if s["bias"] is not None:
            keys = keys + s["bias"].cpu().numpy()
        keys = np.where(live, keys, -np.inf)
    if G > 1:
        split = np.sort(keys.reshape(T, G, -1), axis=2)[:, :, ::-1][:, :, :c["group_best"]]
        gk = np.where(split[:, :, 0] > -np.inf, np.where(split > -np.inf, split, 0).sum(2, dtype=keys.dtype), -np.inf)
        out = np.ones((T, G), bool)
        for _ in range(c["top_groups"]):
            g = np.where(out, gk, -np.inf).argmax(1)
            out[np.arange(T), g] = False
        keys = np.where(np.repeat(out, E // G, axis=1), -np.inf, keys)
    at = np.full((T, k), -1)
    for j in range(k):
        i = keys.argmax(1)
        ok = keys[np.arange(T), i] > -np.inf
        at[ok, j] = i[ok]
        keys[np.arange(T), i] = -np.inf
    return at, p


def exact(case, seed):
    c = case
    if work(c)["flops"] > 2e12:
        return None
    s = prepare(case, seed)
    if c["op"] in ("route", "route_backward"):
        at, p = _exact_route(s, c) if c["op"] == "route" else (s["indices"].cpu().numpy(), None)
        if c["op"] == "route":
            w = np.where(at < 0, 0.0, np.take_along_axis(p, np.maximum(at, 0), 1))
            if c["renorm"]:
                w = w / np.maximum(w.sum(1, keepdims=True), 1e-300)
            return {"weights": torch.from_numpy(w), "indices": torch.from_numpy(at), "counts": torch.from_numpy(np.bincount(at[at >= 0], minlength=c["E"]))}
        z = s["logits"].double()
        dead = torch.isinf(z)
        z = z.masked_fill(dead, -1e4).requires_grad_()
        q = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z, 1)
        at = s["indices"].long()
        w = q.gather(1, at.clamp_min(0)) * (at >= 0)
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
        (w * s["dweights"].double()).sum().backward()
        return z.grad.masked_fill(dead, 0.0)
    x = s["x"].double()
    wide = lambda n: s[n].double() if s.get(n) is not None else None  # noqa: E731
    if c["op"] == "linear":
        y = _unit(x, wide("weight"), wide("bias"), c["act"], c["gated"])
        return y if s["residual"] is None else y + wide("residual")
    if c["op"] == "linear_backward":
        x.requires_grad_()
        w, b = wide("weight").requires_grad_(), wide("bias")
        if b is not None:
            b.requires_grad_()
        _unit(x, w, b, c["act"], c["gated"]).backward(wide("dy"))
        out = {"dx": x.grad, "dweight": w.grad}
        if b is not None:
            out["dbias"] = b.grad
        return out
    back = c["op"] == "experts_backward"
    wt = s["weights"].double()
    dx = torch.zeros_like(x)
    y = torch.zeros_like(x) if s.get("residual") is None else wide("residual")
    dwt = torch.zeros_like(wt)
    grads = {n: torch.zeros(s[n].shape, dtype=torch.float64, device=x.device) if back and s[n] is not None else None for n in ("w1", "w2", "b1", "b2")}
    for e in range(c["E"]):
        tok, place = (s["indices"] == e).nonzero(as_tuple=True)
        if not len(tok):
            continue
        xe = x[tok].requires_grad_(back)
        we = wt[tok, place].requires_grad_(back)
        part = {n: s[n][e].double().requires_grad_(back) if s[n] is not None else None for n in ("w1", "w2", "b1", "b2")}
        o = torch.nn.functional.linear(_unit(xe, part["w1"], part["b1"], c["act"], c["gated"]), part["w2"], part["b2"]) * we[:, None]
        if not back:
            y = y.index_add(0, tok, o)
            continue
        o.backward(s["dy"][tok].double())
        dx.index_add_(0, tok, xe.grad)
        dwt[tok, place] = we.grad
        for n in grads:
            if part[n] is not None:
                grads[n][e] = part[n].grad
    if not back:
        return y
    out = {"dx": dx, "dweights": dwt, "dw1": grads["w1"], "dw2": grads["w2"]}
    if s["b1"] is not None:
        out |= {"db1": grads["b1"], "db2": grads["b2"]}
    return out
