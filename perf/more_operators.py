"""Cases of the operators that train and serve the dense layers (`paper_2608_24067_b200.layers`), their plain forms and their
definitions in 64 bits.

* norm        y = (h - mean) / sqrt(variance + eps) * weight + bias over the rows of h = x + residual (rounded to x's type: it is
              returned, and what the gradient starts from), and the gradient: dx, dweight, dbias;
* adamw       one step over many tensors at once.  m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
              p = p (1 - rate decay) - rate (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps), with m and v in 32 bits, or in 8 bits
              with one exponent for 256 of them and a rounding that random bits decide;
* quantize    blocks of 32 values of a row as 4-bit floating point (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with a power
              of two for each block, and back;
* linear4     y = act(q(x) q(W)^T + b) + r with q(.) such a quantisation, W quantised once, x in the call.

`own = False` computes them with elementary torch operations in fp32; `own = True` calls the library.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5
RATE, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.05
BLOCK = 256  # elements that share an exponent of an 8-bit state
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
        # one token's norm with the residual stream's sum: decoding, launch latency
        {"name": "norm_step", "op": "norm", "T": 1, "D": 4096, "residual": True, "affine": True, "weights": "same", "type": "bf16"},
        # a prompt's norm in front of a block
        {"name": "norm_prompt", "op": "norm", "T": 8192, "D": 4096, "residual": True, "affine": True, "weights": "same", "type": "bf16"},
        # a training step's gradient, odd number of tokens, added to the residual stream's gradient
        {"name": "norm_train", "op": "norm_backward", "T": 16381, "D": 2048, "residual": True, "affine": True, "weights": "fp32", "type": "bf16"},
        # the step of one small layer of experts, fp32 masters with bf16 copies: launch latency
        {"name": "adamw_small", "op": "adamw", "bits": 32, "layers": 1, "D": 256, "E": 16, "I": 128, "param": "fp32", "grad": "bf16", "copy": "bf16", "scaled": False},
        # two layers of experts, 200 million parameters, the same
        {"name": "adamw_large", "op": "adamw", "bits": 32, "layers": 2, "D": 2048, "E": 16, "I": 1024, "param": "fp32", "grad": "bf16", "copy": "bf16", "scaled": False},
        # the same parameters where memory is short: bf16 parameters, states in 8 bits, read back in full as for a checkpoint
        {"name": "adamw8_large", "op": "adamw", "bits": 8, "layers": 2, "D": 2048, "E": 16, "I": 1024, "param": "bf16", "grad": "bf16", "copy": "none", "scaled": False},
        # odd sizes, tensors that end inside a block, fp16 gradients scaled up
        {"name": "adamw8_odd", "op": "adamw", "bits": 8, "layers": 3, "D": 333, "E": 7, "I": 215, "param": "fp32", "grad": "fp16", "copy": "fp16", "scaled": True},
        # weights prepared for serving
        {"name": "quantize_weights", "op": "quantize", "T": 16384, "D": 4096, "type": "bf16"},
        # a few tokens, as in front of a product
        {"name": "quantize_tokens", "op": "quantize", "T": 77, "D": 2080, "type": "fp32"},
        # one token through a gated projection: decoding, where the weights' bytes and the launch are all there is
        {"name": "linear4_step", "op": "linear4", "T": 1, "D": 4096, "F": 4096, "act": "silu", "gated": True, "bias": False, "residual": False, "type": "bf16"},
        # a batch of single tokens
        {"name": "linear4_batch", "op": "linear4", "T": 77, "D": 2048, "F": 4104, "act": "none", "gated": False, "bias": True, "residual": True, "type": "fp16"},
        # a prompt, everything in the epilogue
        {"name": "linear4_prompt", "op": "linear4", "T": 8192, "D": 4096, "F": 4096, "act": "gelu", "gated": False, "bias": True, "residual": True, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges that the listed ones stand for, no larger than the largest of them."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["norm", "norm_backward", "adamw", "adamw", "quantize", "linear4", "linear4"])
        if op in ("norm", "norm_backward"):
            c = {"op": op, "T": _log(rng, 1, 16384), "D": _log(rng, 64, 8192), "residual": rng.random() < 0.6, "affine": rng.random() < 0.8,
                 "weights": rng.choice(["same", "fp32"]), "type": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
        elif op == "adamw":
            param = rng.choice(["fp32", "fp32", "bf16", "fp16"])
            grad = rng.choice(["fp32", "bf16", "fp16"]) if param == "fp32" else rng.choice(["fp32", param])
            c = {"op": op, "bits": rng.choice([32, 8]), "layers": rng.randint(1, 3), "D": _log(rng, 64, 2048), "E": _log(rng, 2, 16), "I": _log(rng, 32, 1024),
                 "param": param, "grad": grad, "copy": rng.choice(["none", "bf16", "fp16"]) if param == "fp32" else "none", "scaled": rng.random() < 0.4}
        elif op == "quantize":
            c = {"op": op, "T": _log(rng, 1, 16384), "D": 32 * _log(rng, 2, 128), "type": rng.choice(["bf16", "fp16", "fp32"])}
        else:
            c = {"op": op, "T": _log(rng, 1, 8192), "D": 32 * _log(rng, 4, 128), "F": 8 * _log(rng, 8, 512), "act": rng.choice(["none", "relu", "gelu", "silu"]),
                 "gated": rng.random() < 0.4, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5, "type": rng.choice(["bf16", "fp16"])}
        if _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def _size(kind):
    return {"fp32": 4, "none": 0}.get(kind, 2)


def _shapes(c):
    """The tensors of `layers` layers of experts: norm, router, both products."""
    one = [(c["D"],), (c["D"],), (c["E"], c["D"]), (c["E"], 2 * c["I"], c["D"]), (c["E"], c["D"], c["I"])]
    return one * c["layers"]


def work(case):
    """Bytes and operations that a pass cannot do without."""
    c = case
    if c["op"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(c))
        each = 2 * _size(c["param"]) + _size(c["grad"]) + _size(c["copy"])
        # states in 8 bits: read, written, and read back once as 16-bit values that hold them exactly
        each += 16 if c["bits"] == 32 else 4 + 2 + 4
        return {"bytes": n * each, "flops": 16 * n}
    T, D, s = c["T"], c["D"], _size(c["type"])
    if c["op"] in ("norm", "norm_backward"):
        w = 2 * D * (4 if c["weights"] == "fp32" else s) if c["affine"] else 0
        if c["op"] == "norm":
            return {"bytes": T * D * s * (4 if c["residual"] else 2) + w, "flops": 8 * T * D}
        return {"bytes": T * D * s * (4 if c["residual"] else 3) + 3 * w // 2, "flops": 14 * T * D}
    if c["op"] == "quantize":
        return {"bytes": T * D * 2 * s + 2 * (T * D // 2 + T * D // 32), "flops": 4 * T * D}
    F = c["F"]
    rows = F * (2 if c["gated"] else 1)
    return {"bytes": s * (T * D + T * F * (2 if c["residual"] else 1) + (rows if c["bias"] else 0)) + rows * D // 2 + rows * D // 32, "flops": 2 * T * D * rows}


# ---- inputs ---------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    s = {"case": c}
    if c["op"] == "adamw":
        shapes = _shapes(c)
        s["scale"] = torch.full((1,), 2.0 ** -10, device=DEV) if c["scaled"] else None
        s["params"], s["grads"], s["copies"], s["m"], s["v"] = [], [], [], [], []
        s["step"], s["seed"] = 700 + seed % 100, seed % 1000003
        for shape in shapes:
            size = 10 ** float(torch.empty((), device="cpu").uniform_(-4, -2, generator=torch.Generator().manual_seed(seed + len(s["m"]))))
            p = normal(*shape, scale=shape[-1] ** -0.5)
            # gradients of tensors, and of their rows, differ in size; some elements get none
            row = torch.exp(normal(*shape[:-1], 1))
            grad = normal(*shape, scale=size) * row * (torch.rand(*shape, generator=g, device=DEV) > 0.02)
            s["params"].append(p.to(TYPES[c["param"]]))
            s["grads"].append((grad * (2.0 ** 10 if c["scaled"] else 1.0)).to(TYPES[c["grad"]]))
            s["copies"].append(p.to(TYPES[c["copy"]]) if c["copy"] != "none" else None)
            m, v = normal(*shape, scale=0.3 * size) * row, (normal(*shape, scale=size) * row).square() * 0.8
            if c["bits"] == 8:
                m, v = _encode(m, True, 0, 0), _encode(v, False, 0, 0)
            s["m"].append(m)
            s["v"].append(v)
        if own:  # the optimiser that a program keeps, with its states
            from paper_2608_24067_b200 import layers
            s["optimizer"] = layers.AdamW(_layers(), s["params"], copies=s["copies"] if c["copy"] != "none" else None, bits=c["bits"])
            s["optimizer"].load(s["m"], s["v"])
        return s
    t = TYPES[c["type"]]
    T, D = c["T"], c["D"]
    if c["op"] in ("norm", "norm_backward"):
        # channels with their own offsets and sizes, as a residual stream has them
        loud = torch.exp(0.5 * torch.randn(D, generator=g, device=DEV))
        offset = 0.5 * torch.randn(D, generator=g, device=DEV)
        s["x"] = (torch.randn(T, D, generator=g, device=DEV) * loud + offset).to(t)
        wt = t if c["weights"] == "same" else torch.float32
        s["weight"] = (1 + normal(D, scale=0.2)).to(wt) if c["affine"] else None
        s["bias"] = normal(D, scale=0.1, dtype=wt) if c["affine"] else None
        if c["op"] == "norm":
            s["residual"] = normal(T, D, dtype=t) if c["residual"] else None
        else:
            s["dy"] = normal(T, D, dtype=t)
            s["dsum"] = normal(T, D, dtype=t) if c["residual"] else None
    elif c["op"] == "quantize":
        loud = torch.exp(torch.randn(D, generator=g, device=DEV))
        s["x"] = (torch.randn(T, D, generator=g, device=DEV) * loud).to(t)
    else:
        F = c["F"]
        rows = F * (2 if c["gated"] else 1)
        s["x"] = normal(T, D, dtype=t)
        w = normal(rows, D, scale=D ** -0.5, dtype=t)
        if own:  # the weights as a serving program keeps them
            s["weight"] = _layers().quantize_fp4(w)
        else:
            s["weight"] = _quantize(w)
        s["bias"] = normal(rows, scale=0.1, dtype=t) if c["bias"] else None
        s["residual"] = normal(T, F, dtype=t) if c["residual"] else None
    return s


# ---- one pass -------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        L = _layers()
        if c["op"] == "norm":
            return L.norm(s["x"], s["weight"], s["bias"], s["residual"], eps=EPS)
        if c["op"] == "norm_backward":
            return L.norm_backward(s["x"], s["weight"], s["dy"], s["bias"], s["dsum"], eps=EPS)
        if c["op"] == "adamw":
            o = s["optimizer"]
            o.step(s["grads"], rate=RATE, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, decay=DECAY, step=s["step"], scale=s["scale"], seed=s["seed"])
            m, v = o.moments()
            return {"params": s["params"], "copies": s["copies"], "m": m, "v": v}
        if c["op"] == "quantize":
            return L.values_fp4(L.quantize_fp4(s["x"]), dtype=s["x"].dtype)
        return L.linear_fp4(s["x"], s["weight"], s["bias"], s["residual"], act=c["act"], gated=c["gated"])
    return {"norm": _norm, "norm_backward": _norm_backward, "adamw": _adamw, "quantize": _there_and_back, "linear4": _linear4}[c["op"]](s, c)


def _norm(s, c):
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
    v = h.float()
    v = v - v.mean(1, keepdim=True)
    y = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    if s["weight"] is not None:
        y = y * s["weight"].float() + s["bias"].float()
    y = y.to(h.dtype)
    return y if s["residual"] is None else {"y": y, "sum": h}


def _norm_backward(s, c):
    x, dy = s["x"].float(), s["dy"].float()
    v = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    n = v * r
    d = dy if s["weight"] is None else dy * s["weight"].float()
    dx = r * (d - d.mean(1, keepdim=True) - n * (d * n).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    out = {"dx": dx.to(s["x"].dtype)}
    if s["weight"] is not None:
        out |= {"dweight": (dy * n).sum(0).to(s["weight"].dtype), "dbias": dy.sum(0).to(s["bias"].dtype)}
    return out


def _mix(x):
    """Bits of whole numbers below 2^32, well mixed."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B9) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(n, seed, tensor, device):
    """32 random bits for each of n elements of the tensor with this number."""
    i = torch.arange(n, device=device)
    block = _mix(torch.arange(-(-n // BLOCK), device=device))
    key = _mix(block ^ ((seed + tensor * 0x9E3779B9) & 0xFFFFFFFF))
    return _mix((key[i // BLOCK] + (i % BLOCK) * 0x6A09E667) & 0xFFFFFFFF)


def _encode(x, signed, bits, nonzero):
    """8-bit codes of fp32 values and the exponent of each block of 256 (that of the largest magnitude, one more where its fraction is above the
    codes' last, 7 / 8): the code is the top of the fp32 number scaled so that the block's exponent is 15 (signed: a sign, 4 bits of
    exponent and 3 of fraction) or 31 (5 and 3), rounded up where the 20 bits below, plus 20 random ones (16 drawn), pass 2^20.
    nonzero: a positive value does not become 0."""
    flat = x.reshape(-1)
    n, blocks = flat.numel(), -(-flat.numel() // BLOCK)
    a = flat.abs()
    e = torch.zeros(blocks * BLOCK, dtype=torch.int32, device=x.device).index_copy_(0, torch.arange(n, device=x.device), a.view(torch.int32))
    e = (e.view(blocks, BLOCK).amax(1).clamp_max(0x7F800000) + 0x100000) >> 23
    up = torch.exp2((127 - e).double()).float()[torch.arange(n, device=x.device) // BLOCK]
    scaled = (a * up) * (2.0 ** -112 if signed else 2.0 ** -96)
    code = ((scaled.view(torch.int32) + (bits << 4)) >> 20).clamp_max(127 if signed else 255)
    if signed:
        code = code | ((flat < 0).int() << 7)
    if nonzero:
        code = torch.where((flat > 0) & (code == 0), 1, code)
    return code.to(torch.uint8), e.to(torch.uint8)


def _decode(state, signed, shape):
    code, e = state[0].int(), state[1]
    at = torch.arange(code.numel(), device=code.device) // BLOCK
    v = ((code & 127 if signed else code) << 20).view(torch.float32) * (2.0 ** 112 if signed else 2.0 ** 96)
    v = v * torch.exp2(e.double() - 127).float()[at]
    return (torch.where(code > 127, -v, v) if signed else v).view(shape)


def _adamw_one(s, c, i):
    p, copy, m, v = s["params"][i], s["copies"][i], s["m"][i], s["v"][i]
    g = s["grads"][i].float()
    if s["scale"] is not None:
        g = g * s["scale"]
    if c["bits"] == 8:
        m, v = _decode(m, True, p.shape), _decode(v, False, p.shape)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    t = s["step"]
    change = (m * (1 / (1 - BETA1 ** t))) / (torch.sqrt(v * (1 / (1 - BETA2 ** t))) + ADAM_EPS)
    new = p.float() * (1 - RATE * DECAY) - change * RATE
    p.copy_(new)
    if copy is not None:
        copy.copy_(new)
    if c["bits"] == 32:
        s["m"][i].copy_(m)
        s["v"][i].copy_(v)
        return s["m"][i], s["v"][i]
    r = _random_bits(p.numel(), s["seed"], i, p.device)
    s["m"][i], s["v"][i] = _encode(m, True, (r & 0xFFFF).int(), False), _encode(v, False, (r >> 16).int(), True)
    return _decode(s["m"][i], True, p.shape).bfloat16(), _decode(s["v"][i], False, p.shape).bfloat16()


def _adamw(s, c):
    states = [_adamw_one(s, c, i) for i in range(len(s["params"]))]
    return {"params": s["params"], "copies": s["copies"], "m": [a for a, _ in states], "v": [b for _, b in states]}


def _steps_of(device):
    """Between which 4-bit values a magnitude lies: half way to the next; a tie goes to the even code."""
    return torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=device), torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=device)


def _quantize(x):
    """Codes (0 to 15, two a byte, the even column in the low half) and the exponents of the blocks of 32.  The block's power of two is that
    of its largest magnitude over 4, one more where that magnitude is 1.75 times a power of two or more (it would round to 8)."""
    v = x.float().view(x.shape[0], -1, 32)
    a = v.abs()
    top = a.amax(2, keepdim=True).view(torch.int32)
    e = ((top + 0x200000) >> 23) - 127 - 2  # the carry of a fraction of 0.75 and more goes into the exponent
    e = e.clamp_min(-127)
    scaled = a * torch.exp2(-e.double()).float()
    half, _ = _steps_of(x.device)
    code = torch.bucketize(scaled, half)  # a tie goes down here,
    code = code + ((code % 2 == 1) & (scaled == half[code.clamp_max(6)]))  # and up where the lower code is odd
    code = (code | (torch.signbit(v).long() << 3)).view(x.shape).to(torch.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), (e.squeeze(2) + 127).to(torch.uint8)


def _values(q):
    pairs, e = q
    code = torch.stack([pairs & 15, pairs >> 4], 2).view(pairs.shape[0], -1).int()
    _, value = _steps_of(code.device)
    v = value[code & 7]
    v = torch.where(code > 7, -v, v)
    return (v.view(v.shape[0], -1, 32) * torch.exp2(e.double() - 127).float()[:, :, None]).view(v.shape)


def _there_and_back(s, c):
    return _values(_quantize(s["x"])).to(s["x"].dtype)


def _act(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _linear4(s, c):
    z = _values(_quantize(s["x"])) @ _values(s["weight"]).t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    if c["gated"]:
        a, b = z.chunk(2, dim=1)
        y = _act(a, c["act"]) * b
    else:
        y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------

_F = {"none": lambda v: v, "relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


def _exact_fp4(x):
    """The values that a matrix in 4 bits stands for, by search of the nearest."""
    v = x.double().view(x.shape[0], -1, 32)
    top = v.abs().amax(2, keepdim=True)
    fraction, power = torch.frexp(top)  # top = fraction 2^power, fraction in [0.5, 1)
    unit = torch.exp2((power - 3 + (fraction >= 0.875)).double().clamp_min(-127))
    a = v.abs() / unit
    best = torch.zeros_like(a)
    for k, value in enumerate((0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), start=1):
        near, far = (a - best).abs(), (a - value).abs()
        best = torch.where((far < near) | ((far == near) & (k % 2 == 0)), value, best)
    return (torch.copysign(best, v) * unit).view(x.shape)


def _exact_state(state, signed, shape):
    """What the 8-bit codes say: (1 + f / 8) 2^(e - top), f / 8 2^(1 - top) where e is 0, times 2 to the block's exponent."""
    code, e = state[0].long(), state[1].double()
    top = 15 if signed else 31
    size = code & 127 if signed else code
    exponent, f = size >> 3, (size & 7).double() / 8
    v = torch.where(exponent > 0, (1 + f) * torch.exp2((exponent - top).double()), f * 2.0 ** (1 - top))
    v = v * torch.exp2(e - 127).repeat_interleave(BLOCK)[:code.numel()]
    return (torch.where(code > 127, -v, v) if signed else v).view(shape)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = (h + s["residual"].double()).to(s["x"].dtype).double()
        wide = [v.double() if v is not None else None for v in (s["weight"], s["bias"])]
        y = torch.nn.functional.layer_norm(h, (c["D"],), *wide, EPS)
        return y if s["residual"] is None else {"y": y, "sum": s["x"].double() + s["residual"].double()}
    if c["op"] == "norm_backward":
        x = s["x"].double().requires_grad_()
        w, b = (v.double().requires_grad_() if v is not None else None for v in (s["weight"], s["bias"]))
        torch.nn.functional.layer_norm(x, (c["D"],), w, b, EPS).backward(s["dy"].double())
        out = {"dx": x.grad if s["dsum"] is None else x.grad + s["dsum"].double()}
        if w is not None:
            out |= {"dweight": w.grad, "dbias": b.grad}
        return out
    if c["op"] == "adamw":
        out = {"params": [], "copies": [], "m": [], "v": []}
        for p, g, m, v, copy in zip(s["params"], s["grads"], s["m"], s["v"], s["copies"]):
            g = g.double() * (s["scale"].double() if s["scale"] is not None else 1.0)
            if c["bits"] == 8:
                m, v = _exact_state(m, True, p.shape), _exact_state(v, False, p.shape)
            m = torch.lerp(m.double(), g, 1 - BETA1)
            v = torch.lerp(v.double(), g.square(), 1 - BETA2)
            t = s["step"]
            new = p.double() - RATE * (DECAY * p.double() + (m / -math.expm1(t * math.log(BETA1))) / ((v / -math.expm1(t * math.log(BETA2))).sqrt() + ADAM_EPS))
            out["params"].append(new)
            out["copies"].append(new if copy is not None else None)
            # which of two neighbouring 8-bit codes is taken is the random bits' choice, not a value of its own
            out["m"].append(m if c["bits"] == 32 else None)
            out["v"].append(v if c["bits"] == 32 else None)
        return out
    if c["op"] == "quantize":
        return _exact_fp4(s["x"])
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = TYPES[c["type"]]  # the weights before their quantisation, drawn again
    torch.randn(c["T"], c["D"], generator=g, device=DEV)
    rows = c["F"] * (2 if c["gated"] else 1)
    w = (torch.randn(rows, c["D"], generator=g, device=DEV) * c["D"] ** -0.5).to(t)
    z = torch.nn.functional.linear(_exact_fp4(s["x"]), _exact_fp4(w), s["bias"].double() if s["bias"] is not None else None)
    y = _F[c["act"]](z[:, :c["F"]]) * z[:, c["F"]:] if c["gated"] else _F[c["act"]](z)
    return y if s["residual"] is None else y + s["residual"].double()
