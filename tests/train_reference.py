"""Definitions in 64 bits of the operators around the dense layers (norm, AdamW, matrices in 4 bits), and what fp32 may lose.

A sum of n terms in fp32 whose longest chain of additions has k links is off by at most k 2^-24 times the sum of the terms'
magnitudes (to first order); every other operation by 2^-24 of its result.  The tolerances below count those and the last rounding."""
import numpy as np
import torch

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(t):
    """The last rounding: half a step relative to the value, and half of the smallest subnormal (2^-149, bf16 2^-133, fp16 2^-24)."""
    return torch.finfo(t).eps / 2, {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}[t]


def chain(n):
    """Links of the longest chain of additions in a sum of n: at most n / 64 in a row in a thread, then a tree or 32 parts."""
    return n / 64 + 48


def norm(x, weight, bias, residual, eps):
    """y, sum and y's tolerance."""
    t, D = x.dtype, x.shape[1]
    h = x.double()
    if residual is not None:
        h = (x.float() + residual.float()).to(t).double()
    mean = h.mean(1, keepdim=True)
    c = h - mean
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    n = c * r
    w = weight.double() if weight is not None else torch.ones(D, dtype=torch.float64, device=x.device)
    b = bias.double() if bias is not None else torch.zeros(D, dtype=torch.float64, device=x.device)
    y = n * w + b
    # the mean's error (times r), the subtraction's, r's (half of the variance's) and five more operations'
    lost = normed_error(h, n, r)
    rel, least = half_step(t)
    return y, h, rel * y.abs() + least + w.abs() * lost + 2 * U * (y.abs() + b.abs())


def normed_error(h, n, r):
    k = chain(h.shape[1])
    mean_off = (k + 2) * U * h.abs().mean(1, keepdim=True) * r
    # a mean off by e changes the variance by e^2 and, through the differences, by 2 e times their mean (0): r moves by that squared
    return mean_off + n.abs() * (k / 2 + 8 + 0.5 * (mean_off ** 2) / U) * U + U * h.abs() * r


def norm_backward(x, weight, dy, dsum, eps):
    """{"dx", "dweight", "dbias"} and their tolerances (the weights' in the sums alone, without the last rounding)."""
    h, D, T = x.double(), x.shape[1], x.shape[0]
    mean = h.mean(1, keepdim=True)
    c = h - mean
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    n = c * r
    g = dy.double()
    w = weight.double() if weight is not None else torch.ones(D, dtype=torch.float64, device=x.device)
    d = g * w
    dm, dn = d.mean(1, keepdim=True), (d * n).mean(1, keepdim=True)
    dx = r * (d - dm - n * dn)
    out = {"dx": dx if dsum is None else dx + dsum.double(), "dweight": (g * n).sum(0), "dbias": g.sum(0)}
    off, k = normed_error(h, n, r), chain(D)
    rel, least = half_step(x.dtype)
    abs_dn = (d * n).abs().mean(1, keepdim=True)
    dn_off = (k + 4) * U * abs_dn + (d.abs() * off).mean(1, keepdim=True)
    r_rel = (k / 2 + 8) * U + (off * n.abs()).mean(1, keepdim=True)
    tol = {"dx": rel * out["dx"].abs() + least + r * ((k + 4) * U * d.abs().mean(1, keepdim=True) + 4 * U * d.abs() + n.abs() * dn_off + off * dn.abs())
           + r_rel * dx.abs() + 4 * U * r * (d.abs() + dm.abs() + (n * dn).abs()) + 2 * U * out["dx"].abs(),
           "dweight": (g.abs() * off).sum(0) + (chain(T) + 4) * U * (g * n).abs().sum(0), "dbias": (chain(T) + 4) * U * g.abs().sum(0)}
    return out, tol


# ---- AdamW -----------------------------------------------------------------------------------------------------

M32 = 0xFFFFFFFF


def _mix(x):
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x9E3779B9)) & np.uint64(M32)
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0xBB67AE85)) & np.uint64(M32)
    return x ^ (x >> np.uint64(16))


def random_bits(n, seed, number):
    i = np.arange(n, dtype=np.uint64)
    key = _mix(_mix(i >> np.uint64(8)) ^ np.uint64((seed + number * 0x9E3779B9) & M32))
    return _mix((key + (i & np.uint64(255)) * np.uint64(0x6A09E667)) & np.uint64(M32))


def encode(x, signed, bits):
    """Codes and exponents of fp32 values, by whole numbers: the magnitude in steps of the code's last place."""
    n = x.size
    top = 15 if signed else 31
    e = np.zeros(-(-n // 256) * 256, np.int64)
    e[:n] = np.abs(x).view(np.uint32).astype(np.int64)
    e = np.minimum((e.reshape(-1, 256).max(1) + 0x100000) >> 23, 255)  # 1.875 times a power of two and more: the next power
    # |x| 2^(127 - e) 2^(top - 127): its fp32 bits with 20 places below the code's last; what is below the smallest subnormal is rounded to even
    a = np.abs(x).astype(np.float64) * np.exp2(127.0 - np.repeat(e, 256)[:n])
    a = a.astype(np.float32).astype(np.float64) * 2.0 ** (top - 127)
    raw = a.astype(np.float32).view(np.uint32).astype(np.int64)
    r = (bits.astype(np.int64) & 0xFFFF if signed else bits.astype(np.int64) >> 16) << 4
    code = np.minimum((raw + r) >> 20, 127 if signed else 255)
    if signed:
        code = code | np.where(x < 0, 128, 0)
    else:
        code = np.where((x > 0) & (code == 0), 1, code)
    return code.astype(np.uint8), e.astype(np.uint8)


def decode(code, e, signed):
    top = 15 if signed else 31
    size = (code & 127 if signed else code).astype(np.int64)
    exponent, f = size >> 3, (size & 7) / 8.0
    v = np.where(exponent > 0, (1 + f) * np.exp2(exponent - top), f * 2.0 ** (1 - top))
    v = v * np.exp2(np.repeat(e.astype(np.float64) - 127, 256)[:code.size])
    return np.where(code > 127, -v, v) if signed else v


def moments_step(m, v, g, b1, b2):
    """The new moments in fp32, every operation rounded by itself."""
    f = np.float32
    with np.errstate(all="ignore"):
        return m * f(b1) + g * f(1 - b1), v * f(b2) + (g * g) * f(1 - b2)


def param_step(p, m, v, rate, b1, b2, eps, decay, t):
    """The new parameter in 64 bits from fp32 moments, and its tolerance without the last rounding."""
    c1, c2 = -np.expm1(t * np.log(b1)) if b1 else 1.0, -np.expm1(t * np.log(b2)) if b2 else 1.0
    with np.errstate(all="ignore"):
        change = rate * (m.astype(np.float64) / c1) / (np.sqrt(v.astype(np.float64) / c2) + eps)
        new = p.astype(np.float64) * (1 - rate * decay) - change
    return new, 4 * U * np.abs(p) + 16 * U * np.abs(change) + U * np.abs(new) + 2.0 ** -149


# ---- matrices in 4 bits ----------------------------------------------------------------------------------------

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def fp4(x):
    """(values in 64 bits, codes 0 to 15, scale bytes [rows][blocks]) of a matrix, by search of the nearest."""
    v = x.double().cpu().view(x.shape[0], -1, 32)
    top = v.abs().amax(2, keepdim=True)
    lost = ~torch.isfinite(v).all(2, keepdim=True)
    v = torch.where(lost, torch.zeros_like(v), v)
    top = torch.where(lost, torch.ones_like(top), top)
    fraction, power = torch.frexp(top)
    e = (power - 3 + (fraction >= 0.875)).double().clamp(-127, 125)
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    a = v.abs() / torch.exp2(e)
    code = torch.zeros_like(a, dtype=torch.long)
    best = torch.zeros_like(a)
    for k, value in enumerate(GRID):
        near, far = (a - best).abs(), (a - value).abs()
        take = (far < near) | ((far == near) & (k % 2 == 0))
        code, best = torch.where(take, k, code), torch.where(take, value, best)
    value = torch.copysign(best, v) * torch.exp2(e)
    value = torch.where(lost, torch.full_like(value, float("nan")), value)
    code = code + 8 * torch.signbit(v).long()
    byte = torch.where(lost, torch.full_like(e, 255), e + 127).long().squeeze(2)
    return value.view(x.shape), code.view(x.shape), byte


def scale_at(row, block, D):
    return ((row // 128) * ((D + 255) // 256) + block // 8) * 1024 + (block // 4 % 2) * 512 + (row % 32) * 16 + (row // 32 % 4) * 4 + block % 4


ACTS = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}
SLOPE = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "silu": 1.1}  # the steepest that an activation gets


def fp4_linear(x, w, bias, residual, act, gated):
    """y in 64 bits and its tolerance; w: the values of the weights."""
    xv, wv = fp4(x)[0].to(x.device), w.double()
    z, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    # products of 4-bit values are exact; sums of D in fp32, where the matrix instructions may cut instead of round: twice the step
    off = 2 * (x.shape[1] / 32 + 16) * U * size
    lost = 2.0 ** -21  # an activation's own computation, relative to its argument (see the error of its formula: 1.5e-7, two approximations)
    if gated:
        F = z.shape[1] // 2
        a = ACTS[act](z[:, :F])
        y = a * z[:, F:]
        tol = (SLOPE[act] * off[:, :F] + lost * z[:, :F].abs()) * z[:, F:].abs() + a.abs() * off[:, F:] + off[:, :F] * off[:, F:]
    else:
        y, tol = ACTS[act](z), SLOPE[act] * off + lost * z.abs()
    if residual is not None:
        y = y + residual.double()
    rel, least = half_step(x.dtype)
    return y, tol + (rel + 4 * U) * y.abs() + least + U * (residual.double().abs() if residual is not None else 0)
