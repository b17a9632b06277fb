"""Plain 64-bit forms of the operators on token rows, with bounds on what rounding may do to the kernels' results (not a test module).

Half a rounding step relative to the value is finfo(type).eps / 2.  Every bound is a sum of such steps over what the kernel rounds."""
import bisect
import math

import torch

from tests import heads_util as U

STEP, F32, check = U.STEP, U.F32, U.check
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MARK = 7.0
CHAIN = 64     # additions behind each other in a sum over a row: at most 32 channels of a lane, 6 steps over lanes, 8 waves, and some


# ---- layer norm

def norm(x, w, b, eps, io, dout=None):
    """x [rows, channels] of one set of weights, all in 64 bits.  Returns {name: (value, bound)}: out and, with dout, dx, dw, db."""
    L, n = CHAIN, x.shape[1]
    mean, var = x.mean(1, keepdim=True), x.var(1, correction=0, keepdim=True)
    r = 1.0 / torch.sqrt(var + eps)
    h = (x - mean) * r
    off = L * F32 * x.abs().mean(1, keepdim=True)                # the mean in fp32, which the kernel subtracts first
    d = (x - mean).abs() + off                                   # sizes of the centred values that it works on
    md = d.mean(1, keepdim=True)
    re = (L + 4) * F32 * (var + off * off) / (var + eps) / 2 + 4 * F32      # relative error of r
    he = r * (2 * F32 * d + (L + 3) * F32 * md) + h.abs() * re
    out = h * w + b
    step = STEP[io] * (1 + 2.0 ** -6)
    res = {"out": (out, he * w.abs() + 2 * F32 * ((h * w).abs() + b.abs()) + step * out.abs() + 1e-30)}
    if dout is None:
        return res
    g = dout * w
    mg, mgh = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    mg_e = (L + 2) * F32 * g.abs().mean(1, keepdim=True)
    mgh_e = r * ((L + 4) * F32 * (g.abs() * d).mean(1, keepdim=True) + (L + 3) * F32 * md * g.abs().mean(1, keepdim=True)) + re * mgh.abs()
    dx = r * (g - mg - h * mgh)
    dx_e = re * dx.abs() + r * (he * mgh.abs() + h.abs() * mgh_e + mg_e + 5 * F32 * (g.abs() + mg.abs() + (h * mgh).abs())) + step * dx.abs() + 1e-30
    rows = x.shape[0] + CHAIN
    res["dx"] = (dx, dx_e)
    res["dw"] = ((dout * h).sum(0), (dout.abs() * he).sum(0) + rows * F32 * (dout * h).abs().sum(0) + 1e-30)
    res["db"] = (dout.sum(0), rows * F32 * dout.abs().sum(0) + 1e-30)
    return res


# ---- 8-bit codes of rows

def code_rows(x):
    """Codes and fp32 scales of x [rows, channels] (bf16 or fp32, on the host): comparisons without rounding in 64 bits."""
    v = x.double()
    odd = ~torch.isfinite(v).all(1)
    v = torch.where(odd[:, None], 0.0, v)
    a = v.abs().amax(1, keepdim=True)
    k = torch.floor(127 * v.abs() / torch.where(a > 0, a, 1.0)).clamp(0, 127)
    for _ in range(2):     # (the quotient may have been rounded across a whole number)
        k = torch.where(127 * v.abs() < k * a, k - 1, k)
        k = torch.where(127 * v.abs() >= (k + 1) * a, k + 1, k) if bool((a > 0).any()) else k
    k = torch.where(a > 0, k, 0.0)
    low, high = 254 * v.abs(), (2 * k + 1) * a      # 24 + 8 bits on either side
    up = (low > high) | ((low == high) & (k % 2 == 1))
    codes = torch.where(a > 0, (k + up.double()), 0.0) * torch.sign(v)
    scales = a[:, 0].float() / torch.tensor(127.0)
    return codes.to(torch.int8), torch.where(odd, math.nan, scales)


# ---- caches held in 8 bits

def _value(code):
    s, e, m = code >> 7, code >> 3 & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    v = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
    return -v if s else v


VALUES = [_value(c) for c in range(256)]
TABLE = torch.tensor(VALUES, dtype=torch.float64)


def e4m3(x):
    """The code nearest to x, ties to the even code; NaN for NaN and infinities."""
    if not math.isfinite(x):
        return 0x7f
    a = abs(x)
    i = bisect.bisect_left(VALUES[:127], a)      # 0x7e is 448
    if i == 127:
        i = 126
    elif i > 0 and VALUES[i] != a:
        lo, hi = a - VALUES[i - 1], VALUES[i] - a
        i = i - 1 if lo < hi or (lo == hi and (i - 1) % 2 == 0) else i
    return i | (0x80 if math.copysign(1.0, x) < 0 else 0)


def least_byte(top):
    m, e = math.frexp(top)                       # top = m 2^e, m in [0.5, 1): top <= 0.875 * 2^9 * 2^(byte - 127)
    return max(10, e - 9 + 127 + (1 if m > 0.875 else 0)) if top > 0 else 10


def append(codes, scales, block, new, length):
    """Appends new [rows, d] (host) to one sequence and head: codes [rows, d] and scales [blocks] as lists of numbers, changed in place."""
    first = length - len(new)
    for lo in range(max(first, 0) // block * block, length, block):
        at = range(max(lo, first, 0), min(lo + block, length))
        if not at:
            continue
        rows = [[float(x) for x in new[i - first]] for i in at]
        e = least_byte(max([abs(x) for r in rows for x in r if math.isfinite(x)], default=0.0))
        old = range(lo, at[0])
        if old:
            was = scales[lo // block]
            e = max(e, was)
            if e != was:
                for i in old:
                    codes[i] = [e4m3(math.ldexp(VALUES[c], was - e)) if not math.isnan(VALUES[c]) else c for c in codes[i]]
        for i, r in zip(at, rows):
            codes[i] = [e4m3(math.ldexp(x, 127 - e)) if math.isfinite(x) else 0x7f for x in r]
        scales[lo // block] = e


def cache_values(codes, scales, block):
    """Values in 64 bits of codes [sequences, rows, heads, d] uint8 with scales [sequences, blocks, heads] uint8."""
    v = TABLE[codes.long()]
    s = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127)).repeat_interleave(block, 1)[:, :v.shape[1]]
    return v * s[..., None]
