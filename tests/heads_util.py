"""Plain 64-bit forms of the operators around the layer, with bounds on what rounding may do to the kernels' results (not a test module).

Half a rounding step relative to the value is finfo(type).eps / 2.  Every bound below is a sum of such steps over what the kernel rounds."""
import math

import torch

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F32 = 2.0 ** -24


def check(name, got, want, bound):
    got, want, bound = got.detach().cpu().double(), want.detach().cpu().double(), bound.detach().cpu().double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (name, "NaN", int(torch.isnan(got).sum()), int(torch.isnan(want).sum()))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), (name, "infinities")
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (name, "over its bound by", float(over.max()), "error", float((got - want)[fine].abs().max()),
                                                         "bound", float(bound[fine].max()))


# ---- rotary positions and norms

def frequencies(axis_dims, base, scaling, factor, context, fast=32.0, slow=1.0):
    """Radians per position of every pair, the axis of every pair, and the amplitude; scaling 0 plain, 1 linear, 2 ntk, 3 by parts."""
    theta, axis = [], []
    for a, n in enumerate(axis_dims):
        b = base * factor ** (n / (n - 2)) if scaling == 2 and n > 2 else base
        for j in range(n // 2):
            w = b ** (-2.0 * j / n)
            if scaling == 1:
                w /= factor
            if scaling == 3:
                keep = min(1.0, max(0.0, (context * w / (2 * math.pi) - slow) / (fast - slow)))
                w = w * (keep + (1 - keep) / factor)
            theta.append(w)
            axis.append(a)
    return torch.tensor(theta, dtype=torch.float64), torch.tensor(axis), (0.1 * math.log(factor) + 1.0 if scaling == 3 else 1.0)


def rotate(x, positions, theta, axis, amplitude, layout, inverse=False):
    """x [batch, tokens, heads, d] in 64 bits, positions [batch, tokens, axes]."""
    phi = (positions.double()[..., axis] * theta)[:, :, None]
    c, s = amplitude * phi.cos(), amplitude * phi.sin() * (-1 if inverse else 1)
    h = len(theta)
    a, b = (slice(0, h), slice(h, 2 * h)) if layout == 0 else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def rotate_size(x, n, amplitude, layout):
    """A |a| + A |b| for the channels of a pair, |x| elsewhere: what roundings of the rotation are relative to."""
    x = x.abs()
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == 0 else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y = x.clone()
    y[..., a] = y[..., b] = amplitude * (x[..., a] + x[..., b])
    return y


# ---- attention over sequences

def attend(q, k, v, causal, scale, io, dout=None):
    """One sequence and head in 64 bits, q [nq, d], k, v [nk, d].  Returns {name: (value, bound)}: out, lse and, with dout, dq, dk, dv."""
    step = STEP[io]
    nq, nk, d = q.shape[0], k.shape[0], q.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    seen = torch.ones(nq, nk, dtype=torch.bool)
    if causal:
        seen = torch.arange(nk)[None] <= torch.arange(nq)[:, None] + nk - nq
    some = seen.any(1)
    if nk == 0:
        some = torch.zeros(nq, dtype=torch.bool)
    s = (q @ k.T * scale).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
    p = torch.where(seen, torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
    zero = lambda x: torch.where(seen[:, :, None], x, 0.0)   # noqa: E731
    out = p @ v
    # score: d products and sums in fp32 and a few steps more; a probability moves by as much relative to itself, in the sum too
    se = F32 * (d + 8) * torch.where(seen, q.abs() @ k.abs().T * scale + s.abs().masked_fill(~seen, 0.0), 0.0).amax(1, keepdim=True) if nk else torch.zeros(nq, 1).double()
    pe = 2 * se + (nk + 16) * F32                       # relative error of a probability kept in fp32
    rounded = pe + (step if io is torch.bfloat16 else 0.0)   # ... rounded to bf16 as an operand of a product
    ob = (p @ v.abs()) * (rounded + nk * F32) + step * out.abs() * (1 + 2.0 ** -6) + 1e-30
    res = {"out": (out, ob), "lse": (lse, (pe[:, 0] + 4 * F32 * lse.abs()).masked_fill(~some, 0.0))}
    if dout is None:
        return res
    do = dout.double()
    delta = (do * out).sum(1, keepdim=True)
    delta_e = (do.abs() * ob).sum(1, keepdim=True) + d * F32 * (do * out).abs().sum(1, keepdim=True)   # from the stored out
    dp = do @ v.T
    dp_e = F32 * (d + 4) * (do.abs() @ v.abs().T)
    ds = p * (dp - delta)
    ds_e = p * (dp_e + delta_e) + ds.abs() * rounded
    sums = (nq + nk + 8) * F32
    dq, dk, dv = scale * ds @ k, scale * ds.T @ q, p.T @ do
    dq_b = scale * (ds_e + ds.abs() * sums) @ k.abs() + step * dq.abs() * (1 + 2.0 ** -6) + 1e-30
    dk_b = scale * (ds_e + ds.abs() * sums).T @ q.abs()
    dv_b = (p * (rounded + sums)).T @ do.abs()
    res.update(dq=(dq, dq_b), dk=(dk, dk_b), dv=(dv, dv_b))   # (of a group's heads the last two are added up; the step of their store comes then)
    return res


def spans(offsets, lengths, rows, n):
    """(batch entry, first row, rows) of every sequence."""
    out = []
    for i in range(n):
        b, first, count = (i, 0, rows) if offsets is None else (0, offsets[i], offsets[i + 1] - offsets[i])
        if lengths is not None:
            count = min(count, lengths[i])
        out.append((b, first, count))
    return out


def attend_all(q, k, v, causal, scale, q_spans, k_spans, dout=None):
    """All sequences and heads; tensors [batch, rows, heads, d] on the host in the type of the call.  Returns {name: (value, bound, inside)}; rows outside the
    sequences have inside False."""
    io, group = q.dtype, q.shape[2] // k.shape[2]
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64)   # noqa: E731
    names = {"out": q, "lse": q[..., 0]} | ({"dq": q, "dk": k, "dv": k} if dout is not None else {})
    res = {n: [z(t), z(t), torch.zeros(t.shape, dtype=torch.bool)] for n, t in names.items()}
    for (qb, q0, qn), (kb, k0, kn) in zip(q_spans, k_spans):
        for h in range(q.shape[2]):
            qi, ki = (qb, slice(q0, q0 + qn), h), (kb, slice(k0, k0 + kn), h // group)
            r = attend(q[qi], k[ki], v[ki], causal, scale, io, None if dout is None else dout[qi])
            for n, (value, bound) in r.items():
                at = ki if n in ("dk", "dv") else qi
                res[n][0][at] += value
                res[n][1][at] += bound
                res[n][2][at] = True
    if dout is not None:
        for n in ("dk", "dv"):
            res[n][1] += (STEP[io] * (1 + 2.0 ** -6) + group * F32) * res[n][0].abs() + 1e-30
    return res
