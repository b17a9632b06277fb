"""What the operators around the frequency-domain attention are measured on: rotary positions, norms of queries and keys with the rotation,
and dense attention over packed or padded sequences, each at the sizes a user of the framework meets.

A case is a dict of plain values.  "op" names the operator: "rotary", "qk_norm" or "attention"; "train" adds the backward pass.  With `own` false,
run() computes the plain form (elementary torch operations in 32 bits); with `own` true it calls the framework's kernels.
"""
import math

import torch


own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "parts": 3}


def _binding():
    from paper_2604_22808_amd import binding
    return binding


# ---------------------------------------------------------------------------------------------------------------- cases

def _rot(layout, axes, scaling="plain", factor=1.0, context=0, grid="", first=0):
    """axes: channels that rotate, per position axis; grid: positions are the coordinates of this grid; first: position of the first token."""
    return dict(layout=layout, axes=axes, base=10000.0, scaling=scaling, factor=factor, context=context, grid=grid, first=first)


def _rotary(name, dtype, batch, tokens, heads, d, rot, inverse=False, head_major=False):
    return dict(name=name, op="rotary", dtype=dtype, batch=batch, tokens=tokens, heads=heads, head_dim=d, inverse=inverse,
                head_major=head_major, **rot)


def _qk(name, dtype, batch, tokens, heads, k_heads, d, rot, train=False):
    return dict(name=name, op="qk_norm", dtype=dtype, batch=batch, tokens=tokens, heads=heads, k_heads=k_heads, head_dim=d, train=train, **rot)


def _attention(name, dtype, form, heads, kv_heads, d, q_lengths, k_lengths, causal, train=False, capacity=0):
    """form: "packed" (rows of all sequences behind each other), "cache" (keys in a [sequences, capacity, heads, d] cache that is filled to the
    lengths, queries [sequences, rows, heads, d]) or "heads" ([sequences, heads, rows, d], all sequences of one length)."""
    return dict(name=name, op="attention", dtype=dtype, form=form, heads=heads, kv_heads=kv_heads, head_dim=d, q_lengths=q_lengths,
                k_lengths=k_lengths, causal=causal, train=train, capacity=capacity)


def listed():
    return [
        # one new token of each of 16 requests, far beyond the trained context: launch latency is all there is
        _rotary("rotary_one_token", "bf16", 16, 1, 16, 64, _rot("half", "64", "parts", 8.0, 16384, first=120000)),
        # gradient of a partial rotation, fp32, an odd number of tokens: plain streaming
        _rotary("rotary_partial_inverse", "f32", 1, 131071, 8, 128, _rot("half", "64", "ntk", 4.0, 32768), inverse=True, head_major=True),
        # one new token of 64 requests: norms and rotation of grouped heads in front of a decode step
        _qk("qk_norm_one_token", "bf16", 64, 1, 32, 8, 128, _rot("half", "128", first=4000)),
        # the 64K-token workload's queries and keys: out of a fused projection into the layout that freqattn_forward reads, T, H, W rotation
        _qk("qk_norm_grid_64k", "bf16", 1, 65536, 24, 24, 64, _rot("interleaved", "16,24,24", grid="16,64,64")),
        # a training step of the same at head_dim 128 on 128K tokens
        _qk("qk_norm_train_128k", "bf16", 1, 131072, 16, 16, 128, _rot("half", "44,42,42", grid="32,64,64"), train=True),
        # one token of one request against a short cache: latency
        _attention("decode_short", "bf16", "cache", 16, 2, 64, "1", "777", True, capacity=1000),
        # one token of 32 requests against long caches of different fill: the bytes of the caches
        _attention("decode_batch", "bf16", "cache", 32, 8, 128, ",".join(["1"] * 32),
                   ",".join(str(200 + 509 * i) for i in range(31)) + ",16384", True, capacity=16384),
        # prompts of very different lengths behind each other
        _attention("prefill_packed", "bf16", "packed", 8, 2, 128, "4500,1,2900,640,17,2222,4096,333,64,1290", "", True),
        # one long causal sequence, all heads on one key head
        _attention("prefill_32k", "bf16", "packed", 4, 1, 128, "32768", "", True),
        # training on packed sequences
        _attention("train_packed", "bf16", "packed", 16, 4, 128, "2500,129,1800,2048,63,1025,2400,500", "", True, train=True),
        # training on the 16K-token grid, every token sees every token, in the framework's head-major layout
        _attention("train_grid_16k", "bf16", "heads", 8, 8, 64, "16384", "", False, train=True),
        # fp32 training, odd head size and lengths
        _attention("train_f32_odd", "f32", "packed", 6, 3, 48, "701,100,333", "", True, train=True),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_rot(rng, d, tokens, full):
    layout = rng.choice(["half", "interleaved"])
    if rng.random() < 0.35:   # a grid of about that many tokens
        t = rng.randint(1, max(1, min(32, tokens)))
        h = max(1, round(math.sqrt(tokens / t)))
        w = max(1, tokens // (t * h))
        a = 2 * max(1, d // 6)
        return t * h * w, _rot(layout, "%d,%d,%d" % (d - 2 * a, a, a), grid="%d,%d,%d" % (t, h, w))
    part = d if full or rng.random() < 0.5 else 8 * rng.randint(1, d // 8)
    scaling = rng.choice(["plain", "plain", "linear", "ntk", "parts"])
    factor, context = (1.0, 0) if scaling == "plain" else (rng.choice([2.0, 4.0, 7.5, 16.0]), rng.choice([4096, 16384, 32768]))
    return tokens, _rot(layout, str(part), scaling, factor, context, first=rng.choice([0, 0, 17, 5000, 250000]))


def draw(rng):
    op = rng.choice(["rotary", "qk_norm", "attention", "attention"])
    if op != "attention":
        dtype, d = rng.choice(["bf16", "bf16", "f32"]), rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 256])
        heads, batch = round(_log(rng, 1, 40)), rng.choice([1, 1, 2, 3, 8, 64])
        group = rng.choice([1, 1, 2, 4])
        k_heads = max(1, heads // group)
        tokens = 1 if rng.random() < 0.2 else max(1, round(_log(rng, 3e4, 2e8) / (d * batch * (heads + k_heads))))
        tokens, rot = _draw_rot(rng, d, tokens, False)
        if op == "rotary":
            c = _rotary("", dtype, batch, tokens, heads, d, rot, rng.random() < 0.5, rng.random() < 0.5)
        else:
            c = _qk("", dtype, batch, tokens, heads, k_heads, d, rot, rng.random() < 0.6)
    else:
        dtype, d = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice([32, 64, 64, 72, 96, 128, 128, 128])
        kv_heads, group = round(_log(rng, 1, 9)), rng.choice([1, 1, 2, 3, 4, 8])
        form, n = rng.choice(["packed", "packed", "cache", "heads"]), round(_log(rng, 1, 24))
        heads = kv_heads * group
        if form == "cache":
            rows = rng.choice([1, 1, 1, 2, 5, 16])
            most = max(64, min(20000, round(2e8 / (n * heads * d))))
            k = [rng.randint(rows, most) for _ in range(n)]
            c = _attention("", dtype, form, heads, kv_heads, d, ",".join([str(rows)] * n), ",".join(map(str, k)), True, capacity=most + rng.choice([0, 3, 64]))
        else:
            pairs = (2e7 if dtype == "f32" else 2e9) * rng.uniform(0.02, 0.5)
            most = max(2, min(8000, round(math.sqrt(pairs / (n * heads)))))
            train = rng.random() < 0.6
            if form == "heads":
                q = ",".join([str(most)] * n)
            else:
                q = ",".join(str(rng.choice([most, rng.randint(1, most), round(_log(rng, 1, most))])) for _ in range(n))
            c = _attention("", dtype, form, heads, kv_heads, d, q, "", rng.random() < 0.7, train)
    del c["name"]
    return c


def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _lengths(c):
    q = _ints(c["q_lengths"])
    return q, (_ints(c["k_lengths"]) or q)


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "attention":
        q, k = _lengths(c)
        d = c["head_dim"]
        pairs = sum((min(a, b) * b - min(a, b) * (min(a, b) - 1) // 2 if c["causal"] else a * b) for a, b in zip(q, k)) * c["heads"]
        qo, kv = sum(q) * c["heads"] * d * size, sum(k) * c["kv_heads"] * d * size
        once = 2 * qo + 2 * kv
        # training: forward, and then q, k, v, out, dout in, dq, dk, dv out
        return {"bytes": once + (4 * qo + 4 * kv if c["train"] else 0), "flops": 4 * d * pairs * (3.5 if c["train"] else 1)}
    n = c["batch"] * c["tokens"] * c["head_dim"]
    if c["op"] == "rotary":
        return {"bytes": 2 * n * c["heads"] * size, "flops": 3 * n * c["heads"]}
    n *= c["heads"] + c["k_heads"]
    return {"bytes": n * size * (5 if c["train"] else 2), "flops": n * (17 if c["train"] else 7)}


# ---------------------------------------------------------------------------------------------------------------- inputs

def _positions(c, device):
    """int32 [batch, tokens, axes], or None where the tokens' own order or grid gives them."""
    if c["grid"] or not c["first"]:
        return None
    p = c["first"] + torch.arange(c["tokens"], device=device, dtype=torch.int32)
    return (p[None, :, None] + 131 * torch.arange(c["batch"], device=device, dtype=torch.int32)[:, None, None]).contiguous()


def prepare(case, seed):
    c, dev, t = case, "cuda", TYPES[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, device=dev, generator=g).to(t)

    d = c["head_dim"]
    s = {"c": c, "t": t}
    if c["op"] == "attention":
        q, k = _lengths(c)
        s["q_len"], s["k_len"] = torch.tensor(q, device=dev, dtype=torch.int32), torch.tensor(k, device=dev, dtype=torch.int32)
        hq, hk = c["heads"], c["kv_heads"]
        if c["form"] == "packed":
            s["offsets"] = torch.tensor([0] + q, device=dev, dtype=torch.int32).cumsum(0).to(torch.int32)
            s["q"], s["k"], s["v"] = randn(sum(q), hq, d), randn(sum(q), hk, d), randn(sum(q), hk, d)
        elif c["form"] == "cache":   # rows behind a request's length hold what an earlier request left
            s["q"], s["k"], s["v"] = randn(len(q), q[0], hq, d), randn(len(q), c["capacity"], hk, d), randn(len(q), c["capacity"], hk, d)
        else:
            s["q"], s["k"], s["v"] = (randn(len(q), h, q[0], d).transpose(1, 2) for h in (hq, hk, hk))
        s["out"] = torch.zeros_like(s["q"])
        if c["train"]:
            s["dout"] = torch.empty_like(s["q"]).copy_(randn(*s["q"].shape))
            s["lse"] = torch.zeros(hq, s["q"].shape[0] if c["form"] == "packed" else s["q"].shape[0] * s["q"].shape[1], device=dev)
            s["dq"], s["dk"], s["dv"] = (torch.zeros_like(s[n]) for n in "qkv")
        return s
    b, n, h = c["batch"], c["tokens"], c["heads"]
    s["positions"] = _positions(c, dev)
    if own:
        s["rotary"] = _binding().Rotary(d, _ints(c["axes"]), layout=LAYOUTS[c["layout"]], base=c["base"], scaling=SCALINGS[c["scaling"]],
                                        factor=c["factor"], context=c["context"], grid=tuple(_ints(c["grid"])) or None)
    if c["op"] == "rotary":
        s["x"] = randn(b, h, n, d).transpose(1, 2) if c["head_major"] else randn(b, n, h, d)
        s["out"] = torch.empty_like(s["x"])
        return s
    hk = c["k_heads"]
    qkv = randn(b, n, h + 2 * hk, d)   # a fused projection, with channels of different sizes
    qkv *= torch.exp(torch.randn(d, device=dev, generator=g)).to(t)
    s["q"], s["k"] = qkv[:, :, :h], qkv[:, :, h:h + hk]
    s["wq"], s["wk"] = (1 + 0.3 * torch.randn(d, device=dev, generator=g)).to(t), (1 + 0.3 * torch.randn(d, device=dev, generator=g)).to(t)
    s["q_out"], s["k_out"] = (torch.empty(b, x, n, d, device=dev, dtype=t).transpose(1, 2) for x in (h, hk))
    if c["train"]:
        s["dq_out"], s["dk_out"] = randn(b, h, n, d).transpose(1, 2), randn(b, hk, n, d).transpose(1, 2)
        dqkv = torch.zeros_like(qkv)
        s["dq"], s["dk"] = dqkv[:, :, :h], dqkv[:, :, h:h + hk]
        s["dwq"], s["dwk"] = torch.empty(d, device=dev), torch.empty(d, device=dev)
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms

def _angles(c, positions, device):
    """cos and sin [batch or 1, tokens, 1, pairs] in 32 bits from angles in 64, and the amplitude."""
    dims = torch.tensor(_ints(c["axes"]), device=device, dtype=torch.float64)
    half = (dims / 2).to(torch.int64)
    axis = torch.repeat_interleave(torch.arange(len(dims), device=device), half)
    j = torch.arange(axis.numel(), device=device) - (torch.cumsum(half, 0) - half)[axis]
    n, f = dims[axis], c["factor"]
    base = torch.full_like(n, c["base"])
    if c["scaling"] == "ntk":
        base = torch.where(n > 2, c["base"] * f ** (n / (n - 2).clamp(min=1)), base)
    theta = base ** (-2.0 * j / n)
    amplitude = 1.0
    if c["scaling"] == "linear":
        theta = theta / f
    if c["scaling"] == "parts":
        keep = ((c["context"] * theta / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        theta = theta * (keep + (1.0 - keep) / f)
        amplitude = 0.1 * math.log(f) + 1.0
    if positions is None:
        i = torch.arange(c["tokens"], device=device)
        g = _ints(c["grid"])
        p = (torch.stack([i // (g[1] * g[2]), i // g[2] % g[1], i % g[2]], -1) if g else i[:, None])[None]
    else:
        p = positions
    phi = p.to(torch.float64)[..., axis] * theta
    return (amplitude * phi.cos()).float()[:, :, None], (amplitude * phi.sin()).float()[:, :, None]


def _turn(c, x, cos, sin):
    """Rotates float x [batch, tokens, heads, d]; sin negated turns back."""
    r = 2 * cos.shape[-1]
    rot, rest = x[..., :r], x[..., r:]
    if c["layout"] == "half":
        a, b = rot[..., :r // 2], rot[..., r // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)
    a, b = rot[..., 0::2], rot[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)


def _plain_rotary(s):
    c, x = s["c"], s["x"]
    cos, sin = _angles(c, s["positions"], x.device)
    s["out"].copy_(_turn(c, x.float(), cos, -sin if c["inverse"] else sin))
    return s["out"]


EPS = 1e-6


def _plain_qk(s):
    c = s["c"]
    cos, sin = _angles(c, s["positions"], s["q"].device)

    def forward(x, w, out):
        x = x.float()
        out.copy_(_turn(c, x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float(), cos, sin))
        return out

    def backward(x, w, dy, dx, dw):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        g = _turn(c, dy.float(), cos, -sin)
        dw.copy_((g * x * r).double().sum((0, 1, 2)))
        g = g * w.float()
        dx.copy_(r * (g - x * r * r * (g * x).mean(-1, keepdim=True)))
        return dx, dw

    out = [forward(s["q"], s["wq"], s["q_out"]), forward(s["k"], s["wk"], s["k_out"])]
    if c["train"]:
        dq, dwq = backward(s["q"], s["wq"], s["dq_out"], s["dq"], s["dwq"])
        dk, dwk = backward(s["k"], s["wk"], s["dk_out"], s["dk"], s["dwk"])
        out += [dq, dk, dwq, dwk]
    return out


def _plain_attention(s):
    c = s["c"]
    dev, group = s["q"].device, c["heads"] // c["kv_heads"]
    lq, lk = max(_lengths(c)[0]), max(_lengths(c)[1])
    i, j = torch.arange(lq, device=dev), torch.arange(lk, device=dev)
    q_in, k_in = i < s["q_len"][:, None], j < s["k_len"][:, None]                     # rows of a sequence
    seen = q_in[:, None, :, None] & k_in[:, None, None, :]
    if c["causal"]:
        seen = seen & (j <= i[:, None] + (s["k_len"] - s["q_len"])[:, None, None, None])
    if c["form"] == "packed":
        qi = (s["offsets"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
        ki = (s["offsets"][:-1, None] + j).clamp(max=s["k"].shape[0] - 1)

    def rows(x, inside, repeat, queries):
        """[sequences, heads, rows, d] in 32 bits, zero behind a sequence's end."""
        x = x[qi if queries else ki] if c["form"] == "packed" else x[:, :inside.shape[1]]
        x = torch.where(inside[:, :, None, None], x.float(), 0.0).transpose(1, 2)
        return x.repeat_interleave(repeat, 1) if repeat > 1 else x.contiguous()

    def store(x, inside, target):
        """x [sequences, heads, rows, d] into the rows of the sequences; other rows stay."""
        x = x.transpose(1, 2)
        if c["form"] == "packed":
            target.copy_(x[inside].to(target.dtype))
        else:
            part = target[:, :inside.shape[1]]
            part.copy_(torch.where(inside[:, :, None, None], x.to(target.dtype), part))
        return target

    q, k, v = rows(s["q"], q_in, 1, True), rows(s["k"], k_in, group, False), rows(s["v"], k_in, group, False)
    scale = 1.0 / math.sqrt(c["head_dim"])
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True).clamp(min=-3e38)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total.clamp(min=1e-38))
    o = torch.matmul(p, v)
    store(o, q_in, s["out"])
    if not c["train"]:
        return s["out"]
    lse = (top + total.log())[..., 0]                                                   # [sequences, heads, rows]
    if c["form"] == "packed":
        s["lse"].copy_(lse.transpose(0, 1)[:, q_in])
    else:
        s["lse"].copy_(lse.transpose(0, 1).flatten(1))
    do = rows(s["dout"], q_in, 1, True)
    folded = (len(s["q_len"]), c["kv_heads"], group, lk, c["head_dim"])
    store(torch.matmul(p.transpose(-1, -2).contiguous(), do).view(folded).sum(2), k_in, s["dv"])
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = dp.sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    store(torch.matmul(ds, k), q_in, s["dq"])
    store(torch.matmul(ds.transpose(-1, -2).contiguous(), q).view(folded).sum(2), k_in, s["dk"])
    return [s[n] for n in ("out", "lse", "dq", "dk", "dv")]


# -------------------------------------------------------------------------------------------------------- one pass of each

def _own_attention(s):
    B, c = _binding(), s["c"]
    how = {"causal": c["causal"]}
    if c["form"] == "packed":
        how.update(q_offsets=s["offsets"], k_offsets=s["offsets"])
    elif c["form"] == "cache":
        how.update(k_lengths=s["k_len"])
    B.sequence_attention(s["q"], s["k"], s["v"], s["out"], lse=s.get("lse"), **how)
    if not c["train"]:
        return s["out"]
    B.sequence_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dq"], s["dk"], s["dv"], **how)
    return [s[n] for n in ("out", "lse", "dq", "dk", "dv")]


def run(state):
    s, c = state, state["c"]
    if c["op"] == "attention":
        return _own_attention(s) if own else _plain_attention(s)
    if c["op"] == "rotary":
        return _binding().rotary_apply(s["rotary"], s["x"], s["out"], positions=s["positions"], inverse=c["inverse"]) if own else _plain_rotary(s)
    if not own:
        return _plain_qk(s)
    B = _binding()
    at = dict(eps=EPS, rotary=s["rotary"], positions=s["positions"])
    B.qk_norm(s["q"], s["k"], s["wq"], s["wk"], s["q_out"], s["k_out"], **at)
    if not c["train"]:
        return [s["q_out"], s["k_out"]]
    B.qk_norm_backward(s["q"], s["k"], s["wq"], s["wk"], s["dq_out"], s["dk_out"], s["dq"], s["dk"], s["dwq"], s["dwk"], **at)
    return [s[n] for n in ("q_out", "k_out", "dq", "dk", "dwq", "dwk")]


# --------------------------------------------------------------------------------------- the definition in 64 bits, by itself

def _exact_rotation(c, positions, device):
    """One complex number per batch entry, token and pair of channels."""
    f = c["factor"]
    tokens = torch.arange(c["tokens"], device=device, dtype=torch.float64)
    g = _ints(c["grid"])
    out = []
    for a, n in enumerate(_ints(c["axes"])):
        base = c["base"] * (f ** (n / (n - 2)) if c["scaling"] == "ntk" and n > 2 else 1.0)
        if positions is not None:
            p = positions[:, :, a].double()
        elif g:
            inner = math.prod(g[a + 1:])
            p = torch.remainder(torch.floor(tokens / inner), g[a])[None]
        else:
            p = tokens[None]
        for j in range(n // 2):
            w = base ** (-2 * j / n)
            if c["scaling"] == "linear":
                w /= f
            elif c["scaling"] == "parts":
                turns = c["context"] * w / (2 * math.pi)
                keep = min(1.0, max(0.0, (turns - 1) / (32 - 1)))
                w = (1 - keep) * w / f + keep * w
            out.append(p * w)
    amplitude = 1 + math.log(f) / 10 if c["scaling"] == "parts" else 1.0
    phi = torch.stack(out, -1)[:, :, None]
    return torch.polar(torch.full_like(phi, amplitude), phi)


def _exact_turn(c, x, z):
    r = 2 * z.shape[-1]
    y = x.clone()
    if c["layout"] == "half":
        first, second = slice(0, r // 2), slice(r // 2, r)
    else:
        first, second = slice(0, r, 2), slice(1, r, 2)
    w = torch.complex(x[..., first], x[..., second]) * z
    y[..., first], y[..., second] = w.real, w.imag
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    dev = s["out"].device if "out" in s else s["q_out"].device
    if c["op"] == "rotary":
        z = _exact_rotation(c, s["positions"], dev)
        return _exact_turn(c, s["x"].double(), z.conj() if c["inverse"] else z)
    if c["op"] == "qk_norm":
        z = _exact_rotation(c, s["positions"], dev)
        out, grads, weights = [], [], []
        for x, w, n in ((s["q"], s["wq"], "q"), (s["k"], s["wk"], "k")):
            x, w = x.double(), w.double()
            norm = (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
            unit = x / norm
            out.append(_exact_turn(c, unit * w, z))
            if c["train"]:
                g = _exact_turn(c, s["d%s_out" % n].double(), z.conj())
                weights.append((g * unit).sum((0, 1, 2)))
                g = g * w
                grads.append((g - unit * (unit * g).sum(-1, keepdim=True) / x.shape[-1]) / norm)
            del x, unit
        return out + grads + weights
    ql, kl = _lengths(c)
    group, d = c["heads"] // c["kv_heads"], c["head_dim"]
    res = [torch.zeros(s[n].shape, device=dev, dtype=torch.float64) for n in (("out", "lse", "dq", "dk", "dv") if c["train"] else ("out",))]
    start = 0
    for b, (nq, nk) in enumerate(zip(ql, kl)):
        at = (slice(start, start + nq),) if c["form"] == "packed" else (b, slice(0, nq))
        kat = (slice(start, start + nk),) if c["form"] == "packed" else (b, slice(0, nk))
        far = torch.arange(nk, device=dev)[None, :] > torch.arange(nq, device=dev)[:, None] + (nk - nq)
        for h in range(c["heads"]):
            q, k, v = s["q"][at][:, h].double(), s["k"][kat][:, h // group].double(), s["v"][kat][:, h // group].double()
            if c["train"]:
                q, k, v = q.requires_grad_(), k.requires_grad_(), v.requires_grad_()
            score = q @ k.T / math.sqrt(d)
            if c["causal"]:
                score = score.masked_fill(far, -math.inf)
            lse = torch.logsumexp(score, 1)
            o = torch.exp(score - lse[:, None]) @ v
            res[0][at][:, h] = o.detach()
            if c["train"]:
                row = start if c["form"] == "packed" else b * nq
                res[1][h, row:row + nq] = lse.detach()
                gq, gk, gv = torch.autograd.grad(o, (q, k, v), s["dout"][at][:, h].double())
                res[2][at][:, h] = gq
                res[3][kat][:, h // group] += gk
                res[4][kat][:, h // group] += gv
        start += nq
    return res if c["train"] else res[0]
