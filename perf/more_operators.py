"""What the token-side operators around the attention are measured on: layer norm with its gradients, products in 8-bit integers with a scale for every
token and channel, and caches held in 8 bits with a scale for every block of tokens and head - filling them, reading them back, attention over them.

A case is a dict of plain values.  "op" names the operator: "norm" ("train" adds the backward pass), "product" (rows coded and multiplied), "fill" (rows
appended to a cache, and the cache's values read back) or "attend" (attention over a filled cache).  With `own` false, run() computes the plain form
(elementary torch operations in 32 bits); with `own` true it calls the framework's kernels.
"""
import math

import torch


own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
TOP = 448.0        # the largest e4m3 value
LEAST = 10         # the smallest exponent byte of a block's scale that filling writes


def _binding():
    from paper_2604_22808_amd import binding
    return binding


# ---------------------------------------------------------------------------------------------------------------- cases

def _norm(name, dtype, batch, rows, channels, each=False, train=False):
    """each: weights of their own for every batch entry."""
    return dict(name=name, op="norm", dtype=dtype, batch=batch, rows=rows, channels=channels, each=each, train=train)


def _product(name, dtype, rows, channels, outputs, bias=False):
    return dict(name=name, op="product", dtype=dtype, rows=rows, channels=channels, outputs=outputs, bias=bias)


def _fill(name, dtype, heads, d, block, new, lengths, capacity):
    """new: rows appended to every sequence, packed; lengths: rows of its cache that are filled then."""
    return dict(name=name, op="fill", dtype=dtype, kv_heads=heads, head_dim=d, block=block, new=new, lengths=lengths, capacity=capacity)


def _attend(name, dtype, heads, kv_heads, d, block, new, lengths, capacity):
    """new: query rows, the last rows of every sequence (packed; all one count: [sequences, rows, heads, d]); lengths: filled rows of the caches."""
    return dict(name=name, op="attend", dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=d, block=block, new=new, lengths=lengths, capacity=capacity)


def listed():
    return [
        # one new token of each of 64 requests in front of their projections: launch latency
        _norm("norm_one_token", "bf16", 64, 1, 2048),
        # a training step of both guidance branches of a 64K-token clip, whose scale and shift come from each branch's own conditioning
        _norm("norm_train_branches", "bf16", 2, 65536, 1536, each=True, train=True),
        # fp32 training, odd numbers of rows and channels
        _norm("norm_train_f32_odd", "f32", 1, 10007, 999, train=True),
        # one new token of 16 requests into the fused projection of queries, keys and values: the weights' bytes
        _product("product_one_token", "bf16", 16, 2048, 6144),
        # a short prompt with an odd number of tokens into a projection back to the model's width, fp32 in and out
        _product("product_short_f32", "f32", 333, 1000, 1100),
        # queries, keys and values of the 64K-token workload's clip
        _product("product_qkv_64k", "bf16", 65536, 1536, 4608),
        # the output projection of 128K tokens at d_model 2048
        _product("product_out_128k", "bf16", 131072, 2048, 2048, bias=True),
        # one new token of 16 requests whose last blocks are partly filled
        _fill("fill_one_token", "bf16", 2, 64, 16, ",".join(["1"] * 16), ",".join(str(40 + 17 * i) for i in range(16)), 300),
        # prompts of different lengths, some behind what earlier chunks left
        _fill("fill_prompts", "bf16", 8, 128, 64, "4096,1,2900,640,17,2222,3333,333", "4096,1000,3900,640,4000,2222,3333,2000", 4100),
        # one token of one request against a short cache: latency
        _attend("attend_one_short", "bf16", 16, 2, 64, 16, "1", "777", 1000),
        # one token of 32 requests against long caches of different fill: the bytes of the caches
        _attend("attend_one_batch", "bf16", 32, 8, 128, 64, ",".join(["1"] * 32), ",".join(str(200 + 509 * i) for i in range(31)) + ",16384", 16384),
        # chunks of prompts against what earlier chunks left, and a lone token
        _attend("attend_chunks", "bf16", 16, 4, 128, 64, "1500,512,2048,1", "9000,16000,4500,777", 16384),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _wide(rng, lo, hi):
    """A width: whole pieces mostly, sometimes odd."""
    n = _log(rng, lo, hi)
    return rng.choice([max(1, round(n)), 8 * max(1, round(n / 8)), 64 * max(1, round(n / 64)), 256 * max(1, round(n / 256))])


def draw(rng):
    op = rng.choice(["norm", "norm", "product", "product", "fill", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        channels, batch = _wide(rng, 48, 8200), rng.choice([1, 1, 2, 5, 16])
        rows = 1 if rng.random() < 0.15 else max(1, round(_log(rng, 2e4, 1.5e8) / (channels * batch)))
        c = _norm("", dtype, batch, rows, channels, rng.random() < 0.4, rng.random() < 0.6)
    elif op == "product":
        channels, outputs = _wide(rng, 64, 8200), _wide(rng, 48, 8200)
        rows = round(_log(rng, 1, 64)) if rng.random() < 0.35 else max(1, round(min(1e5, _log(rng, 1e8, 4e11) / (channels * outputs))))
        c = _product("", dtype, rows, channels, outputs, rng.random() < 0.5)
    else:
        kv_heads, n = round(_log(rng, 1, 9)), round(_log(rng, 1, 24))
        d, block = rng.choice([32, 64, 64, 72, 96, 128, 128, 128]), rng.choice([16, 32, 64, 64, 128, 256])
        if op == "fill":
            most = max(4, min(5000, round(_log(rng, 1e4, 1.5e7) / (n * kv_heads * d))))
            new = [rng.choice([1, most, rng.randint(1, most)]) for _ in range(n)]
            old = [rng.choice([0, rng.randint(0, most)]) for _ in range(n)]
            c = _fill("", dtype, kv_heads, d, block, ",".join(map(str, new)), ",".join(str(a + b) for a, b in zip(new, old)),
                      max(a + b for a, b in zip(new, old)) + rng.choice([0, 3, 64]))
        else:
            heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
            if rng.random() < 0.6:     # single tokens, or a few
                rows = rng.choice([1, 1, 1, 2, 5, 16])
                most = max(64, min(20000, round(2e8 / (n * heads * d))))
                new, lengths = [rows] * n, [rng.randint(rows, most) for _ in range(n)]
            else:
                dtype = rng.choice(["bf16", "bf16", "bf16", dtype])
                pairs = (2e7 if dtype == "f32" else 4e8) * rng.uniform(0.02, 0.5)
                most = max(2, min(16000, round(math.sqrt(4 * pairs / (n * heads)))))
                lengths = [rng.choice([most, rng.randint(1, most)]) for _ in range(n)]
                new = [rng.randint(1, max(1, min(x, most // 3))) for x in lengths]
            c = _attend("", dtype, heads, kv_heads, d, block, ",".join(map(str, new)), ",".join(map(str, lengths)), most + rng.choice([0, 3, 64]))
    del c["name"]
    return c


def _ints(text):
    return [int(x) for x in text.split(",")]


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "norm":
        n, sets = c["batch"] * c["rows"] * c["channels"], c["batch"] if c["each"] else 1
        # forward: x in, y out; backward: x, dy in, dx out
        return {"bytes": n * size * (5 if c["train"] else 2) + sets * c["channels"] * (3 * size + 8 if c["train"] else 2 * size), "flops": n * (22 if c["train"] else 8)}
    if c["op"] == "product":
        m, k, n = c["rows"], c["channels"], c["outputs"]
        return {"bytes": m * k * size + n * k + 4 * n + m * n * size, "flops": 2 * m * k * n}
    new, lengths = _ints(c["new"]), _ints(c["lengths"])
    if c["op"] == "fill":    # new rows in, their codes out; codes of the filled rows in, their values out
        row = c["kv_heads"] * c["head_dim"]
        return {"bytes": 2 * row * (sum(new) * (size + 1) + sum(lengths) * (1 + size)), "flops": 2 * row * (3 * sum(new) + sum(lengths))}
    pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(new, lengths)) * c["heads"]
    return {"bytes": c["head_dim"] * (2 * sum(new) * c["heads"] * size + 2 * sum(lengths) * c["kv_heads"]), "flops": 4 * c["head_dim"] * pairs}


# ---------------------------------------------------------------------------------------------------------------- inputs

def _blocks(x, block):
    """[sequences, rows, heads, d] as [sequences, blocks, block, heads, d], zeros behind the last row."""
    s, r, h, d = x.shape
    pad = -r % block
    if pad:
        x = torch.cat([x, x.new_zeros(s, pad, h, d)], 1)
    return x.view(s, (r + pad) // block, block, h, d)


def _least_byte(top):
    """The smallest byte e, LEAST at least, with top <= 448 * 2^(e - 127)."""
    m, e = torch.frexp(top.double() / TOP)                # m in [0.5, 1): top / 448 = m 2^e
    return torch.where(top > 0, e + 127 - (m == 0.5).int(), LEAST).clamp(min=LEAST)


def _power(byte):
    return (byte.int() << 23).view(torch.float32)          # 2^(byte - 127), byte 1 to 254


def _each_row(byte, block, rows):
    """Scales of the blocks as a factor for every row: [sequences, rows, heads, 1]."""
    return _power(byte).repeat_interleave(block, 1)[:, :rows, :, None]


def prepare(case, seed):
    c, dev, t = case, "cuda", TYPES[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, device=dev, generator=g)

    s = {"c": c}
    if c["op"] == "norm":
        b, r, n = c["batch"], c["rows"], c["channels"]
        # a residual stream: channels of different sizes, rows with a mean
        x = randn(b, r, n)
        x *= torch.exp(0.7 * randn(n))
        x += randn(b, r, 1)
        s["x"] = x.to(t)
        shape = (b, n) if c["each"] else (n,)
        s["w"], s["b"] = (1 + 0.3 * randn(*shape)).to(t), (0.3 * randn(*shape)).to(t)
        s["out"] = torch.empty_like(s["x"])
        if c["train"]:
            s["dout"], s["dx"] = randn(b, r, n).to(t), torch.empty_like(s["x"])
            s["dw"], s["db"] = torch.empty(shape, device=dev), torch.empty(shape, device=dev)
        return s
    if c["op"] == "product":
        m, k, n = c["rows"], c["channels"], c["outputs"]
        x = randn(m, k)
        x *= torch.exp(0.5 * randn(k))
        s["x"] = x.to(t)
        w = randn(n, k)       # weights coded once, a scale for every output channel
        top = w.abs().amax(1, keepdim=True)
        s["w"], s["w_scales"] = torch.round(w * (127 / top)).to(torch.int8), (top[:, 0] * (0.02 / 127)).contiguous()
        s["bias"] = randn(n).to(t) if c["bias"] else None
        s["codes"], s["scales"] = torch.empty(m, k, device=dev, dtype=torch.int8), torch.empty(m, device=dev)
        s["out"] = torch.empty(m, n, device=dev, dtype=t)
        return s
    new, lengths = _ints(c["new"]), _ints(c["lengths"])
    n, h, d, block, cap = len(new), c["kv_heads"], c["head_dim"], c["block"], c["capacity"]
    s["new"], s["lengths"] = (torch.tensor(v, device=dev, dtype=torch.int32) for v in (new, lengths))
    s["offsets"] = torch.tensor([0] + new, device=dev, dtype=torch.int32).cumsum(0).to(torch.int32)
    # what earlier rows and earlier requests left in the cache: blocks of different sizes
    for name in ("k", "v"):
        x = randn(n, cap, h, d)
        x *= torch.exp(randn(n, (cap + block - 1) // block, h)).repeat_interleave(block, 1)[:, :cap, :, None] if c["op"] == "fill" else 1.0
        byte = _least_byte(_blocks(x, block).abs().amax((2, 4)))
        s["cache_" + name] = (x / _each_row(byte, block, cap)).to(torch.float8_e4m3fn)
        s[name + "_scales"] = byte.to(torch.uint8)
    if c["op"] == "fill":
        s["k"], s["v"] = randn(sum(new), h, d).to(t), randn(sum(new), h, d).to(t)
        s["k_out"], s["v_out"] = torch.zeros(n, cap, h, d, device=dev, dtype=t), torch.zeros(n, cap, h, d, device=dev, dtype=t)
        return s
    s["packed"] = len(set(new)) > 1
    s["q"] = randn(*((sum(new),) if s["packed"] else (n, new[0])), c["heads"], d).to(t)
    s["out"] = torch.empty_like(s["q"])
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms

def _plain_norm(s):
    c, x = s["c"], s["x"].float()
    w, b = s["w"].float(), s["b"].float()
    if c["each"]:
        w, b = w[:, None], b[:, None]
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    h = x.mul_(r)
    s["out"].copy_(h * w + b)
    if not c["train"]:
        return s["out"]
    g = s["dout"].float()
    over = (1,) if c["each"] else (0, 1)
    s["dw"].copy_((g * h).sum(over, dtype=torch.float64))
    s["db"].copy_(g.sum(over, dtype=torch.float64))
    g = g * w
    s["dx"].copy_(r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True)))
    return [s[n] for n in ("out", "dx", "dw", "db")]


def _plain_product(s):
    x = s["x"].double()          # (values beside the border between two codes)
    top = x.abs().amax(1, keepdim=True)
    codes = torch.round(x * 127.0 / torch.where(top > 0, top, 1.0)).float()
    y = torch.matmul(codes, s["w"].float().t().contiguous()) * (top / 127.0).float() * s["w_scales"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    s["out"].copy_(y)
    return s["out"]


def _plain_fill(s):
    c, block, cap = s["c"], s["c"]["block"], s["c"]["capacity"]
    j = torch.arange(cap, device=s["new"].device)
    old = (s["lengths"] - s["new"])[:, None]
    is_new, is_old = (j >= old) & (j < s["lengths"][:, None]), j < old
    at = (s["offsets"][:-1, None] + j - old).clamp(0, max(0, s["k"].shape[0] - 1))
    has_old = _blocks(is_old[..., None, None].int(), block).amax((2, 4)) > 0
    has_new = _blocks(is_new[..., None, None].int(), block).amax((2, 4)) > 0
    for name in ("k", "v"):
        x = torch.where(is_new[:, :, None, None], s[name].float()[at], 0.0)
        was = s[name + "_scales"].int()
        need = _least_byte(_blocks(x, block).abs().amax((2, 4)))
        now = torch.where(has_new, torch.where(has_old, torch.maximum(was, need), need), was)
        codes = s["cache_" + name].float()
        kept = codes * _each_row(was, block, cap)
        x = torch.where(is_new[:, :, None, None], x, kept)
        fresh = (x / _each_row(now, block, cap)).to(torch.float8_e4m3fn).float()
        inside = (is_new | is_old)[:, :, None, None]
        codes = torch.where(inside, fresh, codes)
        s["cache_" + name].copy_(codes)
        s[name + "_scales"].copy_(now)
        values = codes * _each_row(now, block, cap)
        s[name + "_out"].copy_(torch.where(inside, values.to(s[name].dtype), s[name + "_out"]))
    return [s["k_out"], s["v_out"]]


def _plain_attend(s):
    c, dev, block = s["c"], s["q"].device, s["c"]["block"]
    group, most, rows = c["heads"] // c["kv_heads"], max(_ints(c["lengths"])), max(_ints(c["new"]))
    i, j = torch.arange(rows, device=dev), torch.arange(most, device=dev)
    q_in, k_in = i < s["new"][:, None], j < s["lengths"][:, None]
    if s["packed"]:
        q = torch.where(q_in[:, :, None, None], s["q"][(s["offsets"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1)].float(), 0.0)
    else:
        q = s["q"].float()

    def values(name):
        x = s["cache_" + name][:, :most].float() * _each_row(s[name + "_scales"], block, most)
        x = torch.where(k_in[:, :, None, None], x, 0.0).transpose(1, 2)
        return x.repeat_interleave(group, 1) if group > 1 else x.contiguous()

    seen = k_in[:, None, None, :] & (j <= i[:, None] + (s["lengths"] - s["new"])[:, None, None, None])
    p = torch.matmul(q.transpose(1, 2).contiguous(), values("k").transpose(-1, -2).contiguous()).mul_(1.0 / math.sqrt(c["head_dim"])).masked_fill_(~seen, -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp(min=1e-38))
    o = torch.matmul(p, values("v")).transpose(1, 2)
    s["out"].copy_(o[q_in] if s["packed"] else o)
    return s["out"]


# -------------------------------------------------------------------------------------------------------- one pass of each

def _own_norm(B, s):
    B.layer_norm(s["x"], s["w"], s["b"], s["out"], eps=EPS)
    if not s["c"]["train"]:
        return s["out"]
    B.layer_norm_backward(s["x"], s["w"], s["dout"], s["dx"], s["dw"], s["db"], eps=EPS)
    return [s[n] for n in ("out", "dx", "dw", "db")]


def _own_product(B, s):
    B.quantize_rows(s["x"], s["codes"], s["scales"])
    return B.product_i8(s["codes"], s["scales"], s["w"], s["w_scales"], s["out"], bias=s["bias"])


def _own_fill(B, s):
    cache = (s["cache_k"], s["cache_v"], s["k_scales"], s["v_scales"], s["c"]["block"])
    B.cache8_append(s["k"], s["v"], *cache, q_offsets=s["offsets"], k_lengths=s["lengths"])
    B.cache8_read(*cache, s["k_out"], s["v_out"], k_lengths=s["lengths"])
    return [s["k_out"], s["v_out"]]


def _own_attend(B, s):
    return B.cache8_attention(s["q"], s["cache_k"], s["cache_v"], s["k_scales"], s["v_scales"], s["c"]["block"], s["out"], causal=True,
                              q_offsets=s["offsets"] if s["packed"] else None, k_lengths=s["lengths"])


_PLAIN = {"norm": _plain_norm, "product": _plain_product, "fill": _plain_fill, "attend": _plain_attend}
_OWN = {"norm": _own_norm, "product": _own_product, "fill": _own_fill, "attend": _own_attend}


def run(state):
    op = state["c"]["op"]
    return _OWN[op](_binding(), state) if own else _PLAIN[op](state)


# --------------------------------------------------------------------------------------- the definition in 64 bits, by itself

def _exact_norm(c, s):
    shared = not c["each"]
    w, b = s["w"].double(), s["b"].double()
    out, dx = (torch.empty(s["x"].shape, device=w.device, dtype=torch.float64) for _ in range(2))
    dw, db = torch.zeros_like(w), torch.zeros_like(w)
    for i in range(c["batch"]):
        for at in range(0, c["rows"], 8192):
            part = (i, slice(at, at + 8192))
            x = s["x"][part].double()
            wi, bi = (w, b) if shared else (w[i], b[i])
            var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
            unit = (x - mean) / (var + EPS).sqrt()
            out[part] = unit * wi + bi
            if c["train"]:
                g = s["dout"][part].double()
                to = Ellipsis if shared else i
                dw[to] += (g * unit).sum(0)
                db[to] += g.sum(0)
                g = g * wi
                n = c["channels"]
                dx[part] = (n * g - g.sum(1, keepdim=True) - unit * (g * unit).sum(1, keepdim=True)) / (n * (var + EPS).sqrt())
    return [out, dx, dw, db] if c["train"] else out


def _exact_product(c, s):
    w = (s["w"].double() * s["w_scales"].double()[:, None]).t().contiguous()
    out = torch.empty(s["out"].shape, device=w.device, dtype=torch.float64)
    for at in range(0, c["rows"], 16384):
        x = s["x"][at:at + 16384].double()
        most = x.abs().max(1).values[:, None]
        whole = 127 * x / torch.where(most > 0, most, 1.0)
        out[at:at + 16384] = (torch.round(whole) * (most / 127)) @ w
    return out + s["bias"].double() if c["bias"] else out


def _exact_e4m3(x):
    """To the nearest e4m3 value, ties to even, of |x| <= 448 in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_fill(c, s):
    res = []
    block = c["block"]
    start = [0]
    for a in _ints(c["new"]):
        start.append(start[-1] + a)
    for name in ("k", "v"):
        out = s[name + "_out"].double()
        for i, (a, n) in enumerate(zip(_ints(c["new"]), _ints(c["lengths"]))):
            first = n - a
            rows = torch.cat([s["cache_" + name][i, :first].float().double(), s[name][start[i]:start[i] + a].double()])   # old codes, new values
            for lo in range(0, n, block):
                hi = min(lo + block, n)
                was = torch.exp2(s[name + "_scales"][i, lo // block].double() - 127)[None, :, None]
                part, k = rows[lo:hi], max(0, min(first - lo, hi - lo))      # k: old rows of the block
                part[:k] *= was
                if k < hi - lo:
                    top = part[k:].abs().amax((0, 2), keepdim=True)
                    need = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / TOP)).clamp(min=LEAST - 127.0))
                    scale = torch.maximum(was, need) if k else need
                    part = _exact_e4m3(part / scale) * scale
                out[i, lo:hi] = part
        res.append(out)
    return res


def _exact_attend(c, s):
    group, d, block = c["heads"] // c["kv_heads"], c["head_dim"], c["block"]
    out = torch.empty(s["out"].shape, device=s["q"].device, dtype=torch.float64)
    at = 0
    for i, (a, n) in enumerate(zip(_ints(c["new"]), _ints(c["lengths"]))):
        byte = torch.arange(n, device=out.device) // block
        k, v = (s["cache_" + x][i, :n].float().double() * torch.exp2(s[x + "_scales"][i].double() - 127)[byte][:, :, None] for x in "kv")
        rows = slice(at, at + a) if s["packed"] else i
        far = torch.arange(n, device=out.device)[None, :] > torch.arange(a, device=out.device)[:, None] + (n - a)
        for h in range(c["heads"]):
            score = (s["q"][rows][:, h].double() @ k[:, h // group].t().contiguous() / math.sqrt(d)).masked_fill(far, -math.inf)
            out[rows][:, h] = torch.softmax(score, 1) @ v[:, h // group].contiguous()
        at += a
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "product": _exact_product, "fill": _exact_fill, "attend": _exact_attend}[case["op"]](case, s)
