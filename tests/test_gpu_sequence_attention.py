"""Attention over packed, padded and cached sequences on the GPU, forward and backward, against the plain 64-bit form."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import heads_util as U

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32).cuda()


def randn(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float64)


MARK = 7.0    # what outputs hold before a call: rows of no sequence still hold it afterwards


class Call:
    """One call's tensors.  Host tensors are [batch, rows, heads, d] (packed: batch 1); device tensors are given as the entry points take them."""

    def __init__(self, seed, dtype, heads, kv_heads, d, q_rows, k_rows, batch=None, q_offsets=None, k_offsets=None, q_lengths=None, k_lengths=None,
                 causal=False, scale=0.0, spoil=False, order="rows", pad=0, spread=1.0):
        self.io, gen = TYPES[dtype], torch.Generator().manual_seed(seed)
        self.n = batch if q_offsets is None else len(q_offsets) - 1
        qb, kb = (1 if q_offsets else batch), (1 if k_offsets else batch)
        self.q_spans = U.spans(q_offsets, q_lengths, q_rows, self.n)
        self.k_spans = U.spans(k_offsets, k_lengths, k_rows, self.n)
        host = {"q": spread * randn(gen, qb, q_rows, heads, d), "k": spread * randn(gen, kb, k_rows, kv_heads, d), "v": randn(gen, kb, k_rows, kv_heads, d),
                "dout": randn(gen, qb, q_rows, heads, d)}
        self.host = {n: t.to(self.io) for n, t in host.items()}
        if spoil:   # rows of no sequence hold NaN
            for n, t in self.host.items():
                inside = torch.zeros(t.shape[:2], dtype=torch.bool)
                for b, first, count in (self.q_spans if n in ("q", "dout") else self.k_spans):
                    inside[b, first:first + count] = True
                t[~inside] = math.nan
        self.how = dict(causal=causal, scale=scale, q_offsets=ints(q_offsets), k_offsets=ints(k_offsets), q_lengths=ints(q_lengths), k_lengths=ints(k_lengths))
        self.packed = (q_offsets is not None, k_offsets is not None)
        self.causal, self.scale = causal, scale if scale > 0 else 1.0 / math.sqrt(d)

        def place(t, packed):
            b, r, h, c = t.shape
            if order == "heads":
                x = torch.empty(b, h, r, c + pad, dtype=self.io, device="cuda").transpose(1, 2)[..., :c]
            else:
                x = torch.empty(b, r, h, c + pad, dtype=self.io, device="cuda")[..., pad:]
            x.copy_(t)
            return x[0] if packed else x

        self.dev = {n: place(t, self.packed[n in ("k", "v")]) for n, t in self.host.items()}
        self.out = {n: place(torch.full_like(self.host[s], MARK), self.packed[s == "k"]) for n, s in (("out", "q"), ("dq", "q"), ("dk", "k"), ("dv", "k"))}
        self.lse = torch.full((heads, qb * q_rows), MARK, device="cuda")

    def forward(self, lse=True):
        d = self.dev
        B.sequence_attention(d["q"], d["k"], d["v"], self.out["out"], lse=self.lse if lse else None, **self.how)

    def backward(self):
        d, o = self.dev, self.out
        B.sequence_attention_backward(d["dout"], d["q"], d["k"], d["v"], o["out"], self.lse, o["dq"], o["dk"], o["dv"], **self.how)

    def results(self):
        r = {n: (t[None] if t.dim() == 3 else t) for n, t in self.out.items()}
        qb, q_rows, heads, _ = self.host["q"].shape
        r["lse"] = self.lse.view(heads, qb, q_rows).permute(1, 2, 0)
        return r

    def check(self, train=True, names=None):
        h = self.host
        want = U.attend_all(h["q"], h["k"], h["v"], self.causal, self.scale, self.q_spans, self.k_spans, h["dout"] if train else None)
        got = self.results()
        for n, (value, bound, inside) in want.items():
            if names and n not in names:
                continue
            g = got[n].cpu()
            U.check(n, g[inside], value[inside], bound[inside])
            assert torch.equal(g[~inside], torch.full_like(g[~inside], MARK)), (n, "rows of no sequence were written")


def offsets(*lengths, first=0):
    out = [first]
    for n in lengths:
        out.append(out[-1] + n)
    return out


# heads, kv heads, head_dim, lengths of the queries and of the keys (packed both)
PACKED = [
    (2, 2, 64, (1,), (1,)),
    (1, 1, 128, (33,), (65,)),
    (4, 1, 64, (130, 1, 0, 64, 127), (130, 1, 0, 64, 127)),
    (6, 3, 128, (200, 31, 129), (200, 31, 129)),
    (3, 3, 128, (5, 70), (300, 257)),          # queries are the last of their keys
    (2, 1, 64, (70, 5, 3, 40), (20, 5, 0, 39)),  # causal: the first queries of three sequences see nothing
    (8, 1, 64, (1, 1, 1), (513, 64, 1)),
    (5, 1, 128, (40,), (96,)),                 # a group that divides no tile
    (2, 2, 48, (77, 19), (77, 19)),
    (2, 1, 100, (50,), (70,)),
    (2, 2, 1, (9,), (40,)),
    (4, 2, 72, (129, 64), (140, 64)),
    (16, 2, 32, (100,), (33,)),
    (1, 1, 128, (300,), (300,)),
]


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", PACKED, ids=str)
def test_packed_sequences(case, dtype, causal):
    heads, kv_heads, d, ql, kl = case
    c = Call(sum(map(ord, str(case))), dtype, heads, kv_heads, d, sum(ql) + 5, sum(kl) + 3, q_offsets=offsets(*ql, first=2), k_offsets=offsets(*kl),
             causal=causal, spoil=True)
    c.forward()
    c.check(train=False)
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_lanes(dtype):
    """100 sequences: short ones (tiles of few rows), and with some long ones among them; packed and batched with lengths."""
    short = [(7 * i) % 5 for i in range(100)]
    mixed = [(7 * i) % 5 + (300 if i % 40 == 3 else 0) for i in range(100)]
    for causal, lengths in ((True, short), (False, mixed), (True, mixed)):
        c = Call(121, dtype, 4, 2, 64, sum(lengths) + 1, sum(lengths), q_offsets=offsets(*lengths), k_offsets=offsets(*lengths), causal=causal, spoil=True)
        c.forward()
        c.backward()
        c.check()
    c = Call(122, dtype, 2, 1, 64, 40, 50, batch=70, q_lengths=[i % 41 for i in range(70)], k_lengths=[50 - i % 51 for i in range(70)], causal=True, spoil=True)
    c.forward()
    c.backward()
    c.check()


def test_one_head_of_any_stride():
    """The stride of an axis of one entry is not used: a single head sliced out of rows of 65 channels keeps to the aligned kernels' results."""
    c = Call(131, "bf16", 1, 1, 64, 200, 200, q_offsets=[0, 200], k_offsets=[0, 200], causal=True)
    for n, t in c.dev.items():
        c.dev[n] = torch.as_strided(t, (200, 1, 64), (64, 65, 1))
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("order", ["rows", "heads"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_padded_batches(causal, dtype, order):
    """[sequences, rows, heads, d] and its head-major order, lengths of zero, of one row and beyond the rows there are."""
    c = Call(21, dtype, 4, 2, 64, 70, 90, batch=5, q_lengths=[70, 0, 1, 33, 99], k_lengths=[90, 40, 17, 0, 1000], causal=causal, spoil=True, order=order)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("rows,heads,kv_heads,d,dtype", [(1, 8, 2, 128, "bf16"), (1, 1, 1, 64, "bf16"), (4, 8, 1, 64, "bf16"), (1, 6, 2, 128, "f32"),
                                                         (3, 40, 1, 128, "bf16"), (1, 4, 4, 80, "bf16"), (2, 3, 1, 36, "bf16")])
def test_tokens_against_a_cache(rows, heads, kv_heads, d, dtype):
    """A few new tokens per request, keys in a cache of more rows than are filled; long enough that the keys are split."""
    c = Call(rows * 100 + heads, dtype, heads, kv_heads, d, rows, 5000, batch=4, k_lengths=[5000, rows, 1023, 2049], causal=True, spoil=True)
    c.forward(lse=False)
    c.check(train=False, names=("out",))
    c.forward()
    c.check(train=False)
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_rows_that_are_no_aligned_pieces(pad, dtype):
    """Channels that start and rows that lie between 16-byte pieces."""
    for d in (64, 44):
        c = Call(31, dtype, 4, 2, d, 150, 150, q_offsets=[0, 140], k_offsets=[0, 140], causal=True, pad=pad)
        c.forward()
        c.backward()
        c.check()


def test_packed_queries_against_a_cache_and_a_batch_against_packed_keys():
    c = Call(41, "bf16", 4, 2, 64, 40, 300, batch=3, q_offsets=[0, 30, 31, 38], k_lengths=[200, 300, 7], causal=True, spoil=True)
    c.forward()
    c.backward()
    c.check()
    c = Call(42, "bf16", 4, 2, 64, 16, 333, batch=3, k_offsets=[0, 30, 31, 333], q_lengths=[16, 1, 9], causal=False, spoil=True)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-3, 0.5, 3.0])
def test_scales_and_large_scores(scale, dtype):
    """Scores of some hundreds: the softmax is a choice of one key, later tiles move the maximum far."""
    c = Call(51, dtype, 2, 2, 64, 200, 333, q_offsets=[0, 200], k_offsets=[0, 333], causal=True, scale=scale, spread=2.0)
    for n in ("q", "k"):     # growing along the sequence
        ramp = torch.linspace(0.1, 2.0, c.host[n].shape[1])[None, :, None, None].double()
        c.host[n] = (c.host[n].double() * ramp).to(c.io)
        c.dev[n].copy_(c.host[n][0])
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_that_are_not_seen_reach_nothing(dtype, value):
    """One key and value row in the middle is not finite: queries before it keep their bits, output and gradient of q; those after it see it."""
    args = dict(q_offsets=[0, 300], k_offsets=[0, 300], causal=True)
    clean = Call(61, dtype, 2, 1, 64, 300, 300, **args)
    bad = Call(61, dtype, 2, 1, 64, 300, 300, **args)
    at = 150
    for n in ("k", "v"):
        bad.dev[n][at] = value
    for c in (clean, bad):
        c.forward()
        c.backward()
    for n in ("out", "dq"):
        assert torch.equal(clean.out[n][:at], bad.out[n][:at]), n
        assert not torch.isfinite(bad.out["out"][at:]).all(-1).any()
    assert torch.equal(clean.lse[:, :at], bad.lse[:, :at])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_that_do_not_see_a_key_give_it_no_gradient(dtype):
    """Query and gradient rows before position 150 are not finite: keys from there on are seen by later queries alone and keep their gradients' bits."""
    args = dict(q_offsets=[0, 300], k_offsets=[0, 300], causal=True)
    clean = Call(62, dtype, 2, 1, 64, 300, 300, **args)
    bad = Call(62, dtype, 2, 1, 64, 300, 300, **args)
    bad.dev["q"][149] = math.nan
    bad.dev["dout"][100] = math.inf
    for c in (clean, bad):
        c.forward()
        c.backward()
    for n in ("dk", "dv"):
        assert torch.equal(clean.out[n][150:], bad.out[n][150:]), n
        assert not torch.isfinite(bad.out[n][:100]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_value_that_is_seen(dtype):
    """v alone holds an infinity: rows that see it get it in its channel, all else is as without."""
    c = Call(63, dtype, 2, 1, 64, 200, 200, q_offsets=[0, 200], k_offsets=[0, 200], causal=True)
    c.dev["v"][70, 0, 5] = math.inf
    c.forward()
    out = c.out["out"].float()
    assert bool((out[70:, :, 5] == math.inf).all())
    out[70:, :, 5] = 0
    assert bool(torch.isfinite(out).all())


def test_wrong_offsets_stay_inside():
    """Offsets that point outside, descend or overlap give some result from inside the tensors and an end to the call."""
    for off in ([0, 500, 120], [-7, 50, 2 ** 31 - 1], [90, 60, 30], [-2 ** 31, -5, -1]):
        c = Call(71, "bf16", 2, 1, 64, 100, 100, q_offsets=[0, 60, 100], k_offsets=[0, 60, 100], causal=True)
        c.how["q_offsets"], c.how["k_offsets"] = ints(off), ints(off[::-1])
        c.how["k_lengths"] = ints([-3, 2 ** 30])
        c.forward()
        c.backward()
        torch.cuda.synchronize()


def test_no_sequences_no_rows_no_keys():
    e = torch.empty
    z = lambda *s: torch.full(s, MARK, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    B.sequence_attention(z(0, 4, 2, 64), z(0, 4, 2, 64), z(0, 4, 2, 64), z(0, 4, 2, 64))
    B.sequence_attention(z(0, 2, 64), z(9, 2, 64), z(9, 2, 64), z(0, 2, 64), q_offsets=ints([0, 0]), k_offsets=ints([0, 9]))
    q, k, out, dk, dv, dq = z(3, 5, 2, 64), z(3, 0, 2, 64), z(3, 5, 2, 64), z(3, 0, 2, 64), z(3, 0, 2, 64), z(3, 5, 2, 64)
    lse = e(2, 15, device="cuda")
    B.sequence_attention(q, k, k, out, lse=lse)
    B.sequence_attention_backward(q, q, k, k, out, lse, dq, dk, dv)
    assert float(out.abs().sum()) == 0 and float(dq.abs().sum()) == 0 and bool((lse == -math.inf).all())
    q, k, dk, dv = z(2, 0, 2, 64), z(2, 5, 2, 64), z(2, 5, 2, 64), z(2, 5, 2, 64)
    B.sequence_attention_backward(q, q, k, k, q, e(2, 0, device="cuda"), q, dk, dv)
    assert float(dk.abs().sum()) == 0 and float(dv.abs().sum()) == 0


def test_a_cache_beyond_32_bits():
    """Rows of the cache lie up to 6 GB from its start, read by one token and by a tile of queries, with gradients."""
    rows, stride = 40, 80 * 1000 * 1000
    for n in (1, 40):
        k = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").as_strided((1, rows, 2, 64), (0, stride, 64, 1))
        v = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").as_strided((1, rows, 2, 64), (0, stride, 64, 1))
        c = Call(81, "bf16", 4, 2, 64, n, rows, batch=1, causal=True)
        k.copy_(c.host["k"])
        v.copy_(c.host["v"])
        c.dev["k"], c.dev["v"] = k, v
        c.forward()
        c.backward()
        c.check()


def test_equal_calls_give_equal_bits_and_streams_do_not_matter():
    lengths = (300, 17, 500)
    c = Call(91, "bf16", 8, 2, 128, sum(lengths), sum(lengths), q_offsets=offsets(*lengths), k_offsets=offsets(*lengths), causal=True)
    d = Call(92, "bf16", 4, 2, 64, 1, 4000, batch=3, k_lengths=[4000, 3, 1500], causal=True)
    for x in (c, d):
        x.forward()
        x.backward()
    torch.cuda.synchronize()
    want = [[t.clone() for t in (*x.out.values(), x.lse)] for x in (c, d)]
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for x, st in zip((c, d), s):     # both at once, each on its stream
            with torch.cuda.stream(st):
                x.forward()
                x.backward()
        torch.cuda.synchronize()
        for x, w in zip((c, d), want):
            assert all(torch.equal(a, b) for a, b in zip((*x.out.values(), x.lse), w))


def test_captured_and_replayed_with_other_lengths():
    """Lengths are read on the device: a graph serves a growing cache.  Two graphs that are replayed at the same time do not share a workspace."""
    def make(seed):
        x = Call(seed, "bf16", 8, 2, 64, 1, 3000, batch=2, k_lengths=[100, 200], causal=True)
        x.forward()
        x.backward()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.forward()
            x.backward()
        return x, g

    pairs = [make(101), make(102)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for lengths in ([101, 201], [3000, 1], [1, 2999], [1500, 64]):
        for x, _ in pairs:
            x.how["k_lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        for t in [t for x, _ in pairs for t in (*x.out.values(), x.lse)]:
            t.fill_(MARK)
        torch.cuda.synchronize()
        for (x, g), st in zip(pairs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for x, _ in pairs:
            x.k_spans = U.spans(None, lengths, 3000, 2)
            x.check()


def test_backward_against_differences():
    """fp32 gradients against central differences of the forward pass: h^2 / 6 of the third derivative and fp32 steps / h."""
    c = Call(111, "f32", 2, 1, 16, 12, 15, q_offsets=[0, 12], k_offsets=[0, 15], causal=True)
    c.forward()
    c.backward()
    grads = {n: c.out["d" + n].clone() for n in "qkv"}
    w = c.dev["dout"].double()
    h = 2.0 ** -6

    def loss():
        c.forward()
        return float((c.out["out"].double() * w).sum())

    for n in "qkv":
        t = c.dev[n]
        for i in range(8):
            at = (t.shape[0] - 1 - i, i % t.shape[1], i)
            x = float(t[at])
            t[at] = x + h
            hi, eh = loss(), float(t[at])
            t[at] = x - h
            lo, el = loss(), float(t[at])
            t[at] = x
            # scores move by at most scale |other| h with scale |other| <= 1 here: a third derivative within 8 sum |w| |v|; outputs of size <= 4 in fp32
            bound = h * h / 6 * 8 * float(w.abs().sum()) / 12 + float(w.abs().sum()) * 4 * 16 * U.F32 / (2 * h)
            assert abs((hi - lo) / (eh - el) - float(grads[n][at])) < bound, (n, at)
